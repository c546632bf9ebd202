// Entry points of the router, of 8-bit rows and products, and of the experts in them:
// argument checks, workspace layout, dispatch.
#include <algorithm>
#include <cmath>

#include "host.h"
#include "i8.h"
#include "route.h"

namespace {

using mla::aligned16;
using mla::fail;
using mla::hip_fail;

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

mla_status check_i8(int64_t n_rows, int32_t n_cols, const void* x, int64_t x_stride, const void* codes, const float* scales) {
  if (n_rows < 0) return fail(MLA_ERR_SHAPE, "n_rows = %lld", (long long)n_rows);
  if (n_cols < 16 || n_cols % 16 != 0) return fail(MLA_ERR_SHAPE, "n_cols = %d must be a positive multiple of 16", n_cols);
  if (n_cols > MLA_I8_MAX_COLS) return fail(MLA_ERR_UNSUPPORTED, "n_cols = %d; built: up to %d", n_cols, MLA_I8_MAX_COLS);
  if (x_stride < n_cols || x_stride % 8 != 0)
    return fail(MLA_ERR_SHAPE, "x_stride = %lld must be a multiple of 8, at least n_cols", (long long)x_stride);
  if (n_rows > INT64_MAX / 2 / x_stride) return fail(MLA_ERR_SHAPE, "n_rows * x_stride overflows");
  if (n_rows > 0 && (x == nullptr || codes == nullptr || scales == nullptr))
    return fail(MLA_ERR_NULL, "x, codes and scales are required");
  if (!aligned16(x) || !aligned16(codes)) return fail(MLA_ERR_SHAPE, "x and codes must be 16-byte aligned");
  if (!aligned(scales, 4)) return fail(MLA_ERR_SHAPE, "scales must be 4-byte aligned");
  return MLA_OK;
}

// Where the tables and intermediates of mla_moe_experts_i8 lie in its workspace.  `total` never
// falls as rows are added, though tiles get taller and h and the parts lie apart up to
// kExpertsFewPairs pairs alone: bytes that do for a batch do for a smaller one.
struct ExpertsSplit {
  int32_t tile_rows;
  bool few;
  int64_t off_hist, off_head, off_tiles, off_pairs, off_xq, off_xs, off_h, off_hq, off_hs, off_part;
  size_t total;
};

mla_status experts_split(const mla_moe_layer* L, int64_t n_rows, int32_t out_dtype, ExpertsSplit* S) {
  if (L == nullptr) return fail(MLA_ERR_NULL, "layer is NULL");
  if (n_rows < 0) return fail(MLA_ERR_SHAPE, "n_rows = %lld", (long long)n_rows);
  if (L->d_model < 64 || L->d_model % 64 != 0 || L->d_ffn < 64 || L->d_ffn % 64 != 0)
    return fail(MLA_ERR_SHAPE, "d_model = %d, d_ffn = %d must be positive multiples of 64", L->d_model, L->d_ffn);
  if (L->d_model > MLA_I8_MAX_COLS || L->d_ffn > MLA_I8_MAX_COLS)
    return fail(MLA_ERR_UNSUPPORTED, "d_model = %d, d_ffn = %d; built: up to %d", L->d_model, L->d_ffn, MLA_I8_MAX_COLS);
  if (L->n_experts < 1 || L->first_expert < 0 || L->first_expert > INT32_MAX - L->n_experts)
    return fail(MLA_ERR_SHAPE, "n_experts = %d, first_expert = %d", L->n_experts, L->first_expert);
  if (L->n_experts > mla::kExpertsMax)
    return fail(MLA_ERR_UNSUPPORTED, "n_experts = %d; built: up to %d", L->n_experts, mla::kExpertsMax);
  if (L->top_k < 1) return fail(MLA_ERR_SHAPE, "top_k = %d", L->top_k);
  if (L->top_k > mla::kExpertsMaxPairs)
    return fail(MLA_ERR_UNSUPPORTED, "top_k = %d; built: up to %d", L->top_k, mla::kExpertsMaxPairs);
  if (out_dtype != MLA_BF16 && out_dtype != MLA_F32) return fail(MLA_ERR_SHAPE, "out_dtype %d", out_dtype);
  if (n_rows > INT64_MAX / 8 / L->top_k / L->d_model) return fail(MLA_ERR_SHAPE, "n_rows * top_k * d_model overflows");
  const int64_t rows = std::min<int64_t>(n_rows, mla::kExpertsChunk), pairs = rows * L->top_k, d = L->d_model, f = L->d_ffn;
  S->tile_rows = mla::experts_tile_rows(pairs, L->n_experts);
  int64_t at = 0;
  auto take = [&at](int64_t bytes) {
    const int64_t was = at;
    at += (bytes + 255) / 256 * 256;
    return was;
  };
  S->off_hist = take((int64_t)mla::kDispatchBlocks * L->n_experts * 4);
  S->off_head = take(16);
  S->off_tiles = take(mla::experts_most_tiles(pairs, L->n_experts) * (int64_t)sizeof(mla::ExpertTile));
  S->off_pairs = take(pairs * (int64_t)sizeof(int2));
  S->off_xq = take(rows * d);
  S->off_xs = take(rows * 4);
  S->off_hq = take(pairs * f);
  S->off_hs = take(pairs * 4);
  S->few = n_rows * L->top_k <= mla::kExpertsFewPairs;
  const int64_t before = at, few = std::min<int64_t>(rows, mla::kExpertsFewPairs / L->top_k) * L->top_k;
  S->off_h = take(few * f * 2);
  S->off_part = take(few * d * 4);
  if (!S->few) {   // h is read for the last time before the first of the parts is written
    const int64_t apart = at;
    at = before;
    S->off_h = S->off_part = take(pairs * std::max(f * 2, d * 4));
    at = std::max(at, apart);
  }
  S->total = (size_t)std::max<int64_t>(at, 256);
  return MLA_OK;
}

}  // namespace

extern "C" {

mla_status mla_moe_route(int64_t n_rows, int32_t n_experts, const void* logits, int32_t logits_dtype, int64_t logits_stride,
                         const float* bias, const mla_route_cfg* cfg, int32_t* expert_idx, float* expert_w, int32_t* fanout,
                         int32_t* expert_count, void* stream) {
  mla::clear_detail();
  if (cfg == nullptr) return fail(MLA_ERR_NULL, "cfg is NULL");
  if (n_rows < 0) return fail(MLA_ERR_SHAPE, "n_rows = %lld", (long long)n_rows);
  if (cfg->scoring != MLA_SOFTMAX && cfg->scoring != MLA_SIGMOID) return fail(MLA_ERR_SHAPE, "scoring %d", cfg->scoring);
  if (logits_dtype != MLA_BF16 && logits_dtype != MLA_F32) return fail(MLA_ERR_SHAPE, "logits_dtype %d", logits_dtype);
  const int32_t k = cfg->top_k;
  if (k < 1 || k > mla::kMoeMaxTopK) return fail(MLA_ERR_UNSUPPORTED, "top_k = %d; built: 1 .. %d", k, mla::kMoeMaxTopK);
  if (cfg->min_k < 1 || cfg->min_k > k) return fail(MLA_ERR_SHAPE, "min_k = %d outside [1, top_k = %d]", cfg->min_k, k);
  if (n_experts < k) return fail(MLA_ERR_SHAPE, "n_experts = %d < top_k = %d", n_experts, k);
  if (n_experts > mla::kMoeMaxExperts)
    return fail(MLA_ERR_UNSUPPORTED, "n_experts = %d; built: up to %d", n_experts, mla::kMoeMaxExperts);
  const int32_t g = cfg->n_groups, kept = cfg->top_groups;
  if (g < 1 || n_experts % g != 0) return fail(MLA_ERR_SHAPE, "n_groups = %d must divide n_experts = %d", g, n_experts);
  if (g > mla::kRouteMaxGroups) return fail(MLA_ERR_UNSUPPORTED, "n_groups = %d; built: up to %d", g, mla::kRouteMaxGroups);
  if (kept < 1 || kept > g || (int64_t)kept * (n_experts / g) < k)
    return fail(MLA_ERR_SHAPE, "top_groups = %d of %d groups of %d experts, top_k = %d", kept, g, n_experts / g, k);
  if (cfg->group_best != 1 && cfg->group_best != 2) return fail(MLA_ERR_SHAPE, "group_best = %d, expected 1 or 2", cfg->group_best);
  if (!std::isfinite(cfg->scale)) return fail(MLA_ERR_SHAPE, "scale is not finite");
  if (std::isnan(cfg->tau)) return fail(MLA_ERR_SHAPE, "tau is NaN");
  if (n_rows > INT32_MAX) return fail(MLA_ERR_UNSUPPORTED, "n_rows = %lld; built: up to 2^31-1", (long long)n_rows);
  if (logits_stride < n_experts) return fail(MLA_ERR_SHAPE, "logits_stride = %lld < n_experts = %d", (long long)logits_stride, n_experts);
  if (n_rows > INT64_MAX / 8 / logits_stride) return fail(MLA_ERR_SHAPE, "n_rows * logits_stride overflows");
  if (n_rows > 0 && (logits == nullptr || expert_idx == nullptr || expert_w == nullptr))
    return fail(MLA_ERR_NULL, "logits, expert_idx and expert_w are required");
  if (!aligned(logits, logits_dtype == MLA_BF16 ? 2 : 4)) return fail(MLA_ERR_SHAPE, "logits must be aligned to their type");
  const void* ptrs[] = {bias, expert_idx, expert_w, fanout, expert_count};
  for (const void* q : ptrs)
    if (!aligned(q, 4)) return fail(MLA_ERR_SHAPE, "arrays must be 4-byte aligned");
  mla::RouteArgs a{};
  a.logits = logits;
  a.bias = bias;
  a.expert_idx = expert_idx;
  a.expert_w = expert_w;
  a.fanout = fanout;
  a.expert_count = expert_count;
  a.n_rows = n_rows;
  a.stride = logits_stride;
  a.n_experts = n_experts;
  a.logits_bf16 = logits_dtype == MLA_BF16;
  a.sigmoid = cfg->scoring == MLA_SIGMOID;
  a.n_groups = g;
  a.top_groups = kept;
  a.group_best = cfg->group_best;
  a.top_k = k;
  a.min_k = cfg->min_k;
  a.renormalize = cfg->renormalize != 0;
  a.scale = cfg->scale;
  a.tau = cfg->tau;
  const hipError_t e = mla::launch_moe_route(a, reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? MLA_OK : hip_fail(e, "router kernel");
}

mla_status mla_i8_quantize(int64_t n_rows, int32_t n_cols, const void* x, int64_t x_stride, void* codes, float* scales, void* stream) {
  mla::clear_detail();
  const mla_status st = check_i8(n_rows, n_cols, x, x_stride, codes, scales);
  if (st != MLA_OK || n_rows == 0) return st;
  const hipError_t e = mla::launch_i8_quantize(mla::I8Args{x, codes, scales, n_rows, x_stride, n_cols, nullptr, nullptr},
                                               reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? MLA_OK : hip_fail(e, "8-bit quantize kernel");
}

mla_status mla_i8_dequantize(int64_t n_rows, int32_t n_cols, const void* codes, const float* scales, void* x, int64_t x_stride,
                             void* stream) {
  mla::clear_detail();
  const mla_status st = check_i8(n_rows, n_cols, x, x_stride, codes, scales);
  if (st != MLA_OK || n_rows == 0) return st;
  const hipError_t e =
      mla::launch_i8_dequantize(mla::I8Args{x, const_cast<void*>(codes), const_cast<float*>(scales), n_rows, x_stride, n_cols, nullptr, nullptr},
                                reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? MLA_OK : hip_fail(e, "8-bit dequantize kernel");
}

mla_status mla_shared_wb_i8(int64_t n_rows, int32_t d_in, int32_t d_out, const void* z_codes, const float* z_scales,
                            const void* w_codes, const float* w_scales, int32_t out_dtype, void* y, void* stream) {
  mla::clear_detail();
  if (n_rows < 0) return fail(MLA_ERR_SHAPE, "n_rows = %lld", (long long)n_rows);
  if (d_in < 64 || d_in % 64 != 0) return fail(MLA_ERR_SHAPE, "d_in = %d must be a positive multiple of 64", d_in);
  if (d_in > MLA_I8_MAX_COLS) return fail(MLA_ERR_UNSUPPORTED, "d_in = %d; built: up to %d", d_in, MLA_I8_MAX_COLS);
  if (d_out < 1) return fail(MLA_ERR_SHAPE, "d_out = %d", d_out);
  if (d_out > MLA_WB_I8_MAX_D_OUT) return fail(MLA_ERR_UNSUPPORTED, "d_out = %d; built: up to %d", d_out, MLA_WB_I8_MAX_D_OUT);
  if (out_dtype != MLA_BF16 && out_dtype != MLA_F32) return fail(MLA_ERR_SHAPE, "out_dtype %d", out_dtype);
  if (n_rows > (1 << 27) || n_rows / 256 + 1 > (int64_t)(1 << 22) / (d_out / 256 + 1))
    return fail(MLA_ERR_UNSUPPORTED, "n_rows = %lld, d_out = %d: too many tiles", (long long)n_rows, d_out);
  if (n_rows == 0) return MLA_OK;
  if (z_codes == nullptr || z_scales == nullptr || w_codes == nullptr || w_scales == nullptr || y == nullptr)
    return fail(MLA_ERR_NULL, "z_codes, z_scales, w_codes, w_scales and y are required");
  if (!aligned16(z_codes) || !aligned16(w_codes) || !aligned16(y))
    return fail(MLA_ERR_SHAPE, "z_codes, w_codes and y must be 16-byte aligned");
  if (!aligned(z_scales, 4) || !aligned(w_scales, 4)) return fail(MLA_ERR_SHAPE, "scales must be 4-byte aligned");
  const mla::WbI8Args a{reinterpret_cast<const int8_t*>(z_codes), z_scales, reinterpret_cast<const int8_t*>(w_codes), w_scales, y,
                        n_rows, d_in, d_out, out_dtype == MLA_BF16 ? 1 : 0};
  const hipError_t e = mla::launch_wb_i8(a, reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? MLA_OK : hip_fail(e, "8-bit W_b kernel");
}

mla_status mla_moe_experts_i8_query(const mla_moe_layer* layer, int64_t n_rows, int32_t out_dtype, size_t* ws_bytes) {
  mla::clear_detail();
  if (ws_bytes == nullptr) return fail(MLA_ERR_NULL, "ws_bytes is NULL");
  ExpertsSplit S;
  const mla_status st = experts_split(layer, n_rows, out_dtype, &S);
  if (st != MLA_OK) return st;
  *ws_bytes = S.total;
  return MLA_OK;
}

mla_status mla_moe_experts_i8(const mla_moe_layer* layer, int64_t n_rows, const void* x, int64_t x_stride, const int32_t* expert_idx,
                              const float* expert_w, const int32_t* fanout, const void* w_gate_up, const float* s_gate_up,
                              const void* w_down, const float* s_down, int32_t out_dtype, void* y, void* workspace, size_t ws_bytes,
                              void* stream) {
  mla::clear_detail();
  ExpertsSplit S;
  const mla_status st = experts_split(layer, n_rows, out_dtype, &S);
  if (st != MLA_OK) return st;
  if (x_stride < layer->d_model || x_stride % 8 != 0)
    return fail(MLA_ERR_SHAPE, "x_stride = %lld must be a multiple of 8, at least d_model", (long long)x_stride);
  if (n_rows > INT64_MAX / 2 / x_stride) return fail(MLA_ERR_SHAPE, "n_rows * x_stride overflows");
  if (n_rows == 0) return MLA_OK;
  if (x == nullptr || expert_idx == nullptr || expert_w == nullptr || w_gate_up == nullptr || s_gate_up == nullptr ||
      w_down == nullptr || s_down == nullptr || y == nullptr || workspace == nullptr)
    return fail(MLA_ERR_NULL, "x, expert_idx, expert_w, the weights, their scales, y and workspace are required");
  const void* wide[] = {x, w_gate_up, s_gate_up, w_down, s_down, y};
  for (const void* q : wide)
    if (!aligned16(q)) return fail(MLA_ERR_SHAPE, "x, the weights, their scales and y must be 16-byte aligned");
  if (!aligned(expert_idx, 4) || !aligned(expert_w, 4) || !aligned(fanout, 4))
    return fail(MLA_ERR_SHAPE, "expert_idx, expert_w and fanout must be 4-byte aligned");
  if (!aligned(workspace, 256)) return fail(MLA_ERR_SHAPE, "workspace must be 256-byte aligned");
  if (ws_bytes < S.total) return fail(MLA_ERR_WORKSPACE, "workspace %zu bytes < required %zu", ws_bytes, S.total);
  unsigned char* W = reinterpret_cast<unsigned char*>(workspace);
  mla::ExpertsArgs a{};
  a.x = reinterpret_cast<const uint16_t*>(x);
  a.idx = expert_idx;
  a.ew = expert_w;
  a.fanout = fanout;
  a.w_gu = reinterpret_cast<const int8_t*>(w_gate_up);
  a.s_gu = s_gate_up;
  a.w_down = reinterpret_cast<const int8_t*>(w_down);
  a.s_down = s_down;
  a.y = y;
  a.n_rows = n_rows;
  a.x_stride = x_stride;
  a.d_model = layer->d_model;
  a.d_ffn = layer->d_ffn;
  a.n_experts = layer->n_experts;
  a.first = layer->first_expert;
  a.top_k = layer->top_k;
  a.y_bf16 = out_dtype == MLA_BF16;
  a.hist = reinterpret_cast<int32_t*>(W + S.off_hist);
  a.head = reinterpret_cast<int32_t*>(W + S.off_head);
  a.tiles = reinterpret_cast<mla::ExpertTile*>(W + S.off_tiles);
  a.pairs = reinterpret_cast<int2*>(W + S.off_pairs);
  a.xq = reinterpret_cast<int8_t*>(W + S.off_xq);
  a.xs = reinterpret_cast<float*>(W + S.off_xs);
  a.h = reinterpret_cast<uint16_t*>(W + S.off_h);
  a.hq = reinterpret_cast<int8_t*>(W + S.off_hq);
  a.hs = reinterpret_cast<float*>(W + S.off_hs);
  a.part = reinterpret_cast<float*>(W + S.off_part);
  a.tile_rows = S.tile_rows;
  a.few = S.few;
  const hipError_t e = mla::launch_experts(a, reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? MLA_OK : hip_fail(e, "experts' kernels");
}

}  // extern "C"

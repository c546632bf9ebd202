// Entry points of the 4-bit format, the paged 4-bit latent cache and the attention over
// it: argument checks, the attention's split of the work, dispatch.
#include <algorithm>
#include <cmath>

#include "host.h"
#include "mx4.h"

namespace {

using mla::aligned16;
using mla::fail;
using mla::hip_fail;

mla_status check_cache_geom(const mla_geom* g) {
  const mla_status st = mla::check_geom(g, false);
  if (st != MLA_OK) return st;
  if (g->d_latent != 512 || g->d_rope != 64)
    return fail(MLA_ERR_UNSUPPORTED, "the paged cache is built for (d_latent, d_rope) = (512, 64)");
  if (g->value_rope) return fail(MLA_ERR_UNSUPPORTED, "the paged cache is built for the latent as the value");
  return MLA_OK;
}

mla_status check_pages(int32_t page_rows) {
  if (page_rows < mla::kCacheTile || page_rows % mla::kCacheTile != 0)
    return fail(MLA_ERR_SHAPE, "page_rows = %d must be a positive multiple of %d", page_rows, mla::kCacheTile);
  if (page_rows > MLA_CACHE_MAX_PAGE_ROWS)
    return fail(MLA_ERR_UNSUPPORTED, "page_rows = %d; built: up to %d", page_rows, MLA_CACHE_MAX_PAGE_ROWS);
  return MLA_OK;
}

mla_status check_cache(int64_t cache_pages, int32_t page_rows) {
  const mla_status st = check_pages(page_rows);
  if (st != MLA_OK) return st;
  if (cache_pages < 1) return fail(MLA_ERR_SHAPE, "cache_pages = %lld", (long long)cache_pages);
  if (cache_pages > INT32_MAX / page_rows)
    return fail(MLA_ERR_UNSUPPORTED, "%lld pages of %d rows: more than 2^31-1 rows", (long long)cache_pages, page_rows);
  return MLA_OK;
}

mla_status check_rows_call(const mla_geom* geom, int64_t n_rows, const void* kv, int64_t kv_stride, const int32_t* slots,
                           int64_t cache_pages, int32_t page_rows, const void* cache) {
  mla_status st = check_cache_geom(geom);
  if (st != MLA_OK) return st;
  if ((st = check_cache(cache_pages, page_rows)) != MLA_OK) return st;
  if (n_rows < 0) return fail(MLA_ERR_SHAPE, "n_rows = %lld", (long long)n_rows);
  const int32_t d = geom->d_latent + geom->d_rope;
  if (kv_stride < d || kv_stride % 8 != 0)
    return fail(MLA_ERR_SHAPE, "kv_stride = %lld must be a multiple of 8, at least %d", (long long)kv_stride, d);
  if (n_rows > INT64_MAX / 2 / kv_stride) return fail(MLA_ERR_SHAPE, "n_rows * kv_stride overflows");
  if (n_rows > 0 && (kv == nullptr || slots == nullptr || cache == nullptr))
    return fail(MLA_ERR_NULL, "kv, slots and cache are required");
  if (!aligned16(kv) || !aligned16(cache)) return fail(MLA_ERR_SHAPE, "kv and cache must be 16-byte aligned");
  if ((reinterpret_cast<uintptr_t>(slots) & 3u) != 0) return fail(MLA_ERR_SHAPE, "slots must be 4-byte aligned");
  return MLA_OK;
}

// RoPE frequencies in revolutions, base^(-2j/d_r) / (2 pi), as powers of the first ratio:
// 32 pow() calls would be a fifth of a small call's time.  The ratio is off by up to two half
// steps (2^-53 of it each) and every product adds one: the j-th by up to 3 j + 1.  At position
// 2^31 that is an angle of 1e-6 for base 10000 and of 2.3e-5 for bases next to 1, at 2^18 a
// 8192th of it; the sine's own error is 4e-7.
void rope_turns(const mla_geom* g, double* theta) {
  const double ratio = std::pow(g->rope_base, -2.0 / g->d_rope);
  double v = 1.0 / 6.283185307179586476925286766559;
  for (int j = 0; j < g->d_rope / 2; ++j, v *= ratio) theta[j] = v;
}

mla::CacheRowsArgs rows_args(const mla_geom* geom, int64_t n_rows, const void* kv, int64_t kv_stride, const int32_t* pos,
                             const int32_t* slots, int64_t cache_pages, int32_t page_rows, const void* cache) {
  mla::CacheRowsArgs a{};
  a.kv = const_cast<void*>(kv);
  a.pos = pos;
  a.slots = slots;
  a.cache = reinterpret_cast<unsigned char*>(const_cast<void*>(cache));
  a.n_rows = n_rows;
  a.kv_stride = kv_stride;
  a.n_slots = (int32_t)(cache_pages * page_rows);
  a.page_rows = page_rows;
  rope_turns(geom, a.rope.theta);
  return a;
}

mla_status check_mx4(int64_t n_rows, int32_t n_cols, const void* x, int64_t x_stride, const void* codes, const void* scales) {
  if (n_rows < 0) return fail(MLA_ERR_SHAPE, "n_rows = %lld", (long long)n_rows);
  if (n_cols < 32 || n_cols % 32 != 0) return fail(MLA_ERR_SHAPE, "n_cols = %d must be a positive multiple of 32", n_cols);
  if (n_cols > MLA_MX4_MAX_COLS) return fail(MLA_ERR_UNSUPPORTED, "n_cols = %d; built: up to %d", n_cols, MLA_MX4_MAX_COLS);
  if (x_stride < n_cols || x_stride % 8 != 0)
    return fail(MLA_ERR_SHAPE, "x_stride = %lld must be a multiple of 8, at least n_cols", (long long)x_stride);
  if (n_rows > INT64_MAX / 2 / x_stride) return fail(MLA_ERR_SHAPE, "n_rows * x_stride overflows");
  if (n_rows > 0 && (x == nullptr || codes == nullptr || scales == nullptr))
    return fail(MLA_ERR_NULL, "x, codes and scales are required");
  if (!aligned16(x) || !aligned16(codes)) return fail(MLA_ERR_SHAPE, "x and codes must be 16-byte aligned");
  return MLA_OK;
}

// How mla_cache_attend splits its work, and its workspace
struct AttendSplit {
  int32_t block, n_blocks, shares;
  int64_t off_long, off_ml, off_o;
  size_t total;
};

// Head-rows per workgroup: 64, or 32 or 16 where a request has no more (a block's scores
// and outputs are paid whole).  Shares: one workgroup a compute unit over all blocks.
mla_status attend_split(const mla_geom* geom, int32_t n_seqs, int32_t n_q, int32_t max_pages, int32_t page_rows, AttendSplit* S) {
  mla_status st = check_cache_geom(geom);
  if (st != MLA_OK) return st;
  if ((st = check_pages(page_rows)) != MLA_OK) return st;
  if (n_seqs < 0 || n_q < 1 || max_pages < 0)
    return fail(MLA_ERR_SHAPE, "n_seqs = %d, n_q = %d, max_pages = %d", n_seqs, n_q, max_pages);
  if (n_seqs > 65535) return fail(MLA_ERR_UNSUPPORTED, "n_seqs = %d; built: up to 65535", n_seqs);
  const int64_t rows = (int64_t)n_q * geom->n_heads;
  if (rows > MLA_CACHE_MAX_HEAD_ROWS)
    return fail(MLA_ERR_UNSUPPORTED, "n_q * n_heads = %lld; built: up to %d", (long long)rows, MLA_CACHE_MAX_HEAD_ROWS);
  if ((int64_t)n_seqs * max_pages > INT32_MAX / (page_rows / mla::kCacheTile))
    return fail(MLA_ERR_UNSUPPORTED, "n_seqs * max_pages = %lld: too many tiles", (long long)n_seqs * max_pages);
  S->block = rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
  S->n_blocks = (int32_t)((rows + S->block - 1) / S->block);
  S->shares = std::max(1, mla::kMaxShares / S->n_blocks);
  auto up = [](int64_t x) { return (x + 255) / 256 * 256; };
  const int64_t part_rows = (int64_t)2 * S->shares * S->n_blocks * S->block;
  S->off_long = up(((int64_t)n_seqs + 1) * 4);
  S->off_ml = S->off_long + up(mla::kMaxShares / mla::kLongShares * 4);
  S->off_o = S->off_ml + up(part_rows * 4 * 4);
  S->total = (size_t)(S->off_o + part_rows * 512 * 4);
  return MLA_OK;
}

}  // namespace

extern "C" {

mla_status mla_mx4_quantize(int64_t n_rows, int32_t n_cols, const void* x, int64_t x_stride, void* codes, void* scales,
                            void* stream) {
  mla::clear_detail();
  const mla_status st = check_mx4(n_rows, n_cols, x, x_stride, codes, scales);
  if (st != MLA_OK || n_rows == 0) return st;
  const mla::Mx4Args a{x, codes, scales, n_rows, x_stride, n_cols};
  const hipError_t e = mla::launch_mx4_quantize(a, reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? MLA_OK : hip_fail(e, "quantize kernel");
}

mla_status mla_mx4_dequantize(int64_t n_rows, int32_t n_cols, const void* codes, const void* scales, void* x,
                              int64_t x_stride, void* stream) {
  mla::clear_detail();
  const mla_status st = check_mx4(n_rows, n_cols, x, x_stride, codes, scales);
  if (st != MLA_OK || n_rows == 0) return st;
  const mla::Mx4Args a{x, const_cast<void*>(codes), const_cast<void*>(scales), n_rows, x_stride, n_cols};
  const hipError_t e = mla::launch_mx4_dequantize(a, reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? MLA_OK : hip_fail(e, "dequantize kernel");
}

mla_status mla_shared_wb_mx4(int64_t n_rows, int32_t d_in, int32_t d_out, const void* z, const void* w_codes,
                             const void* w_scales, int32_t out_dtype, void* y, void* stream) {
  mla::clear_detail();
  if (n_rows < 0) return fail(MLA_ERR_SHAPE, "n_rows = %lld", (long long)n_rows);
  if (d_in < 64 || d_in % 64 != 0) return fail(MLA_ERR_SHAPE, "d_in = %d must be a positive multiple of 64", d_in);
  if (d_in > MLA_WB_MAX_D_IN) return fail(MLA_ERR_UNSUPPORTED, "d_in = %d; built: up to %d", d_in, MLA_WB_MAX_D_IN);
  if (d_out < 1) return fail(MLA_ERR_SHAPE, "d_out = %d", d_out);
  if (d_out > MLA_WB_MX4_MAX_D_OUT)
    return fail(MLA_ERR_UNSUPPORTED, "d_out = %d; built: up to %d", d_out, MLA_WB_MX4_MAX_D_OUT);
  if (out_dtype != MLA_BF16 && out_dtype != MLA_F32) return fail(MLA_ERR_SHAPE, "out_dtype %d", out_dtype);
  if (n_rows > MLA_WB_MX4_MAX_ROWS)
    return fail(MLA_ERR_UNSUPPORTED, "n_rows = %lld; built: up to %d (mla_mx4_dequantize, then mla_shared_wb)",
                (long long)n_rows, MLA_WB_MX4_MAX_ROWS);
  if (n_rows == 0) return MLA_OK;
  if (z == nullptr || w_codes == nullptr || w_scales == nullptr || y == nullptr)
    return fail(MLA_ERR_NULL, "z, w_codes, w_scales and y are required");
  if (!aligned16(z) || !aligned16(w_codes) || !aligned16(y))
    return fail(MLA_ERR_SHAPE, "z, w_codes and y must be 16-byte aligned");
  if ((reinterpret_cast<uintptr_t>(w_scales) & 3u) != 0) return fail(MLA_ERR_SHAPE, "w_scales must be 4-byte aligned");
  const mla::WbMx4Args a{reinterpret_cast<const uint16_t*>(z), reinterpret_cast<const uint8_t*>(w_codes),
                         reinterpret_cast<const uint8_t*>(w_scales), y, n_rows, d_in, d_out,
                         out_dtype == MLA_BF16 ? 1 : 0};
  const hipError_t e = mla::launch_wb_mx4(a, reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? MLA_OK : hip_fail(e, "4-bit W_b kernel");
}

mla_status mla_cache_append(const mla_geom* geom, int64_t n_rows, const void* kv, int64_t kv_stride, const int32_t* pos,
                            const int32_t* slots, int64_t cache_pages, int32_t page_rows, void* cache, void* stream) {
  mla::clear_detail();
  const mla_status st = check_rows_call(geom, n_rows, kv, kv_stride, slots, cache_pages, page_rows, cache);
  if (st != MLA_OK || n_rows == 0) return st;
  if ((reinterpret_cast<uintptr_t>(pos) & 3u) != 0) return fail(MLA_ERR_SHAPE, "pos must be 4-byte aligned");
  const hipError_t e =
      mla::launch_cache_append(rows_args(geom, n_rows, kv, kv_stride, pos, slots, cache_pages, page_rows, cache),
                               reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? MLA_OK : hip_fail(e, "append kernel");
}

mla_status mla_cache_gather(const mla_geom* geom, int64_t n_rows, const int32_t* slots, int64_t cache_pages,
                            int32_t page_rows, const void* cache, void* kv, int64_t kv_stride, void* stream) {
  mla::clear_detail();
  const mla_status st = check_rows_call(geom, n_rows, kv, kv_stride, slots, cache_pages, page_rows, cache);
  if (st != MLA_OK || n_rows == 0) return st;
  const hipError_t e =
      mla::launch_cache_gather(rows_args(geom, n_rows, kv, kv_stride, nullptr, slots, cache_pages, page_rows, cache),
                               reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? MLA_OK : hip_fail(e, "gather kernel");
}

mla_status mla_cache_attend_query(const mla_geom* geom, int32_t n_seqs, int32_t n_q, int32_t max_pages, int32_t page_rows,
                                  size_t* ws_bytes) {
  mla::clear_detail();
  if (ws_bytes == nullptr) return fail(MLA_ERR_NULL, "ws_bytes is NULL");
  AttendSplit S;
  const mla_status st = attend_split(geom, n_seqs, n_q, max_pages, page_rows, &S);
  if (st != MLA_OK) return st;
  *ws_bytes = S.total;
  return MLA_OK;
}

mla_status mla_cache_attend(const mla_geom* geom, int32_t n_seqs, int32_t n_q, const void* q, const int32_t* pos,
                            const mla_page* pages, const int32_t* seq_pages, int32_t max_pages, int64_t cache_pages,
                            int32_t page_rows, const void* cache, void* out_o, float* out_lse, void* workspace,
                            size_t ws_bytes, void* stream) {
  mla::clear_detail();
  AttendSplit S;
  mla_status st = attend_split(geom, n_seqs, n_q, max_pages, page_rows, &S);
  if (st != MLA_OK) return st;
  if ((st = check_cache(cache_pages, page_rows)) != MLA_OK) return st;
  if (n_seqs == 0) return MLA_OK;
  if (q == nullptr || pos == nullptr || seq_pages == nullptr || cache == nullptr || out_o == nullptr || workspace == nullptr)
    return fail(MLA_ERR_NULL, "q, pos, seq_pages, cache, out_o and workspace are required");
  if (max_pages > 0 && pages == nullptr) return fail(MLA_ERR_NULL, "pages is NULL");
  if (!aligned16(q) || !aligned16(pages) || !aligned16(cache) || !aligned16(out_o))
    return fail(MLA_ERR_SHAPE, "q, pages, cache and out_o must be 16-byte aligned");
  if (((reinterpret_cast<uintptr_t>(pos) | reinterpret_cast<uintptr_t>(seq_pages) | reinterpret_cast<uintptr_t>(out_lse)) & 3u) != 0)
    return fail(MLA_ERR_SHAPE, "pos, seq_pages and out_lse must be 4-byte aligned");
  if ((reinterpret_cast<uintptr_t>(workspace) & 255u) != 0) return fail(MLA_ERR_SHAPE, "workspace must be 256-byte aligned");
  if (ws_bytes < S.total) return fail(MLA_ERR_WORKSPACE, "workspace %zu bytes < required %zu", ws_bytes, S.total);
  unsigned char* W = reinterpret_cast<unsigned char*>(workspace);
  mla::CacheAttendArgs a{};
  a.cache = reinterpret_cast<const unsigned char*>(cache);
  a.q = reinterpret_cast<const uint16_t*>(q);
  a.pos = pos;
  a.pages = pages;
  a.seq_pages = seq_pages;
  a.out_o = reinterpret_cast<uint16_t*>(out_o);
  a.out_lse = out_lse;
  a.tile_base = reinterpret_cast<int32_t*>(W);
  a.long_seq = reinterpret_cast<int32_t*>(W + S.off_long);
  a.part_ml = reinterpret_cast<float*>(W + S.off_ml);
  a.part_o = reinterpret_cast<float*>(W + S.off_o);
  a.n_seqs = n_seqs;
  a.n_q = n_q;
  a.n_heads = geom->n_heads;
  a.max_pages = max_pages;
  a.page_rows = page_rows;
  a.cache_pages = (int32_t)cache_pages;
  a.page_tiles = page_rows / mla::kCacheTile;
  a.inv_page_tiles = 1.0 / a.page_tiles;
  a.inv_shares = 1.0 / S.shares;
  a.inv_blocks = 1.0 / S.n_blocks;
  a.block = S.block;
  a.n_blocks = S.n_blocks;
  a.shares = S.shares;
  a.scale_log2 = geom->softmax_scale * 1.4426950408889634f;
  rope_turns(geom, a.rope.theta);
  const hipError_t e = mla::launch_cache_attend(a, reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? MLA_OK : hip_fail(e, "cache attention kernels");
}

}  // extern "C"

// Routing of token rows to experts.  Scores s are the softmax or the sigmoid of the router's
// logits, c = s + bias chooses: the best groups of experts by the sum of their best c, among
// them the top_k experts, equal ones to the lower index.  Weights are the chosen s.
//
// Which expert comes first hangs on values next to one another, so choices and the fanout are
// those of 64-bit scores.
#include "route.h"

#include <algorithm>

namespace mla {
namespace {

__device__ __forceinline__ float logit(const RouteArgs& a, int64_t r, int e) {
  return a.logits_bf16 ? __uint_as_float((uint32_t)((const uint16_t*)a.logits)[r * a.stride + e] << 16)
                       : ((const float*)a.logits)[r * a.stride + e];
}

// order of a value among 64-bit ones, NaN before all
__device__ __forceinline__ uint64_t order_bits(double v) {
  if (v != v) return 0;
  const uint64_t u = (uint64_t)__double_as_longlong(v + 0.0);   // -0 as +0
  return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}

__device__ __forceinline__ double wave_max(double v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v = fmax(v, __shfl_xor(v, d, 64));
  return v;
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d, 64);
  return v;
}

// A row by a whole wave in 64 bits; lane holds experts lane, lane + 64, ...  `group` is LDS of
// the wave, [E].
template <int NV>
__device__ void route_exact(const RouteArgs& a, int64_t r, int lane, double* group) {
  const int E = a.n_experts;
  double s[NV];
  uint64_t key[NV];   // order of c, or of the logit without a bias
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int e = 64 * i + lane;
    s[i] = e < E ? (double)logit(a, r, e) : -INFINITY;
    key[i] = order_bits(s[i]);
  }
  if (a.sigmoid) {
#pragma unroll
    for (int i = 0; i < NV; ++i) s[i] = 1.0 / (1.0 + exp(-s[i]));
  } else {
    double m = -INFINITY, sum = 0.0;
#pragma unroll
    for (int i = 0; i < NV; ++i) m = fmax(m, s[i]);
    m = wave_max(m);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      // a row of -infinity has no weight; lanes past E add none
      s[i] = 64 * i + lane < E && !(m == -INFINITY && s[i] == m) ? exp(s[i] - m) : 0.0;
      sum += s[i];
    }
    sum = wave_sum(sum);
    if (sum != 0.0)
#pragma unroll
      for (int i = 0; i < NV; ++i) s[i] /= sum;
  }
  uint32_t open = 0;   // experts of the lane that may be chosen
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int e = 64 * i + lane;
    if (e >= E) continue;
    open |= 1u << i;
    double c = s[i];
    if (a.bias != nullptr) {
      c += (double)a.bias[e];
      key[i] = order_bits(c);
    }
    if (a.top_groups < a.n_groups) group[e] = c;
  }
  if (a.top_groups < a.n_groups) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");   // the wave's own LDS accesses, in order
    const int G = a.n_groups, size = E / G;
    uint64_t score = 0;
    if (lane < G) {
      double v0 = -INFINITY, v1 = -INFINITY;
      uint64_t k0 = 0, k1 = 0;
      bool any = false;
      for (int i = 0; i < size; ++i) {
        const double v = group[lane * size + i];
        const uint64_t k = order_bits(v);
        if (!any || k > k0) {
          v1 = v0;
          k1 = k0;
          v0 = v;
          k0 = k;
          any = true;
        } else if (i == 1 || k > k1) {
          v1 = v;
          k1 = k;
        }
      }
      score = order_bits(a.group_best > 1 && size > 1 ? v0 + v1 : v0);
    }
    int before = 0;
    for (int g = 0; g < G; ++g) {
      const uint64_t o = (uint64_t)__shfl((long long)score, g, 64);
      before += o > score || (o == score && g < lane);
    }
    const uint64_t kept = __ballot(lane < G && before < a.top_groups);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int e = 64 * i + lane;
      if (e < E && !((kept >> (e / size)) & 1)) open &= ~(1u << i);
    }
  }
  int idx[kMoeMaxTopK];
  double w[kMoeMaxTopK], total = 0.0;
#pragma unroll
  for (int j = 0; j < kMoeMaxTopK; ++j) {
    idx[j] = 0;
    w[j] = 0.0;
    if (j >= a.top_k) continue;
    uint64_t bk = 0;
    int be = INT32_MAX;   // none left
    double bs = 0.0;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (((open >> i) & 1) && (be == INT32_MAX || key[i] > bk)) {
        bk = key[i];
        be = 64 * i + lane;
        bs = s[i];
      }
    const int mine = be;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const uint64_t ok = (uint64_t)__shfl_xor((long long)bk, d, 64);
      const int oe = __shfl_xor(be, d, 64);
      const double os = __shfl_xor(bs, d, 64);
      if (oe != INT32_MAX && (be == INT32_MAX || ok > bk || (ok == bk && oe < be))) {
        bk = ok;
        be = oe;
        bs = os;
      }
    }
    if (mine == be) open &= ~(1u << (be >> 6));
    idx[j] = be;
    w[j] = bs;
    total += bs;
  }
  double upto = 0.0, div = a.renormalize && total != 0.0 ? total : 1.0;
  int K = a.top_k;
  bool done = false;
#pragma unroll
  for (int j = 0; j < kMoeMaxTopK; ++j) {
    if (j >= a.top_k) continue;
    upto += w[j];
    if (!done && j + 1 >= a.min_k && total > 0.0 && upto >= (double)a.tau * total) {
      K = j + 1;
      done = true;
    }
    if (lane == j) {
      a.expert_idx[r * a.top_k + j] = idx[j];
      a.expert_w[r * a.top_k + j] = (float)(w[j] / div * (double)a.scale);
    }
  }
  if (lane == 0 && a.fanout != nullptr) a.fanout[r] = K;
}

template <int NV>
__global__ __launch_bounds__(256) void route_wave_kernel(RouteArgs a) {
  __shared__ double group[4][64 * NV];
  if (a.expert_count != nullptr && blockIdx.x == 0)
    for (int i = threadIdx.x; i < a.n_experts; i += 256) a.expert_count[i] = 0;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int64_t r = (int64_t)blockIdx.x * 4 + wave; r < a.n_rows; r += (int64_t)gridDim.x * 4) {
    route_exact<NV>(a, r, lane, group[wave]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
  }
}

}  // namespace

hipError_t launch_moe_route(const RouteArgs& a, hipStream_t s) {
  if (a.n_rows == 0 && a.expert_count == nullptr) return hipSuccess;
  const dim3 grid((unsigned)std::max<int64_t>(1, std::min<int64_t>((a.n_rows + 3) / 4, 4096))), blk(256);   // no row: the counts are cleared
  const int E = a.n_experts;
  if (E <= 64) route_wave_kernel<1><<<grid, blk, 0, s>>>(a);
  else if (E <= 128) route_wave_kernel<2><<<grid, blk, 0, s>>>(a);
  else if (E <= 256) route_wave_kernel<4><<<grid, blk, 0, s>>>(a);
  else if (E <= 512) route_wave_kernel<8><<<grid, blk, 0, s>>>(a);
  else route_wave_kernel<16><<<grid, blk, 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.expert_count == nullptr || a.n_rows == 0) return e;
  MoeArgs c{};
  c.expert_idx = a.expert_idx;
  c.fanout = a.fanout;
  c.expert_count = a.expert_count;
  c.n_rows = a.n_rows;
  c.n_experts = E;
  c.top_k = a.top_k;
  return launch_moe_count(c, s);
}

}  // namespace mla

// Routing of token rows to experts.  Scores s are the softmax or the sigmoid of the router's
// logits, c = s + bias chooses: the best groups of experts by the sum of their best c, among
// them the top_k experts, equal ones to the lower index.  Weights are the chosen s.
//
// Which expert comes first hangs on values next to one another, so choices and fanouts are those
// of 64-bit scores.  route_exact computes them so, a row a wave.  Up to 256 experts a row is
// first tried in 32 bits by 16 lanes (route_row_kernel, four rows a wave): c becomes a 24-bit
// fixed-point code over its whole range, above the inverted index in a 32-bit key, and whatever
// hangs on two codes that the errors could have swapped sends its row to route_exact: one in some
// hundreds of rows of random logits.
#include "rank.h"
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

// What ranks a row's experts in route_row_kernel
enum RouteBy {
  kByLogit,     // no bias: the order of the logits themselves
  kBySigmoid,   // c = sigmoid + bias
  kBySoftmax,   // c = softmax + bias
};

__device__ __forceinline__ float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }

template <int CTRL>
__device__ __forceinline__ float fmax_dpp(float v) {
  return fmaxf(v, __uint_as_float(dpp<CTRL>(__float_as_uint(v))));
}
__device__ __forceinline__ float row_max(float v) {
  v = fmax_dpp<0xB1>(v);
  v = fmax_dpp<0x4E>(v);
  v = fmax_dpp<0x141>(v);
  return fmax_dpp<0x140>(v);
}
__device__ __forceinline__ float row_sum(float v) {
  v += __uint_as_float(dpp<0xB1>(__float_as_uint(v)));
  v += __uint_as_float(dpp<0x4E>(__float_as_uint(v)));
  v += __uint_as_float(dpp<0x141>(__float_as_uint(v)));
  return v + __uint_as_float(dpp<0x140>(__float_as_uint(v)));
}

// lanes of the row whose key is above this lane's
template <int R>
__device__ __forceinline__ uint32_t above(uint32_t key) {
  const uint32_t n = dpp<0x120 + R>(key) > key ? 1u : 0u;   // row_ror:R
  if constexpr (R > 1) return n + above<R - 1>(key);
  return n;
}

// M consecutive logits of row r from expert M sl on, as f32; past E: -infinity
template <int M, bool BF16>
__device__ __forceinline__ void load_logits(const RouteArgs& a, bool wide, int64_t r, int sl, float (&v)[M]) {
  const int e0 = M * sl, E = a.n_experts;
  constexpr int V = M % 4 == 0 ? 4 : 2;
#pragma unroll
  for (int i = 0; i < M; i += V) {
    const int e = e0 + i;
    if (wide && e + V <= E) {
      if constexpr (BF16) {
        const uint32_t* p = (const uint32_t*)((const uint16_t*)a.logits + r * a.stride + e);
        uint32_t u[V / 2];
        if constexpr (V == 4) {
          const u32x2 w = *(const u32x2*)p;
          u[0] = w[0];
          u[1] = w[1];
        } else {
          u[0] = *p;
        }
#pragma unroll
        for (int k = 0; k < V / 2; ++k) {
          v[i + 2 * k] = bf16_lo(u[k]);
          v[i + 2 * k + 1] = bf16_hi(u[k]);
        }
      } else {
        const float* p = (const float*)a.logits + r * a.stride + e;
        if constexpr (V == 4) {
          const f32x4 w = *(const f32x4*)p;
#pragma unroll
          for (int k = 0; k < 4; ++k) v[i + k] = w[k];
        } else {
          const u32x2 w = *(const u32x2*)p;
          v[i] = __uint_as_float(w[0]);
          v[i + 1] = __uint_as_float(w[1]);
        }
      }
    } else {
#pragma unroll
      for (int k = 0; k < V; ++k) v[i + k] = e + k < E ? logit(a, r, e + k) : -INFINITY;
    }
  }
}

// 16 lanes a row, four rows a wave; lane sl holds experts M sl .. M sl + M - 1, so that with groups
// (E = 16 M, n_groups divides 16) a group is 16 / n_groups whole lanes.  Each lane keeps its DEPTH
// largest keys sorted (a max and medians per key); a round takes the row's maximum of the lanes'
// largest in four DPP steps and the owner drops it.
//
// Errors of the codes, in steps of 2^-24 of the range 1 + 2 B of c (B the largest finite |bias|):
// the sigmoid's exponential is off by (1.5 |l| + 2) 2^-24 of itself, of which s (1 - s) <= 1/4 and
// s (1 - s) |l| < 0.23 reach s; 1 + e, its reciprocal and the bias add 3 s + 1 + B: below 5 (1 + B).
// With the conversion's two a code is off by at most 7, and the order of two that are 17 apart is
// certain.  A softmax score takes the sum's error besides (its terms' 1.5 d + 2 weighted by e^-d,
// and 20 additions): below 50, 113 apart.  A group's score is the sum of two codes: twice that.  In
// kByLogit codes are the upper 24 bits of the logit's order: exact for bf16, else equal codes are
// not certain.
template <int M, bool BF16, int BY>
__global__ __launch_bounds__(256, 4) void route_row_kernel(RouteArgs a, bool wide, bool count) {
  __shared__ double group[4][256];
  __shared__ uint32_t hist[256];
  if (count) {   // the only workgroup: it counts as well
    hist[threadIdx.x] = 0;
    __syncthreads();
  } else if (a.expert_count != nullptr && blockIdx.x == 0) {
    if ((int)threadIdx.x < a.n_experts) a.expert_count[threadIdx.x] = 0;
  }
  constexpr int DEPTH = M < 6 ? M : 6;
  constexpr uint32_t APART = BY == kBySigmoid ? 17 : BY == kBySoftmax ? 113 : BF16 ? 0 : 1;
  constexpr uint32_t kNegInfCode = 0x007FFFFFu >> 8;   // of total_order_bits(-infinity)
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sl = lane & 15, slot = lane >> 4;
  const int E = a.n_experts, TK = a.top_k, LG = 16 / a.n_groups;
  const bool groups = a.top_groups < a.n_groups;
  float bias[BY == kByLogit ? 1 : M], low = 0.f, unit = 0.f;
  if constexpr (BY != kByLogit) {
    float b = 0.f;
#pragma unroll
    for (int i = 0; i < M; ++i) {
      bias[i] = a.bias != nullptr && M * sl + i < E ? a.bias[M * sl + i] : 0.f;
      if (fabsf(bias[i]) < INFINITY) b = fmaxf(b, fabsf(bias[i]));
    }
    low = row_max(b);
    unit = 16777200.f / (1.f + 2.f * low);   // codes 1 .. 2^24 - 1, larger c (an infinite bias) clamped
  }
  const int64_t stride = (int64_t)gridDim.x * 16, last = a.n_rows - 1;
  int64_t r = ((int64_t)blockIdx.x * 4 + wave) * 4 + slot;
  // every lane runs the same number of turns (rows past the end work on a copy of the last and
  // write nothing), so the DPP exchanges see whole rows
  const int64_t first = r - slot;
  uint64_t again = 0;
  int turn = 0;
  float cur[M];
  if (r - slot <= last) load_logits<M, BF16>(a, wide, r < last ? r : last, sl, cur);
  for (; r - slot <= last; r += stride) {
    const int64_t rc = r < last ? r : last;
    float top = 0.f, total = 0.f;   // softmax: largest logit, sum of exponentials
    if (!a.sigmoid) {
      top = cur[0];
#pragma unroll
      for (int i = 1; i < M; ++i) top = fmaxf(top, cur[i]);
      top = row_max(top);
      float part[4] = {};
#pragma unroll
      for (int i = 0; i < M; ++i) {
        const float e = exp_fast(cur[i] - top);   // past E: 0
        part[i & 3] += e;
        if constexpr (BY == kBySoftmax) cur[i] = e;
      }
      total = row_sum((part[0] + part[1]) + (part[2] + part[3]));
    }
    const float inv = BY == kBySoftmax ? __builtin_amdgcn_rcpf(total) : 0.f;
    uint32_t m[DEPTH];
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) m[d] = 0;
#pragma unroll
    for (int i = 0; i < M; ++i) {
      const int e = M * sl + i;
      uint32_t code;
      if constexpr (BY == kByLogit) {
        code = total_order_bits(fmaxf(cur[i], -INFINITY) + 0.0f) >> 8;   // NaN as -infinity, -0 as 0
      } else {
        const float s = BY == kBySigmoid ? __builtin_amdgcn_rcpf(1.f + exp_fast(-cur[i])) : cur[i] * inv;
        // v_cvt takes NaN and what is below 0 to 0
        code = (uint32_t)fminf(fmaxf(((s + bias[i]) + low) * unit + 1.f, 1.f), 16777215.f);
      }
      uint32_t x = (code << 8) | (uint32_t)(255 - e);
      x = e < E ? x : 0u;
#pragma unroll
      for (int d = DEPTH - 1; d > 0; --d) m[d] = med_u32(m[d - 1], m[d], x);
      m[0] = max_u32(m[0], x);
    }
    // the next row, over the registers just consumed
    if (r - slot + stride <= last) load_logits<M, BF16>(a, wide, r + stride < last ? r + stride : last, sl, cur);
    bool unsure = false;
    if (groups) {
      uint32_t g0 = m[0] >> 8, g1 = m[1] >> 8;
      auto join = [&](uint32_t o0, uint32_t o1) {
        const uint32_t lo = g0 < o0 ? g0 : o0;
        g0 = max_u32(g0, o0);
        g1 = max_u32(lo, max_u32(g1, o1));
      };
      if (LG > 1) join(dpp<0xB1>(g0), dpp<0xB1>(g1));
      if (LG > 2) join(dpp<0x4E>(g0), dpp<0x4E>(g1));
      if (LG > 4) join(dpp<0x141>(g0), dpp<0x141>(g1));
      const uint32_t score = BY != kByLogit && a.group_best > 1 ? g0 + g1 : g0;
      const uint32_t key = (score << 4) | (uint32_t)(15 - sl / LG);
      const bool kept = (int)above<15>(key) < a.top_groups * LG;
      // the least kept score and the largest other
      const uint32_t least = ~row_max_u32(kept ? ~score : 0u), most = row_max_u32(kept ? 0u : score);
      unsure = least < most + 2 * APART || (BY == kByLogit && least <= kNegInfCode);
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) m[d] = kept ? m[d] : 0u;
    }
    const bool full = M > DEPTH && m[DEPTH - 1] != 0;
    int32_t my_id = 0;
    uint32_t before = 0xFFFFFFFFu;   // code of the rank before
    int drops = 0;
#pragma unroll
    for (int j = 0; j < kMoeMaxTopK; ++j) {
      if (j < TK) {
        const uint32_t top_key = row_max_u32(m[0]);
        if (sl == j) my_id = 255 - (int32_t)(top_key & 0xFFu);
        unsure |= before - (top_key >> 8) < APART;
        before = top_key >> 8;
        const bool own = m[0] == top_key;
        drops += own;
#pragma unroll
        for (int d = 0; d + 1 < DEPTH; ++d) m[d] = own ? m[d + 1] : m[d];
        m[DEPTH - 1] = own ? 0u : m[DEPTH - 1];
      }
    }
    unsure |= before - (row_max_u32(m[0]) >> 8) < APART;   // the runner-up; nothing left: code 0
    unsure |= full && drops >= DEPTH;                      // the lane's next key is not known
    unsure |= BY == kByLogit ? before <= kNegInfCode : before <= APART + 1;
    // the ranks' scores: lane j of the row holds rank j
    const bool rank = sl < TK;
    const float x = rank ? logit(a, rc, my_id) : 0.f;
    const float d = a.sigmoid ? -fabsf(x) : x - top;
    float e = expf(d);
    if (!a.sigmoid) e += e * ((x - d) - top);   // what the rounding of the difference took
    float s = a.sigmoid ? (x < 0.f ? e : 1.f) / (1.f + e) : e / total;
    s = rank ? s : 0.f;
    const float sum = row_sum(s);
    // the sum decides little where it is tiny or not a number
    unsure |= !(sum > 1e-30f);
    float upto = 0.f;
    int K = TK;
    const float want = a.tau * sum, near = 0x1p-18f * sum;
    auto step = [&](float v, int j) {
      if (j < TK) {
        upto += v;
        if (j + 1 >= a.min_k && j + 1 < TK) {
          unsure |= fabsf(upto - want) <= near;
          if (K == TK && upto >= want) K = j + 1;
        }
      }
    };
    step(row_bcast<0>(s), 0);
    step(row_bcast<1>(s), 1);
    step(row_bcast<2>(s), 2);
    step(row_bcast<3>(s), 3);
    step(row_bcast<4>(s), 4);
    step(row_bcast<5>(s), 5);
    step(row_bcast<6>(s), 6);
    step(row_bcast<7>(s), 7);
    const uint64_t odd = __ballot(unsure && r <= last);
    if (r <= last && (odd >> (16 * slot) & 0xFFFF) == 0) {
      if (rank) {
        a.expert_idx[r * TK + sl] = my_id;
        a.expert_w[r * TK + sl] = (a.renormalize ? s / sum : s) * a.scale;
      }
      if (sl == 0 && a.fanout != nullptr) a.fanout[r] = K;
    }
    // a bit a row and turn
    again |= (uint64_t)((odd & 0xFFFF) != 0 | ((odd >> 16 & 0xFFFF) != 0) << 1 | ((odd >> 32 & 0xFFFF) != 0) << 2 | ((odd >> 48) != 0) << 3)
             << (4 * turn);
    ++turn;
  }
  // rows whose order is not certain, each by the whole wave
  for (; again != 0; again &= again - 1) {
    const int at = __builtin_ctzll(again);
    route_exact<4>(a, first + (at >> 2) * stride + (at & 3), lane, group[wave]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
  }
  if (count) {
    __syncthreads();   // the rows are written
    const int n = (int)a.n_rows * TK;
    if ((int)threadIdx.x < n) {
      const int row = threadIdx.x / TK;
      if ((int)threadIdx.x - row * TK < (a.fanout != nullptr ? a.fanout[row] : TK)) atomicAdd(&hist[a.expert_idx[threadIdx.x]], 1u);
    }
    __syncthreads();
    if ((int)threadIdx.x < E) a.expert_count[threadIdx.x] = (int32_t)hist[threadIdx.x];
  }
}

constexpr int64_t kRouteOneBlock = 16;   // rows of a call that one workgroup routes and counts
constexpr int kRouteTurns = 16;          // of a wave, four rows each: a bit of a word a row

template <int M, bool BF16>
hipError_t launch_rows(const RouteArgs& a, bool wide, bool count, hipStream_t s) {
  const int64_t blocks = (a.n_rows + 15) / 16;
  const dim3 grid((unsigned)std::max(std::min<int64_t>(blocks, 2048), (blocks + kRouteTurns - 1) / kRouteTurns)), blk(256);
  if (a.bias == nullptr && (a.top_groups == a.n_groups || a.group_best == 1))
    route_row_kernel<M, BF16, kByLogit><<<grid, blk, 0, s>>>(a, wide, count);
  else if (a.sigmoid) route_row_kernel<M, BF16, kBySigmoid><<<grid, blk, 0, s>>>(a, wide, count);
  else route_row_kernel<M, BF16, kBySoftmax><<<grid, blk, 0, s>>>(a, wide, count);
  return hipGetLastError();
}

template <bool BF16>
hipError_t launch_by_width(const RouteArgs& a, int m, bool count, hipStream_t s) {
  // vectors of 4 (2 where a lane's share is not whole fours) logits
  const int64_t bytes = (m % 4 == 0 ? 4 : 2) * (BF16 ? 2 : 4);
  const bool wide = reinterpret_cast<uintptr_t>(a.logits) % bytes == 0 && a.stride * (BF16 ? 2 : 4) % bytes == 0;
  switch (m) {
    case 4: return launch_rows<4, BF16>(a, wide, count, s);
    case 8: return launch_rows<8, BF16>(a, wide, count, s);
    case 10: return launch_rows<10, BF16>(a, wide, count, s);
    case 12: return launch_rows<12, BF16>(a, wide, count, s);
    default: return launch_rows<16, BF16>(a, wide, count, s);
  }
}

// experts a lane of route_row_kernel, or 0 where the row does not fit it
int row_share(const RouteArgs& a) {
  for (int m : {4, 8, 10, 12, 16}) {
    if (a.n_experts > 16 * m) continue;
    if (a.top_groups == a.n_groups || (a.n_experts == 16 * m && 16 % a.n_groups == 0)) return m;
    return 0;
  }
  return 0;
}

}  // namespace

hipError_t launch_moe_route(const RouteArgs& a, hipStream_t s) {
  if (a.n_rows == 0 && a.expert_count == nullptr) return hipSuccess;
  const int E = a.n_experts, share = a.n_rows > 0 ? row_share(a) : 0;
  hipError_t e;
  if (share != 0) {
    const bool count = a.expert_count != nullptr && a.n_rows <= kRouteOneBlock;
    e = a.logits_bf16 ? launch_by_width<true>(a, share, count, s) : launch_by_width<false>(a, share, count, s);
    if (count) return e;
  } else {
    const dim3 grid((unsigned)std::max<int64_t>(1, std::min<int64_t>((a.n_rows + 3) / 4, 4096))), blk(256);   // no row: the counts are cleared
    if (E <= 64) route_wave_kernel<1><<<grid, blk, 0, s>>>(a);
    else if (E <= 128) route_wave_kernel<2><<<grid, blk, 0, s>>>(a);
    else if (E <= 256) route_wave_kernel<4><<<grid, blk, 0, s>>>(a);
    else if (E <= 512) route_wave_kernel<8><<<grid, blk, 0, s>>>(a);
    else route_wave_kernel<16><<<grid, blk, 0, s>>>(a);
    e = hipGetLastError();
  }
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

// Routing of token rows to experts.  Scores s are the softmax or the sigmoid of the router's
// logits, c = s + bias chooses: the best groups of experts by the sum of their best c, among
// them the top_k experts, equal ones to the lower index.  Weights are the chosen s.
//
// Which expert comes first hangs on values next to one another, so choices and fanouts are those
// of 64-bit scores.  route_exact computes them so, a row a wave.  A row is first tried in 32 bits
// (route_row_kernel, by 16 lanes up to 256 experts, else by a wave): c becomes a fixed-point code of
// 24 or 22 bits over its whole range, above the inverted index in a 32-bit key, and whatever hangs
// on two codes that the errors could have swapped sends its row to route_exact: one in some
// hundreds to thousands of rows of random logits, and more where the biases share an offset, which widens
// the range (264,192 rows of 256: 109 us, with an offset of 5 133, of 50 181).  A lane keeps its 5 or 6
// largest keys, so rows also go there where the groups kept lie on few lanes: all of them where one
// group of one lane gives 6 or more (66,048 rows of 256 in 16 groups, top 8: 335 us, of two groups 125, of
// five 52; in 8 groups, one kept, 170, four 54; one row of the first 20, of the last 8).  Where groups
// do not fit the lanes every row does.
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

__device__ __forceinline__ double from_order_bits(uint64_t k) {
  if (k == 0) return __longlong_as_double(0x7ff8000000000000ll);
  return __longlong_as_double((long long)((k >> 63) ? (k & 0x7FFFFFFFFFFFFFFFull) : ~k));
}

// The wave's own LDS accesses, in order
__device__ __forceinline__ void in_order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup"); }

// A row by a whole wave in 64 bits; lane holds experts lane, lane + 64, ...; `score` and `key` are
// LDS of the wave, [E].  Lane j returns the expert of rank j if the row executes it, else -1.
// Loops stay rolled: where this runs for one row in hundreds its time is that of fetching its
// instructions (unrolled by four, some 150 rows of 264,192 cost 30 us).
__device__ int route_exact(const RouteArgs& a, int64_t r, int lane, double* score, uint64_t* key) {
  const int E = a.n_experts;
  double m = -INFINITY, sum = 0.0;
  if (!a.sigmoid) {
#pragma unroll 1
    for (int e = lane; e < E; e += 64) m = fmax(m, (double)logit(a, r, e));
#pragma unroll 1
    for (int d = 1; d < 64; d *= 2) m = fmax(m, __shfl_xor(m, d, 64));
  }
#pragma unroll 1
  for (int e = lane; e < E; e += 64) {
    const double x = logit(a, r, e), y = exp(a.sigmoid ? -x : x - m);
    // a row of -infinity alone has no weight
    const double s = a.sigmoid ? 1.0 / (1.0 + y) : m == -INFINITY && x == m ? 0.0 : y;
    sum += s;
    score[e] = s;
    key[e] = order_bits(x);
  }
#pragma unroll 1
  for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d, 64);
  uint32_t open = 0;   // experts of the lane that may be chosen
#pragma unroll 1
  for (int e = lane; e < E; e += 64) {
    open |= 1u << (e >> 6);
    if (!a.sigmoid && sum != 0.0) score[e] /= sum;
    if (a.bias != nullptr) key[e] = order_bits(score[e] + (double)a.bias[e]);
  }
  in_order();
  if (a.top_groups < a.n_groups) {
    const int G = a.n_groups, size = E / G;
    uint64_t best = 0;
    if (lane < G) {
      uint64_t k0 = 0, k1 = 0;   // the two largest, NaN as 0
#pragma unroll 1
      for (int e = lane * size; e < (lane + 1) * size; ++e) {
        const uint64_t k = a.bias != nullptr ? key[e] : order_bits(score[e]);
        k1 = k > k0 ? k0 : k > k1 ? k : k1;
        k0 = k > k0 ? k : k0;
      }
      best = a.group_best > 1 && size > 1 ? order_bits(from_order_bits(k0) + from_order_bits(k1)) : k0;
    }
    int before = 0;
#pragma unroll 1
    for (int g = 0; g < G; ++g) {
      const uint64_t o = (uint64_t)__shfl((long long)best, g, 64);
      before += o > best || (o == best && g < lane);
    }
    const uint64_t kept = __ballot(lane < G && before < a.top_groups);
#pragma unroll 1
    for (int e = lane; e < E; e += 64)
      if (!((kept >> (e / size)) & 1)) open &= ~(1u << (e >> 6));
  }
  int idx = 0;   // lane j: rank j and its score
  double w = 0.0, total = 0.0;
#pragma unroll 1
  for (int j = 0; j < a.top_k; ++j) {
    uint64_t bk = 0;
    int be = INT32_MAX;   // none left
#pragma unroll 1
    for (uint32_t rest = open; rest != 0; rest &= rest - 1) {
      const int e = 64 * __builtin_ctz(rest) + lane;
      const uint64_t k = key[e];
      if (be == INT32_MAX || k > bk) {
        bk = k;
        be = e;
      }
    }
    const int mine = be;
#pragma unroll 1
    for (int d = 1; d < 64; d *= 2) {
      const uint64_t ok = (uint64_t)__shfl_xor((long long)bk, d, 64);
      const int oe = __shfl_xor(be, d, 64);
      if (oe != INT32_MAX && (be == INT32_MAX || ok > bk || (ok == bk && oe < be))) {
        bk = ok;
        be = oe;
      }
    }
    if (mine == be) open &= ~(1u << (be >> 6));
    const double s = score[be];
    total += s;
    if (lane == j) {
      idx = be;
      w = s;
    }
  }
  double upto = 0.0;
  int K = a.top_k;
#pragma unroll 1
  for (int j = 0; j + 1 < a.top_k; ++j) {
    upto += __shfl(w, j, 64);
    if (j + 1 >= a.min_k && total > 0.0 && upto >= (double)a.tau * total) {
      K = j + 1;
      break;
    }
  }
  if (lane < a.top_k) {
    a.expert_idx[r * a.top_k + lane] = idx;
    a.expert_w[r * a.top_k + lane] = (float)(w / (a.renormalize && total != 0.0 ? total : 1.0) * (double)a.scale);
  }
  if (lane == 0 && a.fanout != nullptr) a.fanout[r] = K;
  in_order();
  return lane < (a.fanout != nullptr ? K : a.top_k) ? idx : -1;
}

// any row, a wave each
template <int E_MAX>
__global__ __launch_bounds__(256) void route_wave_kernel(RouteArgs a) {
  __shared__ double score[4][E_MAX];
  __shared__ uint64_t key[4][E_MAX];
  if (a.expert_count != nullptr && blockIdx.x == 0)
    for (int i = threadIdx.x; i < a.n_experts; i += 256) a.expert_count[i] = 0;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int64_t r = (int64_t)blockIdx.x * 4 + wave; r < a.n_rows; r += (int64_t)gridDim.x * 4)
    route_exact(a, r, lane, score[wave], key[wave]);
}

// What ranks a row's experts in route_row_kernel
enum RouteBy {
  kByLogit,     // no bias: the order of the logits themselves
  kByPair,      // the same, groups by the scores of their two best
  kBySigmoid,   // c = sigmoid + bias
  kBySoftmax,   // c = softmax + bias
};

__device__ __forceinline__ float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }

// the conversion itself: in C++ it is undefined past the type's range
__device__ __forceinline__ uint32_t to_u32(float v) {
  uint32_t u;
  asm("v_cvt_u32_f32 %0, %1" : "=v"(u) : "v"(v));
  return u;
}

// Over the L lanes (16 or 64) of a row, in each of them
template <int L, class F>
__device__ __forceinline__ uint32_t over_row(uint32_t v, F&& f) {
  v = f(v, dpp<0xB1>(v));
  v = f(v, dpp<0x4E>(v));
  v = f(v, dpp<0x141>(v));
  v = f(v, dpp<0x140>(v));
  if constexpr (L == 64) {
    const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = f(p[0], p[1]);
    const auto q = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = f(q[0], q[1]);
  }
  return v;
}
template <int L>
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
  return over_row<L>(v, [](uint32_t x, uint32_t y) { return max_u32(x, y); });
}
template <int L>
__device__ __forceinline__ float row_max(float v) {
  return __uint_as_float(over_row<L>(__float_as_uint(v), [](uint32_t x, uint32_t y) {
    return __float_as_uint(fmaxf(__uint_as_float(x), __uint_as_float(y)));
  }));
}
template <int L>
__device__ __forceinline__ float row_sum(float v) {
  return __uint_as_float(over_row<L>(__float_as_uint(v), [](uint32_t x, uint32_t y) {
    return __float_as_uint(__uint_as_float(x) + __uint_as_float(y));
  }));
}

// groups of LG lanes of 16, all with the group's key, whose key is above this lane's
template <int LG, int R = 16 - LG>
__device__ __forceinline__ int above(uint32_t key) {
  if constexpr (R > 0) return (dpp<0x120 + R>(key) > key ? 1 : 0) + above<LG, R - LG>(key);   // row_ror:R
  return 0;
}

// Vectors of logits are loaded in a lane's places below its end, or in all, or in none
enum { kNarrow, kWide, kWhole };

// M consecutive logits of row r from expert e0 on, as f32; from `end` on: -infinity
template <int M, bool BF16>
__device__ __forceinline__ void load_logits(const RouteArgs& a, int wide, int64_t r, int e0, int end, float (&v)[M]) {
  constexpr int V = M % 4 == 0 ? 4 : 2;
#pragma unroll
  for (int i = 0; i < M; i += V) {
    const int e = e0 + i;
    if (wide == kWhole || (wide == kWide && e + V <= end)) {
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
      for (int k = 0; k < V; ++k) v[i + k] = e + k < end ? logit(a, r, e + k) : -INFINITY;
    }
  }
}

// L lanes a row: 16, four rows a wave, up to 256 experts, or the whole wave; a lane holds M
// consecutive experts, and with groups a group has 1, 2, 4, ... lanes (`lg`), the last of which may
// have places past its end.  Each lane keeps its DEPTH largest keys sorted (a max and medians per key); a round takes the row's maximum
// of the lanes' largest and the owner drops it.
//
// Errors of the codes, in steps of 2^-24 of the range 1 + 2 B of c (B the largest finite |bias|):
// the sigmoid's exponential is off by (1.5 |l| + 2) 2^-24 of itself, of which s (1 - s) <= 1/4 and
// s (1 - s) |l| < 0.23 reach s; 1 + e and its reciprocal add 3 s: below 4.  The bias in code units
// is off by 2, the fma by 1/2, the conversion by 1: a code by less than 8, and the order of two
// that are 17 apart is certain.  A softmax score takes the sum's error besides (its terms' 2.3 d + 2
// at a distance d from the largest logit, whose mean weighted by e^-d is at most 4.5 with 1024
// experts, and 11 additions), relative, below 50, and its factor's 2: with the bias's 2 and the last
// two below 56 of its range, the row's largest score + 2 B: 113 apart.  Codes of 22 bits, under
// indexes of 10, are off by a quarter of that and by the last two: less than 4 and 16.  A group's score is the
// sum of two codes: twice that.  Without a bias codes are the upper bits of the logit's order: exact
// for bf16, else equal codes are not certain.  What is no number, or -infinity, has a code at the
// bottom of its kind, as have the places past the end: a row that comes down to it is not certain
// either.  Ranks nearer than that are certain all the same if logits and biases are equal (bf16
// logits often are): then so are c, and the lower index has the larger key.
template <int L, int M, bool BF16, int BY>
__global__ __launch_bounds__(256, 4) void route_row_kernel(RouteArgs a, int lg, int wide, bool count) {
  constexpr int ROWS = 64 / L, E_MAX = L * M, IB = L == 16 ? 8 : 10;   // rows a wave, bits of an index
  constexpr int DEPTH = L == 64 ? (M < 5 ? M : 5) : (M < 6 ? M : 6);
  constexpr bool LOGIT = BY == kByLogit || BY == kByPair;
  constexpr uint32_t APART = BY == kBySigmoid ? (L == 16 ? 17 : 7) : BY == kBySoftmax ? (L == 16 ? 113 : 31) : BF16 ? 0 : 1;
  constexpr uint32_t kNegInfCode = 0x007FFFFFu >> IB;   // of total_order_bits(-infinity)
  constexpr uint32_t kIndex = (1u << IB) - 1;
  constexpr uint32_t kTwo = 2 * 0x3f800000u;   // bits of 1 twice: kTwo - bits of l carries on from 1 the order of 2 - l
  // a buffer of the 64-bit path for each wave, or (whole waves a row) one for each in turn
  constexpr int BUFS = L == 16 ? 4 : 1;
  __shared__ double score[BUFS][E_MAX];
  __shared__ uint64_t key_of[BUFS][E_MAX];
  __shared__ uint32_t hist[E_MAX];
  const int E = a.n_experts, TK = a.top_k;
  if (count) {   // the only workgroup: it counts as well
    for (int i = threadIdx.x; i < E_MAX; i += 256) hist[i] = 0;
    __syncthreads();
  } else if (a.expert_count != nullptr && blockIdx.x == 0) {
    for (int i = threadIdx.x; i < E; i += 256) a.expert_count[i] = 0;
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sl = lane % L, slot = lane / L;
  const bool groups = a.top_groups < a.n_groups;
  int e0 = M * sl, end = E;   // the lane's experts
  if (groups) {
    const int size = E / a.n_groups, g = sl / lg;
    e0 = g < a.n_groups ? g * size + M * (sl % lg) : 0;
    end = g < a.n_groups ? (g + 1) * size : 0;
  }
  float bias[LOGIT ? 1 : M], unit = 0.f, two_b = 0.f;   // c's code is (s + b + B) unit + 1: from 1 to 15 below the largest
  if constexpr (!LOGIT) {
    float b = 0.f;
#pragma unroll
    for (int i = 0; i < M; ++i) {
      bias[i] = e0 + i < end ? a.bias[e0 + i] : -INFINITY;
      if (fabsf(bias[i]) < INFINITY) b = fmaxf(b, fabsf(bias[i]));
    }
    b = row_max<L>(b);
    two_b = 2.f * b;
    unit = (float)((1 << (32 - IB)) - 16) / (1.f + two_b);   // of a softmax for each row
#pragma unroll
    for (int i = 0; i < M; ++i) bias[i] = BY == kBySoftmax ? bias[i] + b : (bias[i] + b) * unit + 1.f;
  }
  const int64_t stride = (int64_t)gridDim.x * (4 * ROWS), last = a.n_rows - 1;
  const int64_t first = ((int64_t)blockIdx.x * 4 + wave) * ROWS;
  int64_t r = first + slot;
  // every lane runs the same number of turns (rows past the end work on a copy of the last and
  // write nothing), so the exchanges see whole rows
  uint64_t again = 0;
  int turn = 0, taken = -1;   // taken: the expert that a lane's rank of the last turn executes
  float cur[M];
  if (r - slot <= last) load_logits<M, BF16>(a, wide, r < last ? r : last, e0, end, cur);
  for (; r - slot <= last; r += stride) {
    const int64_t rc = r < last ? r : last;
    float top = 0.f, total = 0.f;   // softmax: largest logit, sum of exponentials
    if (!a.sigmoid) {
      top = cur[0];
#pragma unroll
      for (int i = 1; i < M; ++i) top = fmaxf(top, cur[i]);
      top = row_max<L>(top);
      float part[4] = {};
#pragma unroll
      for (int i = 0; i < M; ++i) {
        const float e = exp_fast(cur[i] - top);   // past the end: 0
        part[i & 3] += e;
        if constexpr (BY == kBySoftmax) cur[i] = e;
      }
      total = row_sum<L>((part[0] + part[1]) + (part[2] + part[3]));
    }
    float inv = 0.f;
    if constexpr (BY == kBySoftmax) {   // the row's largest score: its codes span that and 2 B
      inv = __builtin_amdgcn_rcpf(total);
      unit = (float)((1 << (32 - IB)) - 16) * __builtin_amdgcn_rcpf(inv + two_b);
      inv *= unit;
    }
    typedef uint32_t Keys __attribute__((ext_vector_type(DEPTH)));   // an array's selects become indexed ones
    Keys m = 0;
    bool unsure = false;
#pragma unroll
    for (int i = 0; i < M; ++i) {
      const int e = e0 + i;
      uint32_t code;
      if constexpr (BY == kByPair) unsure |= cur[i] != cur[i];   // a group's sum with it is no number
      if constexpr (LOGIT) {
        code = total_order_bits(fmaxf(cur[i], -INFINITY) + 0.0f) >> IB;   // NaN as -infinity, -0 as 0
      } else {
        // v_cvt takes NaN and what is below 0 to 0, +infinity to 2^32 - 1: the largest code
        if constexpr (BY == kBySigmoid) code = to_u32(fmaf(__builtin_amdgcn_rcpf(1.f + exp_fast(-cur[i])), unit, bias[i]));
        else code = to_u32(fmaf(cur[i], inv, fmaf(bias[i], unit, 1.f)));
      }
      const uint32_t x = (code << IB) | (kIndex - (uint32_t)e);
#pragma unroll
      for (int d = DEPTH - 1; d > 0; --d) m[d] = med_u32(m[d - 1], m[d], x);
      m[0] = max_u32(m[0], x);
    }
    // the next row, over the registers just consumed
    if (r - slot + stride <= last) load_logits<M, BF16>(a, wide, r + stride < last ? r + stride : last, e0, end, cur);
    if (groups) {
      uint32_t g0 = m[0] >> IB, g1 = m[1] >> IB;
      auto join = [&](uint32_t o0, uint32_t o1) {
        const uint32_t lo = g0 < o0 ? g0 : o0;
        g0 = max_u32(g0, o0);
        g1 = max_u32(lo, max_u32(g1, o1));
      };
      if (lg > 1) join(dpp<0xB1>(g0), dpp<0xB1>(g1));
      if (lg > 2) join(dpp<0x4E>(g0), dpp<0x4E>(g1));
      if (lg > 4) join(dpp<0x141>(g0), dpp<0x141>(g1));
      if (L == 64) {
        if (lg > 8) join(dpp<0x140>(g0), dpp<0x140>(g1));
        if (lg > 16) join((uint32_t)__shfl_xor((int)g0, 16, 64), (uint32_t)__shfl_xor((int)g1, 16, 64));
      }
      uint32_t score;
      uint32_t lo = 0, hi = 0;   // kByPair: the order of a sum less and plus its error
      if constexpr (BY == kByPair) {
        // The scores (a softmax's without its sum) of the middles of the two codes: the logit is off by
        // |x| 2^(IB - 24), the exponential by (2.3 * 70 + 2) 2^-24 of itself and what follows by 6.  Taken
        // twice and more, in relative terms.  Sigmoids that add up to more than 1 are ordered by what
        // lacks to 2, sigmoid(-x) each, which has its bits where they have none.
        float sum = 0.f, err = 0.f, lack = 0.f, lack_err = 0.f;
        auto add = [&](uint32_t code) {
          const float x = code <= kNegInfCode ? -1e30f : fminf(from_total_order_bits((code << IB) | (1u << (IB - 1))), 1e30f);
          const float off = fabsf(x) * (1.f / (1 << (22 - IB))) + 0x1p-15f;
          const float s = a.sigmoid ? __builtin_amdgcn_rcpf(1.f + exp_fast(-x)) : exp_fast(x - top);
          sum += s;
          err += s * off;
          if (a.sigmoid) {
            const float l = __builtin_amdgcn_rcpf(1.f + exp_fast(x));
            lack += l;
            lack_err += l * off;
          }
        };
        add(g0);
        add(g1);
        const bool by_lack = a.sigmoid && sum > 1.f;
        auto order = [&](float v, float l) { return by_lack ? kTwo - __float_as_uint(fmaxf(l, 0.f)) : __float_as_uint(fmaxf(v, 0.f)); };
        const bool group = sl / lg < a.n_groups;
        score = group ? order(sum, lack) >> (L == 16 ? 3 : 5) : 0u;
        lo = order(sum - err, lack + lack_err);
        hi = group ? order(sum + err, lack - lack_err) : 0u;
      } else {
        // the second best at the bottom (-infinity or NaN): the sum is as well
        score = !LOGIT && a.group_best > 1 && a.n_groups < E ? (g1 == 0 ? 0 : g0 + g1) : g0;
      }
      // places past the last group come behind every group
      const uint32_t key = L == 16 ? (score << 4) | (uint32_t)(15 - sl / lg) : (score << 6) | (uint32_t)(63 - sl / lg);
      int over = 0;
      if constexpr (L == 16) {
        over = lg == 1 ? above<1>(key) : lg == 2 ? above<2>(key) : lg == 4 ? above<4>(key) : above<8>(key);
      } else {
        for (int g = 0; g < a.n_groups; ++g) over += (uint32_t)__builtin_amdgcn_readlane((int)key, g * lg) > key ? 1 : 0;
      }
      const bool kept = over < a.top_groups;
      if constexpr (BY == kByPair) {
        // a sum of next to nothing, or 2^-33 from 2, may have 64-bit equals
        const uint32_t least = ~row_max<L>(kept ? ~lo : 0u), most = row_max<L>(kept ? 0u : hi);
        unsure |= !(least > most && least > __builtin_bit_cast(uint32_t, 1e-30f)) || (a.sigmoid && most > kTwo - __builtin_bit_cast(uint32_t, 0x1p-33f));
      } else {
        // the least kept score and the largest other
        const uint32_t least = ~row_max<L>(kept ? ~score : 0u), most = row_max<L>(kept ? 0u : score);
        unsure = least < most + 2 * APART;
        if constexpr (LOGIT) {
          // Groups go by scores, and those of different logits may be equal in 64 bits: a sigmoid next to
          // 1 or to 1/2, an exponential of next to `top` or out of range.  Codes apart are logits 2^-16
          // of themselves apart, which elsewhere is far above a step of the score.
          const float x = from_total_order_bits(least << IB);
          unsure |= least <= kNegInfCode || !(fabsf(x) >= 0x1p-20f * fmaxf(1.f, fabsf(top)) && top - x < 600.f && !(a.sigmoid && x > 24.f));
        }
      }
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) m[d] = kept ? m[d] : 0u;
    }
    const bool full = M > DEPTH && m[DEPTH - 1] != 0;
    uint32_t my_key = 0, before = 0;   // key of the lane's rank, and of the last one
    int drops = 0;
    auto drop = [&](uint32_t top_key, bool there) {
      const bool own = there && m[0] == top_key;
      drops += own;
#pragma unroll
      for (int d = 0; d + 1 < DEPTH; ++d) m[d] = own ? m[d + 1] : m[d];
      m[DEPTH - 1] = own ? 0u : m[DEPTH - 1];
    };
#pragma unroll
    for (int j = 0; j < kMoeMaxTopK; ++j) {
      if (j < TK) {
        before = row_max<L>(m[0]);
        if (sl == j) my_key = before;
        drop(before, true);
      }
    }
    unsure |= LOGIT ? before >> IB <= kNegInfCode : before >> IB <= APART + 1;
    // logit and bias of a key's expert; a place past E is not certain, see above
    auto expert = [&](uint32_t key) { return (int32_t)(kIndex - (key & kIndex)); };
    auto values = [&](uint32_t key, float& x, float& b) {
      const int32_t e = expert(key) < E ? expert(key) : 0;
      x = logit(a, rc, e);
      b = LOGIT ? 0.f : a.bias[e];
    };
    // the ranks' scores: lane j of the row holds rank j
    const bool rank = sl < TK;
    const int32_t my_id = expert(my_key);
    float x = 0.f, b = 0.f;
    if (rank) values(my_key, x, b);
    uint32_t next = row_max<L>(m[0]);   // the runner-up; nothing left: code 0
    if constexpr (APART > 0) {
      const uint32_t prev = dpp<0x111>(my_key);   // row_shr:1
      const bool same = x == __uint_as_float(dpp<0x111>(__float_as_uint(x))) && b == __uint_as_float(dpp<0x111>(__float_as_uint(b)));
      unsure |= rank && sl > 0 && (prev >> IB) - (my_key >> IB) < APART && !same;
      // runners-up equal to the last rank come behind it: the first that is not decides
      bool near = (before >> IB) - (next >> IB) < APART;
      for (int more = 0; more < DEPTH && __ballot(near) != 0; ++more) {
        float xn, bn;
        values(next, xn, bn);
        const int from = lane - sl + TK - 1;
        const bool equal = near && xn == __shfl(x, from, 64) && bn == __shfl(b, from, 64);
        unsure |= near && !equal;
        drop(next, equal);
        next = row_max<L>(m[0]);
        near = equal && (before >> IB) - (next >> IB) < APART;
      }
      unsure |= near;
    }
    unsure |= full && drops >= DEPTH;   // the lane's next key is not known
    const float d = a.sigmoid ? -fabsf(x) : x - top;
    float e = expf(d);
    if (!a.sigmoid) {   // what the rounding of the difference took, whichever of the two is larger
      const float x1 = d + top, top1 = x1 - d;
      e += e * ((x - x1) - (top - top1));
    }
    float s = a.sigmoid ? (x < 0.f ? e : 1.f) * __builtin_amdgcn_rcpf(1.f + e) : e * __builtin_amdgcn_rcpf(total);
    s = rank ? s : 0.f;
    float upto = s;   // sums of the ranks up to the lane's
    upto += __uint_as_float(dpp<0x111>(__float_as_uint(upto)));   // row_shr:1, 2, 4: ranks are below 8
    upto += __uint_as_float(dpp<0x112>(__float_as_uint(upto)));
    upto += __uint_as_float(dpp<0x114>(__float_as_uint(upto)));
    const float sum = row_bcast<7>(upto), want = a.tau * sum;   // of whole waves in the first 16 lanes
    const bool asked = sl + 1 >= a.min_k && sl + 1 < TK;
    // the sum decides little where it is tiny or not a number
    unsure |= (sl < 16 && !(sum > 1e-30f)) || (asked && fabsf(upto - want) <= 0x1p-18f * sum);
    const uint32_t enough = (uint32_t)(__ballot(asked && upto >= want) >> (16 * (L == 16 ? slot : 0))) & 0xFFFFu;
    const int K = enough != 0 ? __builtin_ctz(enough) + 1 : TK;
    const uint64_t odd = __ballot(unsure && r <= last), mine = L == 16 ? 0xFFFFull << (16 * slot) : ~0ull;
    if (r <= last && (odd & mine) == 0) {
      taken = sl < (a.fanout != nullptr ? K : TK) ? my_id : -1;
      if (rank) {
        a.expert_idx[r * TK + sl] = my_id;
        a.expert_w[r * TK + sl] = (a.renormalize ? s * __builtin_amdgcn_rcpf(sum) : s) * a.scale;
      }
      if (sl == 0 && a.fanout != nullptr) a.fanout[r] = K;
    }
    // a bit a row and turn
#pragma unroll
    for (int k = 0; k < ROWS; ++k)
      if ((L == 16 ? odd >> (16 * k) & 0xFFFF : odd) != 0) again |= 1ull << (ROWS * turn + k);
    ++turn;
  }
  // rows whose order is not certain, each by the whole wave
  for (int w = 0; w < (BUFS == 1 ? 4 : 1); ++w) {
    if (BUFS == 4 || wave == w)
      for (; again != 0; again &= again - 1) {
        const int at = __builtin_ctzll(again);
        const int expert = route_exact(a, first + (at / ROWS) * stride + (at % ROWS), lane, score[wave % BUFS], key_of[wave % BUFS]);
        if (count && expert >= 0) atomicAdd(&hist[expert], 1u);
      }
    if (BUFS == 1) __syncthreads();
  }
  if (count) {   // one turn
    if (taken >= 0) atomicAdd(&hist[taken], 1u);
    __syncthreads();
    for (int i = threadIdx.x; i < E; i += 256) a.expert_count[i] = (int32_t)hist[i];
  }
}

// How a row lies on the lanes of route_row_kernel: L of them, M experts each, lg a group; L = 0
// where it does not fit
struct RowShape {
  int L, M, lg;
};

RowShape row_shape(const RouteArgs& a) {
  const int E = a.n_experts, G = a.top_groups < a.n_groups ? a.n_groups : 1, size = E / G;
  for (const int L : {16, 64})
    for (const int M : {2, 4, 8, 10, 12, 16}) {
      if (L == 64 && (M < 8 || M == 10)) continue;   // not built
      if (G == 1) {
        if (M > 2 && E <= L * M) return {L, M, L};
        continue;
      }
      int lg = 1;
      while (lg * M < size) lg *= 2;
      if (G * lg <= L) return {L, M, lg};
    }
  return {0, 0, 0};
}

template <int L, int M, bool BF16>
hipError_t launch_rows(const RouteArgs& a, int lg, bool count, hipStream_t s) {
  constexpr int ROWS = 4 * (64 / L);   // of a workgroup; a wave takes 64 rows at most, a bit of a word each
  const int64_t blocks = (a.n_rows + ROWS - 1) / ROWS;
  const dim3 grid((unsigned)std::max(std::min<int64_t>(blocks, 2048), (blocks + L - 1) / L)), blk(256);
  // vectors of 4 (2 where a lane's share is not whole fours) logits
  const int64_t vec = M % 4 == 0 ? 4 : 2, bytes = vec * (BF16 ? 2 : 4);
  const bool groups = a.top_groups < a.n_groups;
  const bool fit = reinterpret_cast<uintptr_t>(a.logits) % bytes == 0 && a.stride * (BF16 ? 2 : 4) % bytes == 0 &&
                   (!groups || a.n_experts / a.n_groups % vec == 0);
  const int wide = !fit ? kNarrow : a.n_experts == L * M ? kWhole : kWide;   // E places: no lane has one past its end
  if (a.bias == nullptr && groups && a.group_best > 1) route_row_kernel<L, M, BF16, kByPair><<<grid, blk, 0, s>>>(a, lg, wide, count);
  else if (a.bias == nullptr) route_row_kernel<L, M, BF16, kByLogit><<<grid, blk, 0, s>>>(a, lg, wide, count);
  else if (a.sigmoid) route_row_kernel<L, M, BF16, kBySigmoid><<<grid, blk, 0, s>>>(a, lg, wide, count);
  else route_row_kernel<L, M, BF16, kBySoftmax><<<grid, blk, 0, s>>>(a, lg, wide, count);
  return hipGetLastError();
}

template <bool BF16>
hipError_t launch_shape(const RouteArgs& a, const RowShape& S, bool count, hipStream_t s) {
  if (S.L == 64) {
    if (S.M == 8) return launch_rows<64, 8, BF16>(a, S.lg, count, s);
    if (S.M == 12) return launch_rows<64, 12, BF16>(a, S.lg, count, s);
    return launch_rows<64, 16, BF16>(a, S.lg, count, s);
  }
  switch (S.M) {
    case 2: return launch_rows<16, 2, BF16>(a, S.lg, count, s);
    case 4: return launch_rows<16, 4, BF16>(a, S.lg, count, s);
    case 8: return launch_rows<16, 8, BF16>(a, S.lg, count, s);
    case 10: return launch_rows<16, 10, BF16>(a, S.lg, count, s);
    case 12: return launch_rows<16, 12, BF16>(a, S.lg, count, s);
    default: return launch_rows<16, 16, BF16>(a, S.lg, count, s);
  }
}

}  // namespace

hipError_t launch_moe_route(const RouteArgs& a, hipStream_t s) {
  if (a.n_rows == 0 && a.expert_count == nullptr) return hipSuccess;
  const int E = a.n_experts;
  const RowShape S = a.n_rows > 0 ? row_shape(a) : RowShape{0, 0, 0};
  hipError_t e;
  if (S.L != 0) {
    // as many rows as one workgroup takes at once: it counts them too
    const bool count = a.expert_count != nullptr && a.n_rows <= 4 * (64 / S.L);
    e = a.logits_bf16 ? launch_shape<true>(a, S, count, s) : launch_shape<false>(a, S, count, s);
    if (count) return e;
  } else {
    const dim3 grid((unsigned)std::max<int64_t>(1, std::min<int64_t>((a.n_rows + 3) / 4, 4096))), blk(256);   // no row: the counts are cleared
    if (E <= 256) route_wave_kernel<256><<<grid, blk, 0, s>>>(a);
    else if (E <= 512) route_wave_kernel<512><<<grid, blk, 0, s>>>(a);
    else route_wave_kernel<1024><<<grid, blk, 0, s>>>(a);
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

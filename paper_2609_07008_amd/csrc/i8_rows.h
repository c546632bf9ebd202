// Quantizing rows of bf16 into 8 bits, for the kernels that do.
#pragma once

#include <algorithm>

#include "i8.h"

namespace mla {

__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }

// Codes of a row whose largest magnitude is `top` (bf16 bits without the sign, finite).  The
// quotient n / A of n = 127 x 2^-e and A = top 2^-e is taken as one Newton step on v_rcp: its
// error is far below 2^-18, the least distance of such a quotient (8 by 8 bits) from a tie, and
// a quotient that is a tie has at most 8 bits and comes out exact, so rint rounds as the exact
// quotient does.  The scaling keeps n in range: e is top's exponent, and no less than -100.
struct I8Coder {
  float mul, a, inv;
  __device__ __forceinline__ explicit I8Coder(uint32_t top) {
    const int e = std::max((int)(top >> 7), 27) - 127;
    const float two = __uint_as_float((uint32_t)(127 - e) << 23);   // 2^-e; 2^-128 is subnormal and top < 2^128, e <= 127
    const float t = __uint_as_float(top << 16);
    mul = e == 127 ? 127.0f * 0x1p-127f : 127.0f * two;
    a = e == 127 ? t * 0x1p-127f : t * two;
    inv = a > 0.0f ? __builtin_amdgcn_rcpf(a) : 0.0f;
  }
  __device__ __forceinline__ int code(float x) const {
    const float n = x * mul, t0 = n * inv;
    return (int)__builtin_rintf(__builtin_fmaf(__builtin_fmaf(-t0, a, n), inv, t0));
  }
};

__device__ __forceinline__ u32x2 codes8(const I8Coder& c, u32x4 v) {
  u32x2 q;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int c0 = c.code(bf16_lo(v[2 * i])), c1 = c.code(bf16_hi(v[2 * i]));
    const int c2 = c.code(bf16_lo(v[2 * i + 1])), c3 = c.code(bf16_hi(v[2 * i + 1]));
    q[i] = (uint32_t)(c0 & 255) | (uint32_t)(c1 & 255) << 8 | (uint32_t)(c2 & 255) << 16 | (uint32_t)c3 << 24;
  }
  return q;
}

__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v = umax(v, (uint32_t)__shfl_xor((int)v, d, 64));
  return v;
}

// Rows r, r + step, ... below n of a, each by T threads (a wave, or 256 threads of a workgroup),
// read once and kept in registers: 3 bytes moved a value.  With T = 256 every thread of the
// workgroup calls this with r of its 256, and `part` is LDS of 8 words for each 256 threads: the
// row's wave maxima of this turn and the last, one barrier a row.
template <int T, int NV>
__device__ __forceinline__ void quantize_rows(const I8Args& a, int64_t n, int64_t r, int64_t step, int* part) {
  const int t = threadIdx.x % T;
  int* mine = part + threadIdx.x / 256 * 8;
  int turn = 0;
  // the rows of a workgroup's first threads decide how many turns it takes
  for (int64_t r0 = r - threadIdx.x / T; r0 < n; r0 += step, r += step, turn ^= 4) {
    const bool there = r < n;
    const uint16_t* x = (const uint16_t*)a.x + (there ? r : r0) * a.x_stride;
    u32x4 v[NV];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * T + t) * 8;
      v[i] = c < a.n_cols ? *(const u32x4*)(x + c) : u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) m = umax(m, umax(v[i][k] & 0x7fffu, (v[i][k] >> 16) & 0x7fffu));
    m = wave_max(m);
    if (T == 256) {
      if ((threadIdx.x & 63) == 0) mine[turn + (threadIdx.x >> 6 & 3)] = (int)m;
      __syncthreads();
      m = (uint32_t)std::max(std::max(mine[turn], mine[turn + 1]), std::max(mine[turn + 2], mine[turn + 3]));
    }
    if (!there) continue;
    const bool finite = m < 0x7f80u;
    const I8Coder coder(finite ? m : 0);
    int8_t* q = (int8_t*)a.codes + r * a.n_cols;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * T + t) * 8;
      if (c < a.n_cols) *(u32x2*)(q + c) = finite ? codes8(coder, v[i]) : u32x2{0, 0};
    }
    if (t == 0) a.scales[a.at != nullptr ? a.at[r].y : r] = finite ? __uint_as_float(m << 16) / 127.0f : __uint_as_float(0x7fc00000u);
  }
}

}  // namespace mla

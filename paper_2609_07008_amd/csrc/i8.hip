// 8-bit integers with a scale for each row, and y = W_b z in them.
//
// A row x of bf16 is held as codes q = round(127 x / max|x|) and the scale max|x| / 127.  The
// sum of a product of codes is a whole number below 127^2 * 16384 < 2^31 and is exact in i32,
// so a product does not depend on its order, tile or split: every form gives the same bits.
#include "i8.h"

#include <algorithm>

namespace mla {
namespace {

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

// A row by T threads (a wave, or a workgroup of 256), read once and kept in registers: 3 bytes
// moved a value.
template <int T, int NV>
__global__ __launch_bounds__(256) void i8_quantize_kernel(I8Args a) {
  __shared__ uint32_t part[2][4];   // of this turn and the last: one barrier a row
  const int t = threadIdx.x % T;
  const int64_t n = a.n_dev != nullptr ? std::min<int64_t>(*a.n_dev, a.n_rows) : a.n_rows;
  int turn = 0;
  for (int64_t r0 = (int64_t)blockIdx.x * (256 / T); r0 < n; r0 += (int64_t)gridDim.x * (256 / T), turn ^= 1) {
    const int64_t r = r0 + threadIdx.x / T;
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
      if ((threadIdx.x & 63) == 0) part[turn][threadIdx.x >> 6] = m;
      __syncthreads();
      m = umax(umax(part[turn][0], part[turn][1]), umax(part[turn][2], part[turn][3]));
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
    if (t == 0) a.scales[r] = finite ? __uint_as_float(m << 16) / 127.0f : __uint_as_float(0x7fc00000u);
  }
}

__global__ __launch_bounds__(256) void i8_dequantize_kernel(I8Args a, int segs) {
  const int lane = threadIdx.x & 63;
  const int64_t units = a.n_rows * segs;
  for (int64_t u = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); u < units; u += (int64_t)gridDim.x * 4) {
    const int64_t row = u / segs;
    const int c = (int)(u - row * segs) * 512 + lane * 8;
    if (c >= a.n_cols) continue;   // whole eights: n_cols is a multiple of 16
    const float s = a.scales[row];
    const u32x2 q = *(const u32x2*)((const int8_t*)a.codes + row * a.n_cols + c);
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = q[i / 2] >> (16 * (i & 1));
      v[i] = pack_bf16x2((float)(int8_t)(w & 255) * s, (float)(int8_t)((w >> 8) & 255) * s);
    }
    *(u32x4*)((uint16_t*)const_cast<void*>(a.x) + row * a.x_stride + c) = v;
  }
}

// 64 rows x 64 channels a workgroup, 16 rows a wave, fragments from memory
template <bool OUT_BF16>
__global__ __launch_bounds__(256) void wb_i8_kernel(WbI8Args a, int n_tiles) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lg = lane >> 4, lc = lane & 15;
  const int64_t m = (int64_t)(blockIdx.x / n_tiles) * 64 + wave * 16 + lc;
  const int n0 = (int)(blockIdx.x % n_tiles) * 64;
  const int8_t* z = a.z + std::min<int64_t>(m, a.n_rows - 1) * a.d_in + lg * 16;
  const int8_t* w[4];
  i32x4 acc[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    w[j] = a.w + (int64_t)std::min(n0 + 16 * j + lc, a.d_out - 1) * a.d_in + lg * 16;
    acc[j] = i32x4{0, 0, 0, 0};
  }
  for (int k = 0; k < a.d_in; k += 64) {
    const i32x4 fz = *(const i32x4*)(z + k);
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(*(const i32x4*)(w[j] + k), fz, acc[j], 0, 0, 0);
  }
  if (m >= a.n_rows) return;
  const float zs = a.z_scale[m];
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int n = n0 + 16 * j + lg * 4 + e;
      if (n >= a.d_out) continue;
      const float v = (float)acc[j][e] * a.w_scale[n] * zs;
      if (OUT_BF16)
        ((__bf16*)a.y)[m * a.d_out + n] = (__bf16)v;
      else
        ((float*)a.y)[m * a.d_out + n] = v;
    }
}

}  // namespace

hipError_t launch_i8_quantize(const I8Args& a, hipStream_t s) {
  const int64_t most = 1 << 22;   // workgroups: the rows beyond are a next turn
  const dim3 by4((unsigned)std::min((a.n_rows + 3) / 4, most)), by1((unsigned)std::min(a.n_rows, most)), blk(256);
  if (a.n_cols <= 512) i8_quantize_kernel<64, 1><<<by4, blk, 0, s>>>(a);
  else if (a.n_cols <= 2048) i8_quantize_kernel<64, 4><<<by4, blk, 0, s>>>(a);
  else if (a.n_cols <= 4096) i8_quantize_kernel<256, 2><<<by1, blk, 0, s>>>(a);
  else if (a.n_cols <= 8192) i8_quantize_kernel<256, 4><<<by1, blk, 0, s>>>(a);
  else i8_quantize_kernel<256, 8><<<by1, blk, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_i8_dequantize(const I8Args& a, hipStream_t s) {
  const int segs = (a.n_cols + 511) / 512;
  const int64_t blocks = std::min<int64_t>((a.n_rows * segs + 3) / 4, (int64_t)1 << 24);
  i8_dequantize_kernel<<<dim3((unsigned)blocks), dim3(256), 0, s>>>(a, segs);
  return hipGetLastError();
}

hipError_t launch_wb_i8(const WbI8Args& a, hipStream_t s) {
  const int n_tiles = (a.d_out + 63) / 64;
  const dim3 grid((unsigned)((a.n_rows + 63) / 64 * n_tiles));
  if (a.y_bf16) wb_i8_kernel<true><<<grid, dim3(256), 0, s>>>(a, n_tiles);
  else wb_i8_kernel<false><<<grid, dim3(256), 0, s>>>(a, n_tiles);
  return hipGetLastError();
}

}  // namespace mla

// mx4 quantization and dequantization of a matrix, and y = W_b z with W_b in mx4.
#include "mx4.h"

#include <algorithm>

namespace mla {
namespace {

// Both directions move 2 + 17/32 bytes a value and are bound by that: a wave takes 512
// consecutive values of a row, eight a lane (16 bytes of bf16, four of codes), so every
// access of a wave is one contiguous run.
__global__ __launch_bounds__(256) void mx4_quantize_kernel(Mx4Args a, int segs) {
  const int lane = threadIdx.x & 63;
  const int64_t units = a.n_rows * segs;
  for (int64_t u = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); u < units; u += (int64_t)gridDim.x * 4) {
    const int64_t row = u / segs;
    const int c = (int)(u - row * segs) * 512 + lane * 8;
    if (c >= a.n_cols) continue;   // whole quads: n_cols is a multiple of 32
    const u32x4 x = *(const u32x4*)((const uint16_t*)a.x + row * a.x_stride + c);
    uint32_t e;
    const uint32_t codes = mx4_codes(x, e);
    *(uint32_t*)((unsigned char*)a.codes + (row * a.n_cols + c) / 2) = codes;
    if ((lane & 3) == 0) ((unsigned char*)a.scales)[(row * a.n_cols + c) / 32] = (unsigned char)e;
  }
}

__global__ __launch_bounds__(256) void mx4_dequantize_kernel(Mx4Args a, int segs) {
  const int lane = threadIdx.x & 63;
  const int64_t units = a.n_rows * segs;
  for (int64_t u = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); u < units; u += (int64_t)gridDim.x * 4) {
    const int64_t row = u / segs;
    const int c = (int)(u - row * segs) * 512 + lane * 8;
    if (c >= a.n_cols) continue;
    const uint32_t codes = *(const uint32_t*)((const unsigned char*)a.codes + (row * a.n_cols + c) / 2);
    const uint32_t e = ((const unsigned char*)a.scales)[(row * a.n_cols + c) / 32];
    *(bf16x8*)((uint16_t*)const_cast<void*>(a.x) + row * a.x_stride + c) = mx4_values(codes, mx4_scale(e));
  }
}

// y = W z.  A workgroup takes 16 NB output channels and 16 MB rows of z; its eight waves
// split d_in into runs of 128-wide slabs and each adds its own in order, so an element's
// sum has the same order whatever NB, MB and the number of rows.  A lane holds 32
// consecutive values of a channel (16 bytes, one group): they feed four 16x16x32 MFMAs,
// the j-th taking values 8 j .. +7 of each of the four groups of a slab, from W and z alike.
template <bool OUT_BF16, int NB, int MB>
__global__ __launch_bounds__(512, 2) void wb_mx4_kernel(WbMx4Args a) {
  constexpr int WAVES = 8;
  __shared__ __attribute__((aligned(16))) float red[WAVES][NB * MB][64][4];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lg = lane >> 4, lc = lane & 15;
  const int n0 = blockIdx.x * (16 * NB);
  const int64_t m0 = (int64_t)blockIdx.y * (16 * MB);
  const int slabs = (a.d_in + 127) / 128;
  const int s_lo = slabs * wave / WAVES, s_hi = slabs * (wave + 1) / WAVES;
  // rows and channels past the end repeat the last one; their results are not stored
  const uint8_t* wc[NB];
  const uint8_t* ws[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    const int64_t ch = std::min(n0 + n * 16 + lc, a.d_out - 1);
    wc[n] = a.codes + ch * (a.d_in / 2);
    ws[n] = a.scales + ch * (a.d_in / 32);
  }
  const uint16_t* zr[MB];
#pragma unroll
  for (int m = 0; m < MB; ++m) zr[m] = a.z + std::min<int64_t>(m0 + m * 16 + lc, a.n_rows - 1) * a.d_in;
  f32x4 acc[NB][MB];
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int m = 0; m < MB; ++m) acc[n][m] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int s = s_lo; s < s_hi; ++s) {
    const int k = s * 128 + lg * 32;
    const bool in = k < a.d_in;   // a last slab of 64: its upper groups are zero on both sides
    const int kk = in ? k : 0;
    u32x4 c[NB];
    float sc[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      c[n] = *(const u32x4*)(wc[n] + kk / 2);
      sc[n] = mx4_scale(ws[n][kk / 32]);
    }
    bf16x8 z[MB][4];
#pragma unroll
    for (int m = 0; m < MB; ++m)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        z[m][j] = *(const bf16x8*)(zr[m] + kk + j * 8);
        if (!in) z[m][j] = bf16x8{};
      }
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        bf16x8 w = mx4_values(c[n][j], sc[n]);
        if (!in) w = bf16x8{};
#pragma unroll
        for (int m = 0; m < MB; ++m) acc[n][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, z[m][j], acc[n][m], 0, 0, 0);
      }
  }
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int m = 0; m < MB; ++m) *(f32x4*)red[wave][n * MB + m][lane] = acc[n][m];
  __syncthreads();
  for (int i = tid; i < NB * MB * 64; i += 512) {
    const int blk = i >> 6, ln = i & 63;
    f32x4 v = *(const f32x4*)red[0][blk][ln];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v += *(const f32x4*)red[w][blk][ln];
    const int64_t row = m0 + (blk % MB) * 16 + (ln & 15);
    const int ch = n0 + (blk / MB) * 16 + (ln >> 4) * 4;
    if (row >= a.n_rows) continue;
    const int64_t at = row * a.d_out + ch;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (ch + e >= a.d_out) continue;
      if (OUT_BF16)
        ((__bf16*)a.y)[at + e] = (__bf16)v[e];
      else
        ((float*)a.y)[at + e] = v[e];
    }
  }
}

template <int NB, int MB>
hipError_t launch_wb_tile(const WbMx4Args& a, hipStream_t s) {
  const dim3 grid((unsigned)((a.d_out + 16 * NB - 1) / (16 * NB)), (unsigned)((a.n_rows + 16 * MB - 1) / (16 * MB)));
  if (a.y_bf16)
    wb_mx4_kernel<true, NB, MB><<<grid, dim3(512), 0, s>>>(a);
  else
    wb_mx4_kernel<false, NB, MB><<<grid, dim3(512), 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

namespace {
unsigned mx4_grid(int64_t units) { return (unsigned)std::min<int64_t>((units + 3) / 4, 1 << 20); }
}  // namespace

hipError_t launch_mx4_quantize(const Mx4Args& a, hipStream_t s) {
  const int segs = (a.n_cols + 511) / 512;
  mx4_quantize_kernel<<<dim3(mx4_grid(a.n_rows * segs)), dim3(256), 0, s>>>(a, segs);
  return hipGetLastError();
}

hipError_t launch_mx4_dequantize(const Mx4Args& a, hipStream_t s) {
  const int segs = (a.n_cols + 511) / 512;
  mx4_dequantize_kernel<<<dim3(mx4_grid(a.n_rows * segs)), dim3(256), 0, s>>>(a, segs);
  return hipGetLastError();
}

hipError_t launch_wb_mx4(const WbMx4Args& a, hipStream_t s) {
  if (a.n_rows <= 16) return launch_wb_tile<1, 1>(a, s);
  if (a.n_rows <= 32) return launch_wb_tile<1, 2>(a, s);
  return launch_wb_tile<1, 4>(a, s);
}

}  // namespace mla

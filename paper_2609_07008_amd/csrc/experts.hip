// The experts of a mixture-of-experts layer in 8-bit integers:
//   y_n = sum_{j < K_n} w_nj W_down[e] h_nj,  h_nj = silu(W_gate[e] x_n) * (W_up[e] x_n),  e = expert_idx[n, j]
// Pairs (n, j) are put in expert order; x is quantized a row; the products run over blocks of
// rows of one expert; h is rounded to bf16, a layer's activation, and quantized a row; the
// pairs of a token are joined in rank order.  Within an expert the order of the pairs hangs on
// atomics, but rows do not meet and the products are exact in i32: the result does not.
#include "i8.h"

#include <algorithm>

namespace mla {
namespace {

// expert of pair p, or -1 where it is not here or past the token's fanout
__device__ __forceinline__ int pair_expert(const ExpertsArgs& a, int32_t p) {
  const int n = p / a.top_k, j = p - n * a.top_k;
  const uint32_t e = (uint32_t)a.idx[p] - (uint32_t)a.first;
  if (e >= (uint32_t)a.n_experts) return -1;
  return a.fanout != nullptr && j >= a.fanout[n] ? -1 : (int)e;
}

__global__ __launch_bounds__(256) void experts_zero_kernel(ExpertsArgs a) {
  for (int i = threadIdx.x; i < a.n_experts; i += 256) a.counts[i] = 0;
}

__global__ __launch_bounds__(256) void experts_count_kernel(ExpertsArgs a) {
  __shared__ int hist[kExpertsMax];
  for (int i = threadIdx.x; i < a.n_experts; i += 256) hist[i] = 0;
  __syncthreads();
  const int64_t n_pairs = a.n_rows * a.top_k;
  for (int64_t p = (int64_t)blockIdx.x * 256 + threadIdx.x; p < n_pairs; p += (int64_t)gridDim.x * 256) {
    const int e = pair_expert(a, (int32_t)p);
    if (e >= 0) atomicAdd(&hist[e], 1);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < a.n_experts; i += 256)
    if (hist[i]) atomicAdd(&a.counts[i], hist[i]);
}

// counts -> each expert's first place (its cursor), the tiles, the totals
__global__ __launch_bounds__(1024) void experts_scan_kernel(ExpertsArgs a) {
  __shared__ int rows[kExpertsMax], blocks[kExpertsMax];
  const int e = threadIdx.x;
  const int c = e < a.n_experts ? a.counts[e] : 0, b = (c + a.tile_rows - 1) / a.tile_rows;
  rows[e] = c;
  blocks[e] = b;
  __syncthreads();
  for (int d = 1; d < kExpertsMax; d *= 2) {
    const int x = e >= d ? rows[e - d] : 0, y = e >= d ? blocks[e - d] : 0;
    __syncthreads();
    rows[e] += x;
    blocks[e] += y;
    __syncthreads();
  }
  if (e < a.n_experts) {
    const int row = rows[e] - c, t0 = blocks[e] - b;
    a.counts[a.n_experts + e] = row;
    for (int i = 0; i < b; ++i) a.tiles[t0 + i] = ExpertTile{e, row + i * a.tile_rows, std::min(a.tile_rows, c - i * a.tile_rows), 0};
  }
  if (e == kExpertsMax - 1) {
    a.head[0] = rows[e];
    a.head[1] = blocks[e];
  }
}

__global__ __launch_bounds__(256) void experts_place_kernel(ExpertsArgs a) {
  __shared__ int hist[kExpertsMax];
  for (int i = threadIdx.x; i < a.n_experts; i += 256) hist[i] = 0;
  __syncthreads();
  const int64_t n_pairs = a.n_rows * a.top_k, per = (n_pairs + gridDim.x - 1) / gridDim.x;
  const int64_t lo = blockIdx.x * per, hi = std::min(lo + per, n_pairs);
  for (int64_t p = lo + threadIdx.x; p < hi; p += 256) {
    const int e = pair_expert(a, (int32_t)p);
    if (e >= 0) atomicAdd(&hist[e], 1);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < a.n_experts; i += 256)
    if (hist[i]) hist[i] = atomicAdd(&a.counts[a.n_experts + i], hist[i]);
  __syncthreads();
  for (int64_t p = lo + threadIdx.x; p < hi; p += 256) {
    const int e = pair_expert(a, (int32_t)p);
    if (e >= 0) a.pairs[atomicAdd(&hist[e], 1)] = (int32_t)p;
  }
}

__device__ __forceinline__ float silu(float g) { return g / (1.0f + __expf(-g)); }

// 64 rows x 32 channels of h, 16 rows a wave, fragments from memory
__global__ __launch_bounds__(256) void experts_gate_up_kernel(ExpertsArgs a) {
  if ((int)blockIdx.x >= a.head[1]) return;
  const ExpertTile t = a.tiles[blockIdx.x];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lg = lane >> 4, lc = lane & 15;
  const int f0 = blockIdx.y * 32;
  for (int r0 = wave * 16; r0 < t.count; r0 += 64) {
    const int r = r0 + lc, rc = t.row + std::min(r, t.count - 1);
    const int64_t n = a.pairs[rc] / a.top_k;
    const int8_t* x = a.xq + n * a.d_model + lg * 16;
    const int8_t* w = a.w_gu + ((int64_t)t.expert * 2 * a.d_ffn + f0 + lc) * a.d_model + lg * 16;
    const int64_t up = (int64_t)a.d_ffn * a.d_model, b16 = 16 * (int64_t)a.d_model;
    i32x4 acc[4] = {};
    for (int k = 0; k < a.d_model; k += 64) {
      const i32x4 fx = *(const i32x4*)(x + k);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(*(const i32x4*)(w + (j >> 1) * up + (j & 1) * b16 + k), fx, acc[j], 0, 0, 0);
    }
    if (r >= t.count) continue;
    const float xs = a.xs[n];
    const float* s = a.s_gu + (int64_t)t.expert * 2 * a.d_ffn + f0;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int f = 16 * j + lg * 4 + e;
        const float g = (float)acc[j][e] * s[f] * xs, u = (float)acc[2 + j][e] * s[a.d_ffn + f] * xs;
        ((__bf16*)a.h)[(int64_t)rc * a.d_ffn + f0 + f] = (__bf16)(silu(g) * u);
      }
  }
}

__global__ __launch_bounds__(256) void experts_down_kernel(ExpertsArgs a) {
  if ((int)blockIdx.x >= a.head[1]) return;
  const ExpertTile t = a.tiles[blockIdx.x];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lg = lane >> 4, lc = lane & 15;
  const int c0 = blockIdx.y * 64;
  for (int r0 = wave * 16; r0 < t.count; r0 += 64) {
    const int r = r0 + lc, rc = t.row + std::min(r, t.count - 1);
    const int8_t* h = a.hq + (int64_t)rc * a.d_ffn + lg * 16;
    const int8_t* w = a.w_down + ((int64_t)t.expert * a.d_model + c0 + lc) * a.d_ffn + lg * 16;
    i32x4 acc[4] = {};
    for (int k = 0; k < a.d_ffn; k += 64) {
      const i32x4 fh = *(const i32x4*)(h + k);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(*(const i32x4*)(w + (int64_t)j * 16 * a.d_ffn + k), fh, acc[j], 0, 0, 0);
    }
    if (r >= t.count) continue;
    const float hs = a.hs[rc];
    const float* s = a.s_down + (int64_t)t.expert * a.d_model + c0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int c = 16 * j + lg * 4 + e;
        a.part[(int64_t)a.pairs[rc] * a.d_model + c0 + c] = (float)acc[j][e] * s[c] * hs;
      }
  }
}

template <bool OUT_BF16>
__global__ __launch_bounds__(256) void experts_join_kernel(ExpertsArgs a) {
  const int64_t units = a.n_rows * (a.d_model / 4);
  for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < units; u += (int64_t)gridDim.x * 256) {
    const int64_t n = u / (a.d_model / 4);
    const int c = (int)(u - n * (a.d_model / 4)) * 4;
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j < a.top_k; ++j) {
      const int32_t p = (int32_t)(n * a.top_k + j);
      if (pair_expert(a, p) < 0) continue;
      y += a.ew[p] * *(const f32x4*)(a.part + (int64_t)p * a.d_model + c);
    }
    if (OUT_BF16)
      *(u32x2*)((uint16_t*)a.y + n * a.d_model + c) = u32x2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
    else
      *(f32x4*)((float*)a.y + n * a.d_model + c) = y;
  }
}

}  // namespace

int32_t experts_tile_rows(int64_t n_pairs, int32_t n_experts) { return 64; }

hipError_t launch_experts(const ExpertsArgs& a, hipStream_t s) {
  hipError_t e;
  const int64_t n_pairs = a.n_rows * a.top_k;
  experts_zero_kernel<<<dim3(1), dim3(256), 0, s>>>(a);
  if ((e = launch_i8_quantize(I8Args{a.x, a.xq, a.xs, a.n_rows, a.x_stride, a.d_model, nullptr}, s)) != hipSuccess) return e;
  const unsigned blocks = (unsigned)std::min<int64_t>((n_pairs + 1023) / 1024, 256);
  experts_count_kernel<<<dim3(blocks), dim3(256), 0, s>>>(a);
  experts_scan_kernel<<<dim3(1), dim3(kExpertsMax), 0, s>>>(a);
  experts_place_kernel<<<dim3(blocks), dim3(256), 0, s>>>(a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  experts_gate_up_kernel<<<dim3((unsigned)a.max_tiles, (unsigned)(a.d_ffn / 32)), dim3(256), 0, s>>>(a);
  if ((e = launch_i8_quantize(I8Args{a.h, a.hq, a.hs, n_pairs, a.d_ffn, a.d_ffn, a.head}, s)) != hipSuccess) return e;
  experts_down_kernel<<<dim3((unsigned)a.max_tiles, (unsigned)(a.d_model / 64)), dim3(256), 0, s>>>(a);
  const unsigned join = (unsigned)std::min<int64_t>((a.n_rows * (a.d_model / 4) + 255) / 256, 1 << 16);
  if (a.y_bf16) experts_join_kernel<true><<<dim3(join), dim3(256), 0, s>>>(a);
  else experts_join_kernel<false><<<dim3(join), dim3(256), 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace mla

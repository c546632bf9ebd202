// Rows into and out of the paged 4-bit latent cache (mx4.h).
#include "mx4.h"

#include <algorithm>

namespace mla {
namespace {

struct RowPlaces {
  unsigned char *codes, *scales, *rope;
};
__device__ __forceinline__ RowPlaces row_places(unsigned char* cache, int32_t slot, int32_t page_rows) {
  const int32_t page = slot / page_rows, r = slot - page * page_rows;
  unsigned char* p = cache + (int64_t)page * page_rows * kCacheRow;
  return {p + r * (int64_t)kCacheCodes, p + page_rows * (int64_t)kCacheCodes + r * kCacheScales,
          p + page_rows * (int64_t)(kCacheCodes + kCacheScales) + r * (int64_t)kCacheRope};
}

// A wave takes a row: eight latent values a lane, and in lanes 0 .. 31 the pair (j, j + 32)
// of the RoPE key, turned by pos theta_j (reduced in 64 bits, in revolutions).  Bound by
// memory: 1152 bytes read and 400 written a row.
__global__ __launch_bounds__(256) void cache_append_kernel(CacheRowsArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t step = (int64_t)gridDim.x * 4;
  for (int64_t n = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); n < a.n_rows; n += step) {
    const int32_t slot = a.slots[n];
    if (slot < 0 || slot >= a.n_slots) continue;
    const uint16_t* src = (const uint16_t*)a.kv + n * a.kv_stride;
    const u32x4 x = *(const u32x4*)(src + lane * 8);
    const int j = lane & 31;
    const uint32_t k1 = src[512 + j], k2 = src[544 + j];
    const RowPlaces p = row_places(a.cache, slot, a.page_rows);
    uint32_t e;
    const uint32_t codes = mx4_codes(x, e);
    ((uint32_t*)p.codes)[lane] = codes;
    if ((lane & 3) == 0) p.scales[lane >> 2] = (unsigned char)e;
    if (lane < 32) {
      uint16_t o1 = (uint16_t)k1, o2 = (uint16_t)k2;
      if (a.pos != nullptr) {
        const double rev = (double)a.pos[n] * a.rope.theta[j];
        const float r = (float)(rev - rint(rev));
        const float sn = __builtin_amdgcn_sinf(r), cn = __builtin_amdgcn_cosf(r);
        const float x1 = bf16_lo(k1), x2 = bf16_lo(k2);
        o1 = __builtin_bit_cast(uint16_t, (__bf16)(x1 * cn - x2 * sn));
        o2 = __builtin_bit_cast(uint16_t, (__bf16)(x1 * sn + x2 * cn));
      }
      ((uint16_t*)p.rope)[j] = o1;
      ((uint16_t*)p.rope)[32 + j] = o2;
    }
  }
}

__global__ __launch_bounds__(256) void cache_gather_kernel(CacheRowsArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t step = (int64_t)gridDim.x * 4;
  for (int64_t n = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); n < a.n_rows; n += step) {
    const int32_t slot = a.slots[n];
    if (slot < 0 || slot >= a.n_slots) continue;
    const RowPlaces p = row_places(a.cache, slot, a.page_rows);
    uint16_t* dst = (uint16_t*)a.kv + n * a.kv_stride;
    const uint32_t codes = ((const uint32_t*)p.codes)[lane];
    const uint32_t e = p.scales[lane >> 2];
    if (lane < 8) *(u32x4*)(dst + 512 + lane * 8) = ((const u32x4*)p.rope)[lane];
    *(bf16x8*)(dst + lane * 8) = mx4_values(codes, mx4_scale(e));
  }
}

unsigned row_grid(int64_t n) { return (unsigned)std::min<int64_t>((n + 3) / 4, 1 << 20); }

}  // namespace

hipError_t launch_cache_append(const CacheRowsArgs& a, hipStream_t s) {
  cache_append_kernel<<<dim3(row_grid(a.n_rows)), dim3(256), 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_cache_gather(const CacheRowsArgs& a, hipStream_t s) {
  cache_gather_kernel<<<dim3(row_grid(a.n_rows)), dim3(256), 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace mla

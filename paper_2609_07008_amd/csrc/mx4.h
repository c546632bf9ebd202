// The library's 4-bit format (mx4): groups of 32 consecutive values, e2m1 codes
// (sign, 0 .5 1 1.5 2 3 4 6) two a byte, the even value in the low nibble, and one
// scale byte e a group that stands for 2^(e - 127); e = 255 makes the group NaN.
// Every bf16 step of quantizing is exact, so results do not depend on who computes
// them; what a code stands for is exact in bf16.
#pragma once

#include "common.h"

namespace mla {

typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));

// The scale as the conversion instructions take it: they read the exponent field alone
// (0 is 2^-127, 255 gives NaN; checked over all scales and bytes).
__device__ __forceinline__ float mx4_scale(uint32_t e) { return __uint_as_float(e << 23); }

// 16 bytes a lane from memory to LDS, lane after lane
__device__ __forceinline__ void dma16(const void* from, unsigned char MLA_LDS* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (MLA_LDS void*)to, 16, 0, 0);
}

// eight codes (one register) as eight bf16 values, in order
__device__ __forceinline__ bf16x8 mx4_values(uint32_t codes, float scale) {
  const bf16x2v a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
  const bf16x2v b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
  const bf16x2v c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
  const bf16x2v d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Eight consecutive values a lane, a group in four neighbouring lanes: the lane's codes
// and the group's scale byte.  The scale is 2^(floor(log2 max) - 2), one step more where
// the largest value is 7 units of it or more (6 is the largest code; 7 is half way to the
// next): no value is off by more than half the top step.  A group with a NaN or an
// infinity gets scale 255 and codes 0.
__device__ __forceinline__ uint32_t mx4_codes(u32x4 x, uint32_t& scale_byte) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  auto mag = [](uint32_t v) { return __builtin_bit_cast(u16x2, v & 0x7fff7fffu); };
  const u16x2 m = __builtin_elementwise_max(__builtin_elementwise_max(mag(x[0]), mag(x[1])),
                                            __builtin_elementwise_max(mag(x[2]), mag(x[3])));
  int a = m[0] > m[1] ? m[0] : m[1];
  // maximum over the four lanes of the quad
  int o = __builtin_amdgcn_mov_dpp(a, 0xB1, 0xf, 0xf, true);   // lanes 1 0 3 2
  a = o > a ? o : a;
  o = __builtin_amdgcn_mov_dpp(a, 0x4E, 0xf, 0xf, true);       // lanes 2 3 0 1
  a = o > a ? o : a;
  const int ex = (a >> 7) - 2 + ((a & 0x7f) >= 0x60 ? 1 : 0);
  const bool odd = a >= 0x7f80;
  const int e = odd ? 255 : (ex > 0 ? ex : 0);
  scale_byte = (uint32_t)e;
  const float s = mx4_scale((uint32_t)e);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2v, (uint32_t)x[0]), s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2v, (uint32_t)x[1]), s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2v, (uint32_t)x[2]), s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2v, (uint32_t)x[3]), s, 3);
  return odd ? 0u : c;
}

struct Mx4Args {
  const void* x;         // [n_rows, n_cols] bf16, rows x_stride elements apart (quantize: read, else written)
  void* codes;           // [n_rows, n_cols / 2]
  void* scales;          // [n_rows, n_cols / 32]
  int64_t n_rows;
  int64_t x_stride;
  int32_t n_cols;        // a multiple of 32
};
hipError_t launch_mx4_quantize(const Mx4Args& a, hipStream_t s);
hipError_t launch_mx4_dequantize(const Mx4Args& a, hipStream_t s);

// y = W z with W in mx4
struct WbMx4Args {
  const uint16_t* z;       // [n_rows, d_in] bf16
  const uint8_t* codes;    // [d_out, d_in / 2]
  const uint8_t* scales;   // [d_out, d_in / 32]
  void* y;                 // [n_rows, d_out] f32 or bf16
  int64_t n_rows;
  int32_t d_in;            // a multiple of 64
  int32_t d_out;
  int32_t y_bf16;
};
hipError_t launch_wb_mx4(const WbMx4Args& a, hipStream_t s);

// ----------------------------------------------------------------------------
// the paged latent cache (512 + 64): a row takes 256 bytes of codes, 16 of scales
// and its RoPE key in bf16; a page holds these as planes, codes first
// ----------------------------------------------------------------------------
constexpr int kCacheCodes = 256, kCacheScales = 16, kCacheRope = 128;
constexpr int kCacheRow = kCacheCodes + kCacheScales + kCacheRope;
constexpr int kCacheTile = 64;   // keys per attention tile; page_rows is a multiple

struct RopeTable {
  double theta[kMaxRopePairs];   // RoPE frequencies in revolutions
};

struct CacheRowsArgs {
  void* kv;                // [n_rows, 576] bf16, rows kv_stride elements apart
  const int32_t* pos;      // [n_rows] or NULL: RoPE part as given
  const int32_t* slots;    // [n_rows]; outside [0, n_slots): skipped
  unsigned char* cache;
  int64_t n_rows;
  int64_t kv_stride;
  int32_t n_slots;         // cache_pages * page_rows
  int32_t page_rows;
  RopeTable rope;
};
hipError_t launch_cache_append(const CacheRowsArgs& a, hipStream_t s);
hipError_t launch_cache_gather(const CacheRowsArgs& a, hipStream_t s);

constexpr int kMaxShares = 256;   // of the attention's work: a workgroup a compute unit
constexpr int kLongShares = 32;   // a request that more shares than this hold is joined by whole workgroups

struct CacheAttendArgs {
  const unsigned char* cache;
  const uint16_t* q;          // [n_seqs, n_q, n_heads, 576] bf16
  const int32_t* pos;         // [n_seqs, n_q]
  const mla_page* pages;      // [n_seqs, max_pages]
  const int32_t* seq_pages;   // [n_seqs]
  uint16_t* out_o;            // [n_seqs, n_q, n_heads, 512] bf16
  float* out_lse;             // [n_seqs, n_q, n_heads] or NULL
  float* part_o;              // [2 shares, n_blocks, block / 16, 32, 64, 4]: sums of a request that several shares hold, as 16-dim fragments
  float* part_ml;             // [2 shares, n_blocks, block, 4]: reference (log2 units), row sums of the weights and of their bf16 values
  int32_t* tile_base;         // [n_seqs + 1]: tiles before each request
  int32_t* long_seq;          // [kMaxShares / kLongShares], k: the request of more than kLongShares shares whose first share of an index kLongShares divides is kLongShares k, or -1
  int32_t n_seqs, n_q, n_heads;
  int32_t max_pages, page_rows, cache_pages;
  int32_t page_tiles;         // page_rows in tiles
  int32_t block;              // head-rows per workgroup: 16, 32 or 64
  int32_t n_blocks;           // blocks of a request's n_q * n_heads head-rows
  int32_t shares;             // equal runs of the batch's tiles
  float scale_log2;
  double inv_page_tiles, inv_shares, inv_blocks;   // reciprocals
  RopeTable rope;
};
hipError_t launch_cache_attend(const CacheAttendArgs& a, hipStream_t s);

}  // namespace mla

// The K loop of products in 8-bit integers, C = A B^T with both operands K-contiguous: tiles of
// 32 MI rows x BN channels per workgroup of 8 waves (2 x 4, each 16 MI x BN / 4 by 16x16x64
// MFMAs, i32 sums).  The plan is that of the bf16 product in wb.hip: a row of a slice is 128
// bytes in both, here 128 of K, and an MFMA of 16 clocks takes twice the products.  The
// operands come in by direct global->LDS loads, NST slices in LDS; the barrier of a slice sits
// between a step's halves, so that a half's MFMAs, their fragments already in registers, run
// over the LDS reads of the next half and the direct loads.
#pragma once

#include <algorithm>
#include <type_traits>

#include "i8.h"

namespace mla {

constexpr int I8_WAVES = 8;
constexpr int I8_ROWB = 128;   // bytes of a row of a slice

__device__ __forceinline__ int i8_swz(int r) { return (r >> 1) & 7; }

// waves a SIMD: two workgroups a unit where both fit its LDS
constexpr int i8_occupancy(int mi, int bn, int nst) { return (32 * mi + bn) * I8_ROWB * nst <= 80 * 1024 ? 4 : 2; }

template <int MI, int BN, int NST>
struct I8Tile {
  static constexpr int NI = BN / 64, BM = 32 * MI;
  static constexpr int A_BYTES = BM * I8_ROWB, STAGE = A_BYTES + BN * I8_ROWB;
  static constexpr int NLOADS = STAGE / 1024;                      // 1 KB direct loads (8 rows each) a slice
  static constexpr int LPW = (NLOADS + I8_WAVES - 1) / I8_WAVES;   // a wave; past the end the last one again
  static constexpr int LDS = NST * STAGE;

  const unsigned char* src[LPW];
  uint32_t voff[LPW];
  int q[LPW];
  i32x4 acc[MI][NI];

  // Load q of a slice fills LDS bytes [1024 q, +1024) of its stage: the slice's A rows, then its
  // B rows, 8 each; chunk c of row r sits at slot c ^ i8_swz(r).  `row(is_a, r0, r)` gives the
  // wave-uniform address that row r of A or B (r0: the first of its 8) is taken relative to and
  // the row's offset from it.
  template <class Row>
  __device__ __forceinline__ void aim(int wave, int lane, Row&& row) {
#pragma unroll
    for (int j = 0; j < LPW; ++j) {
      q[j] = std::min(wave + I8_WAVES * j, NLOADS - 1);
      const bool is_a = q[j] < A_BYTES / 1024;
      const int r0 = 8 * (is_a ? q[j] : q[j] - A_BYTES / 1024), r = r0 + (lane >> 3);
      row(is_a, r0, r, src[j], voff[j]);
      voff[j] += ((lane & 7) ^ i8_swz(r)) * 16;
    }
  }

  // row of the tile that block i of 16 begins at, for the waves of half wm: a tile's first rows
  // are shared by both halves
  static __device__ __forceinline__ int row_of(int wm, int i) { return 32 * i + 16 * wm; }

  // acc = A B^T over `d_in` of K, a multiple of 64.  Of a last slice of 64 the upper chunks, past
  // the rows' ends, are taken from the lower ones and not used.  Of a tile with fewer rows than
  // it has room for, the blocks i >= mi take no products (their sums are 0).
  __device__ __forceinline__ void product(unsigned char* lds, int wave, int lane, int d_in, int mi = MI) {
    if (mi >= MI) steps<false>(lds, wave, lane, d_in, MI);
    else steps<true>(lds, wave, lane, d_in, mi);
  }

  template <bool SOME>
  __device__ __forceinline__ void steps(unsigned char* lds, int wave, int lane, int d_in, int mi) {
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
    const int nk = (d_in + I8_ROWB - 1) / I8_ROWB, cut = d_in % I8_ROWB ? nk - 1 : nk;
    auto load_one = [&](int j, int kt, int st) {
      uint32_t v = voff[j];
      if (kt == cut) v -= (((lane >> 2) ^ q[j]) & 1) * 64;   // bit 2 of the chunk: i8_swz of the 8 rows has q's lowest there
      dma16(src[j] + (int64_t)kt * I8_ROWB, v, (const unsigned char MLA_LDS*)(lds + st + 1024 * q[j]));
    };
    // fragments (16 rows x 64 of K): lane group lg holds chunk 4 h + lg of row lc; the rows'
    // swizzle repeats every 16, so blocks are immediate offsets
    const int wm = wave >> 2, wn = wave & 3, lg = lane >> 4, lc = lane & 15;
    const int fa = (wm * 16 + lc) * I8_ROWB + ((lg ^ i8_swz(lc)) * 16);
    const int fb = A_BYTES + (wn * (BN / 4) + lc) * I8_ROWB + ((lg ^ i8_swz(lc)) * 16);
    struct Frags {
      i32x4 a[MI], b[NI];
    };
    auto frag = [&](int base, int st, int h, int rows) -> i32x4 {
      return *(const i32x4 MLA_LDS*)((const unsigned char MLA_LDS*)lds + ((st + base) ^ (h * 64)) + rows * I8_ROWB);
    };
    auto half = [&](const Frags& f, Frags& nx, int nst, int nh, auto LOAD, int kt, int lst) {
      constexpr int R = MI + NI;                 // fragments to read, spread over the rows of MFMAs
      constexpr int PER = (R + MI - 1) / MI;
      int rd = 0, ld = 0;
#pragma unroll
      for (int i = 0; i < MI; ++i) {
#pragma unroll
        for (int k = 0; k < PER; ++k, ++rd)
          if (rd < NI) nx.b[rd] = frag(fb, nst, nh, 16 * rd);
          else if (rd < R && (!SOME || rd - NI < mi)) nx.a[rd - NI] = frag(fa, nst, nh, 32 * (rd - NI));
        if constexpr (decltype(LOAD)::value) {
#pragma unroll
          for (int k = 0; k < (LPW + MI - 1) / MI; ++k, ++ld)
            if (ld < LPW) load_one(ld, kt, lst);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (!SOME || i < mi) {
#pragma unroll
          for (int jj = 0; jj < NI; ++jj) {
            const int j = i & 1 ? NI - 1 - jj : jj;   // neighbours share an operand
            acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(f.b[j], f.a[i], acc[i][j], 0, 0, 0);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    // Slices 0 .. NST-1 go out first.  Step kt: the first half's MFMAs beside the reads of the
    // second half's fragments; one barrier (slice kt is read by every wave, so its buffer is
    // free; slice kt + 1 has landed); the second half's MFMAs beside the loads of slice kt + NST
    // and the reads of slice kt + 1's first half.
#pragma unroll
    for (int p = 0; p < NST; ++p)
      if (p < nk)
#pragma unroll
        for (int j = 0; j < LPW; ++j) load_one(j, p, p * STAGE);
    if (nk >= NST) dma_barrier<(NST - 1) * LPW>(); else dma_barrier<0>();
    Frags f0, f1;
#pragma unroll
    for (int j = 0; j < NI; ++j) f0.b[j] = frag(fb, 0, 0, 16 * j);
#pragma unroll
    for (int i = 0; i < MI; ++i) f0.a[i] = frag(fa, 0, 0, 32 * i);
    int st = 0, kt = 0;
    for (; kt + NST < nk; ++kt) {
      half(f0, f1, st, 1, std::false_type{}, 0, 0);
      dma_barrier<(NST - 2) * LPW>();
      const int nst = st == (NST - 1) * STAGE ? 0 : st + STAGE;
      half(f1, f0, nst, 0, std::true_type{}, kt + NST, st);
      st = nst;
    }
    for (; kt < nk; ++kt) {
      half(f0, f1, st, 1, std::false_type{}, 0, 0);
      dma_barrier<0>();
      const int nst = st == (NST - 1) * STAGE ? 0 : st + STAGE;
      if (kt != cut) half(f1, f0, nst, 0, std::false_type{}, 0, 0);   // after the last slice: reads of a stale buffer, not used
      st = nst;
    }
    dma_barrier<0>();
  }
};

}  // namespace mla

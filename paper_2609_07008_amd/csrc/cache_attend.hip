// Absorbed-MLA attention of new tokens over the paged 4-bit latent cache (mx4.h): the
// decode form of Alg. 2's SelectiveMLA, each page in its own RoPE frame (the query is
// turned by t - frame, eq:rope), 512 + 64 latent, the latent as the value.
//
// A request's head-rows (its n_q tokens' heads) share its keys.  A workgroup takes 16 NB of
// them and a run of 64-key tiles, with two kinds of waves that work a tile apart and meet
// once a tile:
//   score    four.  S^T = K Q^T for 16 head-rows a wave, queries in registers; with fewer
//            than 64 head-rows the waves of the same 16 share the tile's keys.  The turned
//            RoPE part of the query goes in twice, as its bf16 value and the bf16 of what
//            that lost: the scores are then as exact as the products, which a request of a
//            few keys shows in its lse.  Softmax against a reference that moves (and sums
//            are rescaled) only when a tile exceeds it by 2^8, so weights stay below 2^9
//            and sums in 32 bits lose nothing.  Weights in bf16: half a step of each, next
//            to an output of the same width; outputs are divided by the sum of the rounded
//            weights, so that a request of one key answers with its value, and the lse takes
//            the sum of the weights themselves.
//   value    four, eight with fewer than 64 head-rows, 512 / waves dims each: O^T += V^T P^T.
//            They convert their dims of the tiles too (v_cvt_scalef32_pk_bf16_fp4), once,
//            into LDS as bf16 in the layout of the online attention's tiles
//            (attend_pair.hip): the key of the scores and, by transposing reads, the value.
// A key that no row of the call sees (behind a page's rows, past the last position) is
// zero in LDS whatever the page holds there.
//
// Work is split by tiles, not by requests: the batch's tiles, in order, form `shares`
// equal runs, one a workgroup (and head-row block).  A request inside one run is written
// at once; one that crosses runs leaves sums to the joining kernels.
//
// Measured, whole calls with the joining, by card: 64 requests of ~16k keys (18,474 tiles), 64
// heads 200 to 215 us, 2.5 us a tile and compute unit; a tile's products keep the matrix cores
// busy 2300 of its 5000 clocks, its LDS traffic takes 2600, its vector instructions 2100: the
// two kinds of waves hide each other only in part (207 us; without the latent's score products
// and their reads 174, without the value products 186, without softmax or conversion 203 to 206,
// all keys from one page 190 of 215).  16 requests of ~8k, 256 head-rows 85 to 89 us; one of
// 264k, 64 heads 63 to 66.  48 of ~6k, 16 heads 41 to 43, and 46 to 47 where other calls have
// used the last-level cache in between; 8 of it are the start (three dependent reads from
// memory before the first tile) and 5 the joining.  No part alone bounds a tile there (without
// conversion 40.5 of 41.3, score products 39.2, value products 38.5): what is left is the way
// through one from barrier to barrier, and eight value waves against four take 41.4 against
// 43.5.
#include "mx4.h"

#include <algorithm>

namespace mla {
namespace {

constexpr int kWaves = 8, kThreads = kWaves * 64;   // of the joining kernels

typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kLong = kLongShares;   // see cache_merge_mixed_kernel

template <int NB>
struct CaCfg {
  static constexpr int BM = 16 * NB;         // head-rows of a workgroup
  static constexpr int KW = 4 / NB;          // score waves that share 16 head-rows, each with its keys
  static constexpr int KB = NB;              // 16-key blocks of a score wave
  // value waves: eight up to 32 head-rows (41.4 against 43.5 us with four, 48 requests of 6k keys
  // and 16 heads); at NB = 4 eight, in 168 registers each, take as long as four
  static constexpr int VW = NB == 4 ? 4 : 8;
  static constexpr int WAVES = 4 + VW, THREADS = 64 * WAVES;
  static constexpr int ND = 32 / VW;         // 16-dim fragments of a value wave
  static constexpr int GW = 16 / VW;         // groups of a row that it converts
  static constexpr int NI = GW;              // loads of a tile's codes in it, 64 / GW keys each
  static constexpr int KBL = 8 * 1024 + 128; // latent of an 8-key block: a kilobyte per 64 dims
  static constexpr int LAT = 8 * KBL;        // a tile
  static constexpr int P_OFF = 2 * LAT;      // weights of two tiles, [32 keys][NB] KB in the layout of the MFMA operand
  static constexpr int P_BYTES = 2 * NB * 1024;
  static constexpr int M_OFF = P_OFF + 2 * P_BYTES;     // [2][KW][BM]: references of the tile's weights
  static constexpr int L_OFF = M_OFF + 2 * KW * BM * 4; // [KW][BM][2]: row sums at the end, of the weights and of their bf16 values
  static constexpr int TH_OFF = L_OFF + KW * BM * 8;
  static constexpr int LDS = TH_OFF + kMaxRopePairs * 8;
  static constexpr int Q_OFF = LAT;          // queries on their way to registers, 1152 bytes a head-row
  static_assert(Q_OFF + BM * 1152 <= M_OFF, "before the second tile and the weights are stored");
  static_assert(LDS <= 160 * 1024, "LDS of a compute unit");
};

// slot of 16-byte chunk c of key k in its kilobyte: c ^ key_swz(k) (see attend_pair.hip)
__device__ __forceinline__ int key_swz(int k) { return k ^ ((~k & 1) << 2); }

// four bytes a lane from memory to LDS, lane after lane
__device__ __forceinline__ void dma4(const unsigned char* from, unsigned char MLA_LDS* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (MLA_LDS void*)to, 4, 0, 0);
}
static_assert(sizeof(RopeTable) == 64 * 4, "a dword a lane");

// this wave's LDS accesses are done, then all waves meet (loads from memory stay in flight)
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// The lane, opaque to the compiler: addresses formed from it in one kind of wave are not
// kept in registers through the code of the other.
__device__ __forceinline__ int lane_now() {
  int v;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(v));
  return v;
}

// x / d for 0 <= x < 2^31, inv = 1 / d: the product is off by less than one
__device__ __forceinline__ int quotient(int x, int d, double inv) {
  uint32_t q = (uint32_t)((double)x * inv);
  if (q * (uint32_t)d > (uint32_t)x) --q;
  if ((q + 1) * (uint32_t)d <= (uint32_t)x) ++q;
  return __builtin_amdgcn_readfirstlane((int)q);
}

struct Tile {       // wave-uniform
  int page, off;    // page to read (0 where there is none), the tile's first row in it
  int rows;         // rows of the tile that hold keys, 0 .. 64
  int frame, pos0;  // RoPE frame, request position of the page's first row
};

// The tiles of a request from tile u on.  Lanes hold 16 page entries, four words each, and
// the next 16, so that a tile's entry is there when it is asked for.
struct Cursor {
  const mla_page* entries;
  int e, sub, tpp, e_last, held;   // entry and tile of it to describe next; first entry held
  int32_t word, ahead;
  __device__ __forceinline__ int32_t fetch(int first) const {
    const int lane = lane_now(), at = first + (lane >> 2);
    return ((const int32_t*)(entries + (at < e_last ? at : e_last)))[lane & 3];
  }
  __device__ __forceinline__ void open(const CacheAttendArgs& a, int b, int u0, int u1) {
    entries = a.pages + (int64_t)b * a.max_pages;
    tpp = a.page_tiles;
    e = quotient(u0, tpp, a.inv_page_tiles);
    sub = u0 - e * tpp;
    e_last = quotient(u1 - 1, tpp, a.inv_page_tiles);
    held = e;
    word = fetch(e);
    ahead = fetch(e + 16);
  }
  __device__ __forceinline__ Tile next(const CacheAttendArgs& a) {
    if (__builtin_expect(e - held == 16, 0)) {
      held = e;
      word = ahead;
      ahead = fetch(e + 16);
    }
    const int l = (e - held) * 4;
    Tile t;
    const int page = __builtin_amdgcn_readlane(word, l), rows = __builtin_amdgcn_readlane(word, l + 1);
    const bool there = (unsigned)page < (unsigned)a.cache_pages;
    t.page = there ? page : 0;
    t.off = sub * kCacheTile;
    const int left = (there ? (rows < a.page_rows ? rows : a.page_rows) : 0) - t.off;
    t.rows = left < 0 ? 0 : left < kCacheTile ? left : kCacheTile;
    t.pos0 = __builtin_amdgcn_readlane(word, l + 2);
    t.frame = __builtin_amdgcn_readlane(word, l + 3);
    if (++sub == tpp) {
      sub = 0;
      ++e;
    }
    return t;
  }
};

// keys of the tile that a row at position t sees, 0 .. 64
__device__ __forceinline__ int seen_keys(const Tile& x, int t) {
  const int64_t d = (int64_t)t - x.pos0 - x.off + 1;
  return t < 0 || d < 0 ? 0 : d < x.rows ? (int)d : x.rows;
}

// maximum / sum over the four lanes (l, l ^ 16, l ^ 32, l ^ 48) that hold a head-row's keys
__device__ __forceinline__ float quad_max(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float quad_sum(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

__device__ __forceinline__ int tiles_of(const CacheAttendArgs& a, int b) {
  int n = a.seq_pages[b];
  n = n < 0 ? 0 : n < a.max_pages ? n : a.max_pages;
  return n * a.page_tiles;
}

// The batch's tiles as `shares` runs in order: the first r of them a tile longer.
struct Runs {
  int q, r;
  __device__ __forceinline__ Runs(const CacheAttendArgs& a, int total) : q(quotient(total, a.shares, a.inv_shares)), r(total - q * a.shares) {}
  __device__ __forceinline__ int first(int s) const { return q * s + (s < r ? s : r); }   // share s's first tile
  __device__ __forceinline__ int share(int tile) const {                                  // the share that holds it
    const int longer = r * (q + 1);
    return tile < longer ? tile / (q + 1) : r + (tile - longer) / q;
  }
};

template <int NB>
__global__ __launch_bounds__(CaCfg<NB>::THREADS, CaCfg<NB>::WAVES / 4) void cache_attend_kernel(CacheAttendArgs a) {
  using C = CaCfg<NB>;
  constexpr int BM = C::BM, KB = C::KB, ND = C::ND, GW = C::GW, NI = C::NI;
  __shared__ __attribute__((aligned(16))) unsigned char lds[C::LDS];
  unsigned char MLA_LDS* L = (unsigned char MLA_LDS*)lds;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int R = a.n_q * a.n_heads;

  // all arguments in one go: taken as they are needed, each of their lines would cost a
  // trip to the host's memory before the first key
  asm volatile("" ::"s"(a.cache), "s"(a.q), "s"(a.pos), "s"(a.pages), "s"(a.seq_pages), "s"(a.tile_base), "s"(a.n_seqs),
               "s"(a.n_q), "s"(a.n_heads), "s"(a.max_pages), "s"(a.page_rows), "s"(a.cache_pages), "s"(a.page_tiles),
               "s"(a.n_blocks), "s"(a.shares), "s"(a.scale_log2), "s"(a.inv_page_tiles), "s"(a.inv_shares),
               "s"(a.inv_blocks));
  // Workgroups go to the 8 XCDs round-robin; the blocks of a share follow each other on one.
  // Shares are dealt to the XCDs in turn, so that a few tiles use all of them, or, where that
  // does not come out even, each XCD takes an eighth of the (share, block) pairs (16 requests
  // of 3 tokens, 85 shares: 79 us where dealing shares out took 129; one of 32 tokens and 128
  // heads, 4 shares: 100 against 181).
  int share, hb;
  {
    const int xcd = blockIdx.x & 7, at = blockIdx.x >> 3;
    const int pairs = a.shares * a.n_blocks, per_xcd = (pairs + 7) / 8;
    const int pair = a.shares % 8 == 0 ? at : xcd * per_xcd + at;
    if (pair >= pairs) return;
    share = quotient(pair, a.n_blocks, a.inv_blocks);
    hb = pair - share * a.n_blocks;
    if (a.shares % 8 == 0) share = share * 8 + xcd;
  }
  double MLA_LDS* theta = (double MLA_LDS*)(L + C::TH_OFF);

  // tiles before each request, by a scan over the batch; the request that holds the
  // share's first tile
  int first_b, first_base, first_n, total;
  {
    int MLA_LDS* sums = (int MLA_LDS*)L;
    const int per = (a.n_seqs + C::THREADS - 1) / C::THREADS;
    const int b0 = tid * per < a.n_seqs ? tid * per : a.n_seqs;
    const int b1 = b0 + per < a.n_seqs ? b0 + per : a.n_seqs;
    int mine = 0;
#pragma unroll 4
    for (int b = b0; b < b1; ++b) mine += tiles_of(a, b);
    int inc = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(inc, o, 64);
      if (lane >= o) inc += v;
    }
    if (lane == 63) sums[wave] = inc;
    if (blockIdx.x == 0 && tid < kMaxShares / kLong) a.long_seq[tid] = -1;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < C::WAVES; ++w) {
      const int v = sums[w];
      before += w < wave ? v : 0;
      total += v;
    }
    int base = before + inc - mine;
    const Runs runs(a, total);   // total is the same in all lanes
    const int lo = runs.first(share);
    const bool writes = blockIdx.x == 0;
    for (int b = b0; b < b1; ++b) {
      const int n = per == 1 ? mine : tiles_of(a, b);
      if (writes) {
        a.tile_base[b] = base;
        if (n > kLong && n > (int64_t)(kLong - 1) * runs.q) {
          const int s0 = runs.share(base), s1 = runs.share(base + n - 1);
          if (s1 - s0 >= kLong) a.long_seq[(s0 + kLong - 1) / kLong] = b;   // at the first kLong-th share that it has
        }
      }
      if (lo >= base && lo < base + n) {
        sums[16] = b;
        sums[17] = base;
        sums[18] = n;
      }
      base += n;
    }
    if (writes && tid == 0) a.tile_base[a.n_seqs] = total;
    __syncthreads();
    first_b = __builtin_amdgcn_readfirstlane(sums[16]);
    first_base = __builtin_amdgcn_readfirstlane(sums[17]);
    first_n = __builtin_amdgcn_readfirstlane(sums[18]);
    total = __builtin_amdgcn_readfirstlane(total);
  }
  const Runs runs(a, total);
  const int lo = runs.first(share), hi = runs.first(share + 1);
  if (lo >= hi) return;

  const uint32_t plane_s = (uint32_t)a.page_rows * kCacheCodes, plane_r = plane_s + (uint32_t)a.page_rows * kCacheScales;

  // Lanes hold the tiles of 64 requests, so that the next one with any is found at once,
  // however many of a padded batch lie between.
  int b = first_b, base = first_base, n = first_n, held = first_b;
  auto tiles_from = [&](int from) { return from + lane < a.n_seqs ? tiles_of(a, from + lane) : 0; };
  int next_tiles = tiles_from(held);
  for (;;) {
    const int u0 = lo > base ? lo - base : 0, u1 = hi < base + n ? hi - base : n;
    const int seq_base = base;
    base += n;
    Cursor cur;
    cur.open(a, b, u0, u1);
    const int32_t* tseq = a.pos + (int64_t)b * a.n_q;
    lds_barrier();   // the tables, and what the previous request left in LDS, are read
    if (wave < 4) {
      // ------------------------------------------------------------------ score wave
      // 16-key blocks kw KB .. of the tile, block rw of the head-rows; rows past the end
      // repeat the last one and are not stored.
      const int kw = wave % C::KW, rw = wave / C::KW;
      const int lane = lane_now(), lg = lane >> 4, lc = lane & 15;
      const unsigned char* qb = (const unsigned char*)a.q + ((int64_t)b * R + hb * BM) * 1152;
      if (wave == 0 && b == first_b)
        dma4((const unsigned char*)__builtin_amdgcn_kernarg_segment_ptr() + offsetof(CacheAttendArgs, rope) + lane * 4, L + C::TH_OFF);
      const int q_last = R - 1 - hb * BM, row = rw * 16 + lc;   // of the block
      // The block's queries come through LDS: as fragments, sixteen rows a load, they would keep
      // the address unit four times as long.  A row's 16-byte chunk c lies at c ^ (row & 7).
#pragma unroll
      for (int j = wave; j < 18 * NB; j += 4) {
        const int at = j * 64 + lane, r = at / 72, c = at - r * 72;
        dma16(qb + (uint32_t)((r < q_last ? r : q_last) * 1152 + (c ^ (r & 7)) * 16), L + C::Q_OFF + j * 1024);
      }
      const int t_row = tseq[(hb * BM + (row < q_last ? row : q_last)) / a.n_heads];
      bf16x8 qf[16], qraw[2], qh[2], ql[2];   // Q fragments (B operand): dims ks*32 + lg*8 .. +7 of head-row lc
      // the RoPE part in a page's frame: the bf16 value and the bf16 of what it lost
      auto relocate = [&](int frame) {
        const double dd = (double)((int64_t)t_row - frame);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const double rev = dd * theta[lg * 8 + i];
          const float r = (float)(rev - rint(rev));
          const float sn = __builtin_amdgcn_sinf(r), cn = __builtin_amdgcn_cosf(r);
          const float f1 = (float)qraw[0][i], f2 = (float)qraw[1][i];
          const float y1 = f1 * cn - f2 * sn, y2 = f1 * sn + f2 * cn;
          qh[0][i] = (__bf16)y1;
          qh[1][i] = (__bf16)y2;
          ql[0][i] = (__bf16)(y1 - (float)qh[0][i]);
          ql[1][i] = (__bf16)(y2 - (float)qh[1][i]);
        }
      };
      // RoPE keys as K fragments: key kb*16 + lc of the wave's, chunks lg and lg + 4
      bf16x8 kr[KB][2];
      auto load_rope = [&](const Tile& t) {
        const unsigned char* p = a.cache + (int64_t)t.page * a.page_rows * kCacheRow + plane_r;
        const uint32_t at = (uint32_t)(t.off + kw * KB * 16 + lc) * kCacheRope + (uint32_t)lg * 16;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
          kr[kb][0] = *(const bf16x8*)(p + at + kb * 16 * kCacheRope);
          kr[kb][1] = *(const bf16x8*)(p + at + kb * 16 * kCacheRope + 64);
        }
      };
      // K fragments (A operand, 16 keys x 32 dims): key kb*16 + lc, chunk 4 ks + lg
      const int kat = (kw * KB * 2 + (lc >> 3)) * C::KBL + (lc & 7) * 128 + ((lg ^ key_swz(lc & 7)) * 16);
      Tile t = cur.next(a);
      load_rope(t);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      lds_barrier();   // the queries have landed
      {
        const unsigned char MLA_LDS* q0 = L + C::Q_OFF + row * 1152;
#pragma unroll
        for (int ks = 0; ks < 18; ++ks) {
          const bf16x8 v = *(const bf16x8 MLA_LDS*)(q0 + (ks >> 1) * 128 + ((((ks & 1) * 4 + lg) ^ (row & 7)) * 16));
          (ks < 16 ? qf[ks & 15] : qraw[ks & 1]) = v;
        }
      }
      relocate(t.frame);
      float m_run = -INFINITY, l_run = 0.f, r_run = 0.f;   // reference; row sums of the weights and of their bf16 values
      int buf = 0, pb = 0;
      lds_barrier();   // tile 0 is stored
      __builtin_amdgcn_s_setprio(1);
      for (int u = u0; u < u1; ++u) {
        f32x4 s[KB];
        const int k0 = buf + kat, k1 = k0 ^ 64;
        auto kfrag = [&](int f) -> bf16x8 {   // f = ks * KB + kb
          const int ks = f / KB, kb = f % KB;
          return *(const bf16x8 MLA_LDS*)(L + (ks & 1 ? k1 : k0) + (ks >> 1) * 1024 + kb * 2 * C::KBL);
        };
        constexpr int KD = 6;   // fragments in the ring, one of them in use
        bf16x8 ka[KD];
#pragma unroll
        for (int j = 0; j < KD - 1; ++j) ka[j] = kfrag(j);
        float met = m_run;      // the largest reference that the waves of these head-rows left
        if (C::KW > 1 && u > u0)
#pragma unroll
          for (int k = 0; k < C::KW; ++k) met = fmaxf(met, *(const float MLA_LDS*)(L + C::M_OFF + (((pb ^ 1) * C::KW + k) * BM + row) * 4));
        __builtin_amdgcn_sched_barrier(0);
        // the RoPE steps while the first latent fragments arrive
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
            s[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kr[kb][j & 1], j < 2 ? ql[j & 1] : qh[j & 1],
                                                            j == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[kb], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        const Tile now = t;
        if (u + 1 < u1) {
          t = cur.next(a);
          load_rope(t);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int f = 0; f < 16 * KB; ++f) {
          if (f + KD - 1 < 16 * KB) ka[(f + KD - 1) % KD] = kfrag(f + KD - 1);
          __builtin_amdgcn_sched_barrier(0);
          s[f % KB] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka[f % KD], qf[f / KB], s[f % KB], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
        // register i of s[kb]: key kb*16 + lg*4 + i of the wave's, head-row lc
        const int seen = seen_keys(now, t_row);
        if (__builtin_amdgcn_ballot_w64(seen < kCacheTile) != 0) {
          const int rel = seen - kw * KB * 16 - lg * 4;
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (kb * 16 + i >= rel) s[kb][i] = -INFINITY;
        }
        float m = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3]));
#pragma unroll
        for (int kb = 1; kb < KB; ++kb) m = fmaxf(m, fmaxf(fmaxf(s[kb][0], s[kb][1]), fmaxf(s[kb][2], s[kb][3])));
        m = quad_max(m) * a.scale_log2;
        if ((m > met + 8.f) | ((met == -INFINITY) & (m > -INFINITY))) met = ceilf(m);
        if (met != m_run) {
          const float al = __builtin_amdgcn_exp2f(m_run - met);
          l_run *= al;
          r_run *= al;
          m_run = met;
        }
        const float ref = m_run == -INFINITY ? 0.f : m_run;   // nothing seen yet: every weight is 0
        if (lg == 0) *(float MLA_LDS*)(L + C::M_OFF + ((pb * C::KW + kw) * BM + row) * 4) = m_run;
        // From 2^23 on a rounded product of score and scale, as the reference is one, is off by more
        // than half a unit: against the product as it is, weights would pass 2^9 and then the
        // range.  There the products are rounded like the reference.
        float scale = a.scale_log2;
        if (fabsf(ref) >= 8388608.f) {
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[kb][i] *= scale;
          scale = 1.f;
        }
        float l = 0.f, r = 0.f;
        u32x2 b[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
          float w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][i], scale, -ref));
          l += (w[0] + w[1]) + (w[2] + w[3]);
          b[kb] = u32x2{pack_bf16x2(w[0], w[1]), pack_bf16x2(w[2], w[3])};
          r += (bf16_lo(b[kb][0]) + bf16_hi(b[kb][0])) + (bf16_lo(b[kb][1]) + bf16_hi(b[kb][1]));
        }
        // key blocks 2 k2 and 2 k2 + 1 of the tile: a lane's eight keys of a fragment
        unsigned char MLA_LDS* at = L + C::P_OFF + pb * C::P_BYTES + rw * 1024 + lane * 16;
        if constexpr (KB == 1) {
          *(u32x2 MLA_LDS*)(at + (kw >> 1) * NB * 1024 + (kw & 1) * 8) = b[0];
        } else {
#pragma unroll
          for (int k = 0; k < KB / 2; ++k)
            *(u32x4 MLA_LDS*)(at + (kw * KB / 2 + k) * NB * 1024) = u32x4{b[2 * k][0], b[2 * k][1], b[2 * k + 1][0], b[2 * k + 1][1]};
        }
        l_run += l;
        r_run += r;
        if (t.frame != now.frame) {
          const unsigned char* q0 = qb + (uint32_t)((row < q_last ? row : q_last) * 1152 + 1024 + lg * 16);
          qraw[0] = *(const bf16x8*)q0;
          qraw[1] = *(const bf16x8*)(q0 + 64);
          relocate(t.frame);
        }
        buf ^= C::LAT;
        pb ^= 1;
        if (u + 1 == u1) {
          l = quad_sum(l_run);
          r = quad_sum(r_run);
          if (lg == 0) *(f32x2 MLA_LDS*)(L + C::L_OFF + (kw * BM + row) * 8) = f32x2{l, r};
        }
        lds_barrier();   // step u - u0 of the score waves
      }
      __builtin_amdgcn_s_setprio(0);
      lds_barrier();
    } else {
      // ------------------------------------------------------------------ value wave
      // Dims 512 / VW w .. of every head-row; it also converts its dims of the tiles: once
      // it has read them as the value of tile u, tile u + 2 may take their place, since the
      // score waves took tile u in the step before.
      const int w = wave - 4;
      const int lane = lane_now(), lg = lane >> 4, lc = lane & 15;
      // codes of key (64 / GW) i + lane / GW, group GW w + lane % GW
      const int key = lane / GW, grp = lane % GW;
      struct Codes {
        u32x4 c[NI];
        uint32_t s[NI];
      };
      auto load_codes = [&](Codes& x, const Tile& t) {
        const unsigned char* p = a.cache + (int64_t)t.page * a.page_rows * kCacheRow;
        const uint32_t row = (uint32_t)(t.off + key), g = (uint32_t)(GW * w + grp);
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          x.c[i] = *(const u32x4*)(p + row * kCacheCodes + g * 16 + i * (64 / GW) * kCacheCodes);
          x.s[i] = (p + plane_s)[row * kCacheScales + g + i * (64 / GW) * kCacheScales];
        }
      };
      const int sat = (key >> 3) * C::KBL + (key & 7) * 128 + (GW * w + grp) / 2 * 1024 +
                      (((grp & 1) * 4) ^ (grp >> 1) ^ key_swz(key & 7)) * 16;
      auto clear = [&](Codes& x, int seen) {   // keys that no row sees: zeros
        if (seen < kCacheTile)
#pragma unroll
          for (int i = 0; i < NI; ++i)
            if (i * (64 / GW) + key >= seen) {
              x.c[i] = u32x4{0, 0, 0, 0};
              x.s[i] = 127;
            }
      };
      // Chunk j of a group; lanes of the upper groups take neighbours
      // swapped, so that a store meets all banks.  With a key's first chunk its byte turns into
      // the scale in place: kept in both forms, one is a copy that waits for its load (231 us
      // where 205 are, 64 requests of 16k).
      auto store_chunk = [&](Codes& x, int buf, int i, int j) {
        const uint32_t c = grp >> 1 ? x.c[i][j ^ 1] : x.c[i][j];
        if (j == 0) x.s[i] = __float_as_uint(mx4_scale(x.s[i]));
        *(bf16x8 MLA_LDS*)(L + ((buf + sat) ^ (j * 16)) + i * (8 / GW) * C::KBL) = mx4_values(c, __uint_as_float(x.s[i]));
      };
      auto store_keys = [&](Codes& x, int buf, int i0) {
#pragma unroll
        for (int i = i0; i < NI; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) store_chunk(x, buf, i, j);
      };
      // A weight of 0 times a value that is NaN or infinite (from scale byte 253 on one may be)
      // would be NaN in rows that do not see its key: once the scores are taken, such values
      // become 0.  Rows that see the key have its NaN or infinity from the score.
      auto has_odd = [&](const Codes& x) {   // of the lane's keys
        uint32_t top = x.s[0];
#pragma unroll
        for (int i = 1; i < NI; ++i) top = top > x.s[i] ? top : x.s[i];
        return top >= __float_as_uint(mx4_scale(253));
      };
      auto drop_odd = [&](int buf) {
#pragma unroll 1
        for (int i = 0; i < NI; ++i)
#pragma unroll 1
          for (int j = 0; j < 4; ++j) {
            u32x4 MLA_LDS* at = (u32x4 MLA_LDS*)(L + ((buf + sat) ^ (j * 16)) + i * (8 / GW) * C::KBL);
            u32x4 v = *at;
#pragma unroll
            for (int c = 0; c < 4; ++c)
              v[c] &= ((v[c] & 0x7f80u) == 0x7f80u ? 0u : 0xffffu) | ((v[c] & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u);
            *at = v;
          }
        asm volatile("" ::: "memory");
      };
      Tile t = cur.next(a);
      Codes next{};
      int odd = 0;             // bit 0: the tile to multiply holds such values, bit 1: the one behind it
      int t_max = INT32_MIN;   // the last position of the block's rows
      {
        Codes first;
        const Tile t0 = t;
        load_codes(first, t);
        if (u0 + 1 < u1) {
          t = cur.next(a);
          load_codes(next, t);
        }
        {
          const int last = (hb + 1) * BM < R ? (hb + 1) * BM : R;
          for (int j = hb * BM / a.n_heads; j <= (last - 1) / a.n_heads; ++j) {
            const int t = __builtin_amdgcn_readfirstlane(tseq[j]);
            t_max = t > t_max ? t : t_max;
          }
        }
        lds_barrier();   // the queries have landed
        clear(first, seen_keys(t0, t_max));
        store_keys(first, 0, 0);
        odd = has_odd(first) ? 1 : 0;
        lds_barrier();   // tile 0 is stored; the queries have left the second tile's place
        if (u0 + 1 < u1) {
          clear(next, seen_keys(t, t_max));
          store_keys(next, C::LAT, 0);
          odd |= has_odd(next) ? 2 : 0;
        }
      }
      if (u0 + 2 < u1) {
        t = cur.next(a);
        load_codes(next, t);
      }
      f32x4 o[ND][NB];
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int h = 0; h < NB; ++h) o[d][h] = f32x4{0.f, 0.f, 0.f, 0.f};
      // V^T fragments (A operand, 16 dims x 32 keys) by transposing reads (see attend_pair.hip)
      const int vkey = (lg & 1) * 4 + (lc >> 2), vcb = lc & 3;
      const int vat = (lg >> 1) * C::KBL + vkey * 128 + (((vcb >> 1) ^ key_swz(vkey)) * 16) + (vcb & 1) * 8 + w * ND * 256;
      float mc[NB];   // reference of the sums, head-row lc
#pragma unroll
      for (int h = 0; h < NB; ++h) mc[h] = -INFINITY;
      int buf = 0, pb = 0;
      lds_barrier();   // the weights of tile 0 are written, tile 1 is stored
      for (int u = u0; u < u1; ++u) {
        auto vfrag = [&](int f) -> bf16x8 {   // f = k2 * ND + d
          const unsigned char MLA_LDS* vp = L + ((buf + vat) ^ ((f & 3) * 32)) + (f % ND) / 4 * 1024 + f / ND * 4 * C::KBL;
          const bf16x4 vl = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((MLA_LDS bf16x4*)vp);
          const bf16x4 vh = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((MLA_LDS bf16x4*)(vp + 2 * C::KBL));
          return __builtin_shufflevector(vl, vh, 0, 1, 2, 3, 4, 5, 6, 7);
        };
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(odd & 1) != 0, 0)) drop_odd(buf);
        constexpr int VD = 3;
        bf16x8 vt[VD], p[2][NB];
        float mk[C::KW][NB];
#pragma unroll
        for (int k = 0; k < C::KW; ++k)
#pragma unroll
          for (int h = 0; h < NB; ++h) mk[k][h] = *(const float MLA_LDS*)(L + C::M_OFF + ((pb * C::KW + k) * BM + h * 16 + lc) * 4);
#pragma unroll
        for (int h = 0; h < NB; ++h) p[0][h] = *(const bf16x8 MLA_LDS*)(L + C::P_OFF + pb * C::P_BYTES + h * 1024 + lane * 16);
#pragma unroll
        for (int j = 0; j < VD - 1; ++j) vt[j] = vfrag(j);
#pragma unroll
        for (int h = 0; h < NB; ++h) p[1][h] = *(const bf16x8 MLA_LDS*)(L + C::P_OFF + pb * C::P_BYTES + (NB + h) * 1024 + lane * 16);
        // Where the references differ, all move to the largest: they are whole numbers, so the
        // weights change by a power of two and stay exact.
        bool moved = false;
#pragma unroll
        for (int k = 0; k < C::KW; ++k)
#pragma unroll
          for (int h = 0; h < NB; ++h) moved |= mk[k][h] != mc[h];
        if (__builtin_amdgcn_ballot_w64(moved) != 0) {
#pragma unroll
          for (int h = 0; h < NB; ++h) {
            float top = mc[h];
#pragma unroll
            for (int k = 0; k < C::KW; ++k) top = fmaxf(top, mk[k][h]);
            const float ref = top == -INFINITY ? 0.f : top;
            const float al = __builtin_amdgcn_exp2f(mc[h] - ref);
            mc[h] = top;
#pragma unroll
            for (int d = 0; d < ND; ++d) o[d][h] *= al;
#pragma unroll
            for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
              for (int i = 0; i < 8; ++i)
                p[k2][h][i] = (__bf16)((float)p[k2][h][i] * __builtin_amdgcn_exp2f(mk[(k2 * 2 + i / 4) * C::KW / 4][h] - ref));
          }
        }
        clear(next, seen_keys(t, t_max));
        __builtin_amdgcn_s_setprio(2);   // the longer way: 85 us where the scores alone come first takes 86 (16 requests, 256 head-rows)
        auto values = [&](int f) {
          if (f + VD - 1 < 2 * ND) vt[(f + VD - 1) % VD] = vfrag(f + VD - 1);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int h = 0; h < NB; ++h)
            o[f % ND][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt[f % VD], p[f / ND][h], o[f % ND][h], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        };
        // keys 0 .. 31 of tile u + 2 take the place of those just multiplied while the others are
        // (behind the last tile, codes that nobody reads)
#pragma unroll
        for (int f = 0; f < 2 * ND; ++f) {
          values(f);
          if (f >= ND) store_chunk(next, buf, (f - ND) / 4, f % 4);
        }
        __builtin_amdgcn_s_setprio(0);
        odd >>= 1;
        if (u + 2 < u1) {
          store_keys(next, buf, NI / 2);
          odd |= has_odd(next) ? 2 : 0;
        }
        if (u + 3 < u1) {
          t = cur.next(a);
          load_codes(next, t);
        }
        buf ^= C::LAT;
        pb ^= 1;
        lds_barrier();   // step u - u0 of the value waves; after the last one the sums are written
      }
      const bool whole = u0 == 0 && u1 == n;
      const int slot = seq_base <= lo ? 2 * share : 2 * share + 1;
#pragma unroll
      for (int h = 0; h < NB; ++h) {
        float l = 0.f, r = 0.f;
#pragma unroll
        for (int k = 0; k < C::KW; ++k) {
          const int at = k * BM + h * 16 + lc;
          const float mk = *(const float MLA_LDS*)(L + C::M_OFF + ((pb ^ 1) * C::KW * BM + at) * 4);
          const f32x2 lr = *(const f32x2 MLA_LDS*)(L + C::L_OFF + at * 8);
          const float al = mk == mc[h] ? 1.f : __builtin_amdgcn_exp2f(mk - mc[h]);
          l += lr[0] * al;   // a NaN stays
          r += lr[1] * al;
        }
        const float m = mc[h];
        const int row = hb * BM + h * 16 + lc;
        if (whole) {
          // Through LDS, in which no tile is read any more, to rows: stored as they lie, sixteen
          // head-rows a store, they would keep the address unit four times as long.
          constexpr int RS = ND * 32 + 16, CR = ND * 2;   // a row's bytes there; its 16-byte chunks
          unsigned char MLA_LDS* own = L + w * 16 * RS;
          const float inv = r == 0.f ? 0.f : 1.f / r;
#pragma unroll
          for (int d = 0; d < ND; ++d)
            *(u32x2 MLA_LDS*)(own + lc * RS + d * 32 + lg * 8) =
                u32x2{pack_bf16x2(o[d][h][0] * inv, o[d][h][1] * inv), pack_bf16x2(o[d][h][2] * inv, o[d][h][3] * inv)};
#pragma unroll
          for (int i = 0; i < CR / 4; ++i) {
            const int rr = i * (64 / CR) + lane / CR, at_row = hb * BM + h * 16 + rr;
            const u32x4 v = *(const u32x4 MLA_LDS*)(own + rr * RS + lane % CR * 16);
            if (at_row < R) *(u32x4*)(a.out_o + ((int64_t)b * R + at_row) * 512 + w * ND * 16 + lane % CR * 8) = v;
          }
          if (w == 0 && lg == 0 && a.out_lse != nullptr && row < R)
            a.out_lse[(int64_t)b * R + row] = l == 0.f ? -INFINITY : (m + __log2f(l)) * 0.6931471805599453f;
        } else {
          // fragments as they lie in the registers: a kilobyte a store
          const int64_t at = (((int64_t)slot * a.n_blocks + hb) * NB + h) * 16;
#pragma unroll
          for (int d = 0; d < ND; ++d) *(f32x4*)(a.part_o + at * 512 + (w * ND + d) * 256 + lane * 4) = o[d][h];
          if (w == 0 && lg == 0) {
            *(f32x4*)(a.part_ml + (at + lc) * 4) = f32x4{m, l, r, 0.f};
          }
        }
      }
    }
    if (base >= hi) return;
    for (;;) {
      const uint64_t with = __builtin_amdgcn_ballot_w64(next_tiles > 0 && held + lane > b);
      if (with != 0) {
        const int at = __builtin_ctzll(with);
        b = held + at;
        n = __builtin_amdgcn_readlane(next_tiles, at);
        break;
      }
      held += 64;
      if (held >= a.n_seqs) return;
      next_tiles = tiles_from(held);
    }
  }
}

template <int kFrags>
using Joined = f32x4[kFrags + 1][64];   // a wave's sums in LDS

// Joins the sums of requests that several shares hold (and writes those without a tile).  A
// unit is 16 head-rows and 16 kFrags dims, the fragments that the sums are kept in; a wave
// takes every G-th share of it, and G waves of a workgroup join their sums through LDS.
// Requests of more than `most` shares are left out.
template <int G, int kFrags>
__device__ __forceinline__ void join_unit(const CacheAttendArgs& a, int b, int unit, int most, Joined<kFrags>* acc) {
  const int R = a.n_q * a.n_heads;
  const int lane = threadIdx.x & 63, lg = lane >> 4, lc = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), sub = wave % G;
  const int group = unit / (32 / kFrags), frag = unit % (32 / kFrags) * kFrags;   // 16 head-rows; first fragment
  const int base = a.tile_base[b], n = a.tile_base[b + 1] - base;
  const int row = group * 16 + lc;
  const int64_t at = (int64_t)b * R + row;
  if (row - lc >= R) return;
  f32x4 o[kFrags];
#pragma unroll
  for (int f = 0; f < kFrags; ++f) o[f] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f, r = 0.f;
  if (n > 0) {
    const Runs runs(a, a.tile_base[a.n_seqs]);
    const int s0 = runs.share(base), s1 = runs.share(base + n - 1);
    if (s0 == s1 || s1 - s0 >= most) return;
    // share s's sums: its first request's or, where another request ends in it, its last one's
    const int first_slot = base <= runs.first(s0) ? 2 * s0 : 2 * s0 + 1;
    const int nb = a.block / 16, block = group / nb, in_block = group - block * nb;
    constexpr int kAhead = 8 / kFrags;
    for (int s = s0 + sub; s <= s1; s += kAhead * G) {
      f32x4 v[kAhead][kFrags];
      f32x4 ml[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {   // past the end the last one again, not used
        const int sj = s + j * G <= s1 ? s + j * G : s1;
        const int64_t from = (((int64_t)(sj == s0 ? first_slot : 2 * sj) * a.n_blocks + block) * nb + in_block) * 16;
        ml[j] = *(const f32x4*)(a.part_ml + (from + lc) * 4);
#pragma unroll
        for (int f = 0; f < kFrags; ++f) v[j][f] = *(const f32x4*)(a.part_o + from * 512 + (frag + f) * 256 + lane * 4);
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        if (s + j * G > s1) break;
        const float top = fmaxf(m, ml[j][0]), ref = top == -INFINITY ? 0.f : top;
        const float x = __builtin_amdgcn_exp2f(m - ref), y = __builtin_amdgcn_exp2f(ml[j][0] - ref);
        m = top;
        l = l * x + ml[j][1] * y;
        r = r * x + ml[j][2] * y;
#pragma unroll
        for (int f = 0; f < kFrags; ++f) o[f] = o[f] * x + v[j][f] * y;
      }
    }
    if constexpr (G > 1) {
      static_assert(G == 1 || G == kWaves, "the waves of a unit are a workgroup");
#pragma unroll
      for (int f = 0; f < kFrags; ++f) acc[wave][f][lane] = o[f];
      acc[wave][kFrags][lane] = f32x4{m, l, r, 0.f};
      __syncthreads();
      if (wave != 0) return;
#pragma unroll
      for (int w = 1; w < kWaves; ++w) {
        const f32x4 x4 = acc[w][kFrags][lane];
        const float top = fmaxf(m, x4[0]), ref = top == -INFINITY ? 0.f : top;
        const float x = __builtin_amdgcn_exp2f(m - ref), y = __builtin_amdgcn_exp2f(x4[0] - ref);
        m = top;
        l = l * x + x4[1] * y;
        r = r * x + x4[2] * y;
#pragma unroll
        for (int f = 0; f < kFrags; ++f) o[f] = o[f] * x + acc[w][f][lane] * y;
      }
    }
  } else if (sub != 0) {
    return;
  }
  if (row >= R) return;
  const float inv = r == 0.f ? 0.f : 1.f / r;
#pragma unroll
  for (int f = 0; f < kFrags; ++f)
    *(u32x2*)(a.out_o + at * 512 + (frag + f) * 16 + lg * 4) =
        u32x2{pack_bf16x2(o[f][0] * inv, o[f][1] * inv), pack_bf16x2(o[f][2] * inv, o[f][3] * inv)};
  if (frag == 0 && lg == 0 && a.out_lse != nullptr)
    a.out_lse[at] = l == 0.f ? -INFINITY : (m + __log2f(l)) * 0.6931471805599453f;
}

// All waves of a workgroup on one unit
template <int kFrags>
__global__ __launch_bounds__(kThreads) void cache_merge_kernel(CacheAttendArgs a) {
  __shared__ __attribute__((aligned(16))) Joined<kFrags> acc[kWaves];
  join_unit<kWaves, kFrags>(a, blockIdx.y, blockIdx.x, INT32_MAX, acc);
}

// A row of workgroups a request, a wave a unit of it, for requests of up to `most` shares; in
// the rows behind, all waves of a workgroup on a unit of a longer one, of which there is one at
// most for every kLong-th share (the attention's kernel says which).
constexpr int kMixFrags = 2, kMixUnits = 32 / kMixFrags;   // units of 16 head-rows
__global__ __launch_bounds__(kThreads) void cache_merge_mixed_kernel(CacheAttendArgs a, int most) {
  __shared__ __attribute__((aligned(16))) Joined<kMixFrags> acc[kWaves];
  if ((int)blockIdx.y < a.n_seqs) {
    join_unit<1, kMixFrags>(a, blockIdx.y, blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), most, acc);
    return;
  }
  const int units = gridDim.x * kWaves, at = ((int)blockIdx.y - a.n_seqs) * gridDim.x + blockIdx.x, k = at / units;
  if (k * kLong >= a.shares) return;
  const int b = __builtin_amdgcn_readfirstlane(a.long_seq[k]);
  if (b >= 0) join_unit<kWaves, kMixFrags>(a, b, at % units, INT32_MAX, acc);
}

}  // namespace

hipError_t launch_cache_attend(const CacheAttendArgs& a, hipStream_t s) {
  const unsigned grid = 8u * (unsigned)((a.shares * a.n_blocks + 7) / 8);
  if (a.block == 16)
    cache_attend_kernel<1><<<dim3(grid), dim3(CaCfg<1>::THREADS), 0, s>>>(a);
  else if (a.block == 32)
    cache_attend_kernel<2><<<dim3(grid), dim3(CaCfg<2>::THREADS), 0, s>>>(a);
  else
    cache_attend_kernel<4><<<dim3(grid), dim3(CaCfg<4>::THREADS), 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const unsigned groups = (unsigned)(a.n_q * a.n_heads + 15) / 16, n_seqs = (unsigned)a.n_seqs;
  // A wave a unit where it holds all shares of a request in flight at once, else eight (64
  // requests of 4 shares each: 201 against 211 us for the whole call; 48 of 5.3 shares: 43.4
  // against 42.3; one of 256 shares: 151 against 64).  How the shares fall to the requests is
  // known on the device alone: with up to four on average, rows of workgroups behind the
  // requests' take those of more than kLong (one of 264k keys among 63 of 400 keys: 87 us, 166
  // with a wave a unit; with kLong 8 and 16 it is the same within a twentieth, and more
  // workgroups find no work in other batches).  Where the grid holds no row more, a wave a unit.
  // Of half the dims where the units are fewer than the compute units (one of 256 shares: 63.3
  // against 64.4).
  if (a.shares <= 4 * a.n_seqs) {
    const unsigned rows = a.shares > kLong ? (unsigned)(a.shares + kLong - 1) / kLong * kWaves : 0;
    const bool fits = n_seqs + rows <= 65535;
    cache_merge_mixed_kernel<<<dim3(groups * kMixUnits / kWaves, n_seqs + (fits ? rows : 0)), dim3(kThreads), 0, s>>>(a, fits ? kLong : INT32_MAX);
  } else if (groups * 16 * n_seqs >= 256) {
    cache_merge_kernel<2><<<dim3(groups * 16, n_seqs), dim3(kThreads), 0, s>>>(a);
  } else {
    cache_merge_kernel<1><<<dim3(groups * 32, n_seqs), dim3(kThreads), 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace mla

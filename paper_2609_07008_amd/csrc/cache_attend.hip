// Absorbed-MLA attention of new tokens over the paged 4-bit latent cache (mx4.h): the
// decode form of Alg. 2's SelectiveMLA, each page in its own RoPE frame (the query is
// turned by t - frame, eq:rope), 512 + 64 latent, the latent as the value.
//
// A request's head-rows (its n_q tokens' heads) share its keys.  A workgroup of eight
// waves takes up to 32 NBQ of them and a run of 64-key tiles:
//   tile      row-major codes come in through registers two tiles ahead, are converted once
//             (v_cvt_scalef32_pk_bf16_fp4) and laid into LDS as bf16 in the layout of the
//             online attention's tiles (attend_pair.hip): the key of the scores and, by
//             transposing reads, the value
//   scores    wave (kb, hh): 16 keys x 16 NBQ head-rows, S^T = K Q^T, queries in registers.
//             The turned RoPE part of the query goes in twice, as its bf16 value and the
//             bf16 of what that lost: the scores are then as exact as the products, which a
//             request of a few keys shows in its lse
//   softmax   the tile's maximum of each head-row crosses the four key waves through LDS;
//             the reference moves (and sums are rescaled) only when a tile exceeds it by
//             2^8, so weights stay below 2^8 and sums in 32 bits lose nothing
//   values    wave w: dims 64 w .. +63 of all head-rows, O^T += V^T P^T, weights in bf16
//             (half a step, 2^-9 of each, next to an output of the same width)
// A key that no row of the call sees (behind a page's rows, past the last position) is
// zero in LDS whatever the page holds there.
//
// Work is split by tiles, not by requests: the batch's tiles, in order, form `shares`
// equal runs, one a workgroup (and head-row block).  A request inside one run is written
// at once; one that crosses runs leaves sums to cache_merge_kernel.
#include "mx4.h"

#include <algorithm>

namespace mla {
namespace {

constexpr int kWaves = 8, kThreads = kWaves * 64;

template <int NB>
struct CaCfg {
  static constexpr int BM = 16 * NB;         // head-rows of a workgroup
  static constexpr int KBL = 8 * 1024 + 128; // latent of an 8-key block: a kilobyte per 64 dims
  static constexpr int LAT = 8 * KBL;        // a tile
  static constexpr int P_OFF = 2 * LAT;      // weights of two tiles: 2 x NB KB each in the layout of the MFMA operand
  static constexpr int P_BYTES = 2 * NB * 1024;
  static constexpr int AL_OFF = P_OFF + 2 * P_BYTES;   // [2][BM]: factors of the sums before the tile
  static constexpr int ML_OFF = AL_OFF + 2 * BM * 4;   // [BM][2]: reference and row sum at the end
  static constexpr int TH_OFF = ML_OFF + BM * 8;
  static constexpr int LDS = TH_OFF + kMaxRopePairs * 8;
  static_assert(LDS <= 160 * 1024, "LDS of a compute unit");
};

// slot of 16-byte chunk c of key k in its kilobyte: c ^ key_swz(k) (see attend_pair.hip)
__device__ __forceinline__ int key_swz(int k) { return k ^ ((~k & 1) << 2); }

// this wave's LDS accesses are done, then all waves meet (loads from memory stay in flight)
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

struct Tile {       // wave-uniform
  int page, off;    // page to read (0 where there is none), the tile's first row in it
  int rows;         // rows of the tile that hold keys, 0 .. 64
  int frame, pos0;  // RoPE frame, request position of the page's first row
};

// The tiles of a request from tile u on: entries are fetched one tile ahead.
struct Cursor {
  const mla_page* entries;
  int e, sub, e_last, tpp, word;   // entry and tile of it to describe next; its words in lanes 0 .. 3
  __device__ __forceinline__ void fetch() {
    if (e <= e_last) word = ((const int32_t*)(entries + e))[threadIdx.x & 3];
  }
  __device__ __forceinline__ void open(const CacheAttendArgs& a, int b, int u0, int u1, int tiles_per_page) {
    entries = a.pages + (int64_t)b * a.max_pages;
    tpp = tiles_per_page;
    e = u0 / tpp;
    sub = u0 - e * tpp;
    e_last = (u1 - 1) / tpp;
    word = 0;
    fetch();
  }
  __device__ __forceinline__ Tile next(const CacheAttendArgs& a) {
    Tile t;
    const int page = __builtin_amdgcn_readlane(word, 0), rows = __builtin_amdgcn_readlane(word, 1);
    const bool there = (unsigned)page < (unsigned)a.cache_pages;
    t.page = there ? page : 0;
    t.off = sub * kCacheTile;
    const int left = (there ? (rows < a.page_rows ? rows : a.page_rows) : 0) - t.off;
    t.rows = left < 0 ? 0 : left < kCacheTile ? left : kCacheTile;
    t.pos0 = __builtin_amdgcn_readlane(word, 2);
    t.frame = __builtin_amdgcn_readlane(word, 3);
    if (++sub == tpp) {
      sub = 0;
      ++e;
    }
    fetch();
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

__device__ __forceinline__ int tiles_of(const CacheAttendArgs& a, int b, int tpp) {
  int n = a.seq_pages[b];
  n = n < 0 ? 0 : n < a.max_pages ? n : a.max_pages;
  return n * tpp;
}

// The batch's tiles as `shares` runs in order: the first r of them a tile longer.
struct Runs {
  int q, r;
  __device__ __forceinline__ Runs(int total, int shares) : q(total / shares), r(total - total / shares * shares) {}
  __device__ __forceinline__ int first(int s) const { return q * s + (s < r ? s : r); }   // share s's first tile
  __device__ __forceinline__ int share(int tile) const {                                  // the share that holds it
    const int longer = r * (q + 1);
    return tile < longer ? tile / (q + 1) : r + (tile - longer) / q;
  }
};

template <int NB>
__global__ __launch_bounds__(kThreads, 2) void cache_attend_kernel(CacheAttendArgs a) {
  using C = CaCfg<NB>;
  constexpr int BM = C::BM;
  __shared__ __attribute__((aligned(16))) unsigned char lds[C::LDS];
  unsigned char MLA_LDS* L = (unsigned char MLA_LDS*)lds;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lg = lane >> 4, lc = lane & 15;
  const int tpp = a.page_rows / kCacheTile;
  const int R = a.n_q * a.n_heads;

  // workgroups go to the 8 XCDs round-robin: the blocks of a share follow each other on one
  const int kx = blockIdx.x >> 3;
  const int hb = kx % a.n_blocks;
  const int share = (kx / a.n_blocks) * 8 + (blockIdx.x & 7);
  if (share >= a.shares) return;

  // tiles before each request, by a scan over the batch; the request that holds the
  // share's first tile
  int first_b, first_base, total;
  {
    int MLA_LDS* sums = (int MLA_LDS*)L;
    const int per = (a.n_seqs + kThreads - 1) / kThreads;
    const int b0 = tid * per < a.n_seqs ? tid * per : a.n_seqs;
    const int b1 = b0 + per < a.n_seqs ? b0 + per : a.n_seqs;
    int mine = 0;
    for (int b = b0; b < b1; ++b) mine += tiles_of(a, b, tpp);
    int inc = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(inc, o, 64);
      if (lane >= o) inc += v;
    }
    if (lane == 63) sums[wave] = inc;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const int v = sums[w];
      before += w < wave ? v : 0;
      total += v;
    }
    int base = before + inc - mine;
    const int lo = Runs(total, a.shares).first(share);
    const bool writes = blockIdx.x == 0;
    for (int b = b0; b < b1; ++b) {
      const int n = tiles_of(a, b, tpp);
      if (writes) a.tile_base[b] = base;
      if (lo >= base && lo < base + n) {
        sums[16] = b;
        sums[17] = base;
      }
      base += n;
    }
    if (writes && tid == 0) a.tile_base[a.n_seqs] = total;
    __syncthreads();
    first_b = __builtin_amdgcn_readfirstlane(sums[16]);
    first_base = __builtin_amdgcn_readfirstlane(sums[17]);
    total = __builtin_amdgcn_readfirstlane(total);
  }
  const Runs runs(total, a.shares);
  const int lo = runs.first(share), hi = runs.first(share + 1);
  if (lo >= hi) return;

  double MLA_LDS* theta = (double MLA_LDS*)(L + C::TH_OFF);
  float MLA_LDS* ml = (float MLA_LDS*)(L + C::ML_OFF);
  const uint32_t plane_s = (uint32_t)a.page_rows * kCacheCodes, plane_r = plane_s + (uint32_t)a.page_rows * kCacheScales;
  if (tid < kMaxRopePairs) theta[tid] = a.rope.theta[tid];

  int b = first_b, base = first_base;
  for (; base < hi; ++b) {
    const int n = __builtin_amdgcn_readfirstlane(tiles_of(a, b, tpp));
    const int u0 = lo > base ? lo - base : 0, u1 = hi < base + n ? hi - base : n;
    const int seq_base = base;
    base += n;
    if (u0 >= u1) continue;
    Cursor cur;
    cur.open(a, b, u0, u1, tpp);
    const int32_t* tseq = a.pos + (int64_t)b * a.n_q;
    lds_barrier();   // the tables, and what the previous request left in LDS, are read
    if (wave < 4) {
      // ------------------------------------------------------------------ score wave
      // Head-row lc of block `wave`; rows past the end repeat the last one and are not stored.
      if (wave >= NB) {
        lds_barrier();
        for (int u = u0; u <= u1; ++u) lds_barrier();
        continue;
      }
      int hr = hb * BM + wave * 16 + lc;
      hr = hr < R ? hr : R - 1;
      const int t_row = tseq[hr / a.n_heads];
      const uint16_t* qrow = a.q + ((int64_t)b * R + hr) * 576;
      bf16x8 qf[16], qraw[2], qh[2], ql[2];   // Q fragments (B operand): dims ks*32 + lg*8 .. +7 of the head-row
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) qraw[ks] = *(const bf16x8*)(qrow + 512 + ks * 32 + lg * 8);
#pragma unroll
      for (int ks = 0; ks < 16; ++ks) qf[ks] = *(const bf16x8*)(qrow + ks * 32 + lg * 8);
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
      // RoPE keys as K fragments: key kb*16 + lc, chunks lg and lg + 4
      bf16x8 kr[4][2];
      auto load_rope = [&](const Tile& t) {
        const unsigned char* p = a.cache + (int64_t)t.page * a.page_rows * kCacheRow + plane_r;
        const uint32_t at = (uint32_t)(t.off + lc) * kCacheRope + (uint32_t)lg * 16;
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
          kr[kb][0] = *(const bf16x8*)(p + at + kb * 16 * kCacheRope);
          kr[kb][1] = *(const bf16x8*)(p + at + kb * 16 * kCacheRope + 64);
        }
      };
      // K fragments (A operand, 16 keys x 32 dims): key kb*16 + lc, chunk 4 ks + lg
      const int kat = (lc >> 3) * C::KBL + (lc & 7) * 128 + ((lg ^ key_swz(lc & 7)) * 16);
      Tile t = cur.next(a);
      load_rope(t);
      relocate(t.frame);
      float m_run = -INFINITY, l_run = 0.f;
      int buf = 0, pb = 0;
      lds_barrier();   // tiles 0 and 1 are stored
      __builtin_amdgcn_s_setprio(1);
      for (int u = u0; u < u1; ++u) {
        f32x4 s[4];
        const int k0 = buf + kat, k1 = k0 ^ 64;
        auto kfrag = [&](int f) -> bf16x8 {   // f = ks * 4 + kb
          const int ks = f >> 2, kb = f & 3;
          return *(const bf16x8 MLA_LDS*)(L + (ks & 1 ? k1 : k0) + (ks >> 1) * 1024 + kb * 2 * C::KBL);
        };
        constexpr int KD = 6;   // fragments in the ring, one of them in use
        bf16x8 ka[KD];
#pragma unroll
        for (int j = 0; j < KD - 1; ++j) ka[j] = kfrag(j);
        __builtin_amdgcn_sched_barrier(0);
        // the RoPE steps while the first latent fragments arrive
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) s[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kr[kb][0], ql[0], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) s[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kr[kb][1], ql[1], s[kb], 0, 0, 0);
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) s[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kr[kb][0], qh[0], s[kb], 0, 0, 0);
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) s[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kr[kb][1], qh[1], s[kb], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        const Tile now = t;
        if (u + 1 < u1) {
          t = cur.next(a);
          load_rope(t);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int f = 0; f < 64; ++f) {
          if (f + KD - 1 < 64) ka[(f + KD - 1) % KD] = kfrag(f + KD - 1);
          __builtin_amdgcn_sched_barrier(0);
          s[f & 3] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka[f % KD], qf[f >> 2], s[f & 3], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
        // register i of s[kb]: key kb*16 + lg*4 + i, head-row lc
        const int rel = seen_keys(now, t_row) - lg * 4;
        if (__builtin_amdgcn_ballot_w64(rel + lg * 4 < kCacheTile) != 0) {
#pragma unroll
          for (int kb = 0; kb < 4; ++kb)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (kb * 16 + i >= rel) s[kb][i] = -INFINITY;
        }
        float m = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3]));
#pragma unroll
        for (int kb = 1; kb < 4; ++kb) m = fmaxf(m, fmaxf(fmaxf(s[kb][0], s[kb][1]), fmaxf(s[kb][2], s[kb][3])));
        m = quad_max(m) * a.scale_log2;
        float al = 1.f;
        if ((m > m_run + 8.f) | ((m_run == -INFINITY) & (m > -INFINITY))) {
          al = __builtin_amdgcn_exp2f(m_run - m);
          m_run = m;
        }
        const float ref = m_run == -INFINITY ? 0.f : m_run;   // nothing seen yet: every weight is 0
        float w[4][4];
#pragma unroll
        for (int kb = 0; kb < 4; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i) w[kb][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][i], a.scale_log2, -ref));
#pragma unroll
        for (int k2 = 0; k2 < 2; ++k2)
          *(u32x4 MLA_LDS*)(L + C::P_OFF + pb * C::P_BYTES + (k2 * NB + wave) * 1024 + lane * 16) =
              u32x4{pack_bf16x2(w[2 * k2][0], w[2 * k2][1]), pack_bf16x2(w[2 * k2][2], w[2 * k2][3]),
                    pack_bf16x2(w[2 * k2 + 1][0], w[2 * k2 + 1][1]), pack_bf16x2(w[2 * k2 + 1][2], w[2 * k2 + 1][3])};
        if (lg == 0) *(float MLA_LDS*)(L + C::AL_OFF + (pb * BM + wave * 16 + lc) * 4) = al;
        float l = 0.f;
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) l += (w[kb][0] + w[kb][1]) + (w[kb][2] + w[kb][3]);
        l_run = l_run * al + l;
        if (t.frame != now.frame) relocate(t.frame);
        buf ^= C::LAT;
        pb ^= 1;
        lds_barrier();   // step u - u0 of the score waves
      }
      __builtin_amdgcn_s_setprio(0);
      const float l = quad_sum(l_run);
      if (lg == 0) {
        ml[(wave * 16 + lc) * 2] = m_run;
        ml[(wave * 16 + lc) * 2 + 1] = l;
      }
      lds_barrier();
    } else {
      // ------------------------------------------------------------------ value wave
      // Dims 128 w .. +127 of every head-row; it also converts its dims of the tiles: once
      // it has read them as the value of tile u, tile u + 2 may take their place, since the
      // score waves took tile u in the step before.
      const int w = wave - 4;
      int t_max = INT32_MIN;
      {
        const int last = (hb + 1) * BM < R ? (hb + 1) * BM : R;
        for (int j = hb * BM / a.n_heads; j <= (last - 1) / a.n_heads; ++j) {
          const int t = __builtin_amdgcn_readfirstlane(tseq[j]);
          t_max = t > t_max ? t : t_max;
        }
      }
      // codes of 16 i + lane / 4, group 4 w + lane % 4
      const int key = lane >> 2, grp = lane & 3;
      u32x4 cw[4];
      uint32_t sc[4];
      auto load_codes = [&](const Tile& t) {
        const unsigned char* p = a.cache + (int64_t)t.page * a.page_rows * kCacheRow;
        const uint32_t row = (uint32_t)(t.off + key), g = (uint32_t)(4 * w + grp);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          cw[i] = *(const u32x4*)(p + row * kCacheCodes + g * 16 + i * 16 * kCacheCodes);
          sc[i] = (p + plane_s)[row * kCacheScales + g + i * 16 * kCacheScales];
        }
      };
      const int sat = (key >> 3) * C::KBL + (key & 7) * 128 + (2 * w + (grp >> 1)) * 1024 +
                      (((grp & 1) * 4) ^ (grp >> 1) ^ key_swz(key & 7)) * 16;
      auto store_tile = [&](int buf, int seen) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (seen < kCacheTile && i * 16 + key >= seen) {   // a key that no row sees: zeros
            cw[i] = u32x4{0, 0, 0, 0};
            sc[i] = 127;
          }
          const float s = mx4_scale(sc[i]);
          // the four chunks of a group; lanes of the upper groups take neighbours swapped, so
          // that a store meets all banks
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t c = grp >> 1 ? cw[i][j ^ 1] : cw[i][j];
            *(bf16x8 MLA_LDS*)(L + ((buf + sat) ^ (j * 16)) + i * 2 * C::KBL) = mx4_values(c, s);
          }
        }
      };
      Tile t = cur.next(a);
      load_codes(t);
      store_tile(0, seen_keys(t, t_max));
      if (u0 + 1 < u1) {
        t = cur.next(a);
        load_codes(t);
        store_tile(C::LAT, seen_keys(t, t_max));
      }
      if (u0 + 2 < u1) {
        t = cur.next(a);
        load_codes(t);
      }
      f32x4 o[8][NB];
#pragma unroll
      for (int d = 0; d < 8; ++d)
#pragma unroll
        for (int h = 0; h < NB; ++h) o[d][h] = f32x4{0.f, 0.f, 0.f, 0.f};
      // V^T fragments (A operand, 16 dims x 32 keys) by transposing reads (see attend_pair.hip)
      const int vkey = (lg & 1) * 4 + (lc >> 2), vcb = lc & 3;
      const int vat = (lg >> 1) * C::KBL + vkey * 128 + (((vcb >> 1) ^ key_swz(vkey)) * 16) + (vcb & 1) * 8 + w * 2048;
      int buf = 0, pb = 0;
      lds_barrier();   // tiles 0 and 1 are stored
      lds_barrier();   // the weights of tile 0 are written
      for (int u = u0; u < u1; ++u) {
        auto vfrag = [&](int f) -> bf16x8 {   // f = k2 * 8 + d
          const unsigned char MLA_LDS* vp = L + ((buf + vat) ^ ((f & 3) * 32)) + ((f >> 2) & 1) * 1024 + (f >> 3) * 4 * C::KBL;
          const bf16x4 vl = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((MLA_LDS bf16x4*)vp);
          const bf16x4 vh = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((MLA_LDS bf16x4*)(vp + 2 * C::KBL));
          return __builtin_shufflevector(vl, vh, 0, 1, 2, 3, 4, 5, 6, 7);
        };
        constexpr int VD = 3;
        bf16x8 vt[VD], p[2][NB];
        float al[NB];
#pragma unroll
        for (int h = 0; h < NB; ++h) al[h] = *(const float MLA_LDS*)(L + C::AL_OFF + (pb * BM + h * 16 + lc) * 4);
#pragma unroll
        for (int h = 0; h < NB; ++h) p[0][h] = *(const bf16x8 MLA_LDS*)(L + C::P_OFF + pb * C::P_BYTES + h * 1024 + lane * 16);
#pragma unroll
        for (int j = 0; j < VD - 1; ++j) vt[j] = vfrag(j);
#pragma unroll
        for (int h = 0; h < NB; ++h) p[1][h] = *(const bf16x8 MLA_LDS*)(L + C::P_OFF + pb * C::P_BYTES + (NB + h) * 1024 + lane * 16);
        bool moved = false;
#pragma unroll
        for (int h = 0; h < NB; ++h) moved |= al[h] != 1.f;
        if (__builtin_amdgcn_ballot_w64(moved) != 0) {
#pragma unroll
          for (int h = 0; h < NB; ++h)
#pragma unroll
            for (int d = 0; d < 8; ++d) o[d][h] *= al[h];
        }
#pragma unroll
        for (int f = 0; f < 16; ++f) {
          if (f + VD - 1 < 16) vt[(f + VD - 1) % VD] = vfrag(f + VD - 1);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int h = 0; h < NB; ++h)
            o[f & 7][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt[f % VD], p[f >> 3][h], o[f & 7][h], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
        if (u + 2 < u1) {
          store_tile(buf, seen_keys(t, t_max));
          if (u + 3 < u1) {
            t = cur.next(a);
            load_codes(t);
          }
        }
        buf ^= C::LAT;
        pb ^= 1;
        lds_barrier();   // step u - u0 of the value waves; after the last one the sums are written
      }
      const bool whole = u0 == 0 && u1 == n;
      const int slot = seq_base <= lo ? 2 * share : 2 * share + 1;
#pragma unroll
      for (int h = 0; h < NB; ++h) {
        const float m = ml[(h * 16 + lc) * 2], l = ml[(h * 16 + lc) * 2 + 1];
        const int row = hb * BM + h * 16 + lc;
        if (row >= R) continue;
        if (whole) {
          const int64_t at = (int64_t)b * R + row;
          const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
          for (int d = 0; d < 8; ++d)
            *(u32x2*)(a.out_o + at * 512 + w * 128 + d * 16 + lg * 4) =
                u32x2{pack_bf16x2(o[d][h][0] * inv, o[d][h][1] * inv), pack_bf16x2(o[d][h][2] * inv, o[d][h][3] * inv)};
          if (w == 0 && lg == 0 && a.out_lse != nullptr)
            a.out_lse[at] = l == 0.f ? -INFINITY : (m + __log2f(l)) * 0.6931471805599453f;
        } else {
          const int64_t at = ((int64_t)slot * a.n_blocks + hb) * BM + h * 16 + lc;
#pragma unroll
          for (int d = 0; d < 8; ++d) *(f32x4*)(a.part_o + at * 512 + w * 128 + d * 16 + lg * 4) = o[d][h];
          if (w == 0 && lg == 0) {
            a.part_ml[at * 2] = m;
            a.part_ml[at * 2 + 1] = l;
          }
        }
      }
    }
  }
}

// Joins the sums of requests that several shares hold (and writes those without a tile):
// G waves take a head-row, eight dims a lane, and its shares in turn.  Bound by the
// latency of three dependent reads, then by the sums themselves (2 KB a share and head-row).
template <int G>
__global__ __launch_bounds__(kThreads) void cache_merge_kernel(CacheAttendArgs a) {
  __shared__ __attribute__((aligned(16))) float acc[G == 1 ? 1 : kWaves][512];
  const int R = a.n_q * a.n_heads;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int b = blockIdx.y, row = blockIdx.x * (kWaves / G) + wave / G, sub = wave % G;
  if (row >= R) return;   // whole workgroups where waves share a head-row
  const int base = a.tile_base[b], n = a.tile_base[b + 1] - base;
  const int64_t at = (int64_t)b * R + row;
  if (n == 0) {
    if (sub != 0) return;
    *(u32x4*)(a.out_o + at * 512 + lane * 8) = u32x4{0, 0, 0, 0};
    if (lane == 0 && a.out_lse != nullptr) a.out_lse[at] = -INFINITY;
    return;
  }
  const Runs runs(a.tile_base[a.n_seqs], a.shares);
  const int s0 = runs.share(base), s1 = runs.share(base + n - 1);
  if (s0 == s1) return;
  const int block = row / a.block, in_block = row - block * a.block;
  // share s's sums: its first request's or, where another request ends in it, its last one's
  const int first_slot = base <= runs.first(s0) ? 2 * s0 : 2 * s0 + 1;
  auto place = [&](int s) -> int64_t {
    return ((int64_t)(s == s0 ? first_slot : 2 * s) * a.n_blocks + block) * a.block + in_block;
  };
  constexpr int kAhead = 4;
  f32x4 v[kAhead][2];
  auto load = [&](int s) {   // shares s, s + G, ..: past the end the last one again, not used
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int at_s = s + j * G <= s1 ? s + j * G : s1;
      const f32x4* src = (const f32x4*)(a.part_o + place(at_s) * 512 + lane * 8);
      v[j][0] = src[0];
      v[j][1] = src[1];
    }
  };
  load(s0 + sub);
  float m = -INFINITY;
  for (int s = s0 + lane; s <= s1; s += 64) m = fmaxf(m, a.part_ml[place(s) * 2]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  const float ref = m == -INFINITY ? 0.f : m;
  f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = {0.f, 0.f, 0.f, 0.f};
  float l = 0.f;
  for (int c = s0; c <= s1; c += 64) {   // 64 shares: lane j holds the weight of share c + j
    float w = 0.f;
    if (c + lane <= s1) {
      const float* ml = a.part_ml + place(c + lane) * 2;
      w = __builtin_amdgcn_exp2f(ml[0] - ref);
      l += w * ml[1];
    }
    for (int i = sub; i < 64 && c + i <= s1; i += kAhead * G) {
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        if (c + i + j * G > s1) break;
        const float wj = __shfl(w, i + j * G, 64);
        x += v[j][0] * wj;
        y += v[j][1] * wj;
      }
      if (c + i + kAhead * G <= s1) load(c + i + kAhead * G);
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) l += __shfl_xor(l, o, 64);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if (sub == 0 && lane == 0 && a.out_lse != nullptr)
    a.out_lse[at] = l == 0.f ? -INFINITY : (ref + __log2f(l)) * 0.6931471805599453f;
  if constexpr (G == 1) {
    *(u32x4*)(a.out_o + at * 512 + lane * 8) = u32x4{pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv),
                                                     pack_bf16x2(y[0] * inv, y[1] * inv), pack_bf16x2(y[2] * inv, y[3] * inv)};
  } else {
    static_assert(G == 1 || G == kWaves, "a head-row's waves are a workgroup");
    *(f32x4*)&acc[wave][lane * 8] = x;
    *(f32x4*)&acc[wave][lane * 8 + 4] = y;
    __syncthreads();
    float o = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) o += acc[w][threadIdx.x];
    a.out_o[at * 512 + threadIdx.x] = __builtin_bit_cast(uint16_t, (__bf16)(o * inv));
  }
}

}  // namespace

hipError_t launch_cache_attend(const CacheAttendArgs& a, hipStream_t s) {
  const unsigned grid = 8u * (unsigned)a.n_blocks * (unsigned)((a.shares + 7) / 8);
  if (a.block == 16)
    cache_attend_kernel<1><<<dim3(grid), dim3(kThreads), 0, s>>>(a);
  else if (a.block == 32)
    cache_attend_kernel<2><<<dim3(grid), dim3(kThreads), 0, s>>>(a);
  else
    cache_attend_kernel<4><<<dim3(grid), dim3(kThreads), 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const unsigned R = (unsigned)(a.n_q * a.n_heads), n_seqs = (unsigned)a.n_seqs;
  // A wave a head-row where it can hold all its shares' sums in flight at once, else eight
  // (64 requests of 16k keys, 4 shares each: 209 against 216 us for the whole call; 48
  // requests of 6k, 5.3 shares: 47.7 against 47.0; one of 264k, 256 shares: 99 against 64)
  if (a.shares <= 4 * a.n_seqs)
    cache_merge_kernel<1><<<dim3((R + kWaves - 1) / kWaves, n_seqs), dim3(kThreads), 0, s>>>(a);
  else
    cache_merge_kernel<kWaves><<<dim3(R, n_seqs), dim3(kThreads), 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace mla

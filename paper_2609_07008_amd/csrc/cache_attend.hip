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

#define MLA_CONST __attribute__((address_space(4)))

constexpr int kWaves = 8, kThreads = kWaves * 64;

template <int NBQ>
struct CaCfg {
  static constexpr int BM = 32 * NBQ;        // head-rows of a workgroup
  static constexpr int NB = 2 * NBQ;         // in blocks of 16
  static constexpr int KBL = 8 * 1024 + 128; // latent of an 8-key block: a kilobyte per 64 dims
  static constexpr int LAT = 8 * KBL;
  static constexpr int KBR = 1024 + 128;     // RoPE keys of an 8-key block
  static constexpr int ROPE_OFF = 2 * LAT;   // two latent buffers; RoPE keys are read before the next tile's arrive
  static constexpr int P_OFF = ROPE_OFF + 8 * KBR;
  static constexpr int QLO_OFF = P_OFF + 2 * NB * 1024;
  static constexpr int EX_OFF = QLO_OFF + 2 * NB * 1024;   // [BM][4]: a value of each key wave
  static constexpr int TH_OFF = EX_OFF + BM * 16;
  static constexpr int LDS = TH_OFF + kMaxRopePairs * 8;
  static_assert(LDS <= 160 * 1024, "LDS of a compute unit");
};

// slot of 16-byte chunk c of key k in its kilobyte: c ^ key_swz(k) (see attend_pair.hip)
__device__ __forceinline__ int key_swz(int k) { return k ^ ((~k & 1) << 2); }

// this wave's LDS accesses are done, then all waves meet (loads from memory stay in flight)
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

struct Tile {       // wave-uniform
  int page, sub;    // page to read (0 where there is none), tile of the page
  int rows;         // rows of the tile that hold keys, 0 .. 64
  int frame;
  int64_t pos0;     // request position of the tile's first row
};

__device__ __forceinline__ Tile tile_of(const CacheAttendArgs& a, const mla_page MLA_CONST* entries, int u, int tpp) {
  const int e = u / tpp;
  Tile t;
  t.sub = u - e * tpp;
  const mla_page MLA_CONST* en = entries + e;
  const int rows = en->rows < a.page_rows ? en->rows : a.page_rows;
  const bool there = (unsigned)en->page < (unsigned)a.cache_pages;
  t.page = there ? en->page : 0;
  const int left = (there ? rows : 0) - t.sub * kCacheTile;
  t.rows = left < 0 ? 0 : left < kCacheTile ? left : kCacheTile;
  t.frame = en->frame;
  t.pos0 = (int64_t)en->req_pos + t.sub * kCacheTile;
  return t;
}

// keys of the tile that a row at position t sees, 0 .. 64
__device__ __forceinline__ int seen_keys(const Tile& x, int t) {
  const int64_t d = (int64_t)t - x.pos0 + 1;
  const int n = t < 0 || d < 0 ? 0 : d < x.rows ? (int)d : x.rows;
  return n;
}

__device__ __forceinline__ float quad_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
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

template <int NBQ>
__global__ __launch_bounds__(kThreads, 2) void cache_attend_kernel(CacheAttendArgs a) {
  using C = CaCfg<NBQ>;
  constexpr int NB = C::NB, BM = C::BM;
  __shared__ __attribute__((aligned(16))) unsigned char lds[C::LDS];
  unsigned char MLA_LDS* L = (unsigned char MLA_LDS*)lds;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lg = lane >> 4, lc = lane & 15;
  const int kb = wave & 3, hh = wave >> 2;
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
    const int lo = (int)((int64_t)total * share / a.shares);
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
  const int lo = (int)((int64_t)total * share / a.shares);
  const int hi = (int)((int64_t)total * (share + 1) / a.shares);
  if (lo >= hi) return;

  double MLA_LDS* theta = (double MLA_LDS*)(L + C::TH_OFF);
  float MLA_LDS* ex = (float MLA_LDS*)(L + C::EX_OFF);

  // this lane's part of a tile's loads: row 8 wave + r of the tile, groups gq and gq + 8,
  // RoPE chunk gq
  const int r8 = lane & 7, gq = lane >> 3;
  u32x4 cw[2], rp;
  uint32_t sc[2];
  auto load_tile = [&](const Tile& t) {
    const unsigned char* p = a.cache + (int64_t)t.page * a.page_rows * kCacheRow;
    const uint32_t row = (uint32_t)(t.sub * kCacheTile + wave * 8 + r8);
    const unsigned char* ps = p + (uint32_t)a.page_rows * kCacheCodes;
    const unsigned char* pr = ps + (uint32_t)a.page_rows * kCacheScales;
    cw[0] = *(const u32x4*)(p + row * kCacheCodes + gq * 16);
    cw[1] = *(const u32x4*)(p + row * kCacheCodes + gq * 16 + 128);
    sc[0] = ps[row * kCacheScales + gq];
    sc[1] = ps[row * kCacheScales + gq + 8];
    rp = *(const u32x4*)(pr + row * kCacheRope + gq * 16);
  };
  auto store_tile = [&](int buf, int seen) {
    const bool live = wave * 8 + r8 < seen;
    unsigned char MLA_LDS* d = L + buf + wave * C::KBL + r8 * 128;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int g = gq + 8 * h;
      const float s = mx4_scale(live ? sc[h] : 127u);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(bf16x8 MLA_LDS*)(d + (g >> 1) * 1024 + ((((g & 1) * 4 + i) ^ key_swz(r8)) * 16)) = mx4_values(live ? cw[h][i] : 0u, s);
    }
    *(u32x4 MLA_LDS*)(L + C::ROPE_OFF + wave * C::KBR + r8 * 128 + ((gq ^ key_swz(r8)) * 16)) = live ? rp : u32x4{0, 0, 0, 0};
  };

  // K fragments (A operand, 16 keys x 32 dims) and V^T fragments (16 dims x 32 keys)
  const int ksw = (lg ^ key_swz(lc & 7)) * 16;
  const int kat = (kb * 2 + (lc >> 3)) * C::KBL + (lc & 7) * 128 + ksw;
  const int rat = C::ROPE_OFF + (kb * 2 + (lc >> 3)) * C::KBR + (lc & 7) * 128 + ksw;
  const int vkey = (lg & 1) * 4 + (lc >> 2), vcb = lc & 3;
  const int vat = (lg >> 1) * C::KBL + vkey * 128 + (((vcb >> 1) ^ key_swz(vkey)) * 16) + (vcb & 1) * 8 + wave * 1024;

  if (tid < kMaxRopePairs) theta[tid] = a.rope.theta[tid];

  int b = first_b, base = first_base;
  for (; base < hi; ++b) {
    const int n = __builtin_amdgcn_readfirstlane(tiles_of(a, b, tpp));
    const int u0 = lo > base ? lo - base : 0, u1 = hi < base + n ? hi - base : n;
    const int seq_base = base;
    base += n;
    if (u0 >= u1) continue;
    const mla_page MLA_CONST* entries = (const mla_page MLA_CONST*)(uintptr_t)(a.pages + (int64_t)b * a.max_pages);

    // the head-rows: block row i is head-row hb BM + i of the request; rows past the end
    // repeat the last one and are not stored
    const uint16_t* qrow[NBQ];
    int tq[NBQ];
    int t_max = INT32_MIN, t_min = INT32_MAX;
#pragma unroll
    for (int nb = 0; nb < NBQ; ++nb) {
      int hr = hb * BM + (hh * NBQ + nb) * 16 + lc;
      hr = hr < R ? hr : R - 1;
      tq[nb] = a.pos[(int64_t)b * a.n_q + hr / a.n_heads];
      qrow[nb] = a.q + ((int64_t)b * R + hr) * 576;
    }
    {
      const int last = (hb + 1) * BM < R ? (hb + 1) * BM : R;
      for (int j = hb * BM / a.n_heads; j <= (last - 1) / a.n_heads; ++j) {
        const int t = __builtin_amdgcn_readfirstlane(a.pos[(int64_t)b * a.n_q + j]);
        t_max = t > t_max ? t : t_max;
        t_min = t < t_min ? t : t_min;
      }
    }
    Tile cur = tile_of(a, entries, u0, tpp);
    load_tile(cur);
    bf16x8 qf[16][NBQ], qr[2][NBQ];
#pragma unroll
    for (int nb = 0; nb < NBQ; ++nb)
#pragma unroll
      for (int ks = 0; ks < 16; ++ks) qf[ks][nb] = *(const bf16x8*)(qrow[nb] + ks * 32 + lg * 8);
    // the query's RoPE part in the page's frame: rounded in registers, the rest in LDS
    auto relocate = [&](int frame) {
#pragma unroll
      for (int nb = 0; nb < NBQ; ++nb) {
        const bf16x8 x1 = *(const bf16x8*)(qrow[nb] + 512 + lg * 8);
        const bf16x8 x2 = *(const bf16x8*)(qrow[nb] + 544 + lg * 8);
        const double dd = (double)((int64_t)tq[nb] - frame);
        bf16x8 l1, l2;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const double rev = dd * theta[lg * 8 + i];
          const float r = (float)(rev - rint(rev));
          const float sn = __builtin_amdgcn_sinf(r), cn = __builtin_amdgcn_cosf(r);
          const float y1 = (float)x1[i] * cn - (float)x2[i] * sn, y2 = (float)x1[i] * sn + (float)x2[i] * cn;
          qr[0][nb][i] = (__bf16)y1;
          qr[1][nb][i] = (__bf16)y2;
          l1[i] = (__bf16)(y1 - (float)qr[0][nb][i]);
          l2[i] = (__bf16)(y2 - (float)qr[1][nb][i]);
        }
        if (kb == 0) {
          unsigned char MLA_LDS* p = L + C::QLO_OFF + (hh * NBQ + nb) * 2048 + lane * 16;
          *(bf16x8 MLA_LDS*)p = l1;
          *(bf16x8 MLA_LDS*)(p + 1024) = l2;
        }
      }
    };
    lds_barrier();   // the tables and what the previous request left in LDS are read
    relocate(cur.frame);
    store_tile(0, seen_keys(cur, t_max));
    Tile nxt = cur;
    if (u0 + 1 < u1) {
      nxt = tile_of(a, entries, u0 + 1, tpp);
      load_tile(nxt);
    }
    f32x4 o[4][NB];
    float m_run[NB], l_run[NBQ];
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int h = 0; h < NB; ++h) o[d][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int h = 0; h < NB; ++h) m_run[h] = -INFINITY;
#pragma unroll
    for (int nb = 0; nb < NBQ; ++nb) l_run[nb] = 0.f;
    lds_barrier();

    int buf = 0;
    for (int u = u0; u < u1; ++u) {
      Tile nn = nxt;
      if (u + 2 < u1) nn = tile_of(a, entries, u + 2, tpp);
      // ---- scores
      f32x4 s[NBQ];
#pragma unroll
      for (int nb = 0; nb < NBQ; ++nb) s[nb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < 16; ++ks) {
        const bf16x8 k = *(const bf16x8 MLA_LDS*)(L + ((buf + kat) ^ ((ks & 1) * 64)) + (ks >> 1) * 1024);
#pragma unroll
        for (int nb = 0; nb < NBQ; ++nb) s[nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, qf[ks][nb], s[nb], 0, 0, 0);
      }
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const bf16x8 k = *(const bf16x8 MLA_LDS*)(L + (rat ^ (ks * 64)));
#pragma unroll
        for (int nb = 0; nb < NBQ; ++nb) {
          const bf16x8 ql = *(const bf16x8 MLA_LDS*)(L + C::QLO_OFF + (hh * NBQ + nb) * 2048 + ks * 1024 + lane * 16);
          s[nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, ql, s[nb], 0, 0, 0);
          s[nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, qr[ks][nb], s[nb], 0, 0, 0);
        }
      }
      // register i of s[nb]: key kb*16 + lg*4 + i, head-row lc of the block
      if (seen_keys(cur, t_min) < kCacheTile) {
#pragma unroll
        for (int nb = 0; nb < NBQ; ++nb) {
          const int rel = seen_keys(cur, tq[nb]) - (kb * 16 + lg * 4);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (i >= rel) s[nb][i] = -INFINITY;
        }
      }
#pragma unroll
      for (int nb = 0; nb < NBQ; ++nb) {
        const float m = quad_max(fmaxf(fmaxf(s[nb][0], s[nb][1]), fmaxf(s[nb][2], s[nb][3]))) * a.scale_log2;
        if (lg == 0) ex[((hh * NBQ + nb) * 16 + lc) * 4 + kb] = m;
      }
      lds_barrier();
      // ---- reference, weights
      bool moves = false;
      float m_new[NB];
#pragma unroll
      for (int h = 0; h < NB; ++h) {
        const f32x4 v = *(const f32x4 MLA_LDS*)(ex + (h * 16 + lc) * 4);
        const float m = fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3]));
        const bool up = m > m_run[h] + 8.f || (m_run[h] == -INFINITY && m > -INFINITY);
        m_new[h] = up ? m : m_run[h];
        moves |= up;
      }
      if (__builtin_amdgcn_ballot_w64(moves) != 0) {
#pragma unroll
        for (int h = 0; h < NB; ++h) {
          const float al = m_new[h] == m_run[h] ? 1.f : __builtin_amdgcn_exp2f(m_run[h] - m_new[h]);
          m_run[h] = m_new[h];
#pragma unroll
          for (int d = 0; d < 4; ++d) o[d][h] *= al;
#pragma unroll
          for (int nb = 0; nb < NBQ; ++nb)
            if (h == hh * NBQ + nb) l_run[nb] *= al;
        }
      }
#pragma unroll
      for (int nb = 0; nb < NBQ; ++nb) {
        float m = hh ? m_run[NBQ + nb] : m_run[nb];
        m = m == -INFINITY ? 0.f : m;   // nothing seen yet: every weight is 0
        float w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          w[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[nb][i], a.scale_log2, -m));
          l_run[nb] += w[i];
        }
        *(u32x2 MLA_LDS*)(L + C::P_OFF + ((kb >> 1) * NB + hh * NBQ + nb) * 1024 + lane * 16 + (kb & 1) * 8) =
            u32x2{pack_bf16x2(w[0], w[1]), pack_bf16x2(w[2], w[3])};
      }
      // ---- the next tile into the other buffer, the one after it on its way
      if (u + 1 < u1) {
        store_tile(buf ^ C::LAT, seen_keys(nxt, t_max));
        if (nxt.frame != cur.frame) relocate(nxt.frame);
        if (u + 2 < u1) load_tile(nn);
      }
      lds_barrier();
      // ---- values
#pragma unroll
      for (int k2 = 0; k2 < 2; ++k2) {
        bf16x8 p[NB];
#pragma unroll
        for (int h = 0; h < NB; ++h) p[h] = *(const bf16x8 MLA_LDS*)(L + C::P_OFF + (k2 * NB + h) * 1024 + lane * 16);
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          const unsigned char MLA_LDS* vp = L + ((buf + vat) ^ (d * 32)) + k2 * 4 * C::KBL;
          const bf16x4 vl = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((MLA_LDS bf16x4*)vp);
          const bf16x4 vh = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((MLA_LDS bf16x4*)(vp + 2 * C::KBL));
          const bf16x8 v = __builtin_shufflevector(vl, vh, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
          for (int h = 0; h < NB; ++h) o[d][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[h], o[d][h], 0, 0, 0);
        }
      }
      cur = nxt;
      nxt = nn;
      buf ^= C::LAT;
    }
    // ---- row sums across lanes and key waves, then the rows
    // (ex: every wave has read the last tile's maxima before the barrier above)
#pragma unroll
    for (int nb = 0; nb < NBQ; ++nb) {
      const float l = quad_sum(l_run[nb]);
      if (lg == 0) ex[((hh * NBQ + nb) * 16 + lc) * 4 + kb] = l;
    }
    lds_barrier();
    const bool whole = u0 == 0 && u1 == n;
    const int slot = seq_base <= lo ? 2 * share : 2 * share + 1;
#pragma unroll
    for (int h = 0; h < NB; ++h) {
      const f32x4 lv = *(const f32x4 MLA_LDS*)(ex + (h * 16 + lc) * 4);
      const float l = lv[0] + lv[1] + lv[2] + lv[3];
      const int row = hb * BM + h * 16 + lc;
      if (row >= R) continue;
      if (whole) {
        const int64_t at = (int64_t)b * R + row;
        const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int d = 0; d < 4; ++d)
          *(u32x2*)(a.out_o + at * 512 + wave * 64 + d * 16 + lg * 4) =
              u32x2{pack_bf16x2(o[d][h][0] * inv, o[d][h][1] * inv), pack_bf16x2(o[d][h][2] * inv, o[d][h][3] * inv)};
        if (wave == 0 && lg == 0 && a.out_lse != nullptr)
          a.out_lse[at] = l == 0.f ? -INFINITY : (m_run[h] + __log2f(l)) * 0.6931471805599453f;
      } else {
        const int64_t at = ((int64_t)slot * a.n_blocks + hb) * BM + h * 16 + lc;
#pragma unroll
        for (int d = 0; d < 4; ++d) *(f32x4*)(a.part_o + at * 512 + wave * 64 + d * 16 + lg * 4) = o[d][h];
        if (wave == 0 && lg == 0) {
          a.part_ml[at * 2] = m_run[h];
          a.part_ml[at * 2 + 1] = l;
        }
      }
    }
  }
}

// Joins the sums of requests that several shares hold (and writes those without a tile):
// a workgroup takes a head-row, its waves the shares in turn, eight dims a lane.
__global__ __launch_bounds__(kThreads) void cache_merge_kernel(CacheAttendArgs a) {
  __shared__ __attribute__((aligned(16))) float acc[kWaves][512];
  __shared__ float sums[kWaves];
  const int R = a.n_q * a.n_heads;
  const int b = blockIdx.y, row = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int base = a.tile_base[b], n = a.tile_base[b + 1] - base;
  const int64_t total = a.tile_base[a.n_seqs];
  const int64_t at = (int64_t)b * R + row;
  if (n == 0) {
    a.out_o[at * 512 + tid] = 0;
    if (tid == 0 && a.out_lse != nullptr) a.out_lse[at] = -INFINITY;
    return;
  }
  // the last share s with total s / shares <= tile
  const int s0 = (int)((((int64_t)base + 1) * a.shares - 1) / total);
  const int s1 = (int)((((int64_t)base + n) * a.shares - 1) / total);
  if (s0 == s1) return;
  auto place = [&](int s) -> int64_t {
    const int lo = (int)(total * s / a.shares);
    const int slot = base <= lo ? 2 * s : 2 * s + 1;
    return ((int64_t)slot * a.n_blocks + row / a.block) * a.block + row % a.block;
  };
  float m = -INFINITY;
  for (int s = s0 + lane; s <= s1; s += 64)
    if (total * s / a.shares < total * (s + 1) / a.shares) m = fmaxf(m, a.part_ml[place(s) * 2]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  const float ref = m == -INFINITY ? 0.f : m;
  f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = {0.f, 0.f, 0.f, 0.f};
  float l = 0.f;
  for (int s = s0 + wave; s <= s1; s += kWaves) {
    if (total * s / a.shares >= total * (s + 1) / a.shares) continue;   // a share without tiles
    const int64_t p = place(s);
    const float w = __builtin_amdgcn_exp2f(a.part_ml[p * 2] - ref);
    l += w * a.part_ml[p * 2 + 1];
    const f32x4* src = (const f32x4*)(a.part_o + p * 512 + lane * 8);
    x += src[0] * w;
    y += src[1] * w;
  }
  *(f32x4*)&acc[wave][lane * 8] = x;
  *(f32x4*)&acc[wave][lane * 8 + 4] = y;
  if (lane == 0) sums[wave] = l;
  __syncthreads();
  float v = 0.f, lt = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    v += acc[w][tid];
    lt += sums[w];
  }
  a.out_o[at * 512 + tid] = __builtin_bit_cast(uint16_t, (__bf16)(lt == 0.f ? 0.f : v / lt));
  if (tid == 0 && a.out_lse != nullptr) a.out_lse[at] = lt == 0.f ? -INFINITY : (ref + __log2f(lt)) * 0.6931471805599453f;
}

}  // namespace

hipError_t launch_cache_attend(const CacheAttendArgs& a, hipStream_t s) {
  const unsigned grid = 8u * (unsigned)a.n_blocks * (unsigned)((a.shares + 7) / 8);
  if (a.block == 32)
    cache_attend_kernel<1><<<dim3(grid), dim3(kThreads), 0, s>>>(a);
  else
    cache_attend_kernel<2><<<dim3(grid), dim3(kThreads), 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  cache_merge_kernel<<<dim3((unsigned)(a.n_q * a.n_heads), (unsigned)a.n_seqs), dim3(kThreads), 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace mla

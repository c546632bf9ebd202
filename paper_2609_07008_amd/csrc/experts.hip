// The experts of a mixture-of-experts layer in 8-bit integers:
//   y_n = sum_{j < K_n} w_nj W_down[e] h_nj,  h_nj = silu(W_gate[e] x_n) * (W_up[e] x_n),  e = expert_idx[n, j]
// Pairs (n, j) are put in expert order; x is quantized a row; the products run over tiles of
// rows of one expert (i8_tiles.h); h is rounded to bf16, a layer's activation, and quantized a
// row; the pairs of a token are joined in rank order, in f32.  Within an expert the order of the
// pairs hangs on LDS atomics, but rows do not meet and the products are exact in i32: the result
// does not.
// With few rows an expert the time is that of its weights: 64 tokens over 256 experts 4096 x 2048, of
// which 129 are met, 505 us, 6.3 TB/s.  With many it is the products': 33,792 tokens 5.3 ms, of which
// gate and up 2.68 (1.9 POP/s), down 1.76, the join 0.53, quantizing x and h 0.08 and 0.15.
#include "i8_rows.h"
#include "i8_tiles.h"

namespace mla {
namespace {

// expert of pair p, or -1 where it is not here or past the token's fanout
__device__ __forceinline__ int pair_expert(const ExpertsArgs& a, int32_t p) {
  const int n = p / a.top_k, j = p - n * a.top_k;
  const uint32_t e = (uint32_t)a.idx[p] - (uint32_t)a.first;
  if (e >= (uint32_t)a.n_experts) return -1;
  return a.fanout != nullptr && j >= a.fanout[n] ? -1 : (int)e;
}

// counts of all experts, one a thread of the first n_experts (1024 threads) -> the place of
// each expert's first pair, in `place`; with `out`, the tiles and totals into memory
__device__ void scan_counts(const ExpertsArgs& a, int c, int* place, int* wave_sums, bool out) {
  const int e = threadIdx.x, lane = e & 63, wave = e >> 6;
  const int b = (c + a.tile_rows - 1) / a.tile_rows;
  int rows = c, blocks = b;   // inclusive sums
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int x = __shfl_up(rows, d, 64), y = __shfl_up(blocks, d, 64);
    if (lane >= d) {
      rows += x;
      blocks += y;
    }
  }
  if (lane == 63) {
    wave_sums[2 * wave] = rows;
    wave_sums[2 * wave + 1] = blocks;
  }
  __syncthreads();
  for (int w = 0; w < wave; ++w) {
    rows += wave_sums[2 * w];
    blocks += wave_sums[2 * w + 1];
  }
  if (e < a.n_experts) place[e] = rows - c;
  if (!out) return;
  if (e == 1023) {
    a.head[0] = rows;
    a.head[1] = blocks;
  }
  if (b > 0) a.tiles[blocks - b] = ExpertTile{e, blocks - b, rows - c, c};
  // the other tiles of an expert by all lanes of its wave: one expert may have most of them
  for (uint64_t more = __ballot(b > 1); more != 0; more &= more - 1) {
    const int l = __builtin_ctzll(more);
    const int n = __shfl(b, l, 64), first = __shfl(blocks - b, l, 64), row0 = __shfl(rows - c, l, 64), count = __shfl(c, l, 64);
    for (int i = 1 + lane; i < n; i += 64) a.tiles[first + i] = ExpertTile{(e & ~63) + l, first, row0, count};
  }
}

constexpr int kBlockPairs = 4;                       // pairs of a thread while they are counted and placed
constexpr int kOneBlockPairs = 2048 * kBlockPairs;   // pairs that one workgroup counts and places

// experts of up to N pairs of each thread from lo on, all loads under way at once
template <int N>
struct Pairs {
  int e[N];
  __device__ __forceinline__ Pairs(const ExpertsArgs& a, int64_t lo, int64_t hi) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int64_t p = lo + i * 1024 + threadIdx.x;
      e[i] = p < hi ? pair_expert(a, (int32_t)p) : -1;
    }
  }
  __device__ __forceinline__ void count(int* hist) const {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (e[i] >= 0) atomicAdd(&hist[e[i]], 1);
  }
  __device__ __forceinline__ void place(const ExpertsArgs& a, int64_t lo, int* at) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int p = (int)lo + i * 1024 + threadIdx.x;
      if (e[i] >= 0) a.pairs[atomicAdd(&at[e[i]], 1)] = int2{p / a.top_k, p};
    }
  }
};

// Workgroups [0, blocks): the pairs of each expert, counted a share each; a single one places
// them as well.  The others quantize rows of x.
template <int NV>
__global__ __launch_bounds__(1024) void experts_start_kernel(ExpertsArgs a, int blocks) {
  __shared__ int hist[kExpertsMax], sums[32];
  if ((int)blockIdx.x >= blocks) {
    quantize_rows<256, NV>(I8Args{a.x, a.xq, a.xs, a.n_rows, a.x_stride, a.d_model, nullptr, nullptr}, a.n_rows,
                           ((int64_t)blockIdx.x - blocks) * 4 + threadIdx.x / 256, ((int64_t)gridDim.x - blocks) * 4, hist);
    return;
  }
  const int64_t n_pairs = a.n_rows * a.top_k;
  if (blocks == 1) {
    const Pairs<2 * kBlockPairs> mine(a, 0, n_pairs);
    for (int i = threadIdx.x; i < a.n_experts; i += 1024) hist[i] = 0;
    __syncthreads();
    mine.count(hist);
    __syncthreads();
    scan_counts(a, (int)threadIdx.x < a.n_experts ? hist[threadIdx.x] : 0, hist, sums, true);
    __syncthreads();
    mine.place(a, 0, hist);
    return;
  }
  for (int i = threadIdx.x; i < a.n_experts; i += 1024) hist[i] = 0;
  __syncthreads();
  const int64_t per = (n_pairs + blocks - 1) / blocks, lo = blockIdx.x * per, hi = std::min(lo + per, n_pairs);
  for (int64_t p = lo; p < hi; p += 1024 * kBlockPairs) Pairs<kBlockPairs>(a, p, hi).count(hist);
  __syncthreads();
  for (int i = threadIdx.x; i < a.n_experts; i += 1024) a.hist[blockIdx.x * a.n_experts + i] = hist[i];
}

// every workgroup adds up the counts of all, and so knows where its own pairs go
__global__ __launch_bounds__(1024) void experts_place_kernel(ExpertsArgs a) {
  __shared__ int place[kExpertsMax], sums[32];
  const int64_t n_pairs = a.n_rows * a.top_k, per = (n_pairs + gridDim.x - 1) / gridDim.x;
  const int64_t lo = blockIdx.x * per, hi = std::min(lo + per, n_pairs);
  Pairs<kBlockPairs> mine(a, lo, hi);
  int total = 0, before = 0;
  if ((int)threadIdx.x < a.n_experts) {
    const int* h = a.hist + threadIdx.x;
#pragma unroll 8
    for (int b = 0; b < (int)gridDim.x; ++b) {
      const int c = h[b * a.n_experts];
      total += c;
      before += b < (int)blockIdx.x ? c : 0;
    }
  }
  scan_counts(a, total, place, sums, blockIdx.x == 0);
  if ((int)threadIdx.x < a.n_experts) place[threadIdx.x] += before;
  __syncthreads();
  mine.place(a, lo, place);
  for (int64_t p = lo + 1024 * kBlockPairs; p < hi; p += 1024 * kBlockPairs) Pairs<kBlockPairs>(a, p, hi).place(a, p, place);
}

constexpr int kExpertsGroup = 8;   // row tiles per column tile in the walk of an expert

// The expert tile and column tile of a workgroup.  The tiles that exist are known on the device
// alone: XCD x takes a contiguous range of them, an expert's tiles column by column over 8 row
// tiles, which share the weights in its L2.
struct Place {
  int expert, row, rows, col;   // first place of the tile's rows, rows of it (1 .. BM)
  bool any;
};
__device__ __forceinline__ Place my_tile(const ExpertsArgs& a, int cols) {
  Place p{};
  const int total = a.head[1] * cols, per = (total + 7) / 8;
  const int t = (int)(blockIdx.x % 8) * per + (int)(blockIdx.x / 8);
  if ((int)(blockIdx.x / 8) >= per || t >= total) return p;
  const ExpertTile e = a.tiles[t / cols];
  const int mt = (e.count + a.tile_rows - 1) / a.tile_rows;
  const int r = t - e.first_tile * cols;
  const int group = r / (kExpertsGroup * cols), rem = r % (kExpertsGroup * cols), gm = std::min(kExpertsGroup, mt - group * kExpertsGroup);
  const int m = group * kExpertsGroup + rem % gm;
  p.col = rem / gm;
  p.expert = e.expert;
  p.row = e.row0 + m * a.tile_rows;
  p.rows = std::min(a.tile_rows, e.count - m * a.tile_rows);
  p.any = true;
  return p;
}

// silu(g) = g / (1 + e^-g), or g e^g / (1 + e^g), by the one of them whose exponential does not grow: e = e^-|g|.
// The exponent -|g| log2(e) is split into whole and rest before it is rounded (as one f32 its error would be
// |g| / 2 steps of 2^-24 of e), with log2(e) in two parts; a Newton step takes the quotient to its last
// bit.  Below 6 steps in all, 0.11 ms of gate and up of 33,792 rows.  |g| > 120 counts as 120: e is 0.
__device__ __forceinline__ float silu(float g) {
  const float t = fmaxf(-fabsf(g), -120.0f), n = __builtin_rintf(t * 0x1.715476p+0f);
  const float rest = __builtin_fmaf(t, 0x1.4ae0cp-26f, __builtin_fmaf(t, 0x1.715476p+0f, -n));
  const float e = __builtin_ldexpf(__builtin_amdgcn_exp2f(rest), (int)n);
  const float num = g < 0.0f ? g * e : g, den = 1.0f + e, r = __builtin_amdgcn_rcpf(den), q = num * r;
  return __builtin_fmaf(__builtin_fmaf(-q, den, num), r, q);
}

// h of 32 MI rows x BN / 2 channels: of a wave's BN / 4 columns the first half are gate
// channels, the second the same channels of up.
template <int MI, int BN, int NST>
__device__ __forceinline__ void gate_up_tile(const ExpertsArgs& a, const Place& at, unsigned char* lds) {
  using Tile = I8Tile<MI, BN, NST>;
  constexpr int NI = Tile::NI, W = BN / 8;   // channels of a wave
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int f0 = at.col * (BN / 2), d = a.d_model, f = a.d_ffn;
  const int8_t* w = a.w_gu + (int64_t)at.expert * 2 * f * d;
  Tile tile;
  // rows and channels past the end are clamped to the last one (their results are not stored)
  tile.aim(wave, lane, [&](bool is_a, int r0, int r, const unsigned char*& src, uint32_t& off) {
    if (is_a) {
      src = (const unsigned char*)a.xq;
      off = (uint32_t)a.pairs[at.row + std::min(r, at.rows - 1)].x * (uint32_t)d;
    } else {
      auto row = [&](int q) { return (q / W & 1) * f + std::min(f0 + q / (2 * W) * W + q % W, f - 1); };
      src = (const unsigned char*)w + (int64_t)row(r0) * d;
      off = (uint32_t)((row(r) - row(r0)) * d);
    }
  });
  tile.product(lds, wave, lane, d, (at.rows + 31) / 32);
  const int wm = wave >> 2, wn = wave & 3, lg = lane >> 4, lc = lane & 15;
  const float* s = a.s_gu + (int64_t)at.expert * 2 * f;
  f32x4 sg[NI / 2], su[NI / 2];
#pragma unroll
  for (int j = 0; j < NI / 2; ++j) {
    const int c = std::min(f0 + wn * W + j * 16 + lg * 4, f - 4);
    sg[j] = *(const f32x4*)(s + c);
    su[j] = *(const f32x4*)(s + f + c);
  }
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int r = Tile::row_of(wm, i) + lc;
    if (r >= at.rows) continue;
    const float xs = a.xs[a.pairs[at.row + r].x];
#pragma unroll
    for (int j = 0; j < NI / 2; ++j) {
      const int c = f0 + wn * W + j * 16 + lg * 4;
      if (c >= f) continue;   // whole fours: d_ffn is a multiple of 64
      float h[4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        h[e] = silu((float)tile.acc[i][j][e] * sg[j][e] * xs) * ((float)tile.acc[i][j + NI / 2][e] * su[j][e] * xs);
      *(u32x2*)(a.h + (int64_t)(at.row + r) * f + c) = u32x2{pack_bf16x2(h[0], h[1]), pack_bf16x2(h[2], h[3])};
    }
  }
}

// W_down h of 32 MI rows x BN channels, in f32 and without the scale of h: that is one number a pair,
// which the join has at hand (here it is a load that waits for a load; down and join of 33,792 rows
// 2.44 ms with it, 2.27 without).  Rows leave through LDS, whole lines of each pair's part: 2.5 GB out,
// and in again at the join.
template <int MI, int BN, int NST>
__device__ __forceinline__ void down_tile(const ExpertsArgs& a, const Place& at, unsigned char* lds) {
  using Tile = I8Tile<MI, BN, NST>;
  constexpr int NI = Tile::NI;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n0 = at.col * BN, d = a.d_model, f = a.d_ffn;
  Tile tile;
  tile.aim(wave, lane, [&](bool is_a, int r0, int r, const unsigned char*& src, uint32_t& off) {
    const int last = is_a ? at.rows - 1 : d - 1 - n0, first = std::min(r0, last);
    src = (const unsigned char*)(is_a ? a.hq + (int64_t)(at.row + first) * f : a.w_down + ((int64_t)at.expert * d + n0 + first) * f);
    off = (uint32_t)((std::min(r, last) - first) * f);
  });
  tile.product(lds, wave, lane, f, (at.rows + 31) / 32);
  const int wm = wave >> 2, wn = wave & 3, lg = lane >> 4, lc = lane & 15;
  constexpr int ROW = BN, CH = ROW / 16, RPI = 64 / CH, SW = CH < 8 ? CH - 1 : 7;   // bytes of a wave's BN / 4 sums
  unsigned char MLA_LDS* sw = (unsigned char MLA_LDS*)lds + wave * (2 * 16 * ROW);
  f32x4 ws[NI];
#pragma unroll
  for (int j = 0; j < NI; ++j)
    ws[j] = *(const f32x4*)(a.s_down + (int64_t)at.expert * d + std::min(n0 + wn * (BN / 4) + j * 16 + lg * 4, d - 4));
  const int rl = lane / CH, cl = lane % CH, n = n0 + wn * (BN / 4) + cl * 4;
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int r0 = Tile::row_of(wm, i);
    if (r0 >= at.rows) break;
    unsigned char MLA_LDS* sb = sw + (i & 1) * (16 * ROW);
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      f32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (float)tile.acc[i][j][e] * ws[j][e];
      *(f32x4 MLA_LDS*)(sb + lc * ROW + (((j * 4 + lg) ^ (lc & SW)) * 16)) = v;
    }
#pragma unroll
    for (int p = 0; p < 16 / RPI; ++p) {
      const int r = p * RPI + rl, m = r0 + r;
      const f32x4 v = *(const f32x4 MLA_LDS*)(sb + r * ROW + ((cl ^ (r & SW)) * 16));
      if (m < at.rows && n < d) *(f32x4*)(a.part + (int64_t)a.pairs[at.row + m].y * d + n) = v;
    }
  }
}

// Few pairs (a new token, or some): what counts is the weights' way and the number of launches, so
// gate and up find their tiles themselves and quantize the rows that they take, and so does down.
// A workgroup takes up to P rows of one expert and 128 rows of its weight; the rows' codes lie in
// LDS over all of K (64 KB; P falls as K grows), and each of 8 waves streams 16 rows of the weight
// through its own stages: it waits for its own loads alone, no barrier in the loop.
// One token through 8 of 256 experts 4096 x 2048: 55.5 -> 50.9 us for the whole call; of 64 experts 16
// pairs 86, and 24 pairs 118 against 112 in tiles, whose workgroups share what these find out each.
constexpr int kFewPanel = 65536, kFewStages = 5;

// The t-th block of up to `most` pairs of one expert, by all lanes of a wave: lane l holds pair l.
// The pairs of the block in row_pair, and how many (0: no such block); `expert` is its expert.
__device__ __forceinline__ int few_block(const ExpertsArgs& a, int n_pairs, int t, int most, int lane, int& expert, int* row_pair) {
  const int e = lane < n_pairs ? pair_expert(a, lane) : -1;
  int nth = 0;   // pairs of the same expert before the lane's
  for (int m = 0; m < n_pairs; ++m) nth += __builtin_amdgcn_readlane(e, m) == e && m < lane;
  const bool first = e >= 0 && nth % most == 0;
  const uint64_t firsts = __ballot(first);
  const uint64_t at = __ballot(first && __popcll(firsts & ((1ull << lane) - 1)) == t);
  if (at == 0) return 0;
  const int l = __builtin_ctzll(at), from = __builtin_amdgcn_readlane(nth, l);
  expert = __builtin_amdgcn_readlane(e, l);
  const bool mine = e == expert && nth >= from && nth < from + most;
  if (mine) row_pair[nth - from] = lane;
  return __popcll(__ballot(mine));
}

// One of the two products: 16 rows of a weight a wave (w_row(q): row of q = 0 .. 15), rows of bf16
// (x_row(r)) quantized.  Codes of k of row r: slice k / 128 of the panel, chunk k / 16 % 8 at slot
// chunk ^ i8_swz(r); NV: vectors of 8 of a lane in a row.
template <int NV, class WRow, class XRow>
__device__ __forceinline__ i32x4 few_product(unsigned char* lds, float* scale, int rows, int k_len, int wave, int lane, WRow&& w_row, XRow&& x_row) {
  constexpr int P = 128 / NV;   // NV = 8, 16, 32: up to 4096, 8192, 16384 of K
  const int nk = (k_len + I8_ROWB - 1) / I8_ROWB, cut = k_len % I8_ROWB ? nk - 1 : nk;
  unsigned char* stage = lds + kFewPanel + wave * (kFewStages * 2048);
  const unsigned char* src[2];
  uint32_t voff[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    src[j] = (const unsigned char*)w_row(8 * j);
    voff[j] = (uint32_t)((const unsigned char*)w_row(8 * j + (lane >> 3)) - src[j]) + (((lane & 7) ^ i8_swz(8 * j + (lane >> 3))) * 16);
  }
  auto load = [&](int kt, int st) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      uint32_t v = voff[j];
      if (kt == cut) v -= (((lane >> 2) ^ j) & 1) * 64;   // of a last half slice the lower chunks again
      dma16(src[j] + (int64_t)kt * I8_ROWB, v, (const unsigned char MLA_LDS*)(stage + st * 2048 + j * 1024));
    }
  };
  u32x4 x[NV];
  auto read = [&](int r) {
    const uint16_t* p = x_row(r);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * 64 + lane) * 8;
      x[i] = c < k_len ? *(const u32x4*)(p + c) : u32x4{0, 0, 0, 0};
    }
  };
  auto code = [&](int r) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) m = umax(m, umax(x[i][k] & 0x7fffu, (x[i][k] >> 16) & 0x7fffu));
    m = wave_max(m);
    const bool finite = m < 0x7f80u;
    const I8Coder coder(finite ? m : 0);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * 64 + lane) * 8;
      if (c < k_len)
        *(u32x2 MLA_LDS*)((unsigned char MLA_LDS*)lds + c / 128 * (P * 128) + r * 128 + ((c / 16 % 8) ^ i8_swz(r)) * 16 + c % 16) =
            finite ? codes8(coder, x[i]) : u32x2{0, 0};
    }
    if (lane == 0) scale[r] = finite ? __uint_as_float(m << 16) / 127.0f : __uint_as_float(0x7fc00000u);
  };
  if (wave < rows) read(wave);
#pragma unroll
  for (int s = 0; s < kFewStages; ++s)
    if (s < nk) load(s, s);
  if (wave < rows) code(wave);
  if (wave + 8 < rows) {
    read(wave + 8);
    code(wave + 8);
  }
  __syncthreads();
  const int lg = lane >> 4, lc = lane & 15;
  const unsigned char MLA_LDS* A = (const unsigned char MLA_LDS*)lds + (lc % P) * 128;
  const unsigned char MLA_LDS* B = (const unsigned char MLA_LDS*)stage + lc * 128;
  const int ca = (lg ^ i8_swz(lc % P)) * 16, cb = (lg ^ i8_swz(lc)) * 16;
  i32x4 acc = {0, 0, 0, 0};
  int st = 0;
  for (int kt = 0; kt < nk; ++kt) {
    // this wave's slice kt has landed; near the end fewer are under way
    if (kt + kFewStages <= nk) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * (kFewStages - 1)) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    const i32x4 b0 = *(const i32x4 MLA_LDS*)(B + st * 2048 + cb), b1 = *(const i32x4 MLA_LDS*)(B + st * 2048 + (cb ^ 64));
    const i32x4 a0 = *(const i32x4 MLA_LDS*)(A + kt * (P * 128) + ca), a1 = *(const i32x4 MLA_LDS*)(A + kt * (P * 128) + (ca ^ 64));
    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(b0, a0, acc, 0, 0, 0);
    if (kt != cut) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(b1, a1, acc, 0, 0, 0);
    if (kt + kFewStages < nk) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the stage is read
      load(kt + kFewStages, st);
    }
    st = st == kFewStages - 1 ? 0 : st + 1;
  }
  return acc;
}

constexpr int kFewLds = kFewPanel + I8_WAVES * kFewStages * 2048;

// h of up to P rows x 64 channels: of a wave's 16 weight rows 8 are gate's, 8 up's
template <int NV>
__global__ __launch_bounds__(I8_WAVES * 64, 2) void experts_few_gate_up_kernel(ExpertsArgs a, int n_pairs, int cols) {
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kFewLds];
  __shared__ int row_pair[16];
  __shared__ float scale[16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t = blockIdx.x / cols, f = a.d_ffn, d = a.d_model;
  int expert = 0;
  // every wave finds the block, and all write the same rows
  const int rows = few_block(a, n_pairs, t, 128 / NV, lane, expert, row_pair);
  if (rows == 0) return;
  __syncthreads();
  const int f0 = (int)(blockIdx.x % cols) * 64 + 8 * wave;
  const int8_t* w = a.w_gu + (int64_t)expert * 2 * f * d;
  const i32x4 acc = few_product<NV>(
      lds, scale, rows, d, wave, lane, [&](int q) { return w + (int64_t)((q >> 3) * f + f0 + (q & 7)) * d; },
      [&](int r) { return a.x + (int64_t)(__builtin_amdgcn_readfirstlane(row_pair[r]) / a.top_k) * a.x_stride; });
  const int lg = lane >> 4, lc = lane & 15, c = f0 + (lg & 1) * 4;   // lg 0, 1: gate; 2, 3: up
  const f32x4 s = *(const f32x4*)(a.s_gu + (int64_t)expert * 2 * f + (lg >> 1) * f + c);
  const float xs = scale[lc < rows ? lc : 0];
  float v[4], h[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[e] = (float)acc[e] * s[e] * xs;
    const float up = __shfl_xor(v[e], 32, 64);
    h[e] = silu(v[e]) * up;
  }
  if (lg < 2 && lc < rows) *(u32x2*)(a.h + (int64_t)row_pair[lc] * f + c) = u32x2{pack_bf16x2(h[0], h[1]), pack_bf16x2(h[2], h[3])};
}

template <int NV>
__global__ __launch_bounds__(I8_WAVES * 64, 2) void experts_few_down_kernel(ExpertsArgs a, int n_pairs, int cols) {
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kFewLds];
  __shared__ int row_pair[16];
  __shared__ float scale[16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t = blockIdx.x / cols, col = (int)(blockIdx.x % cols), f = a.d_ffn, d = a.d_model;
  int expert = 0;
  const int rows = few_block(a, n_pairs, t, 128 / NV, lane, expert, row_pair);
  if (rows == 0) return;
  __syncthreads();
  const int n0 = col * 128 + 16 * wave;
  const int8_t* w = a.w_down + (int64_t)expert * d * f;
  // channels past the end are clamped to the last one (their results are not stored)
  const i32x4 acc = few_product<NV>(
      lds, scale, rows, f, wave, lane, [&](int q) { return w + (int64_t)std::min(n0 + q, d - 1) * f; },
      [&](int r) { return a.h + (int64_t)__builtin_amdgcn_readfirstlane(row_pair[r]) * f; });
  const int lg = lane >> 4, lc = lane & 15, c = n0 + lg * 4;
  if (col == 0 && (int)threadIdx.x < rows) a.hs[row_pair[threadIdx.x]] = scale[threadIdx.x];
  if (lc >= rows || c >= d) return;
  const f32x4 s = *(const f32x4*)(a.s_down + (int64_t)expert * d + c);
  f32x4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = (float)acc[e] * s[e];
  *(f32x4*)(a.part + (int64_t)row_pair[lc] * d + c) = v;
}

// y of a token: its pairs' parts in rank order, 512 channels a wave.  Lane j reads the token's
// pair j; what is chosen by it is then uniform.
template <bool OUT_BF16>
__global__ __launch_bounds__(256) void experts_join_kernel(ExpertsArgs a) {
  constexpr int G = 2;   // parts under way at once (33,792 rows 530 us, with four the same)
  const int lane = threadIdx.x & 63, d = a.d_model, chunks = (d + 511) / 512;
  const int units = (int)a.n_rows * chunks;
  for (int u = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); u < units; u += gridDim.x * 4) {
    const int n = u / chunks, c = (u - n * chunks) * 512 + lane * 8;
    bool mine = false;
    float w = 0.f, hs = 0.f;
    if (lane < a.top_k) {
      const int32_t p = n * a.top_k + lane;
      mine = pair_expert(a, p) >= 0;
      if (mine) {
        w = a.ew[p];
        hs = a.hs[p];
      }
    }
    auto of = [](float v, int j) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), j)); };
    float y[8] = {};
    for (uint64_t here = __ballot(mine); here != 0;) {
      f32x4 v[G][2];
      float wj[G], hj[G];
      int got = 0;
#pragma unroll
      for (int g = 0; g < G; ++g) {
        if (here == 0) break;
        const int j = __builtin_ctzll(here);
        here &= here - 1;
        got = g + 1;
        wj[g] = of(w, j);
        hj[g] = of(hs, j);
        if (c < d) {
          const f32x4* part = (const f32x4*)(a.part + ((int64_t)n * a.top_k + j) * d + c);
          v[g][0] = __builtin_nontemporal_load(part);
          v[g][1] = __builtin_nontemporal_load(part + 1);
        }
      }
#pragma unroll
      for (int g = 0; g < G; ++g) {
        if (g >= got) break;
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] += wj[g] * (v[g][k / 4][k % 4] * hj[g]);
      }
    }
    if (c >= d) continue;
    if (OUT_BF16) {
      *(u32x4*)((uint16_t*)a.y + (int64_t)n * d + c) =
          u32x4{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7])};
    } else {
      f32x4* to = (f32x4*)((float*)a.y + (int64_t)n * d + c);
      to[0] = f32x4{y[0], y[1], y[2], y[3]};
      to[1] = f32x4{y[4], y[5], y[6], y[7]};
    }
  }
}

// LDS of a kernel of tiles of 32 MI rows x BN, three or (MI = 8) two slices, and of the lower ones in it
constexpr int experts_lds(int mi, int bn) {
  const int own = (32 * mi + bn) * I8_ROWB * (mi == 8 ? 2 : 3), low = mi > 2 ? (16 * mi + bn) * I8_ROWB * 3 : 0;
  return own > low ? own : low;
}

// A tile with half of its rows, or a quarter, goes as a lower one: with the sums of the others
// left out, what is left of a step is its loads' way, which more slices in LDS cover.
template <int MI, int BN>
__global__ __launch_bounds__(I8_WAVES * 64, experts_lds(MI, BN) <= 80 * 1024 ? 4 : 2) void experts_gate_up_kernel(ExpertsArgs a) {
  __shared__ __attribute__((aligned(1024))) unsigned char lds[experts_lds(MI, BN)];
  const Place at = my_tile(a, (a.d_ffn + BN / 2 - 1) / (BN / 2));
  if (!at.any) return;
  if (MI == 2 || at.rows > 16 * MI) return gate_up_tile<MI, BN, MI == 8 ? 2 : 3>(a, at, lds);
  if constexpr (MI == 8) {
    if (at.rows > 64) return gate_up_tile<4, BN, 3>(a, at, lds);
  }
  if constexpr (MI > 2) gate_up_tile<2, BN, 3>(a, at, lds);
}

template <int MI, int BN>
__global__ __launch_bounds__(I8_WAVES * 64, experts_lds(MI, BN) <= 80 * 1024 ? 4 : 2) void experts_down_kernel(ExpertsArgs a) {
  __shared__ __attribute__((aligned(1024))) unsigned char lds[experts_lds(MI, BN)];
  const Place at = my_tile(a, (a.d_model + BN - 1) / BN);
  if (!at.any) return;
  if (MI == 2 || at.rows > 16 * MI) return down_tile<MI, BN, MI == 8 ? 2 : 3>(a, at, lds);
  if constexpr (MI == 8) {
    if (at.rows > 64) return down_tile<4, BN, 3>(a, at, lds);
  }
  if constexpr (MI > 2) down_tile<2, BN, 3>(a, at, lds);
}

template <int MI, int BN>
hipError_t launch_gate_up(const ExpertsArgs& a, hipStream_t s) {
  const int64_t total = experts_max_tiles(a.n_rows * a.top_k, a.n_experts, 32 * MI) * ((a.d_ffn + BN / 2 - 1) / (BN / 2));
  experts_gate_up_kernel<MI, BN><<<dim3((unsigned)(8 * ((total + 7) / 8))), dim3(I8_WAVES * 64), 0, s>>>(a);
  return hipGetLastError();
}

template <int MI, int BN>
hipError_t launch_down(const ExpertsArgs& a, hipStream_t s) {
  const int64_t total = experts_max_tiles(a.n_rows * a.top_k, a.n_experts, 32 * MI) * ((a.d_model + BN - 1) / BN);
  experts_down_kernel<MI, BN><<<dim3((unsigned)(8 * ((total + 7) / 8))), dim3(I8_WAVES * 64), 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_start(const ExpertsArgs& a, hipStream_t s) {
  const int64_t n_pairs = a.n_rows * a.top_k;
  const int blocks = n_pairs <= kOneBlockPairs ? 1 : (int)std::min<int64_t>((n_pairs + 2047) / 2048, kDispatchBlocks);
  const dim3 grid((unsigned)(blocks + (a.n_rows + 3) / 4)), blk(1024);
  if (a.d_model <= 4096) experts_start_kernel<2><<<grid, blk, 0, s>>>(a, blocks);
  else if (a.d_model <= 8192) experts_start_kernel<4><<<grid, blk, 0, s>>>(a, blocks);
  else experts_start_kernel<8><<<grid, blk, 0, s>>>(a, blocks);
  if (blocks > 1) experts_place_kernel<<<dim3((unsigned)blocks), blk, 0, s>>>(a);
  return hipGetLastError();
}

template <int NV>
void launch_few_gate_up(const ExpertsArgs& a, int n_pairs, hipStream_t s) {
  const int cols = a.d_ffn / 64;
  experts_few_gate_up_kernel<NV><<<dim3((unsigned)(n_pairs * cols)), dim3(I8_WAVES * 64), 0, s>>>(a, n_pairs, cols);
}

template <int NV>
void launch_few_down(const ExpertsArgs& a, int n_pairs, hipStream_t s) {
  const int cols = (a.d_model + 127) / 128;
  experts_few_down_kernel<NV><<<dim3((unsigned)(n_pairs * cols)), dim3(I8_WAVES * 64), 0, s>>>(a, n_pairs, cols);
}

hipError_t launch_few(const ExpertsArgs& a, hipStream_t s) {
  const int n_pairs = (int)a.n_rows * a.top_k;
  if (a.d_model <= 4096) launch_few_gate_up<8>(a, n_pairs, s);
  else if (a.d_model <= 8192) launch_few_gate_up<16>(a, n_pairs, s);
  else launch_few_gate_up<32>(a, n_pairs, s);
  if (a.d_ffn <= 4096) launch_few_down<8>(a, n_pairs, s);
  else if (a.d_ffn <= 8192) launch_few_down<16>(a, n_pairs, s);
  else launch_few_down<32>(a, n_pairs, s);
  return hipGetLastError();
}

hipError_t launch_many(const ExpertsArgs& a, hipStream_t s) {
  hipError_t e = launch_start(a, s);
  if (e != hipSuccess) return e;
  switch (a.tile_rows) {
    case 64: e = launch_gate_up<2, 128>(a, s); break;
    case 128: e = launch_gate_up<4, 256>(a, s); break;
    default: e = launch_gate_up<8, 256>(a, s); break;
  }
  if (e != hipSuccess) return e;
  e = launch_i8_quantize(I8Args{a.h, a.hq, a.hs, a.n_rows * a.top_k, a.d_ffn, a.d_ffn, a.head, a.pairs}, s);
  if (e != hipSuccess) return e;
  switch (a.tile_rows) {
    case 64: e = launch_down<2, 128>(a, s); break;
    case 128: e = launch_down<4, 256>(a, s); break;
    default: e = launch_down<8, 256>(a, s); break;
  }
  return e;
}

hipError_t launch_chunk(const ExpertsArgs& a, hipStream_t s) {
  const hipError_t e = a.few ? launch_few(a, s) : launch_many(a, s);
  if (e != hipSuccess) return e;
  const unsigned join = (unsigned)std::min<int64_t>((a.n_rows * ((a.d_model + 511) / 512) + 3) / 4, 1 << 16);
  if (a.y_bf16) experts_join_kernel<true><<<dim3(join), dim3(256), 0, s>>>(a);
  else experts_join_kernel<false><<<dim3(join), dim3(256), 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_experts(const ExpertsArgs& all, hipStream_t s) {
  for (int64_t r = 0; r < all.n_rows; r += kExpertsChunk) {
    ExpertsArgs a = all;
    a.n_rows = std::min<int64_t>(all.n_rows - r, kExpertsChunk);
    a.x += r * a.x_stride;
    a.idx += r * a.top_k;
    a.ew += r * a.top_k;
    if (a.fanout != nullptr) a.fanout += r;
    a.y = (unsigned char*)a.y + r * a.d_model * (a.y_bf16 ? 2 : 4);
    const hipError_t e = launch_chunk(a, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace mla

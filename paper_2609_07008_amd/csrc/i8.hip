// 8-bit integers with a scale for each row, and y = W_b z in them.
//
// A row x of bf16 is held as codes q = round(127 x / max|x|) and the scale max|x| / 127.  The
// sum of a product of codes is a whole number of at most 128^2 * 16384 = 2^28 and is exact in i32,
// so a product does not depend on its order, tile or split: every form gives the same bits.
#include "i8_rows.h"
#include "i8_tiles.h"

namespace mla {
namespace {

// Rows up to 2048 wide by a wave, wider ones by a workgroup, so that a row stays in 16 to 32 registers
// a lane and is read once.  264,192 rows x 4096: 0.53 ms, 6.1 TB/s of the 3 bytes a value.
template <int T, int NV>
__global__ __launch_bounds__(256) void i8_quantize_kernel(I8Args a) {
  __shared__ int part[8];
  const int64_t n = a.n_dev != nullptr ? std::min<int64_t>(*a.n_dev, a.n_rows) : a.n_rows;
  quantize_rows<T, NV>(a, n, (int64_t)blockIdx.x * (256 / T) + threadIdx.x / T, (int64_t)gridDim.x * (256 / T), part);
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

constexpr int kWbGroup = 8;                              // row panels per column panel in the tile walk

// y = W_b z in tiles (i8_tiles.h).  Workgroups go to the 8 XCDs round-robin, so XCD x takes a
// contiguous range of tiles, and inside it tiles walk 8 row panels per column panel.  The output
// leaves through LDS as whole 128-byte lines.
// 264,192 rows 4096 -> 4096: 3.4 ms, 2.6 POP/s (fragments straight from memory 36), matrix cores 68 %
// busy at 1.84 GHz.  Of a 256 x 256 tile's 54 us the slices of K take 46.7 (1.46 each), scaling and
// rounding 2.6 and the stores 4, which is what a unit sends: first tiles staggered by up to a
// half changed nothing.
template <bool OUT_BF16, int MI, int BN, int NST>
__global__ __launch_bounds__(I8_WAVES * 64, i8_occupancy(MI, BN, NST)) void wb_i8_tile_kernel(WbI8Args a, int m_tiles, int n_tiles, bool stream_out) {
  using Tile = I8Tile<MI, BN, NST>;
  constexpr int NI = Tile::NI, BM = Tile::BM;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[Tile::LDS];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int total = m_tiles * n_tiles, per = (total + 7) / 8;
  const int t = (int)(blockIdx.x % 8) * per + (int)(blockIdx.x / 8);
  if ((int)(blockIdx.x / 8) >= per || t >= total) return;
  const int group = t / (kWbGroup * n_tiles), rem = t % (kWbGroup * n_tiles);
  const int gm = std::min(kWbGroup, m_tiles - group * kWbGroup);
  const int mt = group * kWbGroup + rem % gm, nt = rem / gm;
  const int64_t m0 = (int64_t)mt * BM;
  const int n0 = nt * BN;

  Tile tile;
  // rows past the end are clamped to the last one (their results are not stored)
  tile.aim(wave, lane, [&](bool is_a, int r0, int r, const unsigned char*& src, uint32_t& off) {
    const int64_t rows = is_a ? a.n_rows - m0 : (int64_t)a.d_out - n0;   // from the tile's first to the last
    const int64_t first = std::min<int64_t>(r0, rows - 1);
    src = (const unsigned char*)(is_a ? a.z : a.w) + ((is_a ? m0 : n0) + first) * a.d_in;
    off = (uint32_t)((std::min<int64_t>(r, rows - 1) - first) * a.d_in);
  });
  tile.product(lds, wave, lane, a.d_in, (int)std::min<int64_t>((a.n_rows - m0 + 31) / 32, MI));

  // 16 rows x BN / 4 channels a wave at a time: scaled and written in the sums' layout (row lc,
  // channels lg * 4 .. + 3 of each block; 16-byte chunk c of row r at c ^ (r & SW)), read back
  // row-contiguous
  const int wm = wave >> 2, wn = wave & 3, lg = lane >> 4, lc = lane & 15;
  constexpr int ES = OUT_BF16 ? 2 : 4, ROW = BN / 4 * ES;   // element and row bytes
  constexpr int CH = ROW / 16, RPI = 64 / CH;               // 16-byte chunks a row, rows a store
  constexpr int SW = CH < 8 ? CH - 1 : 7;
  unsigned char MLA_LDS* sw = (unsigned char MLA_LDS*)lds + wave * (2 * 16 * ROW);
  f32x4 ws[NI];
#pragma unroll
  for (int j = 0; j < NI; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) ws[j][e] = a.w_scale[std::min(n0 + wn * (BN / 4) + j * 16 + lg * 4 + e, a.d_out - 1)];
  float zs[MI];
#pragma unroll
  for (int i = 0; i < MI; ++i) zs[i] = a.z_scale[std::min<int64_t>(m0 + Tile::row_of(wm, i) + lc, a.n_rows - 1)];
  const bool vec = (a.d_out & (16 / ES - 1)) == 0;   // whole chunks: y is 16-byte aligned
  const int rl = lane / CH, cl = lane % CH;
  const int n = n0 + wn * (BN / 4) + cl * (16 / ES);
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    unsigned char MLA_LDS* sb = sw + (i & 1) * (16 * ROW);
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      f32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (float)tile.acc[i][j][e] * ws[j][e] * zs[i];
      if (OUT_BF16)
        *(u32x2 MLA_LDS*)(sb + lc * ROW + (((j * 2 + (lg >> 1)) ^ (lc & SW)) * 16) + (lg & 1) * 8) =
            u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
      else
        *(f32x4 MLA_LDS*)(sb + lc * ROW + (((j * 4 + lg) ^ (lc & SW)) * 16)) = v;
    }
#pragma unroll
    for (int p = 0; p < (16 + RPI - 1) / RPI; ++p) {
      const int r = p * RPI + rl;
      if (RPI > 16 && r >= 16) continue;   // half of the lanes hold all rows
      const u32x4 v = *(const u32x4 MLA_LDS*)(sb + r * ROW + ((cl ^ (r & SW)) * 16));
      const int64_t m = m0 + Tile::row_of(wm, i) + r;
      if (m >= a.n_rows) continue;
      const int64_t at = m * a.d_out + n;
      if (vec && n + 16 / ES <= a.d_out) {
        u32x4* q = (u32x4*)((unsigned char*)a.y + at * ES);
        if (stream_out) __builtin_nontemporal_store(v, q); else *q = v;
      } else {
#pragma unroll
        for (int e = 0; e < 16 / ES; ++e) {
          if (n + e >= a.d_out) continue;
          if (OUT_BF16)
            ((uint16_t*)a.y)[at + e] = (uint16_t)(v[e / 2] >> (16 * (e & 1)));
          else
            ((uint32_t*)a.y)[at + e] = v[e];
        }
      }
    }
  }
}

// Few rows: the weight is read once, so what counts is how much of it is in flight.  A workgroup
// takes 16 output channels and up to 16 MB rows (all of them); its 8 waves bring 1024 of K at a
// time, a kilobyte of one weight or z row a direct load, into NST stages, and wave b < MB runs
// the MFMAs of row block b.  Chunk c of row r sits at c ^ (r & 15).
// 4096 -> 4096 at 1 and 16 rows, weights from memory: 8.1 us (16.8 MB; the launch is about half).
template <bool OUT_BF16, int MB, int NST>
__global__ __launch_bounds__(I8_WAVES * 64) void wb_i8_rows_kernel(WbI8Args a) {
  constexpr int ROWB = 1024, ROWS = 16 + 16 * MB, STAGE = ROWS * ROWB;
  constexpr int LPW = ROWS / I8_WAVES;           // 1 KB direct loads per wave and stage
  static_assert(ROWS % I8_WAVES == 0, "a load takes a row");
  __shared__ __attribute__((aligned(1024))) unsigned char lds[NST * STAGE];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lg = lane >> 4, lc = lane & 15;
  const int n0 = (int)blockIdx.x * 16;
  // rows past the end repeat the last one; their results are not stored
  const unsigned char* src[LPW];
#pragma unroll
  for (int j = 0; j < LPW; ++j) {
    const int r = wave * LPW + j;
    src[j] = (const unsigned char*)(r < 16 ? a.w + (int64_t)std::min(n0 + r, a.d_out - 1) * a.d_in
                                           : a.z + std::min<int64_t>(r - 16, a.n_rows - 1) * a.d_in);
  }
  auto load = [&](int s, int st) {   // past the end of K: the last chunk again, not used
#pragma unroll
    for (int j = 0; j < LPW; ++j) {
      const int r = wave * LPW + j;
      const uint32_t at = std::min((uint32_t)(s * ROWB + (lane ^ (r & 15)) * 16), (uint32_t)(a.d_in - 16));
      dma16(src[j], at, (const unsigned char MLA_LDS*)(lds + st + r * ROWB));
    }
  };
  i32x4 acc = {0, 0, 0, 0};
  const unsigned char MLA_LDS* L = (const unsigned char MLA_LDS*)lds;
  const int nk = a.d_in / 64, ns = (a.d_in + ROWB - 1) / ROWB;
#pragma unroll
  for (int p = 0; p < NST - 1; ++p) load(p, p * STAGE);
  int st = 0;
  for (int s = 0; s < ns; ++s) {
    // stage s has landed, and every wave has read stage s - 1, whose buffer is next
    dma_barrier<(NST - 2) * LPW>();
    load(s + NST - 1, st == 0 ? (NST - 1) * STAGE : st - STAGE);
    if (wave < MB) {
      const unsigned char MLA_LDS* pw = L + st + lc * ROWB;
      const unsigned char MLA_LDS* pz = L + st + (16 + wave * 16 + lc) * ROWB;
      const int left = nk - s * (ROWB / 64);
      constexpr int N = ROWB / 64, AHEAD = 4;   // fragments read ahead of their MFMA
      i32x4 fw[N], fz[N];
      auto frag = [&](int k) {
        const int o = ((k * 4 + lg) ^ lc) * 16;
        fw[k] = *(const i32x4 MLA_LDS*)(pw + o);
        fz[k] = *(const i32x4 MLA_LDS*)(pz + o);
      };
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) frag(k);
#pragma unroll
      for (int k = 0; k < N; ++k) {
        if (k + AHEAD < N) frag(k + AHEAD);
        __builtin_amdgcn_sched_barrier(0);
        if (k < left) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[k], fz[k], acc, 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    st = st == (NST - 1) * STAGE ? 0 : st + STAGE;
  }
  dma_barrier<0>();   // the loads past the end have landed
  if (wave >= MB) return;
  const int64_t m = wave * 16 + lc;
  if (m >= a.n_rows) return;
  const float zs = a.z_scale[m];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int n = n0 + lg * 4 + e;
    if (n >= a.d_out) continue;
    const float v = (float)acc[e] * a.w_scale[n] * zs;
    if (OUT_BF16)
      ((__bf16*)a.y)[m * a.d_out + n] = (__bf16)v;
    else
      ((float*)a.y)[m * a.d_out + n] = v;
  }
}

template <bool OUT_BF16, int MI, int BN>
hipError_t launch_tiles(const WbI8Args& a, hipStream_t s) {
  const int m_tiles = (int)((a.n_rows + 32 * MI - 1) / (32 * MI));
  const int n_tiles = (a.d_out + BN - 1) / BN;
  const int total = m_tiles * n_tiles;
  // an output beyond the L2s' 32 MB cannot stay there: stored past them, it leaves them to the panels
  const bool stream_out = a.n_rows * a.d_out * (OUT_BF16 ? 2 : 4) > (int64_t)32 << 20;
  wb_i8_tile_kernel<OUT_BF16, MI, BN, wb_i8_slices(32 * MI, BN)><<<dim3((unsigned)(8 * ((total + 7) / 8))), dim3(I8_WAVES * 64), 0, s>>>(a, m_tiles, n_tiles, stream_out);
  return hipGetLastError();
}

template <bool OUT_BF16, int MB>
hipError_t launch_few(const WbI8Args& a, hipStream_t s) {
  wb_i8_rows_kernel<OUT_BF16, MB, wb_i8_slices(16 * MB, 16)><<<dim3((unsigned)((a.d_out + 15) / 16)), dim3(I8_WAVES * 64), 0, s>>>(a);
  return hipGetLastError();
}

template <bool OUT_BF16>
hipError_t launch_out(const WbI8Args& a, hipStream_t s) {
  const I8TileShape t = wb_i8_tile(a.n_rows, a.d_out);
  if (t.channels == 16) return t.rows == 16 ? launch_few<OUT_BF16, 1>(a, s) : launch_few<OUT_BF16, 2>(a, s);
  if (t.channels == 64) return t.rows == 32 ? launch_tiles<OUT_BF16, 1, 64>(a, s) : launch_tiles<OUT_BF16, 2, 64>(a, s);
  if (t.channels == 128) {
    switch (t.rows) {
      case 32: return launch_tiles<OUT_BF16, 1, 128>(a, s);
      case 64: return launch_tiles<OUT_BF16, 2, 128>(a, s);
      case 96: return launch_tiles<OUT_BF16, 3, 128>(a, s);
      default: return launch_tiles<OUT_BF16, 4, 128>(a, s);
    }
  }
  switch (t.rows) {
    case 64: return launch_tiles<OUT_BF16, 2, 256>(a, s);
    case 96: return launch_tiles<OUT_BF16, 3, 256>(a, s);
    case 128: return launch_tiles<OUT_BF16, 4, 256>(a, s);
    case 160: return launch_tiles<OUT_BF16, 5, 256>(a, s);
    case 192: return launch_tiles<OUT_BF16, 6, 256>(a, s);
    case 224: return launch_tiles<OUT_BF16, 7, 256>(a, s);
    default: return launch_tiles<OUT_BF16, 8, 256>(a, s);
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
  const int64_t blocks = std::min<int64_t>((a.n_rows * segs + 3) / 4, (int64_t)1 << 22);
  i8_dequantize_kernel<<<dim3((unsigned)blocks), dim3(256), 0, s>>>(a, segs);
  return hipGetLastError();
}

hipError_t launch_wb_i8(const WbI8Args& a, hipStream_t s) {
  return a.y_bf16 ? launch_out<true>(a, s) : launch_out<false>(a, s);
}

}  // namespace mla

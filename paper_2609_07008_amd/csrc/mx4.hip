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

// y = W z.  A workgroup of W waves takes 16 NB CW output channels and 16 MB rows of z.  d_in
// is cut into slabs of 128, and the slabs into eight classes by their index: a class is
// summed in order, then the classes are added in order, so an element's sum has the same
// order whatever the tile and the number of rows.  CW waves side by side take the channels,
// W / CW the slabs of a step.  A lane holds 32 consecutive values of a channel (16 bytes, one
// group): they feed four 16x16x32 MFMAs, the j-th taking values 8 j .. +7 of each of the
// four groups of a slab, from W and z alike.
//   codes  into registers, four lanes a channel's slab, and through a kilobyte of LDS to the
//          lanes of the fragments
//   z      through LDS, a step ahead and double-buffered, [slab][row][16 chunks], chunk c of
//          row r at c ^ z_swz(r)
// Loaded as fragments, 16 channels or rows a load, either would keep the address unit four
// times as long (64 clocks a kilobyte).  Weights from memory: 32 rows x 7168 -> 16384 take 24
// to 25 us (75 with z as fragments from memory; 13 at the rate of a copy), 200 x 4096 -> 7168
// 24 (114; 8 at the rate of a large product), 1 x 4096 -> 4096 5.7, most of it launch and two
// trips to memory.  From the last-level cache the first takes 18 and the last 5.  What is left
// is the conversion of the codes, once a row block, and what a compute unit takes in, 15 bytes
// a clock, two thirds of it z.  Codes are loaded two steps ahead (CA), but the compiler widens
// their scale bytes at the loop's head and waits there for every load, so that each second step
// waits for the codes of the step after as well.  Twice the waves, z three steps ahead or its
// loads in another order on each unit left the times as they are, all with that wait.
// A 16-byte LDS read is served to lanes 0-3, 12-15, 20-27 of a half wave at once, then to
// its others: rows 0-3 and 12-15 at one chunk with rows 4-11 at the chunk behind the next
// four (lane / 16 of the fragment).  With this they lie in all 64 banks.
__device__ __forceinline__ int z_swz(int r) { return (r & 3) | (r & 8 ? 12 : 0); }

// All but the last N loads of this wave have landed and its LDS accesses are done, then all
// waves meet: behind it a load may overwrite what any wave has read before.
template <int N>
__device__ __forceinline__ void meet() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// Loads before it are issued before those after it: meet counts on z before the codes of the
// step after.
__device__ __forceinline__ void in_order() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

template <int W, int CW, int NB, int MB>
struct WbCfg {
  static constexpr int KW = W / CW, CL = 8 / KW;      // slabs of a step, classes of a wave
  static constexpr int CH = 16 * NB * CW, ROWS = 16 * MB;
  static constexpr int ZB = KW * ROWS * 256;          // z of a step
  static constexpr int CA = NB < 4 ? 2 : 1;           // steps from a load of codes to its use, as registers allow (NB = 4 spills two as it is)
  static constexpr int ZI = ROWS / 4 / CW;             // loads of it in a wave
  static constexpr int C_OFF = 2 * ZB;                // codes on their way to the fragments, NB KB a wave
  static constexpr int RQ = 4 * NB * CW;              // quads of channels
  static constexpr int RED = KW * MB * RQ * 272;      // sums of KW classes, [class][16 rows][quad][17] x 16 bytes
  static constexpr int RE = (ROWS * RQ + 64 * W - 1) / (64 * W);  // quads of outputs of a thread
  static constexpr int LDS = C_OFF + W * NB * 1024 > RED ? C_OFF + W * NB * 1024 : RED;
  static constexpr int WAVES_SIMD = LDS <= 80 * 1024 || W == 16 ? 4 : 2;   // two workgroups a unit where LDS allows
  static_assert(LDS <= 160 * 1024, "LDS of a compute unit");
};

template <bool OUT_BF16, int W, int CW, int NB, int MB>
__global__ __launch_bounds__(64 * W, (WbCfg<W, CW, NB, MB>::WAVES_SIMD)) void wb_mx4_kernel(WbMx4Args a) {
  using C = WbCfg<W, CW, NB, MB>;
  constexpr int KW = C::KW;
  __shared__ __attribute__((aligned(16))) unsigned char lds[C::LDS];
  unsigned char MLA_LDS* L = (unsigned char MLA_LDS*)lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lg = lane >> 4, lc = lane & 15;
  const int cw = wave % CW, kw = wave / CW;
  // workgroups go to the 8 XCDs round-robin: the row blocks of the same channels follow each
  // other on one, whose L2 holds the codes
  const int per_xcd = blockIdx.x >> 3, m_blocks = (int)((a.n_rows + C::ROWS - 1) / C::ROWS);
  const int n_block = per_xcd / m_blocks * 8 + (blockIdx.x & 7), m_block = per_xcd % m_blocks;
  const int n0 = n_block * C::CH, m0 = m_block * C::ROWS;
  if (n0 >= a.d_out) return;
  const int rows = a.n_rows - m0 < C::ROWS ? (int)(a.n_rows - m0) : C::ROWS;
  const int slabs = (a.d_in + 127) / 128, steps = (slabs + KW - 1) / KW;

  // Channels past the end repeat the last one; their results are not stored.
  // A lane loads group lane % 4 of channel lane / 4 of a block's slab.
  const int last_group = a.d_in / 32 - 1;
  const uint32_t row_c = (uint32_t)a.d_in / 2, row_s = (uint32_t)a.d_in / 32;
  const uint8_t* codes[NB];
  const uint8_t* scales[NB];
  uint32_t chan[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    const int c0 = std::min(n0 + (cw * NB + n) * 16, a.d_out - 1), left = a.d_out - 1 - c0;
    chan[n] = (uint32_t)((lane >> 2) < left ? lane >> 2 : left);
    codes[n] = a.codes + (int64_t)c0 * row_c;
    scales[n] = a.scales + (int64_t)c0 * row_s;
  }
  struct Codes {
    u32x4 c[NB];
    uint32_t s[NB];
  };
  auto load_codes = [&](Codes& x, int step) {   // past the end the last group again, not used
    const int g0 = (step * KW + kw) * 4 + (lane & 3), g = g0 < last_group ? g0 : last_group;
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      x.c[n] = *(const u32x4*)(codes[n] + chan[n] * row_c + g * 16);
      x.s[n] = scales[n][chan[n] * row_s + g];
    }
  };
  // A load of z takes four rows of a slab, of which a wave has one a step; rows past the end
  // repeat the last one, chunks past it the last one, neither used.
  const unsigned char* z = (const unsigned char*)(a.z + (int64_t)m0 * a.d_in);
  const int zk = wave % KW, zq = wave / KW, quads = (rows + 3) / 4;
  uint32_t z_row[C::ZI], z_chunk[C::ZI];
#pragma unroll
  for (int i = 0; i < C::ZI; ++i) {
    const int r = (zq + i * CW) * 4 + lg;
    z_row[i] = (uint32_t)((r < rows ? r : rows - 1) * a.d_in) * 2;
    z_chunk[i] = (uint32_t)(zk * 16 + (lc ^ z_swz(r))) * 16;
  }
  const uint32_t z_last = (uint32_t)(a.d_in / 8 - 1) * 16;
  auto load_z = [&](int step, int i) {
    if (zq + i * CW >= quads) return;
    const uint32_t c = (uint32_t)step * (KW * 256) + z_chunk[i];
    dma16(z + (z_row[i] + (c < z_last ? c : z_last)), L + (step & 1) * C::ZB + (zk * C::ROWS + (zq + i * CW) * 4) * 256);
  };
  f32x4 acc[C::CL][NB][MB];   // of class k * KW + kw
#pragma unroll
  for (int k = 0; k < C::CL; ++k)
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int m = 0; m < MB; ++m) acc[k][n][m] = f32x4{0.f, 0.f, 0.f, 0.f};
  const unsigned char MLA_LDS* zl = L + kw * C::ROWS * 256 + lc * 256;
  unsigned char MLA_LDS* own = L + C::C_OFF + wave * NB * 1024;
  auto step = [&](int t, Codes& x, f32x4 (&sum)[NB][MB]) {
    // z of this step has landed; the next step's codes may be on their way
    meet<(C::CA - 1) * 2 * NB>();
    float scale[NB];
    u32x4 code[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      *(u32x4 MLA_LDS*)(own + n * 1024 + (lane >> 2) * 64 + (((lane & 3) ^ ((lane >> 3) & 3)) * 16)) = x.c[n];
      scale[n] = mx4_scale((uint32_t)__builtin_amdgcn_ds_bpermute((lc * 4 + lg) * 4, (int)x.s[n]));
    }
#pragma unroll
    for (int n = 0; n < NB; ++n) code[n] = *(const u32x4 MLA_LDS*)(own + n * 1024 + lc * 64 + ((lg ^ ((lc >> 1) & 3)) * 16));
    // the loads of the next steps
    __builtin_amdgcn_sched_barrier(0);
    if (t + 1 < steps)
#pragma unroll
      for (int i = 0; i < C::ZI; ++i) load_z(t + 1, i);
    in_order();
    load_codes(x, t + C::CA);
    in_order();
    const bool whole = (t * KW + kw) * 4 + 3 <= last_group;   // else groups past the end are zero on both sides
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      bf16x8 zf[MB];
#pragma unroll
      for (int m = 0; m < MB; ++m) zf[m] = *(const bf16x8 MLA_LDS*)(zl + (t & 1) * C::ZB + m * 4096 + (((lg * 4 + j) ^ z_swz(lc)) * 16));
      const bool out = !whole && (t * KW + kw) * 4 + lg > last_group;
      if (out)
#pragma unroll
        for (int m = 0; m < MB; ++m) zf[m] = bf16x8{};
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        bf16x8 wf = mx4_values(code[n][j], scale[n]);
        if (out) wf = bf16x8{};
#pragma unroll
        for (int m = 0; m < MB; ++m) sum[n][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf, zf[m], sum[n][m], 0, 0, 0);
      }
    }
  };
  Codes even, odd;
  load_codes(even, 0);
#pragma unroll
  for (int i = 0; i < C::ZI; ++i) load_z(0, i);
  in_order();
  if (C::CA == 2) load_codes(odd, 1);
  in_order();
  for (int t = 0; t < steps; t += 2) {
    step(t, even, acc[0]);
    if (t + 1 < steps) step(t + 1, C::CA == 2 ? odd : even, acc[C::CL - 1]);
  }
  f32x4 out[C::RE];
#pragma unroll
  for (int e = 0; e < C::RE; ++e) out[e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < C::CL; ++k) {   // classes k KW ..
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int m = 0; m < MB; ++m)
        *(f32x4 MLA_LDS*)(L + ((kw * MB + m) * C::RQ + (cw * NB + n) * 4 + lg) * 272 + lc * 16) = acc[k][n][m];
    __syncthreads();
#pragma unroll
    for (int e = 0; e < C::RE; ++e) {
      const int i = tid + e * 64 * W, q = i % C::RQ, row = i / C::RQ;
      if (row >= rows) continue;
#pragma unroll
      for (int c = 0; c < KW; ++c) out[e] += *(const f32x4 MLA_LDS*)(L + ((c * MB + row / 16) * C::RQ + q) * 272 + (row & 15) * 16);
    }
  }
#pragma unroll
  for (int e = 0; e < C::RE; ++e) {
    const int i = tid + e * 64 * W, q = i % C::RQ, row = i / C::RQ, ch = n0 + q * 4;
    if (row >= rows || ch >= a.d_out) continue;
    const f32x4 v = out[e];
    const int64_t at = (int64_t)(m0 + row) * a.d_out + ch;
    if (a.d_out % 4 == 0) {
      if (OUT_BF16)
        *(u32x2*)((uint16_t*)a.y + at) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
      else
        *(f32x4*)((float*)a.y + at) = v;
    } else {
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        if (ch + c >= a.d_out) continue;
        if (OUT_BF16)
          ((__bf16*)a.y)[at + c] = (__bf16)v[c];
        else
          ((float*)a.y)[at + c] = v[c];
      }
    }
  }
}

template <int W, int CW, int NB, int MB>
hipError_t launch_wb_tile(const WbMx4Args& a, hipStream_t s) {
  using C = WbCfg<W, CW, NB, MB>;
  const int64_t n_blocks = ((int64_t)a.d_out + C::CH - 1) / C::CH, m_blocks = (a.n_rows + C::ROWS - 1) / C::ROWS;
  const dim3 grid((unsigned)((n_blocks + 7) / 8 * 8 * m_blocks));
  if (a.y_bf16)
    wb_mx4_kernel<true, W, CW, NB, MB><<<grid, dim3(64 * W), 0, s>>>(a);
  else
    wb_mx4_kernel<false, W, CW, NB, MB><<<grid, dim3(64 * W), 0, s>>>(a);
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
  // The tile of the least cost.  A workgroup a compute unit takes, at d_in = 4096, about 4 us,
  // 0.07 a row and 0.11 a channel (measured, us: 16 x 16 6.7, 32 x 16 8.2, 32 x 32 10.0,
  // 32 x 64 13.8, 64 x 64 17.5, 64 x 128 25); with more workgroups than units the units take
  // them in turn, each after the first without the launch.  So 200 rows to 7168 channels
  // take 24 us in 64 x 128 (224 workgroups) and 28 in 64 x 64 (448), 128 rows 25 and 18.
  // Of all tiles at 1 to 200 rows and 512 to 16384 channels, the rule's is the fastest or, at
  // d_in = 1024 and 4096, within 6 % of it; at 512 and 16384 within 14 % (1 x 16384 -> 16384 39.6
  // us, in 16 x 32 34.9), at 128 within 0.9 us.
  struct Tile {
    int rows, channels;
    hipError_t (*launch)(const WbMx4Args&, hipStream_t);
  };
  static constexpr Tile kTiles[] = {
      {16, 16, launch_wb_tile<8, 1, 1, 1>},  {32, 16, launch_wb_tile<8, 1, 1, 2>},  {16, 32, launch_wb_tile<16, 2, 1, 1>},
      {32, 32, launch_wb_tile<16, 2, 1, 2>}, {16, 64, launch_wb_tile<8, 2, 2, 1>},  {32, 64, launch_wb_tile<8, 2, 2, 2>},
      {64, 64, launch_wb_tile<8, 2, 2, 4>},  {64, 128, launch_wb_tile<8, 2, 4, 4>}};
  const Tile* best = nullptr;
  int64_t least = INT64_MAX;
  for (const Tile& t : kTiles) {
    if (t.rows > 16 && t.rows / 2 >= a.n_rows) continue;   // half of it would do
    const int64_t blocks = ((a.n_rows + t.rows - 1) / t.rows) * (((int64_t)a.d_out + t.channels - 1) / t.channels);
    const int64_t cost = (blocks + 255) / 256 * (5 * std::min<int64_t>(a.n_rows, t.rows) + 8 * t.channels + 80);
    if (cost < least) {
      least = cost;
      best = &t;
    }
  }
  return best->launch(a, s);
}

}  // namespace mla

// 8-bit integers with a scale for each row (a token, an output channel), products of them,
// and the experts of a mixture-of-experts layer in them: argument structs and launchers.
#pragma once

#include "common.h"
#include "i8_rules.h"

namespace mla {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kI8MaxCols = 16384;       // a row is held in registers; 127^2 * 16384 < 2^31
constexpr int kExpertsMaxPairs = 16;    // columns of expert_idx
constexpr int kExpertsMax = 1024;

struct I8Args {
  const void* x;         // [N, n_cols] bf16, rows x_stride apart
  void* codes;           // [N, n_cols] int8
  float* scales;         // [N]
  int64_t n_rows;
  int64_t x_stride;
  int32_t n_cols;        // multiple of 16, <= kI8MaxCols
  const int32_t* n_dev;  // device count of rows, at most n_rows, or null
  const int2* at;        // the scale of row r goes to scales[at[r].y], or null: to scales[r]
};

hipError_t launch_i8_quantize(const I8Args& a, hipStream_t s);
hipError_t launch_i8_dequantize(const I8Args& a, hipStream_t s);

struct WbI8Args {
  const int8_t* z;         // [N, d_in]
  const float* z_scale;    // [N]
  const int8_t* w;         // [d_out, d_in]
  const float* w_scale;    // [d_out]
  void* y;                 // [N, d_out] f32 or bf16
  int64_t n_rows;
  int32_t d_in;            // multiple of 64
  int32_t d_out;
  int32_t y_bf16;
};

hipError_t launch_wb_i8(const WbI8Args& a, hipStream_t s);

constexpr int kExpertsChunk = 65536;    // rows taken at a time: what the workspace holds
constexpr int kExpertsFewPairs = 16;     // pairs of a call whose products find their rows themselves
constexpr int kDispatchBlocks = 128;    // workgroups that count and place pairs, at most

// One block of rows of an expert.  Its pairs lie at places [row0, row0 + count) of the expert
// order and make ceil(count / tile rows) tiles from first_tile on, all with this entry.
struct ExpertTile {
  int32_t expert;
  int32_t first_tile;
  int32_t row0;
  int32_t count;
};

struct ExpertsArgs {
  // the layer
  const uint16_t* x;         // [N, d_model] bf16, rows x_stride apart
  const int32_t* idx;        // [N, top_k]: expert of the whole layer; outside [first, first + n_experts): not here
  const float* ew;           // [N, top_k]
  const int32_t* fanout;     // [N] or null: the first fanout[n] of a row's experts
  const int8_t* w_gu;        // [n_experts, 2 d_ffn, d_model]: gate rows, then up rows
  const float* s_gu;         // [n_experts, 2 d_ffn]
  const int8_t* w_down;      // [n_experts, d_model, d_ffn]
  const float* s_down;       // [n_experts, d_model]
  void* y;                   // [N, d_model] f32 or bf16
  int64_t n_rows;
  int64_t x_stride;
  int32_t d_model, d_ffn, n_experts, first, top_k, y_bf16;
  // the workspace, for min(n_rows, kExpertsChunk) rows
  int32_t* hist;             // [kDispatchBlocks, n_experts] pairs of each expert in each block's share
  int32_t* head;             // [4]: pairs, tiles
  ExpertTile* tiles;         // [max_tiles]
  int2* pairs;               // [rows top_k]: (n, n * top_k + j) of the pair at each place of the expert order
  int8_t* xq;                // [rows, d_model]
  float* xs;                 // [rows]
  uint16_t* h;               // [rows top_k, d_ffn] bf16
  int8_t* hq;                // [rows top_k, d_ffn]
  float* hs;                 // [rows top_k] by pair
  float* part;               // [rows top_k, d_model] by pair: W_down h without the scale of h
  int32_t tile_rows;
  int32_t few;               // the whole call has at most kExpertsFewPairs pairs: h and part lie apart
};

hipError_t launch_experts(const ExpertsArgs& a, hipStream_t s);

}  // namespace mla

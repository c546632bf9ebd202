// 8-bit integers with a scale for each row (a token, an output channel), products of them,
// and the experts of a mixture-of-experts layer in them: argument structs and launchers.
#pragma once

#include "common.h"

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

// One block of rows of an expert: rows [row, row + count) of the pairs in expert order
struct ExpertTile {
  int32_t expert;
  int32_t row;
  int32_t count;
  int32_t pad;
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
  // the workspace
  int32_t* counts;           // [n_experts] pairs of each expert (atomics), then its cursors [n_experts]
  int32_t* head;             // [4]: pairs, tiles
  ExpertTile* tiles;         // [max_tiles]
  int32_t* pairs;            // [N top_k]: pair n * top_k + j at each place of the expert order
  int8_t* xq;                // [N, d_model]
  float* xs;                 // [N]
  uint16_t* h;               // [N top_k, d_ffn] bf16
  int8_t* hq;                // [N top_k, d_ffn]
  float* hs;                 // [N top_k]
  float* part;               // [N top_k, d_model]: W_down h of each pair
  int32_t max_tiles;
  int32_t tile_rows;
};

// rows of a tile, by the largest number of pairs that an expert has on average
int32_t experts_tile_rows(int64_t n_pairs, int32_t n_experts);
hipError_t launch_experts(const ExpertsArgs& a, hipStream_t s);

}  // namespace mla

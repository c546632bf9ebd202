// The tiles that the products in 8 bits go in, by sizes alone.  Plain C++: a test on the CPU asks the
// same functions.
#pragma once

#include <cstdint>
#include <initializer_list>

namespace mla {

constexpr int64_t kI8FewRows = 32, kI8FewBlocks = 256;   // largest requests of W_b's few-row kernel

// A tile of rows x channels; 16 channels: the few-row kernel, for up to that many rows
struct I8TileShape {
  int32_t rows, channels;
};

// slices of K that a tile of y = W_b z keeps in LDS (of the few-row kernel: of 1024 each, else 128)
constexpr int wb_i8_slices(int32_t rows, int32_t channels) {
  switch (channels) {
    case 16: return rows <= 16 ? 4 : 3;
    case 64: return rows <= 32 ? 6 : 5;
    case 128: return rows <= 32 ? 7 : rows <= 64 ? 6 : rows <= 96 ? 5 : 4;
    default: return rows <= 160 ? 3 : 2;
  }
}

inline I8TileShape wb_i8_tile(int64_t n_rows, int32_t d_out) {
  // Up to 32 rows and a workgroup of 16 channels a compute unit, the few-row kernel: 4096 -> 4096
  // at 16 rows 8.2 us, in tiles of 32 x 64 9.4.
  if (n_rows <= kI8FewRows && ((int64_t)d_out + 15) / 16 <= kI8FewBlocks) return {n_rows <= 16 ? 16 : 32, 16};
  // The tile whose rounds over the 256 compute units cost least: a round of 32 mi rows x 256
  // channels taken as 6 (mi + 3), x 128 as 2 (mi + 7), x 64 as 9 and 10 (mi = 1, 2; two fit a unit,
  // and a second round comes in under the first).  At 4096 channels, weights from memory: 64 rows
  // 9.9 us at 32 x 64 against 14.8 at 32 x 128, 300 rows 16.6 at 64 x 128 against 21 at 32 x 64,
  // 1000 rows 23.8 at 128 x 128 against 26.4 at 64 x 256, 2100 rows 41.6 at 160 x 256 against 46.7
  // at 256 x 256, 4096 rows 58 at 256 x 256 against 71 at 128 x 256; 33 rows of 7168 -> 16384 23.7
  // at 64 x 64 against 27.5 at 32 x 128.
  I8TileShape best{256, 256};
  int64_t cost = INT64_MAX;
  auto tile = [&](int mi, int bn, int w, int first) {
    const int64_t tiles = (n_rows + 32 * mi - 1) / (32 * mi) * (((int64_t)d_out + bn - 1) / bn);
    const int64_t c = (tiles + 255) / 256 * w + first;
    if (c < cost) {
      cost = c;
      best = {32 * mi, bn};
    }
  };
  for (int mi = 8; mi >= 2; --mi) tile(mi, 256, 6 * (mi + 3), 0);
  for (int mi = 4; mi >= 1; --mi) tile(mi, 128, 2 * (mi + 7), 0);
  tile(2, 64, 10, 1);
  tile(1, 64, 9, 1);
  return best;
}

// Rows of a tile of the experts' products, by the pairs of an expert on average, an upper bound
// where others hold experts too.  Few: 64 rows x 128 columns, two workgroups a unit, whose time is
// that of the weights (64 tokens, 6 of 256 experts: gate and up 345 us, down 175; 32 x 128 the same,
// 128 x 256 356 and 180).  Enough to fill them: 128 x 256 (2100 tokens, 6 of 64: 109 and 72 us against
// 124 and 76 in 64 x 128, 123 and 81 in 256 x 256), then 256 x 256 (33,792 tokens, 6 of 256: 2.63 and
// 1.73 ms against 2.96 and 1.99 in 128 x 256).
constexpr int64_t kExpertsAvg64 = 128, kExpertsAvg128 = 384;   // the most for 64 and for 128 rows
inline int32_t experts_tile_rows(int64_t n_pairs, int32_t n_experts) {
  const int64_t avg = n_pairs / n_experts;
  return avg <= kExpertsAvg64 ? 64 : avg <= kExpertsAvg128 ? 128 : 256;
}
inline int64_t experts_max_tiles(int64_t n_pairs, int32_t n_experts, int32_t tile_rows) {
  return n_pairs / tile_rows + (n_experts < n_pairs ? n_experts : n_pairs);
}
// the most tiles that any number of pairs up to n_pairs has in the height taken for it
inline int64_t experts_most_tiles(int64_t n_pairs, int32_t n_experts) {
  const int64_t upto64 = (kExpertsAvg64 + 1) * n_experts - 1, upto128 = (kExpertsAvg128 + 1) * n_experts - 1;
  int64_t most = 0;
  for (const int64_t n : {upto64, upto128, n_pairs}) {
    const int64_t met = n < n_pairs ? n : n_pairs, tiles = experts_max_tiles(met, n_experts, experts_tile_rows(met, n_experts));
    most = tiles > most ? tiles : most;
  }
  return most;
}

}  // namespace mla

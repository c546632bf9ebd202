// Answers of the 8-bit products' rules (i8_rules.h) to lines of standard input:
//   wb <rows> <channels>         -> rows, channels and slices of the tile of W_b
//   experts <pairs> <experts>    -> rows of a tile of the experts' products
#include <cinttypes>
#include <cstdio>
#include <cstring>

#include "i8_rules.h"

int main() {
  char what[16];
  int64_t n;
  int32_t m;
  while (std::scanf("%15s %" SCNd64 " %" SCNd32, what, &n, &m) == 3) {
    if (std::strcmp(what, "wb") == 0) {
      const mla::I8TileShape t = mla::wb_i8_tile(n, m);
      std::printf("%d %d %d\n", t.rows, t.channels, mla::wb_i8_slices(t.rows, t.channels));
    } else {
      std::printf("%d\n", mla::experts_tile_rows(n, m));
    }
  }
  return 0;
}

// Rows and tokens that a block of attention over chunks looks things up for, on the host (the kernel's own functions): never one behind the sequence's last.
#include <algorithm>
#include <cstdio>

#include "attn_chunk.cuh"

int main() {
  using namespace sd::ac;
  long checked = 0;
  for (int group : {1, 2, 3, 4, 7, 8, 32, 127, 128, 129, 300})
    for (int n_new = 1; n_new <= 530; n_new += n_new < 140 || n_new % 128 > 124 || n_new % 128 < 3 ? 1 : 17)
      for (int tiles = 1; tiles <= 2; ++tiles) {
        const int rows_all = n_new * group, rows = tiles * TILE_ROWS;
        for (int row0 = (rows_all - 1) / rows * rows; row0 >= 0; row0 -= rows)
          for (int t = 0; t < 2; ++t) {                        // the second tile's warps are there in blocks of one tile too
            const int start = row0 + t * TILE_ROWS, n_rows = t < tiles ? std::max(0, std::min(TILE_ROWS, rows_all - start)) : 0;
            for (int r = 0; r < TILE_ROWS; ++r) {
              const int row = tile_row(row0, t, n_rows, r);
              if (row < 0 || row / group >= n_new) { printf("row %d of %d tokens in groups of %d, block at %d, tile %d of %d\n", row, n_new, group, row0, t, tiles); return 1; }
              if (r < n_rows && row != start + r) { printf("row %d for %d\n", row, start + r); return 1; }
              ++checked;
            }
            int next = n_rows ? start / group : 0;             // every token of the tile once, in order
            for (int i = 0; i < 256; ++i) {
              const int token = tile_token(start, t < tiles ? std::min(TILE_ROWS, rows_all - start) : 0, group, i);
              if (token < 0) continue;
              if (token != next++ || token >= n_new) { printf("token %d of %d\n", token, n_new); return 1; }
            }
            if (n_rows && next != (start + n_rows - 1) / group + 1) { printf("tokens up to %d of %d\n", next, (start + n_rows - 1) / group + 1); return 1; }
          }
      }
  printf("ok %ld\n", checked);
  return 0;
}

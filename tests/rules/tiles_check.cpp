// Walks the rows and elements that a tile's loads read: all of them lie inside the matrix, and those of the tile that the matrix has are the tile's own.
#include <stdio.h>

#include <initializer_list>

#include "../../paper_2303_06324_amd/csrc/dfx_tiles.h"

int main() {
  const uint32_t sizes[] = {1, 2, 8, 63, 64, 65, 81, 127, 128, 129, 255, 256, 257, 2368, 50257};
  for (uint32_t rows : sizes)
    for (uint32_t tile : {64u, 128u, 256u})
      for (uint32_t m0 = 0; m0 < rows; m0 += tile)
        for (uint32_t half = 0; half < 2; ++half) {
          const uint32_t first = m0 + half * (tile / 2);      // behind the last row where the last tile has half of its rows or fewer
          for (uint32_t r = 0; r < tile / 2; ++r) {
            const uint64_t at = (uint64_t)tile_base(first, rows) + tile_row(first, r, rows);
            if (at >= rows || (first + r < rows && at != first + r)) {
              printf("rows %u tile %u first %u row %u: reads row %llu\n", rows, tile, first, r, (unsigned long long)at);
              return 1;
            }
          }
        }
  for (uint32_t cols : {8u, 64u, 128u, 1024u, 4096u})
    for (uint32_t first = 0; first < cols + 256; first += 64)
      for (uint32_t part = 0; part < 32; ++part) {
        const uint32_t at = tile_col(first, part, cols);
        if (at + 8 > cols || (first + part * 8 + 8 <= cols && at != first + part * 8)) {
          printf("cols %u first %u part %u: reads from %u\n", cols, first, part, at);
          return 1;
        }
      }
  puts("ok");
  return 0;
}

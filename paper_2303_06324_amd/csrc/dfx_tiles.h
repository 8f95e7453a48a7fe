// Which rows and elements of a matrix a tile's loads read: pure functions, compiled for the device (dfx_gemm.h) and for the host (tests/rules/tiles_check.cpp walks them
// without a GPU).  A tile, or half of one, may reach beyond the matrix or lie behind it altogether: what lies behind is the last row, or the last 8 elements, once more.
#ifndef DFX_TILES_H
#define DFX_TILES_H

#include <stdint.h>

#if defined(__HIPCC__)
#define DFX_TILE __host__ __device__ __forceinline__
#else
#define DFX_TILE inline
#endif

// The row that addresses of a tile from row `first` on are counted from, of a matrix of rows >= 1.
DFX_TILE uint32_t tile_base(uint32_t first, uint32_t rows) { return first < rows ? first : rows - 1u; }
// The tile's row-th row, counted from there: never behind the last one.  (Counted from `first` itself, the rest of the rows of a half tile behind the last row would wrap.)
DFX_TILE uint32_t tile_row(uint32_t first, uint32_t row, uint32_t rows) {
  const uint32_t from = tile_base(first, rows), left = rows - 1u - from;
  return row < left ? row : left;
}
// The first of eight elements, the part-th eight from `first` on, of rows of cols >= 8.
DFX_TILE uint32_t tile_col(uint32_t first, uint32_t part, uint32_t cols) { return first + part * 8u < cols - 8u ? first + part * 8u : cols - 8u; }

#endif

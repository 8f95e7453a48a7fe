// How calls of the vocabulary's loss are laid out (csrc/dfx_vocab_plan.h).  Without arguments: walks calls of many sizes; what their kernels touch of each part of the
// workspace lies inside it, and the workspace of more rows holds it.  With rows, dim, vocab, type, piece, aligned: which products such a call with gradients takes.
#include <stdio.h>
#include <stdlib.h>

#include <initializer_list>

#include "../../paper_2303_06324_amd/csrc/dfx_vocab_plan.h"

namespace {

int bad(const char* what, size_t rows, size_t dim, size_t vocab, int dtype, bool grad, size_t piece, bool aligned) {
  printf("%s: rows %zu dim %zu vocab %zu type %d grad %d piece %zu aligned %d\n", what, rows, dim, vocab, dtype, (int)grad, piece, (int)aligned);
  return 1;
}

// elements of a matrix in planes: the last plane's last row included
size_t reach(size_t planes, size_t plane, size_t rows, size_t pitch) { return (planes - 1) * plane + rows * pitch; }

int look(size_t rows, size_t dim, size_t vocab, int dtype, bool grad, size_t piece, bool aligned) {
#define TRY(ok, what) if (!(ok)) return bad(what, rows, dim, vocab, dtype, grad, piece, aligned)
  const VocabPlan p = vocab_plan(rows, dim, vocab, dtype, grad, piece, aligned);
  const size_t planes = gemm_planes(dtype), pieces = vocab ? (vocab + p.vp - 1) / p.vp : 0, last = pieces ? (pieces - 1) * p.vp : 0;
  TRY(p.rp >= rows && p.dp >= dim && p.vp % kTileRows == 0 && p.split_rows >= rows && p.split_rows <= p.rp, "rows and elements");
  // rows as tiles of rows have them: of 64 at most for few, else of 128 or 256
  TRY(p.few ? p.split_rows % 64 == 0 : p.split_rows % 256 == 0, "tiles of rows");
  // state and what is known of each row
  TRY(p.idx - p.state >= sizeof(VocabState) + 4 && p.target - p.idx >= 4 * p.rp && p.map - p.target >= 4 * p.rp && p.weight - p.map >= 4 * p.rp && p.zt - p.weight >= 4 * p.rp &&
          p.row_loss - p.zt >= 4 * p.rp && p.row_w - p.row_loss >= 4 * p.rp && p.row - p.row_w >= 4 * p.rp && p.parts - p.row >= sizeof(VocabRow) * p.rp, "rows");
  // the tiles' parts: of few rows those of each launch (what lies before the last piece, and that) begin anew
  size_t tiles = p.tiles;
  if (p.few) {
    const size_t made = (last + p.height - 1) / p.height + (vocab - last + p.height - 1) / p.height;
    TRY(made <= p.tiles, "tiles");
    TRY(p.height % 4 == 0 && p.height <= (p.lone ? 64 : 64 * (size_t)p.mt), "height");
  }
  TRY(p.x - p.parts >= 8 * tiles * p.split_rows, "parts");
  TRY(p.x_plane >= p.split_rows * p.dp && p.w - p.x >= 2 * reach(planes, p.x_plane, p.split_rows, p.dp), "hidden");
  if (!p.few) TRY(p.w_plane >= p.vp * p.dp && p.dz - p.w >= 2 * reach(planes, p.w_plane, p.vp, p.dp), "weight");
  if (grad) {
    TRY(p.dz_plane >= p.split_rows * p.vp && p.z - p.dz >= 2 * reach(planes, p.dz_plane, p.split_rows, p.vp), "dz");
    if (p.keep || p.few) TRY(p.dx - p.z >= 4 * p.split_rows * p.vp, "logits");
    TRY(p.bytes - p.dx >= 4 * p.splits * p.split_rows * p.dq && p.splits >= 1, "dX");
  }
  TRY(vocab_plan(rows, dim, vocab, dtype, grad, piece, !aligned).bytes == p.bytes, "alignment changes the space");
  for (size_t more : {rows + 1, (size_t)128, (size_t)129, (size_t)256, (size_t)1024, (size_t)5000, (size_t)65536, 2 * rows})
    if (more >= rows) TRY(vocab_plan(more, dim, vocab, dtype, grad, piece, true).bytes >= p.bytes, "more rows have less room");
#undef TRY
  return 0;
}

}  // namespace

int main(int argc, char** argv) {
  if (argc == 7) {
    const size_t rows = strtoull(argv[1], nullptr, 10), dim = strtoull(argv[2], nullptr, 10), vocab = strtoull(argv[3], nullptr, 10), piece = strtoull(argv[5], nullptr, 10);
    const VocabPlan p = vocab_plan(rows, dim, vocab, atoi(argv[4]), true, piece, atoi(argv[6]) != 0);
    printf("few=%d keep=%d lone=%d nt=%d mt=%d wide=%zu steps=%zu pieces=%zu vp=%zu splits=%zu dx_wide=%d dw_wide=%d\n", p.few, p.keep, p.lone, p.nt, p.mt, p.wide, p.dp / kGemmK, (vocab + p.vp - 1) / p.vp, p.vp,
           p.splits, !p.few && !p.dx_quarters, !p.few && !p.dw_quarters);
    return 0;
  }
  int wrong = 0;
  for (int dtype : {(int)DFX_F32, (int)DFX_BF16, (int)DFX_F16})
    for (size_t dim : {1, 63, 64, 65, 256, 1001, 1024, 4096, 70000})
      for (size_t vocab : {0, 1, 255, 256, 257, 1000, 8192, 32000, 50257, 65536, 65537, 78592, 78593, 100000, 131072, 131073, 300000, 524288, 524289, 3000000})
        for (size_t rows : {0, 1, 16, 17, 32, 33, 64, 65, 127, 128, 129, 255, 256, 257, 1000, 1024, 1025, 8192, 40000})
          for (size_t piece : {0, 256, 768, 65536, 1 << 20, 1 << 22, 1 << 24})
            for (int how = 0; how < 4; ++how) wrong += wrong < 20 ? look(rows, dim, vocab, dtype, how & 1, piece, how >> 1) : 0;
  if (!wrong) puts("ok");
  return wrong != 0;
}

// How a call of the vocabulary's loss is laid out: which products it takes, in which tiles and pieces, and where things lie in its workspace.  Pure functions, compiled with the kernels
// (dfx_vocab.hip, dfx_gemm.h) and by themselves for the host (tests/rules/vocab_plan_check.cpp walks them without a GPU).
#ifndef DFX_VOCAB_PLAN_H
#define DFX_VOCAB_PLAN_H

#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/dfx.h"

namespace {

constexpr int kGemmK = 64;               // elements of k in a step: 128 bytes of a row
constexpr uint32_t kFewK = 128;          // rows of W in a step of dX of few rows

constexpr int gemm_planes(int dt) { return dt == DFX_F32 ? 3 : 1; }
constexpr int gemm_pairs(int dt) { return dt == DFX_F32 ? 6 : 1; }
constexpr int gemm_few_e(int dt, int nt) { return dt != DFX_F32 && nt == 2 ? 8 : 4; }      // elements of eight rows of W that a lane reads for dX of few rows

struct VocabState { uint32_t count; float g; };       // what is known of a call on the device, first in the workspace: rows that count; scale * largest weight * c / 2^15
struct VocabRow { float m, f, w; int32_t t; };        // largest logit, w / S, w R / S (w: the row's weight, relative, times 2^15), target

constexpr size_t kTileRows = 256;        // rows of hidden and of weight are padded to tiles of so many

// Up to so many rows of at least so many elements go by the products for few rows, which read the weight as it lies (us, by them and by wide tiles with gradients: 64 x 2048 x 32000
// bf16 97 and 117, 64 x 1024 x 32000 in 32 bits 153 and 277; 128 rows 126 and 127, 252 and 295; between 65 and 128 bf16 rows -10 % to +19 %, the better the longer the vocabulary).
constexpr uint32_t kFewRows = 128, kFewDim = 64;
// Elements of dz that are held at a time, and with them the logits of the last piece in 32 bits (8192 x 4096 x 131072: 2^26 24.1 ms, 2^27 23.8, 2^28 23.5: 1.6 GB of a
// workspace of 2.4, which has 0.5 for a weight that cannot be read where it lies; all of it, 2^30, 6.4 of 7.8 GB, a seventh less); rows of a piece at least, at most, of few rows, and where the caller says (offsets within a tile of dz have 32 bits).
constexpr size_t kPieceElems = 256ull << 20, kPieceLeast = 1024, kPieceMost = 65536, kPieceFew = 1ull << 19, kPieceEver = 1ull << 22;
// From so long a vocabulary on, few rows' logits are made by twice as many rows of an unaligned or 32-bit weight to a workgroup (40 x 2001 x 100000 bf16 184 us and 195 by half as many, but 66 x
// 1789 x 30000 in 32 bits 140 and 94).
constexpr size_t kFewWide = 65536;
// The last piece's logits are kept, in 32 bits, where making them again takes longer than writing and reading them: of long rows (us, kept and not: 8192 x 512 x 32768 bf16 1255 and 1143,
// x 1024 1820 and 1931, x 2048 2998 and 3433; 4096 x 128 x 16384 in 32 bits 576 and 552, x 256 810 and 855), and of so few that a launch counts
// (256 elements: 1024 x 8192 55 and 57, 2048 x 16000 146 and 131).
constexpr size_t kKeepDim = 1024, kKeepDimF32 = 256, kKeepElems = 16ull << 20;

inline size_t up(size_t n, size_t to) { return (n + to - 1) / to * to; }

struct VocabPlan {
  size_t rp, dp, dq, vp, pieces, tiles, splits, split_rows;      // rows and elements padded, dX's pitch, rows of a piece, pieces, tiles of the vocabulary, splits of dX and the tiles' rows
  bool few, keep;                        // keep: the logits of the last piece
  int lone;                              // x stays in registers, 32 times so many elements of a wave; or 0
  int nt, mt;                            // tiles of the products for few rows
  size_t height;                         // of a tile of the vocabulary, for few rows
  size_t wide;                           // otherwise: rows of the vocabulary whose logits go by wide tiles, the others' by quarters
  bool dx_quarters, dw_quarters;         // whether the gradients' products do
  size_t x_plane, w_plane, dz_plane;     // elements from one plane to the next
  size_t state, idx, target, map, weight, zt, row_loss, row_w, row, parts, x, w, dz, z, dx, bytes;      // places in the workspace
};

// Whether logits go by workgroups that keep x, and 32 times how many elements of it each of the eight waves has: not where an eighth of those would lie behind a row's end (us by
// them and by the others, bf16 of 1 row by 32000, the weight in the caches: 1024 elements 19.6 and 20.9, 1001 28.1 and 31.8, 1531 42.3 and 46.2, but 1600 28.2 and 26.4, 3200 45.2 and 40.5; from
// HBM, by 50257: 2000 49 and 62, 2048 53 and 57).
inline int vocab_lone(size_t rows, size_t dim, int dtype) {
  if (rows > (dtype == DFX_F32 ? 16 : 32)) return 0;
  for (int kk : {4, 6, 8, 12, 16}) {
    if (kk > (dtype == DFX_F32 || rows > 16 ? 8 : 16)) break;
    const size_t all = 256 * (size_t)kk;
    if (dim <= all) return dim * 8 > all * 7 ? kk : 0;
  }
  return 0;
}

// How long a launch takes of workgroups, one to a compute unit, of two kinds: n of length l each, the longer ones first.
inline double vocab_time(size_t n, double l, size_t n2, double l2) {
  if (l2 > l) { std::swap(n, n2); std::swap(l, l2); }
  const size_t some = n % 256;           // compute units that have one more of the long ones
  const double early = (double)(n / 256) * l, late = some ? early + l : early;
  if (!n2) return late;
  auto done = [&](double t) { return (double)(256 - some) * floor((t - early) / l2 + 1e-9) + (t > late ? (double)some * floor((t - late) / l2 + 1e-9) : 0.0); };
  double k = std::max(1.0, std::max(floor((double)n2 / 256), std::min(ceil((double)n2 / (double)(256 - some)), floor((late - early) / l2))));
  while (done(early + k * l2) < (double)n2) k += 1;
  const double t = early + k * l2, other = t > late ? late + floor((t - late) / l2) * l2 : late;      // (those that come behind the late ones may be the last)
  return std::max(late, other < t && done(other) >= (double)n2 ? other : t);
}

// Tiles of the products of many rows, and splits of dX: what takes the shortest time where a wide tile takes a unit for a step of k and as long as 8 steps besides, and a quarter of it
// 0.4 of both (4096 x 2048 x 8192, logits: 65 us and 25; dW: 117 and 45).
constexpr double kQuarter = 0.4;
inline void vocab_tiles(VocabPlan& p, size_t rows, size_t dim, size_t vocab, size_t pairs) {
  auto over = [](size_t n, size_t by) { return (n + by - 1) / by; };
  const size_t n4 = over(rows, 256), n1 = over(rows, 128), v4 = over(vocab, 256), m4 = over(dim, 256), m1 = over(dim, 128);
  const double logits = (double)(p.dp / kGemmK * pairs) + 8;
  double best = 1e300;
  for (size_t wide : {v4, v4 * n4 / 256 * 256 / n4, (size_t)0}) {
    const double t = vocab_time(wide * n4, logits, n1 * (wide < v4 ? over(vocab - wide * 256, 128) : 0), kQuarter * logits);
    if (t < best) { best = t; p.wide = wide * 256; }
  }
  p.tiles = p.wide / 256 + over(vocab > p.wide ? vocab - p.wide : 0, 128);
  const size_t most = std::max<size_t>(1, std::min(256 / (p.rp / 256 * m4), p.vp / 256)), steps = p.vp / kGemmK;
  const double dw = (double)(over(rows, kGemmK) * pairs) + 8;
  best = 1e300;
  for (int kind = 0; kind < 4; ++kind) {
    const bool xq = kind & 1, wq = kind >> 1;
    for (size_t part = 1; part <= 16; ++part) {
      const size_t splits = over(most * part, 16);
      const double dx = (double)(over(steps, splits) * pairs) + 8;
      const double t = vocab_time(splits * (xq ? n1 * m1 : n4 * m4), xq ? kQuarter * dx : dx, wq ? m1 * over(p.vp, 128) : m4 * (p.vp / 256), wq ? kQuarter * dw : dw) + (double)(splits * rows * dim) * 0.5e-6;
      if (t < best) { best = t; p.splits = splits; p.dx_quarters = xq; p.dw_quarters = wq; }
    }
  }
}

// Splits of dX along the vocabulary: as many workgroups as compute units, of the products for few rows three times as many.  What depends on the number of rows has room for
// any smaller number.  aligned: rows of weight lie at multiples of 16 bytes (which changes nothing of the space).
inline VocabPlan vocab_plan(size_t rows, size_t dim, size_t vocab, int dtype, bool grad, size_t piece, bool aligned) {
  VocabPlan p = {};
  const size_t planes = gemm_planes(dtype);
  p.few = rows <= kFewRows && dim >= kFewDim;
  p.lone = 0;
  p.rp = std::max(kTileRows, up(rows, kTileRows));
  p.dp = up(dim, kGemmK);
  p.dq = up(dim, 4);
  const size_t whole = std::max(kTileRows, up(vocab, kTileRows));
  const size_t most = std::min(whole, piece ? std::min(piece, kPieceEver) : kPieceMost), few_most = std::min(whole, piece ? std::min(piece, kPieceEver) : kPieceFew);
  const bool long_rows = dim >= (dtype == DFX_F32 ? kKeepDimF32 : kKeepDim);
  size_t length = most, dz = p.rp * most;
  if (!piece) {
    length = std::min(most, std::max(kPieceLeast, kPieceElems / p.rp / kTileRows * kTileRows));
    dz = std::min(dz, std::max(kPieceElems, p.rp * kPieceLeast));
  }
  if (p.few) length = few_most;
  p.pieces = (whole + length - 1) / length;
  p.vp = piece ? length : up((whole + p.pieces - 1) / p.pieces, kTileRows);      // (of equal length)
  p.keep = grad && (p.few || long_rows || p.rp * p.vp <= kKeepElems);
  if (p.few) {
    p.nt = rows <= 32 ? 2 : 4;
    p.lone = vocab_lone(rows, dim, dtype);
    p.mt = !p.lone && (aligned || vocab >= kFewWide) ? 2 : 1;
    // so many tiles that whole rounds of workgroups, two to a compute unit, have them all
    const size_t rounds = std::max<size_t>(1, (vocab + 512 * 64 * p.mt - 1) / (512 * 64 * p.mt));
    p.height = std::max<size_t>(16, up((vocab + 512 * rounds - 1) / (512 * rounds), 4));
    p.tiles = (vocab + p.height - 1) / p.height + p.pieces;      // (of each piece by itself)
    p.split_rows = up(std::max<size_t>(rows, 1), 64);
    const size_t dx_wide = 16 * gemm_few_e(dtype, p.nt), groups = up(std::max<size_t>(rows, 1), 16 * p.nt) / (16 * p.nt) * (up(dim, dx_wide) / dx_wide);
    p.splits = std::max<size_t>(1, std::min(768 / groups, p.vp / kFewK));
  } else {
    p.height = 0;
    p.split_rows = p.rp;
    vocab_tiles(p, std::max<size_t>(rows, 1), dim, vocab, gemm_pairs(dtype));
  }
  p.x_plane = p.rp * p.dp;
  p.w_plane = p.vp * p.dp;
  p.dz_plane = p.split_rows * p.vp;
  size_t at = 0;
  auto take = [&](size_t n) { const size_t here = at; at += up(n, 256); return here; };
  p.state = take(sizeof(VocabState) + 4);
  p.idx = take(4 * p.rp); p.target = take(4 * p.rp); p.map = take(4 * p.rp); p.weight = take(4 * p.rp); p.zt = take(4 * p.rp);
  p.row_loss = take(4 * p.rp); p.row_w = take(4 * p.rp); p.row = take(sizeof(VocabRow) * p.rp);
  p.parts = take(2 * sizeof(float) * std::max<size_t>(p.rp * (whole / 128), kFewRows * std::min(whole / 4, whole / 32 + 520)));
  p.x = take(planes * p.rp * p.dp * 2);
  p.w = p.few ? at : take(planes * most * p.dp * 2);
  p.dz = grad ? take(planes * std::max(dz, kFewRows * few_most) * 2) : at;
  p.z = grad ? take(std::max(long_rows ? dz : std::min(dz, kKeepElems), kFewRows * few_most) * 4) : at;
  p.dx = grad ? take(std::max(std::max(256 / (up(dim, 256) / 256), p.rp / 256) * 256, std::max<size_t>(768 / (up(dim, 128) / 128), 1) * kFewRows) * p.dq * 4) : at;
  p.bytes = at;
  return p;
}

// a launch's threads are counted in 32 bits: workgroups of 512 to each tile of the vocabulary by 128 rows at least
inline bool vocab_too_large(const VocabPlan& p) { return p.rp / 128 * p.tiles >= (1ull << 23) - 8; }

}  // namespace

#endif

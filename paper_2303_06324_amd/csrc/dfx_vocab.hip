// Softmax cross entropy over a vocabulary whose logits are never kept, and its gradients: the head of a language model and the loss in one.
//
// With z = hidden weight^T and, for a row, m its largest logit, R = the sum of exp(c (z - m)) but for the target's and S = R + exp(c (z_t - m)):  logp = c (z_t - m) - log S, or
// -log(1 + R) where the target's is the largest, and its dz = -R / S: so that a token that is expected keeps the digits of what is missing from 1.  Tiles of z are made on the matrix
// cores and reduced to (m, R) of each row where they lie; a second kernel joins the tiles' parts.  For the gradients a piece of the vocabulary at
// a time is made again (the last one's logits may be kept), turned into dz = softmax - [target], and goes as the operand into dX += dz W and dW = dz^T X.
//
// Rows that have nothing to learn from are left out first: the others' hidden states are laid one behind the other (and padded to whole steps of
// the products), so that masked rows cost nothing.
//
// dz is held relative to the largest weight of a row and times 2^15, which is at most 2^15 in size: in f16 a probability keeps its digits down to 2e-9
// instead of 6e-5.  What is left out comes back as one factor in 32 bits behind the products.
#include <float.h>
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>

#include "dfx_gemm.h"
#include "dfx_vocab_plan.h"

namespace {

constexpr double kVLog2 = 0.69314718055994530942, kVLog2e = 1.44269504088896340736;
constexpr float kDzScale = 32768.0f;
constexpr uint32_t kRowsThreads = 1024;
// Up to so many rows are found by every workgroup that lays one out, which spares a launch (1024 x 1024 x 2000: 23.4 us and 24.1).
constexpr uint32_t kLayRows = 1024;
// Workgroups of dW of few rows (48 x 1024 x 32000 f16 and 8 x 3840 x 72397 bf16: 768 20.3 and 142 us, 1024 20.0 and 141, 2048 20.0 and 150).
constexpr uint32_t kDwGroups = 1024;
// Rows of a vocabulary whose tiles' parts are joined by a workgroup for each row, with gradients by each of dz's, which spares a launch (200 x 512 x 8000 43.9 us and 46.0, 1024 x 512 x 16000 level);
// of few rows, whose parts lie together (8 x 512 x 60000 78.7 and 81.4, 128 rows 92.3 and 94.0).
constexpr size_t kJoinMost = 16384, kJoinFew = 65536;

struct VocabArgs {
  const int64_t* targets;
  const float *row_weight, *scale;
  float *logp, *loss, *sums;
  VocabState* state;
  int32_t *idx, *target, *map;           // [Rp] rows that count, their targets (-1 behind them); [rows] where a row went, or -1
  float *weight, *zt, *row_loss, *row_w; // [Rp]
  float* top_weight;                     // largest |weight|
  VocabRow* row;                         // [Rp]
  float2* parts;                         // (m, R) of a tile's part of a row, at tile * tile_step + row * row_step: of many rows beside each other as a tile has them, of few a row's tiles
  uint16_t* x;                           // the rows that count, of 16 bits (null: of 32, whose infinite hidden states give NaN)
  uint32_t rows, rp, tile_step, row_step, vocab, tiles, dp;      // dp: elements of a row of x
  double c;
  float k;                               // c / log 2
};

__device__ __forceinline__ float vocab_base(float m) { return m == -INFINITY ? 0.0f : m; }
__device__ __forceinline__ float vocab_exp(float z, float base, float k) { return __builtin_amdgcn_exp2f((z - base) * k); }

__device__ __forceinline__ void vocab_state(const VocabArgs& a, uint32_t count, float top) {
  a.state->count = count;
  a.state->g = count ? (float)((a.scale ? (double)a.scale[0] : 1.0) * (double)top * a.c / (double)kDzScale) : 0.0f;
  *a.top_weight = top;
}

// The rows that count, in their order, by one workgroup; logp and loss of the others.  8192 rows 12.7 us, a chain of rounds of 1024.
__global__ void __launch_bounds__(kRowsThreads) dfx_vocab_rows_kernel(VocabArgs a) {
  constexpr uint32_t W = kRowsThreads / kStepWave;
  __shared__ uint32_t counts[2][W];
  __shared__ float tops[W];
  const uint32_t me = threadIdx.x, wave = me / kStepWave, lane = me % kStepWave;
  uint32_t done = 0, turn = 0;
  float top = 0.0f;
  for (uint32_t first = 0; first < a.rows; first += kRowsThreads, turn ^= 1u) {
    const uint32_t i = first + me;
    const int64_t t = i < a.rows ? a.targets[i] : -1;
    const float w = i < a.rows && a.row_weight ? a.row_weight[i] : 1.0f;
    const bool counts_here = t >= 0 && t < (int64_t)a.vocab && w != 0.0f;
    const uint64_t mask = __ballot(counts_here);
    if (lane == 0) counts[turn][wave] = (uint32_t)__popcll(mask);
    __syncthreads();
    uint32_t before = 0, all = 0;
    for (uint32_t k = 0; k < W; ++k) {
      before += k < wave ? counts[turn][k] : 0u;
      all += counts[turn][k];
    }
    const uint32_t place = done + before + (uint32_t)__popcll(mask & ((1ull << lane) - 1ull));
    if (i < a.rows) {
      a.map[i] = counts_here ? (int32_t)place : -1;
      if (counts_here) {
        a.idx[place] = (int32_t)i; a.target[place] = (int32_t)t; a.weight[place] = w;
        top = fmaxf(top, fabsf(w));
      } else {
        if (a.logp) a.logp[i] = 0.0f;
        if (a.loss) a.loss[i] = 0.0f;
      }
    }
    done += all;
  }
  for (uint32_t i = done + me; i < a.rp; i += kRowsThreads) {
    a.idx[i] = -1; a.target[i] = -1; a.weight[i] = 0.0f;
  }
  top = __uint_as_float(wave_max(__float_as_uint(top)));      // (none is negative)
  if (lane == 0) tops[wave] = top;
  __syncthreads();
  if (me == 0) {
    for (uint32_t k = 1; k < W; ++k) top = fmaxf(top, tops[k]);
    top = fmaxf(top, tops[0]);
    vocab_state(a, done, top);
  }
}

// A row of a matrix for the products, by a workgroup: padded with zeros to whole steps, 32 bits cut into planes.  null: zeros.
template <int DT>
__device__ __forceinline__ void pack_row(const void* row, uint32_t dim, uint32_t padded, uint16_t* to, size_t plane) {
  for (uint32_t e = threadIdx.x * 8u; e < padded; e += 256u * 8u) {
    if constexpr (DT == DFX_F32) {
      float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (row) {
        if (e + 8u <= dim) {
          StepVec<DT, 4> lo, hi;
          lo.load(row, e); hi.load(row, e + 4u);
#pragma unroll
          for (int j = 0; j < 4; ++j) { v[j] = lo.get(j); v[4 + j] = hi.get(j); }
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (e + j < dim) v[j] = step_get<DT>(row, e + j);
        }
      }
      uint32_t p[3][4];
      gemm_cut8(v, p);
#pragma unroll
      for (int q = 0; q < 3; ++q) *(uint4*)(to + q * plane + e) = make_uint4(p[q][0], p[q][1], p[q][2], p[q][3]);
    } else {
      StepVec<DT, 8> v;
      v.w = 0;
      if (row) {
        if (e + 8u <= dim) v.load(row, e);
        else {
          uint16_t x[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) x[j] = e + j < dim ? *((const STEP_GLOBAL uint16_t*)row + e + j) : (uint16_t)0;
          memcpy(&v.w, x, 16);
        }
      }
      *(uint4*)(to + e) = make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]);
    }
  }
}

// idx: which rows (-1: zeros), or null: row for row.  HBM bounds it: 50257 x 1001 in 32 bits 77 us, 0.50 GB.
template <int DT>
__global__ void __launch_bounds__(256) dfx_vocab_pack_kernel(const void* src, size_t stride, const int32_t* idx, uint32_t dim, uint32_t padded, uint16_t* dst, size_t plane) {
  const uint32_t r = blockIdx.x;
  const int64_t from = idx ? (int64_t)idx[r] : (int64_t)r;
  pack_row<DT>(from < 0 ? nullptr : (const unsigned char*)src + (size_t)from * stride * step_elem_bytes(DT), dim, padded, dst + (size_t)r * padded, plane);
}

// The same for up to kLayRows rows in one launch with what dfx_vocab_rows_kernel does: every workgroup finds the rows that count, and lays out the one of its number.  4.2 us for 48, 6.5 for 1023.
template <int DT>
__global__ void __launch_bounds__(256) dfx_vocab_lay_kernel(VocabArgs a, const void* src, size_t stride, uint32_t dim, uint32_t padded, uint16_t* dst, size_t plane) {
  constexpr uint32_t R = kLayRows / 256u;
  __shared__ uint32_t counts[R][4];
  __shared__ float tops[4];
  __shared__ int32_t mine;
  const uint32_t me = threadIdx.x, wave = me / kStepWave, lane = me % kStepWave;
  int64_t t[R];
  float w[R], top = 0.0f;
  uint64_t mask[R];
#pragma unroll
  for (uint32_t r = 0; r < R; ++r) {
    const uint32_t i = r * 256u + me;
    t[r] = i < a.rows ? a.targets[i] : -1;
    w[r] = i < a.rows && a.row_weight ? a.row_weight[i] : 1.0f;
  }
#pragma unroll
  for (uint32_t r = 0; r < R; ++r) {
    const bool counts_here = t[r] >= 0 && t[r] < (int64_t)a.vocab && w[r] != 0.0f;
    mask[r] = __ballot(counts_here);
    if (counts_here) top = fmaxf(top, fabsf(w[r]));
    if (lane == 0) counts[r][wave] = (uint32_t)__popcll(mask[r]);
  }
  top = __uint_as_float(wave_max(__float_as_uint(top)));
  if (lane == 0) tops[wave] = top;
  if (me == 0) mine = -1;
  __syncthreads();
  uint32_t done = 0;
#pragma unroll
  for (uint32_t r = 0; r < R; ++r) {
    uint32_t place = done + (uint32_t)__popcll(mask[r] & ((1ull << lane) - 1ull));
    for (uint32_t k = 0; k < 4; ++k) {
      place += k < wave ? counts[r][k] : 0u;
      done += counts[r][k];
    }
    const bool counts_here = mask[r] >> lane & 1u;
    const uint32_t i = r * 256u + me;
    if (counts_here && place == blockIdx.x) mine = (int32_t)i;
    if (blockIdx.x == 0 && i < a.rows) {
      a.map[i] = counts_here ? (int32_t)place : -1;
      if (counts_here) {
        a.idx[place] = (int32_t)i; a.target[place] = (int32_t)t[r]; a.weight[place] = w[r];
      } else {
        if (a.logp) a.logp[i] = 0.0f;
        if (a.loss) a.loss[i] = 0.0f;
      }
    }
  }
  if (blockIdx.x == 0) {
    for (uint32_t i = done + me; i < a.rp; i += 256u) {
      a.idx[i] = -1; a.target[i] = -1; a.weight[i] = 0.0f;
    }
    if (me == 0) vocab_state(a, done, fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])));
  }
  __syncthreads();
  pack_row<DT>(mine < 0 ? nullptr : (const unsigned char*)src + (size_t)mine * stride * step_elem_bytes(DT), dim, padded, dst + (size_t)blockIdx.x * padded, plane);
}

// A tile's part of each row: (m, R), and the target's logit where it lies here; for the last piece of a call with gradients the logits as well.
struct VocabStats {
  float2* parts;
  float *zt, *z;                         // z: rows of z_pitch, may be null
  const int32_t* target;
  uint32_t tile_step, row_step, z_pitch, left, v0, tile0, height;      // left: rows of the vocabulary from the first of this launch, v0, on; tile0: its first tile; height: of a tile, 0: all of it
  float k;
  template <class TILE>
  __device__ __forceinline__ void operator()(const TILE& tile, const GemmPlace& at, GemmAcc (&acc)[TILE::MT][TILE::NT], unsigned char* lds) const {
    const uint32_t lane = threadIdx.x % kStepWave, wave = threadIdx.x / kStepWave;
    const uint32_t end = min(left, tile.m0 + (height ? height : (uint32_t)TILE::M));
    if (tile.m0 + TILE::M > end) {
#pragma unroll
      for (int i = 0; i < TILE::MT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (tile.m(i) + e >= end)
#pragma unroll
            for (int j = 0; j < TILE::NT; ++j) acc[i][j][e] = -INFINITY;
    }
    if (z)
#pragma unroll
      for (int j = 0; j < TILE::NT; ++j) {
        float* to = z + (size_t)tile.n(j) * z_pitch;
#pragma unroll
        for (int i = 0; i < TILE::MT; ++i)
          if (tile.m(i) < end) *(GemmAcc*)(to + tile.m(i)) = acc[i][j];      // (heights are multiples of 4, and what is behind the vocabulary is not looked at)
      }
    if (!parts) return;                  // (they are known: the logits alone)
    float2* part = (float2*)lds;         // [WM][N]
    __syncthreads();
#pragma unroll
    for (int j = 0; j < TILE::NT; ++j) {
      const uint32_t n = tile.n(j), t = (uint32_t)target[n] - v0;      // (none: far beyond)
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < TILE::MT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) top = fmaxf(top, acc[i][j][e]);
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      if (t >= tile.m0 && t < end)       // (few rows of a tile have their target in it)
#pragma unroll
        for (int i = 0; i < TILE::MT; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (tile.m(i) + e == t) {
              zt[n] = acc[i][j][e];
              acc[i][j][e] = -INFINITY;
            }
      const float base = vocab_base(top);
      float s = 0.0f;
#pragma unroll
      for (int i = 0; i < TILE::MT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) s += vocab_exp(acc[i][j][e], base, k);
      s += __shfl_xor(s, 16);
      s += __shfl_xor(s, 32);
      if (lane < 16) part[wave / TILE::WN * TILE::N + (n - tile.n0)] = make_float2(top, s);
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < TILE::N; i += TILE::THREADS) {
      float2 p[TILE::WM];
      float top = -INFINITY, s = 0.0f;
#pragma unroll
      for (int w = 0; w < TILE::WM; ++w) {
        p[w] = part[w * TILE::N + i];
        top = fmaxf(top, p[w].x);
      }
#pragma unroll
      for (int w = 0; w < TILE::WM; ++w) s += p[w].y * vocab_exp(p[w].x, vocab_base(top), k);
      parts[(size_t)(tile0 + at.m) * tile_step + (size_t)(tile.n0 + i) * row_step] = make_float2(top, s);
    }
  }
  // of 64 logits of N rows, four of a row in each of N 16 threads (thread i: row i % N, logits 4 (i / N) on); lds: 16 N pairs
  template <int N>
  __device__ __forceinline__ void of_fours(uint32_t tile, uint32_t m0, uint32_t end, GemmAcc v, float2* lds) const {
    const uint32_t n = threadIdx.x % N, four = threadIdx.x / N, m = m0 + four * 4u;
    float top = -INFINITY, s = 0.0f;
    if (four < 16u) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (m + e >= end) v[e] = -INFINITY;
      if (z && m < end) *(GemmAcc*)(z + (size_t)n * z_pitch + m) = v;
      const uint32_t t = (uint32_t)target[n] - v0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        top = fmaxf(top, v[e]);
        if (m + e == t && t < end) {
          zt[n] = v[e];
          v[e] = -INFINITY;
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) s += vocab_exp(v[e], vocab_base(top), k);
      lds[four * N + n] = make_float2(top, s);
    }
    if (!parts) return;
    __syncthreads();
    if (threadIdx.x >= N) return;
    for (uint32_t q = 1; q < 16; ++q) top = fmaxf(top, lds[q * N + n].x);
    s = 0.0f;
    for (uint32_t q = 0; q < 16; ++q) s += lds[q * N + n].y * vocab_exp(lds[q * N + n].x, vocab_base(top), k);
    parts[(size_t)(tile0 + tile) * tile_step + (size_t)n * row_step] = make_float2(top, s);
  }
};

// What the n-th of the rows that count comes to, of its largest logit and R; behind them: nothing.
__device__ __forceinline__ VocabRow row_end(const VocabArgs& a, uint32_t n, uint32_t count, float top, float s, bool writes) {
  VocabRow r = {0.0f, 0.0f, 0.0f, -1};
  float logp = 0.0f, loss = 0.0f, w = 0.0f;
  const bool none = n < count && top == -INFINITY && s == 0.0f && a.zt[n] == -INFINITY;      // no logit above -infinity, and the target's, which is not in R, no NaN
  if (n < count && !none) {
    const float base = vocab_base(top), et = vocab_exp(a.zt[n], base, a.k), all = s + et;
    w = a.weight[n];
    if (writes) {
      int two;
      const float f = frexpf(all, &two);
      logp = et == 1.0f ? (float)-log1p((double)s) : (float)(a.c * ((double)a.zt[n] - (double)base) - ((double)two + (double)__builtin_amdgcn_logf(f)) * kVLog2);
      loss = -w * logp;
    }
    const float relative = w / *a.top_weight * kDzScale;
    r = {base, relative / all, relative * (s / all), a.target[n]};
  }
  if (!writes) return r;
  a.row[n] = r;
  a.row_loss[n] = loss;
  a.row_w[n] = w;
  if (n < count) {
    if (a.logp) a.logp[a.idx[n]] = logp;
    if (a.loss) a.loss[a.idx[n]] = loss;
  }
  if (none && a.x)                       // its hidden state, which may be infinite, has no part in the products either: 0 times that is NaN
    for (uint32_t e = 0; e < a.dp; e += 8u) *(uint4*)(a.x + (size_t)n * a.dp + e) = make_uint4(0, 0, 0, 0);
  return r;
}

// The tiles' parts of a row joined by a workgroup of 256: where they are few (4.7 us as a launch of its own).  (Which way they are joined goes by the vocabulary alone, so that a row's logp is the same with
// gradients and without.)
__device__ __forceinline__ float2 join_row(const VocabArgs& a, uint32_t n, bool any) {
  __shared__ float2 lds[4];
  float top = -INFINITY, s = 0.0f;
  if (any)
    for (uint32_t t = threadIdx.x; t < a.tiles; t += 256u) {
      const float2 p = a.parts[(size_t)t * a.tile_step + (size_t)n * a.row_step];
      const float more = fmaxf(top, p.x), base = vocab_base(more);
      s = s * vocab_exp(top, base, a.k) + p.y * vocab_exp(p.x, base, a.k);
      top = more;
    }
  float most = top;
#pragma unroll
  for (uint32_t x = kStepWave / 2; x; x >>= 1) most = fmaxf(most, __shfl_xor(most, (int)x));
  s = wave_sum(s * vocab_exp(top, vocab_base(most), a.k));
  if (threadIdx.x % kStepWave == 0) lds[threadIdx.x / kStepWave] = make_float2(most, s);
  __syncthreads();
  top = fmaxf(fmaxf(lds[0].x, lds[1].x), fmaxf(lds[2].x, lds[3].x));
  s = 0.0f;
#pragma unroll
  for (int k = 0; k < 4; ++k) s += lds[k].y * vocab_exp(lds[k].x, vocab_base(top), a.k);
  return make_float2(top, s);
}
__global__ void __launch_bounds__(256) dfx_vocab_row_kernel(VocabArgs a) {
  const uint32_t n = blockIdx.x, count = a.state->count;
  const float2 all = join_row(a, n, n < count);
  if (threadIdx.x == 0) row_end(a, n, count, all.x, all.y, true);
}

// The tiles' parts of a row joined, and what it comes to.  S threads to a row: few where there are many rows.  512 tiles of 6700 rows 15.9 us.
template <uint32_t S>
__global__ void __launch_bounds__(256) dfx_vocab_join_kernel(VocabArgs a) {
  constexpr uint32_t R = 256 / S;
  __shared__ float2 lds[S][R];
  const uint32_t i = threadIdx.x % R, slice = threadIdx.x / R, n = blockIdx.x * R + i, count = a.state->count;
  float top = -INFINITY, s = 0.0f;
  if (n < count)
    for (uint32_t t = slice; t < a.tiles; t += 4u * S) {
      float2 p[4];
#pragma unroll
      for (uint32_t u = 0; u < 4; ++u) p[u] = t + u * S < a.tiles ? a.parts[(size_t)(t + u * S) * a.tile_step + (size_t)n * a.row_step] : make_float2(-INFINITY, 0.0f);
      float more = top;
#pragma unroll
      for (int u = 0; u < 4; ++u) more = fmaxf(more, p[u].x);
      const float base = vocab_base(more);
      s *= vocab_exp(top, base, a.k);
#pragma unroll
      for (int u = 0; u < 4; ++u) s += p[u].y * vocab_exp(p[u].x, base, a.k);
      top = more;
    }
  lds[slice][i] = make_float2(top, s);
  __syncthreads();
  if (slice || n >= a.rp) return;
  for (uint32_t k = 1; k < S; ++k) top = fmaxf(top, lds[k][i].x);
  s = 0.0f;
  for (uint32_t k = 0; k < S; ++k) s += lds[k][i].y * vocab_exp(lds[k][i].x, vocab_base(top), a.k);
  row_end(a, n, count, top, s, true);
}

// sums over the rows, in an order that is always the same, by a workgroup of 256
__device__ __forceinline__ void vocab_sums(const VocabArgs& a) {
  __shared__ double lds[2][4];
  double s = 0.0, w = 0.0;
  for (uint32_t i = threadIdx.x, n = a.state->count; i < n; i += 256u) {
    s += (double)a.row_loss[i];
    w += (double)a.row_w[i];
  }
  s = wave_sum(s); w = wave_sum(w);
  if (threadIdx.x % kStepWave == 0) {
    lds[0][threadIdx.x / kStepWave] = s;
    lds[1][threadIdx.x / kStepWave] = w;
  }
  __syncthreads();
  if (threadIdx.x < 2) a.sums[threadIdx.x] = (float)(lds[threadIdx.x][0] + lds[threadIdx.x][1] + lds[threadIdx.x][2] + lds[threadIdx.x][3]);
}
__global__ void __launch_bounds__(256) dfx_vocab_sums_kernel(VocabArgs a) { vocab_sums(a); }

// dz of a tile, to the type of the products: 16-bit inputs have it rounded once, to half a step of their type (two matrices of 16 bits are one product, one of 32 with one of 16 three, which would
// take three times as long).  8192 x 4096 x 131072 bf16: the gradients are 1.7e-3 of their norm from those of a dz in 32 bits, 48 x 1024 x 32000 f16 2.6e-4; their errors against 64 bits, the rounding
// of the results among them, grow by 10 to 30 %, of a single row up to twice.  The one scale for all rows keeps f16's steps at 2^-39 of the largest row weight and above: a row of a far smaller weight loses its small probabilities.
template <int DT>
struct VocabDz {
  const VocabRow* row;
  uint16_t* dz;                          // [Rp][pitch], planes of them
  size_t plane;
  uint32_t pitch, left, v0;
  float k;
  // of eight logits of a row
  __device__ __forceinline__ void put(uint32_t n, const VocabRow& r, uint32_t m, const float* z) const {
    const uint32_t t = (uint32_t)r.t - v0;
    uint16_t* to = dz + (size_t)n * pitch + m;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = r.f * vocab_exp(z[e], r.m, k);
      if (m + e == t) v[e] = -r.w;
      if (m + e >= left || r.t < 0) v[e] = 0.0f;      // (a row behind those that count may have NaN for logits: 0 times an infinite weight)
    }
    if constexpr (DT == DFX_F32) {
      uint32_t p[3][4];
      gemm_cut8(v, p);
#pragma unroll
      for (int q = 0; q < 3; ++q) *(uint4*)(to + q * plane) = make_uint4(p[q][0], p[q][1], p[q][2], p[q][3]);
    } else {
      StepVec<DT, 8> o;
      o.put(v);
      *(uint4*)to = make_uint4(o.w[0], o.w[1], o.w[2], o.w[3]);
    }
  }
  template <class TILE>
  __device__ __forceinline__ void operator()(const TILE& tile, const GemmPlace&, GemmAcc (&acc)[TILE::MT][TILE::NT], unsigned char* lds) const {
    gemm_by_rows<8>(tile, acc, lds, [&](uint32_t n, uint32_t m, const float* z) { put(n, row[n], m, z); });
  }
};

// dz of a piece whose logits were kept: a workgroup to 2048 logits of a row.  Rows behind those that count are 0 as far as the products take them.  JOIN: the row's parts are
// joined by each of its workgroups, which spares a launch where they are few.  HBM bounds it: 6700 x 32768 bf16 246 us, 1.3 GB; 921 x 50257 in 32 bits 84 us, 0.46 GB.
template <int DT, bool JOIN>
__global__ void __launch_bounds__(256) dfx_vocab_dz_kernel(VocabArgs a, VocabDz<DT> d, const float* z) {
  const uint32_t n = blockIdx.x, m = (blockIdx.y * 256u + threadIdx.x) * 8u, count = a.state->count;
  const bool in = m < d.pitch, any = n < count;
  float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  if (any && in && m < d.left) memcpy(v, __builtin_assume_aligned(z + (size_t)n * d.pitch + m, 16), 32);      // (left is rounded up to a multiple of 4 at most)
  VocabRow r = {0.0f, 0.0f, 0.0f, -1};
  if constexpr (JOIN) {
    const float2 all = join_row(a, n, any);
    r = row_end(a, n, count, all.x, all.y, blockIdx.y == 0 && threadIdx.x == 0);
  } else if (any) r = d.row[n];
  if (in && n < (count + kGemmK - 1) / kGemmK * kGemmK) d.put(n, r, m, v);
}

// a part of dX, in 32 bits: [splits][rows][pitch]
struct VocabDx {
  float* part;
  uint32_t rows, pitch;
  bool more;                             // not the first piece
  template <class TILE>
  __device__ __forceinline__ void operator()(const TILE& tile, const GemmPlace& at, GemmAcc (&acc)[TILE::MT][TILE::NT], unsigned char*) const {
#pragma unroll
    for (int j = 0; j < TILE::NT; ++j) {
      float* to = part + ((size_t)at.split * rows + tile.n(j)) * pitch;
#pragma unroll
      for (int i = 0; i < TILE::MT; ++i) {
        const uint32_t m = tile.m(i);
        if (m >= pitch) continue;
        GemmAcc* p = (GemmAcc*)(to + m);
        *p = more ? *p + acc[i][j] : acc[i][j];
      }
    }
  }
};

// rows of dW
template <int OUT>
struct VocabDw {
  void* grad;
  size_t stride;
  const VocabState* state;
  uint32_t dim, left;                    // elements of a row; rows from grad's first on
  bool accumulate;
  template <int E>
  __device__ __forceinline__ void put(uint32_t n, uint32_t m, float* v, float g) const {
    if (n >= left || m >= dim) return;
    typedef typename StepElem<OUT>::raw raw;
    raw* to = (raw*)grad + (size_t)n * stride;
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] *= g;
    if (m + E <= dim) {
      StepVec<OUT, E> o;
      if (accumulate) {
        o.load(to, m);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] += o.get(e);
      }
      o.put(v);
      *(STEP_GLOBAL typename StepVec<OUT, E>::words*)((STEP_GLOBAL raw*)to + m) = o.w;
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (m + e < dim) step_put<OUT>(to, m + e, accumulate ? v[e] + step_get<OUT>(to, m + e) : v[e]);
    }
  }
  __device__ __forceinline__ void put8(uint32_t n, uint32_t m, float* v) const {
    if constexpr (OUT == DFX_F32) {
      put<4>(n, m, v, state->g);
      put<4>(n, m + 4u, v + 4, state->g);
    } else put<8>(n, m, v, state->g);
  }
  template <class TILE>
  __device__ __forceinline__ void operator()(const TILE& tile, const GemmPlace&, GemmAcc (&acc)[TILE::MT][TILE::NT], unsigned char* lds) const {
    constexpr int E = 16 / (int)sizeof(typename StepElem<OUT>::raw);
    const float g = state->g;
    gemm_by_rows<E>(tile, acc, lds, [&](uint32_t n, uint32_t m, float* v) { put<E>(n, m, v, g); });
  }
};

// dX: the splits' parts, in their order; rows that do not count are 0.  A workgroup behind them makes the sums, where they are asked for.  6700 x 4096 of one split 31 us, 48 x 1024 of 48 splits 6.9.
template <int DT>
__global__ void __launch_bounds__(256) dfx_vocab_dx_kernel(VocabArgs a, const float* part, uint32_t splits, uint32_t split_rows, uint32_t pitch, void* grad, size_t stride, uint32_t dim) {
  const uint32_t row = blockIdx.x, e = (blockIdx.y * 256u + threadIdx.x) * 4u;
  if (row == a.rows) {                   // one more, for the sums
    if (blockIdx.y == 0) vocab_sums(a);
    return;
  }
  if (e >= dim) return;
  const int32_t n = a.map[row];
  const float g = a.state->g;
  typedef typename StepElem<DT>::raw raw;
  raw* to = (raw*)grad + (size_t)row * stride;
  float v[4] = {0, 0, 0, 0};
  if (n >= 0) {
    GemmAcc sum = *(const GemmAcc*)(part + (size_t)n * pitch + e);
#pragma unroll 8
    for (uint32_t s = 1; s < splits; ++s) sum += *(const GemmAcc*)(part + ((size_t)s * split_rows + n) * pitch + e);
    for (int q = 0; q < 4; ++q) v[q] = g * sum[q];
  }
  if (e + 4u <= dim) {
    StepVec<DT, 4> o;
    o.put(v);
    *(STEP_GLOBAL typename StepVec<DT, 4>::words*)((STEP_GLOBAL raw*)to + e) = o.w;
  } else {
    for (int q = 0; q < 4; ++q)
      if (e + q < dim) step_put<DT>(to, e + q, v[q]);
  }
}

// ------------------------------------------------------------------------------------------
// how a call is laid out
// ------------------------------------------------------------------------------------------
// Whether the weight can be read where it lies by loads to LDS: 16-bit rows of whole steps at multiples of 16 bytes.
bool vocab_aligned(const dfx_vocab_loss_args& u) {
  return u.dtype != DFX_F32 && u.dim % kGemmK == 0 && (uintptr_t)u.weight % 16 == 0 && (u.weight_stride ? u.weight_stride : u.dim) % 8 == 0;
}

// a product as workgroups of a launch from `from` on, of m by n elements
template <class EPI>
GemmTask<EPI> vocab_task(const GemmOperand& a, const GemmOperand& b, GemmShape s, size_t m, size_t n, const EPI& epi, bool quarters, uint32_t from) {
  const size_t tile = quarters ? 128 : 256;
  s.mtiles = (uint32_t)((m + tile - 1) / tile);
  s.ntiles = (uint32_t)((n + tile - 1) / tile);
  return {a, b, s, from, quarters, epi};
}

// what is made of logits, with wide tiles and with quarters
template <int DT, class EPI>
int vocab_logits(const GemmOperand& w, const GemmOperand& x, const GemmShape& s, size_t wide, size_t vocab, size_t rows, const EPI& epi, const EPI& epi_quarters, hipStream_t stream) {
  GemmOperand rest = w;
  rest.p += wide * w.stride; rest.rows = (uint32_t)(vocab - wide);
  const auto one = vocab_task(w, x, s, wide, rows, epi, false, 0);
  const auto two = vocab_task(rest, x, s, vocab - wide, rows, epi_quarters, true, gemm_groups(one.s));
  const uint32_t groups = two.from + gemm_groups(two.s);
  return groups ? step_launch(dfx_gemm_wide_kernel<DT, false, false, EPI>, dim3(groups), GemmWide::THREADS, stream, one, two) : DFX_OK;
}

// the products for few rows: logits, dX, dW
template <int DT, class EPI>
int vocab_few(const VocabPlan& p, bool aligned, const GemmSource& w, const GemmOperand& x, GemmShape s, size_t rows, const EPI& epi, hipStream_t stream) {
  s.mtiles = (uint32_t)((w.rows + p.height - 1) / p.height);
  s.height = (uint32_t)p.height;
  if (p.lone) {
    if (!s.mtiles || !rows) return DFX_OK;
    auto go = [&](auto k) { return step_launch(k, dim3(std::min(s.mtiles, p.lone == 4 ? 512u : 256u)), 512, stream, w, x, s.height, epi); };      // (what fits at once)
    if constexpr (DT != DFX_F32) {
      if (rows > 16) return p.lone == 4 ? go(dfx_gemm_lone_kernel<DT, 2, 4, EPI>) : p.lone == 6 ? go(dfx_gemm_lone_kernel<DT, 2, 6, EPI>) : go(dfx_gemm_lone_kernel<DT, 2, 8, EPI>);
      if (p.lone > 8) return p.lone == 12 ? go(dfx_gemm_lone_kernel<DT, 1, 12, EPI>) : go(dfx_gemm_lone_kernel<DT, 1, 16, EPI>);
    }
    return p.lone == 4 ? go(dfx_gemm_lone_kernel<DT, 1, 4, EPI>) : p.lone == 6 ? go(dfx_gemm_lone_kernel<DT, 1, 6, EPI>) : go(dfx_gemm_lone_kernel<DT, 1, 8, EPI>);
  }
  if constexpr (DT != DFX_F32)
    if (aligned) {
      s.ntiles = (uint32_t)((rows + 63) / 64);
      const GemmOperand a = {(const uint16_t*)w.p, 0, (uint32_t)w.stride, w.rows, w.dim};
      return s.mtiles && s.ntiles ? step_launch(p.height <= 64 ? dfx_gemm_flat_kernel<DT, 1, EPI> : dfx_gemm_flat_kernel<DT, 2, EPI>, dim3(gemm_groups(s)), 256, stream, a, x, s, epi) : DFX_OK;
    }
  s.ntiles = (uint32_t)((rows + 16 * p.nt - 1) / (16 * p.nt));
  if (!s.mtiles || !s.ntiles) return DFX_OK;
  constexpr int D2 = DT == DFX_F32 ? 3 : 4, D4 = DT == DFX_F32 ? 2 : 4;
  auto k = p.nt == 2 ? (p.mt == 2 ? dfx_gemm_few_kernel<DT, 2, 2, D2, EPI> : dfx_gemm_few_kernel<DT, 2, 1, D2, EPI>)
                     : (p.mt == 2 ? dfx_gemm_few_kernel<DT, 4, 2, D4, EPI> : dfx_gemm_few_kernel<DT, 4, 1, D4, EPI>);
  return step_launch(k, dim3(gemm_groups(s)), 256, stream, w, x, s, epi);
}

template <int DT>
int vocab_few_dx(const VocabPlan& p, const GemmSource& w, const GemmOperand& z, GemmShape s, size_t rows, float* dx, bool more, hipStream_t stream) {
  const uint32_t wide = 16 * gemm_few_e(DT, p.nt);
  s.mtiles = (w.dim + wide - 1) / wide;
  s.ntiles = (uint32_t)((rows + 16 * p.nt - 1) / (16 * p.nt));
  s.ksteps = (w.rows + kFewK - 1) / kFewK;
  if (!s.ntiles) return DFX_OK;
  return step_launch(p.nt == 2 ? dfx_gemm_few_dx_kernel<DT, 2> : dfx_gemm_few_dx_kernel<DT, 4>, dim3(gemm_groups(s)), 256, stream, w, z, s, dx, (uint32_t)p.split_rows, (uint32_t)p.dq, more);
}

template <int DT, class OUT>
int vocab_few_dw(const GemmOperand& x, const GemmOperand& z, const uint32_t* count, size_t rows, size_t dim, size_t vocab, const OUT& out, hipStream_t stream) {
  const uint32_t mtiles = (uint32_t)((dim + 127) / 128), ntiles = (uint32_t)((vocab + 63) / 64), each = std::min(ntiles, std::max(1u, kDwGroups / mtiles));
  return step_launch(rows <= kGemmK ? dfx_gemm_few_dw_kernel<DT, 1, OUT> : dfx_gemm_few_dw_kernel<DT, 2, OUT>, dim3(mtiles * each), 256, stream, x, z, count, mtiles, ntiles, each, out);
}

// dX and dW of a piece, or one of them, in one launch: the longer ones first
template <int DT, class DW>
int vocab_grads(const VocabPlan& p, const GemmOperand& w, const GemmOperand& z, const GemmShape& sx, size_t dim, size_t rows, const VocabDx* dx, const GemmOperand& x, const GemmShape& sw, size_t vocab, const DW* dw,
                hipStream_t stream) {
  auto one = vocab_task(w, z, sx, dx ? dim : 0, rows, dx ? *dx : VocabDx{}, p.dx_quarters, 0);
  auto two = vocab_task(x, z, sw, dw ? dim : 0, vocab, dw ? *dw : DW{}, p.dw_quarters, 0);
  const uint32_t n1 = gemm_groups(one.s), n2 = gemm_groups(two.s);
  const bool dw_first = (p.dw_quarters ? kQuarter : 1.0) * (double)((rows + kGemmK - 1) / kGemmK) > (p.dx_quarters ? kQuarter : 1.0) * (double)(sx.ksteps / sx.splits);
  if (dw_first) one.from = n2;
  else two.from = n1;
  return n1 + n2 ? step_launch(dfx_gemm_two_kernel<DT, true, false, VocabDx, true, true, DW>, dim3(n1 + n2), GemmWide::THREADS, stream, one, two) : DFX_OK;
}

#define VOCAB_TRY(call) do { const int rc_ = (call); if (rc_ != DFX_OK) return rc_; } while (0)

template <int DT>
int vocab_run(const dfx_vocab_loss_args& u, const VocabPlan& p, hipStream_t stream) {
  unsigned char* ws = (unsigned char*)u.workspace;
  VocabArgs a;
  memset(&a, 0, sizeof(a));
  a.targets = u.targets; a.row_weight = u.row_weight; a.scale = u.scale; a.logp = u.logp; a.loss = u.loss; a.sums = u.sums;
  a.state = (VocabState*)(ws + p.state); a.top_weight = (float*)(a.state + 1);
  a.idx = (int32_t*)(ws + p.idx); a.target = (int32_t*)(ws + p.target); a.map = (int32_t*)(ws + p.map); a.weight = (float*)(ws + p.weight);
  a.zt = (float*)(ws + p.zt); a.row_loss = (float*)(ws + p.row_loss); a.row_w = (float*)(ws + p.row_w); a.row = (VocabRow*)(ws + p.row);
  a.parts = (float2*)(ws + p.parts);
  a.rows = (uint32_t)u.rows; a.rp = (uint32_t)p.rp; a.tile_step = p.few ? 1u : (uint32_t)p.split_rows; a.row_step = p.few ? (uint32_t)p.tiles : 1u; a.vocab = (uint32_t)u.vocab; a.tiles = (uint32_t)p.tiles;
  a.c = u.inv_temperature; a.k = (float)(u.inv_temperature * kVLog2e);
  const size_t eb = step_elem_bytes(DT), ws_stride = u.weight_stride ? u.weight_stride : u.dim;
  const uint32_t* count = &a.state->count;
  uint16_t *x = (uint16_t*)(ws + p.x), *w = (uint16_t*)(ws + p.w), *dz = (uint16_t*)(ws + p.dz);
  float* dx = (float*)(ws + p.dx);
  a.x = DT == DFX_F32 ? nullptr : x; a.dp = (uint32_t)p.dp;

  const size_t hs = u.hidden_stride ? u.hidden_stride : u.dim;
  if (u.rows <= kLayRows) VOCAB_TRY(step_launch(dfx_vocab_lay_kernel<DT>, dim3((uint32_t)p.split_rows), 256, stream, a, u.hidden, hs, (uint32_t)u.dim, (uint32_t)p.dp, x, p.x_plane));
  else {
    VOCAB_TRY(step_launch(dfx_vocab_rows_kernel, dim3(1), kRowsThreads, stream, a));
    VOCAB_TRY(step_launch(dfx_vocab_pack_kernel<DT>, dim3((uint32_t)p.rp), 256, stream, u.hidden, hs, (const int32_t*)a.idx, (uint32_t)u.dim, (uint32_t)p.dp, x, p.x_plane));
  }
  // The weight is read where it lies if its rows are whole steps at multiples of 16 bytes; otherwise a piece at a time is laid out.
  // (The products for few rows take it as it is.)
  const bool direct = !p.few && vocab_aligned(u);
  const GemmOperand ox = {x, p.x_plane, (uint32_t)p.dp, (uint32_t)p.split_rows, (uint32_t)p.dp};
  const size_t pieces = (u.vocab + p.vp - 1) / p.vp;
  GemmOperand ow = {};
  auto take_piece = [&](size_t v0, size_t left) -> int {
    if (direct) {
      ow = {(const uint16_t*)u.weight + v0 * ws_stride, 0, (uint32_t)ws_stride, (uint32_t)left, (uint32_t)u.dim};
      return DFX_OK;
    }
    ow = {w, p.w_plane, (uint32_t)p.dp, (uint32_t)left, (uint32_t)p.dp};
    return step_launch(dfx_vocab_pack_kernel<DT>, dim3((uint32_t)left), 256, stream, (const void*)((const unsigned char*)u.weight + v0 * ws_stride * eb), ws_stride, (const int32_t*)nullptr,
                       (uint32_t)u.dim, (uint32_t)p.dp, w, p.w_plane);
  };
  const GemmShape by_rows = {0, 0, 1, (uint32_t)(p.dp / kGemmK), 0, count, false};
  const size_t last = pieces ? (pieces - 1) * p.vp : 0;
  float* z = p.keep ? (float*)(ws + p.z) : nullptr;
  size_t tile0 = 0;
  auto stats = [&](size_t v0, size_t left, float* keep, size_t tile, float2* parts) {
    return VocabStats{parts, a.zt, keep, a.target, a.tile_step, a.row_step, (uint32_t)p.vp, (uint32_t)left, (uint32_t)v0, (uint32_t)tile, (uint32_t)p.height, a.k};
  };
  GemmSource few_w = {};
  auto few_logits = [&](size_t v0, size_t left, const VocabStats& epi) -> int {      // of rows of weight from v0 on
    few_w = {(const unsigned char*)u.weight + v0 * ws_stride * eb, ws_stride, (uint32_t)left, (uint32_t)u.dim};
    return vocab_few<DT>(p, vocab_aligned(u), few_w, ox, by_rows, u.rows, epi, stream);
  };
  auto wide_of = [&](size_t v0, size_t left) { return p.wide > v0 ? std::min(p.wide - v0, left) : 0; };      // rows of a piece that go by wide tiles
  for (size_t v0 = 0, left; v0 < u.vocab; v0 += left) {      // what lies where it is in one launch, but for a piece whose logits are kept (of few rows always: their tiles begin with it)
    left = direct || p.few ? ((z || p.few) && v0 < last ? last : u.vocab) - v0 : std::min(p.vp, u.vocab - v0);
    if (!p.few) VOCAB_TRY(take_piece(v0, left));
    float* keep = v0 == last ? z : nullptr;
    if (p.few) {
      VOCAB_TRY(few_logits(v0, left, stats(v0, left, keep, tile0, a.parts)));
      tile0 += (left + p.height - 1) / p.height;
    } else {
      const size_t wide = wide_of(v0, left), v1 = v0 + wide;
      VOCAB_TRY((vocab_logits<DT>(ow, ox, by_rows, wide, left, u.rows, stats(v0, wide, keep, v0 / 256, a.parts), stats(v1, left - wide, keep ? keep + wide : nullptr, p.wide / 256 + (v1 - std::min(v1, p.wide)) / 128, a.parts), stream)));
    }
  }
  a.tiles = (uint32_t)(p.few ? tile0 : p.tiles);
  const bool grad = u.grad_hidden || u.grad_weight, by_row = u.vocab <= (p.few ? kJoinFew : kJoinMost), join = grad && z && pieces && by_row;
  if (!join) {
    if (by_row) VOCAB_TRY(step_launch(dfx_vocab_row_kernel, dim3((uint32_t)p.split_rows), 256, stream, a));
    else if (p.few) VOCAB_TRY(step_launch(dfx_vocab_join_kernel<64>, dim3((uint32_t)(p.rp / 4)), 256, stream, a));
    else VOCAB_TRY(step_launch(dfx_vocab_join_kernel<8>, dim3((uint32_t)(p.rp / 32)), 256, stream, a));
  }
  const bool sums_last = u.sums && u.grad_hidden && u.rows;
  if (u.sums && !sums_last && !join) VOCAB_TRY(step_launch(dfx_vocab_sums_kernel, dim3(1), 256, stream, a));
  if (!grad) return DFX_OK;
  for (size_t q = pieces; q-- != 0;) {   // the last one first
    const size_t v0 = q * p.vp, left = std::min(p.vp, u.vocab - v0);
    if (direct || (!p.few && v0 != last)) VOCAB_TRY(take_piece(v0, left));
    const VocabDz<DT> epi = {a.row, dz, p.dz_plane, (uint32_t)p.vp, (uint32_t)left, (uint32_t)v0, a.k};
    if (p.few && v0 != last) VOCAB_TRY(few_logits(v0, left, stats(v0, left, z, 0, nullptr)));
    if (p.few || (z && v0 == last))
      VOCAB_TRY(step_launch(join && v0 == last ? dfx_vocab_dz_kernel<DT, true> : dfx_vocab_dz_kernel<DT, false>, dim3((uint32_t)p.split_rows, (uint32_t)(p.vp / 8 + 255) / 256), 256, stream, a, epi, (const float*)z));
    else {
      const size_t wide = wide_of(v0, left);
      VOCAB_TRY((vocab_logits<DT>(ow, ox, by_rows, wide, left, u.rows, epi, VocabDz<DT>{a.row, dz + wide, p.dz_plane, (uint32_t)p.vp, (uint32_t)(left - wide), (uint32_t)(v0 + wide), a.k}, stream)));
    }
    const GemmOperand oz = {dz, p.dz_plane, (uint32_t)p.vp, (uint32_t)p.split_rows, (uint32_t)p.vp};
    const GemmShape sx = {0, 0, (uint32_t)p.splits, (uint32_t)((left + kGemmK - 1) / kGemmK), 0, count, false}, sw = {0, 0, 1, 0, 0, count, true};
    const VocabDx dx_to = {dx, (uint32_t)p.split_rows, (uint32_t)p.dq, v0 != last};
    const size_t gs = u.grad_weight_stride ? u.grad_weight_stride : u.dim;
    auto both = [&](const auto& dw_to) -> int {
      if (p.few) {
        few_w = {(const unsigned char*)u.weight + v0 * ws_stride * eb, ws_stride, (uint32_t)left, (uint32_t)u.dim};
        if (u.grad_hidden) VOCAB_TRY((vocab_few_dx<DT>(p, few_w, oz, sx, u.rows, dx, v0 != last, stream)));
        return u.grad_weight ? vocab_few_dw<DT>(ox, oz, count, u.rows, u.dim, left, dw_to, stream) : DFX_OK;
      }
      return vocab_grads<DT>(p, ow, oz, sx, u.dim, u.rows, u.grad_hidden && u.rows ? &dx_to : nullptr, ox, sw, left, u.grad_weight ? &dw_to : nullptr, stream);
    };
    if (u.grad_dtype == DFX_F32) VOCAB_TRY(both(VocabDw<DFX_F32>{(float*)u.grad_weight + v0 * gs, gs, a.state, (uint32_t)u.dim, (uint32_t)left, u.accumulate != 0}));
    else if constexpr (DT != DFX_F32) VOCAB_TRY(both(VocabDw<DT>{(uint16_t*)u.grad_weight + v0 * gs, gs, a.state, (uint32_t)u.dim, (uint32_t)left, u.accumulate != 0}));
  }
  if (u.sums && !sums_last && join) VOCAB_TRY(step_launch(dfx_vocab_sums_kernel, dim3(1), 256, stream, a));
  if (u.grad_hidden && u.rows)
    VOCAB_TRY(step_launch(dfx_vocab_dx_kernel<DT>, dim3((uint32_t)u.rows + (sums_last ? 1u : 0u), (uint32_t)((u.dim + 1023) / 1024)), 256, stream, a, (const float*)dx, (uint32_t)p.splits, (uint32_t)p.split_rows, (uint32_t)p.dq, u.grad_hidden,
                          u.grad_hidden_stride ? u.grad_hidden_stride : u.dim, (uint32_t)u.dim));
  return DFX_OK;
}

constexpr size_t kMostRows = (1ull << 24) - 1024, kMostVocab = 1ull << 28, kMostStride = 1ull << 20;

}  // namespace

extern "C" {

size_t dfx_vocab_loss_workspace(size_t rows, size_t dim, size_t vocab, dfx_dtype dtype, int grad, size_t piece) {
  if (dtype != DFX_F32 && dtype != DFX_BF16 && dtype != DFX_F16) return 0;
  if (rows >= kMostRows || vocab >= kMostVocab || !dim || dim >= kMostStride || piece % kTileRows) return 0;
  const VocabPlan p = vocab_plan(rows, dim, vocab, dtype, grad != 0, piece, true);
  return vocab_too_large(p) ? 0 : p.bytes;
}

int dfx_vocab_loss(const dfx_vocab_loss_args* u, void* hip_stream) {
  if (!u || u->struct_bytes != sizeof(*u)) return DFX_ERR_INVALID_ARG;
  if (u->dtype != DFX_F32 && u->dtype != DFX_BF16 && u->dtype != DFX_F16) return DFX_ERR_INVALID_ARG;
  if (u->grad_dtype != u->dtype && u->grad_dtype != DFX_F32) return DFX_ERR_INVALID_ARG;
  if (u->rows >= kMostRows || u->vocab >= kMostVocab || u->dim >= kMostStride) return DFX_ERR_TOO_LARGE;
  const size_t eb = step_elem_bytes(u->dtype), gb = step_elem_bytes(u->grad_dtype);
  const size_t hs = u->hidden_stride ? u->hidden_stride : u->dim, ws = u->weight_stride ? u->weight_stride : u->dim;
  const size_t ghs = u->grad_hidden_stride ? u->grad_hidden_stride : u->dim, gws = u->grad_weight_stride ? u->grad_weight_stride : u->dim;
  for (size_t s : {hs, ws, ghs, gws}) {
    if (s >= kMostStride) return DFX_ERR_TOO_LARGE;
    if (s < u->dim) return DFX_ERR_INVALID_ARG;
  }
  if (!u->dim || u->piece % kTileRows) return DFX_ERR_INVALID_ARG;
  if (!(u->inv_temperature * kVLog2e >= (double)FLT_MIN && u->inv_temperature * kVLog2e <= (double)FLT_MAX)) return DFX_ERR_INVALID_ARG;
  if ((u->rows && (!u->hidden || !u->targets)) || (u->vocab && !u->weight)) return DFX_ERR_INVALID_ARG;
  if ((uintptr_t)u->hidden % eb || (uintptr_t)u->weight % eb || (uintptr_t)u->grad_hidden % eb || (uintptr_t)u->grad_weight % gb || (uintptr_t)u->targets % 8) return DFX_ERR_INVALID_ARG;
  for (const void* p : {(const void*)u->row_weight, (const void*)u->scale, (const void*)u->logp, (const void*)u->loss, (const void*)u->sums})
    if ((uintptr_t)p % 4) return DFX_ERR_INVALID_ARG;
  const VocabPlan p = vocab_plan(u->rows, u->dim, u->vocab, u->dtype, u->grad_hidden || u->grad_weight, u->piece, vocab_aligned(*u));
  if (vocab_too_large(p)) return DFX_ERR_TOO_LARGE;
  if (!u->workspace || (uintptr_t)u->workspace % 256 || u->workspace_bytes < p.bytes) return DFX_ERR_INVALID_ARG;
  auto matrix = [](const void* at, size_t rows, size_t stride, size_t dim, size_t bytes) { return flat(at, rows ? ((rows - 1) * stride + dim) * bytes : 0); };
  const Span reads[] = {matrix(u->hidden, u->rows, hs, u->dim, eb), matrix(u->weight, u->vocab, ws, u->dim, eb), flat(u->targets, 8 * u->rows), flat(u->row_weight, 4 * u->rows), flat(u->scale, 4)};
  const Span writes[] = {flat(u->logp, 4 * u->rows), flat(u->loss, 4 * u->rows), flat(u->sums, 8), matrix(u->grad_hidden, u->rows, ghs, u->dim, eb),
                         matrix(u->grad_weight, u->vocab, gws, u->dim, gb), flat(u->workspace, p.bytes)};
  for (const Span& w : writes) {
    for (const Span& r : reads)
      if (meet(w, r)) return DFX_ERR_INVALID_ARG;
    for (const Span* o = writes; o != &w; ++o)
      if (meet(w, *o)) return DFX_ERR_INVALID_ARG;
  }
  if (u->dtype == DFX_F32) return vocab_run<DFX_F32>(*u, p, (hipStream_t)hip_stream);
  if (u->dtype == DFX_BF16) return vocab_run<DFX_BF16>(*u, p, (hipStream_t)hip_stream);
  return vocab_run<DFX_F16>(*u, p, (hipStream_t)hip_stream);
}

}  // extern "C"

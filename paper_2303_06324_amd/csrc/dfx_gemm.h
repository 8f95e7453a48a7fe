// Products of matrices for the loss over a vocabulary (dfx_vocab.hip): C[n][m] = sum over k of A[m][k] B[n][k] by workgroups that each hold a tile of C in
// registers, and hand it to an epilogue there.  An operand lies in memory with k along its rows, or across them ("turned": [k][m]).
//
// 16-bit elements on the matrix cores, sums in 32 bits.  A 32-bit matrix comes as three planes of bf16, its mantissa's 24 bits cut into three parts of 8,
// which hold it exactly: a = a0 + a1 + a2, |a1| <= 2^-8 |a|, |a2| <= 2^-16 |a|, and a b = a0 b0 + (a0 b1 + a1 b0) + (a1 b1 + a0 b2 + a2 b0) but for
// a1 b2 + a2 b1 + a2 b2, which are below 2^-23 + 2^-32 of it.  These six products follow one another along k, the small ones first, and cost six of a peak that is
// sixteen times that of 32-bit products.
#ifndef DFX_GEMM_H
#define DFX_GEMM_H

#include "dfx_step.h"
#include "dfx_tiles.h"
#include "dfx_vocab_plan.h"

namespace {

typedef __bf16 GemmBf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 GemmF16x8 __attribute__((ext_vector_type(8)));
typedef short GemmShort4 __attribute__((ext_vector_type(4)));
typedef short GemmShort8 __attribute__((ext_vector_type(8)));
typedef float GemmAcc __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) unsigned char GemmLds;

__device__ __forceinline__ int gemm_plane_a(int pair) { return (0x201100 >> (4 * (5 - pair))) & 0xf; }      // (2,0) (0,2) (1,1) (1,0) (0,1) (0,0)
__device__ __forceinline__ int gemm_plane_b(int pair) { return (0x021010 >> (4 * (5 - pair))) & 0xf; }

// rows: of a matrix with k along them, how many there are; of a turned one, how many k's.  cols: of a turned one, elements of a row that may be read
// (a multiple of 8).  Tiles that go beyond read the last row or the last 8 elements again; what is made of those is not used.  Every row begins at a
// multiple of 16 bytes, and rows with k along them hold whole steps.
struct GemmOperand {
  const uint16_t* p;
  size_t plane;                          // elements from one plane to the next
  uint32_t stride, rows, cols;
};

struct GemmShape {
  uint32_t mtiles, ntiles, splits;       // workgroups; splits along k
  uint32_t ksteps;                       // (or of what count says)
  uint32_t height;                       // rows of m from one tile to the next, where they are not all of a tile; otherwise 0
  const uint32_t* count;                 // device, may be null: what it holds bounds n (n_counted), or k
  bool k_counted;
};

// Workgroups go round the 8 XCDs; each XCD gets as many tiles as the others, which lie together, so that what it reads is in its own L2: kGroup tiles of n,
// then the next of m.
struct GemmPlace { uint32_t m, n, split; bool any; };
__device__ __forceinline__ GemmPlace gemm_place(const GemmShape& s, uint32_t ntiles, uint32_t block) {
  constexpr uint32_t kGroup = 8;
  const uint32_t tiles = s.mtiles * ntiles, total = tiles * s.splits, each = (total + 7u) / 8u;
  const uint32_t j = (block & 7u) * each + (block >> 3);
  if (j >= total || (block >> 3) >= each) return {0, 0, 0, false};
  const uint32_t split = j / tiles, t = j % tiles, group = t / (kGroup * s.mtiles), in = t % (kGroup * s.mtiles);
  const uint32_t width = min(kGroup, ntiles - group * kGroup);
  return {in / width, group * kGroup + in % width, split, true};
}
inline __host__ __device__ uint32_t gemm_groups(const GemmShape& s) { return (uint32_t)(((uint64_t)s.mtiles * s.ntiles * s.splits + 7) / 8 * 8); }

// Tiles in LDS.  k along the rows: a row's 128 bytes, whose 16-byte parts are exchanged by the row's number, so that 16 rows' parts of one k lie in
// different banks.  Turned: a k's 2 COLS bytes, whose 32-byte parts (16 elements, a tile of the matrix instruction) are exchanged by k, so that those of four k's
// that are read at once do.
template <int COLS>
__device__ __forceinline__ uint32_t gemm_turned_swap(uint32_t k) { return COLS >= 128 ? (k & 3u) | ((k >> 1) & 4u) : ((k >> 1) & 1u) | ((k >> 2) & 2u); }

template <int COLS, int THREADS, bool TURNED>
__device__ __forceinline__ void gemm_fetch(const GemmOperand& o, int plane, uint32_t first, uint32_t k0, unsigned char* lds) {
  constexpr int LOADS = COLS * 8 / THREADS;
  const uint32_t t = threadIdx.x, wave = t / kStepWave;
  if (!TURNED) {
    const uint32_t from = tile_base(first, o.rows);      // (half a tile may lie behind the last row)
    const uint16_t* base = o.p + (size_t)plane * o.plane + (size_t)from * o.stride + k0;
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(base), 0, -1, 0x00020000);
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const uint32_t row = j * (THREADS / 8) + t / 8, part = (t & 7u) ^ ((row >> 1) & 7u);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(lds + (j * THREADS + wave * kStepWave) * 16), 16, (int)(tile_row(first, row, o.rows) * o.stride * 2u + part * 16u), 0, 0, 0);
    }
  } else {
    constexpr int PARTS = COLS / 8;      // of 16 bytes in a k's row
    const uint16_t* base = o.p + (size_t)plane * o.plane + (size_t)tile_base(k0, o.rows) * o.stride;
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(base), 0, -1, 0x00020000);
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const uint32_t k = j * (THREADS / PARTS) + t / PARTS, slot = t % PARTS;
      const uint32_t part = (((slot >> 1) ^ gemm_turned_swap<COLS>(k)) << 1) | (slot & 1u);
      const uint32_t col = tile_col(first, part, o.cols);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(lds + (j * THREADS + wave * kStepWave) * 16), 16, (int)((tile_row(k0, k, o.rows) * o.stride + col) * 2u), 0, 0, 0);
    }
  }
}

// what a lane holds of 16 rows and 32 k's: row lane % 16, k's 8 (lane / 16) on
__device__ __forceinline__ GemmShort8 gemm_read(const unsigned char* lds, uint32_t first, int kk) {
  const uint32_t lane = threadIdx.x % kStepWave, l = lane % 16u;
  return *(const __attribute__((address_space(3))) GemmShort8*)((GemmLds*)lds + (first + l) * 128u + (((uint32_t)kk * 4u + lane / 16u) ^ ((l >> 1) & 7u)) * 16u);
}

// The same of COUNT tiles of 16 rows at once and both kk, of a turned tile: the reads and the wait for them are one block of assembly, because the compiler,
// which does not know what of LDS a load writes, waits for every load to LDS before a transposing read.
template <int COLS>
__device__ __forceinline__ uint32_t gemm_turned_at(const unsigned char* lds, uint32_t first) {
  const uint32_t lane = threadIdx.x % kStepWave, l = lane % 16u, k = 8u * (lane / 16u) + l / 4u;
  return (uint32_t)(uintptr_t)(GemmLds*)lds + k * (COLS * 2u) + (((first / 16u) ^ gemm_turned_swap<COLS>(k)) * 32u) + (l & 3u) * 8u;
}
template <int COUNT, int COLS>
__device__ __forceinline__ void gemm_read_turned(const unsigned char* lds, uint32_t first, GemmShort8 (*to)[2]) {
  GemmShort4 r[COUNT][4];                // (4 k's further: COLS 8 bytes, 32: COLS 64)
  if constexpr (COUNT == 4)
    asm volatile(
        "ds_read_b64_tr_b16 %0, %16\n\t"
        "ds_read_b64_tr_b16 %1, %16 offset:%20\n\t"
        "ds_read_b64_tr_b16 %2, %16 offset:%21\n\t"
        "ds_read_b64_tr_b16 %3, %16 offset:%22\n\t"
        "ds_read_b64_tr_b16 %4, %17\n\t"
        "ds_read_b64_tr_b16 %5, %17 offset:%20\n\t"
        "ds_read_b64_tr_b16 %6, %17 offset:%21\n\t"
        "ds_read_b64_tr_b16 %7, %17 offset:%22\n\t"
        "ds_read_b64_tr_b16 %8, %18\n\t"
        "ds_read_b64_tr_b16 %9, %18 offset:%20\n\t"
        "ds_read_b64_tr_b16 %10, %18 offset:%21\n\t"
        "ds_read_b64_tr_b16 %11, %18 offset:%22\n\t"
        "ds_read_b64_tr_b16 %12, %19\n\t"
        "ds_read_b64_tr_b16 %13, %19 offset:%20\n\t"
        "ds_read_b64_tr_b16 %14, %19 offset:%21\n\t"
        "ds_read_b64_tr_b16 %15, %19 offset:%22\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(r[0][0]), "=&v"(r[0][1]), "=&v"(r[0][2]), "=&v"(r[0][3]), "=&v"(r[1][0]), "=&v"(r[1][1]), "=&v"(r[1][2]), "=&v"(r[1][3]), "=&v"(r[2][0]), "=&v"(r[2][1]), "=&v"(r[2][2]), "=&v"(r[2][3]), "=&v"(r[3][0]), "=&v"(r[3][1]), "=&v"(r[3][2]), "=&v"(r[3][3])
        : "v"(gemm_turned_at<COLS>(lds, first + 0u)), "v"(gemm_turned_at<COLS>(lds, first + 16u)), "v"(gemm_turned_at<COLS>(lds, first + 32u)), "v"(gemm_turned_at<COLS>(lds, first + 48u)), "i"(COLS * 8), "i"(COLS * 64), "i"(COLS * 72)
        : "memory");
  else
    asm volatile(
        "ds_read_b64_tr_b16 %0, %8\n\t"
        "ds_read_b64_tr_b16 %1, %8 offset:%10\n\t"
        "ds_read_b64_tr_b16 %2, %8 offset:%11\n\t"
        "ds_read_b64_tr_b16 %3, %8 offset:%12\n\t"
        "ds_read_b64_tr_b16 %4, %9\n\t"
        "ds_read_b64_tr_b16 %5, %9 offset:%10\n\t"
        "ds_read_b64_tr_b16 %6, %9 offset:%11\n\t"
        "ds_read_b64_tr_b16 %7, %9 offset:%12\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(r[0][0]), "=&v"(r[0][1]), "=&v"(r[0][2]), "=&v"(r[0][3]), "=&v"(r[1][0]), "=&v"(r[1][1]), "=&v"(r[1][2]), "=&v"(r[1][3])
        : "v"(gemm_turned_at<COLS>(lds, first + 0u)), "v"(gemm_turned_at<COLS>(lds, first + 16u)), "i"(COLS * 8), "i"(COLS * 64), "i"(COLS * 72)
        : "memory");
#pragma unroll
  for (int i = 0; i < COUNT; ++i)
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) to[i][kk] = __builtin_shufflevector(r[i][2 * kk], r[i][2 * kk + 1], 0, 1, 2, 3, 4, 5, 6, 7);
}

// COUNT tiles of 16 rows and 64 k's, either way
template <int COUNT, int COLS, bool TURNED>
__device__ __forceinline__ void gemm_take(const unsigned char* lds, uint32_t first, GemmShort8 (*to)[2]) {
  if constexpr (TURNED) gemm_read_turned<COUNT, COLS>(lds, first, to);
  else
#pragma unroll
    for (int i = 0; i < COUNT; ++i)
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) to[i][kk] = gemm_read(lds, first + i * 16, kk);
}

template <int DT>
__device__ __forceinline__ GemmAcc gemm_mac(GemmShort8 a, GemmShort8 b, GemmAcc c) {
  if (DT == DFX_F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(GemmF16x8, a), __builtin_bit_cast(GemmF16x8, b), c, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(GemmBf16x8, a), __builtin_bit_cast(GemmBf16x8, b), c, 0, 0, 0);
}

// The three planes of two 32-bit values, side by side in a word each, every one the nearest bf16 to what is left (the largest values' first: the largest bf16, where the
// nearest would be infinite).  Of an infinity or NaN one of them is NaN.
__device__ __forceinline__ void gemm_cut(float x, float y, uint32_t* part) {
  const float most = 3.3895313892515355e38f;
  StepPair v = {__builtin_amdgcn_fmed3f(x, -most, most), __builtin_amdgcn_fmed3f(y, -most, most)};
  part[0] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, StepBf16Pair));
  v[0] = x - __uint_as_float(part[0] << 16); v[1] = y - __uint_as_float(part[0] & 0xffff0000u);
  part[1] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, StepBf16Pair));
  v[0] -= __uint_as_float(part[1] << 16); v[1] -= __uint_as_float(part[1] & 0xffff0000u);
  part[2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, StepBf16Pair));
}
// ... of eight, as four words of each plane
__device__ __forceinline__ void gemm_cut8(const float* v, uint32_t (*part)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    uint32_t p[3];
    gemm_cut(v[2 * e], v[2 * e + 1], p);
#pragma unroll
    for (int q = 0; q < 3; ++q) part[q][e] = p[q];
  }
}

// Sums of few rows, whose log-probabilities are looked at one by one, are taken in blocks of k, which are then added up: an addition costs up to a digit of the sum that it meets, and so few of them
// meet one that is nearly whole.  kGemmBlock steps of 16-bit elements to a block; of 32-bit ones, six products to a step, two or three.  Errors of logp of a row (rms, logits of 7.5) as one sum and
// in blocks: 4096 fp32 elements 4.3e-6 and 0.7e-6, 3200 bf16 1.6e-6 and 0.5e-6 (torch's 32-bit product 1.8e-6 and 0.7e-6).  40 x 2001 x 100000 bf16 183 us and 178, 66 x 1789 x 67561 in 32 bits 282
// and 291.
constexpr uint32_t kGemmBlock = 8;
template <int MT, int NT>
__device__ __forceinline__ void gemm_fold(GemmAcc (&all)[MT][NT], GemmAcc (&acc)[MT][NT]) {
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      all[i][j] += acc[i][j];
      acc[i][j] = GemmAcc{0, 0, 0, 0};
    }
}

// Few rows: a tile of 64 MT m by 64 n by 4 waves of 16 MT m each.  A lane holds, of each of its wave's MT NT products of 16 x 16, n = lane % 16 and m = 4 (lane / 16) on.
template <int MT_>
struct GemmFlat {
  static constexpr int WM = 4, WN = 1, MT = MT_, NT = 4, M = 64 * MT, N = 64, THREADS = 256;
  static constexpr int STAGE = (M + N) * kGemmK * 2, LOADS = (M + N) * 8 / THREADS;
  uint32_t m0, n0;                       // of the workgroup's tile
  __device__ __forceinline__ uint32_t wave_m() const { return threadIdx.x / kStepWave * (16u * MT); }
  __device__ __forceinline__ uint32_t m(int mt) const { return m0 + wave_m() + mt * 16 + threadIdx.x % kStepWave / 16 * 4; }
  __device__ __forceinline__ uint32_t n(int nt) const { return n0 + nt * 16 + threadIdx.x % 16; }
  __device__ __forceinline__ uint32_t row(int nt, uint32_t r) const { return n0 + nt * 16 + r; }
  __device__ __forceinline__ uint32_t row_of_pass() const { return threadIdx.x % 16; }
};

// A tile of 256 m by 256 n by 8 waves, in halves of 128 by 128 in which each wave has 64 m by 32 n.
struct GemmWide {
  static constexpr int WM = 2, WN = 4, MT = 8, NT = 4, M = 256, N = 256, THREADS = 512;
  static constexpr int HALF = 128 * kGemmK * 2, STAGE = 4 * HALF, LDS = 2 * STAGE;
  uint32_t m0, n0;
  __device__ __forceinline__ uint32_t wave_m() const { return threadIdx.x / kStepWave / WN * 64u; }
  __device__ __forceinline__ uint32_t wave_n() const { return threadIdx.x / kStepWave % WN * 32u; }
  __device__ __forceinline__ uint32_t m(int mt) const { return m0 + mt / 4 * 128u + wave_m() + mt % 4 * 16u + threadIdx.x % kStepWave / 16 * 4; }
  __device__ __forceinline__ uint32_t n(int nt) const { return n0 + nt / 2 * 128u + wave_n() + nt % 2 * 16u + threadIdx.x % 16; }
  __device__ __forceinline__ uint32_t row(int nt, uint32_t r) const { return n0 + nt / 2 * 128u + r / 16u * 32u + nt % 2 * 16u + r % 16u; }
  __device__ __forceinline__ uint32_t row_of_pass() const { return wave_n() / 2u + threadIdx.x % 16; }
};

// A wave's waits: at most so many of its loads to LDS under way, none of its reads from LDS
template <int LOADS>
__device__ __forceinline__ void gemm_wait() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt((LOADS & 15) | 0x70 | (LOADS >> 4) << 14);
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void gemm_meet() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
}

// What a workgroup has to do: its tile, and steps of k for each pair of planes
template <class TILE>
__device__ __forceinline__ GemmPlace gemm_work(const GemmShape& s, uint32_t block, TILE& tile, uint32_t& begin, uint32_t& end) {
  uint32_t steps = s.ksteps, ntiles = s.ntiles;
  if (s.count) {
    const uint32_t count = *s.count;
    if (s.k_counted) steps = (count + kGemmK - 1) / kGemmK;
    else ntiles = (count + TILE::N - 1) / TILE::N;
  }
  const GemmPlace at = gemm_place(s, ntiles, block);
  tile.m0 = at.m * (s.height ? s.height : TILE::M); tile.n0 = at.n * TILE::N;
  const uint32_t each = (steps + s.splits - 1) / s.splits;
  begin = min(at.split * each, steps); end = min(begin + each, steps);
  return at;
}

// The step of k that is loaded next.  Behind the last one it is loaded again, and not used.
struct GemmNext {
  uint32_t k, begin, end, left;
  int pair;
  __device__ __forceinline__ GemmNext(uint32_t begin_, uint32_t end_, uint32_t total) : k(begin_), begin(begin_), end(end_), left(total), pair(0) {}
  __device__ __forceinline__ void advance() {
    if (--left == 0) left = 1;
    else if (++k == end) { k = begin; ++pair; }
  }
};

// The flat tile: it streams a 16-bit matrix of rows at multiples of 16 bytes through the chip once.  Three or four stages, one of which is used while the others are under way, and
// two workgroups to a compute unit.  HBM bounds it: logits of 64 x 4096 x 131072 bf16 187 us (5.7 TB/s) where the kernel past LDS takes 216, of 48 x 2048 x 32000 30 and 40.
template <int DT, int MT, class EPI>
__global__ void __launch_bounds__(256, 2) dfx_gemm_flat_kernel(GemmOperand a, GemmOperand b, GemmShape s, EPI epi) {
  typedef GemmFlat<MT> TILE;
  constexpr uint32_t STAGES = MT == 1 ? 4 : 3;
  __shared__ __align__(1024) unsigned char lds[TILE::STAGE * STAGES];
  TILE tile;
  uint32_t begin, end;
  const GemmPlace at = gemm_work(s, blockIdx.x, tile, begin, end);
  if (!at.any) return;
  if (s.height) a.rows = min(a.rows, tile.m0 + s.height);
  GemmAcc acc[TILE::MT][TILE::NT], all[TILE::MT][TILE::NT];
#pragma unroll
  for (int i = 0; i < TILE::MT; ++i)
#pragma unroll
    for (int j = 0; j < TILE::NT; ++j) acc[i][j] = all[i][j] = GemmAcc{0, 0, 0, 0};
  const uint32_t total = end - begin, wm = tile.wave_m();
  if (total) {
    GemmNext next(begin, end, total);
    auto load = [&](uint32_t stage) {
      unsigned char* to = lds + stage * TILE::STAGE;
      gemm_fetch<TILE::M, TILE::THREADS, false>(a, 0, tile.m0, next.k * kGemmK, to);
      gemm_fetch<TILE::N, TILE::THREADS, false>(b, 0, tile.n0, next.k * kGemmK, to + TILE::M * kGemmK * 2);
      next.advance();
    };
#pragma unroll
    for (uint32_t q = 0; q < STAGES - 1; ++q) load(q);
    uint32_t stage = 0;
    for (uint32_t q = 0; q < total;) {
      for (const uint32_t till = min(total, q + kGemmBlock); q < till; ++q) {
        gemm_wait<(STAGES - 2) * TILE::LOADS>();
        gemm_meet();                       // this stage has arrived for all, and nobody reads the one before it any more
        load(stage ? stage - 1u : STAGES - 1u);
        const unsigned char* la = lds + stage * TILE::STAGE;
        GemmShort8 fa[TILE::MT][2], fb[TILE::NT][2];
        gemm_take<TILE::NT, TILE::N, false>(la + TILE::M * kGemmK * 2, 0, fb);
        gemm_take<TILE::MT, TILE::M, false>(la, wm, fa);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
          for (int i = 0; i < TILE::MT; ++i)
#pragma unroll
            for (int j = 0; j < TILE::NT; ++j) acc[i][j] = gemm_mac<DT>(fa[i][kk], fb[j][kk], acc[i][j]);
        stage = stage + 1u == STAGES ? 0u : stage + 1u;
      }
      gemm_fold(all, acc);
    }
    gemm_wait<0>();
    gemm_meet();
  }
  epi(tile, at, all, lds);
}

// A tile by its rows of n: f(n, m, v) for E elements that follow one another from m on, of one row by threads beside each other, so that what they write lies
// together.  Through LDS, WN 16 rows at a time, which lie 16 bytes further in the banks each.
template <int E, class TILE, class F>
__device__ __forceinline__ void gemm_by_rows(const TILE& tile, const GemmAcc (&acc)[TILE::MT][TILE::NT], unsigned char* lds, const F& f) {
  constexpr uint32_t ROWS = TILE::WN * 16, PITCH = TILE::M + 4, PARTS = TILE::M / E;
  float* at = (float*)lds;
#pragma unroll
  for (int j = 0; j < TILE::NT; ++j) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < TILE::MT; ++i) *(GemmAcc*)(at + tile.row_of_pass() * PITCH + tile.m(i) - tile.m0) = acc[i][j];
    __syncthreads();
#pragma unroll
    for (uint32_t q = threadIdx.x; q < ROWS * PARTS; q += TILE::THREADS) {
      const uint32_t r = q / PARTS, m = q % PARTS * E;
      float v[E];
#pragma unroll
      for (int e = 0; e < E; e += 4) {
        const GemmAcc four = *(const GemmAcc*)(at + r * PITCH + m + e);
#pragma unroll
        for (int x = 0; x < 4; ++x) v[e + x] = four[x];
      }
      f(tile.row(j, r), tile.m0 + m, v);
    }
  }
}

// The wide tile.  Two waves share a SIMD, and while one of them has the matrix core the other fetches: a step is four turns, one for each quarter of a wave's
// products, and a turn is a part that reads LDS and starts loads, and a part of 16 products; waves 4 to 7 run one part behind waves 0 to 3.  Halves of the
// tiles are read in the order n0, m0, n1, m1, and as soon as both sets of waves have read one, the loads of the step after next may begin to overwrite it: a
// load has seven turns to arrive, 12 younger ones of a wave under way behind it.  The matrix cores' power bounds it: logits of 6700 x 4096 x 131072 bf16 1.30 PFLOP/s, dX with dW 1.21 (as
// one set of waves 29.4 ms in all, now 22.1); 32-bit ones as six products 1.15 PFLOP/s of bf16.  Products of 32 x 32 x 16 were 6 % slower, a step in two turns 3 %.
template <int DT, bool TA, bool TB, class EPI>
__device__ __forceinline__ void gemm_wide(const GemmOperand& a, const GemmOperand& b, const GemmShape& s, const EPI& epi, uint32_t block, unsigned char* gemm_lds) {
  GemmWide tile;
  uint32_t begin, end;
  const GemmPlace at = gemm_work(s, block, tile, begin, end);
  if (!at.any) return;
  GemmAcc acc[GemmWide::MT][GemmWide::NT];
#pragma unroll
  for (int i = 0; i < GemmWide::MT; ++i)
#pragma unroll
    for (int j = 0; j < GemmWide::NT; ++j) acc[i][j] = GemmAcc{0, 0, 0, 0};
  const uint32_t total = (end - begin) * gemm_pairs(DT);
  if (total) {
    const uint32_t wm = tile.wave_m(), wn = tile.wave_n();
    GemmNext next(begin, end, total);
    auto load_a = [&](uint32_t stage, int half) {
      gemm_fetch<128, GemmWide::THREADS, TA>(a, gemm_planes(DT) == 1 ? 0 : gemm_plane_a(next.pair), tile.m0 + half * 128u, next.k * kGemmK, gemm_lds + stage * GemmWide::STAGE + half * GemmWide::HALF);
    };
    auto load_b = [&](uint32_t stage, int half) {
      gemm_fetch<128, GemmWide::THREADS, TB>(b, gemm_planes(DT) == 1 ? 0 : gemm_plane_b(next.pair), tile.n0 + half * 128u, next.k * kGemmK, gemm_lds + stage * GemmWide::STAGE + (2 + half) * GemmWide::HALF);
    };
    GemmShort8 fa[4][2], fb[3][2][2];    // of n0 in an even step, n1, n0 in an odd one
    auto read_a = [&](uint32_t stage, int half) { gemm_take<4, 128, TA>(gemm_lds + stage * GemmWide::STAGE + half * GemmWide::HALF, wm, fa); };
    auto read_b = [&](uint32_t stage, int half, int to) { gemm_take<2, 128, TB>(gemm_lds + stage * GemmWide::STAGE + (2 + half) * GemmWide::HALF, wn, fb[to]); };
    auto products = [&](int mh, int nh, int from) {
      gemm_meet();
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) acc[mh * 4 + i][nh * 2 + j] = gemm_mac<DT>(fa[i][kk], fb[from][j][kk], acc[mh * 4 + i][nh * 2 + j]);
      __builtin_amdgcn_s_setprio(0);
      gemm_meet();
    };
    for (uint32_t q = 0; q < 2; ++q) {
      load_b(q, 0); load_a(q, 0); load_b(q, 1); load_a(q, 1);
      next.advance();
    }
    auto step = [&](uint32_t stage) {
      load_b(stage, 0);
      read_a(stage, 0);
      gemm_wait<12>();
      products(0, 0, 2 * stage);
      load_a(stage, 0);
      read_b(stage, 1, 1);
      gemm_wait<12>();
      products(0, 1, 1);
      load_b(stage, 1);
      read_a(stage, 1);
      gemm_wait<12>();
      products(1, 1, 1);
      load_a(stage, 1);
      next.advance();
      read_b(stage ^ 1u, 0, 2 - 2 * stage);
      gemm_wait<12>();
      products(1, 0, 2 * stage);
    };
    gemm_wait<14>();
    gemm_meet();
    read_b(0, 0, 0);
    gemm_wait<12>();
    gemm_meet();
    if (threadIdx.x >= 256) gemm_meet();       // one part behind
    for (uint32_t q = 0; q < total; q += 2) {
      step(0);
      if (q + 1 < total) step(1);
    }
    if (threadIdx.x < 256) gemm_meet();
    gemm_wait<0>();
    gemm_meet();
  }
  epi(tile, at, acc, gemm_lds);
}

// A quarter of it: 128 by 128, of which each of the eight waves has 64 by 32.
struct GemmQuarter {
  static constexpr int WM = 2, WN = 4, MT = 4, NT = 2, M = 128, N = 128, THREADS = 512;
  static constexpr int HALF = 128 * kGemmK * 2, STAGE = 2 * HALF, STAGES = 4, LOADS = 4;
  uint32_t m0, n0;
  __device__ __forceinline__ uint32_t wave_m() const { return threadIdx.x / kStepWave / WN * 64u; }
  __device__ __forceinline__ uint32_t wave_n() const { return threadIdx.x / kStepWave % WN * 32u; }
  __device__ __forceinline__ uint32_t m(int mt) const { return m0 + wave_m() + mt * 16u + threadIdx.x % kStepWave / 16 * 4; }
  __device__ __forceinline__ uint32_t n(int nt) const { return n0 + wave_n() + nt * 16u + threadIdx.x % 16; }
  __device__ __forceinline__ uint32_t row(int nt, uint32_t r) const { return n0 + r / 16u * 32u + nt * 16u + r % 16u; }
  __device__ __forceinline__ uint32_t row_of_pass() const { return wave_n() / 2u + threadIdx.x % 16; }
};
static_assert(GemmQuarter::STAGES * GemmQuarter::STAGE <= GemmWide::LDS, "a workgroup takes either tile");

// Where wide tiles would leave compute units idle.  Four stages, three of which are under way; the waves of a SIMD fill each other's waits.  It needs twice the bytes from L2 for a
// product, which bound it (12 TB/s): 0.39 of a wide tile's time for a quarter of its work.  650 x 1984 x 2368 bf16 with gradients: 111 us by wide tiles, 61 by these.
template <int DT, bool TA, bool TB, class EPI>
__device__ __forceinline__ void gemm_quarter(const GemmOperand& a, const GemmOperand& b, const GemmShape& s, const EPI& epi, uint32_t block, unsigned char* lds) {
  typedef GemmQuarter TILE;
  TILE tile;
  uint32_t begin, end;
  const GemmPlace at = gemm_work(s, block, tile, begin, end);
  if (!at.any) return;
  GemmAcc acc[TILE::MT][TILE::NT];
#pragma unroll
  for (int i = 0; i < TILE::MT; ++i)
#pragma unroll
    for (int j = 0; j < TILE::NT; ++j) acc[i][j] = GemmAcc{0, 0, 0, 0};
  const uint32_t total = (end - begin) * gemm_pairs(DT);
  if (total) {
    GemmNext next(begin, end, total);
    auto load = [&](uint32_t stage) {
      gemm_fetch<128, TILE::THREADS, TA>(a, gemm_planes(DT) == 1 ? 0 : gemm_plane_a(next.pair), tile.m0, next.k * kGemmK, lds + stage * TILE::STAGE);
      gemm_fetch<128, TILE::THREADS, TB>(b, gemm_planes(DT) == 1 ? 0 : gemm_plane_b(next.pair), tile.n0, next.k * kGemmK, lds + stage * TILE::STAGE + TILE::HALF);
      next.advance();
    };
    for (uint32_t q = 0; q < 3; ++q) load(q);
    for (uint32_t q = 0; q < total; ++q) {
      gemm_wait<2 * TILE::LOADS>();
      gemm_meet();                       // this stage has arrived for all, and nobody reads the one before it any more
      load((q + 3u) & 3u);
      const unsigned char* at_a = lds + (q & 3u) * TILE::STAGE;
      GemmShort8 fa[TILE::MT][2], fb[TILE::NT][2];
      gemm_take<TILE::NT, 128, TB>(at_a + TILE::HALF, tile.wave_n(), fb);
      gemm_take<TILE::MT, 128, TA>(at_a, tile.wave_m(), fa);
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int i = 0; i < TILE::MT; ++i)
#pragma unroll
          for (int j = 0; j < TILE::NT; ++j) acc[i][j] = gemm_mac<DT>(fa[i][kk], fb[j][kk], acc[i][j]);
    }
    gemm_wait<0>();
    gemm_meet();
  }
  epi(tile, at, acc, lds);
}

// What the workgroups of a launch from `from` on do: a product by wide tiles or by quarters
template <class EPI>
struct GemmTask {
  GemmOperand a, b;
  GemmShape s;
  uint32_t from;
  bool quarters;
  EPI epi;
};
template <int DT, bool TA, bool TB, class EPI>
__device__ __forceinline__ bool gemm_task(const GemmTask<EPI>& t, unsigned char* lds) {
  const uint32_t block = blockIdx.x - t.from;
  if (block >= gemm_groups(t.s)) return false;
  if (t.quarters) gemm_quarter<DT, TA, TB>(t.a, t.b, t.s, t.epi, block, lds);
  else gemm_wide<DT, TA, TB>(t.a, t.b, t.s, t.epi, block, lds);
  return true;
}

// Two products in one launch, the one of the longer sums first: the other's tiles fill the compute units that its last round leaves idle.
template <int DT, bool TA, bool TB, class EPI, bool TA2, bool TB2, class EPI2>
__global__ void __launch_bounds__(GemmWide::THREADS, 2) dfx_gemm_two_kernel(GemmTask<EPI> one, GemmTask<EPI2> two) {
  __shared__ __align__(1024) unsigned char lds[GemmWide::LDS];
  if (!gemm_task<DT, TA, TB>(one, lds)) gemm_task<DT, TA2, TB2>(two, lds);
}
// ... of which both are one, some of its tiles wide
template <int DT, bool TA, bool TB, class EPI>
__global__ void __launch_bounds__(GemmWide::THREADS, 2) dfx_gemm_wide_kernel(GemmTask<EPI> wide, GemmTask<EPI> quarters) {
  __shared__ __align__(1024) unsigned char lds[GemmWide::LDS];
  if (blockIdx.x < quarters.from) gemm_wide<DT, TA, TB>(wide.a, wide.b, wide.s, wide.epi, blockIdx.x, lds);
  else gemm_quarter<DT, TA, TB>(quarters.a, quarters.b, quarters.s, quarters.epi, blockIdx.x - quarters.from, lds);
}

// ------------------------------------------------------------------------------------------
// Few rows: the larger matrix, W, goes through the chip once and past LDS, from its own type at any alignment straight into the registers that the matrix
// instructions take, steps ahead; the other operand, small and in planes, comes through LDS.  HBM bounds these.
// ------------------------------------------------------------------------------------------
// A matrix as the caller has it.  dim >= 64 elements of a row.
struct GemmSource {
  const void* p;
  size_t stride;
  uint32_t rows, dim;
};

// 16 bytes of a row from element e on, or the last 16 bytes of the row where it ends before: `over` elements further on
template <int DT>
__device__ __forceinline__ StepVec<DT, 16 / (int)sizeof(typename StepElem<DT>::raw)> gemm_row_part(const void* row, uint32_t e, uint32_t dim) {
  constexpr uint32_t N = 16 / sizeof(typename StepElem<DT>::raw);
  StepVec<DT, (int)N> v;
  v.load(row, min(e, dim - N));
  return v;
}
// ... put right: elements that lie behind the row's end are 0
template <int DT, int N>
__device__ __forceinline__ void gemm_row_end(StepVec<DT, N>& v, uint32_t e, uint32_t dim) {
  constexpr uint32_t BITS = 8 * sizeof(typename StepElem<DT>::raw), WORDS = sizeof(v.w) / 4;
  const uint32_t over = e + N > dim ? min(e + N - dim, (uint32_t)N) : 0u, words = over * BITS / 32u, half = over * BITS % 32u;
  uint32_t x[WORDS + 1];
#pragma unroll
  for (uint32_t k = 0; k < WORDS; ++k) {
    x[k] = 0;
#pragma unroll
    for (uint32_t j = 0; j < WORDS; ++j)
      if (k + words == j) x[k] = v.w[j];
  }
  x[WORDS] = 0;
#pragma unroll
  for (uint32_t k = 0; k < WORDS; ++k) v.w[k] = half ? x[k] >> 16 | x[k + 1] << 16 : x[k];
}

template <int NT_, int MT_>
struct GemmFew {
  static constexpr int WM = 4, WN = 1, MT = MT_, NT = NT_, M = 64 * MT, N = 16 * NT, THREADS = 256;
  uint32_t m0, n0;
  __device__ __forceinline__ uint32_t wave_m() const { return threadIdx.x / kStepWave * (MT * 16); }
  __device__ __forceinline__ uint32_t m(int mt) const { return m0 + wave_m() + mt * 16 + threadIdx.x % kStepWave / 16 * 4; }
  __device__ __forceinline__ uint32_t n(int nt) const { return n0 + nt * 16 + threadIdx.x % 16; }
  __device__ __forceinline__ uint32_t row(int nt, uint32_t r) const { return n0 + nt * 16 + r; }
  __device__ __forceinline__ uint32_t row_of_pass() const { return threadIdx.x % 16; }
};

// planes of eight 32-bit values, or eight 16-bit ones as they are
template <int DT>
__device__ __forceinline__ void gemm_parts(const StepVec<DT, 16 / (int)sizeof(typename StepElem<DT>::raw)>* v, GemmShort8* to) {
  if constexpr (DT == DFX_F32) {
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = v[e / 4].get(e % 4);
    uint32_t p[3][4];
    gemm_cut8(x, p);
#pragma unroll
    for (int q = 0; q < 3; ++q) to[q] = __builtin_bit_cast(GemmShort8, p[q]);
  } else to[0] = __builtin_bit_cast(GemmShort8, v[0].w);
}

// Logits: M rows of W by N rows of x, along both; loads of W are DEPTH steps ahead.  66 x 1789 x 67561 in 32 bits 171 us (2.8 TB/s; cut into planes and laid out first 548).
template <int DT, int NT, int MT, int DEPTH, class EPI>
__global__ void __launch_bounds__(256, 2) dfx_gemm_few_kernel(GemmSource w, GemmOperand b, GemmShape s, EPI epi) {
  typedef GemmFew<NT, MT> TILE;
  constexpr int P = gemm_planes(DT), V = DT == DFX_F32 ? 2 : 1, N = 16 / (int)sizeof(typename StepElem<DT>::raw), PLANE = TILE::N * kGemmK * 2, STAGE = P * PLANE, LOADS = MT * 2 * V + P * NT / 2;
  constexpr int STAGES = DEPTH + 1;
  __shared__ __align__(1024) unsigned char lds[STAGES * STAGE > 16 * (TILE::M + 4) * 4 ? STAGES * STAGE : 16 * (TILE::M + 4) * 4];
  TILE tile;
  uint32_t begin, end;
  const GemmPlace at = gemm_work(s, blockIdx.x, tile, begin, end);
  if (!at.any) return;
  GemmAcc acc[MT][NT], all[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = all[i][j] = GemmAcc{0, 0, 0, 0};
  if (s.height) w.rows = min(w.rows, tile.m0 + s.height);
  const uint32_t lane = threadIdx.x % kStepWave, g = lane / 16u;
  const void* row[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) row[i] = (const typename StepElem<DT>::raw*)w.p + (size_t)min(tile.m0 + tile.wave_m() + i * 16u + lane % 16u, w.rows - 1u) * w.stride;
  StepVec<DT, N> raw[DEPTH][MT][2][V];
  GemmNext next(begin, end, end - begin);
  auto load = [&](int set, uint32_t stage) {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int v = 0; v < V; ++v) raw[set][i][kk][v] = gemm_row_part<DT>(row[i], next.k * kGemmK + kk * 32u + g * 8u + v * N, w.dim);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int p = 0; p < P; ++p) gemm_fetch<TILE::N, 256, false>(b, p, tile.n0, next.k * kGemmK, lds + stage * STAGE + p * PLANE);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    next.advance();
  };
#pragma unroll
  for (int d = 0; d < DEPTH; ++d) load(d, d);
  uint32_t stage = 0;
  auto step = [&](int set, uint32_t k) {
    gemm_wait<LOADS * (DEPTH - 1)>();
    gemm_meet();                         // this step's operands have arrived, and nobody reads the stage of the one before any more
    GemmShort8 fa[MT][2][P];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        if ((k + 1u) * kGemmK > w.dim)
#pragma unroll
          for (int v = 0; v < V; ++v) gemm_row_end(raw[set][i][kk][v], k * kGemmK + kk * 32u + g * 8u + v * N, w.dim);
        gemm_parts<DT>(raw[set][i][kk], fa[i][kk]);
      }
    load(set, stage ? stage - 1u : STAGES - 1u);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      GemmShort8 fb[P][2];
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) fb[p][kk] = gemm_read(lds + stage * STAGE + p * PLANE, j * 16, kk);
#pragma unroll
      for (int pair = 0; pair < gemm_pairs(DT); ++pair)
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
          for (int i = 0; i < MT; ++i) acc[i][j] = gemm_mac<DT>(fa[i][kk][P == 1 ? 0 : gemm_plane_a(pair)], fb[P == 1 ? 0 : gemm_plane_b(pair)][kk], acc[i][j]);
    }
    if (P == 1 && k % kGemmBlock == kGemmBlock - 1u) gemm_fold(all, acc);
    stage = stage + 1u == STAGES ? 0u : stage + 1u;
  };
  for (uint32_t k = begin; k < end; k += DEPTH) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
      if (k + d < end) step(d, k + d);
    if (P > 1) gemm_fold(all, acc);      // (of 32 bits every DEPTH steps)
  }
  gemm_fold(all, acc);
  gemm_wait<0>();
  gemm_meet();
  epi(tile, at, all, lds);
}

// Logits of 16 NT rows at most: x stays in registers, of each of eight waves 32 KK elements of all rows.  A wave reads so much of a row of W at a time, which lies together (the
// memory is quicker at that than at 128 bytes of each of many rows), a tile of 16 rows ahead, also where the next tile of 64 rows begins: as many workgroups as fit at once go
// through all of W.  The waves' sums meet in LDS at the end of 64 rows.  HBM bounds it: 1 row of bf16, 2048 x 50257, 43 us (4.8 TB/s; a workgroup for each 64 rows 47, by 128 bytes
// of 64 rows past LDS 47; 2000 elements 39 and 52; 4096 x 32000 47 and 53); 32-bit rows of 1024 elements 49 and 55, of 2048 79 and 102.
template <int DT, int NT, int KK, class EPI>
__global__ void __launch_bounds__(512, 2) dfx_gemm_lone_kernel(GemmSource w, GemmOperand x, uint32_t height, EPI epi) {
  constexpr int P = gemm_planes(DT), V = DT == DFX_F32 ? 2 : 1, N = 16 / (int)sizeof(typename StepElem<DT>::raw), ROWS = 16 * NT, PITCH = ROWS + 1;
  constexpr int PART = DT == DFX_F32 ? 4 : 8, H = (KK + PART - 1) / PART, CK = KK / H;      // a row's elements are taken in H parts, which the registers hold twice
  __shared__ __align__(16) float sums[8 * 64 * PITCH];
  __shared__ float2 pairs[16 * ROWS];
  const uint32_t wave = threadIdx.x / kStepWave, lane = threadIdx.x % kStepWave, l = lane % 16u, g = lane / 16u, k0 = wave * KK * 32u + g * 8u;
  uint32_t m0 = blockIdx.x * height, end = min(w.rows, m0 + height);
  StepVec<DT, N> raw[2][CK][V];
  auto load = [&](int set, int i, int h) {
    const void* row = (const typename StepElem<DT>::raw*)w.p + (size_t)min(m0 + i * 16u + l, end - 1u) * w.stride;
#pragma unroll
    for (int kk = 0; kk < CK; ++kk)
#pragma unroll
      for (int v = 0; v < V; ++v) raw[set][kk][v] = gemm_row_part<DT>(row, k0 + (h * CK + kk) * 32u + v * N, w.dim);
  };
  load(0, 0, 0);
  GemmShort8 fx[NT][KK][P];              // (x is 0 from dim to its padded length, and here behind that)
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const uint32_t e = k0 + kk * 32u;
        fx[j][kk][p] = GemmShort8{0, 0, 0, 0, 0, 0, 0, 0};
        if (e < x.cols) fx[j][kk][p] = *(const STEP_GLOBAL GemmShort8*)(x.p + (size_t)p * x.plane + (size_t)(j * 16 + l) * x.stride + e);
      }
  for (uint32_t tile = blockIdx.x;;) {
    const uint32_t here = m0, till = end;
    GemmAcc acc[NT];
#pragma unroll
    for (int q = 0; q < 4 * H; ++q) {
      const int i = q / H, h = q % H, set = q & 1;
      if (q == 4 * H - 1) {              // the next tile's first rows
        m0 = min(m0 + gridDim.x * height, w.rows - 1u); end = min(w.rows, m0 + height);
      }
      load(set ^ 1, (q + 1) / H & 3, (q + 1) % H);
      if (h == 0)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[j] = GemmAcc{0, 0, 0, 0};
#pragma unroll
      for (int kk = 0; kk < CK; ++kk) {
        if ((wave + 1u) * KK * 32u > w.dim)
#pragma unroll
          for (int v = 0; v < V; ++v) gemm_row_end(raw[set][kk][v], k0 + (h * CK + kk) * 32u + v * N, w.dim);
        GemmShort8 fa[P];
        gemm_parts<DT>(raw[set][kk], fa);
#pragma unroll
        for (int pair = 0; pair < gemm_pairs(DT); ++pair)
#pragma unroll
          for (int j = 0; j < NT; ++j) acc[j] = gemm_mac<DT>(fa[P == 1 ? 0 : gemm_plane_a(pair)], fx[j][h * CK + kk][P == 1 ? 0 : gemm_plane_b(pair)], acc[j]);
      }
      if (h == H - 1)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) sums[(wave * 64u + i * 16u + 4u * g + e) * PITCH + j * 16 + l] = acc[j][e];
    }
    __syncthreads();
    GemmAcc v = {0, 0, 0, 0};
    const uint32_t n = threadIdx.x % ROWS, four = threadIdx.x / ROWS;
    if (four < 16u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = sums[(four * 4u + e) * PITCH + n];
#pragma unroll
        for (uint32_t q = 1; q < 8; ++q) v[e] += sums[(q * 64u + four * 4u + e) * PITCH + n];
      }
    epi.template of_fours<ROWS>(tile, here, till, v, pairs);
    tile += gridDim.x;
    if (tile * height >= w.rows) break;
    __syncthreads();
  }
}

// A part of dX: 16 E elements of a row of W, by N rows of dz, summed over rows of W, 32 of each 128 by each of four waves.  A lane reads E elements of eight rows, and
// so holds eight k's of each of E tiles whose rows are E elements apart.  (E = 8, 16 bytes of 16-bit rows, takes too many registers by 64 rows: 48 x 1024 x 32000 22.5 us and 18.)
// 8 x 3840 x 72397 bf16 112 us, 5.0 TB/s.
template <int DT, int NT>
__global__ void __launch_bounds__(256, DT == DFX_F32 && NT == 4 ? 1 : 2) dfx_gemm_few_dx_kernel(GemmSource w, GemmOperand b, GemmShape s, float* part, uint32_t rows, uint32_t pitch, bool more) {
  constexpr int E = gemm_few_e(DT, NT);
  GemmFew<NT, E / 4> tile;
  constexpr int P = gemm_planes(DT), PLANE = 16 * NT * kGemmK * 2, STAGE = 2 * P * PLANE, PITCH = 16 * E + 4, SUMS = 4 * 16 * PITCH * 4;
  __shared__ __align__(1024) unsigned char lds[2 * STAGE > SUMS ? 2 * STAGE : SUMS];
  uint32_t begin, end;
  const GemmPlace at = gemm_work(s, blockIdx.x, tile, begin, end);
  if (!at.any) return;
  GemmAcc acc[E][NT];
#pragma unroll
  for (int i = 0; i < E; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = GemmAcc{0, 0, 0, 0};
  const uint32_t wave = threadIdx.x / kStepWave, lane = threadIdx.x % kStepWave, g = lane / 16u, l = lane % 16u, e = tile.m0 + E * l;
  StepVec<DT, E> raw[2][8];
  GemmNext next(begin, end, end - begin);
  auto load_w = [&](int set) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t v = min(next.k * kFewK + wave * 32u + g * 8u + j, w.rows - 1u);
      raw[set][j].load((const typename StepElem<DT>::raw*)w.p + (size_t)v * w.stride, min(e, w.dim - E));
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  auto load_b = [&](uint32_t k, uint32_t stage) {
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int p = 0; p < P; ++p) gemm_fetch<16 * NT, 256, false>(b, p, tile.n0, k * kFewK + half * kGemmK, lds + stage * STAGE + (half * P + p) * PLANE);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  auto step = [&](int set, uint32_t k) {
    gemm_wait<8>();                      // dz of this step and its part of W; the next one's rows of W are under way
    gemm_meet();
    if (tile.m0 + 16u * E > w.dim)
#pragma unroll
      for (int j = 0; j < 8; ++j) gemm_row_end(raw[set][j], e, w.dim);
    GemmShort8 fa[E][P];
#pragma unroll
    for (int t = 0; t < E; ++t) {
      if constexpr (DT == DFX_F32) {
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = raw[set][j].get(t);
        uint32_t p[3][4];
        gemm_cut8(x, p);
#pragma unroll
        for (int q = 0; q < 3; ++q) fa[t][q] = __builtin_bit_cast(GemmShort8, p[q]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) fa[t][0][j] = (short)(raw[set][j].w[t / 2] >> (t % 2 * 16));
      }
    }
    load_b(min(k + 1u, end - 1u), set ^ 1);
    load_w(set);
    next.advance();
    const unsigned char* lb = lds + set * STAGE + wave / 2u * P * PLANE;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      GemmShort8 fb[P];
#pragma unroll
      for (int p = 0; p < P; ++p) fb[p] = gemm_read(lb + p * PLANE, j * 16, wave % 2u);
#pragma unroll
      for (int pair = 0; pair < gemm_pairs(DT); ++pair)
#pragma unroll
        for (int t = 0; t < E; ++t) acc[t][j] = gemm_mac<DT>(fa[t][P == 1 ? 0 : gemm_plane_a(pair)], fb[P == 1 ? 0 : gemm_plane_b(pair)], acc[t][j]);
    }
  };
  if (begin < end) {
    load_w(0);
    next.advance();
    load_b(begin, 0);
    load_w(1);
    next.advance();
    for (uint32_t k = begin; k < end; k += 2) {
      step(0, k);
      if (k + 1u < end) step(1, k + 1u);
    }
    gemm_wait<0>();
    gemm_meet();
  }
  float* sums = (float*)lds;             // [wave][n][PITCH]
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    __syncthreads();
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int t = 0; t < E; t += 4) {
        const GemmAcc four = {acc[t][j][x], acc[t + 1][j][x], acc[t + 2][j][x], acc[t + 3][j][x]};
        *(GemmAcc*)(sums + (wave * 16u + l) * PITCH + E * (4u * g + x) + t) = four;
      }
    __syncthreads();
#pragma unroll
    for (uint32_t q = threadIdx.x; q < 16u * 4u * E; q += 256u) {
      const uint32_t n = q / (4u * E), d = q % (4u * E) * 4u;
      GemmAcc sum = *(const GemmAcc*)(sums + n * PITCH + d);
#pragma unroll
      for (uint32_t x = 1; x < 4; ++x) sum += *(const GemmAcc*)(sums + (x * 16u + n) * PITCH + d);
      if (tile.m0 + d < pitch) {
        GemmAcc* to = (GemmAcc*)(part + ((size_t)at.split * rows + tile.n0 + j * 16 + n) * pitch + tile.m0 + d);
        *to = more ? *to + sum : sum;
      }
    }
  }
}

// dW of few rows, whose sums are a step or two long: writing it is what takes the time.  A wave has 32 elements of x's rows in registers, all the sums' length, and goes from
// 64 rows of dW to others; the next ones' dz is on its way meanwhile.  Its two tiles' rows are exchanged in fours, so that a lane has eight elements of dW side by side.
// 48 x 1024 x 32000 f16 20 us, 8 x 3840 x 72397 bf16 141 us: 3.3 and 3.9 TB/s, all of it writes.
template <int DT, int STEPS, class OUT>
__global__ void __launch_bounds__(256, DT == DFX_F32 ? 1 : 3) dfx_gemm_few_dw_kernel(GemmOperand x, GemmOperand z, const uint32_t* count, uint32_t mtiles, uint32_t ntiles, uint32_t each, OUT out) {
  constexpr int P = gemm_planes(DT), PLANE = 64 * kGemmK * 2, STAGE = STEPS * P * PLANE, WIDE = 128, NT = 4;
  constexpr int LDS = 2 * STAGE > WIDE * kGemmK * 2 ? 2 * STAGE : WIDE * kGemmK * 2;
  __shared__ __align__(1024) unsigned char lds[LDS];
  const uint32_t m0 = blockIdx.x % mtiles * WIDE, first = blockIdx.x / mtiles, wave = threadIdx.x / kStepWave, lane = threadIdx.x % kStepWave, l = lane % 16u, g = lane / 16u;
  const uint32_t steps = min((*count + kGemmK - 1) / kGemmK, (uint32_t)STEPS);
  GemmShort8 fa[2][STEPS][2][P];
#pragma unroll
  for (int s = 0; s < STEPS; ++s)
#pragma unroll
    for (int p = 0; p < P; ++p) {
      if ((uint32_t)s < steps) gemm_fetch<WIDE, 256, true>(x, p, m0, s * kGemmK, lds);
      __syncthreads();
      const uint32_t k = 8u * g + l / 4u, q = l & 3u;
      GemmLds* at = (GemmLds*)lds + k * (WIDE * 2u) + (((wave * 2u + q / 2u) ^ gemm_turned_swap<WIDE>(k)) * 32u) + (q & 1u) * 16u;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
          const GemmShort4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) GemmShort4*)(at + kk * 32 * WIDE * 2 + t * 8));
          const GemmShort4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) GemmShort4*)(at + kk * 32 * WIDE * 2 + 4 * WIDE * 2 + t * 8));
          fa[t][s][kk][p] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
      __syncthreads();
    }
  auto load = [&](uint32_t n, uint32_t stage) {
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
      if ((uint32_t)s < steps)
#pragma unroll
        for (int p = 0; p < P; ++p) gemm_fetch<64, 256, true>(z, p, n * 64u, s * kGemmK, lds + stage * STAGE + (s * P + p) * PLANE);
  };
  if (first < ntiles) load(first, 0);
  uint32_t stage = 0;
  for (uint32_t n = first; n < ntiles; n += each, stage ^= 1u) {
    gemm_wait<0>();
    gemm_meet();
    if (n + each < ntiles) load(n + each, stage ^ 1u);
    GemmAcc acc[2][NT];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[t][j] = GemmAcc{0, 0, 0, 0};
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
      if ((uint32_t)s < steps) {
        GemmShort8 fb[P][NT][2];
#pragma unroll
        for (int p = 0; p < P; ++p) gemm_read_turned<NT, 64>(lds + stage * STAGE + (s * P + p) * PLANE, 0, fb[p]);
#pragma unroll
        for (int pair = 0; pair < gemm_pairs(DT); ++pair)
#pragma unroll
          for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
              for (int t = 0; t < 2; ++t) acc[t][j] = gemm_mac<DT>(fa[t][s][kk][P == 1 ? 0 : gemm_plane_a(pair)], fb[P == 1 ? 0 : gemm_plane_b(pair)][j][kk], acc[t][j]);
      }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = acc[e / 4][j][e % 4];
      out.put8(n * 64u + j * 16u + l, m0 + wave * 32u + g * 8u, v);
    }
  }
}

}  // namespace

#endif

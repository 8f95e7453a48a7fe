// Rows of an embedding table by token, and the table's gradient.
//
// The gradient of a row is the sum of the gradients of its token's places.  The places are sorted by token (stable, so that each token's stand in
// their order), and the sums are taken along the sorted places, so many at a time whatever the tokens are: a token that stands in every other place
// of a batch is shared by as many workgroups as its places are worth.  No atomics, so that the same call gives the same bits.
#include <float.h>
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>

#include "dfx_step.h"

namespace {

constexpr int kEmbedThreads = 256;
constexpr uint32_t kSortThreads = 512, kSortWaves = kSortThreads / kStepWave, kSortChunks = 256, kSortChunk = 2048;      // chunks at most, places of one at least
constexpr uint32_t kDigitBits = 10;      // at most
// places of a block of the sums at most; blocks, where they are fewer (us, on the same memory each time, some of it in the caches: 16384 x 4096 bf16 onto 131072 rows 256 98, 512 78, 1024 91;
// x 1024 87, 65, 62; 4000 x 1024 onto 50000 28, 25, 30)
constexpr uint32_t kSumMost = 64, kSumBlocks = 512;

struct EmbedArgs {
  const int64_t* tokens;
  const void* table;
  void* out;
  size_t table_stride, out_stride;
  uint32_t rows, dim, vocab, lanes, lanes_log2;      // lanes: threads to a row, a power of two
  float scale;
};

// N elements from element e on of a row: whole, or what there is of them
template <int DT, int N>
__device__ __forceinline__ void part_take(const void* row, uint32_t e, uint32_t dim, float* v) {
  if (e + N <= dim) {
    StepVec<DT, N> a;
    a.load(row, e);
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = a.get(k);
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = e + k < dim ? step_get<DT>(row, e + k) : 0.0f;
  }
}
template <int DT, int N, bool STREAM = false>
__device__ __forceinline__ void part_put(void* row, uint32_t e, uint32_t dim, const float* v) {
  if (e + N <= dim) {
    if constexpr (N * (DT == DFX_F32 ? 4 : 2) == 32) {
      StepVec<DT, N / 2> a, b;
      a.put(v); b.put(v + N / 2);
      typedef typename StepVec<DT, N / 2>::words words;
      STEP_GLOBAL words* to = (STEP_GLOBAL words*)((STEP_GLOBAL typename StepElem<DT>::raw*)row + e);
      to[0] = a.w; to[1] = b.w;
    } else {
      StepVec<DT, N> a;
      a.put(v);
      if (STREAM) a.stream(row, e);
      else *(STEP_GLOBAL typename StepVec<DT, N>::words*)((STEP_GLOBAL typename StepElem<DT>::raw*)row + e) = a.w;
    }
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (e + k < dim) step_put<DT>(row, e + k, v[k]);
  }
}

// a.lanes threads to a row; what is written goes past the caches.  HBM's writes bound it: 16384 x 4096 bf16 31 us, 6.1 TB/s; one row 1.7.
template <int DT>
__global__ void __launch_bounds__(kEmbedThreads) dfx_embed_kernel(EmbedArgs a) {
  typedef typename StepElem<DT>::raw raw;
  constexpr uint32_t N = 16 / sizeof(raw);
  const uint32_t row = blockIdx.x * (kEmbedThreads >> a.lanes_log2) + (threadIdx.x >> a.lanes_log2);
  if (row >= a.rows) return;
  const int64_t t = ((const STEP_GLOBAL int64_t*)a.tokens)[row];
  const bool any = t >= 0 && t < (int64_t)a.vocab;
  const raw* from = (const raw*)a.table + (any ? (size_t)t : 0) * a.table_stride;
  raw* to = (raw*)a.out + (size_t)row * a.out_stride;
  for (uint32_t e = (blockIdx.y * a.lanes + (threadIdx.x & (a.lanes - 1u))) * N; e < a.dim; e += gridDim.y * a.lanes * N) {
    float v[N];
    if (any) {
      part_take<DT, N>(from, e, a.dim, v);
#pragma unroll
      for (int k = 0; k < (int)N; ++k) v[k] *= a.scale;
    } else {
#pragma unroll
      for (int k = 0; k < (int)N; ++k) v[k] = 0.0f;
    }
    part_put<DT, N, true>(to, e, a.dim, v);
  }
}

// ------------------------------------------------------------------------------------------
// places sorted by token: passes over digits, the lowest first, each of which counts a chunk's digits and then moves its places
// ------------------------------------------------------------------------------------------
struct SortArgs {
  const int64_t* tokens;                 // of the first pass, else null
  const uint2* from;                     // (token, place)
  uint2* to;
  uint32_t* counts;                      // [chunks][digits]
  uint32_t n, vocab, chunk, shift, bits;
};

// A token's key: itself, or vocab for none.
__device__ __forceinline__ uint2 sort_take(const SortArgs& a, uint32_t i) {
  if (!a.tokens) return a.from[i];
  const int64_t t = a.tokens[i];
  return make_uint2(t >= 0 && t < (int64_t)a.vocab ? (uint32_t)t : a.vocab, i);
}
__device__ __forceinline__ uint32_t sort_digit(const SortArgs& a, uint32_t key) { return (key >> a.shift) & ((1u << a.bits) - 1u); }

__global__ void __launch_bounds__(kSortThreads) dfx_embed_count_kernel(SortArgs a) {
  __shared__ uint32_t hist[1u << kDigitBits];
  const uint32_t digits = 1u << a.bits;
  for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads) hist[d] = 0;
  __syncthreads();
  const uint32_t begin = blockIdx.x * a.chunk, end = min(a.n, begin + a.chunk);
  for (uint32_t i = begin + threadIdx.x; i < end; i += kSortThreads) atomicAdd(&hist[sort_digit(a, sort_take(a, i).x)], 1u);
  __syncthreads();
  for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads) a.counts[blockIdx.x * digits + d] = hist[d];
}

// Where a digit's places begin: those of smaller digits, then those of earlier chunks, then those of earlier waves, each of which has its own part of
// the chunk.  A wave takes 64 places at a time; lanes of one digit find each other by its bits.
__global__ void __launch_bounds__(kSortThreads) dfx_embed_move_kernel(SortArgs a) {
  __shared__ uint32_t at[kSortWaves][1u << kDigitBits];
  __shared__ uint32_t sums[kSortWaves];
  const uint32_t digits = 1u << a.bits, me = threadIdx.x, wave = me / kStepWave, lane = me % kStepWave;
  for (uint32_t d = me; d < kSortWaves * digits; d += kSortThreads) at[d / digits][d % digits] = 0;
  __syncthreads();
  const uint32_t begin = blockIdx.x * a.chunk, end = min(a.n, begin + a.chunk), each = (a.chunk + kSortWaves - 1u) / kSortWaves;
  const uint32_t mine = min(end, begin + wave * each), stop = min(end, mine + each);
  for (uint32_t i = mine + lane; i < stop; i += kStepWave) atomicAdd(&at[wave][sort_digit(a, sort_take(a, i).x)], 1u);
  __syncthreads();
  // a thread has one or two digits that follow one another
  const uint32_t per = digits > kSortThreads ? digits / kSortThreads : 1u;
  uint32_t total = 0, earlier[2] = {0, 0}, own[2] = {0, 0};
  for (uint32_t q = 0; q < per; ++q) {
    const uint32_t d = me * per + q;
    if (d >= digits) break;
    uint32_t all = 0;
    for (uint32_t c = 0; c < gridDim.x; ++c) {
      const uint32_t k = a.counts[c * digits + d];
      earlier[q] += c < blockIdx.x ? k : 0u;
      all += k;
    }
    own[q] = total;                      // (of this thread's digits before)
    total += all;
  }
  uint32_t sum = total;                  // over the threads up to this one
  for (uint32_t d = 1; d < kStepWave; d <<= 1) {
    const uint32_t more = __shfl_up(sum, d);
    if (lane >= d) sum += more;
  }
  if (lane == kStepWave - 1u) sums[wave] = sum;
  __syncthreads();
  uint32_t before = sum - total;
  for (uint32_t w = 0; w < wave; ++w) before += sums[w];
  for (uint32_t q = 0; q < per; ++q) {
    const uint32_t d = me * per + q;
    if (d >= digits) break;
    uint32_t place = before + own[q] + earlier[q];
    for (uint32_t w = 0; w < kSortWaves; ++w) {
      const uint32_t k = at[w][d];
      at[w][d] = place;
      place += k;
    }
  }
  __syncthreads();
  for (uint32_t first = mine; first < stop; first += kStepWave) {
    const uint32_t i = first + lane;
    const bool has = i < stop;
    const uint2 x = has ? sort_take(a, i) : make_uint2(0, 0);
    const uint32_t d = sort_digit(a, x.x);
    uint64_t same = __ballot(has);
    for (uint32_t b = 0; b < a.bits; ++b) {
      const uint64_t set = __ballot((d >> b) & 1u);
      same &= (d >> b) & 1u ? set : ~set;
    }
    if (has) {
      const uint32_t place = at[wave][d];
      a.to[place + (uint32_t)__popcll(same & ((1ull << lane) - 1ull))] = x;
      if (lane == (uint32_t)__ffsll((long long)same) - 1u) at[wave][d] = place + (uint32_t)__popcll(same);      // (behind every lane's read: a wave's LDS accesses keep their order)
    }
  }
}

// The same in one launch where there are few places and not very many tokens: a workgroup has the tokens of one remainder by kOwners.  It looks at all places, counts those
// of smaller remainders, which come first, keeps its own in LDS in their order, and sorts them by the quotient: places of a quotient are counted, and one wave moves them, 64
// at a time.  The workgroups behind clear the table's gradient meanwhile.  16384 places 19.6 us: the chain of one wave's rounds over its share and the counts before it.  In all, by this and by
// the passes, on the same memory each time: 4000 x 1024 28 us and 37, 16384 x 4096 82 and 86 (from HBM 104).
constexpr uint32_t kOwnMost = 16384, kOwnBits = 7, kOwners = 1u << kOwnBits, kOwnThreads = 1024, kOwnWaves = kOwnThreads / kStepWave, kOwnQuotients = 2 * kOwnThreads;

template <int OUT>
__device__ __forceinline__ void clear_row(void* out, size_t stride, uint32_t dim, uint32_t row) {
  constexpr uint32_t N = 16 / sizeof(typename StepElem<OUT>::raw);
  typename StepElem<OUT>::raw* at = (typename StepElem<OUT>::raw*)out + (size_t)row * stride;
  float zero[N];
#pragma unroll
  for (int k = 0; k < (int)N; ++k) zero[k] = 0.0f;
  for (uint32_t e = threadIdx.x * N; e < dim; e += blockDim.x * N) part_put<OUT, N, true>(at, e, dim, zero);
}

// The whole table, by `groups` workgroups of which this one is the group-th: where its rows follow one another as one piece of memory, in vectors at multiples of 16 bytes (35146 rows of
// 657 bf16: row for row 62 us of the gradient of 758 places, so 28).
template <int OUT>
__device__ __forceinline__ void clear_table(void* out, size_t stride, uint32_t dim, uint32_t vocab, uint32_t group, uint32_t groups) {
  typedef typename StepElem<OUT>::raw raw;
  if (stride != dim) {
    for (uint32_t row = group; row < vocab; row += groups) clear_row<OUT>(out, stride, dim, row);
    return;
  }
  constexpr uint32_t N = 16 / sizeof(raw);
  const size_t all = (size_t)vocab * dim, head = min(all, (size_t)((16u - (uint32_t)((uintptr_t)out & 15u)) & 15u) / sizeof(raw)), vectors = (all - head) / N;
  StepVec<OUT, (int)N> zero;
  zero.w = 0;
  raw* body = (raw*)out + head;
  for (size_t v = (size_t)group * blockDim.x + threadIdx.x; v < vectors; v += (size_t)groups * blockDim.x) zero.stream(body, v * N);
  if (group == 0 && threadIdx.x < 2 * N) {
    const size_t i = threadIdx.x < N ? (size_t)threadIdx.x : head + vectors * N + threadIdx.x - N;      // in front of the vectors, behind them
    if (threadIdx.x < N ? i < head : i < all) step_put<OUT>(out, i, 0.0f);
  }
}

template <int OUT>
__global__ void __launch_bounds__(kOwnThreads) dfx_embed_own_kernel(SortArgs a, void* out, size_t stride, uint32_t dim) {
  constexpr uint32_t U = kOwnMost / kOwnThreads;
  __shared__ uint16_t quotient[kOwnMost], place[kOwnMost];
  __shared__ uint32_t bin[kOwnQuotients], sums[kOwnWaves];
  __shared__ uint32_t counts[3][kOwnWaves];      // of smaller remainders, of this one, without a token
  const uint32_t me = threadIdx.x, wave = me / kStepWave, lane = me % kStepWave;
  if (blockIdx.x >= kOwners) {
    clear_table<OUT>(out, stride, dim, a.vocab, blockIdx.x - kOwners, gridDim.x - kOwners);
    return;
  }
  bin[2u * me] = bin[2u * me + 1u] = 0;
  // a wave has places that follow one another
  const uint32_t each = ((a.n + kOwnWaves - 1u) / kOwnWaves + kStepWave - 1u) / kStepWave * kStepWave;
  const uint32_t begin = min(a.n, wave * each), end = min(a.n, begin + each);
  uint32_t t[U], smaller = 0, here = 0, none = 0;
#pragma unroll
  for (uint32_t u = 0; u < U; ++u) {
    const uint32_t i = begin + u * kStepWave + lane;
    t[u] = i < end ? sort_take(a, i).x : ~0u;
  }
#pragma unroll
  for (uint32_t u = 0; u < U; ++u) {
    const uint32_t own = t[u] < a.vocab ? t[u] % kOwners : kOwners;
    smaller += (uint32_t)__popcll(__ballot(own < blockIdx.x));
    here += (uint32_t)__popcll(__ballot(own == blockIdx.x));
    none += (uint32_t)__popcll(__ballot(t[u] == a.vocab));
  }
  if (lane == 0) { counts[0][wave] = smaller; counts[1][wave] = here; counts[2][wave] = none; }
  __syncthreads();
  uint32_t base = 0, at = 0, all = 0, left = 0;
  for (uint32_t w = 0; w < kOwnWaves; ++w) {
    base += counts[0][w];
    at += w < wave ? counts[1][w] : 0u;
    all += counts[1][w];
    left += counts[2][w];
  }
#pragma unroll
  for (uint32_t u = 0; u < U; ++u) {
    const bool mine = t[u] < a.vocab && t[u] % kOwners == blockIdx.x;
    const uint64_t mask = __ballot(mine);
    if (mine) {
      const uint32_t to = at + (uint32_t)__popcll(mask & ((1ull << lane) - 1ull));
      quotient[to] = (uint16_t)(t[u] / kOwners);
      place[to] = (uint16_t)(begin + u * kStepWave + lane);
      atomicAdd(&bin[t[u] / kOwners], 1u);
    }
    at += (uint32_t)__popcll(mask);
  }
  __syncthreads();
  const uint32_t one = bin[2u * me], two = one + bin[2u * me + 1u];
  uint32_t sum = two;
#pragma unroll
  for (uint32_t d = 1; d < kStepWave; d <<= 1) {
    const uint32_t more = __shfl_up(sum, d);
    if (lane >= d) sum += more;
  }
  if (lane == kStepWave - 1u) sums[wave] = sum;
  __syncthreads();
  uint32_t before = base + sum - two;
  for (uint32_t w = 0; w < wave; ++w) before += sums[w];
  bin[2u * me] = before; bin[2u * me + 1u] = before + one;
  __syncthreads();
  if (wave == 0)
    for (uint32_t first = 0; first < all; first += kStepWave) {
      const uint32_t i = first + lane, q = i < all ? quotient[i] : 0u;
      uint64_t same = __ballot(i < all);
#pragma unroll
      for (uint32_t b = 0; b < 11; ++b) {
        const uint64_t set = __ballot((q >> b) & 1u);
        same &= (q >> b) & 1u ? set : ~set;
      }
      if (i < all) {
        const uint32_t to = bin[q];
        a.to[to + (uint32_t)__popcll(same & ((1ull << lane) - 1ull))] = make_uint2(q << kOwnBits | blockIdx.x, place[i]);
        if (lane == (uint32_t)__ffsll((long long)same) - 1u) bin[q] = to + (uint32_t)__popcll(same);      // (behind every lane's read)
      }
    }
  if (blockIdx.x == 0)                   // behind all tokens: as many places without one
    for (uint32_t i = me; i < left; i += kOwnThreads) a.to[a.n - 1u - i] = make_uint2(a.vocab, 0u);
}

// ------------------------------------------------------------------------------------------
// sums along the sorted places: 16384 x 4096 bf16 onto 131072 rows 72 us, 0.24 GB; a row onto the table waits for what the table holds, one token after the other
// ------------------------------------------------------------------------------------------
struct SumArgs {
  const uint2* sorted;
  const void* grad;
  void* out;
  float* part;                           // [blocks][2][dim]: of a block's first token that began before it, and of its last one that goes on behind it
  size_t grad_stride, out_stride;
  uint32_t n, dim, vocab, block, blocks, lanes, lanes_log2;
  float scale;
  bool accumulate;
};

template <int OUT, int N>
__device__ __forceinline__ void sum_put(const SumArgs& a, uint32_t token, uint32_t e, float* s) {
  typename StepElem<OUT>::raw* row = (typename StepElem<OUT>::raw*)a.out + (size_t)token * a.out_stride;
  float old[N];
#pragma unroll
  for (int k = 0; k < N; ++k) old[k] = 0.0f;
  if (a.accumulate) {
    if constexpr (N * (OUT == DFX_F32 ? 4 : 2) == 32) {
      part_take<OUT, N / 2>(row, e, a.dim, old);
      part_take<OUT, N / 2>(row, e + N / 2, a.dim, old + N / 2);
    } else part_take<OUT, N>(row, e, a.dim, old);
  }
#pragma unroll
  for (int k = 0; k < N; ++k) s[k] = a.accumulate ? fmaf(s[k], a.scale, old[k]) : s[k] * a.scale;
  part_put<OUT, N>(row, e, a.dim, s);
}

template <int DT, int OUT>
__global__ void __launch_bounds__(kEmbedThreads) dfx_embed_sum_kernel(SumArgs a) {
  typedef typename StepElem<DT>::raw raw;
  constexpr int N = 16 / (int)sizeof(raw), U = 8;
  const uint32_t b = blockIdx.x * (kEmbedThreads >> a.lanes_log2) + (threadIdx.x >> a.lanes_log2);
  const uint32_t e = (blockIdx.y * a.lanes + (threadIdx.x & (a.lanes - 1u))) * N;
  if (b >= a.blocks || e >= a.dim) return;
  const uint32_t begin = b * a.block, end = min(a.n, begin + a.block);
  float s[N];
#pragma unroll
  for (int k = 0; k < N; ++k) s[k] = 0.0f;
  uint32_t token = a.sorted[begin].x;
  if (token == a.vocab) return;          // (and all behind it: places without a token)
  bool from_before = begin > 0 && a.sorted[begin - 1].x == token;
  auto close = [&](bool goes_on) {
    if (from_before || goes_on) {
      float* to = a.part + ((size_t)b * 2u + (from_before ? 0u : 1u)) * a.dim;
#pragma unroll
      for (int k = 0; k < N; ++k)
        if (e + k < a.dim) to[e + k] = s[k];
    } else sum_put<OUT, N>(a, token, e, s);
  };
  for (uint32_t i = begin; i < end; i += U) {
    uint2 x[U];
    float v[U][N];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = i + u < end ? a.sorted[i + u] : make_uint2(a.vocab, 0);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (x[u].x != a.vocab) part_take<DT, N>((const raw*)a.grad + (size_t)x[u].y * a.grad_stride, e, a.dim, v[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u >= end) break;
      if (x[u].x != token) {
        close(false);
        from_before = false;
        token = x[u].x;
        if (token == a.vocab) return;
#pragma unroll
        for (int k = 0; k < N; ++k) s[k] = 0.0f;
      }
#pragma unroll
      for (int k = 0; k < N; ++k) s[k] += v[u][k];
    }
  }
  close(end < a.n && a.sorted[end].x == token);
}

// A token whose places go on behind the block that they begin in: its blocks' parts, in their order.  15 us of the same.
template <int OUT>
__global__ void __launch_bounds__(kEmbedThreads) dfx_embed_join_kernel(SumArgs a) {
  constexpr int N = 4;
  const uint32_t b = blockIdx.x * (kEmbedThreads >> a.lanes_log2) + (threadIdx.x >> a.lanes_log2);
  const uint32_t e = (blockIdx.y * a.lanes + (threadIdx.x & (a.lanes - 1u))) * N;
  if (b + 1u >= a.blocks || e >= a.dim) return;
  const uint32_t begin = b * a.block, end = begin + a.block, token = a.sorted[end - 1u].x;
  if (token == a.vocab || a.sorted[end].x != token) return;
  if (a.sorted[begin].x == token && begin > 0 && a.sorted[begin - 1u].x == token) return;      // (began before)
  float s[N];
  part_take<DFX_F32, N>(a.part + ((size_t)b * 2u + 1u) * a.dim, e, a.dim, s);
  constexpr uint32_t U = 16;             // blocks at once
  bool on = true;
  for (uint32_t c = b + 1u; on; c += U) {
    bool has[U];
    float v[U][N];
#pragma unroll
    for (uint32_t u = 0; u < U; ++u) has[u] = c + u < a.blocks && a.sorted[(size_t)(c + u) * a.block].x == token;
#pragma unroll
    for (uint32_t u = 0; u < U; ++u)
      if (has[u]) part_take<DFX_F32, N>(a.part + (size_t)(c + u) * 2u * a.dim, e, a.dim, v[u]);
#pragma unroll
    for (uint32_t u = 0; u < U; ++u)
      if (has[u])
#pragma unroll
        for (int k = 0; k < N; ++k) s[k] += v[u][k];
    on = has[U - 1u];
  }
  sum_put<OUT, N>(a, token, e, s);
}

// ------------------------------------------------------------------------------------------
// few places: no sort.  A workgroup finds the places of its rows of the table among all of them, in their order.  Onto the gradient that is there: a workgroup to a
// place, which does nothing if its token stood before; otherwise a workgroup to eight rows of the table.
// In all, by this and by the sort: 300 x 1024 bf16 7.0 us and 16.9, 500 x 4096 11.0 and 18.1.  A workgroup that has a frequent token adds up all its places in its part of the row: 300 x 1001 fp32,
// whole table of 5003 rows, 8.7 us without tokens (20 MB of zeros), 11 with tokens of three places at most, 15 with one of 16, 115 where all are the same (1024 elements, whose vectors lie at
// multiples of 16 bytes: 8.4, 10.2, 10.5, 37).
// ------------------------------------------------------------------------------------------
constexpr uint32_t kFewPlaces = 512, kFewTable = 8;
// From so many rows on, the table is cleared first, a launch more, and the sums added onto it (us, cleared first and not: 300 x 368 by 86505 fp32 28 and 47, 129 x 448 by 21904 bf16 10 and 15, 26 x
// 1001 by 10000 fp32 level, 300 x 1001 by 5003 14.7 and 16.2; below, it goes by the launch that it spares).
constexpr size_t kFewClear = 16384;
constexpr size_t kClearGroups = 8192;    // workgroups of the clearing, at most: 86505 x 368 fp32 in some 20 us, 6 TB/s

template <int DT, int OUT>
__global__ void __launch_bounds__(kEmbedThreads) dfx_embed_few_kernel(SumArgs a, const int64_t* tokens) {
  typedef typename StepElem<DT>::raw raw;
  constexpr int N = 16 / (int)sizeof(raw), U = 64 / N;
  constexpr uint32_t W = kFewPlaces / kStepWave, R = kFewPlaces / kEmbedThreads;      // groups of 64 places; a thread's places
  __shared__ uint32_t place[kFewPlaces], counts[kFewTable][W], start[kFewTable + 1];
  const uint32_t me = threadIdx.x, lane = me % kStepWave;
  int64_t first = (int64_t)blockIdx.x * kFewTable;
  uint32_t table = kFewTable;
  if (a.accumulate) {
    first = tokens[blockIdx.x]; table = 1;
    if (first < 0 || first >= (int64_t)a.vocab) return;
  }
  uint64_t same[R];                      // lanes whose places have this one's token
  uint32_t row[R];
  bool stood = false;
#pragma unroll
  for (uint32_t r = 0; r < R; ++r) {
    const uint32_t i = r * kEmbedThreads + me;
    const int64_t t = i < a.n ? tokens[i] : -1;
    row[r] = t >= first && t < first + table && t < (int64_t)a.vocab ? (uint32_t)(t - first) : kFewTable;
    stood = stood || (a.accumulate && row[r] < kFewTable && i < blockIdx.x);
    for (uint32_t q = 0; q < table; ++q) {
      const uint64_t mask = __ballot(row[r] == q);
      if (row[r] == q) same[r] = mask;
      if (lane == 0) counts[q][i / kStepWave] = (uint32_t)__popcll(mask);
    }
  }
  if (__syncthreads_or(stood)) return;
  if (me <= table) {
    uint32_t before = 0;
    for (uint32_t q = 0; q < me; ++q)
      for (uint32_t w = 0; w < W; ++w) before += counts[q][w];
    start[me] = before;
  }
  __syncthreads();
#pragma unroll
  for (uint32_t r = 0; r < R; ++r)
    if (row[r] < kFewTable) {
      uint32_t to = start[row[r]] + (uint32_t)__popcll(same[r] & ((1ull << lane) - 1ull));
      for (uint32_t w = 0; w < (r * kEmbedThreads + me) / kStepWave; ++w) to += counts[row[r]][w];
      place[to] = r * kEmbedThreads + me;
    }
  __syncthreads();
  for (uint32_t q = 0; q < table; ++q) {
    const int64_t v = first + q;
    if (v >= (int64_t)a.vocab) return;
    const uint32_t begin = start[q], end = start[q + 1];
    for (uint32_t e = (blockIdx.y * kEmbedThreads + me) * N; e < a.dim; e += gridDim.y * kEmbedThreads * N) {
      float s[N];
#pragma unroll
      for (int k = 0; k < N; ++k) s[k] = 0.0f;
      for (uint32_t i = begin; i < end; i += U) {
        float x[U][N];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (i + u < end) part_take<DT, N>((const raw*)a.grad + (size_t)place[i + u] * a.grad_stride, e, a.dim, x[u]);
          else
#pragma unroll
            for (int k = 0; k < N; ++k) x[u][k] = 0.0f;
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int k = 0; k < N; ++k) s[k] += x[u][k];
      }
      sum_put<OUT, N>(a, (uint32_t)v, e, s);
    }
  }
}

template <int OUT>
__global__ void __launch_bounds__(kEmbedThreads) dfx_embed_clear_kernel(void* out, size_t stride, uint32_t dim, uint32_t vocab) {
  clear_table<OUT>(out, stride, dim, vocab, blockIdx.x, gridDim.x);
}

// ------------------------------------------------------------------------------------------
constexpr size_t kMostRows = (1ull << 31) - 1024, kMostStride = 1ull << 20;
constexpr size_t kRowsAtOnce = 1ull << 22;      // workgroups of a launch (whose threads are counted in 32 bits)

uint32_t lanes_log2(uint32_t vectors) {
  uint32_t k = 0;
  while ((1u << k) < vectors && (1u << k) < (uint32_t)kEmbedThreads) ++k;
  return k;
}

struct SortPlan {
  uint32_t chunk, chunks, bits, passes, block, blocks;
  size_t pairs[2], counts, part, bytes;
};
size_t up(size_t n, size_t to) { return (n + to - 1) / to * to; }

SortPlan sort_plan(size_t rows, size_t dim, size_t vocab) {
  SortPlan p;
  memset(&p, 0, sizeof(p));
  p.chunk = (uint32_t)std::max<size_t>(kSortChunk, (rows + kSortChunks - 1) / kSortChunks);
  p.chunks = (uint32_t)((rows + p.chunk - 1) / p.chunk);
  uint32_t bits = 1;
  while ((uint64_t)vocab >> bits) ++bits;
  p.passes = (bits + kDigitBits - 1) / kDigitBits;
  p.bits = (bits + p.passes - 1) / p.passes;
  uint32_t block = 4;
  while (block < kSumMost && (rows + block - 1) / block > kSumBlocks) block *= 2;
  p.block = block;
  p.blocks = (uint32_t)((rows + block - 1) / block);
  // (the parts of the sums have room for any number of rows up to these)
  const size_t most = std::max<size_t>(std::min<size_t>((rows + 3) / 4, kSumBlocks), (rows + kSumMost - 1) / kSumMost);
  size_t at = 0;
  auto take = [&](size_t n) { const size_t here = at; at += up(n, 256); return here; };
  p.pairs[0] = take(rows * sizeof(uint2));
  p.pairs[1] = take(rows * sizeof(uint2));
  p.counts = take(std::min<size_t>(kSortChunks, (rows + kSortChunk - 1) / kSortChunk) * (1u << kDigitBits) * 4);
  p.part = take(most * 2 * dim * 4);
  p.bytes = std::max<size_t>(at, 16);
  return p;
}

bool embed_types(int dtype, int out) { return (dtype == DFX_F32 || dtype == DFX_BF16 || dtype == DFX_F16) && (out == dtype || out == DFX_F32); }

template <int DT, int OUT>
int embed_sums(const SumArgs& a, hipStream_t s) {
  constexpr uint32_t N = 16 / sizeof(typename StepElem<DT>::raw);
  SumArgs x = a;
  const uint32_t vectors = (a.dim + N - 1) / N, quads = (a.dim + 3) / 4;
  x.lanes_log2 = lanes_log2(vectors); x.lanes = 1u << x.lanes_log2;
  const uint32_t groups = kEmbedThreads >> x.lanes_log2;
  const int rc = step_launch(dfx_embed_sum_kernel<DT, OUT>, dim3((a.blocks + groups - 1) / groups, (vectors + x.lanes - 1) / x.lanes), kEmbedThreads, s, x);
  if (rc != DFX_OK || a.blocks < 2) return rc;
  x.lanes_log2 = lanes_log2(quads); x.lanes = 1u << x.lanes_log2;
  const uint32_t more = kEmbedThreads >> x.lanes_log2;
  return step_launch(dfx_embed_join_kernel<OUT>, dim3((a.blocks + more - 1) / more, (quads + x.lanes - 1) / x.lanes), kEmbedThreads, s, x);
}

}  // namespace

extern "C" {

int dfx_embed(const dfx_embed_args* u, void* hip_stream) {
  if (!u || u->struct_bytes != sizeof(*u) || !embed_types(u->dtype, u->dtype)) return DFX_ERR_INVALID_ARG;
  if (u->rows >= kMostRows || u->vocab >= kMostRows || u->dim >= kMostStride || u->table_stride >= kMostStride || u->out_stride >= kMostStride) return DFX_ERR_TOO_LARGE;
  const size_t eb = step_elem_bytes(u->dtype), ts = u->table_stride ? u->table_stride : u->dim, os = u->out_stride ? u->out_stride : u->dim;
  if (ts < u->dim || os < u->dim || !step_fits(u->scale)) return DFX_ERR_INVALID_ARG;
  if (!u->rows || !u->dim) return DFX_OK;
  if (!u->tokens || (uintptr_t)u->tokens % 8 || !u->out || (uintptr_t)u->out % eb || (u->vocab && !u->table) || (uintptr_t)u->table % eb) return DFX_ERR_INVALID_ARG;
  const Span out = flat(u->out, ((u->rows - 1) * os + u->dim) * eb);
  if (meet(out, flat(u->tokens, 8 * u->rows)) || (u->vocab && meet(out, flat(u->table, ((u->vocab - 1) * ts + u->dim) * eb)))) return DFX_ERR_INVALID_ARG;
  EmbedArgs a;
  memset(&a, 0, sizeof(a));
  a.tokens = u->tokens; a.table = u->table; a.out = u->out; a.table_stride = ts; a.out_stride = os;
  a.rows = (uint32_t)u->rows; a.dim = (uint32_t)u->dim; a.vocab = (uint32_t)u->vocab; a.scale = (float)u->scale;
  const uint32_t N = 16 / (uint32_t)eb, vectors = (a.dim + N - 1) / N;
  a.lanes_log2 = lanes_log2(vectors); a.lanes = 1u << a.lanes_log2;
  const uint32_t groups = kEmbedThreads >> a.lanes_log2;
  auto k = u->dtype == DFX_F32 ? dfx_embed_kernel<DFX_F32> : u->dtype == DFX_BF16 ? dfx_embed_kernel<DFX_BF16> : dfx_embed_kernel<DFX_F16>;
  for (size_t first = 0; first < u->rows; first += kRowsAtOnce) {
    a.tokens = u->tokens + first; a.out = (unsigned char*)u->out + first * os * eb;
    a.rows = (uint32_t)std::min(kRowsAtOnce, u->rows - first);
    const int rc = step_launch(k, dim3((a.rows + groups - 1) / groups, std::min(4u, (vectors + a.lanes - 1) / a.lanes)), kEmbedThreads, (hipStream_t)hip_stream, a);
    if (rc != DFX_OK) return rc;
  }
  return DFX_OK;
}

size_t dfx_embed_grad_workspace(size_t rows, size_t dim, size_t vocab, dfx_dtype dtype) {
  (void)dtype;
  if (rows >= kMostRows || vocab >= kMostRows || dim >= kMostStride) return 0;
  return sort_plan(rows, dim, vocab).bytes;
}

int dfx_embed_grad(const dfx_embed_grad_args* u, void* hip_stream) {
  if (!u || u->struct_bytes != sizeof(*u) || !embed_types(u->dtype, u->out_dtype)) return DFX_ERR_INVALID_ARG;
  if (u->rows >= kMostRows || u->vocab >= kMostRows || u->dim >= kMostStride || u->grad_stride >= kMostStride || u->table_grad_stride >= kMostStride) return DFX_ERR_TOO_LARGE;
  const size_t eb = step_elem_bytes(u->dtype), ob = step_elem_bytes(u->out_dtype), gs = u->grad_stride ? u->grad_stride : u->dim, os = u->table_grad_stride ? u->table_grad_stride : u->dim;
  if (gs < u->dim || os < u->dim || !step_fits(u->scale)) return DFX_ERR_INVALID_ARG;
  if (!u->vocab || !u->dim) return DFX_OK;
  if ((u->rows && (!u->tokens || !u->grad)) || (uintptr_t)u->tokens % 8 || (uintptr_t)u->grad % eb || !u->table_grad || (uintptr_t)u->table_grad % ob) return DFX_ERR_INVALID_ARG;
  const SortPlan p = sort_plan(u->rows, u->dim, u->vocab);
  if (!u->workspace || (uintptr_t)u->workspace % 16 || u->workspace_bytes < p.bytes) return DFX_ERR_INVALID_ARG;
  const Span tokens = flat(u->tokens, 8 * u->rows), grad = flat(u->grad, u->rows ? ((u->rows - 1) * gs + u->dim) * eb : 0), work = flat(u->workspace, p.bytes);
  const Span out = flat(u->table_grad, ((u->vocab - 1) * os + u->dim) * ob);
  if (meet(out, tokens) || meet(out, grad) || meet(out, work) || meet(work, tokens) || meet(work, grad)) return DFX_ERR_INVALID_ARG;
  hipStream_t s = (hipStream_t)hip_stream;
  unsigned char* ws = (unsigned char*)u->workspace;
  SumArgs a;
  memset(&a, 0, sizeof(a));
  a.grad = u->grad; a.out = u->table_grad; a.part = (float*)(ws + p.part); a.grad_stride = gs; a.out_stride = os;
  a.n = (uint32_t)u->rows; a.dim = (uint32_t)u->dim; a.vocab = (uint32_t)u->vocab; a.block = p.block; a.blocks = p.blocks; a.scale = (float)u->scale; a.accumulate = u->accumulate != 0;
  auto clear = [&]() -> int {
    auto k = u->out_dtype == DFX_F32 ? dfx_embed_clear_kernel<DFX_F32> : u->out_dtype == DFX_BF16 ? dfx_embed_clear_kernel<DFX_BF16> : dfx_embed_clear_kernel<DFX_F16>;
    const size_t groups = os == u->dim ? u->vocab * u->dim * ob / (16 * kEmbedThreads) + 1 : u->vocab;
    return step_launch(k, dim3((uint32_t)std::min(groups, kClearGroups)), kEmbedThreads, s, u->table_grad, os, (uint32_t)u->dim, (uint32_t)u->vocab);
  };
  if (u->rows && u->rows <= kFewPlaces) {
    if (!a.accumulate && u->vocab >= kFewClear) {
      const int rc = clear();
      if (rc != DFX_OK) return rc;
      a.accumulate = true;
    }
    const uint32_t at_once = kEmbedThreads * 16 / (uint32_t)eb;      // elements of a row that a workgroup has
    const dim3 grid(a.accumulate ? a.n : (uint32_t)((u->vocab + kFewTable - 1) / kFewTable), std::min(8u, (a.dim + at_once - 1) / at_once));
    const bool wide = u->out_dtype == DFX_F32;
    auto k = u->dtype == DFX_F32 ? dfx_embed_few_kernel<DFX_F32, DFX_F32> : u->dtype == DFX_BF16 ? (wide ? dfx_embed_few_kernel<DFX_BF16, DFX_F32> : dfx_embed_few_kernel<DFX_BF16, DFX_BF16>)
                                                                        : (wide ? dfx_embed_few_kernel<DFX_F16, DFX_F32> : dfx_embed_few_kernel<DFX_F16, DFX_F16>);
    return step_launch(k, grid, kEmbedThreads, s, a, u->tokens);
  }
  uint2* pairs[2] = {(uint2*)(ws + p.pairs[0]), (uint2*)(ws + p.pairs[1])};
  const bool few = u->rows && u->rows <= kOwnMost && u->vocab <= (size_t)kOwnQuotients * kOwners;
  if (few) {
    auto k = u->out_dtype == DFX_F32 ? dfx_embed_own_kernel<DFX_F32> : u->out_dtype == DFX_BF16 ? dfx_embed_own_kernel<DFX_BF16> : dfx_embed_own_kernel<DFX_F16>;
    const SortArgs x = {u->tokens, nullptr, pairs[0], nullptr, (uint32_t)u->rows, (uint32_t)u->vocab, 0, 0, 0};
    const int rc = step_launch(k, dim3(kOwners + (u->accumulate ? 0u : (uint32_t)std::min<size_t>(u->vocab, 4096))), kOwnThreads, s, x, u->table_grad, os, (uint32_t)u->dim);
    if (rc != DFX_OK) return rc;
    a.sorted = pairs[0];
  } else if (!u->accumulate) {
    const int rc = clear();
    if (rc != DFX_OK) return rc;
  }
  if (!u->rows) return DFX_OK;
  if (!few) {
    for (uint32_t k = 0; k < p.passes; ++k) {
      const SortArgs x = {k ? nullptr : u->tokens, k ? pairs[(k - 1) & 1] : nullptr, pairs[k & 1], (uint32_t*)(ws + p.counts), (uint32_t)u->rows, (uint32_t)u->vocab, p.chunk, k * p.bits, p.bits};
      int rc = step_launch(dfx_embed_count_kernel, dim3(p.chunks), kSortThreads, s, x);
      if (rc == DFX_OK) rc = step_launch(dfx_embed_move_kernel, dim3(p.chunks), kSortThreads, s, x);
      if (rc != DFX_OK) return rc;
    }
    a.sorted = pairs[(p.passes - 1) & 1];
  }
  if (u->dtype == DFX_F32) return embed_sums<DFX_F32, DFX_F32>(a, s);
  if (u->dtype == DFX_BF16) return u->out_dtype == DFX_F32 ? embed_sums<DFX_BF16, DFX_F32>(a, s) : embed_sums<DFX_BF16, DFX_BF16>(a, s);
  return u->out_dtype == DFX_F32 ? embed_sums<DFX_F16, DFX_F32>(a, s) : embed_sums<DFX_F16, DFX_F16>(a, s);
}

}  // extern "C"

// The clipped policy loss with a KL term over rows of logits, forward and backward, in front of a step's gradient all-reduce.
//
// A row's softmax is taken around its largest logit m: S = sum exp(c (z - m)), logp = c (z_t - m) - log S, and the gradient of z_j is
// g ([j = t] - exp(c (z_j - m)) / S) with one number g for the row.  So a row is read, reduced to (m, S), and written once g is known.
#include <float.h>
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>

#include "dfx_step.h"

namespace {

constexpr int kSums = 5;
constexpr uint32_t kGroups = 4096;       // workgroups of a call, at most: each leaves its share of the sums
constexpr int kSumWaves = 3;             // waves that share a sum
constexpr int kSumThreads = kSums * kSumWaves * kStepWave;
// Few rows of a long vocabulary are split over workgroups.
constexpr int kSplitThreads = 256;
constexpr uint32_t kSplitGroups = 512;   // workgroups, at most
constexpr uint32_t kSplitRows = 64;      // rows, at most
constexpr uint32_t kSplitGrad = 20000, kSplitForward = 65536;      // elements of a row, at least

struct LossPart { float m, s, zt, has; };       // of a segment of a row; zt: the target's logit, where the segment has it (has = 1, else both 0)

struct LossArgs {
  const void* logits;
  void* grad;
  size_t logits_stride, grad_stride;
  const int64_t* targets;
  const float *old_logp, *ref_logp, *advantage, *weight, *scale;      // absent: the targets' address, so that all are read alike (has_...)
  float *logp, *loss, *sums;
  double* part;                          // [kSums][workgroups]
  LossPart* parts;                       // [rows][segments], where rows are split
  uint32_t rows, vocab;
  double c;                              // 1 / temperature
  float least, most, kl_coef;            // 1 - clip_low, 1 + clip_high
  float k;                               // c / log 2: exponents are taken to base 2
  bool has_old, has_ref, has_advantage, has_weight, has_scale;
};

// exp(c (z - m)) = 2^(k (z - m)), k = c / log 2.  The difference first: it is 0 for the largest logit, exact where it matters, and cannot
// overflow for logits of the type's lowest or largest value.
// The product is rounded to 32 bits, k as well: an exponential is off by 4e-7 of its size at a distance of 10, 9e-7 at 20, and weighs as little in
// the sum.  It shows in single elements of 32-bit gradients that far from the largest.
struct MaxSum { float m, s; };           // s = sum 2^(k (z - m)); nothing seen yet: m = -infinity, s = 0

// m to take differences from: where only -infinity was seen, any finite one (2^(-infinity - 0) = 0, and NaN stays NaN)
__device__ __forceinline__ float loss_base(float m) { return m == -INFINITY ? 0.0f : m; }
__device__ __forceinline__ float loss_exp(float z, float base, float k) { return __builtin_amdgcn_exp2f((z - base) * k); }

// over each n (a power of two) lanes' entries, for all of them
__device__ __forceinline__ MaxSum join_lanes(MaxSum ms, float k, uint32_t n) {
  float top = ms.m;
  for (uint32_t d = n / 2; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, (int)d));
  ms.s *= loss_exp(ms.m, loss_base(top), k);
  for (uint32_t d = n / 2; d; d >>= 1) ms.s += __shfl_xor(ms.s, (int)d);
  return {top, ms.s};
}

// over a workgroup of T threads, for all of them; one barrier.  lds: T / 64 entries that nobody reads any more
template <int T>
__device__ __forceinline__ MaxSum join_all(MaxSum ms, float k, MaxSum* lds) {
  ms = join_lanes(ms, k, kStepWave);
  if ((threadIdx.x & (kStepWave - 1)) == 0) lds[threadIdx.x / kStepWave] = ms;
  __syncthreads();
  return join_lanes(lds[threadIdx.x % (T / kStepWave)], k, T / kStepWave);      // every wave joins them once more, an entry a lane
}

constexpr double kLog2 = 0.69314718055994530942, kLog2e = 1.44269504088896340736;

__device__ __forceinline__ float loss_exp_of(double x) { return __builtin_amdgcn_exp2f((float)(x * kLog2e)); }

// exp(d) - 1, which the gradient takes, and the penalty exp(d) - 1 - d, each rounded once.  Near 0, where they cancel, by the penalty's series, whose
// next term is d^10 / 10! (d = 1/2: 3e-10 of 0.15); elsewhere by the exponential, so that neither carries the other's rounding (exp(d) - 1 as d + penalty
// would be off by |d| units).  d = -infinity, a token that the reference bans: -1 and infinity; d = +infinity: infinity twice.
struct LossPenalty { float grows, kl; };
__device__ __forceinline__ LossPenalty loss_penalty(double d) {
  const float x = (float)d;
  if (fabsf(x) > 0.5f) {
    const double e = (double)loss_exp_of(d);
    return {(float)(e - 1.0), e == INFINITY ? INFINITY : (float)(e - 1.0 - d)};
  }
  float r = 1.0f / 362880.0f;
  r = fmaf(r, x, 1.0f / 40320.0f);
  r = fmaf(r, x, 1.0f / 5040.0f);
  r = fmaf(r, x, 1.0f / 720.0f);
  r = fmaf(r, x, 1.0f / 120.0f);
  r = fmaf(r, x, 1.0f / 24.0f);
  r = fmaf(r, x, 1.0f / 6.0f);
  r = fmaf(r, x, 0.5f);
  r = r * x * x;
  return {(float)(d + (double)r), r};
}

// What is known of a row before its logits.  Read at once when the row is begun, through the scalar cache (nobody writes it while the kernel
// runs), so that no wait for it comes behind the reduction.
struct RowIn { int64_t t; float w, A, old, ref, scale; };

#define LOSS_CONST __attribute__((address_space(4)))
__device__ __forceinline__ RowIn row_in(const LossArgs& a, uint32_t row) {
  const LOSS_CONST float *w = (const LOSS_CONST float*)a.weight, *A = (const LOSS_CONST float*)a.advantage, *old = (const LOSS_CONST float*)a.old_logp, *ref = (const LOSS_CONST float*)a.ref_logp, *scale = (const LOSS_CONST float*)a.scale;
  const RowIn in = {((const LOSS_CONST int64_t*)a.targets)[row], w[row], A[row], old[row], ref[row], scale[0]};
  return {in.t, a.has_weight ? in.w : 1.0f, in.A, in.old, in.ref, a.has_scale ? in.scale : 1.0f};
}

// whether it has anything to learn from, as far as that says
__device__ __forceinline__ bool row_counts(const LossArgs& a, const RowIn& in) { return in.t >= 0 && in.t < (int64_t)a.vocab && in.w != 0.0f; }

// What a row comes to.  far: z_t - m in 64 bits; s: the sum around that m.  log2 s = e + log2 f, f in [1/2, 1): what 32 bits lose there is
// 6e-8 of a logarithm, the sum's own error is more.  Differences of log-probabilities are taken in 64 bits (a logp of -10 holds 5e-7 in
// 32, which would be the ratio's error), what is made of them in 32.
struct RowValue { float logp, loss, pg, kl, clipped, w, g; };      // pg, kl, clipped times the weight w; nothing: all 0

__device__ __forceinline__ RowValue row_value(const LossArgs& a, const RowIn& in, double far, float s) {
  RowValue e = {0, 0, 0, 0, 0, 0, 0};
  if (s == 0.0f) return e;               // no logit above -infinity
  int two;
  const float f = frexpf(s, &two);
  const double logp = a.c * far - ((double)two + (double)__builtin_amdgcn_logf(f)) * kLog2;
  e.logp = (float)logp;
  if (!a.has_advantage) return e;
  e.w = in.w;
  const float A = in.A, r = a.has_old ? loss_exp_of(logp - (double)in.old) : 1.0f;
  const bool up = A >= 0.0f, clipped = up ? r > a.most : r < a.least;
  const float pg = -A * (clipped ? up ? a.most : a.least : r);
  float slope = clipped ? 0.0f : -A * r, value = pg;
  if (a.has_ref) {
    const LossPenalty x = loss_penalty((double)in.ref - logp);
    e.kl = e.w * x.kl;
    if (a.kl_coef != 0.0f) {             // (0 times an infinite penalty is not a number)
      slope -= a.kl_coef * x.grows;
      value = fmaf(a.kl_coef, x.kl, pg);
    }
  }
  e.pg = e.w * pg; e.clipped = clipped ? e.w : 0.0f;
  e.loss = e.w * value;
  e.g = (float)a.c * e.w * slope * in.scale;
  return e;
}

__device__ __forceinline__ void add_sums(double* sums, const RowValue& e) {
  sums[0] += (double)e.loss; sums[1] += (double)e.pg; sums[2] += (double)e.kl; sums[3] += (double)e.clipped; sums[4] += (double)e.w;
}

// ... by every thread alike; one of them writes it down.  Returns g
__device__ __forceinline__ float row_end(const LossArgs& a, uint32_t row, const RowIn& in, double far, float s, bool writes, double* sums) {
  const RowValue e = row_value(a, in, far, s);
  if (writes) {
    if (a.logp) a.logp[row] = e.logp;
    if (a.loss) a.loss[row] = e.loss;
    if (sums) add_sums(sums, e);
  }
  return e.g;
}

// How a row of logits lies in memory: head elements up to a multiple of 128 bytes (PEEL), nvec vectors of N, and at most N - 1 elements behind
// them.  A wave's vectors then fill whole lines, of the gradient too, whose rows begin where the logits' do.  Rows of an odd length, with gradient:
// 4096 x 50257 bf16 182 us, from a multiple of 16 bytes on 155, of 128 148; fp32 338 and 310; x 32001 bf16 130 and 111.  Short rows, of workgroups
// below 512, are quicker without a head (x 8001 27.5 and 30.9).
template <int DT, bool PEEL>
struct RowPlace {
  static constexpr uint32_t N = 16 / sizeof(typename StepElem<DT>::raw);
  uint32_t head, nvec, vocab;
  __device__ __forceinline__ RowPlace(const void* row, uint32_t vocab_) : vocab(vocab_) {
    head = !PEEL ? 0u : min((uint32_t)(-(uintptr_t)row & 127u) / (uint32_t)sizeof(typename StepElem<DT>::raw), vocab);
    nvec = (vocab - head) / N;
  }
  // the i-th of the elements outside the vectors; from vocab on: there is none
  __device__ __forceinline__ uint32_t end_element(uint32_t i) const { return i < head ? i : nvec * N + i; }
  __device__ __forceinline__ bool in_vectors(uint32_t t) const { return t - head < nvec * N; }
  __device__ __forceinline__ uint32_t vector_of(uint32_t t) const { return (t - head) / N; }
};

// what of a row is in vectors, joined into ms
template <int DT, int N, int U>
__device__ __forceinline__ void take_vectors(StepVec<DT, N>* r, float k, MaxSum& ms) {
  float z = -INFINITY;
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int j = 0; j < N; ++j) z = fmaxf(z, r[u].get(j));
  const float m = fmaxf(ms.m, z), base = loss_base(m);
  float s = ms.s * loss_exp(ms.m, base, k);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    r[u].again();
#pragma unroll
    for (int j = 0; j < N; ++j) s += loss_exp(r[u].get(j), base, k);
  }
  ms = {m, s};
}

template <int DT, int N>
__device__ __forceinline__ void grad_vector(const StepVec<DT, N>& r, float k, float base, float gs, void* out, uint32_t bytes) {
  float x[N];
#pragma unroll
  for (int j = 0; j < N; ++j) x[j] = gs * loss_exp(r.get(j), base, k);
  StepVec<DT, N> o;
  o.put(x);
  o.stream_at(out, bytes);
}

// what every lane holds alike, in a scalar register
__device__ __forceinline__ float uniform(float v) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v))); }

// this thread's number; what is made of it is made where it is used, not kept from row to row
__device__ __forceinline__ uint32_t thread_here() {
  uint32_t me = threadIdx.x;
  asm("" : "+v"(me));
  return me;
}

// 16 bytes a lane from an address that is a multiple of 16, straight to LDS: lane i's to the i-th place behind `to`, which all lanes share
__device__ __forceinline__ void load_to_lds(const void* p, uint32_t bytes, uint4* to) {
  __builtin_amdgcn_global_load_lds((const STEP_GLOBAL uint32_t*)((const STEP_GLOBAL unsigned char*)p + bytes), (__attribute__((address_space(3))) uint32_t*)to, 16, 0, 0);
}

template <int DT, int T>
__device__ __forceinline__ void zero_row(typename StepElem<DT>::raw* out, uint32_t vocab) {
  const RowPlace<DT, false> at(out, vocab);
  const uint32_t me = thread_here(), end = at.end_element(me);
  StepVec<DT, (int)RowPlace<DT, false>::N> zero;
  zero.w = 0;
  for (uint32_t v = me; v < at.nvec; v += T) zero.stream_at(out + at.head, v * 16u);
  if (end < vocab) step_put<DT>(out, end, 0.0f);
}

// A workgroup of T threads per row.  From the reduction to the gradient a thread keeps the row's vectors v = thread + u T, u < U, in registers
// and the next L of them in LDS, where loads put them without a register in between; what a longer row has beyond these is read again, from
// its end, and comes from the memory-side cache.
//
// HBM bounds it, with reads and writes of 512 rows at once (5.2 TB/s; the exponentials keep the vector units busy for 57 % of 16-bit rows' time, and
// fewer instructions do not make it shorter).  So that one row's reads pass while another's exponentials do, a kernel has at most 64 registers and
// half of the LDS, and two workgroups of 1024 fit a compute unit: 4096 x 131072 bf16, every sixth row masked, 370 us; with one workgroup of up
// to 128 registers 417 to 435, with workgroups of 512 that read more of the row again 450, without LDS 384.  1024 x 50257 fp32 74.5 us (5.2 TB/s);
// loads of what stays in registers go past the caches, which keep the rest of the row instead (without: 84).  Behind the matrix product that leaves
// its logits in the memory-side cache that costs nothing (1024 x 50257 bf16 29 and 28 us, forward 16 and 14; 2048 x 50257 65 and 98, 30 and 63).
// Forward 2048 x 32000 bf16 21.2 us (5.3 TB/s), with workgroups of 1024 29, of 256 42.
template <int DT, int T, int U, int L, bool GRAD>
__global__ void __launch_bounds__(T, 8) dfx_loss_rows_kernel(LossArgs a) {
  typedef typename StepElem<DT>::raw raw;
  constexpr int N = 16 / (int)sizeof(raw);
  constexpr bool LINES = T >= 512;       // vectors fill whole lines, and what stays in registers is read past the caches
  __shared__ struct {
    uint4 kept[L * T + 1];               // (at 0, as where loads straight to LDS go is said in 16 bits)
    MaxSum lds[2][T / kStepWave];
    double sums[kSums];                  // (thread 0's)
  } sh;
  const float k = a.k;
  if (threadIdx.x == 0)
    for (int i = 0; i < kSums; ++i) sh.sums[i] = 0.0;
  uint32_t turn = 0;
  for (uint32_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const raw* z = (const raw*)a.logits + (size_t)row * a.logits_stride;
    raw* out = GRAD ? (raw*)a.grad + (size_t)row * a.grad_stride : nullptr;
    const RowIn in = row_in(a, row);
    if (!row_counts(a, in)) {            // (the whole workgroup)
      if (threadIdx.x == 0) {
        if (a.logp) a.logp[row] = 0.0f;
        if (a.loss) a.loss[row] = 0.0f;
      }
      if (GRAD) zero_row<DT, T>(out, a.vocab);
      continue;
    }
    const uint32_t t = (uint32_t)in.t;
    const RowPlace<DT, LINES> at(z, a.vocab);
    const uint32_t nvec = at.nvec;
    const raw* zv = z + at.head;
    uint32_t me = thread_here();
    const uint32_t end = at.end_element(me);
    StepVec<DT, N> r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t v = u * T + me;
      if (v < nvec) r[u].template load_at<LINES>(zv, v * 16u);
      else r[u].fill_lowest();
    }
#pragma unroll
    for (int l = 0; l < L; ++l)
      if ((U + l) * T + me < nvec) load_to_lds(zv, ((U + l) * T + me) * 16u, &sh.kept[l * T + (threadIdx.x & ~(kStepWave - 1u))]);
    const float zt = step_get<DT>(z, t);
    MaxSum ms = {-INFINITY, 0.0f};
    float last = -INFINITY;
    if (end < a.vocab) {
      last = step_get<DT>(z, end);
      ms = {last, loss_exp(last, loss_base(last), k)};
    }
    take_vectors<DT, N, U>(r, k, ms);
    if (L) loads_arrived();
#pragma unroll 1
    for (int l = 0; l < L; ++l)
      if ((U + l) * T + me < nvec) {
        StepVec<DT, N> more;
        more.from(sh.kept[l * T + me]);
        take_vectors<DT, N, 1>(&more, k, ms);
      }
    for (uint32_t v = (U + L) * T + me; v < nvec; v += T) {
      StepVec<DT, N> more;
      more.load_at(zv, v * 16u);
      take_vectors<DT, N, 1>(&more, k, ms);
    }
    ms = join_all<T>(ms, k, sh.lds[turn]);
    turn ^= 1u;                          // (of the rows that come here: whoever writes a half again is behind the other one's barrier)
    ms = {uniform(loss_base(ms.m)), uniform(ms.s)};
    const float g = uniform(row_end(a, row, in, (double)zt - (double)ms.m, ms.s, threadIdx.x == 0, sh.sums));
    if (!GRAD) continue;
    if (ms.s == 0.0f) {                  // no logit above -infinity
      zero_row<DT, T>(out, a.vocab);
      continue;
    }
    const float base = ms.m, gs = -g / ms.s;
    asm("" : "+v"(me));
    raw* ov = out + at.head;
    if ((U + L) * T + me < nvec)
      for (uint32_t n = (nvec - 1u - (U + L) * T - me) / T + 1u; n-- != 0;) {
        const uint32_t bytes = ((U + L) * T + me + n * T) * 16u;
        StepVec<DT, N> more;
        more.load_at(zv, bytes);
        grad_vector<DT, N>(more, k, base, gs, ov, bytes);
      }
#pragma unroll 1
    for (int l = 0; l < L; ++l)
      if ((U + l) * T + me < nvec) {
        StepVec<DT, N> more;
        more.from(sh.kept[l * T + me]);
        grad_vector<DT, N>(more, k, base, gs, ov, ((U + l) * T + me) * 16u);
      }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t v = u * T + me;
      r[u].again();
      if (v < nvec) grad_vector<DT, N>(r[u], k, base, gs, ov, v * 16u);
    }
    if (end < a.vocab) step_put<DT>(out, end, gs * loss_exp(last, base, k));
    // the target's element once more, by the thread that has just written it
    if (at.in_vectors(t) ? at.vector_of(t) % T == threadIdx.x : t == end) step_put<DT>(out, t, gs * loss_exp(zt, base, k) + g);
  }
  if (a.sums && threadIdx.x == 0)
    for (int i = 0; i < kSums; ++i) a.part[(size_t)i * gridDim.x + blockIdx.x] = sh.sums[i];
}

// ------------------------------------------------------------------------------------------
// few rows: each split over workgroups, in two kernels: the segments' parts, then all of them joined by everyone who needs them.  No row's
// logits are read behind a write of another workgroup, so the gradient may take their place.
// ------------------------------------------------------------------------------------------
// Segments of a row (at most 64), vectors of a segment (a multiple of kSplitThreads), and the power of two that holds the segments.  What lies outside
// a row's vectors goes with the last segment.
struct Split { uint32_t segments, vectors, lanes, lanes_log2; };

template <int DT>
__device__ __forceinline__ bool segment_has(const Split& sp, const RowPlace<DT, true>& at, uint32_t seg, uint32_t t) {
  return at.in_vectors(t) ? at.vector_of(t) - seg * sp.vectors < sp.vectors : seg + 1u == sp.segments;
}

template <int DT>
__global__ void __launch_bounds__(kSplitThreads) dfx_loss_parts_kernel(LossArgs a, Split sp) {
  constexpr int T = kSplitThreads, N = 16 / (int)sizeof(typename StepElem<DT>::raw), U = 2;
  __shared__ MaxSum lds[T / kStepWave];
  const uint32_t row = blockIdx.y, seg = blockIdx.x;
  const RowIn in = row_in(a, row);
  if (!row_counts(a, in)) return;
  const auto* z = (const typename StepElem<DT>::raw*)a.logits + (size_t)row * a.logits_stride;
  const RowPlace<DT, true> at(z, a.vocab);
  const uint32_t end = min(at.nvec, (seg + 1u) * sp.vectors), t = (uint32_t)in.t;
  const float k = a.k;
  MaxSum ms = {-INFINITY, 0.0f};
  for (uint32_t v = seg * sp.vectors + threadIdx.x; v < end; v += U * T) {
    StepVec<DT, N> r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (v + u * T < end) r[u].load_at(z + at.head, (v + u * T) * 16u);
      else r[u].fill_lowest();
    }
    take_vectors<DT, N, U>(r, k, ms);
  }
  const uint32_t lone = at.end_element(threadIdx.x);
  if (seg + 1u == sp.segments && lone < a.vocab) {
    const float x = step_get<DT>(z, lone), m = fmaxf(ms.m, x), base = loss_base(m);
    ms = {m, ms.s * loss_exp(ms.m, base, k) + loss_exp(x, base, k)};
  }
  ms = join_all<T>(ms, k, lds);
  if (threadIdx.x == 0) {
    const bool has = segment_has(sp, at, seg, t);
    a.parts[row * sp.segments + seg] = {ms.m, ms.s, has ? step_get<DT>(z, t) : 0.0f, has ? 1.0f : 0.0f};
  }
}

// The sums over split rows, by one workgroup beside the rows' own: as many lanes to a row as it has segments, so that a few steps do for any
// number of rows (their product is bounded).
template <int DT>
__device__ __forceinline__ void split_sums(const LossArgs& a, const Split& sp) {
  constexpr int T = kSplitThreads;
  __shared__ double lds[T / kStepWave][kSums];
  const uint32_t me = threadIdx.x, i = me & (sp.lanes - 1u), step = T >> sp.lanes_log2;
  double s[kSums] = {0, 0, 0, 0, 0};
  for (uint32_t first = 0; first < a.rows; first += step) {
    const uint32_t row = first + (me >> sp.lanes_log2);
    LossPart part = {-INFINITY, 0.0f, 0.0f, 0.0f};
    RowIn in = {-1, 0, 0, 0, 0, 0};
    if (row < a.rows) in = row_in(a, row);
    const bool counts = row_counts(a, in);
    if (counts && i < sp.segments) part = a.parts[row * sp.segments + i];
    const MaxSum ms = join_lanes({part.m, part.s}, a.k, sp.lanes);
    float zt = part.zt;                  // (0 but where the target is)
    for (uint32_t d = sp.lanes / 2u; d; d >>= 1) zt += __shfl_xor(zt, (int)d);
    if (counts && i == 0) add_sums(s, row_value(a, in, (double)zt - (double)loss_base(ms.m), ms.s));
  }
  for (int q = 0; q < kSums; ++q) {
    s[q] = wave_sum(s[q]);
    if ((me & (kStepWave - 1)) == 0) lds[me / kStepWave][q] = s[q];
  }
  __syncthreads();
  if (me < kSums) {
    double all = lds[0][me];
    for (int w = 1; w < T / kStepWave; ++w) all += lds[w][me];
    a.sums[me] = (float)all;
  }
}

// Every workgroup joins its row's parts again.
template <int DT, bool GRAD>
__global__ void __launch_bounds__(kSplitThreads) dfx_loss_split_kernel(LossArgs a, Split sp) {
  constexpr int T = kSplitThreads, N = 16 / (int)sizeof(typename StepElem<DT>::raw), U = 2;
  const float k = a.k;
  const uint32_t row = blockIdx.y, seg = blockIdx.x, lane = threadIdx.x % kStepWave;      // (without gradient there is one of a row)
  if (row == a.rows) {
    if (seg == 0) split_sums<DT>(a, sp);
    return;
  }
  typedef typename StepElem<DT>::raw raw;
  const raw* z = (const raw*)a.logits + (size_t)row * a.logits_stride;
  raw* out = GRAD ? (raw*)a.grad + (size_t)row * a.grad_stride : nullptr;
  const RowPlace<DT, true> at(z, a.vocab);
  const raw* zv = z + at.head;
  raw* ov = out + at.head;
  const uint32_t first = seg * sp.vectors + threadIdx.x, end = min(at.nvec, (seg + 1u) * sp.vectors);
  const uint32_t lone = seg + 1u == sp.segments ? at.end_element(threadIdx.x) : a.vocab;
  const RowIn in = row_in(a, row);
  const bool writes = seg == 0 && threadIdx.x == 0, counts = row_counts(a, in);
  float s = 0.0f, g = 0.0f, base = 0.0f, zt = 0.0f;
  StepVec<DT, N> r[U];
  if (GRAD && counts)                    // (under way while the parts are joined)
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (first + u * T < end) r[u].load_at(zv, (first + u * T) * 16u);
  const uint32_t t = (uint32_t)in.t;
  if (counts) {
    LossPart part = {-INFINITY, 0.0f, 0.0f, 0.0f};
    if (lane < sp.segments) part = a.parts[row * sp.segments + lane];
    zt = __shfl(part.zt, __ffsll(__ballot(part.has != 0.0f)) - 1);      // (a target that counts lies in one of them)
    MaxSum ms = {part.m, part.s};
    ms = join_lanes(ms, k, kStepWave);
    base = loss_base(ms.m); s = ms.s;
    g = row_end(a, row, in, (double)zt - (double)base, s, writes, nullptr);
  } else if (writes) {
    if (a.logp) a.logp[row] = 0.0f;
    if (a.loss) a.loss[row] = 0.0f;
  }
  if (!GRAD) return;
  const float gs = s == 0.0f ? 0.0f : -g / s;
  if (s == 0.0f) {                       // nothing to learn from (the whole workgroup)
    StepVec<DT, N> zero;
    zero.w = 0;
    for (uint32_t v = first; v < end; v += T) zero.stream_at(ov, v * 16u);
    if (lone < a.vocab) step_put<DT>(out, lone, 0.0f);
    return;
  }
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (first + u * T < end) grad_vector<DT, N>(r[u], k, base, gs, ov, (first + u * T) * 16u);
  for (uint32_t v = first + U * T; v < end; v += T) {
    r[0].load_at(zv, v * 16u);
    grad_vector<DT, N>(r[0], k, base, gs, ov, v * 16u);
  }
  if (lone < a.vocab) step_put<DT>(out, lone, gs * loss_exp(step_get<DT>(z, lone), base, k));
  if (at.in_vectors(t) ? segment_has(sp, at, seg, t) && at.vector_of(t) % T == threadIdx.x : t == lone) step_put<DT>(out, t, gs * loss_exp(zt, base, k) + g);
}

// the workgroups' shares, in an order that is always the same: a wave to a sum, three waves to each
__global__ void __launch_bounds__(kSumThreads) dfx_loss_sums_kernel(const double* part, uint32_t n, float* out) {
  __shared__ double lds[kSumThreads / kStepWave];
  const uint32_t wave = threadIdx.x / kStepWave, lane = threadIdx.x % kStepWave;
  const double* mine = part + (size_t)(wave % kSums) * n;
  constexpr uint32_t U = 8, stride = kSumWaves * kStepWave;
  double s = 0.0;
  for (uint32_t i = wave / kSums * kStepWave + lane; i < n; i += U * stride) {      // (eight loads under way at once)
    double x[U];
#pragma unroll
    for (uint32_t u = 0; u < U; ++u) x[u] = i + u * stride < n ? mine[i + u * stride] : 0.0;
#pragma unroll
    for (uint32_t u = 0; u < U; ++u) s += x[u];
  }
  s = wave_sum(s);
  if (lane == 0) lds[wave] = s;
  __syncthreads();
  if (threadIdx.x < kSums) {
    double t = lds[threadIdx.x];
    for (int w = 1; w < kSumWaves; ++w) t += lds[threadIdx.x + w * kSums];
    out[threadIdx.x] = (float)t;
  }
}

uint32_t loss_groups(uint64_t rows) { return (uint32_t)std::min<uint64_t>(rows, kGroups); }
uint32_t loss_parts(uint64_t rows) { return (uint32_t)std::min<uint64_t>(rows * kStepWave, kSplitGroups); }      // at most

// How a call is split, or segments = 0.  A row alone on its workgroup takes as long as that needs for its elements.  One row of bf16, us, alone and
// split: with gradient and sums (two kernels either way) 20000 elements 7.8 and 6.7, 50257 10.3 and 7.2, 131072 19.2 and 7.2; forward (a launch
// more, which costs the host 3) 32000 4.4 and 4.9, 70000 6.7 and 4.9, 131072 10.5 and 5.1.  64 rows with gradient 9.1 and 8.7, 12.1 and 9.7, 21.8 and
// 12.5.  A split row is read twice, so that it gains less the more rows there are: 128 rows 9.6 and 9.7, 12.6 and 11.9, 23.4 and 20.7, 200 of 131072 27.5 and
// 33.6.  Between 64, where every length gains, and 200 the place where the ways meet depends on the length and was not looked for.
Split loss_split(const LossArgs& a, uint32_t elem_bytes) {
  Split sp = {0, 0, 1, 0};
  if (a.rows == 0 || a.rows > kSplitRows || a.vocab < (a.grad ? kSplitGrad : kSplitForward)) return sp;
  const uint32_t nvec = a.vocab / (16u / elem_bytes), want = std::min<uint32_t>(kStepWave, kSplitGroups / a.rows);
  sp.vectors = ((nvec + want - 1) / want + kSplitThreads - 1) / kSplitThreads * kSplitThreads;
  sp.segments = (nvec + sp.vectors - 1) / sp.vectors;
  for (; sp.lanes < sp.segments; sp.lanes *= 2) ++sp.lanes_log2;
  return sp;
}

template <int DT>
int launch_split(const LossArgs& a, const Split& sp, hipStream_t s) {
  const uint32_t more = a.sums ? 1u : 0u;
  const int rc = step_launch(dfx_loss_parts_kernel<DT>, dim3(sp.segments, a.rows), kSplitThreads, s, a, sp);
  if (rc != DFX_OK) return rc;
  if (a.grad) return step_launch(dfx_loss_split_kernel<DT, true>, dim3(sp.segments, a.rows + more), kSplitThreads, s, a, sp);
  return step_launch(dfx_loss_split_kernel<DT, false>, dim3(1, a.rows + more), kSplitThreads, s, a, sp);
}

template <int DT>
int launch_rows(const LossArgs& a, uint32_t groups, hipStream_t s) {
  const uint32_t nvec = a.vocab / (16 / step_elem_bytes(DT));
#define ROWS(T, U, L, F) return step_launch(a.grad ? dfx_loss_rows_kernel<DT, T, U, L, true> : dfx_loss_rows_kernel<DT, T, F, 0, false>, dim3(groups), T, s, a)
  if (nvec <= 256) ROWS(128, 2, 0, 2);
  if (nvec <= 512) ROWS(128, 4, 0, 4);
  if (nvec <= 1024) ROWS(256, 4, 0, 4);
  if (nvec <= 2048) ROWS(512, 4, 0, 4);
  if (nvec <= 4096) ROWS(512, 8, 0, 8);  // (with gradient 32 to 40 bytes a thread are spilled; 4096 x 32000 bf16 103 us)
  if (nvec <= 10240) ROWS(1024, 6, 4, 6);
  ROWS(1024, 8, 4, 6);                   // (where more is read again, a few spilled registers are the lesser evil: 4096 x 131072 bf16 380 and 375 us; x 65536 195 and 199)
#undef ROWS
}

// rows of n elements, stride elements apart, from p on: [first, second) in bytes
struct Extent { uintptr_t lo, hi; };
Extent extent(const void* p, size_t rows, size_t vocab, size_t stride, size_t eb) {
  return {(uintptr_t)p, (uintptr_t)p + ((rows - 1) * stride + vocab) * eb};
}

// n pieces of so many bytes, step bytes from one to the next; nothing: n = 0
struct Span { uintptr_t at; size_t n, bytes, step; };
Span flat(const void* p, size_t bytes) { return {(uintptr_t)p, p && bytes ? (size_t)1 : 0, bytes, bytes}; }

// whether a span of one piece shares a byte with another: with the last piece that begins at or before it, or the one behind that
bool meet(const Span& one, const Span& s) {
  if (!one.n || !s.n) return false;
  const uintptr_t lo = one.at, hi = lo + one.bytes;
  const size_t k = lo <= s.at ? 0 : std::min<size_t>((lo - s.at) / s.step, s.n - 1);
  const uintptr_t p = s.at + k * s.step;
  return (lo < p + s.bytes && p < hi) || (k + 1 < s.n && p + s.step < hi);
}

}  // namespace

extern "C" {

size_t dfx_policy_loss_workspace(size_t rows, size_t vocab, dfx_dtype dtype) {
  (void)vocab; (void)dtype;
  return loss_parts(rows) * sizeof(LossPart) + std::max(1u, loss_groups(rows)) * kSums * sizeof(double);
}

int dfx_policy_loss(const dfx_policy_loss_args* u, void* hip_stream) {
  if (!u || u->struct_bytes != sizeof(*u)) return DFX_ERR_INVALID_ARG;
  if (u->dtype != DFX_F32 && u->dtype != DFX_BF16 && u->dtype != DFX_F16) return DFX_ERR_INVALID_ARG;
  if (u->rows > 0x7fffffffull || u->vocab >= (1ull << 30)) return DFX_ERR_TOO_LARGE;
  if (!(u->inv_temperature * kLog2e >= (double)FLT_MIN && u->inv_temperature * kLog2e <= (double)FLT_MAX)) return DFX_ERR_INVALID_ARG;
  const size_t eb = step_elem_bytes(u->dtype), ls = u->logits_stride ? u->logits_stride : u->vocab, gs = u->grad_stride ? u->grad_stride : u->vocab;
  if (ls < u->vocab || (u->grad && gs < u->vocab)) return DFX_ERR_INVALID_ARG;
  if (u->rows && ((ls > SIZE_MAX / 8 / u->rows) || (u->grad && gs > SIZE_MAX / 8 / u->rows))) return DFX_ERR_TOO_LARGE;
  if (!isfinite(u->clip_low) || u->clip_low < 0.0 || u->clip_low > 1.0 || !isfinite(u->clip_high) || u->clip_high < 0.0 || !step_fits(u->kl_coef)) return DFX_ERR_INVALID_ARG;
  if (u->kl_coef != 0.0 && !u->ref_logp) return DFX_ERR_INVALID_ARG;
  if (!u->advantage && (u->loss || u->sums || u->grad)) return DFX_ERR_INVALID_ARG;
  if (u->rows && (!u->targets || (u->vocab && !u->logits))) return DFX_ERR_INVALID_ARG;
  for (const void* p : {(const void*)u->old_logp, (const void*)u->ref_logp, (const void*)u->advantage, (const void*)u->weight, (const void*)u->scale, (const void*)u->logp, (const void*)u->loss, (const void*)u->sums})
    if ((uintptr_t)p & 3u) return DFX_ERR_INVALID_ARG;
  if (((uintptr_t)u->targets & 7u) || ((uintptr_t)u->logits % eb) || ((uintptr_t)u->grad % eb)) return DFX_ERR_INVALID_ARG;
  if (u->sums && (!u->workspace || ((uintptr_t)u->workspace & 7u) || u->workspace_bytes < dfx_policy_loss_workspace(u->rows, u->vocab, u->dtype))) return DFX_ERR_INVALID_ARG;
  if (u->grad && u->rows && u->vocab && !(u->grad == u->logits && gs == ls)) {
    const Extent a = extent(u->logits, u->rows, u->vocab, ls, eb), b = extent(u->grad, u->rows, u->vocab, gs, eb);
    if (a.lo < b.hi && b.lo < a.hi) return DFX_ERR_INVALID_ARG;
  }
  // What is written lies apart from what is read (but for the gradient in the logits' place) and from what else is written: rows are read by some
  // workgroups while others write theirs, and the sums of split rows while the rows are written.
  const size_t rows = u->rows, work = dfx_policy_loss_workspace(u->rows, u->vocab, u->dtype);
  const bool has_work = u->workspace && !((uintptr_t)u->workspace & 7u) && u->workspace_bytes >= work;
  const Span z = {(uintptr_t)u->logits, u->vocab ? rows : 0, u->vocab * eb, ls * eb}, g = {(uintptr_t)u->grad, u->grad && u->vocab ? rows : 0, u->vocab * eb, gs * eb};
  const Span reads[] = {flat(u->targets, 8 * rows), flat(u->old_logp, 4 * rows), flat(u->ref_logp, 4 * rows), flat(u->advantage, 4 * rows), flat(u->weight, 4 * rows), flat(u->scale, rows ? 4 : 0)};
  const Span writes[] = {flat(u->logp, 4 * rows), flat(u->loss, 4 * rows), flat(u->sums, 4 * kSums), flat(u->workspace, has_work ? work : 0)};
  for (size_t k = 0; k < sizeof(writes) / sizeof(writes[0]); ++k) {
    if (meet(writes[k], z) || meet(writes[k], g)) return DFX_ERR_INVALID_ARG;
    for (const Span& r : reads)
      if (meet(writes[k], r)) return DFX_ERR_INVALID_ARG;
    for (size_t j = 0; j < k; ++j)
      if (meet(writes[k], writes[j])) return DFX_ERR_INVALID_ARG;
  }
  for (const Span& r : reads)
    if (meet(r, g)) return DFX_ERR_INVALID_ARG;
  LossArgs a;
  memset(&a, 0, sizeof(a));
  a.logits = u->logits; a.grad = u->grad; a.logits_stride = ls; a.grad_stride = gs;
  a.targets = u->targets;
  const float* any = (const float*)u->targets;       // (8 bytes a row)
  a.old_logp = u->old_logp ? u->old_logp : any; a.ref_logp = u->ref_logp ? u->ref_logp : any; a.advantage = u->advantage ? u->advantage : any;
  a.weight = u->weight ? u->weight : any; a.scale = u->scale ? u->scale : any;
  a.has_old = u->old_logp; a.has_ref = u->ref_logp; a.has_advantage = u->advantage; a.has_weight = u->weight; a.has_scale = u->scale;
  a.logp = u->logp; a.loss = u->loss; a.sums = u->sums; a.parts = (LossPart*)u->workspace; a.part = (double*)(a.parts + loss_parts(u->rows));
  a.rows = (uint32_t)u->rows; a.vocab = (uint32_t)u->vocab;
  a.least = (float)(1.0 - u->clip_low); a.most = (float)std::min(1.0 + u->clip_high, (double)FLT_MAX); a.kl_coef = (float)u->kl_coef; a.c = u->inv_temperature;
  a.k = (float)(u->inv_temperature * kLog2e);
  hipStream_t s = (hipStream_t)hip_stream;
  const uint32_t groups = loss_groups(u->rows);
  const Split sp = has_work ? loss_split(a, (uint32_t)eb) : Split{0, 0, 1, 0};
  const bool f32 = u->dtype == DFX_F32, bf16 = u->dtype == DFX_BF16;
  if (sp.segments) return f32 ? launch_split<DFX_F32>(a, sp, s) : bf16 ? launch_split<DFX_BF16>(a, sp, s) : launch_split<DFX_F16>(a, sp, s);
  if (groups) {
    const int rc = f32 ? launch_rows<DFX_F32>(a, groups, s) : bf16 ? launch_rows<DFX_BF16>(a, groups, s) : launch_rows<DFX_F16>(a, groups, s);
    if (rc != DFX_OK) return rc;
  }
  return u->sums ? step_launch(dfx_loss_sums_kernel, dim3(1), kSumThreads, s, (const double*)a.part, groups, u->sums) : DFX_OK;
}

}  // extern "C"

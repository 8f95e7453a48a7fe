// Operators over lists of tensors, behind the gradient all-reduce of a step: the norm of all gradients, clipping, AdamW.
//
// A list is cut into chunks once, when it is made: a chunk lies in one tensor, has at most kChunk elements and is one entry {address,
// elements, type} of a table in device memory.  Lists of equal counts have equal tables but for the addresses and types, so a kernel
// over several lists takes entry c of each.  A call is one kernel (the norm and clipping: two), allocates nothing and copies nothing.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <vector>

#include "dfx_step.h"

namespace {

constexpr uint32_t kChunk = 8192;        // elements
constexpr int kNormThreads = 512;
constexpr int kNormGroups = 512;         // workgroups of a norm, at most: each leaves one partial result
constexpr uint32_t kNormTurn = 32;       // workgroups that draw their tickets from one counter
constexpr int kClipThreads = 1024;
constexpr int kAdamThreads = 1024;
constexpr int kAdamParts = 2;            // workgroups that share a chunk
constexpr uint32_t kAdamStaged = 640;    // chunks from which on a thread's loads wait for one another
constexpr uint32_t kMaxGroups = 1u << 20;      // (a grid's threads are counted in 32 bits) of a launch over a list

struct ListChunk { uint64_t ptr; uint32_t n; int32_t dtype; };
static_assert(sizeof(ListChunk) == 16, "a chunk is one 16-byte load");

struct ListSpan { uintptr_t lo, hi; size_t k; };      // a tensor's memory, and its place in the list

struct ListScratch {
  double part[kNormGroups];
  // count workgroups through, 0 again when the last one is: a counter (128 bytes apart) for every kNormTurn of them, and one for these
  uint32_t tickets[kNormGroups / kNormTurn + 1][32];
};

}  // namespace

struct dfx_list {
  int device = 0;
  uint32_t nchunks = 0;
  bool all_f32 = true;
  std::vector<dfx_tensor> tensors;
  std::vector<size_t> counts;            // the tensors', for comparisons between lists
  std::vector<ListSpan> spans;           // of the tensors that have elements, in the order of their addresses
  bool apart = true;                     // none of them shares memory with another
  ListChunk* chunks = nullptr;           // device
  ListScratch* scratch = nullptr;        // device
};

namespace {

// ------------------------------------------------------------------------------------------
// norm: sum of squares (or the largest magnitude) over all elements
//
// Squares and their sum are held in 64 bits: no gradient of 32 or 16 bits is too large or too small to be squared there, so no second,
// scaled pass is needed, and the products cost nothing beside the reads (with sums in 32 bits the times are the same).
//
// HBM bounds it.  Two workgroups a compute unit, all loads of a chunk under way at once (8 MiB of 16 bits, 16 of 32): sixteen 25 MiB bf16 buckets 69 us (6.1 TB/s),
// 1 GiB of fp32 170 us (6.3 TB/s).  Half as many threads 113 and 195 us; 2048 workgroups of 256, all the waves that fit, 85 and 191 us:
// what is in flight beyond about 16 MiB only gets in its own way.  A short list is its chain of waits (table, data, ticket): 4.0 us.
// ------------------------------------------------------------------------------------------
template <int DT, bool MAXIMUM>
__device__ __forceinline__ void norm_chunk(const ListChunk& c, double& sum, uint32_t& top) {
  constexpr int N = 16 / (int)sizeof(typename StepElem<DT>::raw), U = (int)kChunk / (N * kNormThreads);
  const void* p = (const void*)c.ptr;
  auto take = [&](float x) {
    if (MAXIMUM) top = max(top, __float_as_uint(x) & 0x7fffffffu);       // as integers: magnitudes in order, NaN above infinity
    else sum = fma((double)x, (double)x, sum);
  };
  if (c.n == kChunk) {                   // every load of the chunk is under way before the first is waited for
    StepVec<DT, N> r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) r[u].load(p, (size_t)(u * kNormThreads + threadIdx.x) * N);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int k = 0; k < N; ++k) take(r[u].get(k));
    return;
  }
  const uint32_t nvec = c.n / N;
  for (uint32_t v = threadIdx.x; v < nvec; v += kNormThreads) {
    StepVec<DT, N> r;
    r.load(p, (size_t)v * N);
#pragma unroll
    for (int k = 0; k < N; ++k) take(r.get(k));
  }
  const uint32_t i = nvec * N + threadIdx.x;
  if (i < c.n) take(step_get<DT>(p, i));
}

// Whether this is the last of n tickets.  The counter starts over behind it, in the same atomic: a multiple of n draws leaves 0, also where two calls on one
// list overlapped after all and drew from it together (with a reset of its own a draw in between was lost, and every later norm of the list wrong).
__device__ __forceinline__ bool draw(uint32_t* counter, uint32_t n) { return atomicInc(counter, n - 1u) == n - 1u; }

template <bool MAXIMUM>
__global__ void __launch_bounds__(kNormThreads) dfx_norm_kernel(const ListChunk* __restrict__ chunks, uint32_t nchunks, ListScratch* scratch, double scale, float* norm) {
  __shared__ double lds[kNormThreads / kStepWave];
  __shared__ uint32_t last;
  double sum = 0.0;
  uint32_t top = 0;
  for (uint32_t c = blockIdx.x; c < nchunks; c += gridDim.x) {
    const ListChunk e = chunks[c];
    if (e.dtype == DFX_F32) norm_chunk<DFX_F32, MAXIMUM>(e, sum, top);
    else if (e.dtype == DFX_BF16) norm_chunk<DFX_BF16, MAXIMUM>(e, sum, top);
    else norm_chunk<DFX_F16, MAXIMUM>(e, sum, top);
  }
  auto joined = [&]() -> double {       // over the workgroup; valid in thread 0
    const double w = MAXIMUM ? (double)wave_max(top) : wave_sum(sum);
    if ((threadIdx.x & (kStepWave - 1)) == 0) lds[threadIdx.x / kStepWave] = w;
    __syncthreads();
    double r = lds[0];
    for (int k = 1; k < kNormThreads / kStepWave; ++k) r = MAXIMUM ? fmax(r, lds[k]) : r + lds[k];
    return r;
  };
  auto norm_of = [&](double r) { return (float)(fabs(scale) * (MAXIMUM ? (double)__uint_as_float((uint32_t)r) : sqrt(r))); };
  double all = joined();
  if (gridDim.x == 1) {
    if (threadIdx.x == 0) *norm = norm_of(all);
    return;
  }
  if (threadIdx.x == 0) {
    __hip_atomic_store(&scratch->part[blockIdx.x], all, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // The result is stored past the caches of this XCD and has arrived before the ticket is drawn (a ticket that also writes these caches
    // back costs 50 ns a workgroup, one after the other).  A counter takes 12 ns a ticket: with one for all, 488 workgroups took 9.7 us.
    __builtin_amdgcn_s_waitcnt(0);
    const uint32_t turns = (gridDim.x + kNormTurn - 1u) / kNormTurn, mine = blockIdx.x / kNormTurn;
    last = draw(scratch->tickets[mine], min(kNormTurn, gridDim.x - mine * kNormTurn)) && (turns == 1u || draw(scratch->tickets[kNormGroups / kNormTurn], turns));
  }
  __syncthreads();
  if (!last) return;
  // the last workgroup adds up the others' results, in an order that does not depend on who came when
  sum = 0.0; top = 0;
  for (uint32_t k = threadIdx.x; k < gridDim.x; k += kNormThreads) {
    const double p = __hip_atomic_load(&scratch->part[k], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (MAXIMUM) top = max(top, (uint32_t)p);
    else sum += p;
  }
  all = joined();
  if (threadIdx.x == 0) *norm = norm_of(all);
}

// ------------------------------------------------------------------------------------------
// clipping
//
// A workgroup per chunk, which ends with it; stores go past the caches, which have nothing to keep of them (into fp32, norm and clipping of
// the sixteen buckets: 250 us, with ordinary stores 289; of the 250, the clipping takes 182, or 6.9 TB/s).  The chunks are taken from the
// list's end: the norm has just read them in the other order, and the memory-side cache holds the last 256 MiB of that (from the front,
// with workgroups of 256: 278 instead of 263 us).
// ------------------------------------------------------------------------------------------
// What a gradient is multiplied with: its scale and, where the norm (of the scaled gradients) is above max_norm, the factor that brings
// it there.  A norm of infinity gives 0 (and NaN from infinite gradients), a norm of NaN gives NaN.
__device__ __forceinline__ float clip_factor(float norm, float max_norm, float scale) {
  const float q = max_norm / (norm + 1e-6f);
  return scale * (q > 1.0f ? 1.0f : q);
}

template <int SD, int DD, int N>
__device__ __forceinline__ StepVec<DD, N> clip_vector(const StepVec<SD, N>& r, float f) {
  float x[N];
#pragma unroll
  for (int k = 0; k < N; ++k) x[k] = r.get(k) * f;
  StepVec<DD, N> o;
  o.put(x);
  return o;
}

template <int SD, int DD>
__device__ __forceinline__ void clip_chunk(const ListChunk& s, const ListChunk& d, float f) {
  constexpr int N = 4, U = (int)kChunk / (N * kClipThreads);
  const void* from = (const void*)s.ptr;
  void* to = (void*)d.ptr;
  if (s.n == kChunk) {
    StepVec<SD, N> r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) r[u].load(from, (size_t)(u * kClipThreads + threadIdx.x) * N);
#pragma unroll
    for (int u = 0; u < U; ++u) clip_vector<SD, DD, N>(r[u], f).stream(to, (size_t)(u * kClipThreads + threadIdx.x) * N);
    return;
  }
  const uint32_t nvec = s.n / N;
  for (uint32_t v = threadIdx.x; v < nvec; v += kClipThreads) {
    StepVec<SD, N> r;
    r.load(from, (size_t)v * N);
    clip_vector<SD, DD, N>(r, f).stream(to, (size_t)v * N);
  }
  const uint32_t i = nvec * N + threadIdx.x;
  if (i < s.n) step_put<DD>(to, i, step_get<SD>(from, i) * f);
}

template <int SD>
__device__ __forceinline__ void clip_chunk_to(const ListChunk& s, const ListChunk& d, float f) {
  if (d.dtype == DFX_F32) clip_chunk<SD, DFX_F32>(s, d, f);
  else if (d.dtype == DFX_BF16) clip_chunk<SD, DFX_BF16>(s, d, f);
  else clip_chunk<SD, DFX_F16>(s, d, f);
}

// (src and dst may be the same tensors: no __restrict__ on what the chunks point to)
__global__ void __launch_bounds__(kClipThreads) dfx_clip_kernel(const ListChunk* __restrict__ src, const ListChunk* __restrict__ dst, uint32_t nchunks, const float* norm, float max_norm, float scale, bool in_place) {
  const float f = clip_factor(*norm, max_norm, scale);
  if (in_place && f == 1.0f) return;      // the gradients are what they are to become
  for (uint32_t k = blockIdx.x; k < nchunks; k += gridDim.x) {
    const uint32_t c = nchunks - 1u - k;
    const ListChunk s = src[c], d = dst[c];
    if (s.dtype == DFX_F32) clip_chunk_to<DFX_F32>(s, d, f);
    else if (s.dtype == DFX_BF16) clip_chunk_to<DFX_BF16>(s, d, f);
    else clip_chunk_to<DFX_F16>(s, d, f);
  }
}

// ------------------------------------------------------------------------------------------
// AdamW
//
// HBM bounds it: 28 bytes of a parameter with a 16-bit gradient and copy pass through, 372 M of them in 1740 us (6.0 TB/s).  A thread takes one
// vector of four of every list and its workgroup ends, which leaves the order of requests to the dispatcher.  The lists of a model lie alike in
// memory, so a thread's loads go to the same channels at the same moment; in a long list the second waits for the first to arrive, and the
// others for the second: 1740 instead of 2069 us.  Below about 700 chunks the waits cost more than they give (4 M parameters 19.5 and 19.2
// us, 8 M 43 and 45, 500 k 4.8 and 4.5).  Persistent workgroups (2048 of 256) 2400 us, with ordinary stores 2540.  A step number that is read on
// the device costs every thread two powers in 64 bits ahead of its loads: the 372 M then take 2100 us, 500 k 7.0 a call instead of 6.4.
// ------------------------------------------------------------------------------------------
struct AdamArgs {
  const ListChunk *p, *g, *m, *v, *copy;      // copy: may be null
  const float* norm;                          // may be null: nothing is clipped
  const uint32_t* step_dev;                   // may be null: correct1 / correct2 hold
  const float* lr_dev;                        // may be null: lr holds
  double beta1_d, beta2_d;
  float lr, beta1, beta2, one_beta1, one_beta2, eps, decay, scale, max_norm;
  float correct1, correct2;                   // 1 / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
};

struct AdamRates { float f, decay, beta1, one_beta1, beta2, one_beta2, rate, correct2, eps; };

__device__ __forceinline__ void adam_element(const AdamRates& a, float& p, float g, float& m, float& v) {
  g *= a.f;
  m = fmaf(a.beta1, m, a.one_beta1 * g);
  v = fmaf(a.beta2, v, a.one_beta2 * g * g);
  // (what p loses is made up apart from p: 1 - lr decay holds 32-bit numbers below 1 to 6e-8 only, which is all of a decay of lr 1e-6 and 0.01)
  p -= fmaf(a.decay, p, a.rate * m / fmaf(sqrtf(v), a.correct2, a.eps));
}

template <int GD, int CD, bool STAGED>      // CD < 0: no copy
__device__ __forceinline__ void adam_vector(const AdamRates& a, const ListChunk& p, const ListChunk& g, const ListChunk& m, const ListChunk& v, const ListChunk& copy, size_t i) {
  constexpr int N = 4, C = CD < 0 ? DFX_F32 : CD;
  StepVec<DFX_F32, N> rp, rm, rv;
  StepVec<GD, N> rg;
  rp.load((const void*)p.ptr, i);
  if (STAGED) loads_arrived();
  rm.load((const void*)m.ptr, i);
  if (STAGED) loads_arrived();
  rv.load((const void*)v.ptr, i);
  rg.load((const void*)g.ptr, i);
  float xp[N], xm[N], xv[N];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    xp[j] = rp.get(j); xm[j] = rm.get(j); xv[j] = rv.get(j);
    adam_element(a, xp[j], rg.get(j), xm[j], xv[j]);
  }
  rp.put(xp); rm.put(xm); rv.put(xv);
  rp.stream((void*)p.ptr, i);
  rm.stream((void*)m.ptr, i);
  rv.stream((void*)v.ptr, i);
  if (CD >= 0) {
    StepVec<C, N> rc;
    rc.put(xp);
    rc.stream((void*)copy.ptr, i);
  }
}

template <int GD, int CD, bool STAGED>
__device__ __forceinline__ void adam_chunk(const AdamRates& a, const ListChunk& p, const ListChunk& g, const ListChunk& m, const ListChunk& v, const ListChunk& copy, uint32_t part) {
  constexpr int N = 4, C = CD < 0 ? DFX_F32 : CD;
  constexpr uint32_t stride = kAdamThreads * kAdamParts;
  const uint32_t nvec = p.n / N, me = part * kAdamThreads + threadIdx.x;
  static_assert(kChunk == stride * N, "a whole chunk is a vector for each thread of its workgroups");
  if (p.n == kChunk) {
    adam_vector<GD, CD, STAGED>(a, p, g, m, v, copy, me * N);
    return;
  }
  if (me < nvec) adam_vector<GD, CD, STAGED>(a, p, g, m, v, copy, me * N);
  const uint32_t i = nvec * N + me;
  if (i < p.n) {
    float xp = step_get<DFX_F32>((const void*)p.ptr, i), xm = step_get<DFX_F32>((const void*)m.ptr, i), xv = step_get<DFX_F32>((const void*)v.ptr, i);
    adam_element(a, xp, step_get<GD>((const void*)g.ptr, i), xm, xv);
    step_put<DFX_F32>((void*)p.ptr, i, xp);
    step_put<DFX_F32>((void*)m.ptr, i, xm);
    step_put<DFX_F32>((void*)v.ptr, i, xv);
    if (CD >= 0) step_put<C>((void*)copy.ptr, i, xp);
  }
}

template <int GD, bool STAGED>
__device__ __forceinline__ void adam_chunk_copy(const AdamRates& a, const ListChunk& p, const ListChunk& g, const ListChunk& m, const ListChunk& v, const ListChunk& copy, uint32_t part, bool has_copy) {
  if (!has_copy) adam_chunk<GD, -1, STAGED>(a, p, g, m, v, copy, part);
  else if (copy.dtype == DFX_BF16) adam_chunk<GD, DFX_BF16, STAGED>(a, p, g, m, v, copy, part);
  else if (copy.dtype == DFX_F16) adam_chunk<GD, DFX_F16, STAGED>(a, p, g, m, v, copy, part);
  else adam_chunk<GD, DFX_F32, STAGED>(a, p, g, m, v, copy, part);
}

template <bool STAGED>
__global__ void __launch_bounds__(kAdamThreads) dfx_adamw_kernel(AdamArgs a) {
  float f = a.scale, lr = a.lr, c1 = a.correct1, c2 = a.correct2;
  if (a.norm) {
    const float norm = *a.norm;
    if (!(norm < INFINITY)) return;       // (infinite or NaN: the gradients overflowed, the step is left out)
    f = clip_factor(norm, a.max_norm, a.scale);
  }
  if (a.lr_dev) lr = *a.lr_dev;
  if (a.step_dev) {
    const double t = (double)*a.step_dev;
    if (t == 0.0) return;                 // (no update has this number: the corrections would be infinite and every parameter NaN)
    c1 = (float)(1.0 / (1.0 - pow(a.beta1_d, t)));
    c2 = (float)(1.0 / sqrt(1.0 - pow(a.beta2_d, t)));
  }
  const AdamRates r = {f, lr * a.decay, a.beta1, a.one_beta1, a.beta2, a.one_beta2, lr * c1, c2, a.eps};
  const uint32_t c = blockIdx.x / kAdamParts, part = blockIdx.x % kAdamParts;
  const ListChunk p = a.p[c], g = a.g[c], m = a.m[c], v = a.v[c], copy = a.copy ? a.copy[c] : ListChunk{0, 0, 0};
  if (g.dtype == DFX_F32) adam_chunk_copy<DFX_F32, STAGED>(r, p, g, m, v, copy, part, a.copy != nullptr);
  else if (g.dtype == DFX_BF16) adam_chunk_copy<DFX_BF16, STAGED>(r, p, g, m, v, copy, part, a.copy != nullptr);
  else adam_chunk_copy<DFX_F16, STAGED>(r, p, g, m, v, copy, part, a.copy != nullptr);
}

__global__ void dfx_zero_norm_kernel(float* norm) { *norm = 0.0f; }

// ------------------------------------------------------------------------------------------
// host
// ------------------------------------------------------------------------------------------
bool on_its_device(const dfx_list* l) {
  int device = -1;
  return hipGetDevice(&device) == hipSuccess && device == l->device;
}

bool same_counts(const dfx_list* a, const dfx_list* b) {
  return a == b || (a->device == b->device && a->counts.size() == b->counts.size() && (a->counts.empty() || !memcmp(a->counts.data(), b->counts.data(), a->counts.size() * sizeof(size_t))));
}

// Whether no tensor of dst, whose own lie apart, shares memory with one of src, but for the same tensor at the same place.  Both go by addresses, so one
// walk does; lists in buckets of their own do not meet at all.
bool written_apart(const dfx_list* src, const dfx_list* dst) {
  const std::vector<ListSpan>&s = src->spans, &d = dst->spans;
  if (s.empty() || d.empty() || d.back().hi <= s.front().lo || (src->apart && s.back().hi <= d.front().lo)) return true;
  size_t j = 0;
  for (const ListSpan& x : s) {
    while (j < d.size() && d[j].hi <= x.lo) ++j;
    for (size_t i = j; i < d.size() && d[i].lo < x.hi; ++i)
      if (d[i].k != x.k || d[i].lo != x.lo || src->tensors[x.k].dtype != dst->tensors[x.k].dtype) return false;
    if (j == d.size()) break;
  }
  return true;
}

int check_norm(const dfx_list* l, int kind, double scale, const float* norm) {
  if (!l || !norm || ((uintptr_t)norm & 3u) || (kind != DFX_NORM_2 && kind != DFX_NORM_INF) || !isfinite(scale)) return DFX_ERR_INVALID_ARG;
  return on_its_device(l) ? DFX_OK : DFX_ERR_INVALID_ARG;
}

int check_clip(const dfx_list* src, const dfx_list* dst, const float* norm, double max_norm, double scale) {
  if (!src || !norm || ((uintptr_t)norm & 3u) || !(max_norm > 0.0) || !step_normal(scale)) return DFX_ERR_INVALID_ARG;
  if (!(dst ? dst : src)->apart || (dst && dst != src && (!same_counts(src, dst) || !written_apart(src, dst)))) return DFX_ERR_INVALID_ARG;
  return on_its_device(src) ? DFX_OK : DFX_ERR_INVALID_ARG;
}

// in 32 bits: none is above the largest, so that a norm of infinity is above each
float max_norm_of(double max_norm) { return (float)std::min(max_norm, (double)FLT_MAX); }

int launch_norm(const dfx_list* l, int kind, double scale, float* norm, hipStream_t stream) {
  if (!l->nchunks) {
    return step_launch(dfx_zero_norm_kernel, dim3(1), 1, stream, norm);
  }
  const dim3 grid(std::min<uint32_t>(l->nchunks, (uint32_t)kNormGroups));
  return step_launch(kind == DFX_NORM_2 ? dfx_norm_kernel<false> : dfx_norm_kernel<true>, grid, kNormThreads, stream, l->chunks, l->nchunks, l->scratch, scale, norm);
}

int launch_clip(const dfx_list* src, const dfx_list* dst, const float* norm, double max_norm, double scale, hipStream_t stream) {
  if (!dst) dst = src;
  if (!src->nchunks) return DFX_OK;
  return step_launch(dfx_clip_kernel, dim3(std::min(src->nchunks, kMaxGroups)), kClipThreads, stream, src->chunks, dst->chunks, src->nchunks, norm, max_norm_of(max_norm), (float)scale, dst == src);
}

}  // namespace

extern "C" {

int dfx_list_create(dfx_list** out, const dfx_tensor* tensors, int n) {
  if (out) *out = nullptr;
  if (!out || n < 0 || (n && !tensors)) return DFX_ERR_INVALID_ARG;
  uint64_t nchunks = 0;
  for (int k = 0; k < n; ++k) {
    const dfx_tensor& t = tensors[k];
    if (t.reserved0 || (t.dtype != DFX_F32 && t.dtype != DFX_BF16 && t.dtype != DFX_F16)) return DFX_ERR_INVALID_ARG;
    if (t.count && (!t.ptr || ((uintptr_t)t.ptr % step_elem_bytes(t.dtype)))) return DFX_ERR_INVALID_ARG;
    if (t.count > (SIZE_MAX >> 4)) return DFX_ERR_TOO_LARGE;
    nchunks += (t.count + kChunk - 1) / kChunk;
    if (nchunks > 0x3fffffffu) return DFX_ERR_TOO_LARGE;
  }
  dfx_list* l = nullptr;
  int rc = DFX_OK;
  try {
    l = new dfx_list;
    l->tensors.assign(tensors, tensors + n);
    for (const dfx_tensor& t : l->tensors) {
      l->counts.push_back(t.count);
      l->all_f32 = l->all_f32 && t.dtype == DFX_F32;
      if (t.count) l->spans.push_back({(uintptr_t)t.ptr, (uintptr_t)t.ptr + t.count * step_elem_bytes(t.dtype), l->counts.size() - 1});
    }
    const auto before = [](const ListSpan& a, const ListSpan& b) { return a.lo < b.lo; };
    if (!std::is_sorted(l->spans.begin(), l->spans.end(), before)) std::sort(l->spans.begin(), l->spans.end(), before);
    for (size_t k = 1; k < l->spans.size(); ++k) l->apart = l->apart && l->spans[k - 1].hi <= l->spans[k].lo;
    l->nchunks = (uint32_t)nchunks;
    // scratch in front, zeroed with the table's upload
    const size_t at = (sizeof(ListScratch) + 255) / 256 * 256, bytes = at + nchunks * sizeof(ListChunk);
    std::vector<unsigned char> host(bytes, 0);
    ListChunk* c = (ListChunk*)(host.data() + at);
    for (const dfx_tensor& t : l->tensors)
      for (size_t i = 0; i < t.count; i += kChunk) *c++ = {(uint64_t)(uintptr_t)t.ptr + i * step_elem_bytes(t.dtype), (uint32_t)std::min<size_t>(kChunk, t.count - i), (int32_t)t.dtype};
    unsigned char* dev = nullptr;
    if (hipGetDevice(&l->device) != hipSuccess || hipMalloc((void**)&dev, bytes) != hipSuccess) rc = DFX_ERR_HIP;
    else {
      l->scratch = (ListScratch*)dev;
      l->chunks = (ListChunk*)(dev + at);
      if (hipMemcpy(dev, host.data(), bytes, hipMemcpyHostToDevice) != hipSuccess) rc = DFX_ERR_HIP;
    }
  } catch (...) {                          // (host memory)
    rc = DFX_ERR_NO_RESOURCES;
  }
  if (rc != DFX_OK) {
    if (l && l->scratch) (void)hipFree(l->scratch);
    delete l;
    return rc;
  }
  *out = l;
  return DFX_OK;
}

int dfx_list_destroy(dfx_list* l) {
  if (!l) return DFX_ERR_INVALID_ARG;
  const hipError_t e = hipFree(l->scratch);
  delete l;
  return e == hipSuccess ? DFX_OK : DFX_ERR_HIP;
}

int dfx_grad_norm(dfx_list* grads, dfx_norm_kind kind, double grad_scale, float* norm_dev, void* hip_stream) {
  const int rc = check_norm(grads, kind, grad_scale, norm_dev);
  return rc != DFX_OK ? rc : launch_norm(grads, kind, grad_scale, norm_dev, (hipStream_t)hip_stream);
}

int dfx_grad_clip(dfx_list* src, dfx_list* dst, const float* norm_dev, double max_norm, double grad_scale, void* hip_stream) {
  const int rc = check_clip(src, dst, norm_dev, max_norm, grad_scale);
  return rc != DFX_OK ? rc : launch_clip(src, dst, norm_dev, max_norm, grad_scale, (hipStream_t)hip_stream);
}

int dfx_clip_grad_norm(dfx_list* src, dfx_list* dst, dfx_norm_kind kind, double max_norm, double grad_scale, float* norm_dev, void* hip_stream) {
  int rc = check_norm(src, kind, grad_scale, norm_dev);
  if (rc == DFX_OK) rc = check_clip(src, dst, norm_dev, max_norm, grad_scale);
  if (rc == DFX_OK) rc = launch_norm(src, kind, grad_scale, norm_dev, (hipStream_t)hip_stream);
  return rc != DFX_OK ? rc : launch_clip(src, dst, norm_dev, max_norm, grad_scale, (hipStream_t)hip_stream);
}

int dfx_adamw_default(dfx_adamw_config* cfg) {
  if (!cfg) return DFX_ERR_INVALID_ARG;
  memset(cfg, 0, sizeof(*cfg));
  cfg->struct_bytes = sizeof(*cfg);
  cfg->step = 1;
  cfg->lr = 1e-3; cfg->beta1 = 0.9; cfg->beta2 = 0.999; cfg->eps = 1e-8; cfg->weight_decay = 0.01;
  cfg->grad_scale = 1.0; cfg->max_norm = 1.0;
  return DFX_OK;
}

int dfx_adamw(dfx_list* params, dfx_list* grads, dfx_list* exp_avg, dfx_list* exp_avg_sq, dfx_list* copies, const dfx_adamw_config* cfg, const float* norm_dev, void* hip_stream) {
  if (!params || !grads || !exp_avg || !exp_avg_sq || !cfg || cfg->struct_bytes != sizeof(*cfg)) return DFX_ERR_INVALID_ARG;
  if (!(cfg->beta1 >= 0.0 && cfg->beta1 < 1.0) || !(cfg->beta2 >= 0.0 && cfg->beta2 < 1.0) || !(cfg->eps >= 0.0) || !step_normal(cfg->eps) || !step_fits(cfg->lr) ||
      !step_fits(cfg->weight_decay) || !step_normal(cfg->grad_scale) || (!cfg->step_dev && !cfg->step) || (norm_dev && !(cfg->max_norm > 0.0)))
    return DFX_ERR_INVALID_ARG;
  if (((uintptr_t)norm_dev & 3u) || ((uintptr_t)cfg->step_dev & 3u) || ((uintptr_t)cfg->lr_dev & 3u)) return DFX_ERR_INVALID_ARG;
  if (!same_counts(params, grads) || !same_counts(params, exp_avg) || !same_counts(params, exp_avg_sq) || (copies && !same_counts(params, copies))) return DFX_ERR_INVALID_ARG;
  if (params == exp_avg || params == exp_avg_sq || exp_avg == exp_avg_sq || params == grads || grads == exp_avg || grads == exp_avg_sq || (copies && (copies == params || copies == grads || copies == exp_avg || copies == exp_avg_sq))) return DFX_ERR_INVALID_ARG;
  if (!params->apart || !exp_avg->apart || !exp_avg_sq->apart || (copies && !copies->apart)) return DFX_ERR_INVALID_ARG;
  if (!params->all_f32 || !exp_avg->all_f32 || !exp_avg_sq->all_f32 || !on_its_device(params)) return DFX_ERR_INVALID_ARG;
  if (!params->nchunks) return DFX_OK;
  AdamArgs a;
  memset(&a, 0, sizeof(a));
  a.p = params->chunks; a.g = grads->chunks; a.m = exp_avg->chunks; a.v = exp_avg_sq->chunks; a.copy = copies ? copies->chunks : nullptr;
  a.norm = norm_dev; a.step_dev = cfg->step_dev; a.lr_dev = cfg->lr_dev;
  a.beta1_d = cfg->beta1; a.beta2_d = cfg->beta2;
  a.lr = (float)cfg->lr; a.beta1 = (float)cfg->beta1; a.beta2 = (float)cfg->beta2;
  a.one_beta1 = (float)(1.0 - cfg->beta1); a.one_beta2 = (float)(1.0 - cfg->beta2);
  a.eps = (float)cfg->eps; a.decay = (float)cfg->weight_decay; a.scale = (float)cfg->grad_scale; a.max_norm = max_norm_of(cfg->max_norm);
  a.correct1 = (float)(1.0 / (1.0 - pow(cfg->beta1, (double)cfg->step)));
  a.correct2 = (float)(1.0 / sqrt(1.0 - pow(cfg->beta2, (double)cfg->step)));
  for (uint32_t done = 0; done < params->nchunks; done += kMaxGroups) {      // (more than one launch beyond 2^20 chunks)
    const uint32_t n = std::min(params->nchunks - done, kMaxGroups);
    const int rc = step_launch(params->nchunks >= kAdamStaged ? dfx_adamw_kernel<true> : dfx_adamw_kernel<false>, dim3(n * kAdamParts), kAdamThreads, (hipStream_t)hip_stream, a);
    if (rc != DFX_OK) return rc;
    a.p += n; a.g += n; a.m += n; a.v += n;
    if (a.copy) a.copy += n;
  }
  return DFX_OK;
}

}  // extern "C"

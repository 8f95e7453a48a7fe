// The clipped policy loss with a KL term over rows of logits, forward and backward, in front of a step's gradient all-reduce.
//
// A row's softmax is taken around its largest logit m: S = sum exp(c (z - m)), logp = c (z_t - m) - log S, and the gradient of z_j is
// g ([j = t] - exp(c (z_j - m)) / S) with one number g for the row.  So a row is read, reduced to (m, S), and written once g is known.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>

#include "dfx_step.h"

namespace {

constexpr uint32_t kGroups = 2048;       // workgroups of a call, at most: each leaves its share of the sums
constexpr int kSums = 5;
constexpr int kSumThreads = 256;

struct LossArgs {
  const void* logits;
  void* grad;
  size_t logits_stride, grad_stride;
  const int64_t* targets;
  const float *old_logp, *ref_logp, *advantage, *weight, *scale;
  float *logp, *loss, *sums;
  double* part;                          // [workgroups][kSums]
  uint32_t rows, vocab;
  double clip_low, clip_high, kl_coef, c;
  float c_log2e;                         // c / log 2: exponents are taken to base 2
};

// exp(c (z - m)): the difference first, which is exact where it matters and cannot overflow for logits of the type's lowest value
__device__ __forceinline__ float loss_exp(float z, float m, float c_log2e) { return __builtin_amdgcn_exp2f((z - m) * c_log2e); }

struct MaxSum { float m, s; };           // s = sum exp(c (z - m)); nothing seen yet: m = -infinity, s = 0

// m to take differences from: of a row that has only seen -infinity, any finite one (exp(-infinity - 0) = 0, and NaN stays NaN)
__device__ __forceinline__ float loss_base(float m) { return m == -INFINITY ? 0.0f : m; }

__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b, float c_log2e) {
  const float m = fmaxf(a.m, b.m), base = loss_base(m);
  return {m, a.s * loss_exp(a.m, base, c_log2e) + b.s * loss_exp(b.m, base, c_log2e)};
}

// What a row comes to, by one thread.  In 64 bits: a logp of -10 holds no more than 5e-7 in 32, which would be the ratio's error.
struct RowEnd { double logp, loss, pg, kl, clipped, w; float g; };

__device__ __forceinline__ RowEnd row_end(const LossArgs& a, uint32_t row, MaxSum ms, float zt) {
  RowEnd e = {0, 0, 0, 0, 0, 0, 0};
  if (ms.s == 0.0f) return e;            // no logit above -infinity
  e.logp = a.c * ((double)zt - (double)loss_base(ms.m)) - log((double)ms.s);
  if (!a.advantage) return e;
  e.w = a.weight ? (double)a.weight[row] : 1.0;
  const double A = (double)a.advantage[row];
  const double r = a.old_logp ? exp(e.logp - (double)a.old_logp[row]) : 1.0;
  const bool clipped = A >= 0.0 ? r > 1.0 + a.clip_high : r < 1.0 - a.clip_low;
  const double used = clipped ? (A >= 0.0 ? 1.0 + a.clip_high : 1.0 - a.clip_low) : r;
  e.pg = e.w * (-A * used);
  double slope = clipped ? 0.0 : -A * r;
  if (a.ref_logp) {
    const double d = (double)a.ref_logp[row] - e.logp, x = expm1(d);
    e.kl = e.w * (x - d);
    slope -= a.kl_coef * x;
  }
  e.clipped = clipped ? e.w : 0.0;
  e.loss = e.pg + a.kl_coef * e.kl;
  e.g = (float)(a.c * e.w * slope * (a.scale ? (double)*a.scale : 1.0));
  return e;
}

// whether a row has anything to learn from, by what is known before its logits
__device__ __forceinline__ bool row_counts(const LossArgs& a, uint32_t row) {
  const int64_t t = a.targets[row];
  return t >= 0 && t < (int64_t)a.vocab && (!a.weight || a.weight[row] != 0.0f);
}

template <int DT, int THREADS>
__global__ void __launch_bounds__(THREADS) dfx_loss_rows_kernel(LossArgs a) {
  typedef typename StepElem<DT>::raw raw;
  constexpr int N = 16 / (int)sizeof(raw), WAVES = THREADS / kStepWave;
  __shared__ MaxSum lds[WAVES];
  __shared__ float row_g, row_m, row_s;
  const uint32_t nvec = a.vocab / N, rest = nvec * N + threadIdx.x;
  double sums[kSums] = {0, 0, 0, 0, 0};
  for (uint32_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const raw* z = (const raw*)a.logits + (size_t)row * a.logits_stride;
    raw* out = a.grad ? (raw*)a.grad + (size_t)row * a.grad_stride : nullptr;
    const bool counts = row_counts(a, row);
    MaxSum ms = {-INFINITY, 0.0f};
    float zt = 0.0f;
    if (counts) {
      for (uint32_t v = threadIdx.x; v < nvec; v += THREADS) {
        StepVec<DT, N> r;
        r.load(z, (size_t)v * N);
        float x[N], m = ms.m;
#pragma unroll
        for (int k = 0; k < N; ++k) { x[k] = r.get(k); m = fmaxf(m, x[k]); }
        const float base = loss_base(m);
        float s = ms.s * loss_exp(ms.m, base, a.c_log2e);
#pragma unroll
        for (int k = 0; k < N; ++k) s += loss_exp(x[k], base, a.c_log2e);
        ms = {m, s};
      }
      if (rest < a.vocab) {
        const float x = step_get<DT>(z, rest);
        ms = join(ms, {x, x == -INFINITY ? 0.0f : 1.0f}, a.c_log2e);
      }
      if (threadIdx.x == 0) zt = step_get<DT>(z, (size_t)a.targets[row]);
#pragma unroll
      for (int d = kStepWave / 2; d; d >>= 1) ms = join(ms, {__shfl_xor(ms.m, d), __shfl_xor(ms.s, d)}, a.c_log2e);
      if ((threadIdx.x & (kStepWave - 1)) == 0) lds[threadIdx.x / kStepWave] = ms;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      RowEnd e = {0, 0, 0, 0, 0, 0, 0};
      if (counts) {
        ms = lds[0];
        for (int k = 1; k < WAVES; ++k) ms = join(ms, lds[k], a.c_log2e);
        e = row_end(a, row, ms, zt);
      }
      row_g = e.g; row_m = loss_base(ms.m); row_s = ms.s == 0.0f ? 0.0f : 1.0f / ms.s;
      if (a.logp) a.logp[row] = (float)e.logp;
      if (a.loss) a.loss[row] = (float)e.loss;
      sums[0] += e.loss; sums[1] += e.pg; sums[2] += e.kl; sums[3] += e.clipped; sums[4] += e.w;
    }
    __syncthreads();
    if (!out) continue;
    const float g = row_g, m = row_m, gs = -row_g * row_s;
    const uint32_t t = counts ? (uint32_t)a.targets[row] : 0xffffffffu;
    const bool nothing = !counts || row_s == 0.0f;
    for (uint32_t v = threadIdx.x; v < nvec; v += THREADS) {
      float x[N];
      if (nothing) {
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = 0.0f;
      } else {
        StepVec<DT, N> r;
        r.load(z, (size_t)v * N);
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = gs * loss_exp(r.get(k), m, a.c_log2e) + (v * N + k == t ? g : 0.0f);
      }
      StepVec<DT, N> o;
      o.put(x);
      o.store(out, (size_t)v * N);
    }
    if (rest < a.vocab) step_put<DT>(out, rest, nothing ? 0.0f : gs * loss_exp(step_get<DT>(z, rest), m, a.c_log2e) + (rest == t ? g : 0.0f));
  }
  if (a.sums && threadIdx.x == 0)
    for (int k = 0; k < kSums; ++k) a.part[(size_t)blockIdx.x * kSums + k] = sums[k];
}

// the workgroups' shares, in an order that is always the same
__global__ void __launch_bounds__(kSumThreads) dfx_loss_sums_kernel(const double* part, uint32_t n, float* out) {
  __shared__ double lds[kSumThreads / kStepWave][kSums];
  double s[kSums] = {0, 0, 0, 0, 0};
  for (uint32_t i = threadIdx.x; i < n; i += kSumThreads)
    for (int k = 0; k < kSums; ++k) s[k] += part[(size_t)i * kSums + k];
  for (int k = 0; k < kSums; ++k) {
    s[k] = wave_sum(s[k]);
    if ((threadIdx.x & (kStepWave - 1)) == 0) lds[threadIdx.x / kStepWave][k] = s[k];
  }
  __syncthreads();
  if (threadIdx.x < kSums) {
    double t = 0;
    for (int w = 0; w < kSumThreads / kStepWave; ++w) t += lds[w][threadIdx.x];
    out[threadIdx.x] = (float)t;
  }
}

uint32_t loss_groups(uint64_t rows) { return (uint32_t)std::min<uint64_t>(rows, kGroups); }

template <int DT>
void launch_rows(const LossArgs& a, uint32_t groups, hipStream_t s) {
  if (a.vocab <= 4096) hipLaunchKernelGGL((dfx_loss_rows_kernel<DT, 256>), dim3(groups), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((dfx_loss_rows_kernel<DT, 1024>), dim3(groups), dim3(1024), 0, s, a);
}

// rows of n elements, stride elements apart, from p on: [first, second) in bytes
struct Extent { uintptr_t lo, hi; };
Extent extent(const void* p, size_t rows, size_t vocab, size_t stride, size_t eb) {
  return {(uintptr_t)p, (uintptr_t)p + ((rows - 1) * stride + vocab) * eb};
}

}  // namespace

extern "C" {

size_t dfx_policy_loss_workspace(size_t rows, size_t vocab, dfx_dtype dtype) {
  (void)vocab; (void)dtype;
  return std::max<size_t>(1, loss_groups(rows)) * kSums * sizeof(double);
}

int dfx_policy_loss(const dfx_policy_loss_args* u, void* hip_stream) {
  if (!u || u->struct_bytes != sizeof(*u)) return DFX_ERR_INVALID_ARG;
  if (u->dtype != DFX_F32 && u->dtype != DFX_BF16 && u->dtype != DFX_F16) return DFX_ERR_INVALID_ARG;
  if (u->rows > 0x7fffffffull || u->vocab > (1ull << 30)) return DFX_ERR_TOO_LARGE;
  const size_t eb = step_elem_bytes(u->dtype), ls = u->logits_stride ? u->logits_stride : u->vocab, gs = u->grad_stride ? u->grad_stride : u->vocab;
  if (ls < u->vocab || (u->grad && gs < u->vocab)) return DFX_ERR_INVALID_ARG;
  if (u->rows && ((ls > SIZE_MAX / 8 / u->rows) || (u->grad && gs > SIZE_MAX / 8 / u->rows))) return DFX_ERR_TOO_LARGE;
  if (!isfinite(u->clip_low) || u->clip_low < 0.0 || u->clip_low > 1.0 || !isfinite(u->clip_high) || u->clip_high < 0.0 || !isfinite(u->kl_coef) || !isfinite(u->inv_temperature) || !(u->inv_temperature > 0.0)) return DFX_ERR_INVALID_ARG;
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
  LossArgs a;
  memset(&a, 0, sizeof(a));
  a.logits = u->logits; a.grad = u->grad; a.logits_stride = ls; a.grad_stride = gs;
  a.targets = u->targets; a.old_logp = u->old_logp; a.ref_logp = u->ref_logp; a.advantage = u->advantage; a.weight = u->weight; a.scale = u->scale;
  a.logp = u->logp; a.loss = u->loss; a.sums = u->sums; a.part = (double*)u->workspace;
  a.rows = (uint32_t)u->rows; a.vocab = (uint32_t)u->vocab;
  a.clip_low = u->clip_low; a.clip_high = u->clip_high; a.kl_coef = u->kl_coef; a.c = u->inv_temperature;
  a.c_log2e = (float)(u->inv_temperature * 1.4426950408889634);
  hipStream_t s = (hipStream_t)hip_stream;
  const uint32_t groups = loss_groups(u->rows);
  if (groups) {
    if (u->dtype == DFX_F32) launch_rows<DFX_F32>(a, groups, s);
    else if (u->dtype == DFX_BF16) launch_rows<DFX_BF16>(a, groups, s);
    else launch_rows<DFX_F16>(a, groups, s);
    if (hipGetLastError() != hipSuccess) return DFX_ERR_HIP;
  }
  if (u->sums) hipLaunchKernelGGL(dfx_loss_sums_kernel, dim3(1), dim3(kSumThreads), 0, s, a.part, groups, u->sums);
  return hipGetLastError() == hipSuccess ? DFX_OK : DFX_ERR_HIP;
}

}  // extern "C"

// Layer norm over rows, forward and backward.
//
// h = (x - mean) r, r = 1 / sqrt(var + eps), y = h w + b;  with g = dy w:  dx = r (g - mean g - h mean(g h)), dw = sum dy h, db = sum dy.
// A row stays in registers from its mean to its results.  Mean and variance are taken one behind the other, so that a large mean costs the variance nothing; h keeps the mean's own
// rounding, 2^-24 of it or a few times that, over the deviation (as mean d, d = x - mean, it could be summed and taken out: 16384 x 4096 bf16 42 to 45 us forward, 91 to 113 backward; the sum
// of x in 64 bits instead 43 and 98).
// The backward pass makes both again rather than read what the forward pass would have to keep.
#include <float.h>
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>

#include "dfx_step.h"

namespace {

constexpr uint32_t kNormDim = 32768;     // elements of a row, at most: what a workgroup of 1024 keeps in registers
// workgroups of the backward pass, at most: each leaves its share of the sums over rows (us: 16384 x 4096 bf16 256 132, 512 94, 1024 102; 4096 x 1024 14.5, 12.4, 14.0)
constexpr uint32_t kNormGroups = 512;

struct NormArgs {
  const void *x, *dy, *weight, *bias;
  void *y, *dx;
  size_t x_stride, dy_stride, y_stride, dx_stride;
  float* part;                           // [workgroups][2][dim]: a workgroup's share of grad_weight and grad_bias; may be null
  uint32_t rows, dim;
  float eps;
  bool param_f32;
};

// N elements from element e of a row; behind its end: `beyond`
template <int DT, int N>
__device__ __forceinline__ void row_take(const void* row, uint32_t e, uint32_t dim, float* v, float beyond) {
  if (e + N <= dim) {
    if constexpr (N * (DT == DFX_F32 ? 4 : 2) == 32) {
      StepVec<DT, N / 2> a, b;
      a.load(row, e); b.load(row, e + N / 2);
#pragma unroll
      for (int k = 0; k < N / 2; ++k) { v[k] = a.get(k); v[k + N / 2] = b.get(k); }
    } else {
      StepVec<DT, N> a;
      a.load(row, e);
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] = a.get(k);
    }
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = e + k < dim ? step_get<DT>(row, e + k) : beyond;
  }
}
template <int DT, int N>
__device__ __forceinline__ void row_put(void* row, uint32_t e, uint32_t dim, const float* v) {
  if (e + N <= dim) {
    StepVec<DT, N> a;
    a.put(v);
    *(STEP_GLOBAL typename StepVec<DT, N>::words*)((STEP_GLOBAL typename StepElem<DT>::raw*)row + e) = a.w;
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (e + k < dim) step_put<DT>(row, e + k, v[k]);
  }
}
template <int DT, int N>
__device__ __forceinline__ void param_take(const void* p, bool f32, uint32_t e, uint32_t dim, float* v, float absent) {
  if (!p) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = absent;
  } else if (f32) row_take<DFX_F32, N>(p, e, dim, v, 0.0f);
  else row_take<DT, N>(p, e, dim, v, 0.0f);
}

template <int DT>
__device__ __forceinline__ const void* row_of(const void* p, size_t stride, uint32_t row) { return (const typename StepElem<DT>::raw*)p + (size_t)row * stride; }
template <int DT>
__device__ __forceinline__ void* row_of(void* p, size_t stride, uint32_t row) { return (typename StepElem<DT>::raw*)p + (size_t)row * stride; }

// Sums over the T threads of a row, for all of them.  T > 64: through lds, two of whose halves are used in turn, one barrier each.
template <int T, int THREADS, int NUM>
__device__ __forceinline__ void row_sum(float (&s)[NUM], float (*lds)[2][THREADS / kStepWave], uint32_t& turn) {
#pragma unroll
  for (int q = 0; q < NUM; ++q) s[q] = wave_sum(s[q]);
  if constexpr (T > kStepWave) {
    constexpr int W = T / kStepWave;
    const uint32_t wave = threadIdx.x / kStepWave;
    if (threadIdx.x % kStepWave == 0)
#pragma unroll
      for (int q = 0; q < NUM; ++q) lds[turn][q][wave] = s[q];
    __syncthreads();
#pragma unroll
    for (int q = 0; q < NUM; ++q) {
      s[q] = lds[turn][q][wave / W * W];
#pragma unroll
      for (int w = 1; w < W; ++w) s[q] += lds[turn][q][wave / W * W + w];
    }
    turn ^= 1u;
  }
}

// T threads to a row, U vectors a thread, THREADS / T rows of a workgroup at once.  HBM bounds it: 16384 x 4096 bf16 53 us, 5.0 TB/s as a copy; one row 3.0.
template <int DT, int T, int U>
__global__ void __launch_bounds__(T < 256 ? 256 : T) dfx_norm_kernel(NormArgs a) {
  constexpr int THREADS = T < 256 ? 256 : T, ROWS = THREADS / T, N = 16 / (int)sizeof(typename StepElem<DT>::raw);
  __shared__ float lds[2][2][THREADS / kStepWave];
  const uint32_t me = threadIdx.x % T, row = blockIdx.x * ROWS + threadIdx.x / T;
  uint32_t turn = 0;
  if (ROWS > 1 && row >= a.rows) return;  // (T is a wave or more of one: nobody waits for it)
  const void* x = row_of<DT>(a.x, a.x_stride, row);
  float v[U][N], s[1] = {0.0f};
#pragma unroll
  for (int u = 0; u < U; ++u) row_take<DT, N>(x, (u * T + me) * N, a.dim, v[u], 0.0f);
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int k = 0; k < N; ++k) s[0] += v[u][k];
  row_sum<T, THREADS, 1>(s, lds, turn);
  const float mean = s[0] / (float)a.dim;
  s[0] = 0.0f;
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int k = 0; k < N; ++k) {
      v[u][k] = (u * T + me) * N + k < a.dim ? v[u][k] - mean : 0.0f;
      s[0] = fmaf(v[u][k], v[u][k], s[0]);
    }
  row_sum<T, THREADS, 1>(s, lds, turn);
  const float r = 1.0f / sqrtf(s[0] / (float)a.dim + a.eps);
  void* y = row_of<DT>(a.y, a.y_stride, row);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t e = (u * T + me) * N;
    if (e >= a.dim) break;
    float w[N], b[N];
    param_take<DT, N>(a.weight, a.param_f32, e, a.dim, w, 1.0f);
    param_take<DT, N>(a.bias, a.param_f32, e, a.dim, b, 0.0f);
#pragma unroll
    for (int k = 0; k < N; ++k) v[u][k] = fmaf(v[u][k] * r, w[k], b[k]);
    row_put<DT, N>(y, e, a.dim, v[u]);
  }
}

// A row as it is loaded: U vectors a thread, the last of them perhaps of fewer elements.
template <int DT, int T, int U>
struct NormRow {
  static constexpr int N = 16 / (int)sizeof(typename StepElem<DT>::raw);
  StepVec<DT, N> r[U];
  __device__ __forceinline__ void take(const void* row, uint32_t me, uint32_t dim) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t e = (u * T + me) * N;
      if (e + N <= dim) r[u].load(row, e);
      else {
        float v[N];
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = e + k < dim ? step_get<DT>(row, e + k) : 0.0f;
        r[u].put(v);                     // (values of the type: nothing is rounded)
      }
    }
  }
  __device__ __forceinline__ void again() {
#pragma unroll
    for (int u = 0; u < U; ++u) r[u].again();
  }
};

// The same for the gradients.  A thread's columns are the same in every row, so that the weight and the sums over rows stay in its registers, and the next
// row is on its way while one is worked on.  With d = x - mean, mean(g h) = r mean(g d): two rounds of sums over a row, (x, g) and (d^2, g d).
// Workgroups of up to 512, two to a compute unit, have room for that in 128 registers, and so has one of 1024 for rows above 4096 16-bit elements (2048 of 32 bits).  From 8193 16-bit elements on they
// have not: up to 16384 (8192 of 32 bits, which just fit) 25 of them lie in scratch, and above that 40 to 264, where the next row is not fetched and the weight is read again (AHEAD false).
// 16384 x 4096 bf16 92 us, 4.4 TB/s (without the next row on its way 140): HBM, and a workgroup's two rounds of sums for each of its rows.  Longer rows, bf16: 8192 x 8192 108 us (3.7 TB/s),
// 4096 x 16384 162, 2048 x 32768 410 (scratch: 1.0 TB/s); fp32: 8192 x 4096 93 and 4096 x 8192 92 (4.4 TB/s), 4096 x 16384 262, 2048 x 32768 750.
template <int DT, int T, int U, int THREADS, bool AHEAD>
__global__ void __launch_bounds__(THREADS, 4) dfx_norm_grad_kernel(NormArgs a) {
  constexpr int ROWS = THREADS / T, N = 16 / (int)sizeof(typename StepElem<DT>::raw);
  __shared__ float lds[2][2][THREADS / kStepWave];
  const uint32_t me = threadIdx.x % T, sub = threadIdx.x / T, step = gridDim.x * ROWS;
  const float per = 1.0f / (float)a.dim;
  uint32_t turn = 0;
  float dw[U][N], db[U][N], w[U][N];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t e = (u * T + me) * N;
#pragma unroll
    for (int k = 0; k < N; ++k) dw[u][k] = db[u][k] = w[u][k] = 0.0f;
    if (AHEAD && e < a.dim) param_take<DT, N>(a.weight, a.param_f32, e, a.dim, w[u], 1.0f);
  }
  auto weights = [&](int u, float* v) {
    const uint32_t e = (u * T + me) * N;
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = w[u][k];
    if (!AHEAD && e < a.dim) param_take<DT, N>(a.weight, a.param_f32, e, a.dim, v, 1.0f);
    if (!AHEAD) __builtin_amdgcn_sched_barrier(0);      // (one vector's at a time)
  };
  NormRow<DT, T, U> x, y;
  uint32_t row = blockIdx.x * ROWS + sub;
  if (AHEAD && row < a.rows) {
    x.take(row_of<DT>(a.x, a.x_stride, row), me, a.dim);
    y.take(row_of<DT>(a.dy, a.dy_stride, row), me, a.dim);
  }
  for (uint32_t row0 = blockIdx.x * ROWS; row0 < a.rows; row0 += step, row += step) {      // (all of the workgroup as often)
    const bool any = row < a.rows, more = AHEAD && row < a.rows && a.rows - row > step;
    NormRow<DT, T, U> x1, y1;
    if (more) {
      x1.take(row_of<DT>(a.x, a.x_stride, row + step), me, a.dim);
      y1.take(row_of<DT>(a.dy, a.dy_stride, row + step), me, a.dim);
    }
    if (!AHEAD && any) {
      x.take(row_of<DT>(a.x, a.x_stride, row), me, a.dim);
      y.take(row_of<DT>(a.dy, a.dy_stride, row), me, a.dim);
    }
    float s[2] = {0.0f, 0.0f};
    if (any)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float wu[N];
        weights(u, wu);
#pragma unroll
        for (int k = 0; k < N; ++k) {
          s[0] += x.r[u].get(k);
          s[1] = fmaf(y.r[u].get(k), wu[k], s[1]);
        }
      }
    row_sum<T, THREADS, 2>(s, lds, turn);
    const float mean = s[0] * per, c0 = s[1] * per;
    x.again(); y.again();
    s[0] = s[1] = 0.0f;
    if (any)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float wu[N];
        weights(u, wu);
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const float d = (u * T + me) * N + k < a.dim ? x.r[u].get(k) - mean : 0.0f;
          s[0] = fmaf(d, d, s[0]);
          s[1] = fmaf(y.r[u].get(k) * wu[k], d, s[1]);
        }
      }
    row_sum<T, THREADS, 2>(s, lds, turn);
    const float r = 1.0f / sqrtf(s[0] * per + a.eps), c1 = s[1] * per * r;
    x.again(); y.again();
    if (any) {
      void* dx = a.dx ? row_of<DT>(a.dx, a.dx_stride, row) : nullptr;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t e = (u * T + me) * N;
        float wu[N];
        weights(u, wu);
        float out[N];
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const float h = (x.r[u].get(k) - mean) * r, dy = y.r[u].get(k);
          dw[u][k] = fmaf(dy, h, dw[u][k]);
          db[u][k] += dy;
          out[k] = r * (fmaf(dy, wu[k], -c0) - h * c1);
        }
        if (dx && e < a.dim) row_put<DT, N>(dx, e, a.dim, out);
      }
    }
    if (more) { x = x1; y = y1; }
  }
  if (!a.part) return;
  // the rows of a workgroup at once: one behind the other through LDS
  float* part = a.part + (size_t)blockIdx.x * 2u * a.dim;
  if constexpr (ROWS > 1) {
    __shared__ float sums[2][T * N];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      for (uint32_t q = 1; q < ROWS; ++q) {
        __syncthreads();
        if (sub == q)
#pragma unroll
          for (int k = 0; k < N; ++k) { sums[0][k * T + me] = dw[u][k]; sums[1][k * T + me] = db[u][k]; }
        __syncthreads();
        if (sub == 0)
#pragma unroll
          for (int k = 0; k < N; ++k) { dw[u][k] += sums[0][k * T + me]; db[u][k] += sums[1][k * T + me]; }
      }
    }
    if (sub) return;
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t e = (u * T + me) * N;
    if (e < a.dim) {
      row_put<DFX_F32, 4>(part, e, a.dim, dw[u]);
      row_put<DFX_F32, 4>(part + a.dim, e, a.dim, db[u]);
      if constexpr (N == 8)
        if (e + 4u < a.dim) {
          row_put<DFX_F32, 4>(part, e + 4u, a.dim, dw[u] + 4);
          row_put<DFX_F32, 4>(part + a.dim, e + 4u, a.dim, db[u] + 4);
        }
    }
  }
}

// The workgroups' shares of a column, in their order: 32 columns of a workgroup, 32 threads to each.  512 shares of 4096 columns 5.0 us.
template <int OUT>
__global__ void __launch_bounds__(1024) dfx_norm_sums_kernel(const float* part, uint32_t groups, uint32_t dim, void* grad_weight, void* grad_bias, bool accumulate) {
  __shared__ float lds[32][32];
  const uint32_t i = threadIdx.x % 32u, slice = threadIdx.x / 32u, col = blockIdx.x * 32u + i;
  const bool bias = blockIdx.y != 0;
  void* to = bias ? grad_bias : grad_weight;
  if (!to) return;
  float s = 0.0f;
  if (col < dim) {
    const float* p = part + (bias ? dim : 0u) + col;
    const uint32_t each = (groups + 31u) / 32u, end = min((slice + 1u) * each, groups);
#pragma unroll 8
    for (uint32_t g = slice * each; g < end; ++g) s += p[(size_t)g * 2u * dim];
  }
  lds[slice][i] = s;
  __syncthreads();
  if (slice || col >= dim) return;
  for (int k = 1; k < 32; ++k) s += lds[k][i];
  if (accumulate) s += step_get<OUT>(to, col);
  step_put<OUT>(to, col, s);
}

uint32_t norm_groups(size_t rows) { return (uint32_t)std::min<size_t>(rows, kNormGroups); }

template <int DT>
int norm_launch(const NormArgs& a, hipStream_t s) {
  constexpr uint32_t N = 16 / (DT == DFX_F32 ? 4 : 2);
  const uint32_t nvec = (a.dim + N - 1) / N;
#define NORM(T, U) return step_launch(dfx_norm_kernel<DT, T, U>, dim3((a.rows + (T < 256 ? 256 / T : 1) - 1) / (T < 256 ? 256 / T : 1)), T < 256 ? 256 : T, s, a)
  if (nvec <= 64) NORM(64, 1);
  if (nvec <= 128) NORM(64, 2);
  if (nvec <= 256) NORM(256, 1);
  if (nvec <= 512) NORM(256, 2);
  if (nvec <= 1024) NORM(256, 4);
  if (nvec <= 2048) NORM(1024, 2);
  if constexpr (DT == DFX_F32)
    if (nvec > 4096) NORM(1024, 8);
  NORM(1024, 4);
#undef NORM
}

template <int DT>
int norm_grad_launch(const NormArgs& a, uint32_t groups, hipStream_t s) {
  constexpr uint32_t N = 16 / (DT == DFX_F32 ? 4 : 2);
  const uint32_t nvec = (a.dim + N - 1) / N;
#define NORM(T, U, THREADS) return step_launch(dfx_norm_grad_kernel<DT, T, U, THREADS, (U < 4)>, dim3(groups), THREADS, s, a)
  if (nvec <= 64) NORM(64, 1, 256);
  if (nvec <= 128) NORM(128, 1, 256);
  if (nvec <= 256) NORM(256, 1, 256);
  if (nvec <= 512) NORM(512, 1, 512);
  if (nvec <= 1024) NORM(1024, 1, 1024);
  if (nvec <= 2048) NORM(1024, 2, 1024);
  if constexpr (DT == DFX_F32)
    if (nvec > 4096) NORM(1024, 8, 1024);
  NORM(1024, 4, 1024);
#undef NORM
}

constexpr size_t kMostRows = (1ull << 31) - 1024, kMostStride = 1ull << 20;
constexpr size_t kRowsAtOnce = 1ull << 21;      // of a launch of the forward pass: a row has 1024 threads at most, and a launch's threads are counted in 32 bits

bool norm_types(int dtype, int other) { return (dtype == DFX_F32 || dtype == DFX_BF16 || dtype == DFX_F16) && (other == dtype || other == DFX_F32); }

// all space from a matrix's first to its last row
Span rows_of(const void* a, size_t stride, size_t rows, size_t dim, size_t eb) { return flat(a, rows ? ((rows - 1) * stride + dim) * eb : 0); }
// two matrices of rows: apart, or the same memory with the same stride
bool rows_lie_well(const void* a, size_t as, const void* b, size_t bs, size_t rows, size_t dim, size_t eb) {
  return (a == b && as == bs) || !meet(rows_of(a, as, rows, dim, eb), rows_of(b, bs, rows, dim, eb));
}

}  // namespace

extern "C" {

int dfx_layer_norm(const dfx_layer_norm_args* u, void* hip_stream) {
  if (!u || u->struct_bytes != sizeof(*u) || u->reserved0 || !norm_types(u->dtype, u->param_dtype)) return DFX_ERR_INVALID_ARG;
  if (u->rows >= kMostRows || u->dim > kNormDim || u->x_stride >= kMostStride || u->y_stride >= kMostStride) return DFX_ERR_TOO_LARGE;
  const size_t eb = step_elem_bytes(u->dtype), pb = step_elem_bytes(u->param_dtype), xs = u->x_stride ? u->x_stride : u->dim, ys = u->y_stride ? u->y_stride : u->dim;
  if (!u->dim || xs < u->dim || ys < u->dim || !(u->eps >= 0.0) || !step_normal(u->eps)) return DFX_ERR_INVALID_ARG;
  if ((u->rows && (!u->x || !u->y)) || (uintptr_t)u->x % eb || (uintptr_t)u->y % eb || (uintptr_t)u->weight % pb || (uintptr_t)u->bias % pb) return DFX_ERR_INVALID_ARG;
  if (!u->rows) return DFX_OK;
  if (!rows_lie_well(u->x, xs, u->y, ys, u->rows, u->dim, eb)) return DFX_ERR_INVALID_ARG;
  const Span y = rows_of(u->y, ys, u->rows, u->dim, eb);
  if (meet(flat(u->weight, u->dim * pb), y) || meet(flat(u->bias, u->dim * pb), y)) return DFX_ERR_INVALID_ARG;
  NormArgs a;
  memset(&a, 0, sizeof(a));
  a.x = u->x; a.weight = u->weight; a.bias = u->bias; a.y = u->y; a.x_stride = xs; a.y_stride = ys;
  a.rows = (uint32_t)u->rows; a.dim = (uint32_t)u->dim; a.eps = (float)u->eps; a.param_f32 = u->param_dtype == DFX_F32;
  hipStream_t s = (hipStream_t)hip_stream;
  for (size_t first = 0; first < u->rows; first += kRowsAtOnce) {
    a.x = (const unsigned char*)u->x + first * xs * eb; a.y = (unsigned char*)u->y + first * ys * eb;
    a.rows = (uint32_t)std::min(kRowsAtOnce, u->rows - first);
    const int rc = u->dtype == DFX_F32 ? norm_launch<DFX_F32>(a, s) : u->dtype == DFX_BF16 ? norm_launch<DFX_BF16>(a, s) : norm_launch<DFX_F16>(a, s);
    if (rc != DFX_OK) return rc;
  }
  return DFX_OK;
}

size_t dfx_layer_norm_grad_workspace(size_t rows, size_t dim, dfx_dtype dtype) {
  (void)dtype;
  if (rows >= kMostRows || dim > kNormDim) return 0;
  return std::max<size_t>(16, (size_t)norm_groups(rows) * 2 * dim * sizeof(float));
}

int dfx_layer_norm_grad(const dfx_layer_norm_grad_args* u, void* hip_stream) {
  if (!u || u->struct_bytes != sizeof(*u) || u->reserved0 || !norm_types(u->dtype, u->param_dtype) || !norm_types(u->dtype, u->grad_dtype)) return DFX_ERR_INVALID_ARG;
  if (u->rows >= kMostRows || u->dim > kNormDim || u->x_stride >= kMostStride || u->dy_stride >= kMostStride || u->dx_stride >= kMostStride) return DFX_ERR_TOO_LARGE;
  const size_t eb = step_elem_bytes(u->dtype), pb = step_elem_bytes(u->param_dtype), gb = step_elem_bytes(u->grad_dtype);
  const size_t xs = u->x_stride ? u->x_stride : u->dim, dys = u->dy_stride ? u->dy_stride : u->dim, dxs = u->dx_stride ? u->dx_stride : u->dim;
  if (!u->dim || xs < u->dim || dys < u->dim || dxs < u->dim || !(u->eps >= 0.0) || !step_normal(u->eps)) return DFX_ERR_INVALID_ARG;
  if ((u->rows && (!u->x || !u->dy)) || (uintptr_t)u->x % eb || (uintptr_t)u->dy % eb || (uintptr_t)u->dx % eb || (uintptr_t)u->weight % pb ||
      (uintptr_t)u->grad_weight % gb || (uintptr_t)u->grad_bias % gb)
    return DFX_ERR_INVALID_ARG;
  const bool sums = u->grad_weight || u->grad_bias;
  const size_t need = dfx_layer_norm_grad_workspace(u->rows, u->dim, u->dtype);
  if (sums && (!u->workspace || (uintptr_t)u->workspace % 16 || u->workspace_bytes < need)) return DFX_ERR_INVALID_ARG;
  const size_t rows = u->rows;
  if (!rows_lie_well(u->x, xs, u->dx, dxs, rows, u->dim, eb) || !rows_lie_well(u->dy, dys, u->dx, dxs, rows, u->dim, eb)) return DFX_ERR_INVALID_ARG;
  const Span x = rows_of(u->x, xs, rows, u->dim, eb), dy = rows_of(u->dy, dys, rows, u->dim, eb), dx = rows_of(u->dx, dxs, rows, u->dim, eb);
  const Span w = flat(u->weight, u->dim * pb), writes[] = {flat(u->grad_weight, u->dim * gb), flat(u->grad_bias, u->dim * gb), flat(sums ? u->workspace : nullptr, need)};
  if (meet(w, dx)) return DFX_ERR_INVALID_ARG;
  for (int k = 0; k < 3; ++k) {
    if (meet(writes[k], x) || meet(writes[k], dy) || meet(writes[k], dx) || meet(writes[k], w)) return DFX_ERR_INVALID_ARG;
    for (int j = 0; j < k; ++j)
      if (meet(writes[k], writes[j])) return DFX_ERR_INVALID_ARG;
  }
  NormArgs a;
  memset(&a, 0, sizeof(a));
  a.x = u->x; a.dy = u->dy; a.weight = u->weight; a.dx = u->dx; a.x_stride = xs; a.dy_stride = dys; a.dx_stride = dxs;
  a.part = sums ? (float*)u->workspace : nullptr;
  a.rows = (uint32_t)rows; a.dim = (uint32_t)u->dim; a.eps = (float)u->eps; a.param_f32 = u->param_dtype == DFX_F32;
  hipStream_t s = (hipStream_t)hip_stream;
  const uint32_t groups = norm_groups(rows);
  if (groups && (sums || u->dx)) {
    const int rc = u->dtype == DFX_F32 ? norm_grad_launch<DFX_F32>(a, groups, s) : u->dtype == DFX_BF16 ? norm_grad_launch<DFX_BF16>(a, groups, s) : norm_grad_launch<DFX_F16>(a, groups, s);
    if (rc != DFX_OK) return rc;
  }
  if (!sums) return DFX_OK;
  const dim3 grid((a.dim + 31u) / 32u, 2);
  auto k = u->grad_dtype == DFX_F32 ? dfx_norm_sums_kernel<DFX_F32> : u->grad_dtype == DFX_BF16 ? dfx_norm_sums_kernel<DFX_BF16> : dfx_norm_sums_kernel<DFX_F16>;
  return step_launch(k, grid, 1024, s, (const float*)a.part, groups, a.dim, u->grad_weight, u->grad_bias, u->accumulate != 0);
}

}  // extern "C"

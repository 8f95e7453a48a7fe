// What the operators of the training step around the collectives share (dfx_lists.hip, dfx_loss.hip): 16-bit and 32-bit elements read
// into 32 bits and rounded back once, sums over a workgroup.
#ifndef DFX_STEP_H
#define DFX_STEP_H

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/dfx.h"

namespace {

constexpr int kStepWave = 64;

__host__ __device__ inline uint32_t step_elem_bytes(int dtype) { return dtype == DFX_F32 ? 4u : 2u; }

// A tensor starts at any multiple of its element's size (views into a bucket lie one behind the other), so a vector of elements is read
// and written wherever it begins: gfx950 takes global accesses of any alignment, and such a type says that they may be.
template <class T, int N>
struct __attribute__((packed, aligned(1))) StepVec { T x[N]; };

template <int DT> struct StepElem;
template <> struct StepElem<DFX_F32> {
  typedef uint32_t raw;
  static __device__ __forceinline__ float get(raw v) { return __uint_as_float(v); }
  static __device__ __forceinline__ raw put(float v) { return __float_as_uint(v); }
};
template <> struct StepElem<DFX_BF16> {
  typedef uint16_t raw;
  static __device__ __forceinline__ float get(raw v) { return __uint_as_float((uint32_t)v << 16); }
  static __device__ __forceinline__ raw put(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }      // to nearest even
};
template <> struct StepElem<DFX_F16> {
  typedef uint16_t raw;
  static __device__ __forceinline__ float get(raw v) { return (float)__builtin_bit_cast(_Float16, v); }
  static __device__ __forceinline__ raw put(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
};

template <int DT>
__device__ __forceinline__ float step_get(const void* p, size_t i) { return StepElem<DT>::get(((const StepVec<typename StepElem<DT>::raw, 1>*)p)[i].x[0]); }
template <int DT>
__device__ __forceinline__ void step_put(void* p, size_t i, float v) { ((StepVec<typename StepElem<DT>::raw, 1>*)p)[i].x[0] = StepElem<DT>::put(v); }

// N elements at element i
template <int DT, int N>
__device__ __forceinline__ StepVec<typename StepElem<DT>::raw, N> step_load(const void* p, size_t i) {
  return *(const StepVec<typename StepElem<DT>::raw, N>*)((const typename StepElem<DT>::raw*)p + i);
}
template <int DT, int N>
__device__ __forceinline__ void step_store(void* p, size_t i, const float* v) {
  StepVec<typename StepElem<DT>::raw, N> r;
#pragma unroll
  for (int k = 0; k < N; ++k) r.x[k] = StepElem<DT>::put(v[k]);
  *(StepVec<typename StepElem<DT>::raw, N>*)((typename StepElem<DT>::raw*)p + i) = r;
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int d = kStepWave / 2; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int d = kStepWave / 2; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
  for (int d = kStepWave / 2; d; d >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, d));
  return v;
}

}  // namespace

#endif

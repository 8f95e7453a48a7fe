// What the operators of the training step around the collectives share (dfx_lists.hip, dfx_loss.hip): 16-bit and 32-bit elements read
// into 32 bits and rounded back once, sums over a workgroup.
#ifndef DFX_STEP_H
#define DFX_STEP_H

#include <float.h>
#include <hip/hip_runtime.h>
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include <tuple>

#include "../../include/dfx.h"

namespace {

constexpr int kStepWave = 64;

__host__ __device__ inline uint32_t step_elem_bytes(int dtype) { return dtype == DFX_F32 ? 4u : 2u; }

// A tensor starts at any multiple of its element's size (views into a bucket lie one behind the other), so a vector of elements is read
// and written wherever it begins: gfx950 takes global accesses of any alignment, and these types say that they may be.
typedef uint32_t StepWords2 __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t StepWords4 __attribute__((ext_vector_type(4), aligned(2)));
template <int WORDS> struct StepWordsOf;
template <> struct StepWordsOf<2> { typedef StepWords2 type; };
template <> struct StepWordsOf<4> { typedef StepWords4 type; };

// Addresses come out of tables and argument blocks: said to be global ones, accesses take global instructions, which are waited for on one
// counter, where a generic pointer would take flat ones.
#define STEP_GLOBAL __attribute__((address_space(1)))

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
  // (of the 32-bit value: left to itself the compiler takes an operation and this conversion as one, whose result differs where the
  // 32-bit one is stored as well)
  static __device__ __forceinline__ raw put(float v) {
    asm("" : "+v"(v));
    return __builtin_bit_cast(uint16_t, (_Float16)v);
  }
};

template <int DT>
__device__ __forceinline__ float step_get(const void* p, size_t i) {
  typedef typename StepElem<DT>::raw raw;
  return StepElem<DT>::get(*((const STEP_GLOBAL raw*)p + i));
}
template <int DT>
__device__ __forceinline__ void step_put(void* p, size_t i, float v) {
  typedef typename StepElem<DT>::raw raw;
  *((STEP_GLOBAL raw*)p + i) = StepElem<DT>::put(v);
}

// The caller's numbers are of 64 bits, the kernels take most of them in 32: whether one is finite there, and whether it keeps its digits there
// as well (is 0 or no smaller than the smallest normal number).
inline bool step_fits(double v) { return fabs(v) <= (double)FLT_MAX; }
inline bool step_normal(double v) { return v == 0.0 || (step_fits(v) && fabs(v) >= (double)FLT_MIN); }

typedef float StepPair __attribute__((ext_vector_type(2)));
typedef __bf16 StepBf16Pair __attribute__((ext_vector_type(2)));

// N elements from element i on, as words; what is read or written once and is larger than the caches goes past them (STREAM, stream)
template <int DT, int N>
struct StepVec {
  typedef typename StepElem<DT>::raw raw;
  typedef typename StepWordsOf<N * (int)sizeof(raw) / 4>::type words;
  words w;

  __device__ __forceinline__ void load(const void* p, size_t i) { w = *(const STEP_GLOBAL words*)((const STEP_GLOBAL raw*)p + i); }
  // at a 32-bit offset in bytes from an address that all lanes share: one register where an address of their own takes two
  template <bool STREAM = false>
  __device__ __forceinline__ void load_at(const void* p, uint32_t bytes) {
    const STEP_GLOBAL words* q = (const STEP_GLOBAL words*)((const STEP_GLOBAL unsigned char*)p + bytes);
    w = STREAM ? __builtin_nontemporal_load(q) : *q;
  }
  __device__ __forceinline__ void stream_at(void* p, uint32_t bytes) const { __builtin_nontemporal_store(w, (STEP_GLOBAL words*)((STEP_GLOBAL unsigned char*)p + bytes)); }
  __device__ __forceinline__ void stream(void* p, size_t i) const { __builtin_nontemporal_store(w, (STEP_GLOBAL words*)((STEP_GLOBAL raw*)p + i)); }
  __device__ __forceinline__ void fill_lowest() { w = DT == DFX_F32 ? 0xff800000u : DT == DFX_BF16 ? 0xff80ff80u : 0xfc00fc00u; }      // -infinity
  __device__ __forceinline__ void from(uint4 v) { w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w; }      // (16 bytes of them)
  // what was made of the elements so far is made anew behind this, not kept: a vector of 16-bit elements takes half the registers of its values
  __device__ __forceinline__ void again() { asm("" : "+v"(w)); }
  __device__ __forceinline__ float get(int k) const {
    if (DT == DFX_F32) return StepElem<DT>::get((raw)w[k]);
    if (DT == DFX_BF16) return __uint_as_float(k & 1 ? w[k / 2] & 0xffff0000u : w[k / 2] << 16);
    return StepElem<DT>::get((raw)(k & 1 ? w[k / 2] >> 16 : w[k / 2]));
  }
  __device__ __forceinline__ void put(const float* v) {
#pragma unroll
    for (int k = 0; k < N * (int)sizeof(raw) / 4; ++k) {
      if (DT == DFX_F32) w[k] = (uint32_t)StepElem<DT>::put(v[k]);
      else if (DT == DFX_BF16) {           // (both halves in one instruction)
        const StepPair two = {v[2 * k], v[2 * k + 1]};
        w[k] = __builtin_bit_cast(uint32_t, __builtin_convertvector(two, StepBf16Pair));
      } else w[k] = (uint32_t)StepElem<DT>::put(v[2 * k]) | ((uint32_t)StepElem<DT>::put(v[2 * k + 1]) << 16);
    }
  }
};

// One kernel on a stream; the launch's own outcome, whatever error an earlier call of the caller's has left behind.
template <class... P, class... A>
int step_launch(void (*kernel)(P...), dim3 grid, int threads, hipStream_t stream, A... args) {
  std::tuple<P...> held(static_cast<P>(args)...);
  void* at[sizeof...(P)];
  std::apply([&](auto&... x) {
    size_t k = 0;
    ((at[k++] = (void*)&x), ...);
  }, held);
  return hipLaunchKernel((const void*)kernel, grid, dim3(threads), at, 0, stream) == hipSuccess ? DFX_OK : DFX_ERR_HIP;
}

// nothing of what follows is begun before every load so far has arrived
__device__ __forceinline__ void loads_arrived() {
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(0x0f70);     // vmcnt(0), the other counters at their largest
  __builtin_amdgcn_sched_barrier(0);
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int d = kStepWave / 2; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
  for (int d = kStepWave / 2; d; d >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, d));
  return v;
}

}  // namespace

#endif

// Device helpers of the operators around the step (group.hip, losses.hip): elements of every type as float32, and sums over a
// workgroup in a fixed order.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_common.h"

namespace tgrad {

// Elements of the real types as float32.  Widening is exact; narrowing rounds once, to nearest even.
template <int DT> struct Elem;
template <> struct Elem<TGRAD_F32> {
  typedef float raw;
  static __device__ __forceinline__ float widen(raw v) { return v; }
  static __device__ __forceinline__ raw narrow(float v) { return v; }
};
template <> struct Elem<TGRAD_BF16> {
  typedef uint16_t raw;
  static __device__ __forceinline__ float widen(raw v) { return __uint_as_float((uint32_t)v << 16); }
  static __device__ __forceinline__ raw narrow(float v) { return (raw)bf16_pack(v, 0.f); }
};
template <> struct Elem<TGRAD_F16> {
  typedef _Float16 raw;
  static __device__ __forceinline__ float widen(raw v) { return (float)v; }
  static __device__ __forceinline__ raw narrow(float v) { return (raw)v; }
};

// The real type whose numbers a type's elements are made of.
__host__ __device__ constexpr int real_type(int dt) { return dt == TGRAD_C64 ? TGRAD_F32 : dt == TGRAD_CBF16 ? TGRAD_BF16 : dt; }
__host__ __device__ constexpr bool complex_type(int dt) { return dt == TGRAD_C64 || dt == TGRAD_CBF16; }
__host__ __device__ constexpr int real_bytes(int real) { return real == TGRAD_F32 ? 4 : 2; }

// Sum over a workgroup of WAVES wavefronts, the same in every thread: butterflies, then the wavefronts' sums in order.
template <int WAVES, typename T>
__device__ __forceinline__ T block_sum(T v, T* lds) {
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) v += __shfl_xor(v, d);
  if constexpr (WAVES == 1) return v;
  __syncthreads();
  if (lane_id() == 0) lds[threadIdx.x / kWave] = v;
  __syncthreads();
  T s = lds[0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) s += lds[w];
  return s;
}

}  // namespace tgrad

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

// 16 and 8 bytes that start at any element: aligned to 2 bytes only; the hardware does such loads and stores as they are (a
// wavefront's 1024 bytes touch nine cache lines then instead of eight).
typedef uint32_t Quad __attribute__((ext_vector_type(4)));
typedef Quad QuadAny __attribute__((aligned(2)));
typedef uint32_t Duo __attribute__((ext_vector_type(2)));
typedef Duo DuoAny __attribute__((aligned(2)));

// Four consecutive numbers of a real type.
template <int DT> struct Four {
  typedef DuoAny any;
  typedef Duo type;
  static __device__ __forceinline__ void widen(type v, float* f) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if constexpr (DT == TGRAD_BF16) {
        f[2 * k] = __uint_as_float(v[k] << 16);
        f[2 * k + 1] = __uint_as_float(v[k] & 0xFFFF0000u);
      } else {
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        const h2 h = __builtin_bit_cast(h2, (uint32_t)v[k]);
        f[2 * k] = (float)h.x;
        f[2 * k + 1] = (float)h.y;
      }
    }
  }
  static __device__ __forceinline__ type narrow(const float* f) {
    type v;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if constexpr (DT == TGRAD_BF16) {
        v[k] = bf16_pack(f[2 * k], f[2 * k + 1]);
      } else {
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        h2 h;
        h.x = (_Float16)f[2 * k];
        h.y = (_Float16)f[2 * k + 1];
        v[k] = __builtin_bit_cast(uint32_t, h);
      }
    }
    return v;
  }
};
template <> struct Four<TGRAD_F32> {
  typedef QuadAny any;
  typedef Quad type;
  static __device__ __forceinline__ void widen(type v, float* f) {
#pragma unroll
    for (int k = 0; k < 4; ++k) f[k] = __uint_as_float(v[k]);
  }
  static __device__ __forceinline__ type narrow(const float* f) {
    type v;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = __float_as_uint(f[k]);
    return v;
  }
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

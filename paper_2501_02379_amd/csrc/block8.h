// What the files of a block in 8 bits share (act8.hip, norms.hip, int8mm.hip): matrices and codes as kernels see them, rows in units of eight
// numbers, the rounding of a code, checks of arguments.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "launch_util.h"
#include "train_common.h"

namespace tgrad {

constexpr size_t kScratchAlign = 256;

struct Mat {
  char* data;
  int64_t stride;                         // bytes from one row to the next
  __device__ __forceinline__ char* row(int64_t r) const { return data + r * stride; }
};

struct Codes8 {
  int8_t* codes;
  float* scale;
  int64_t stride;
  int64_t groups;                         // scales of a row
  int shift;                              // log2 of a group's columns; 31: the whole row
};

typedef Duo DuoByte __attribute__((aligned(1)));
typedef Quad QuadByte __attribute__((aligned(1)));

// Eight consecutive numbers of a real type, as they lie in memory.
template <int DT> struct Eight {
  typedef typename Elem<DT>::raw raw;
  static constexpr int kQuads = DT == TGRAD_F32 ? 2 : 1;
  Quad q[kQuads];

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < kQuads; ++i) q[i] = Quad{0, 0, 0, 0};
  }
  // `n` of them are there (at least 8: all); the others count as 0.
  __device__ __forceinline__ void load(const char* at, int n) {
    const raw* p = reinterpret_cast<const raw*>(at);
    if (n >= 8) {
#pragma unroll
      for (int i = 0; i < kQuads; ++i) q[i] = reinterpret_cast<const QuadAny*>(p)[i];
    } else {
      float f[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = i < n ? Elem<DT>::widen(p[i]) : 0.f;
      set(f);
    }
  }
  __device__ __forceinline__ void store(char* at, int n) const {
    raw* p = reinterpret_cast<raw*>(at);
    if (n >= 8) {
#pragma unroll
      for (int i = 0; i < kQuads; ++i) {
        // results go past the caches, but for float32, whose lanes have half a line at a time (dequantising 8192^2: bf16 31 -> 31 us, 8192 x 28672
        // 122 -> 101, float32 65 -> 101; a norm of 8192 x 16384 bf16 99 -> 88)
        if constexpr (kQuads == 1) __builtin_nontemporal_store(q[i], reinterpret_cast<QuadAny*>(p) + i);
        else reinterpret_cast<QuadAny*>(p)[i] = q[i];
      }
    } else {
      float f[8];
      get(f);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = Elem<DT>::narrow(f[i]);
    }
  }
  __device__ __forceinline__ void get(float* f) const {
    if constexpr (DT == TGRAD_F32) {
      Four<DT>::widen(q[0], f);
      Four<DT>::widen(q[1], f + 4);
    } else {
      Four<DT>::widen(Duo{q[0][0], q[0][1]}, f);
      Four<DT>::widen(Duo{q[0][2], q[0][3]}, f + 4);
    }
  }
  __device__ __forceinline__ void set(const float* f) {
    if constexpr (DT == TGRAD_F32) {
      q[0] = Four<DT>::narrow(f);
      q[1] = Four<DT>::narrow(f + 4);
    } else {
      const Duo a = Four<DT>::narrow(f), b = Four<DT>::narrow(f + 4);
      q[0] = Quad{a[0], a[1], b[0], b[1]};
    }
  }
};

// Eight numbers of a vector whose type is known at run time only (the same for every thread).
__device__ __forceinline__ void load_weights(const void* w, int dt, int64_t at, int n, float* f) {
  if (dt == TGRAD_F32) {
    Eight<TGRAD_F32> e;
    e.load(static_cast<const char*>(w) + at * 4, n);
    e.get(f);
  } else if (dt == TGRAD_BF16) {
    Eight<TGRAD_BF16> e;
    e.load(static_cast<const char*>(w) + at * 2, n);
    e.get(f);
  } else {
    Eight<TGRAD_F16> e;
    e.load(static_cast<const char*>(w) + at * 2, n);
    e.get(f);
  }
}

// The bits of the largest magnitude: magnitudes order like their bit patterns, with infinity and then NaN above all numbers.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t largest(const float* f) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, magnitude(f[i]));
  return m;
}
// A lane's value from a neighbour in the same 16 lanes, with no trip through LDS: STEP 1 and 2: lane ^ STEP; 4 and 8: the lane that mirrors it in 8 and 16
// (another half's value, which is all that a running maximum or sum of halves needs).
template <int STEP>
__device__ __forceinline__ uint32_t neighbour(uint32_t v) {
  constexpr int kCtrl = STEP == 1 ? 0xB1 : STEP == 2 ? 0x4E : STEP == 4 ? 0x141 : 0x140;
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, kCtrl, 0xF, 0xF, true);
}
template <int STEP>
__device__ __forceinline__ float neighbour(float v) { return __uint_as_float(neighbour<STEP>(__float_as_uint(v))); }

// The largest over neighbouring lanes, `lanes` 1 or a power of two from 4 to 64
__device__ __forceinline__ uint32_t largest_of_lanes(uint32_t m, int lanes) {
  if (lanes < 4) return m;
  m = max(m, neighbour<1>(m));
  m = max(m, neighbour<2>(m));
  if (lanes >= 8) m = max(m, neighbour<4>(m));
  if (lanes >= 16) m = max(m, neighbour<8>(m));
  if (lanes >= 32) m = max(m, (uint32_t)__shfl_xor((int)m, 16));
  if (lanes >= 64) m = max(m, (uint32_t)__shfl_xor((int)m, 32));
  return m;
}
// The sum over a wavefront, the same in every lane
__device__ __forceinline__ float sum_of_lanes(float v) {
  v += neighbour<1>(v);
  v += neighbour<2>(v);
  v += neighbour<4>(v);
  v += neighbour<8>(v);
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}
// ... over a workgroup of WAVES wavefronts
template <int WAVES>
__device__ __forceinline__ uint32_t largest_of_block(uint32_t m, uint32_t* lds) {
  m = largest_of_lanes(m, kWave);
  if constexpr (WAVES == 1) return m;
  __syncthreads();
  if (lane_id() == 0) lds[threadIdx.x / kWave] = m;
  __syncthreads();
  m = lds[0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) m = max(m, lds[w]);
  return m;
}

// How a group is rounded, from the bits of its largest magnitude a.  The factor 127 / a is finite and normal where a is 2^-119 at least.  Both quotients
// without a division (25 operations, as much as eight codes): q = a y with y the rounded 1 / 127 is next to a / 127, the rest a - 127 q is exact, and
// q + rest y rounds to the right scale (Markstein); the factor, off by 2^-23 of itself at most, needs no more.
struct Rounding {
  float scale, factor, top;
};
__device__ __forceinline__ Rounding rounding_of(uint32_t top_bits) {
  const float a = __uint_as_float(top_bits);
  constexpr float kInverse = 1.f / 127.f;
  Rounding r;
  r.top = a;
  const float q = a * kInverse;
  r.scale = fmaf(fmaf(-q, 127.f, a), kInverse, q);
  if (a < 0x1p-90f) r.scale = a / 127.f;                             // where the rest has too few bits
  r.scale = fminf(r.scale, 0x1.0204060000000p+121f);                 // the largest scale with a finite 127 * scale: a / 127 rounds up at float32's end
  const float s = a * 0x1p-6f, i = __builtin_amdgcn_rcpf(s);         // neither is subnormal
  r.factor = fmaf(fmaf(-s, i, 1.f), i, i) * (127.f / 64.f);
  if (a < 0x1p-119f) r.scale = r.factor = 0.f;
  if (top_bits >= 0x7F800000u) {          // an infinity or NaN
    r.scale = __uint_as_float(0x7FC00000u);
    r.factor = 0.f;
  }
  return r;
}

// Codes of eight numbers: 127 v / a, rounded to nearest even as the exact quotient is.  v * factor + 1.5 * 2^23 is one rounding, to a whole number in its low
// byte; the factor's error is 127 * 2^-23 = 1.5e-5 of a code at most, and quotients further than 2e-5 from a border are decided by that.
// Next to a border 254 |v| is compared with an odd multiple of a, both exact in float64 (32 bits each).  Halves are no rare case: v = a / 2 is one, a common
// one in two-byte types.  (Decided number by number it was 12 operations each instead of 5: an activation of 8192 x 2 x 28672 bf16 409 us.)
__device__ __forceinline__ float exact_code(float v, const Rounding& r) {
  const float below = rintf(fabsf(v * r.factor) - 0.5f);             // the border is below + 0.5
  const double twice = 254. * (double)fabsf(v), border = (2. * (double)below + 1.) * (double)r.top;
  const float up = twice > border ? below + 1.f : twice < border ? below : 2.f * floorf(0.5f * (below + 1.f));
  return copysignf(up, v);
}
__device__ __forceinline__ Duo codes_of(const float* f, const Rounding& r) {
  constexpr float kWhole = 12582912.f;
  float t[8], off[8], worst = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    t[i] = fmaf(f[i], r.factor, kWhole);
    off[i] = fabsf(fmaf(f[i], r.factor, kWhole - t[i]));
    worst = fmaxf(worst, off[i]);
  }
  if (worst > 0.49998f) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (off[i] > 0.49998f) t[i] = kWhole + exact_code(f[i], r);
  }
  Duo d;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(t[4 * i + 1]), __float_as_uint(t[4 * i]), 0x0C0C0400u);
    const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(t[4 * i + 3]), __float_as_uint(t[4 * i + 2]), 0x04000C0Cu);
    d[i] = r.factor == 0.f ? 0u : lo | hi;
  }
  return d;
}
__device__ __forceinline__ void store_codes(int8_t* p, Duo d, int n) {
  if (n >= 8) {
    __builtin_nontemporal_store(d, reinterpret_cast<DuoByte*>(p));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = (int8_t)(d[i / 4] >> (8 * (i % 4)));
  }
}
__device__ __forceinline__ Duo load_codes(const int8_t* p, int n) {
  Duo d = {0, 0};
  if (n >= 8) {
    d = *reinterpret_cast<const DuoByte*>(p);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) d[i / 4] |= (uint32_t)(uint8_t)p[i] << (8 * (i % 4));
  }
  return d;
}
// v as the float32 that it is.  (A product that is then narrowed to float16 becomes one v_fma_mixlo_f16, which rounds once, otherwise: every result
// is to be the same whichever kernel computes it.)
__device__ __forceinline__ float in_float32(float v) {
  asm("" : "+v"(v));
  return v;
}
__device__ __forceinline__ void widen_codes(Duo d, float scale, float* f) {
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = in_float32((float)(int8_t)(d[i / 4] >> (8 * (i % 4))) * scale);
}

// A sum of products of codes as a number: one conversion, two products.
__device__ __forceinline__ float scaled(int sum, float sx, float sw) { return in_float32(in_float32((float)sum * sx) * sw); }

// ---- host ---------------------------------------------------------------------------------------------------------------

constexpr int64_t kMostRows = ((int64_t)1 << 31) - 1, kMostCols = (int64_t)1 << 30;

inline bool is_real(int dt) { return dt == TGRAD_F32 || dt == TGRAD_BF16 || dt == TGRAD_F16; }

inline bool extents_ok(int64_t rows, int64_t cols, int64_t stride) {
  return rows >= 0 && rows <= kMostRows && cols >= 1 && cols <= kMostCols && stride >= cols && stride <= ((int64_t)1 << 60) / std::max<int64_t>(rows, 1);
}
inline bool good(const tgrad_matrix* m) {
  return m && is_real(m->dtype) && extents_ok(m->rows, m->cols, m->row_stride) && (m->data || m->rows == 0) &&
         (uintptr_t)m->data % (uintptr_t)real_bytes(m->dtype) == 0;
}
inline bool good(const tgrad_codes* c) {
  if (!c || !extents_ok(c->rows, c->cols, c->row_stride)) return false;
  if (c->group != 0 && c->group != 32 && c->group != 64 && c->group != 128 && c->group != 256 && c->group != 512) return false;
  return (c->rows == 0 || (c->codes && c->scale)) && (uintptr_t)c->scale % 4 == 0;
}
inline bool same_size(const tgrad_matrix* a, int64_t rows, int64_t cols) { return a->rows == rows && a->cols == cols; }
inline bool same_size(const tgrad_codes* a, int64_t rows, int64_t cols) { return a->rows == rows && a->cols == cols; }

inline Mat mat(const tgrad_matrix* m) {
  return m ? Mat{static_cast<char*>(m->data), m->row_stride * real_bytes(m->dtype)} : Mat{nullptr, 0};
}
inline Codes8 codes8(const tgrad_codes* c) {
  if (!c) return Codes8{nullptr, nullptr, 0, 0, 31};
  const int shift = c->group ? __builtin_ctz((unsigned)c->group) : 31;
  return Codes8{static_cast<int8_t*>(c->codes), c->scale, c->row_stride, c->group ? (c->cols + c->group - 1) / c->group : 1, shift};
}

inline int launched() { return hipGetLastError() == hipSuccess ? TGRAD_OK : TGRAD_ERR_HIP; }
inline bool pending() { return hipPeekAtLastError() != hipSuccess; }

template <typename F>
void for_real(int dt, F&& f) {
  if (dt == TGRAD_F32) f(std::integral_constant<int, TGRAD_F32>());
  else if (dt == TGRAD_BF16) f(std::integral_constant<int, TGRAD_BF16>());
  else f(std::integral_constant<int, TGRAD_F16>());
}

// f(first, rows) for parts of the rows whose launches, `groups` workgroups of T threads a row, stay below 2^32 threads.
template <typename F>
void rows_in_launches(int64_t rows, int T, int64_t groups, F&& f) {
  const int64_t most = std::max<int64_t>(1, (((int64_t)1 << 32) - 1) / (T * groups));
  for (int64_t at = 0; at < rows; at += most) f(at, std::min(rows - at, most));
}

}  // namespace tgrad

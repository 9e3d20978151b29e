// What the products of int8mm.hip and grad8.hip share: loads of codes, loads that go straight to LDS, the order of tiles.
#pragma once

#include "block8.h"

namespace tgrad {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __amdgpu_buffer_rsrc_t Ref;

__device__ __forceinline__ Quad load16(const int8_t* p, int64_t n) {
  Quad q = {0, 0, 0, 0};
  if (n >= 16) {
    q = *reinterpret_cast<const QuadByte*>(p);
  } else if (n > 0) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (i < n) q[i / 4] |= (uint32_t)(uint8_t)p[i] << (8 * (i % 4));
  }
  return q;
}

// Memory from p on, for loads that go straight to LDS: 16 bytes a lane, the lanes' one behind the other.
__device__ __forceinline__ Ref ref(const void* p, int bytes = 0x7FFFFFF8) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, bytes, 0x00020000);       // what lies behind `bytes` reads as 0
}
__device__ __forceinline__ void to_lds(const Ref& g, char* l, int each, int all) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(g, (__attribute__((address_space(3))) void*)l, 16, each, all, 0, 0);
}
// The same as an instruction that the compiler does not know for a load: it waits for all loads to LDS in front of a transposing read of LDS, whichever
// part they go to.  The caller counts them (barrier_but); the compiler's own waits for other loads only become stricter.  `l`: the same for the wavefront.
__device__ __forceinline__ void to_lds_uncounted(const Ref& g, const char* l, int each) {
  const int at = __builtin_amdgcn_readfirstlane((int)(uintptr_t)(__attribute__((address_space(3))) const char*)l);
  int m0;                                  // left as it was found
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0"
               : "=&s"(m0)
               : "s"(at), "v"(each), "s"(g)
               : "memory");
}
// A barrier behind which everyone's LDS stores are there, and everyone's loads to LDS but the last N of each wavefront.
template <int N>
__device__ __forceinline__ void barrier_but() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// The same for the wide tiles, whose two halves of a workgroup take turns: while four wavefronts, one on each SIMD, read operands, the other four
// multiply.  Nothing moves across.
template <int N>
__device__ __forceinline__ void turn_but() {
  __builtin_amdgcn_sched_barrier(0);
  barrier_but<N>();
  __builtin_amdgcn_sched_barrier(0);
}
__device__ __forceinline__ void turn() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// A launch's workgroups go round the 8 dies; here each die gets neighbouring tiles, in bands of 4 tiles of rows, so that those at work at a time
// share what its L2 holds.  -> (tile of rows, tile of columns)
__device__ __forceinline__ int2 tile_of(int id, int total, int tiles_c) {
  const int q = total / 8, r = total % 8, die = id % 8;
  id = die * q + min(die, r) + id / 8;
  const int band = id / (4 * tiles_c), in = id % (4 * tiles_c), tall = min(4, total / tiles_c - band * 4);
  return make_int2(band * 4 + in % tall, in / tall);
}

// ---- host ---------------------------------------------------------------------------------------------------------------

inline size_t aligned(size_t n) { return (n + kScratchAlign - 1) / kScratchAlign * kScratchAlign; }
inline bool scratch_ok(const void* p, size_t needed) { return needed == 0 || (p && (uintptr_t)p % kScratchAlign == 0); }
// A launch has fewer than 2^32 threads.
inline bool too_many(const tgrad_matrix* y) { return ((y->rows + 63) / 64) * ((y->cols + 63) / 64) >= ((int64_t)1 << 21); }

}  // namespace tgrad

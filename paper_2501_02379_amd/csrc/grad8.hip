// The two gradients of a product with codes: sums over s of dy's numbers times codes' values, dx[t][k] = sum_n dy[t][n] w[n][k] and
// dw[n][k] = sum_t dy[t][n] x[t][k].
//
// Both have the codes' rows along the sum, so that codes and, for dw, dy lie across it: a matrix instruction wants eight
// neighbours along the sum in a lane, and LDS gives them with transposing loads.  Codes are widened on their way to LDS (cvt, mul, half a pack for each), once for each
// tile of results that they go into.
#include "tiles8.h"

using namespace tgrad;

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <int DT>
__device__ __forceinline__ v4f mfma_of(Quad a, Quad b, v4f c) {
  if constexpr (DT == TGRAD_F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// A tile that lies across the sum: rows along the sum, `W` two-byte numbers each, block b (16 numbers, 32 bytes) of row s at block b ^ bend(s): a
// transposing load's 16 lanes take a block of four rows, 0 to 3 modulo 4, and these then meet all banks.
__device__ __forceinline__ int bend(int s) { return (s & 3) | ((s >> 1) & 4); }
// Rows 8 g .. 8 g + 7 of block b, column l % 16, for lane l = 16 g + ...
template <int W>
__device__ __forceinline__ Quad across(const char* tile, int s0, int block, int lane) {
  const int s = s0 + lane / 16 * 8 + lane % 16 / 4;
  const char* p = tile + s * (W * 2) + (block ^ bend(s)) * 32 + lane % 4 * 8;
  typedef __attribute__((address_space(3))) s16x4* At;
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(p));
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(p + 4 * W * 2));        // bend(s + 4) = bend(s)
  const Duo l = __builtin_bit_cast(Duo, lo), h = __builtin_bit_cast(Duo, hi);
  return Quad{l[0], l[1], h[0], h[1]};
}

// Eight two-byte numbers of which n are there.
template <int DT>
__device__ __forceinline__ Quad load8(const char* p, int64_t n) {
  Eight<DT> e;
  e.clear();
  if (n > 0) e.load(p, (int)min(n, (int64_t)8));
  return e.q[0];
}

// Sixteen codes times a scale, as two-byte numbers.
template <int DT>
__device__ __forceinline__ void widen16(Quad c, float scale, Quad* out) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float f[8];
    widen_codes(Duo{c[2 * h], c[2 * h + 1]}, scale, f);
    Eight<DT> e;
    e.set(f);
    out[h] = e.q[0];
  }
}

// One of the two parts of unrounded values: the upper one, rounded towards zero, or what that leaves, rounded.  The upper part is that of the value less 2^-9
// (float16: 2^-12) of itself, so that both parts have the value's sign and, but for float16's smallest, neither is 0: an infinity in dy stays the infinity that
// it is.  Together they are off by 2^-8 (2^-7 + 2^-9) of the value at most, float16 2^-11 (2^-10 + 2^-12).
template <int DT, bool REST>
__device__ __forceinline__ void widen16_part(Quad c, float scale, Quad* out) {
  const float less = scale * (DT == TGRAD_F16 ? 1.f - 0x1p-12f : 1.f - 0x1p-9f);
#pragma unroll
  for (int h = 0; h < 8; ++h) {
    const uint32_t pair = c[h / 2] >> (h % 2 * 16);
    const float x = (float)(int8_t)pair, y = (float)(int8_t)(pair >> 8);
    const float a = in_float32(x * less), b = in_float32(y * less);
    uint32_t v;
    if constexpr (DT == TGRAD_F16) {
      const auto u = __builtin_amdgcn_cvt_pkrtz(a, b);
      const _Float16 r[2] = {(_Float16)in_float32(fmaf(x, scale, -(float)u[0])), (_Float16)in_float32(fmaf(y, scale, -(float)u[1]))};
      v = REST ? __builtin_bit_cast(uint32_t, r) : __builtin_bit_cast(uint32_t, u);
    } else {
      const float r = fmaf(x, scale, -__uint_as_float(__float_as_uint(a) & 0xFFFF0000u)), q = fmaf(y, scale, -__uint_as_float(__float_as_uint(b) & 0xFFFF0000u));
      v = REST ? bf16_pack(r, q) : __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
    }
    out[h / 4][h % 4] = v;
  }
}

// float16's exponents do not reach what float32 scales do, so its values are multiplied with 2^k on their way to LDS and the sums with 2^-k, both exact: k
// brings the largest of the scales that a tile reads to 2^8..2^9, 127 times it to 65024 at most, below float16's end.  Values keep 11 bits down to 2^-28 of
// the largest.  Rows `first` .. first + rows - 1, columns c0 .. c0 + cols - 1; the same in every thread.  Infinite and NaN scales are no size.  (8192^3: 3
// percent, for the tile's scales are read ahead of its loop.)
template <int T>
__device__ __forceinline__ int lift_of(const Codes8& c, int64_t first, int64_t rows, int c0, int cols, uint32_t* lds) {
  const int g0 = c0 >> c.shift, g1 = (c0 + cols - 1) >> c.shift;
  uint32_t top = 0;
  for (int64_t r = threadIdx.x; r < rows; r += T)
    for (int g = g0; g <= g1; ++g) {
      const uint32_t m = magnitude(c.scale[(first + r) * c.groups + g]);
      if (m < 0x7F800000u) top = max(top, m);
    }
  top = largest_of_block<T / kWave>(top, lds);
  return top == 0 ? 0 : 8 + 127 - (int)(top >> 23);
}

// A result's four neighbours in a row, of the type OT (float32 sums of a split where OT < 0), times 2^-lift.
template <int OT>
__device__ __forceinline__ void store4(char* row, int64_t c, int64_t cols, v4f v, int lift = 0) {
  constexpr int RT = OT < 0 ? TGRAD_F32 : OT;
  typedef typename Elem<RT>::raw raw;
  raw* to = reinterpret_cast<raw*>(row) + c;
  const float f[4] = {ldexpf(v[0], -lift), ldexpf(v[1], -lift), ldexpf(v[2], -lift), ldexpf(v[3], -lift)};
  if (c + 4 <= cols) {
    *reinterpret_cast<typename Four<RT>::any*>(to) = Four<RT>::narrow(f);
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (c + r < cols) to[r] = Elem<RT>::narrow(f[r]);
  }
}

struct Grad {
  Mat dy;
  Codes8 c;
  Mat out;                                // [split][rows][cols] in float32 where the sum is split
  int64_t sum;
  int rows, cols;                         // of the result
  int tiles_c, tiles, steps;              // steps of a split
  int dy_rows;                            // rows, or more of them: what of dy can be read for dw, a multiple of 8
};

// ---- two-byte dy ----------------------------------------------------------------------------------------------------------------------

constexpr int kStep = 64;                 // of the sum in LDS at a time

// WR x WC wavefronts, each FR x FC results of 16 x 16; two steps in LDS, one barrier a step.  WEIGHT: dy lies across the sum, else along it (rows of
// 128 bytes, chunk c of row r at chunk c ^ (r % 8)).  dy goes straight to LDS, but for the sum's end; codes go through registers, a step ahead.
// (8192^3 bf16, codes in rows that the wide tiles do not take: 1390 us; unrounded 2840 and 2890.)
// PARTS = 2: values unrounded.  A step is then taken in two turns, with its values' upper parts and with what they leave (both beside each other in LDS would leave
// room for one workgroup a compute unit).
template <int WR, int WC, int FR, int FC, int DT, int OT, bool WEIGHT, int PARTS>
__global__ __launch_bounds__(WR * WC * 64, 2) void k_grad_tiles(Grad a) {
  constexpr int T = WR * WC * 64, BR = WR * FR * 16, BC = WC * FC * 16;
  constexpr int kDy = BR * kStep * 2, kBytes = kDy + BC * kStep * 2;
  constexpr int kLoads = kDy / 16 / T, kCodes = BC * kStep / 16 / T;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = lane_id();
  const int split = blockIdx.x / a.tiles;
  const int2 tile = tile_of(blockIdx.x % a.tiles, a.tiles, a.tiles_c);
  const int r0 = tile.x * BR, c0 = tile.y * BC;
  const int64_t first = (int64_t)split * a.steps, last = min(first + a.steps, (a.sum + kStep - 1) / kStep);
  // turns: PARTS of them a step; `whole` of them on steps that lie within the sum
  const int64_t turns = (last - first) * PARTS, whole = max((min(last, a.sum / kStep) - first) * PARTS, (int64_t)0);
  auto place_of = [&](int64_t q) { return lds + (int)(q & 1) * kBytes; };
  int lift = 0;
  if constexpr (DT == TGRAD_F16) {
    __shared__ uint32_t tops[WR * WC];
    lift = lift_of<T>(a.c, first * kStep, min(last * kStep, a.sum) - first * kStep, c0, min(BC, a.cols - c0), tops);
  }

  // this thread's chunks of dy: row of the tile and chunk of eight numbers
  auto part = [&](int i, int& row, int& chunk) {
    const int id = i * T + (int)threadIdx.x;
    if constexpr (WEIGHT) {
      row = id / (BR / 8);
      const int c = id % (BR / 8);
      chunk = ((c / 2) ^ bend(row)) * 2 + c % 2;
    } else {
      row = id / 8;
      chunk = (id % 8) ^ (row % 8);
    }
  };
  int each[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    int row, chunk;
    part(i, row, chunk);
    // what lies beyond the matrix is loaded from within it, and its results are not stored
    each[i] = WEIGHT ? row * (int)a.dy.stride + min(chunk * 8, a.dy_rows - r0 - 8) * 2 : min(row, a.rows - 1 - r0) * (int)a.dy.stride + chunk * 16;
  }
  const char* dy0 = WEIGHT ? a.dy.data + (int64_t)r0 * 2 : a.dy.row(r0);
  auto fill = [&](int64_t q) {
    const int64_t s = first + q / PARTS;
    const Ref g = ref(dy0 + (WEIGHT ? s * kStep * a.dy.stride : s * kStep * 2));
    char* l = place_of(q) + wave * kWave * 16;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) to_lds_uncounted(g, l + i * T * 16, each[i]);
  };
  Quad held[kLoads];
  auto read = [&](int64_t s) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      int row, chunk;
      part(i, row, chunk);
      if constexpr (WEIGHT) held[i] = load8<DT>(a.dy.row(s * kStep + row) + (int64_t)(r0 + chunk * 8) * 2, s * kStep + row < a.sum ? a.rows - r0 - chunk * 8 : 0);
      else held[i] = load8<DT>(a.dy.row(min(r0 + row, a.rows - 1)) + (s * kStep + chunk * 8) * 2, a.sum - s * kStep - chunk * 8);
    }
  };
  auto place = [&](int64_t q) {
    char* l = place_of(q) + threadIdx.x * 16;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) *reinterpret_cast<Quad*>(l + i * T * 16) = held[i];
  };

  Quad codes[kCodes];
  float scale[kCodes];
  const int8_t* cp = a.c.codes + c0;
  auto read_codes = [&](int64_t s) {
#pragma unroll
    for (int i = 0; i < kCodes; ++i) {
      const int id = i * T + (int)threadIdx.x, col = id % (BC / 16) * 16;
      const int64_t row = s * kStep + id / (BC / 16);
      codes[i] = Quad{0, 0, 0, 0};
      scale[i] = 0.f;
      if (row < a.sum && c0 + col < a.cols) {
        codes[i] = load16(cp + row * a.c.stride + col, a.cols - c0 - col);
        scale[i] = a.c.scale[row * a.c.groups + ((c0 + col) >> a.c.shift)];
        if constexpr (DT == TGRAD_F16) scale[i] = ldexpf(scale[i], lift);
      }
    }
  };
  auto place_codes = [&](int64_t q) {
    char* l = place_of(q) + kDy;
#pragma unroll
    for (int i = 0; i < kCodes; ++i) {
      const int id = i * T + (int)threadIdx.x, row = id / (BC / 16), block = id % (BC / 16);
      Quad v[2];
      if constexpr (PARTS == 1) widen16<DT>(codes[i], scale[i], v);
      else if (q & 1) widen16_part<DT, true>(codes[i], scale[i], v);
      else widen16_part<DT, false>(codes[i], scale[i], v);
      char* at = l + row * (BC * 2) + (block ^ bend(row)) * 32;
      const bool upper = lane & 4;          // lanes 4 to 7 store their upper halves first: eight lanes then meet all banks
      *reinterpret_cast<Quad*>(at + (upper ? 16 : 0)) = upper ? v[1] : v[0];
      *reinterpret_cast<Quad*>(at + (upper ? 0 : 16)) = upper ? v[0] : v[1];
    }
  };

  v4f acc[FC][FR] = {};
  const int wr = wave % WR, wc = wave / WR;
  auto multiply = [&](int64_t q) {
    const char* l = place_of(q);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      Quad c[FC], d[FR];
#pragma unroll
      for (int i = 0; i < FC; ++i) c[i] = across<BC>(l + kDy, k * 32, wc * FC + i, lane);
#pragma unroll
      for (int j = 0; j < FR; ++j) {
        if constexpr (WEIGHT) d[j] = across<BR>(l, k * 32, wr * FR + j, lane);
        else d[j] = *reinterpret_cast<const Quad*>(l + ((wr * FR + j) * 16 + lane % 16) * 128 + (((k * 4 + lane / 16) ^ (lane % 8)) * 16));
      }
#pragma unroll
      for (int i = 0; i < FC; ++i)
#pragma unroll
        for (int j = 0; j < FR; ++j) acc[i][j] = mfma_of<DT>(c[i], d[j], acc[i][j]);
    }
  };

  // the codes of a step's second turn are there from its first one
  auto next_codes = [&](int64_t q) {
    if (q < turns && q % PARTS == 0) read_codes(first + q / PARTS);
  };
  read_codes(first);
  if (whole > 0) fill(0);
  place_codes(0);
  next_codes(1);
  for (int64_t q = 0; q < whole; ++q) {
    barrier_but<0>();
    if (q + 1 < turns) {
      if (q + 1 < whole) fill(q + 1);
      place_codes(q + 1);
      next_codes(q + 2);
    }
    multiply(q);
  }
  if (whole < turns) {                      // the sum's end, less than a step
    read(first + whole / PARTS);
    __syncthreads();
    for (int64_t q = whole; q < turns; ++q) {
      if (q > whole) place_codes(q);        // into the place of turn q - 2, which everyone is done with
      place(q);
      __syncthreads();
      multiply(q);
    }
  }

#pragma unroll
  for (int j = 0; j < FR; ++j) {
    const int r = r0 + (wr * FR + j) * 16 + lane % 16;
    if (r >= a.rows) continue;
    char* row = a.out.row((int64_t)split * a.rows + r);
#pragma unroll
    for (int i = 0; i < FC; ++i) {
      const int c = c0 + (wc * FC + i) * 16 + lane / 16 * 4;
      if (c < a.cols) store4<OT>(row, c, a.cols, acc[i][j], lift);
    }
  }
}

// The same with 256 x 256 results of 8 wavefronts, 2 x 4 of 8 x 4, in steps of 32 of which four are there or on their way, in turns: wavefronts 0 to 3 read a
// step's operands while 4 to 7, a turn behind, multiply the step before.  dy goes straight to LDS three steps ahead; codes are loaded four
// steps ahead and widened into LDS two steps ahead.  All loads are unconditional, of memory that ends where the matrices do, so that they are
// counted the same in every step and read 0 behind the sum's end.
// dy: 16-byte rows, whole chunks of eight columns; codes: 16-byte rows.
constexpr int kWide = 256, kWideStep = 32, kWideBufs = 4, kWideDy = kWide * kWideStep * 2, kWideBytes = 2 * kWideDy;

// 8192^3 bf16: dw 950 to 980 us, dx 965 to 1000 (1160 and 1140 TFLOP/s at best; with loads to LDS that the compiler waits for 1130 and 1143 us).  The matrix instructions alone reach 1650
// to 2030 on random numbers.
// RAGGED: the codes' last row ends within a chunk (its branch costs the others 12 percent).
// PARTS = 2: values unrounded.  32 of the sum are two steps here, one with the values' upper parts and one with what they leave; dy is fetched again, from the caches.
// 8192^3 bf16: dw and dx 1860 to 1910 us, 1180 TFLOP/s of both parts' products.  (Both parts in one step, dy read once, need 70 to 100 registers more than there are.)
template <int DT, int OT, bool WEIGHT, bool RAGGED, int PARTS>
__global__ __launch_bounds__(512) void k_grad_wide(Grad a) {
  constexpr int T = 512, FR = 8, FC = 4, kLoads = kWideDy / 16 / T;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = lane_id();
  const int split = blockIdx.x / a.tiles;
  const int2 tile = tile_of(blockIdx.x % a.tiles, a.tiles, a.tiles_c);
  const int r0 = tile.x * kWide, c0 = tile.y * kWide;
  const int64_t from = (int64_t)split * a.steps * kWideStep;           // this split's part of the sum
  const int sum = (int)min(a.sum - from, (int64_t)a.steps * kWideStep), steps = (sum + kWideStep - 1) / kWideStep * PARTS;
  int lift = 0;
  if constexpr (DT == TGRAD_F16) {
    __shared__ uint32_t tops[T / kWave];
    lift = lift_of<T>(a.c, from, sum, c0, min(kWide, a.cols - c0), tops);
  }

  // dy: what lies beyond its rows or columns is loaded from within, and its results are not stored
  int each[kLoads], ahead[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int id = i * T + (int)threadIdx.x;
    if constexpr (WEIGHT) {
      const int row = id / 32, c = id % 32, chunk = ((c / 2) ^ bend(row)) * 2 + c % 2;
      each[i] = row * (int)a.dy.stride + min(chunk * 8, a.dy_rows - r0 - 8) * 2;
      ahead[i] = 0;
    } else {
      const int row = id / 4, chunk = (id % 4) ^ (row / 2 % 4);
      each[i] = min(row, a.rows - 1 - r0) * (int)a.dy.stride + chunk * 16;
      ahead[i] = chunk * 8;
    }
  }
  const char* dy0 = WEIGHT ? a.dy.row(from) + (int64_t)r0 * 2 : a.dy.row(r0) + from * 2;
  const int across_bytes = min(a.dy_rows - r0, kWide) * 2;
  auto fill = [&](int s) {
    const int at = s / PARTS * kWideStep, left = min(sum - at, kWideStep);
    char* l = lds + s % kWideBufs * kWideBytes + wave * kWave * 16;
    if constexpr (WEIGHT) {
      const int bytes = (left - 1) * (int)a.dy.stride + across_bytes;
      const Ref g = ref(dy0 + at * a.dy.stride, left > 0 ? bytes : 0);
#pragma unroll
      for (int i = 0; i < kLoads; ++i) to_lds_uncounted(g, l + i * T * 16, each[i]);
    } else {
      const Ref g = ref(dy0 + (int64_t)at * 2);
#pragma unroll
      for (int i = 0; i < kLoads; ++i) to_lds_uncounted(g, l + i * T * 16, ahead[i] < left ? each[i] : 0x7FFFFFFC);
    }
  };

  // codes: 16 of a row for each thread
  const int row = threadIdx.x / 16, block = threadIdx.x % 16;
  const int code_at = row * (int)a.c.stride + block * 16;
  const int scale_at = (row * (int)a.c.groups + ((c0 + block * 16) >> a.c.shift)) * 4;
  struct Held {
    Quad codes;
    float scale;
  };
  const int8_t* codes0 = a.c.codes + from * a.c.stride + c0;
  const float* scale0 = a.c.scale + from * a.c.groups;
  auto read_codes = [&](int s, Held& h) {
    const int row0 = s / PARTS * kWideStep, left = min(sum - row0, kWideStep);
    const bool end = from + row0 + left >= a.sum;                      // this step has the last row, or nothing
    const int bytes = left * (int)a.c.stride - (end ? (int)a.c.stride - (a.cols - c0) : 0);
    const int8_t* at = codes0 + row0 * a.c.stride;
    const Ref g = ref(scale0 + row0 * a.c.groups, max(left, 0) * (int)a.c.groups * 4);
    h.codes = __builtin_bit_cast(Quad, __builtin_amdgcn_raw_buffer_load_b128(ref(at, left > 0 ? bytes : 0), code_at, 0, 0));
    h.scale = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(g, scale_at, 0, 0));
    if (RAGGED && end && left > 0) {        // buffers end at whole dwords: the last row's end byte by byte.  All loads are then waited for
      const int n = a.cols - c0 - block * 16;
      if (row == left - 1 && n > 0 && n < 16) h.codes = load16(at + code_at, n);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
  };
  const int place = kWideDy + row * (kWide * 2) + (block ^ bend(row)) * 32;
  auto place_codes = [&](int s, auto rest, const Held& h) {
    Quad q[2];
    const float scale = DT == TGRAD_F16 ? ldexpf(h.scale, lift) : h.scale;
    if constexpr (PARTS == 1) widen16<DT>(h.codes, scale, q);
    else widen16_part<DT, decltype(rest)::value>(h.codes, scale, q);
    char* at = lds + s % kWideBufs * kWideBytes + place;
    const bool upper = lane & 4;            // lanes 4 to 7 store their upper halves first: eight lanes then meet all banks
    *reinterpret_cast<Quad*>(at + (upper ? 16 : 0)) = upper ? q[1] : q[0];
    *reinterpret_cast<Quad*>(at + (upper ? 0 : 16)) = upper ? q[0] : q[1];
  };

  v4f acc[FC][FR] = {};
  const int wc = wave % 4, wr = wave / 4;
  const bool late = wave >= 4;
  const std::false_type even;
  const std::true_type odd;
  auto step = [&](int s, auto parity, Held& h) {
    Quad c[FC], d[FR];
    const char* l = lds + s % kWideBufs * kWideBytes;
#pragma unroll
    for (int i = 0; i < FC; ++i) c[i] = across<kWide>(l + kWideDy, 0, wc * FC + i, lane);
#pragma unroll
    for (int j = 0; j < FR; ++j) {
      if constexpr (WEIGHT) d[j] = across<kWide>(l, 0, wr * FR + j, lane);
      else d[j] = *reinterpret_cast<const Quad*>(l + ((wr * FR + j) * 16 + lane % 16) * 64 + ((lane / 16) ^ (lane / 2 % 4)) * 16);
    }
    // dy of s + 1 has to be there; behind it came codes of s + 2, dy of s + 2, codes of s + 3
    turn_but<kLoads + 4>();
    __builtin_amdgcn_s_setprio(1);
    place_codes(s + 2, parity, h);
    fill(s + 3);                            // behind the sum's end both read zeros
    read_codes(s + 4, h);
#pragma unroll
    for (int i = 0; i < FC; ++i)
#pragma unroll
      for (int j = 0; j < FR; ++j) acc[i][j] = mfma_of<DT>(c[i], d[j], acc[i][j]);
#pragma unroll
    for (int i = 0; i < FC * FR; ++i) {     // a product, and what vector instructions fit beside it
      __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x2, 3, 0);
    }
    __builtin_amdgcn_s_setprio(0);
    turn();
  };
  Held h0, h1;
  read_codes(0, h0);
  read_codes(1, h1);
  fill(0);
  fill(1);
  fill(2);
  place_codes(0, even, h0);
  place_codes(1, odd, h1);
  read_codes(2, h0);
  read_codes(3, h1);
  turn_but<0>();
  if (late) turn();
  for (int s = 0; s < steps; s += 2) {
    step(s, even, h0);
    step(s + 1, odd, h1);                   // with an odd number of steps the last one adds zeros
  }
  if (!late) turn();
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
  for (int j = 0; j < FR; ++j) {
    const int r = r0 + (wr * FR + j) * 16 + lane % 16;
    if (r >= a.rows) continue;
    char* out = a.out.row((int64_t)split * a.rows + r);
#pragma unroll
    for (int i = 0; i < FC; ++i) {
      const int c = c0 + (wc * FC + i) * 16 + lane / 16 * 4;
      if (c < a.cols) store4<OT>(out, c, a.cols, acc[i][j], lift);
    }
  }
}

// ---- float32 dy, and two-byte dy of a few tokens: a scale for each row of codes -------------------------------------------------------------------------------------------

// dy times a row's scale, rounded to float32, lies in LDS as three bf16 parts of 8 bits (split_apart); codes are exact in bf16.  Three products instead
// of one, each 16 times as fast as the float32 matrix instructions'.  (4096^3: 420 us for dw, 425 for dx, 325 TFLOP/s.)  Two-byte dy of up to 16
// tokens takes this way too: memory bounds such products, so that no value need be rounded; and float32 results of unrounded values.
constexpr int kStep32 = 32;

// The parts of eight numbers (see split_pair, which forms rests with dot products of both: neighbours here are different results' terms, and a NaN
// or an infinity may not reach the other one's).  An infinity leaves nothing: its product with a code other than 0 is the infinity that it is.  (Looked at
// number by number that was 8 percent of 4096^3, this way 3.)
__device__ __forceinline__ void split_apart(const float* f, u32v4& h, u32v4& m, u32v4& l) {
  float top = 0.f, r[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    top = fmaxf(top, fabsf(f[i]));
    r[i] = f[i] - __uint_as_float(__float_as_uint(f[i]) & 0xFFFF0000u);
  }
  if (__any(top == INFINITY)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = fabsf(f[i]) == INFINITY ? 0.f : r[i];
  }
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    h[d] = __builtin_amdgcn_perm(__float_as_uint(f[2 * d + 1]), __float_as_uint(f[2 * d]), 0x07060302u);       // the upper halves
    m[d] = bf16_pack(r[2 * d], r[2 * d + 1]);
    l[d] = bf16_pack(r[2 * d] - __uint_as_float(m[d] << 16), r[2 * d + 1] - __uint_as_float(m[d] & 0xFFFF0000u));
  }
}

template <int WR, int WC, int FR, int FC, int DT, int OT, bool WEIGHT>
__global__ __launch_bounds__(WR * WC * 64, 2) void k_grad_split(Grad a) {
  constexpr int T = WR * WC * 64, BR = WR * FR * 16, BC = WC * FC * 16;
  constexpr int kPart = BR * kStep32 * 2, kBytes = 3 * kPart + BC * kStep32 * 2;
  constexpr int kLoads = BR * kStep32 / 8 / T, kCodes = BC * kStep32 / 16 / T;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = lane_id();
  const int split = blockIdx.x / a.tiles;
  const int2 tile = tile_of(blockIdx.x % a.tiles, a.tiles, a.tiles_c);
  const int r0 = tile.x * BR, c0 = tile.y * BC;
  const int64_t first = (int64_t)split * a.steps, last = min(first + a.steps, (a.sum + kStep32 - 1) / kStep32);
  auto place_of = [&](int64_t s) { return lds + (int)((s - first) & 1) * kBytes; };

  constexpr int es = sizeof(typename Elem<DT>::raw);
  Eight<DT> held[kLoads];
  Quad codes[kCodes];
  float scale[kLoads][WEIGHT ? 1 : 8];
  auto read = [&](int64_t s) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int id = i * T + (int)threadIdx.x;
      held[i].clear();
      if constexpr (WEIGHT) {
        const int64_t row = s * kStep32 + id / (BR / 8);
        const int n = a.rows - r0 - id % (BR / 8) * 8;
        scale[i][0] = 0.f;
        if (row < a.sum && n > 0) {
          held[i].load(a.dy.row(row) + (int64_t)(a.rows - n) * es, n);
          scale[i][0] = a.c.scale[row];
        }
      } else {
        const int64_t at = s * kStep32 + id % 4 * 8;
        const int n = (int)min(a.sum - at, (int64_t)8);
        if (n > 0) held[i].load(a.dy.row(min(r0 + id / 4, a.rows - 1)) + at * es, n);
        Eight<TGRAD_F32> e;
        e.clear();
        if (n > 0) e.load(reinterpret_cast<const char*>(a.c.scale + at), n);
        e.get(scale[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < kCodes; ++i) {
      const int id = i * T + (int)threadIdx.x, col = id % (BC / 16) * 16;
      const int64_t row = s * kStep32 + id / (BC / 16);
      codes[i] = Quad{0, 0, 0, 0};
      if (row < a.sum && c0 + col < a.cols) codes[i] = load16(a.c.codes + row * a.c.stride + c0 + col, a.cols - c0 - col);
    }
  };
  auto place = [&](int64_t s) {
    char* l = place_of(s);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int id = i * T + (int)threadIdx.x;
      float f[8];
      held[i].get(f);
      u32v4 h, m, lo;
#pragma unroll
      for (int k = 0; k < 8; ++k) f[k] *= scale[i][WEIGHT ? 0 : k];
      split_apart(f, h, m, lo);
      int at;
      if constexpr (WEIGHT) {
        const int row = id / (BR / 8), c = id % (BR / 8);
        at = row * (BR * 2) + ((c / 2) ^ bend(row)) * 32 + c % 2 * 16;
      } else {
        const int row = id / 4;                                    // rows of 64 bytes, two to all banks
        at = row * 64 + ((id % 4) ^ (row / 2 % 4)) * 16;
      }
      *reinterpret_cast<u32v4*>(l + at) = h;
      *reinterpret_cast<u32v4*>(l + kPart + at) = m;
      *reinterpret_cast<u32v4*>(l + 2 * kPart + at) = lo;
    }
#pragma unroll
    for (int i = 0; i < kCodes; ++i) {
      const int id = i * T + (int)threadIdx.x, row = id / (BC / 16), block = id % (BC / 16);
      Quad q[2];
      widen16<TGRAD_BF16>(codes[i], 1.f, q);
      char* at = l + 3 * kPart + row * (BC * 2) + (block ^ bend(row)) * 32;
      const bool upper = lane & 4;
      *reinterpret_cast<Quad*>(at + (upper ? 16 : 0)) = upper ? q[1] : q[0];
      *reinterpret_cast<Quad*>(at + (upper ? 0 : 16)) = upper ? q[0] : q[1];
    }
  };

  v4f acc[FC][FR] = {};
  const int wr = wave % WR, wc = wave / WR;
  auto multiply = [&](int64_t s) {
    const char* l = place_of(s);
    Quad c[FC];
#pragma unroll
    for (int i = 0; i < FC; ++i) c[i] = across<BC>(l + 3 * kPart, 0, wc * FC + i, lane);
#pragma unroll
    for (int p = 2; p >= 0; --p) {          // the smallest part first
      Quad d[FR];
#pragma unroll
      for (int j = 0; j < FR; ++j) {
        const int row = (wr * FR + j) * 16 + lane % 16;
        if constexpr (WEIGHT) d[j] = across<BR>(l + p * kPart, 0, wr * FR + j, lane);
        else d[j] = *reinterpret_cast<const Quad*>(l + p * kPart + row * 64 + ((lane / 16) ^ (row / 2 % 4)) * 16);
      }
#pragma unroll
      for (int i = 0; i < FC; ++i)
#pragma unroll
        for (int j = 0; j < FR; ++j) acc[i][j] = mfma_of<TGRAD_BF16>(c[i], d[j], acc[i][j]);
    }
  };

  read(first);
  place(first);
  if (first + 1 < last) read(first + 1);
  for (int64_t s = first; s < last; ++s) {
    __syncthreads();
    if (s + 1 < last) place(s + 1);
    if (s + 2 < last) read(s + 2);
    multiply(s);
  }
#pragma unroll
  for (int j = 0; j < FR; ++j) {
    const int r = r0 + (wr * FR + j) * 16 + lane % 16;
    if (r >= a.rows) continue;
    char* row = a.out.row((int64_t)split * a.rows + r);
#pragma unroll
    for (int i = 0; i < FC; ++i) {
      const int c = c0 + (wc * FC + i) * 16 + lane / 16 * 4;
      if (c < a.cols) store4<OT>(row, c, a.cols, acc[i][j]);
    }
  }
}

// ---- float32 dy or float32 results of unrounded values, a scale for groups of columns: 64 x 64 results a workgroup, 4 x 4 a thread, float32 -------

// 4096^3: 2400 us, 57 TFLOP/s: two reads of LDS feed four products a thread.  Such codes are the activations' checkpoints, whose values go into no product.
template <int DT, bool WEIGHT>
__global__ __launch_bounds__(256) void k_grad_groups(Grad a) {
  __shared__ float as[16][65], bs[16][65];
  const int r0 = blockIdx.x / a.tiles_c * 64, c0 = blockIdx.x % a.tiles_c * 64;
  const int tr = threadIdx.x / 16, tc = threadIdx.x % 16;
  float acc[4][4] = {};
  for (int64_t s0 = 0; s0 < a.sum; s0 += 16) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = threadIdx.x + 256 * i;
      const int s = WEIGHT ? e / 64 : e % 16, r = WEIGHT ? e % 64 : e / 16, v = e / 64, k = e % 64;
      float x = 0.f, y = 0.f;
      if (s0 + s < a.sum && r0 + r < a.rows)
        x = Elem<DT>::widen(reinterpret_cast<const typename Elem<DT>::raw*>(a.dy.row(WEIGHT ? s0 + s : r0 + r))[WEIGHT ? r0 + r : s0 + s]);
      if (s0 + v < a.sum && c0 + k < a.cols)
        y = (float)a.c.codes[(s0 + v) * a.c.stride + c0 + k] * a.c.scale[(s0 + v) * a.c.groups + ((c0 + k) >> a.c.shift)];
      as[s][r] = x;
      bs[v][k] = y;
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < 16; ++s)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] += as[s][tr + 16 * i] * bs[s][tc + 16 * j];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int r = r0 + tr + 16 * i, k = c0 + tc + 16 * j;
      if (r < a.rows && k < a.cols) reinterpret_cast<float*>(a.out.row(r))[k] = acc[i][j];
    }
}

// dy in rows that start at multiples of 16 bytes and end at multiples of eight numbers, with zeros there: eight numbers a thread.
template <int DT>
__global__ __launch_bounds__(256) void k_align(Mat dy, int64_t rows, int64_t cols, char* out) {
  const int64_t per = (cols + 7) / 8, id = (int64_t)blockIdx.x * 256 + threadIdx.x, r = id / per, at = id % per * 8;
  if (r < rows) *reinterpret_cast<Quad*>(out + id * 16) = load8<DT>(dy.row(r) + at * 2, cols - at);
}

// The splits' sums, added up in their order: four results a thread.
template <int OT>
__global__ __launch_bounds__(256) void k_add_splits(const float* __restrict__ part, int splits, int rows, int cols, Mat out) {
  const int64_t per = (cols + 3) / 4, id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int r = (int)(id / per), c = (int)(id % per) * 4;
  if (r >= rows) return;
  v4f sum = {0.f, 0.f, 0.f, 0.f};
  const float* from = part + (int64_t)r * cols + c;
  const int64_t each = (int64_t)rows * cols;
  if (c + 4 <= cols) {
#pragma unroll 8
    for (int s = 0; s < splits; ++s) sum += __builtin_bit_cast(v4f, *reinterpret_cast<const QuadAny*>(from + s * each));
  } else {
    for (int s = 0; s < splits; ++s)
      for (int k = 0; k < cols - c; ++k) sum[k] += from[s * each + k];
  }
  store4<OT>(out.row(r), c, cols, sum);
}

// ---- host -------------------------------------------------------------------------------------------------------------------------------

struct Cut {
  int tile, tiles_c, tiles, splits, steps;
};
// Tiles of 256 x 256, one workgroup a compute unit, where they fill three quarters of the units, by themselves or with the sum in splits of 1024 at
// least that waste no more than a quarter of their results; else tiles of 128 x 128, with splits up to two for every unit.
// (dw of 131072 x 512 x 768 float16: 187 us in tiles of 128, 42 splits of 6 wide ones 142; dx of 2048 x 2048 x 8192 bf16: 104, 4 splits of 64 wide ones 86.)
Cut cut_of(int64_t rows, int64_t cols, int64_t sum, bool wide, int step) {
  auto tiles = [&](int64_t b) { return ((rows + b - 1) / b) * ((cols + b - 1) / b); };
  const int64_t big = std::max<int64_t>(1, tiles(kWide)), all = std::max<int64_t>(1, (sum + kWideStep - 1) / kWideStep);
  int64_t splits = 1;
  if (wide && big < 192) {
    if (rows * cols * 4 >= big * kWide * kWide * 3) splits = std::max<int64_t>(1, std::min<int64_t>(256 / big, all / 32));
    wide = big * splits >= 192;
  }
  Cut c;
  c.tile = wide ? kWide : 128;
  c.tiles_c = (int)((cols + c.tile - 1) / c.tile);
  c.tiles = (int)std::max<int64_t>(1, std::min<int64_t>(tiles(c.tile), kMostRows));
  const int64_t steps = wide ? all : std::max<int64_t>(1, (sum + step - 1) / step);
  if (!wide) splits = std::max<int64_t>(1, std::min<int64_t>(512 / c.tiles, steps / 4));
  c.steps = (int)((steps + splits - 1) / splits);
  c.splits = (int)((steps + c.steps - 1) / c.steps);
  return c;
}

template <typename Kern>
void launch_cut(hipStream_t s, Kern k, int threads, size_t lds, const Cut& c, const Grad& g) {
  allow_lds(k, lds);
  k<<<dim3((uint32_t)(c.tiles * c.splits)), dim3(threads), lds, s>>>(g);
}

template <int DT, int OT, bool WEIGHT, int PARTS>
void launch_tiles(hipStream_t s, const Cut& c, const Grad& g) {
  if (c.tile == kWide && g.cols % 16) launch_cut(s, k_grad_wide<DT, OT, WEIGHT, true, PARTS>, 512, kWideBufs * kWideBytes, c, g);
  else if (c.tile == kWide) launch_cut(s, k_grad_wide<DT, OT, WEIGHT, false, PARTS>, 512, kWideBufs * kWideBytes, c, g);
  else launch_cut(s, k_grad_tiles<2, 2, 4, 4, DT, OT, WEIGHT, PARTS>, 256, 2 * (128 + 128) * kStep * 2, c, g);
}

void launch_add(hipStream_t s, const float* part, int splits, const tgrad_matrix* out) {
  const int64_t threads = out->rows * ((out->cols + 3) / 4);
  for_real(out->dtype, [&](auto t) {
    k_add_splits<decltype(t)::value><<<dim3((uint32_t)((threads + 255) / 256)), dim3(256), 0, s>>>(part, splits, (int)out->rows, (int)out->cols, mat(out));
  });
}

// What goes straight to LDS: rows at multiples of 16 bytes, whole chunks of eight numbers, offsets of 32 bits within a tile.
bool straight(const tgrad_matrix* dy) {
  return (uintptr_t)dy->data % 16 == 0 && dy->row_stride % 8 == 0 && dy->cols % 8 == 0 && dy->row_stride <= ((int64_t)1 << 21);
}
bool straight(const tgrad_codes* c) { return (uintptr_t)c->codes % 16 == 0 && c->row_stride % 16 == 0 && c->row_stride <= ((int64_t)1 << 22); }
size_t copy_bytes(int64_t tokens, int64_t outer) { return aligned((size_t)tokens * ((outer + 7) / 8 * 16)); }

bool one_scale(const tgrad_codes* c) { return c->group == 0 || c->cols <= c->group; }
// float32 sums of numbers with 24 bits: float32 dy, and float32 results of unrounded values.
bool full(const tgrad_matrix* dy, const tgrad_matrix* out, bool unrounded) { return dy->dtype == TGRAD_F32 || (unrounded && out->dtype == TGRAD_F32); }
// dy in parts, or element by element: no tile reads dy's rows as they are, and none is copied.
bool by_element(const tgrad_matrix* dy, const tgrad_codes* c, const tgrad_matrix* out, bool unrounded) {
  return full(dy, out, unrounded) || (dy->rows <= 16 && one_scale(c));
}

template <bool WEIGHT>
void launch_gradient(hipStream_t s, const tgrad_matrix* dy, const tgrad_codes* c, const tgrad_matrix* out, bool unrounded, void* scratch) {
  Grad g{mat(dy), codes8(c), mat(out), WEIGHT ? dy->rows : dy->cols, (int)out->rows, (int)out->cols, 0, 0, 0, (int)out->rows};
  if (full(dy, out, unrounded) && !one_scale(c)) {
    g.tiles_c = (g.cols + 63) / 64;
    for_real(dy->dtype, [&](auto t) {
      k_grad_groups<decltype(t)::value, WEIGHT><<<dim3((uint32_t)((g.rows + 63) / 64 * (int64_t)g.tiles_c)), dim3(256), 0, s>>>(g);
    });
    return;
  }
  char* parts = static_cast<char*>(scratch);
  const bool split = by_element(dy, c, out, unrounded);
  if (!split && !straight(dy) && dy->rows > 0) {
    const int64_t per = (dy->cols + 7) / 8;
    rows_in_launches(dy->rows, 256, (per + 255) / 256, [&](int64_t first, int64_t rows) {
      for_real(dy->dtype, [&](auto t) {
        k_align<decltype(t)::value><<<dim3((uint32_t)((rows * per + 255) / 256)), dim3(256), 0, s>>>(
            Mat{g.dy.data + first * g.dy.stride, g.dy.stride}, rows, dy->cols, parts + first * per * 16);
      });
    });
    g.dy = Mat{parts, per * 16};
    if (WEIGHT) g.dy_rows = (int)(per * 8);
    parts += copy_bytes(dy->rows, dy->cols);
  }
  const Cut cut = cut_of(out->rows, out->cols, g.sum, !split && straight(c) && g.dy.stride <= ((int64_t)1 << 22), split ? kStep32 : kStep);
  g.tiles_c = cut.tiles_c;
  g.tiles = cut.tiles;
  g.steps = cut.steps;
  if (cut.splits > 1) g.out = Mat{parts, out->cols * 4};
  for_real(dy->dtype, [&](auto t) {
    constexpr int DT = decltype(t)::value;
    auto run = [&](auto o) {
      constexpr int OT = decltype(o)::value;
      if (split) launch_cut(s, k_grad_split<2, 2, 4, 4, DT, OT, WEIGHT>, 256, 2 * (3 * 128 + 128) * kStep32 * 2, cut, g);
      else if constexpr (DT != TGRAD_F32) {
        if constexpr (OT != TGRAD_F32) {
          if (unrounded) return launch_tiles<DT, OT, WEIGHT, 2>(s, cut, g);
        }
        launch_tiles<DT, OT, WEIGHT, 1>(s, cut, g);
      }
    };
    if (cut.splits > 1) run(std::integral_constant<int, -1>());
    else if (out->dtype == DT) run(t);
    else run(std::integral_constant<int, TGRAD_F32>());
  });
  if (cut.splits > 1) launch_add(s, reinterpret_cast<const float*>(parts), cut.splits, out);
}

}  // namespace

namespace tgrad {

// Splits' sums, for the type of dy and the alignment that need most.
size_t gradient_scratch(bool weight, bool copy, int64_t tokens, int64_t inner, int64_t outer) {
  const int64_t rows = weight ? outer : tokens, sum = weight ? tokens : outer;
  size_t most = 0;
  for (bool wide : {false, true})
    for (int step : {kStep, kStep32}) {
      const Cut c = cut_of(rows, inner, sum, wide, step);
      if (c.splits > 1) most = std::max(most, (size_t)c.splits * rows * inner * 4);
    }
  return aligned(most) + (copy ? copy_bytes(tokens, outer) : 0);
}

}  // namespace tgrad

namespace {

// Two-byte rows of more than 2^21 numbers, whose tiles 32-bit offsets do not reach, are refused, and so are sums whose steps they do not count.
bool reachable(const tgrad_matrix* dy) { return dy->rows <= ((int64_t)1 << 30) && (dy->dtype == TGRAD_F32 || dy->cols <= ((int64_t)1 << 21)); }

template <bool WEIGHT>
int gradient(const tgrad_matrix* dy, const tgrad_codes* c, const tgrad_matrix* out, bool unrounded, void* workspace_dev, void* hip_stream) {
  if (!good(dy) || !good(c) || !good(out)) return TGRAD_ERR_INVALID_ARG;
  if (out->dtype != dy->dtype && out->dtype != TGRAD_F32) return TGRAD_ERR_INVALID_ARG;
  if (c->rows != (WEIGHT ? dy->rows : dy->cols) || !same_size(out, WEIGHT ? dy->cols : dy->rows, c->cols)) return TGRAD_ERR_INVALID_ARG;
  if (too_many(out) || !reachable(dy)) return TGRAD_ERR_UNSUPPORTED;
  const bool copy = !by_element(dy, c, out, unrounded) && !straight(dy);
  if (!scratch_ok(workspace_dev, gradient_scratch(WEIGHT, copy, dy->rows, c->cols, dy->cols))) return TGRAD_ERR_INVALID_ARG;
  if (pending()) return TGRAD_ERR_HIP;
  if (out->rows == 0) return TGRAD_OK;
  launch_gradient<WEIGHT>(static_cast<hipStream_t>(hip_stream), dy, c, out, unrounded, workspace_dev);
  return launched();
}

}  // namespace

extern "C" {

int tgrad_codes_grad_input(const tgrad_matrix* dy, const tgrad_codes* w, const tgrad_matrix* dx, void* workspace_dev, void* hip_stream) {
  return gradient<false>(dy, w, dx, false, workspace_dev, hip_stream);
}

int tgrad_codes_grad_weight(const tgrad_matrix* dy, const tgrad_codes* x, const tgrad_matrix* dw, void* workspace_dev, void* hip_stream) {
  return gradient<true>(dy, x, dw, false, workspace_dev, hip_stream);
}

int tgrad_codes_gradient(int op, const tgrad_matrix* dy, const tgrad_codes* codes, const tgrad_matrix* out, void* workspace_dev, void* hip_stream) {
  const bool unrounded = op & TGRAD_CODES_UNROUNDED;
  op &= ~(TGRAD_CODES_UNROUNDED | TGRAD_CODES_UNALIGNED);
  if (op == TGRAD_CODES_GRAD_INPUT) return gradient<false>(dy, codes, out, unrounded, workspace_dev, hip_stream);
  if (op == TGRAD_CODES_GRAD_WEIGHT) return gradient<true>(dy, codes, out, unrounded, workspace_dev, hip_stream);
  return TGRAD_ERR_INVALID_ARG;
}

}  // extern "C"

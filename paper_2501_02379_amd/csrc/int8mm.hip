// Tokens times a weight, both as 8-bit codes with a scale a row.
#include "tiles8.h"

using namespace tgrad;

namespace tgrad {
void launch_quantize(hipStream_t s, const tgrad_matrix* x, const tgrad_codes* out);
size_t gradient_scratch(bool weight, bool copy, int64_t tokens, int64_t inner, int64_t outer);
}

namespace {

// ---- codes times codes: tiles of results, v_mfma_i32_16x16x64_i8 ----------------------------------------------------------------------

constexpr int kStep = 128;                // bytes of the sum in LDS at a time: a row of it is 8 chunks of 16

// Four neighbours of a row of results.
template <int OT>
__device__ __forceinline__ void store_scaled(char* row, int n, int outer, i32x4 sum, float sx, const float* sw) {
  typedef typename Elem<OT>::raw raw;
  raw* to = reinterpret_cast<raw*>(row) + n;
  if (n + 4 <= outer) {
    float f[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) f[r] = scaled(sum[r], sx, sw[n + r]);
    *reinterpret_cast<typename Four<OT>::any*>(to) = Four<OT>::narrow(f);
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (n + r < outer) to[r] = Elem<OT>::narrow(scaled(sum[r], sx, sw[n + r]));
  }
}

// y[t][n] = sum_k x[t][k] w[n][k].  WT x WN wavefronts, each FT x FN results of 16 x 16.  A step's 128 bytes of every row lie in LDS, chunk c of row r
// at chunk c ^ (r % 8), so that eight rows' loads of one chunk meet eight banks; `BUFS` steps are there or on their way.  One
// barrier a step: it says that everyone's part of this step has arrived and that everyone is done with the step before, whose place is filled
// next.  OT < 0: sums go to `part`, [split][tokens][outer], and are added up by k_add_parts.
// STAGED: rows that do not start at multiples of 16 bytes go through registers (4096^3: 140 us instead of 69, 8192^3: 861 instead of 428).
// (8192^3 in tiles of 128 x 128, two workgroups a compute unit: 546 us; four wavefronts of 8 x 8 results: 582.)
template <int WT, int WN, int FT, int FN, int BUFS, bool STAGED, int OT>
__global__ __launch_bounds__(WT * WN * 64, 2) void k_codes_tiles(Codes8 x, Codes8 w, int tokens, int outer, int inner, Mat y, int* part, int tiles_n, int tiles,
                                                              int steps_a_split) {
  constexpr int T = WT * WN * 64, BT = WT * FT * 16, BN = WN * FN * 16, kBytes = (BT + BN) * kStep;
  constexpr int kLoads = kBytes / 16 / T, kLoadsN = BN * kStep / 16 / T;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = lane_id();
  const int split = blockIdx.x / tiles;
  const int2 tile = tile_of(blockIdx.x % tiles, tiles, tiles_n);
  const int t0 = tile.x * BT, n0 = tile.y * BN;
  const int8_t* xp = x.codes + (int64_t)t0 * x.stride;
  const int8_t* wp = w.codes + (int64_t)n0 * w.stride;
  const int first = split * steps_a_split, last = min(first + steps_a_split, (inner + kStep - 1) / kStep);
  const int whole = STAGED ? first : min(last, inner / kStep);        // steps that go straight to LDS

  // this thread's chunks of a step: row (rows beyond the matrix are its last one again, and are not stored) and column
  auto row_of = [&](int i) {
    const int r = (i * T + (int)threadIdx.x) / 8;
    return i < kLoadsN ? min(r, outer - 1 - n0) : min(r - BN, tokens - 1 - t0);
  };
  const int chunk = ((int)threadIdx.x % 8 ^ (int)threadIdx.x / 8 % 8) * 16;
  int each[kLoads];
  if constexpr (!STAGED) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) each[i] = row_of(i) * (int)(i < kLoadsN ? w.stride : x.stride) + chunk;
  }
  const Ref xr = ref(xp), wr = ref(wp);
  auto fill = [&](int s) {
    char* l = lds + (s - first) % BUFS * kBytes + wave * kWave * 16;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) to_lds(i < kLoadsN ? wr : xr, l + i * T * 16, each[i], s * kStep);
  };
  Quad held[kLoads];
  auto read = [&](int s) {
    const int at = s * kStep + chunk;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) held[i] = load16((i < kLoadsN ? wp + row_of(i) * w.stride : xp + row_of(i) * x.stride) + at, inner - at);
  };
  auto place = [&](int s) {
    char* l = lds + (s - first) % BUFS * kBytes + threadIdx.x * 16;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) *reinterpret_cast<Quad*>(l + i * T * 16) = held[i];
  };

  i32x4 acc[FN][FT] = {};
  const int wn = wave % WN, wt = wave / WN;
  auto multiply = [&](int s) {
    const char* l = lds + (s - first) % BUFS * kBytes;
    const char* nl = l + (wn * FN * 16 + lane % 16) * kStep;
    const char* tl = l + (BN + wt * FT * 16 + lane % 16) * kStep;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      i32x4 a[FN], b[FT];
      const int c = ((k * 4 + lane / 16) ^ (lane % 8)) * 16;
#pragma unroll
      for (int i = 0; i < FN; ++i) a[i] = *reinterpret_cast<const i32x4*>(nl + i * 16 * kStep + c);
#pragma unroll
      for (int j = 0; j < FT; ++j) b[j] = *reinterpret_cast<const i32x4*>(tl + j * 16 * kStep + c);
#pragma unroll
      for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int j = 0; j < FT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[i], b[j], acc[i][j], 0, 0, 0);
    }
  };

  if constexpr (STAGED) {
    read(first);
    place(first);
    for (int s = first; s < last; ++s) {
      if (s + 1 < last) read(s + 1);
      __syncthreads();
      multiply(s);
      if (s + 1 < last) place(s + 1);
    }
  } else {
#pragma unroll
    for (int i = 0; i < BUFS - 1; ++i)
      if (first + i < whole) fill(first + i);
    for (int s = first; s < whole; ++s) {
      if (s + BUFS - 2 < whole) barrier_but<kLoads * (BUFS - 2)>();
      else barrier_but<0>();
      if (s + BUFS - 1 < whole) fill(s + BUFS - 1);
      multiply(s);
    }
    if (whole < last) {                   // the sum's end, less than a step
      read(whole);
      __syncthreads();
      place(whole);
      __syncthreads();
      multiply(whole);
    }
  }

#pragma unroll
  for (int j = 0; j < FT; ++j) {
    const int t = t0 + (wt * FT + j) * 16 + lane % 16;
    if (t >= tokens) continue;
    const float sx = OT < 0 ? 0.f : x.scale[t];
#pragma unroll
    for (int i = 0; i < FN; ++i) {
      const int n = n0 + (wn * FN + i) * 16 + lane / 16 * 4;
      if (n >= outer) continue;
      if constexpr (OT < 0) {
        int* to = part + ((int64_t)split * tokens + t) * outer + n;
        if (n + 4 <= outer) {
          *reinterpret_cast<QuadAny*>(to) = __builtin_bit_cast(Quad, acc[i][j]);
        } else {
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (n + r < outer) to[r] = acc[i][j][r];
        }
      } else {
        store_scaled<OT>(y.row(t), n, outer, acc[i][j], sx, w.scale);
      }
    }
  }
}

// The same with 256 x 256 results of 8 wavefronts, 2 x 4 of 8 x 4, in steps of 64 bytes of which four are there or on their way (rows of 64 bytes, chunk c of row
// r at chunk c ^ (r / 2 % 4)).  A step is two turns: wavefronts 0 to 3 read the step's operands while 4 to 7, a turn behind, multiply the
// step before.  What is filled in a step was last read three turns ago at least, and is read five or six turns later.
// 8192^3: 428 us in calls behind one another (2570 TOP/s), 450 behind the launch that quantises, 476 from idle; k_codes_tiles of this size takes 460 to 510
// (wavefronts 4 x 2 of 4 x 8: 488).  The card's power is the limit: the matrix
// instructions alone, out of registers, reach 3260 to 4020 on random codes and 4800 on zeros; without its reads of LDS this kernel would take 410 us.
constexpr int kWide = 256, kWideStep = 64, kWideBufs = 4, kWideBytes = 2 * kWide * kWideStep;

template <int OT>
__global__ __launch_bounds__(512) void k_codes_wide(Codes8 x, Codes8 w, int tokens, int outer, int inner, Mat y, int tiles_n, int tiles) {
  constexpr int T = 512, FT = 8, FN = 4, kLoads = kWideBytes / 16 / T, kLoadsN = kLoads / 2;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = lane_id();
  const int2 tile = tile_of(blockIdx.x, tiles, tiles_n);
  const int t0 = tile.x * kWide, n0 = tile.y * kWide;
  const int8_t* xp = x.codes + (int64_t)t0 * x.stride;
  const int8_t* wp = w.codes + (int64_t)n0 * w.stride;
  auto row_of = [&](int i) {
    const int r = (i * T + (int)threadIdx.x) / 4;
    return i < kLoadsN ? min(r, outer - 1 - n0) : min(r - kWide, tokens - 1 - t0);
  };
  const int chunk = ((int)threadIdx.x % 4 ^ (int)threadIdx.x / 8 % 4) * 16;
  int each[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) each[i] = row_of(i) * (int)(i < kLoadsN ? w.stride : x.stride) + chunk;
  const Ref xr = ref(xp), wr = ref(wp);
  auto fill = [&](int s) {
    char* l = lds + s % kWideBufs * kWideBytes + wave * kWave * 16;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) to_lds(i < kLoadsN ? wr : xr, l + i * T * 16, each[i], s * kWideStep);
  };
  i32x4 acc[FN][FT] = {};
  const int wn = wave % 4, wt = wave / 4;
  const int at = lane % 16 * kWideStep + ((lane / 16) ^ (lane / 2 % 4)) * 16;
  i32x4 a[FN], b[FT];
  auto operands = [&](int s) {
    const char* l = lds + s % kWideBufs * kWideBytes + at;
#pragma unroll
    for (int i = 0; i < FN; ++i) a[i] = *reinterpret_cast<const i32x4*>(l + (wn * FN + i) * 16 * kWideStep);
#pragma unroll
    for (int j = 0; j < FT; ++j) b[j] = *reinterpret_cast<const i32x4*>(l + (kWide + (wt * FT + j) * 16) * kWideStep);
  };
  auto multiply = [&]() {
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
      for (int j = 0; j < FT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[i], b[j], acc[i][j], 0, 0, 0);
  };
  const int whole = inner / kWideStep;
  const bool late = wave >= 4;
#pragma unroll
  for (int i = 0; i < 3; ++i)
    if (i < whole) fill(i);
  turn_but<0>();
  if (late) turn();
  for (int s = 0; s < whole; ++s) {
    if (s + 3 < whole) fill(s + 3);
    operands(s);
    if (s + 3 < whole) turn_but<2 * kLoads>();
    else turn_but<0>();
    __builtin_amdgcn_s_setprio(1);
    multiply();
    __builtin_amdgcn_s_setprio(0);
    turn();
  }
  if (!late) turn();
  if (whole * kWideStep < inner) {        // the sum's end, less than a step, through registers; everyone is done with the first place
    char* l = lds + whole % kWideBufs * kWideBytes + threadIdx.x * 16;
    const int from = whole * kWideStep + chunk;
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      *reinterpret_cast<Quad*>(l + i * T * 16) = load16((i < kLoadsN ? wp + row_of(i) * w.stride : xp + row_of(i) * x.stride) + from, inner - from);
    __syncthreads();
    operands(whole);
    multiply();
  }
#pragma unroll
  for (int j = 0; j < FT; ++j) {
    const int t = t0 + (wt * FT + j) * 16 + lane % 16;
    if (t >= tokens) continue;
    const float sx = x.scale[t];
#pragma unroll
    for (int i = 0; i < FN; ++i) store_scaled<OT>(y.row(t), n0 + (wn * FN + i) * 16 + lane / 16 * 4, outer, acc[i][j], sx, w.scale);
  }
}

// Sums of the splits' sums: four results a thread.
template <int OT>
__global__ __launch_bounds__(256) void k_add_parts(const int* __restrict__ part, int splits, int tokens, int outer, const float* sx, const float* sw, Mat y) {
  const int64_t per = (outer + 3) / 4, id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int t = (int)(id / per), n = (int)(id % per) * 4;
  if (t >= tokens) return;
  const int many = min(4, outer - n);
  i32x4 sum = {0, 0, 0, 0};
  const int* from = part + (int64_t)t * outer + n;
  const int64_t each = (int64_t)tokens * outer;
  if (many == 4) {
#pragma unroll 8
    for (int s = 0; s < splits; ++s) sum += __builtin_bit_cast(i32x4, *reinterpret_cast<const QuadAny*>(from + s * each));
  } else {
    for (int s = 0; s < splits; ++s)
      for (int r = 0; r < many; ++r) sum[r] += from[s * each + r];
  }
  typedef typename Elem<OT>::raw raw;
  raw* to = reinterpret_cast<raw*>(y.row(t)) + n;
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (r < many) to[r] = Elem<OT>::narrow(scaled(sum[r], sx[t], sw[n + r]));
}

// ---- up to 32 tokens: the weight is read once, straight to registers --------------------------------------------------------------------

constexpr int kFewWaves = 8, kFewThreads = kFewWaves * kWave, kAhead = 8;
constexpr int kFusedTokens = 4, kFusedCodes = 32768, kFusedUnits = 4;      // what one workgroup quantises by the way

// 16 outputs a workgroup; its wavefronts share the sum, and a matrix instruction takes 64 bytes of 16 rows of the weight and of 16 tokens (FT times).
// XT >= 0: the tokens come as numbers; every workgroup quantises them into LDS for itself while its first loads of the weight are on their way, which
// spares a launch; the first one writes what is kept.  1 x 4096 x 4096: 6 to 7 us, with 9.4 a call; 16 x 8192 x 8192 18.4 a call.
template <int XT, int OT, int FT>
__global__ __launch_bounds__(kFewThreads) void k_codes_few(Mat xm, Codes8 x, bool keep, Codes8 w, int tokens, int outer, int inner, Mat y) {
  extern __shared__ __attribute__((aligned(16))) char lds[];          // sums, scales, then codes of the tokens
  int (*sums)[FT][kWave][4] = reinterpret_cast<int (*)[FT][kWave][4]>(lds);
  float* sx = reinterpret_cast<float*>(lds + sizeof(int) * kFewWaves * FT * kWave * 4);
  uint32_t* tops = reinterpret_cast<uint32_t*>(sx + 16 * FT);
  char* codes = reinterpret_cast<char*>(tops + kFewWaves);
  const int wave = threadIdx.x / kWave, lane = lane_id();
  const int n0 = blockIdx.x * 16;
  const int8_t* wrow = w.codes + (int64_t)min(n0 + lane % 16, outer - 1) * w.stride;
  const int pieces = (inner + 63) / 64, a_wave = (pieces + kFewWaves - 1) / kFewWaves;
  const int first = min(wave * a_wave, pieces), last = min(first + a_wave, pieces);
  const int mine = lane / 16 * 16;
  Quad a[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    const int at = (first + i) * 64 + mine;
    a[i] = load16(wrow + at, first + i < last ? inner - at : 0);
  }
  const int pitch = (inner + 63) / 64 * 64;
  if constexpr (XT >= 0) {
    constexpr int es = sizeof(typename Elem<XT>::raw);
    const int units = pitch / 8;
    for (int t = 0; t < tokens; ++t) {
      Eight<XT> held[kFusedUnits];
      float f[8];
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < kFusedUnits; ++i) {
        const int u = threadIdx.x + i * kFewThreads;
        held[i].clear();
        if (u * 8 < inner) held[i].load(xm.row(t) + (int64_t)u * 8 * es, inner - u * 8);
        held[i].get(f);
        top = max(top, largest(f));
      }
      const Rounding r = rounding_of(largest_of_block<kFewWaves>(top, tops));
      if (threadIdx.x == 0) {
        sx[t] = r.scale;
        if (keep && blockIdx.x == 0) x.scale[t] = r.scale;
      }
#pragma unroll
      for (int i = 0; i < kFusedUnits; ++i) {
        const int u = threadIdx.x + i * kFewThreads;
        held[i].get(f);
        if (u < units) {
          const Duo d = codes_of(f, r);
          *reinterpret_cast<Duo*>(codes + t * pitch + u * 8) = d;
          if (keep && blockIdx.x == 0 && u * 8 < inner) store_codes(x.codes + t * x.stride + u * 8, d, inner - u * 8);
        }
      }
    }
    __syncthreads();
  } else {
    if (threadIdx.x < (uint32_t)tokens) sx[threadIdx.x] = x.scale[threadIdx.x];
  }
  const char* lrow[FT];
  const int8_t* xrow[FT];
#pragma unroll
  for (int j = 0; j < FT; ++j) {
    const int t = min(j * 16 + lane % 16, tokens - 1);
    lrow[j] = codes + t * pitch;
    xrow[j] = x.codes + (int64_t)t * x.stride;
  }
  i32x4 acc[FT] = {};
  for (int p = first; p < last; p += kAhead) {
    Quad b[FT][kAhead];
#pragma unroll
    for (int j = 0; j < FT; ++j)
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int at = (p + i) * 64 + mine;
        if constexpr (XT >= 0) b[j][i] = p + i < last ? *reinterpret_cast<const Quad*>(lrow[j] + at) : Quad{0, 0, 0, 0};
        else b[j][i] = load16(xrow[j] + at, p + i < last ? inner - at : 0);
      }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
#pragma unroll
      for (int j = 0; j < FT; ++j)
        acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a[i]), __builtin_bit_cast(i32x4, b[j][i]), acc[j], 0, 0, 0);
      const int at = (p + kAhead + i) * 64 + mine;
      a[i] = load16(wrow + at, p + kAhead + i < last ? inner - at : 0);
    }
  }
#pragma unroll
  for (int j = 0; j < FT; ++j) *reinterpret_cast<i32x4*>(sums[wave][j][lane]) = acc[j];
  __syncthreads();
  // lane l of a wavefront has token l % 16 and outputs 4 (l / 16) .. + 3
  if (threadIdx.x < 256 * FT) {
    const int t = threadIdx.x / 16, n = threadIdx.x % 16;
    int sum = 0;
#pragma unroll
    for (int i = 0; i < kFewWaves; ++i) sum += sums[i][t / 16][n / 4 * 16 + t % 16][n % 4];
    if (t < tokens && n0 + n < outer) reinterpret_cast<typename Elem<OT>::raw*>(y.row(t))[n0 + n] = Elem<OT>::narrow(scaled(sum, sx[t], w.scale[n0 + n]));
  }
}

// ---- host ---------------------------------------------------------------------------------------------------------------------------

size_t few_lds(int ft, int64_t tokens, int64_t inner) {
  return sizeof(int) * kFewWaves * ft * kWave * 4 + 16 * ft * 4 + kFewWaves * 4 + (size_t)tokens * ((inner + 63) / 64 * 64);
}

// Codes of x that nobody keeps: rows of a multiple of 16 bytes, and a scale each.
int64_t scratch_stride(int64_t inner) { return (inner + 15) / 16 * 16; }
size_t scratch_codes(int64_t tokens, int64_t inner) { return aligned((size_t)tokens * scratch_stride(inner)) + aligned((size_t)tokens * 4); }

// How a product of more tokens is cut.
struct Cut {
  int tile;                               // 256, 128 or 64 results on a side
  int tiles_n, tiles, splits, steps;      // steps of kStep bytes to a split
};
// Codes that go straight to LDS: 16-byte rows, and offsets of 32 bits within a tile.
bool straight(const void* p, int64_t stride) { return (uintptr_t)p % 16 == 0 && stride % 16 == 0 && stride <= ((int64_t)1 << 22); }
// Tiles of 256 x 256 where they fill three quarters of the compute units (one workgroup each), of 128 x 128 otherwise, of 64 outputs for up to 64 tokens, where
// it is the weight's bytes that count.  The sum is split where there are fewer tiles than two (three of 64 outputs) for every compute unit.
// (2048 x 8192 x 2048: 96 us in tiles of 256, 48 of 128; 1024 x 4096 x 4096: 56 and 29; 4096^3: 69 and 75.  23 x 8190 x 10007: 21.9 us in tiles of 64 x 64 and up
// to 1024 of them, 20.2 of 32 x 64 and up to 768.)
Cut cut_of(int64_t tokens, int64_t outer, int64_t inner, bool direct) {
  auto tiles = [&](int64_t b) { return ((tokens + b - 1) / b) * ((outer + b - 1) / b); };
  Cut c;
  c.tile = tokens <= 64 ? 64 : direct && tiles(256) >= 192 ? 256 : 128;
  c.tiles_n = (int)((outer + c.tile - 1) / c.tile);
  c.tiles = (int)std::max<int64_t>(1, std::min<int64_t>(tiles(c.tile), kMostRows));
  const int64_t steps = (inner + kStep - 1) / kStep, want = c.tile == 256 ? 1 : c.tile == 128 ? 512 : 768;
  int64_t splits = std::max<int64_t>(1, std::min<int64_t>(want / c.tiles, steps / 4));
  c.steps = (int)((steps + splits - 1) / splits);
  c.splits = (int)((steps + c.steps - 1) / c.steps);
  return c;
}
// Products of k_codes_few: every workgroup reads all tokens' codes, so beyond 16 tokens the weight has to be small as well.  (Calls, us, k_codes_few / tiles and their
// parts: 32 x 4096 x 4096 10.1 / 14.5, 23 x 8190 x 10007 44 / 24.7.)
bool few(int64_t tokens, int64_t outer, int64_t inner) { return tokens <= 16 || (tokens <= 32 && outer * inner <= ((int64_t)1 << 25)); }
size_t part_bytes(int64_t tokens, int64_t outer, int64_t inner) {
  if (few(tokens, outer, inner)) return 0;
  size_t most = 0;
  for (bool direct : {false, true}) {
    const Cut c = cut_of(tokens, outer, inner, direct);
    if (c.splits > 1) most = std::max(most, (size_t)c.splits * tokens * outer * 4);
  }
  return aligned(most);
}

template <int WT, int WN, int FT, int FN, int BUFS, bool STAGED, int OT>
void launch_tiles_as(hipStream_t s, const Cut& c, const Codes8& x, const Codes8& w, const tgrad_matrix* y, int inner, int* part) {
  constexpr size_t bytes = (size_t)(WT * FT + WN * FN) * 16 * kStep * BUFS;
  auto k = k_codes_tiles<WT, WN, FT, FN, BUFS, STAGED, OT>;
  allow_lds(k, bytes);
  k<<<dim3((uint32_t)(c.tiles * c.splits)), dim3(WT * WN * 64), bytes, s>>>(x, w, (int)y->rows, (int)y->cols, inner, mat(y), part, c.tiles_n, c.tiles, c.steps);
}
template <bool STAGED, int OT>
void launch_tiles(hipStream_t s, const Cut& c, const Codes8& x, const Codes8& w, const tgrad_matrix* y, int inner, int* part) {
  if (c.tile == 64 && y->rows <= 32) launch_tiles_as<1, 4, 2, 1, STAGED ? 2 : 4, STAGED, OT>(s, c, x, w, y, inner, part);
  else if (c.tile == 64) launch_tiles_as<2, 2, 2, 2, STAGED ? 2 : 3, STAGED, OT>(s, c, x, w, y, inner, part);
  else if (STAGED || c.tile == 128) launch_tiles_as<2, 2, 4, 4, 2, STAGED, OT>(s, c, x, w, y, inner, part);
  else if constexpr (OT >= 0) {
    auto k = k_codes_wide<OT>;
    allow_lds(k, kWideBufs * kWideBytes);
    k<<<dim3((uint32_t)c.tiles), dim3(512), kWideBufs * kWideBytes, s>>>(x, w, (int)y->rows, (int)y->cols, inner, mat(y), c.tiles_n, c.tiles);
  }
}

void launch_product(hipStream_t s, const tgrad_codes* x, const tgrad_codes* w, const tgrad_matrix* y, void* parts) {
  const Codes8 cx = codes8(x), cw = codes8(w);
  const int inner = (int)x->cols;
  if (few(y->rows, y->cols, inner)) {
    for_real(y->dtype, [&](auto t) {
      auto run = [&](auto ft) {
        constexpr int FT = decltype(ft)::value;
        k_codes_few<-1, decltype(t)::value, FT><<<dim3((uint32_t)((y->cols + 15) / 16)), dim3(kFewThreads), few_lds(FT, 0, 0), s>>>(
            Mat{nullptr, 0}, cx, false, cw, (int)y->rows, (int)y->cols, inner, mat(y));
      };
      if (y->rows <= 16) run(std::integral_constant<int, 1>());
      else run(std::integral_constant<int, 2>());
    });
    return;
  }
  const bool direct = straight(x->codes, x->row_stride) && straight(w->codes, w->row_stride);
  const Cut c = cut_of(y->rows, y->cols, inner, direct);
  int* part = static_cast<int*>(parts);
  if (c.splits > 1) {
    if (direct) launch_tiles<false, -1>(s, c, cx, cw, y, inner, part);
    else launch_tiles<true, -1>(s, c, cx, cw, y, inner, part);
    const int64_t threads = y->rows * ((y->cols + 3) / 4);
    for_real(y->dtype, [&](auto t) {
      k_add_parts<decltype(t)::value><<<dim3((uint32_t)((threads + 255) / 256)), dim3(256), 0, s>>>(part, c.splits, (int)y->rows, (int)y->cols, x->scale, w->scale, mat(y));
    });
  } else {
    for_real(y->dtype, [&](auto t) {
      if (direct) launch_tiles<false, decltype(t)::value>(s, c, cx, cw, y, inner, nullptr);
      else launch_tiles<true, decltype(t)::value>(s, c, cx, cw, y, inner, nullptr);
    });
  }
}

// A few tokens are quantised by the product's own launch.
bool fused(int64_t tokens, int64_t inner) { return tokens <= kFusedTokens && tokens * inner <= kFusedCodes && inner <= kFewThreads * 8 * kFusedUnits; }

size_t product_scratch(int64_t tokens, int64_t outer, int64_t inner) { return inner <= TGRAD_CODES_MAX_INNER ? part_bytes(tokens, outer, inner) : 0; }
size_t linear_scratch(int64_t tokens, int64_t outer, int64_t inner) {
  return fused(tokens, inner) ? 0 : product_scratch(tokens, outer, inner) + scratch_codes(tokens, inner);
}

}  // namespace

extern "C" {

int tgrad_codes_query_size(int op, int64_t tokens, int64_t inner, int64_t outer, size_t* workspace_bytes) {
  const bool copy = op & TGRAD_CODES_UNALIGNED, gradient = op >= TGRAD_CODES_UNALIGNED;
  if (op > 0) op &= ~(TGRAD_CODES_UNALIGNED | TGRAD_CODES_UNROUNDED);
  if (!workspace_bytes || op < (gradient ? TGRAD_CODES_GRAD_INPUT : TGRAD_CODES_MATMUL) || op > TGRAD_CODES_GRAD_WEIGHT) return TGRAD_ERR_INVALID_ARG;
  if (!extents_ok(tokens, inner, inner) || !extents_ok(outer, inner, inner)) return TGRAD_ERR_INVALID_ARG;
  *workspace_bytes = op == TGRAD_CODES_MATMUL ? product_scratch(tokens, outer, inner)
                   : op == TGRAD_CODES_LINEAR ? linear_scratch(tokens, outer, inner)
                                              : gradient_scratch(op == TGRAD_CODES_GRAD_WEIGHT, copy, tokens, inner, outer);
  return TGRAD_OK;
}

int tgrad_codes_matmul(const tgrad_codes* x, const tgrad_codes* w, const tgrad_matrix* y, void* workspace_dev, void* hip_stream) {
  if (!good(x) || !good(w) || !good(y) || x->group || w->group) return TGRAD_ERR_INVALID_ARG;
  if (x->cols != w->cols || !same_size(y, x->rows, w->rows)) return TGRAD_ERR_INVALID_ARG;
  if (too_many(y) || x->cols > TGRAD_CODES_MAX_INNER) return TGRAD_ERR_UNSUPPORTED;
  if (!scratch_ok(workspace_dev, product_scratch(y->rows, y->cols, x->cols))) return TGRAD_ERR_INVALID_ARG;
  if (pending()) return TGRAD_ERR_HIP;
  if (y->rows == 0) return TGRAD_OK;
  launch_product(static_cast<hipStream_t>(hip_stream), x, w, y, workspace_dev);
  return launched();
}

int tgrad_codes_linear(const tgrad_matrix* x, const tgrad_codes* w, const tgrad_codes* keep, const tgrad_matrix* y, void* workspace_dev,
                      void* hip_stream) {
  if (!good(x) || !good(w) || !good(y) || w->group) return TGRAD_ERR_INVALID_ARG;
  if (x->cols != w->cols || !same_size(y, x->rows, w->rows)) return TGRAD_ERR_INVALID_ARG;
  if (keep && (!good(keep) || keep->group || !same_size(keep, x->rows, x->cols))) return TGRAD_ERR_INVALID_ARG;
  if (too_many(y) || x->cols > TGRAD_CODES_MAX_INNER) return TGRAD_ERR_UNSUPPORTED;
  if (!scratch_ok(workspace_dev, keep ? product_scratch(y->rows, y->cols, x->cols) : linear_scratch(y->rows, y->cols, x->cols))) return TGRAD_ERR_INVALID_ARG;
  if (pending()) return TGRAD_ERR_HIP;
  if (y->rows == 0) return TGRAD_OK;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (fused(x->rows, x->cols)) {
    for_real(x->dtype, [&](auto xt) {
      for_real(y->dtype, [&](auto yt) {
        k_codes_few<decltype(xt)::value, decltype(yt)::value, 1><<<dim3((uint32_t)((y->cols + 15) / 16)), dim3(kFewThreads), few_lds(1, x->rows, x->cols), s>>>(
            mat(x), codes8(keep), keep != nullptr, codes8(w), (int)y->rows, (int)y->cols, (int)x->cols, mat(y));
      });
    });
    return launched();
  }
  tgrad_codes own = {};
  if (!keep) {
    char* at = static_cast<char*>(workspace_dev) + part_bytes(y->rows, y->cols, x->cols);
    own = tgrad_codes{at, reinterpret_cast<float*>(at + aligned((size_t)x->rows * scratch_stride(x->cols))), x->rows, x->cols, scratch_stride(x->cols), 0};
  }
  const tgrad_codes* c = keep ? keep : &own;
  launch_quantize(s, x, c);
  launch_product(s, c, w, y, workspace_dev);
  return launched();
}

}  // extern "C"

// Numbers in 8 bits and back, and an activation whose backward pass reads what it kept in 8 bits.
//
// A group of columns shares a scale, its largest magnitude over 127; codes are the exact quotients rounded to nearest even.  There are 10 to 40
// operations for every 3 to 10 bytes: memory bounds all of it.
#include "block8.h"

using namespace tgrad;

namespace {

// Activations and their derivatives.  FULL, for float32: exponentials whose argument's rounding is made good, so that errors do not grow with it (exp2's
// argument of -30 is off by 2^-20, which is 10 u of the result); two-byte results and codes round that away.  (Float32 8192^2, us, with it and without: result
// 101 and 99, backward pass with gate 170 and 167, gelu 176 and 171; as codes it would be 197 and 137, gelu 357 and 159.)
__device__ __forceinline__ float exp2_of(float t, float rest) {          // 2^(t + rest), a small rest; t <= 0
  t = in_float32(t);                                                     // the rest is that of t as it was rounded
  const float n = rintf(t), e = __builtin_amdgcn_exp2f(t - n);
  return ldexpf(fmaf(e, rest * 0.69314718f, e), (int)n);
}

template <int ACT, bool FULL> struct Act;
template <> struct Act<TGRAD_ACT_SILU, false> {
  static __device__ __forceinline__ float value(float v) { return v * __builtin_amdgcn_rcpf(1.f + __expf(-v)); }
  static __device__ __forceinline__ void both(float v, float& y, float& slope) {
    const float p = __builtin_amdgcn_rcpf(1.f + __expf(-v));
    y = v * p;
    slope = p * (1.f + v * (1.f - p));
  }
};
// From q = exp(-|v|) <= 1: 1 / (1 + q) and q / (1 + q) are p and 1 - p, or the other way round, each with all its digits.
template <> struct Act<TGRAD_ACT_SILU, true> {
  static __device__ __forceinline__ void parts(float v, float& p, float& other) {
    constexpr float kLog2e = 1.44269502f, kLow = 1.92596303e-08f;
    const float z = fminf(fabsf(v), 1000.f), t = z * -kLog2e;
    const float q = exp2_of(t, fmaf(z, -kLow, fmaf(z, -kLog2e, -t)));
    const float r = __builtin_amdgcn_rcpf(1.f + q), s = q * r;
    p = v < 0.f ? s : r;
    other = v < 0.f ? r : s;
  }
  static __device__ __forceinline__ float value(float v) {
    float p, other;
    parts(v, p, other);
    return v * p;
  }
  static __device__ __forceinline__ void both(float v, float& y, float& slope) {
    float p, other;
    parts(v, p, other);
    y = v * p;
    slope = p * fmaf(v, other, 1.f);
  }
};
// The normal distribution function from its tail, Phi(-z) = exp(-z^2 / 2) P(t) with t = 1 / (1 + c z), z = |v|: P(t) = exp(z^2 / 2) Phi(-z) is smooth on 0..1,
// and a polynomial fitted to it by least squares in 64 bits, weighted by 1 / P, is off by 1e-07 of it.  Tails keep their digits that way, which
// (1 + erf) / 2 loses below -2.  (With erfc of the device library: 519 us where silu takes 409.)
template <bool FULL> struct Act<TGRAD_ACT_GELU, FULL> {
  static __device__ __forceinline__ void tail(float v, float& bell, float& q) {
    const float z = fabsf(v);
    if constexpr (FULL) {
      constexpr float kHalf = 0.721347511f, kLow = 9.62981517e-09f;      // log2(e) / 2
      const float w = fminf(z, 64.f), s = w * w, a = s * -kHalf;
      bell = exp2_of(a, fmaf(s, -kLow, fmaf(s, -kHalf, -a)) - fmaf(w, w, -s) * kHalf);
    } else {
      bell = __builtin_amdgcn_exp2f(v * v * -0.72134752f);
    }
    const float t = __builtin_amdgcn_rcpf(fmaf(0.40f, z, 1.f));
    float p = 3.219981867e-02f;
    p = fmaf(p, t, -1.766817470e-01f);
    p = fmaf(p, t, 3.818516465e-01f);
    p = fmaf(p, t, -3.732105289e-01f);
    p = fmaf(p, t, 1.186081176e-01f);
    p = fmaf(p, t, -2.625735117e-02f);
    p = fmaf(p, t, 9.109580981e-02f);
    p = fmaf(p, t, 1.331981479e-01f);
    p = fmaf(p, t, 1.596197832e-01f);
    p = fmaf(p, t, 1.595763111e-01f);
    q = bell * p * t;
  }
  static __device__ __forceinline__ float value(float v) {
    float bell, q;
    tail(v, bell, q);
    return v * (v > 0.f ? 1.f - q : q);
  }
  static __device__ __forceinline__ void both(float v, float& y, float& slope) {
    float bell, q;
    tail(v, bell, q);
    const float p = v > 0.f ? 1.f - q : q;
    y = v * p;
    slope = p + v * 0.39894228f * bell;
  }
};

// ---- a scale for the whole row: a workgroup of T threads a row ------------------------------------------------------------

// 8192^2 bf16: 33 us, 6.1 TB/s.  Units of eight numbers; thread t has units t, t + T, ...; the first NV of each thread stay in registers.
template <int DT, int T, int NV>
__global__ __launch_bounds__(T) void k_quantize_rows(Mat x, int64_t first, int cols, Codes8 out) {
  __shared__ uint32_t lds[T / kWave];
  const int64_t row = first + blockIdx.x;
  const char* src = x.row(row);
  const int units = (cols + 7) / 8, es = sizeof(typename Elem<DT>::raw);
  Eight<DT> held[NV];
  uint32_t top = 0;
  float f[8];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int u = threadIdx.x + i * T;
    held[i].clear();
    if (u < units) held[i].load(src + (int64_t)u * 8 * es, cols - u * 8);
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    held[i].get(f);
    top = max(top, largest(f));
  }
  for (int u = threadIdx.x + NV * T; u < units; u += T) {
    Eight<DT> e;
    e.load(src + (int64_t)u * 8 * es, cols - u * 8);
    e.get(f);
    top = max(top, largest(f));
  }
  const Rounding r = rounding_of(largest_of_block<T / kWave>(top, lds));
  if (threadIdx.x == 0) out.scale[row] = r.scale;
  int8_t* dst = out.codes + row * out.stride;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int u = threadIdx.x + i * T;
    held[i].get(f);
    if (u < units) store_codes(dst + u * 8, codes_of(f, r), cols - u * 8);
  }
  for (int u = threadIdx.x + NV * T; u < units; u += T) {
    Eight<DT> e;
    e.load(src + (int64_t)u * 8 * es, cols - u * 8);
    e.get(f);
    store_codes(dst + (int64_t)u * 8, codes_of(f, r), cols - u * 8);
  }
}

// ---- a scale for 32 to 512 columns: a thread for eight numbers, 4 to 64 neighbouring lanes a group -----------------------------

// Where a thread's eight numbers lie.  Every row has a whole number of groups of threads, so that no group is shared by two rows.
struct Place {
  int64_t row;
  int col;
  bool in;
};
__device__ __forceinline__ Place place_of(int64_t first, int64_t rows, int threads_a_row, int cols) {
  const uint32_t id = blockIdx.x * blockDim.x + threadIdx.x;
  const uint32_t r = id / (uint32_t)threads_a_row;
  Place p;
  p.row = first + r;
  p.col = (int)(id - r * (uint32_t)threads_a_row) * 8;
  p.in = (int64_t)r < rows && p.col < cols;
  return p;
}

__device__ __forceinline__ void keep_group(const float* f, const Place& p, int cols, const Codes8& out) {
  const Rounding r = rounding_of(largest_of_lanes(largest(f), 1 << (out.shift - 3)));
  if (!p.in) return;
  if ((p.col & ((1 << out.shift) - 1)) == 0) out.scale[p.row * out.groups + (p.col >> out.shift)] = r.scale;
  store_codes(out.codes + p.row * out.stride + p.col, codes_of(f, r), cols - p.col);
}

template <int DT>
__global__ __launch_bounds__(256) void k_quantize_groups(Mat x, int64_t first, int64_t rows, int threads_a_row, int cols, Codes8 out) {
  const Place p = place_of(first, rows, threads_a_row, cols);
  Eight<DT> e;
  e.clear();
  if (p.in) e.load(x.row(p.row) + (int64_t)p.col * sizeof(typename Elem<DT>::raw), cols - p.col);
  float f[8];
  e.get(f);
  keep_group(f, p, cols, out);
}

template <int DT>
__global__ __launch_bounds__(256) void k_dequantize(Codes8 c, int64_t first, int64_t rows, int threads_a_row, int cols, Mat out) {
  const Place p = place_of(first, rows, threads_a_row, cols);
  if (!p.in) return;
  float f[8];
  widen_codes(load_codes(c.codes + p.row * c.stride + p.col, cols - p.col), c.scale[p.row * c.groups + (p.col >> c.shift)], f);
  Eight<DT> e;
  e.set(f);
  e.store(out.row(p.row) + (int64_t)p.col * sizeof(typename Elem<DT>::raw), cols - p.col);
}

// ---- activation ---------------------------------------------------------------------------------------------------------------

template <int ACT, bool GATED, bool FULL>
__device__ __forceinline__ void activate(const float* v, const float* g, float* y) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    y[i] = Act<ACT, FULL>::value(v[i]);
    if constexpr (GATED) y[i] *= g[i];
  }
}

// 8192 x 28672 bf16 with a gate: 311 us, 6 TB/s; without the checkpoint 234.
template <int DT, int ACT, bool GATED>
__global__ __launch_bounds__(256) void k_activation(Mat x, Mat gate, int64_t first, int64_t rows, int threads_a_row, int cols, Mat y,
                                                    Codes8 x8, Codes8 gate8) {
  const Place p = place_of(first, rows, threads_a_row, cols);
  const int64_t at = (int64_t)p.col * sizeof(typename Elem<DT>::raw);
  Eight<DT> e, h;
  float v[8], g[8], r[8];
  e.clear();
  h.clear();
  if (p.in) {
    e.load(x.row(p.row) + at, cols - p.col);
    if constexpr (GATED) h.load(gate.row(p.row) + at, cols - p.col);
  }
  e.get(v);
  h.get(g);
  if (p.in) {
    activate<ACT, GATED, DT == TGRAD_F32>(v, g, r);
    Eight<DT> o;
    o.set(r);
    o.store(y.row(p.row) + at, cols - p.col);
  }
  if (x8.codes) {
    keep_group(v, p, cols, x8);
    if constexpr (GATED) keep_group(g, p, cols, gate8);
  }
}

// The same with the result in 8 bits, one scale a row: a workgroup of T threads a row.  The result waits as float32, the first NV units of every thread in
// registers, the next NL in LDS; of longer rows the rest is computed again.  8192 x 28672 bf16 with a gate and its checkpoint: 361 us, 4.5 TB/s, with two
// rows of 512 threads a compute unit, 4 units in registers and 4 in LDS; some 33 operations a number are 6 us of a row.  (1024 threads with all in registers leave
// room for one row, whose arithmetic does not go on under its loads and stores: 401; with all its loads ahead 430; the next row's loads as soon as
// registers are free spill: 711.  3 in registers and 5 in LDS, one row a unit: 589.)
template <int DT, int ACT, bool GATED, int T, int NV, int NL>
__global__ __launch_bounds__(T, NL > 0 ? 4 : 1) void k_activation_rows(Mat x, Mat gate, int64_t first, int cols, Codes8 y8, Codes8 x8, Codes8 gate8) {
  __shared__ uint32_t lds[T / kWave];
  __shared__ __attribute__((aligned(16))) float kept[NL > 0 ? NL * T * 8 : 4];
  const int64_t row = first + blockIdx.x;
  const char* src = x.row(row);
  const char* gsrc = GATED ? gate.row(row) : nullptr;
  const int units = (cols + 7) / 8, es = sizeof(typename Elem<DT>::raw);
  float held[NV][8];
  uint32_t top = 0;
  auto load = [&](int u, Eight<DT>& e, Eight<DT>& h) {
    e.clear();
    h.clear();
    if (u < units) {
      e.load(src + (int64_t)u * 8 * es, cols - u * 8);
      if constexpr (GATED) h.load(gsrc + (int64_t)u * 8 * es, cols - u * 8);
    }
  };
  auto unit = [&](int u, const Eight<DT>& e, const Eight<DT>& h, float* r, bool keep) {
    float v[8], g[8];
    const Place p{row, u * 8, u < units};
    e.get(v);
    h.get(g);
    activate<ACT, GATED, false>(v, g, r);
    if (keep && x8.codes) {
      keep_group(v, p, cols, x8);
      if constexpr (GATED) keep_group(g, p, cols, gate8);
    }
  };
  Eight<DT> e, h;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    load(threadIdx.x + i * T, e, h);
    unit(threadIdx.x + i * T, e, h, held[i], true);
    top = max(top, largest(held[i]));
  }
  if constexpr (NL > 0) {
#pragma unroll 1
    for (int i = 0; i < NL; ++i) {
      float r[8];
      load(threadIdx.x + (NV + i) * T, e, h);
      unit(threadIdx.x + (NV + i) * T, e, h, r, true);
      top = max(top, largest(r));
      float4* to = reinterpret_cast<float4*>(kept) + i * 2 * T + threadIdx.x;
      to[0] = make_float4(r[0], r[1], r[2], r[3]);
      to[T] = make_float4(r[4], r[5], r[6], r[7]);
    }
  }
  for (int u0 = (NV + NL) * T; u0 < units; u0 += T) {      // whole wavefronts: groups are formed across lanes
    float r[8];
    load(u0 + threadIdx.x, e, h);
    unit(u0 + threadIdx.x, e, h, r, true);
    top = max(top, largest(r));
  }
  const Rounding r8 = rounding_of(largest_of_block<T / kWave>(top, lds));
  if (threadIdx.x == 0) y8.scale[row] = r8.scale;
  int8_t* dst = y8.codes + row * y8.stride;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int u = threadIdx.x + i * T;
    if (u < units) store_codes(dst + u * 8, codes_of(held[i], r8), cols - u * 8);
  }
  if constexpr (NL > 0) {
#pragma unroll 1
    for (int i = 0; i < NL; ++i) {
      const int u = threadIdx.x + (NV + i) * T;
      const float4* from = reinterpret_cast<const float4*>(kept) + i * 2 * T + threadIdx.x;
      const float4 p = from[0], q = from[T];
      const float r[8] = {p.x, p.y, p.z, p.w, q.x, q.y, q.z, q.w};
      if (u < units) store_codes(dst + u * 8, codes_of(r, r8), cols - u * 8);
    }
  }
  for (int u = threadIdx.x + (NV + NL) * T; u < units; u += T) {
    float r[8];
    load(u, e, h);
    unit(u, e, h, r, false);
    store_codes(dst + (int64_t)u * 8, codes_of(r, r8), cols - u * 8);
  }
}

// 8192 x 28672 bf16 with a gate: 317 us, 5.9 TB/s.
template <int DT, int ACT, bool GATED>
__global__ __launch_bounds__(256) void k_activation_back(Mat dy, Codes8 x8, Codes8 gate8, int64_t first, int64_t rows, int threads_a_row,
                                                         int cols, Mat dx, Mat dgate) {
  const Place p = place_of(first, rows, threads_a_row, cols);
  if (!p.in) return;
  const int64_t at = (int64_t)p.col * sizeof(typename Elem<DT>::raw);
  const int n = cols - p.col;
  Eight<DT> e;
  e.load(dy.row(p.row) + at, n);
  float d[8], v[8], g[8], a[8], b[8];
  e.get(d);
  widen_codes(load_codes(x8.codes + p.row * x8.stride + p.col, n), x8.scale[p.row * x8.groups + (p.col >> x8.shift)], v);
  if constexpr (GATED)
    widen_codes(load_codes(gate8.codes + p.row * gate8.stride + p.col, n), gate8.scale[p.row * gate8.groups + (p.col >> gate8.shift)], g);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float y, slope;
    Act<ACT, DT == TGRAD_F32>::both(v[i], y, slope);
    a[i] = d[i] * slope;
    if constexpr (GATED) {
      a[i] = d[i] * g[i] * slope;
      b[i] = d[i] * y;
    }
  }
  e.set(a);
  e.store(dx.row(p.row) + at, n);
  if constexpr (GATED) {
    e.set(b);
    e.store(dgate.row(p.row) + at, n);
  }
}

// ---- launches -------------------------------------------------------------------------------------------------------------------

// Threads and units in registers of a workgroup that has a row to itself: the fewest threads whose registers hold it, 4 units each at most, so that several rows
// share a compute unit.  (32768 rows of 1000 bf16 quantised by 256 threads 28 us, by 64 18; activations of them 71 and 45.  Rows of 28672, activations: 512
// threads of 8 units 560 us, 1024 with their registers halved for two rows a unit spill: 1110.)
template <typename F>
void for_row(int64_t rows, int cols, F&& f) {
  const int units = (cols + 7) / 8;
  typedef std::integral_constant<int, 64> t64;
  typedef std::integral_constant<int, 256> t256;
  typedef std::integral_constant<int, 512> t512;
  typedef std::integral_constant<int, 1024> t1024;
  typedef std::integral_constant<int, 1> n1;
  typedef std::integral_constant<int, 2> n2;
  typedef std::integral_constant<int, 4> n4;
  if (units <= 64) f(t64(), n1());
  else if (units <= 128) f(t64(), n2());
  else if (units <= 256) f(t256(), n1());
  else if (units <= 512) f(t256(), n2());
  else if (units <= 1024 && rows > compute_units()) f(t256(), n4());
  else if (units <= 1024) f(t1024(), n1());
  else if (units <= 2048) f(t512(), n4());
  else f(t1024(), n4());
}

// f(first, rows, workgroups, threads a row) for a thread for eight columns, rows in whole groups of `lanes` threads.
template <typename F>
void for_units(int64_t rows, int64_t cols, int64_t lanes, F&& f) {
  const int64_t a_row = ((cols + 7) / 8 + lanes - 1) / lanes * lanes;
  const int64_t most = std::max<int64_t>(1, (((int64_t)1 << 32) - 512) / a_row);
  for (int64_t at = 0; at < rows; at += most) {
    const int64_t n = std::min(rows - at, most);
    f(at, n, (uint32_t)((n * a_row + 255) / 256), (int)a_row);
  }
}

template <typename F>
void for_act(int act, bool gated, F&& f) {
  typedef std::integral_constant<int, TGRAD_ACT_SILU> silu;
  typedef std::integral_constant<int, TGRAD_ACT_GELU> gelu;
  if (act == TGRAD_ACT_SILU) gated ? f(silu(), std::true_type()) : f(silu(), std::false_type());
  else gated ? f(gelu(), std::true_type()) : f(gelu(), std::false_type());
}

}  // namespace

namespace tgrad {

void launch_quantize(hipStream_t s, const tgrad_matrix* x, const tgrad_codes* out) {
  const Mat m = mat(x);
  const Codes8 c = codes8(out);
  const int cols = (int)x->cols;
  for_real(x->dtype, [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    if (out->group == 0) {
      for_row(x->rows, cols, [&](auto t, auto n) {
        constexpr int T = decltype(t)::value, NV = decltype(n)::value;
        rows_in_launches(x->rows, T, 1, [&](int64_t first, int64_t rows) {
          k_quantize_rows<DT, T, NV><<<dim3((uint32_t)rows), dim3(T), 0, s>>>(m, first, cols, c);
        });
      });
    } else {
      for_units(x->rows, cols, out->group / 8, [&](int64_t first, int64_t rows, uint32_t grid, int a_row) {
        k_quantize_groups<DT><<<dim3(grid), dim3(256), 0, s>>>(m, first, rows, a_row, cols, c);
      });
    }
  });
}

}  // namespace tgrad

extern "C" {

int tgrad_quantize(const tgrad_matrix* x, const tgrad_codes* out, void* hip_stream) {
  if (!good(x) || !good(out) || !same_size(out, x->rows, x->cols)) return TGRAD_ERR_INVALID_ARG;
  if (pending()) return TGRAD_ERR_HIP;
  if (x->rows == 0) return TGRAD_OK;
  launch_quantize(static_cast<hipStream_t>(hip_stream), x, out);
  return launched();
}

int tgrad_dequantize(const tgrad_codes* codes, const tgrad_matrix* out, void* hip_stream) {
  if (!good(codes) || !good(out) || !same_size(out, codes->rows, codes->cols)) return TGRAD_ERR_INVALID_ARG;
  if (pending()) return TGRAD_ERR_HIP;
  if (out->rows == 0) return TGRAD_OK;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const Codes8 c = codes8(codes);
  const Mat m = mat(out);
  for_real(out->dtype, [&](auto dt) {
    for_units(out->rows, out->cols, 1, [&](int64_t first, int64_t rows, uint32_t grid, int a_row) {
      k_dequantize<decltype(dt)::value><<<dim3(grid), dim3(256), 0, s>>>(c, first, rows, a_row, (int)out->cols, m);
    });
  });
  return launched();
}

int tgrad_activation(const tgrad_matrix* x, const tgrad_matrix* gate, int act, const tgrad_matrix* y, const tgrad_codes* y8,
                     const tgrad_codes* x8, const tgrad_codes* gate8, void* hip_stream) {
  if (!good(x) || (act != TGRAD_ACT_SILU && act != TGRAD_ACT_GELU) || !y == !y8) return TGRAD_ERR_INVALID_ARG;
  if (gate && (!good(gate) || gate->dtype != x->dtype || !same_size(gate, x->rows, x->cols))) return TGRAD_ERR_INVALID_ARG;
  if (y && (!good(y) || y->dtype != x->dtype || !same_size(y, x->rows, x->cols))) return TGRAD_ERR_INVALID_ARG;
  if (y8 && (!good(y8) || y8->group != 0 || !same_size(y8, x->rows, x->cols))) return TGRAD_ERR_INVALID_ARG;
  if (x8 && (!good(x8) || x8->group == 0 || !same_size(x8, x->rows, x->cols))) return TGRAD_ERR_INVALID_ARG;
  if (gate8 && (!good(gate8) || gate8->group == 0 || !same_size(gate8, x->rows, x->cols))) return TGRAD_ERR_INVALID_ARG;
  if ((gate8 != nullptr) != (x8 && gate)) return TGRAD_ERR_INVALID_ARG;
  if (pending()) return TGRAD_ERR_HIP;
  if (x->rows == 0) return TGRAD_OK;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const int cols = (int)x->cols;
  const Mat mx = mat(x), mg = mat(gate), my = mat(y);
  const Codes8 cx = codes8(x8), cg = codes8(gate8), cy = codes8(y8);
  for_real(x->dtype, [&](auto dt) {
    for_act(act, gate != nullptr, [&](auto a, auto g) {
      constexpr int DT = decltype(dt)::value, ACT = decltype(a)::value;
      constexpr bool GATED = decltype(g)::value;
      if (y) {
        const int lanes = x8 ? std::max(x8->group, gate8 ? gate8->group : 0) / 8 : 1;
        for_units(x->rows, cols, lanes, [&](int64_t first, int64_t rows, uint32_t grid, int a_row) {
          k_activation<DT, ACT, GATED><<<dim3(grid), dim3(256), 0, s>>>(mx, mg, first, rows, a_row, cols, my, cx, cg);
        });
      } else {
        for_row(x->rows, cols, [&](auto t, auto n) {
          constexpr int T = decltype(t)::value, NV = decltype(n)::value;
          rows_in_launches(x->rows, T, 1, [&](int64_t first, int64_t rows) {
            if constexpr (T * NV == 4096) k_activation_rows<DT, ACT, GATED, 512, 4, 4><<<dim3((uint32_t)rows), dim3(512), 0, s>>>(mx, mg, first, cols, cy, cx, cg);
            else k_activation_rows<DT, ACT, GATED, T, NV, 0><<<dim3((uint32_t)rows), dim3(T), 0, s>>>(mx, mg, first, cols, cy, cx, cg);
          });
        });
      }
    });
  });
  return launched();
}

int tgrad_activation_backward(const tgrad_matrix* dy, const tgrad_codes* x8, const tgrad_codes* gate8, int act, const tgrad_matrix* dx,
                              const tgrad_matrix* dgate, void* hip_stream) {
  if (!good(dy) || !good(x8) || !good(dx) || (act != TGRAD_ACT_SILU && act != TGRAD_ACT_GELU)) return TGRAD_ERR_INVALID_ARG;
  if (!gate8 != !dgate || (gate8 && (!good(gate8) || !good(dgate)))) return TGRAD_ERR_INVALID_ARG;
  const int64_t n = dy->rows, m = dy->cols;
  if (!same_size(x8, n, m) || !same_size(dx, n, m) || dx->dtype != dy->dtype) return TGRAD_ERR_INVALID_ARG;
  if (gate8 && (!same_size(gate8, n, m) || !same_size(dgate, n, m) || dgate->dtype != dy->dtype)) return TGRAD_ERR_INVALID_ARG;
  if (pending()) return TGRAD_ERR_HIP;
  if (n == 0) return TGRAD_OK;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const Mat md = mat(dy), mx = mat(dx), mg = mat(dgate);
  const Codes8 cx = codes8(x8), cg = codes8(gate8);
  for_real(dy->dtype, [&](auto dt) {
    for_act(act, gate8 != nullptr, [&](auto a, auto g) {
      for_units(n, m, 1, [&](int64_t first, int64_t rows, uint32_t grid, int a_row) {
        k_activation_back<decltype(dt)::value, decltype(a)::value, decltype(g)::value>
            <<<dim3(grid), dim3(256), 0, s>>>(md, cx, cg, first, rows, a_row, (int)m, mx, mg);
      });
    });
  });
  return launched();
}

}  // extern "C"

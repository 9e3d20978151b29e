// Products with 8-bit codes: tokens times a weight, both as codes, and that product's two gradients, of which one factor is codes.
#include "block8.h"

using namespace tgrad;

namespace tgrad {
void launch_quantize(hipStream_t s, const tgrad_matrix* x, const tgrad_codes* out);
}

namespace {

// ---- codes times codes: 64 x 64 results a workgroup, 4 x 4 a thread, v_dot4_i32_i8 ------------------------------------------------

constexpr int kStep = 64;                 // bytes of the sum that are staged at a time
constexpr int kPitch = kStep + 4;         // an odd number of dwords: rows start in different banks

__device__ __forceinline__ Quad load16(const int8_t* p, int64_t n) {
  Quad q = {0, 0, 0, 0};
  if (n >= 16) {
    q = *reinterpret_cast<const QuadByte*>(p);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (i < n) q[i / 4] |= (uint32_t)(uint8_t)p[i] << (8 * (i % 4));
  }
  return q;
}

template <int OT>
__global__ __launch_bounds__(256) void k_int8_tile(Codes8 x, Codes8 w, int64_t tokens, int64_t outer, int inner, Mat y) {
  __shared__ uint32_t xs[64 * kPitch / 4], ws[64 * kPitch / 4];
  const int64_t t0 = (int64_t)blockIdx.y * 64, n0 = (int64_t)blockIdx.x * 64;
  const int r = threadIdx.x / 4, seg = threadIdx.x % 4;
  const int tr = threadIdx.x / 16, tc = threadIdx.x % 16;
  int acc[4][4] = {};
  for (int k0 = 0; k0 < inner; k0 += kStep) {
    const int at = k0 + seg * 16;
    Quad a = {0, 0, 0, 0}, b = {0, 0, 0, 0};
    if (t0 + r < tokens) a = load16(x.codes + (t0 + r) * x.stride + at, inner - at);
    if (n0 + r < outer) b = load16(w.codes + (n0 + r) * w.stride + at, inner - at);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      xs[r * (kPitch / 4) + seg * 4 + i] = a[i];
      ws[r * (kPitch / 4) + seg * 4 + i] = b[i];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kStep / 4; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[i][j] = __builtin_amdgcn_sdot4((int)xs[(tr + 16 * i) * (kPitch / 4) + k], (int)ws[(tc + 16 * j) * (kPitch / 4) + k], acc[i][j], false);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t t = t0 + tr + 16 * i, n = n0 + tc + 16 * j;
      if (t < tokens && n < outer)
        reinterpret_cast<typename Elem<OT>::raw*>(y.row(t))[n] = Elem<OT>::narrow(scaled(acc[i][j], x.scale[t], w.scale[n]));
    }
}

// ---- gradients: 64 x 64 results a workgroup, 4 x 4 a thread, float32 ---------------------------------------------------------------

template <int DT, int OT, bool WEIGHT>
__global__ __launch_bounds__(256) void k_grad_tile(Mat dy, Codes8 c, int64_t rows, int64_t cols, int64_t sum, Mat out) {
  __shared__ float as[16][65], bs[16][65];
  const int64_t r0 = (int64_t)blockIdx.y * 64, c0 = (int64_t)blockIdx.x * 64;
  const int tr = threadIdx.x / 16, tc = threadIdx.x % 16;
  typedef typename Elem<DT>::raw raw;
  float acc[4][4] = {};
  for (int64_t s0 = 0; s0 < sum; s0 += 16) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = threadIdx.x + 256 * i;
      const int s = WEIGHT ? e / 64 : e % 16, r = WEIGHT ? e % 64 : e / 16;
      float a = 0.f, b = 0.f;
      if (s0 + s < sum && r0 + r < rows) a = Elem<DT>::widen(WEIGHT ? reinterpret_cast<const raw*>(dy.row(s0 + s))[r0 + r] : reinterpret_cast<const raw*>(dy.row(r0 + r))[s0 + s]);
      const int bs_s = e / 64, k = e % 64;
      if (s0 + bs_s < sum && c0 + k < cols) {
        b = (float)c.codes[(s0 + bs_s) * c.stride + c0 + k] * c.scale[(s0 + bs_s) * c.groups + ((c0 + k) >> c.shift)];
        b = Elem<DT>::widen(Elem<DT>::narrow(in_float32(b)));
      }
      as[s][r] = a;
      bs[bs_s][k] = b;
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
      const int64_t r = r0 + tr + 16 * i, k = c0 + tc + 16 * j;
      if (r < rows && k < cols) reinterpret_cast<typename Elem<OT>::raw*>(out.row(r))[k] = Elem<OT>::narrow(acc[i][j]);
    }
}

// ---- host ---------------------------------------------------------------------------------------------------------------------------

size_t aligned(size_t n) { return (n + kScratchAlign - 1) / kScratchAlign * kScratchAlign; }

// Codes of x that nobody keeps: rows of a multiple of 16 bytes, and a scale each.
int64_t scratch_stride(int64_t inner) { return (inner + 15) / 16 * 16; }
size_t scratch_codes(int64_t tokens, int64_t inner) { return aligned((size_t)tokens * scratch_stride(inner)) + aligned((size_t)tokens * 4); }

void launch_product(hipStream_t s, const tgrad_codes* x, const tgrad_codes* w, const tgrad_matrix* y) {
  for_real(y->dtype, [&](auto t) {
    k_int8_tile<decltype(t)::value><<<dim3((uint32_t)((y->cols + 63) / 64), (uint32_t)((y->rows + 63) / 64)), dim3(256), 0, s>>>(
        codes8(x), codes8(w), y->rows, y->cols, (int)x->cols, mat(y));
  });
}

template <bool WEIGHT>
void launch_gradient(hipStream_t s, const tgrad_matrix* dy, const tgrad_codes* c, const tgrad_matrix* out) {
  const int64_t sum = WEIGHT ? dy->rows : dy->cols;
  for_real(dy->dtype, [&](auto t) {
    constexpr int DT = decltype(t)::value;
    const dim3 grid((uint32_t)((out->cols + 63) / 64), (uint32_t)((out->rows + 63) / 64));
    if (out->dtype == DT) k_grad_tile<DT, DT, WEIGHT><<<grid, dim3(256), 0, s>>>(mat(dy), codes8(c), out->rows, out->cols, sum, mat(out));
    else k_grad_tile<DT, TGRAD_F32, WEIGHT><<<grid, dim3(256), 0, s>>>(mat(dy), codes8(c), out->rows, out->cols, sum, mat(out));
  });
}

bool scratch_ok(const void* p) { return p && (uintptr_t)p % kScratchAlign == 0; }

template <bool WEIGHT>
int gradient(const tgrad_matrix* dy, const tgrad_codes* c, const tgrad_matrix* out, void* workspace_dev, void* hip_stream) {
  if (!good(dy) || !good(c) || !good(out) || !scratch_ok(workspace_dev)) return TGRAD_ERR_INVALID_ARG;
  if (out->dtype != dy->dtype && out->dtype != TGRAD_F32) return TGRAD_ERR_INVALID_ARG;
  if (c->rows != (WEIGHT ? dy->rows : dy->cols) || !same_size(out, WEIGHT ? dy->cols : dy->rows, c->cols)) return TGRAD_ERR_INVALID_ARG;
  if (pending()) return TGRAD_ERR_HIP;
  if (out->rows == 0) return TGRAD_OK;
  launch_gradient<WEIGHT>(static_cast<hipStream_t>(hip_stream), dy, c, out);
  return launched();
}

}  // namespace

extern "C" {

int tgrad_codes_query_size(int op, int64_t tokens, int64_t inner, int64_t outer, size_t* workspace_bytes) {
  if (!workspace_bytes || op < TGRAD_CODES_MATMUL || op > TGRAD_CODES_GRAD_WEIGHT) return TGRAD_ERR_INVALID_ARG;
  if (!extents_ok(tokens, inner, inner) || !extents_ok(outer, inner, inner)) return TGRAD_ERR_INVALID_ARG;
  *workspace_bytes = kScratchAlign + (op == TGRAD_CODES_LINEAR ? scratch_codes(tokens, inner) : 0);
  return TGRAD_OK;
}

int tgrad_codes_matmul(const tgrad_codes* x, const tgrad_codes* w, const tgrad_matrix* y, void* workspace_dev, void* hip_stream) {
  if (!good(x) || !good(w) || !good(y) || x->group || w->group || !scratch_ok(workspace_dev)) return TGRAD_ERR_INVALID_ARG;
  if (x->cols != w->cols || !same_size(y, x->rows, w->rows)) return TGRAD_ERR_INVALID_ARG;
  if (x->cols > TGRAD_CODES_MAX_INNER) return TGRAD_ERR_UNSUPPORTED;
  if (pending()) return TGRAD_ERR_HIP;
  if (y->rows == 0) return TGRAD_OK;
  launch_product(static_cast<hipStream_t>(hip_stream), x, w, y);
  return launched();
}

int tgrad_codes_linear(const tgrad_matrix* x, const tgrad_codes* w, const tgrad_codes* keep, const tgrad_matrix* y, void* workspace_dev,
                      void* hip_stream) {
  if (!good(x) || !good(w) || !good(y) || w->group || !scratch_ok(workspace_dev)) return TGRAD_ERR_INVALID_ARG;
  if (x->cols != w->cols || !same_size(y, x->rows, w->rows)) return TGRAD_ERR_INVALID_ARG;
  if (keep && (!good(keep) || keep->group || !same_size(keep, x->rows, x->cols))) return TGRAD_ERR_INVALID_ARG;
  if (x->cols > TGRAD_CODES_MAX_INNER) return TGRAD_ERR_UNSUPPORTED;
  if (pending()) return TGRAD_ERR_HIP;
  if (y->rows == 0) return TGRAD_OK;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  char* ws = static_cast<char*>(workspace_dev) + kScratchAlign;
  tgrad_codes own{ws, reinterpret_cast<float*>(ws + aligned((size_t)x->rows * scratch_stride(x->cols))), x->rows, x->cols, scratch_stride(x->cols), 0};
  const tgrad_codes* c = keep ? keep : &own;
  launch_quantize(s, x, c);
  launch_product(s, c, w, y);
  return launched();
}

int tgrad_codes_grad_input(const tgrad_matrix* dy, const tgrad_codes* w, const tgrad_matrix* dx, void* workspace_dev, void* hip_stream) {
  return gradient<false>(dy, w, dx, workspace_dev, hip_stream);
}

int tgrad_codes_grad_weight(const tgrad_matrix* dy, const tgrad_codes* x, const tgrad_matrix* dw, void* workspace_dev, void* hip_stream) {
  return gradient<true>(dy, x, dw, workspace_dev, hip_stream);
}

}  // extern "C"

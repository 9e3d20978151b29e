// A group of tensors of any types and sizes: global gradient norm, clipping, AdamW.
//
// The list of tensors lies in device memory and is cut into pieces of kPiece elements; a table says for every piece which
// tensor it belongs to, so that one launch serves any number of tensors and small ones cost no more than their bytes.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "launch_util.h"
#include "train_common.h"

using namespace tgrad;

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int64_t kPiece = 4096;          // elements
constexpr int kMaxSums = 1024;            // workgroups that leave a partial sum
constexpr int kTicketGrid = 256;          // up to this many, the last of them forms the norm
constexpr int kPut = 32;                  // tensors per launch that writes the list

struct Entry {                            // a tensor as the kernels see it
  void* grad;
  void* out;
  void* param;
  void* m;
  void* v;
  int64_t numel;
  int32_t grad_dtype, param_dtype;
  float lr_scale, weight_decay;
};

struct Piece {
  int32_t entry, index;                   // elements index * kPiece ... of that tensor
};

struct PutArgs {
  Entry e[kPut];
  int32_t first_piece[kPut];
};

// Writes entries first .. first + gridDim.x - 1, and their part of the table where `pieces` is not null.
__global__ void k_group_put(PutArgs a, int first, Entry* entries, Piece* pieces) {
  const int b = blockIdx.x;
  const Entry e = a.e[b];
  if (threadIdx.x == 0) entries[first + b] = e;
  if (!pieces) return;
  const int64_t n = (e.numel + kPiece - 1) / kPiece;
  for (int64_t i = threadIdx.x; i < n; i += blockDim.x) pieces[a.first_piece[b] + i] = Piece{first + b, (int32_t)i};
}

__global__ void k_group_zero(uint32_t* ticket) { *ticket = 0; }

// Real numbers of a piece: [first, first + count) of the tensor's.
struct Span {
  int64_t first;
  int count;
};
__device__ __forceinline__ Span piece_span(const Entry& e, int index, bool cplx) {
  const int64_t at = (int64_t)index * kPiece, left = e.numel - at;
  const int n = (int)(left < kPiece ? left : kPiece);
  return cplx ? Span{at * 2, n * 2} : Span{at, n};
}

template <typename F>
__device__ __forceinline__ void for_real(int real, F&& f) {
  if (real == TGRAD_F32) f(std::integral_constant<int, TGRAD_F32>());
  else if (real == TGRAD_BF16) f(std::integral_constant<int, TGRAD_BF16>());
  else f(std::integral_constant<int, TGRAD_F16>());
}

// U units of four numbers of a thread from unit `first` on; past the end the last one again.  LAST: nobody reads them again soon.  With
// that hint on loads and stores norm and scaling of 136 M complex64 took 545 us instead of 608, norm and AdamW of 478 M numbers 2365
// instead of 2488.
template <int DT, int U, bool LAST>
__device__ __forceinline__ void load_units(typename Four<DT>::type* q, const void* base, int64_t at, int first, int units) {
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = first + u * kThreads + (int)threadIdx.x;
    const typename Four<DT>::any* p = reinterpret_cast<const typename Four<DT>::any*>(
        static_cast<const typename Elem<DT>::raw*>(base) + at + (int64_t)(i < units ? i : units - 1) * 4);
    q[u] = LAST ? __builtin_nontemporal_load(p) : *p;
  }
}
template <int DT>
__device__ __forceinline__ void store_unit(void* base, int64_t at, int unit, const float* f) {
  __builtin_nontemporal_store(Four<DT>::narrow(f), reinterpret_cast<typename Four<DT>::any*>(
                                                       static_cast<typename Elem<DT>::raw*>(base) + at + (int64_t)unit * 4));
}
// Everything above is on its way before anything below: the compiler would move each load to the branch that uses it.
__device__ __forceinline__ void loads_issued() { asm volatile("" ::: "memory"); }

// sum |g|^2, bounded by the read: 136 M complex64 in 181 to 183 us, 5.7 TB/s and what the caches give besides.  Squares and sums in float64:
// the square of a float32 is exact there, and no finite gradient overflows.  Every workgroup leaves one partial sum; the last one to come
// adds them up in the order of the workgroups, so that the result does not depend on which one that is.
template <int DT>
__device__ __forceinline__ double piece_sumsq(const void* g, Span s) {
  constexpr int U = 4;
  const int units = s.count / 4, rest = s.count % 4;
  double acc[4] = {0., 0., 0., 0.};
  for (int first = 0; first < units; first += U * kThreads) {
    typename Four<DT>::type q[U];
    load_units<DT, U, false>(q, g, s.first, first, units);
    loads_issued();
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (first + u * kThreads + (int)threadIdx.x < units) {
        float f[4];
        Four<DT>::widen(q[u], f);
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[k] = fma((double)f[k], (double)f[k], acc[k]);
      }
    }
  }
  if ((int)threadIdx.x < rest) {
    const double v = (double)Elem<DT>::widen(static_cast<const typename Elem<DT>::raw*>(g)[s.first + units * 4 + threadIdx.x]);
    acc[0] = fma(v, v, acc[0]);
  }
  return (acc[0] + acc[1]) + (acc[2] + acc[3]);
}

struct NormArgs {
  double* sums;
  uint32_t* ticket;
  float max_norm;
  const double* add;
  tgrad_norm* out;
};

// The partial sums in the order of the workgroups that left them, and what follows from them.
__device__ __forceinline__ void finish_norm(const NormArgs& a, int n, double* lds) {
  double acc = 0.;
  for (int i = threadIdx.x; i < n; i += kThreads) acc += __hip_atomic_load(a.sums + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  acc = block_sum<kWaves>(acc, lds);
  if (threadIdx.x == 0) {
    if (a.add) acc += *a.add;
    const float norm = (float)sqrt(acc);
    const float c = norm == INFINITY ? 0.f : a.max_norm / (norm + 1e-6f);   // for max_norm = INFINITY too (no clipping)
    a.out->sumsq = acc;
    a.out->norm = norm;
    a.out->coef = c > 1.f ? 1.f : c;      // a NaN stays one
  }
}

// FINISH: the last workgroup to come does k_group_norm's work; which one that is does not change the result.  For few workgroups: the
// counter, with what it makes visible, costs every one of them some 50 ns, mostly behind one another (2048 of them: 90 us of 290; counters
// in two levels were no better), k_group_norm a launch.
template <bool FINISH>
__global__ __launch_bounds__(kThreads) void k_group_sumsq(const Entry* __restrict__ entries, const Piece* __restrict__ pieces,
                                                          int64_t npieces, NormArgs a) {
  __shared__ double lds[kWaves];
  __shared__ uint32_t last;
  double acc = 0.;
  for (int64_t p = blockIdx.x; p < npieces; p += gridDim.x) {
    const Piece pc = pieces[p];
    const Entry& e = entries[pc.entry];
    const Span s = piece_span(e, pc.index, complex_type(e.grad_dtype));
    for_real(real_type(e.grad_dtype), [&](auto dt) { acc += piece_sumsq<dt.value>(e.grad, s); });
  }
  acc = block_sum<kWaves>(acc, lds);
  if constexpr (!FINISH) {
    if (threadIdx.x == 0) a.sums[blockIdx.x] = acc;
  } else {
    if (threadIdx.x == 0) {
      __hip_atomic_store(a.sums + blockIdx.x, acc, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      last = __hip_atomic_fetch_add(a.ticket, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    finish_norm(a, gridDim.x, lds);
    if (threadIdx.x == 0) *a.ticket = 0;
  }
}

__global__ __launch_bounds__(kThreads) void k_group_norm(NormArgs a, int n) {
  __shared__ double lds[kWaves];
  finish_norm(a, n, lds);
}

template <int DT>
__device__ __forceinline__ void piece_scale(const void* g, void* out, Span s, float coef) {
  constexpr int U = 4;
  const int units = s.count / 4, rest = s.count % 4;
  for (int first = 0; first < units; first += U * kThreads) {
    typename Four<DT>::type q[U];
    load_units<DT, U, true>(q, g, s.first, first, units);
    loads_issued();
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = first + u * kThreads + (int)threadIdx.x;
      float f[4];
      Four<DT>::widen(q[u], f);
#pragma unroll
      for (int k = 0; k < 4; ++k) f[k] *= coef;
      if (i < units) store_unit<DT>(out, s.first, i, f);
    }
  }
  if ((int)threadIdx.x < rest) {
    typedef typename Elem<DT>::raw raw;
    const int64_t i = s.first + units * 4 + threadIdx.x;
    static_cast<raw*>(out)[i] = Elem<DT>::narrow(coef * Elem<DT>::widen(static_cast<const raw*>(g)[i]));
  }
}

// One workgroup per piece: workgroups that stay for more of them, one piece behind the other, are slower (norm and AdamW of
// 478 M numbers 2690 us instead of 2488).  136 M complex64: 382 to 385 us, 5.7 TB/s.
__global__ __launch_bounds__(kThreads) void k_group_scale(const Entry* __restrict__ entries, const Piece* __restrict__ pieces,
                                                          const tgrad_norm* norm) {
  const float coef = norm->coef;
  const Piece pc = pieces[blockIdx.x];
  const Entry& e = entries[pc.entry];
  if (coef == 1.f && e.out == e.grad) return;
  const Span s = piece_span(e, pc.index, complex_type(e.grad_dtype));
  for_real(real_type(e.grad_dtype), [&](auto dt) { piece_scale<dt.value>(e.grad, e.out, s, coef); });
}

struct AdamK {
  double lr;
  float beta1, beta2, one_beta1, one_beta2, inv_c1, inv_c2, eps;
  bool skip_nonfinite;
};
struct AdamRates {                         // a tensor's
  float decay, step;                       // 1 - lr wd; lr / (1 - beta1^tau)
};

// Four numbers: of four real elements, or of two complex ones, whose v are v[0] and v[1].
template <bool CX>
__device__ __forceinline__ void adamw_unit(const AdamK& h, AdamRates r, float coef, const float* g, float* p, float* m, float* v) {
  float gs[4], d[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    gs[k] = coef * g[k];
    m[k] = h.beta1 * m[k] + h.one_beta1 * gs[k];
  }
#pragma unroll
  for (int k = 0; k < (CX ? 2 : 4); ++k) {
    const float sq = CX ? gs[2 * k] * gs[2 * k] + gs[2 * k + 1] * gs[2 * k + 1] : gs[k] * gs[k];
    v[k] = h.beta2 * v[k] + h.one_beta2 * sq;
    d[k] = r.step / (sqrtf(v[k] * h.inv_c2) + h.eps);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) p[k] = r.decay * p[k] - d[CX ? k / 2 : k] * m[k];
}

template <int GR, int PR, bool CX>
__device__ __forceinline__ void piece_adamw(const Entry& e, int index, const AdamK& h, AdamRates r, float coef) {
  constexpr int U = 4;
  const Span s = piece_span(e, index, CX);
  const int64_t vfirst = CX ? s.first / 2 : s.first;
  const int units = s.count / 4, rest = s.count % 4;
  float* M = static_cast<float*>(e.m);
  float* V = static_cast<float*>(e.v);
  for (int first = 0; first < units; first += U * kThreads) {
    typename Four<GR>::type g[U];
    typename Four<PR>::type p[U];
    Quad m[U], v[U];
    load_units<GR, U, true>(g, e.grad, s.first, first, units);
    load_units<PR, U, true>(p, e.param, s.first, first, units);
    load_units<TGRAD_F32, U, true>(m, M, s.first, first, units);
    if constexpr (CX) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = first + u * kThreads + (int)threadIdx.x;
        const Duo w = *reinterpret_cast<const DuoAny*>(V + vfirst + (int64_t)(i < units ? i : units - 1) * 2);
        v[u] = Quad{w[0], w[1], 0u, 0u};
      }
    } else {
      load_units<TGRAD_F32, U, true>(v, V, vfirst, first, units);
    }
    loads_issued();
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = first + u * kThreads + (int)threadIdx.x;
      if (i < units) {
        float fg[4], fp[4], fm[4], fv[4];
        Four<GR>::widen(g[u], fg);
        Four<PR>::widen(p[u], fp);
        Four<TGRAD_F32>::widen(m[u], fm);
        Four<TGRAD_F32>::widen(v[u], fv);
        adamw_unit<CX>(h, r, coef, fg, fp, fm, fv);
        store_unit<PR>(e.param, s.first, i, fp);
        store_unit<TGRAD_F32>(M, s.first, i, fm);
        if constexpr (CX) *reinterpret_cast<DuoAny*>(V + vfirst + (int64_t)i * 2) = Duo{__float_as_uint(fv[0]), __float_as_uint(fv[1])};
        else store_unit<TGRAD_F32>(V, vfirst, i, fv);
      }
    }
  }
  // up to three real elements, or one complex element, by one thread each
  constexpr int W = CX ? 2 : 1;
  if ((int)threadIdx.x < rest / W) {
    const int64_t i = s.first + units * 4 + (int64_t)threadIdx.x * W, iv = vfirst + units * 4 / W + threadIdx.x;
    const typename Elem<GR>::raw* G = static_cast<const typename Elem<GR>::raw*>(e.grad);
    typename Elem<PR>::raw* P = static_cast<typename Elem<PR>::raw*>(e.param);
    float fg[4] = {0.f, 0.f, 0.f, 0.f}, fp[4] = {0.f, 0.f, 0.f, 0.f}, fm[4] = {0.f, 0.f, 0.f, 0.f}, fv[4] = {1.f, 1.f, 1.f, 1.f};
#pragma unroll
    for (int k = 0; k < W; ++k) {
      fg[k] = Elem<GR>::widen(G[i + k]);
      fp[k] = Elem<PR>::widen(P[i + k]);
      fm[k] = M[i + k];
    }
    fv[0] = V[iv];
    adamw_unit<CX>(h, r, coef, fg, fp, fm, fv);
#pragma unroll
    for (int k = 0; k < W; ++k) {
      P[i + k] = Elem<PR>::narrow(fp[k]);
      M[i + k] = fm[k];
    }
    V[iv] = fv[0];
  }
}

// Seven streams, 26 to 28 bytes a number: 478 M numbers with bf16 gradients in 2180 to 2200 us behind the norm, 5.7 TB/s.  Backwards: what
// k_group_sumsq has read last is still in the caches (norm and step 2320 us, forwards 2343).
__global__ __launch_bounds__(kThreads) void k_group_adamw(const Entry* __restrict__ entries, const Piece* __restrict__ pieces, AdamK h,
                                                          const tgrad_norm* norm) {
  const float coef = norm ? norm->coef : 1.f;
  if (h.skip_nonfinite && !(fabsf(norm->norm) < INFINITY)) return;
  const Piece pc = pieces[gridDim.x - 1 - blockIdx.x];
  const Entry& e = entries[pc.entry];
  const double lr = h.lr * (double)e.lr_scale;
  const AdamRates r{(float)(1. - lr * (double)e.weight_decay), (float)(lr * (double)h.inv_c1)};
  const bool cplx = complex_type(e.grad_dtype);
  for_real(real_type(e.grad_dtype), [&](auto g) {
    for_real(real_type(e.param_dtype), [&](auto p) {
      if (!cplx) piece_adamw<g.value, p.value, false>(e, pc.index, h, r, coef);
      else if constexpr (g.value != TGRAD_F16 && p.value != TGRAD_F16) piece_adamw<g.value, p.value, true>(e, pc.index, h, r, coef);
    });
  });
}

constexpr size_t kAlign = 256;
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

struct Layout {
  int64_t npieces = 0;
  size_t entries = 0, pieces = 0, sums = 0, ticket = 0, bytes = 0;
};

bool known_type(int32_t dt) { return dt >= TGRAD_C64 && dt <= TGRAD_F16; }
bool aligned(const void* p, int real) { return (uintptr_t)p % (uintptr_t)real_bytes(real) == 0; }

int layout(const tgrad_tensor* t, int64_t n, Layout* l) {
  if (!t || n < 1) return TGRAD_ERR_INVALID_ARG;
  if (n > ((int64_t)1 << 20)) return TGRAD_ERR_UNSUPPORTED;
  for (int64_t i = 0; i < n; ++i) {
    if (t[i].numel < 0) return TGRAD_ERR_INVALID_ARG;
    if (t[i].numel > ((int64_t)1 << 40)) return TGRAD_ERR_UNSUPPORTED;
    l->npieces += (t[i].numel + kPiece - 1) / kPiece;
    if (l->npieces > ((int64_t)1 << 31) - 1) return TGRAD_ERR_UNSUPPORTED;
  }
  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t at = o; o += align_up(bytes); return at; };
  l->entries = take((size_t)n * sizeof(Entry));
  l->pieces = take((size_t)l->npieces * sizeof(Piece));
  l->sums = take(kMaxSums * sizeof(double));
  l->ticket = take(sizeof(uint32_t));
  l->bytes = o;
  return TGRAD_OK;
}

int check_tensor(const tgrad_tensor& t) {
  if (!known_type(t.grad_dtype)) return TGRAD_ERR_INVALID_ARG;
  if (!(std::isfinite(t.lr_scale) && std::isfinite(t.weight_decay) && t.lr_scale >= 0.f && t.weight_decay >= 0.f))
    return TGRAD_ERR_INVALID_ARG;
  const int gr = real_type(t.grad_dtype);
  if (t.numel > 0 && !t.grad) return TGRAD_ERR_INVALID_ARG;
  if (!aligned(t.grad, gr) || !aligned(t.out, gr)) return TGRAD_ERR_INVALID_ARG;
  if (!t.param) return t.exp_avg || t.exp_avg_sq ? TGRAD_ERR_INVALID_ARG : TGRAD_OK;
  if (!known_type(t.param_dtype) || complex_type(t.param_dtype) != complex_type(t.grad_dtype)) return TGRAD_ERR_INVALID_ARG;
  if (t.numel > 0 && (!t.exp_avg || !t.exp_avg_sq)) return TGRAD_ERR_INVALID_ARG;
  if (!aligned(t.param, real_type(t.param_dtype)) || !aligned(t.exp_avg, TGRAD_F32) || !aligned(t.exp_avg_sq, TGRAD_F32))
    return TGRAD_ERR_INVALID_ARG;
  if (t.numel > 0 && (t.param == t.grad || t.exp_avg == t.exp_avg_sq || t.param == t.exp_avg || t.param == t.exp_avg_sq))
    return TGRAD_ERR_INVALID_ARG;
  return TGRAD_OK;
}

// Host record of a tensor: what a later bind may not change.
struct Kind {
  int64_t numel;
  int32_t grad_dtype, param_dtype;
  bool out, param;
};

}  // namespace

struct tgrad_group {
  Layout lay;
  char* ws;
  hipStream_t stream;
  std::vector<Kind> kinds;
  bool steps;                              // every tensor has a parameter and moments

  const Entry* entries() const { return reinterpret_cast<const Entry*>(ws + lay.entries); }
  const Piece* pieces() const { return reinterpret_cast<const Piece*>(ws + lay.pieces); }
};

namespace {

int launched() { return hipGetLastError() == hipSuccess ? TGRAD_OK : TGRAD_ERR_HIP; }
bool pending() { return hipPeekAtLastError() != hipSuccess; }

// The list goes to the device as kernel arguments: ordered on the stream, and the caller's array is free at once.
void put(tgrad_group* g, const tgrad_tensor* t, bool table) {
  const int64_t n = (int64_t)g->kinds.size();
  int64_t piece = 0;
  for (int64_t a = 0; a < n; a += kPut) {
    PutArgs args;
    const int cnt = (int)(n - a < kPut ? n - a : kPut);
    for (int j = 0; j < cnt; ++j) {
      const tgrad_tensor& x = t[a + j];
      args.e[j] = Entry{x.grad, x.out ? x.out : x.grad, x.param, x.exp_avg, x.exp_avg_sq, x.numel,
                        x.grad_dtype, x.param ? x.param_dtype : x.grad_dtype, x.lr_scale, x.weight_decay};
      args.first_piece[j] = (int32_t)piece;
      piece += (x.numel + kPiece - 1) / kPiece;
    }
    k_group_put<<<dim3(cnt), dim3(256), 0, g->stream>>>(args, (int)a, reinterpret_cast<Entry*>(g->ws + g->lay.entries),
                                                        table ? reinterpret_cast<Piece*>(g->ws + g->lay.pieces) : nullptr);
  }
}

// f(pieces, workgroups) for parts of the table, the last one first, whose launches stay below 2^32 threads.
template <typename F>
void by_pieces(const tgrad_group* g, F&& f) {
  constexpr int64_t kMost = (((int64_t)1 << 32) - 1) / kThreads;
  for (int64_t end = g->lay.npieces; end > 0; end -= kMost) {
    const int64_t first = end > kMost ? end - kMost : 0;
    f(g->pieces() + first, (uint32_t)(end - first));
  }
}

int sum_grid(const tgrad_group* g) {
  const int64_t most = std::min<int64_t>(compute_units() * 4, kMaxSums);
  return (int)std::max<int64_t>(1, std::min(g->lay.npieces, most));
}

}  // namespace

extern "C" {

int tgrad_group_query_size(const tgrad_tensor* tensors, int64_t n, size_t* workspace_bytes) {
  if (!workspace_bytes) return TGRAD_ERR_INVALID_ARG;
  Layout l;
  const int rc = layout(tensors, n, &l);
  if (rc == TGRAD_OK) *workspace_bytes = l.bytes;
  return rc;
}

int tgrad_group_init(tgrad_group** out, const tgrad_tensor* tensors, int64_t n, void* workspace_dev, void* hip_stream) {
  if (!out) return TGRAD_ERR_INVALID_ARG;
  *out = nullptr;
  Layout l;
  const int rc = layout(tensors, n, &l);
  if (rc != TGRAD_OK) return rc;
  if (!workspace_dev || (uintptr_t)workspace_dev % kAlign) return TGRAD_ERR_INVALID_ARG;
  for (int64_t i = 0; i < n; ++i)
    if (check_tensor(tensors[i]) != TGRAD_OK) return TGRAD_ERR_INVALID_ARG;
  if (pending()) return TGRAD_ERR_HIP;
  tgrad_group* g = new (std::nothrow) tgrad_group();
  if (!g) return TGRAD_ERR_INVALID_ARG;
  try {
    g->kinds.resize((size_t)n);
  } catch (...) {
    delete g;
    return TGRAD_ERR_INVALID_ARG;
  }
  g->lay = l;
  g->ws = static_cast<char*>(workspace_dev);
  g->stream = static_cast<hipStream_t>(hip_stream);
  g->steps = true;
  for (int64_t i = 0; i < n; ++i) {
    const tgrad_tensor& t = tensors[i];
    g->kinds[(size_t)i] = Kind{t.numel, t.grad_dtype, t.param_dtype, t.out != nullptr, t.param != nullptr};
    g->steps = g->steps && (t.param || t.numel == 0);
  }
  put(g, tensors, true);
  k_group_zero<<<dim3(1), dim3(1), 0, g->stream>>>(reinterpret_cast<uint32_t*>(g->ws + l.ticket));
  if (launched() != TGRAD_OK) {
    delete g;
    return TGRAD_ERR_HIP;
  }
  *out = g;
  return TGRAD_OK;
}

int tgrad_group_bind(tgrad_group* group, const tgrad_tensor* tensors) {
  if (!group || !tensors) return TGRAD_ERR_INVALID_ARG;
  for (size_t i = 0; i < group->kinds.size(); ++i) {
    const Kind& k = group->kinds[i];
    const tgrad_tensor& t = tensors[i];
    if (t.numel != k.numel || t.grad_dtype != k.grad_dtype || (t.out != nullptr) != k.out || (t.param != nullptr) != k.param ||
        (k.param && t.param_dtype != k.param_dtype) || check_tensor(t) != TGRAD_OK)
      return TGRAD_ERR_INVALID_ARG;
  }
  if (pending()) return TGRAD_ERR_HIP;
  put(group, tensors, false);
  return launched();
}

int tgrad_group_grad_norm(tgrad_group* group, float max_norm, const double* add_sumsq_dev, tgrad_norm* norm_dev) {
  if (!group || !norm_dev || !(max_norm >= 0.f) || (uintptr_t)norm_dev % 8 || (uintptr_t)add_sumsq_dev % 8)
    return TGRAD_ERR_INVALID_ARG;
  if (pending()) return TGRAD_ERR_HIP;
  const int grid = sum_grid(group);
  const NormArgs a{reinterpret_cast<double*>(group->ws + group->lay.sums), reinterpret_cast<uint32_t*>(group->ws + group->lay.ticket),
                   max_norm, add_sumsq_dev, norm_dev};
  if (grid <= kTicketGrid) {
    k_group_sumsq<true><<<dim3(grid), dim3(kThreads), 0, group->stream>>>(group->entries(), group->pieces(), group->lay.npieces, a);
  } else {
    k_group_sumsq<false><<<dim3(grid), dim3(kThreads), 0, group->stream>>>(group->entries(), group->pieces(), group->lay.npieces, a);
    k_group_norm<<<dim3(1), dim3(kThreads), 0, group->stream>>>(a, grid);
  }
  return launched();
}

int tgrad_group_scale(tgrad_group* group, const tgrad_norm* norm_dev) {
  if (!group || !norm_dev || (uintptr_t)norm_dev % 8) return TGRAD_ERR_INVALID_ARG;
  if (pending()) return TGRAD_ERR_HIP;
  by_pieces(group, [&](const Piece* pieces, uint32_t grid) {
    k_group_scale<<<dim3(grid), dim3(kThreads), 0, group->stream>>>(group->entries(), pieces, norm_dev);
  });
  return launched();
}

int tgrad_group_clip(tgrad_group* group, float max_norm, const double* add_sumsq_dev, tgrad_norm* norm_dev) {
  const int rc = tgrad_group_grad_norm(group, max_norm, add_sumsq_dev, norm_dev);
  return rc == TGRAD_OK ? tgrad_group_scale(group, norm_dev) : rc;
}

int tgrad_group_adamw(tgrad_group* group, const tgrad_adamw* hyper, int64_t t, const tgrad_norm* norm_dev) {
  if (!group || !hyper || t < 0 || !group->steps || (uintptr_t)norm_dev % 8) return TGRAD_ERR_INVALID_ARG;
  const tgrad_adamw& h = *hyper;
  if (!(std::isfinite(h.lr) && h.lr >= 0. && h.beta1 >= 0. && h.beta1 < 1. && h.beta2 >= 0. && h.beta2 < 1. &&
        std::isfinite(h.eps) && h.eps >= 0.) ||
      h.skip_nonfinite < 0 || h.skip_nonfinite > 1 || (h.skip_nonfinite && !norm_dev))
    return TGRAD_ERR_INVALID_ARG;
  if (pending()) return TGRAD_ERR_HIP;
  const double tau = (double)(t + 1);
  AdamK k;
  k.lr = h.lr;
  k.beta1 = (float)h.beta1;
  k.beta2 = (float)h.beta2;
  k.one_beta1 = (float)(1. - h.beta1);
  k.one_beta2 = (float)(1. - h.beta2);
  k.inv_c1 = (float)(1. / (1. - std::pow(h.beta1, tau)));
  k.inv_c2 = (float)(1. / (1. - std::pow(h.beta2, tau)));
  k.eps = (float)h.eps;
  k.skip_nonfinite = h.skip_nonfinite != 0;
  by_pieces(group, [&](const Piece* pieces, uint32_t grid) {
    k_group_adamw<<<dim3(grid), dim3(kThreads), 0, group->stream>>>(group->entries(), pieces, k, norm_dev);
  });
  return launched();
}

int tgrad_group_destroy(tgrad_group* group) {
  if (!group) return TGRAD_ERR_INVALID_ARG;
  delete group;
  return TGRAD_OK;
}

}  // extern "C"

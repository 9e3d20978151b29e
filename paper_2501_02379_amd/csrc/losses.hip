// The loss at the head of a training step, on logits x (rows, vocab): log-probabilities of given tokens, the clipped policy loss
// with a KL term, the preference loss on paired log ratios, and their gradients with respect to the logits.
//
// Both losses depend on a row through logp = z_y - lse, lse = log sum_v exp z_v (z = x / temperature), alone, so the gradient is
// d loss / d logp times (1[v = y] - exp(z_v - lse)) / temperature.  Exponentials are those of 2, of (x - max) log2(e) / temperature.
#include <hip/hip_runtime.h>

#include <cmath>

#include "launch_util.h"
#include "train_common.h"

using namespace tgrad;

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr double kLog2e = 1.4426950408889634;

struct Logits {
  const void* x;
  int64_t rows, stride;
  const int64_t* targets;
  int vocab;
  float scale;                            // 1 / temperature
  float scale2;                           // log2(e) / temperature
};

// Running maximum and sum of 2^((x - max) scale2).  A maximum of -inf belongs to a sum of nothing, 0; a NaN entry is no maximum and
// makes the sum NaN, and so does +inf.
struct Soft {
  float m, s;
};
__device__ __forceinline__ float soft_base(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ Soft soft_join(Soft a, Soft b, float scale2) {
  const float m = fmaxf(a.m, b.m), base = soft_base(m);
  return Soft{m, a.s * exp2f((a.m - base) * scale2) + b.s * exp2f((b.m - base) * scale2)};
}
__device__ __forceinline__ Soft soft_add(Soft a, float x, float scale2) {
  const float m = fmaxf(a.m, x), base = soft_base(m);
  return Soft{m, a.s * exp2f((a.m - base) * scale2) + exp2f((x - base) * scale2)};
}

// What a row needs: maximum and log of the sum, in units of z.
struct RowSum {
  float m;                                // maximum of x
  float log_s;                            // log sum exp((x - m) scale)
};

template <int DT>
__device__ __forceinline__ RowSum row_sum(const typename Elem<DT>::raw* x, int vocab, float scale2, Soft* lds) {
  Soft a{-INFINITY, 0.f};
  for (int i = threadIdx.x; i < vocab; i += kThreads) a = soft_add(a, Elem<DT>::widen(x[i]), scale2);
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const Soft b{__shfl_xor(a.m, d), __shfl_xor(a.s, d)};
    a = soft_join(a, b, scale2);
  }
  __syncthreads();
  if (lane_id() == 0) lds[threadIdx.x / kWave] = a;
  __syncthreads();
  a = lds[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) a = soft_join(a, lds[w], scale2);
  return RowSum{a.m, logf(a.s)};
}

// dlogits of a row: d (1[v = y] - exp(x scale - lse)) with d = dlogp * scale, given lse = m scale + log_s.
template <int DT>
__device__ __forceinline__ void row_gradient(const typename Elem<DT>::raw* x, typename Elem<DT>::raw* out, int vocab, int64_t y,
                                             float m, float log2_s, float scale2, float d) {
  for (int i = threadIdx.x; i < vocab; i += kThreads) {
    const float p = exp2f((Elem<DT>::widen(x[i]) - m) * scale2 - log2_s);
    out[i] = Elem<DT>::narrow(i == y ? d - d * p : -d * p);
  }
}

template <int DT>
__device__ __forceinline__ void row_zero(typename Elem<DT>::raw* out, int vocab) {
  for (int i = threadIdx.x; i < vocab; i += kThreads) out[i] = Elem<DT>::narrow(0.f);
}

template <int DT>
__global__ __launch_bounds__(kThreads) void k_logprobs(Logits L, const float* weight, float* logp, float* lse, float2* stat) {
  typedef typename Elem<DT>::raw raw;
  __shared__ Soft lds[kWaves];
  const int64_t n = blockIdx.x;
  const int64_t y = L.targets[n];
  const bool live = y >= 0 && y < L.vocab && (!weight || weight[n] != 0.f);
  RowSum r{0.f, 0.f};
  float lp = 0.f, l = 0.f;
  if (live) {
    const raw* x = static_cast<const raw*>(L.x) + n * L.stride;
    r = row_sum<DT>(x, L.vocab, L.scale2, lds);
    lp = (Elem<DT>::widen(x[y]) - r.m) * L.scale - r.log_s;
    l = r.m * L.scale + r.log_s;
  }
  if (threadIdx.x == 0) {
    if (logp) logp[n] = lp;
    if (lse) lse[n] = l;
    if (stat) stat[n] = make_float2(r.m, r.log_s);
  }
}

// stat: maximum and log of the sum of every row; lse instead where stat is null (then its rounding is the gradient's error).
template <int DT>
__global__ __launch_bounds__(kThreads) void k_logprobs_back(Logits L, const float* lse, const float2* stat, const float* dlogp,
                                                            void* dx, int64_t dstride) {
  typedef typename Elem<DT>::raw raw;
  const int64_t n = blockIdx.x;
  const int64_t y = L.targets[n];
  const float d = dlogp[n];
  raw* out = static_cast<raw*>(dx) + n * dstride;
  if (!(y >= 0 && y < L.vocab) || d == 0.f) return row_zero<DT>(out, L.vocab);
  const raw* x = static_cast<const raw*>(L.x) + n * L.stride;
  const float m = stat ? stat[n].x : 0.f, log_s = stat ? stat[n].y : lse[n];
  row_gradient<DT>(x, out, L.vocab, y, m, log_s * (float)kLog2e, L.scale2, d * L.scale);
}

struct PolicyArgs {
  float low, high;                        // the ratio's bounds
  float kl_beta;
  const float* weight;
  const float* advantage;
  const float* old_logp;
  const float* ref_logp;
  const float* dloss;
  float4* each;                           // every row's part of the four sums
  float* logp;
  void* dx;
  int64_t dstride;
};

template <int DT>
__global__ __launch_bounds__(kThreads) void k_policy(Logits L, PolicyArgs a) {
  typedef typename Elem<DT>::raw raw;
  __shared__ Soft lds[kWaves];
  const int64_t n = blockIdx.x;
  const int64_t y = L.targets[n];
  const float w = a.weight[n];
  const bool live = y >= 0 && y < L.vocab && w != 0.f;
  raw* out = a.dx ? static_cast<raw*>(a.dx) + n * a.dstride : nullptr;
  if (!live) {
    if (threadIdx.x == 0) {
      a.each[n] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (a.logp) a.logp[n] = 0.f;
    }
    if (out) row_zero<DT>(out, L.vocab);
    return;
  }
  const raw* x = static_cast<const raw*>(L.x) + n * L.stride;
  const float xy = Elem<DT>::widen(x[y]);
  const RowSum r = row_sum<DT>(x, L.vocab, L.scale2, lds);
  const float logp = (xy - r.m) * L.scale - r.log_s;
  const float adv = a.advantage[n];
  const float ratio = expf(logp - a.old_logp[n]);
  const float whole = ratio * adv, cut = fminf(fmaxf(ratio, a.low), a.high) * adv;
  const bool clipped = cut < whole;
  const float pg = clipped ? -cut : -whole;
  float dlogp = clipped ? 0.f : -whole, kl = 0.f;
  if (a.ref_logp) {
    const float d = a.ref_logp[n] - logp, e = expm1f(d);
    kl = e - d;
    if (a.kl_beta != 0.f) dlogp -= a.kl_beta * e;
  }
  if (threadIdx.x == 0) {
    const float term = a.kl_beta != 0.f ? pg + a.kl_beta * kl : pg;
    a.each[n] = make_float4(w * term, w * pg, w * kl, clipped ? w : 0.f);
    if (a.logp) a.logp[n] = logp;
  }
  if (!out) return;
  const float d = w * dlogp * (a.dloss ? *a.dloss : 1.f) * L.scale;
  if (d == 0.f) return row_zero<DT>(out, L.vocab);
  row_gradient<DT>(x, out, L.vocab, y, r.m, r.log_s * (float)kLog2e, L.scale2, d);
}

__global__ __launch_bounds__(kThreads) void k_policy_sums(const float4* each, int64_t rows, float* stats) {
  __shared__ double lds[kWaves];
  double s[4] = {0., 0., 0., 0.};
  for (int64_t n = threadIdx.x; n < rows; n += kThreads) {
    const float4 e = each[n];
    s[0] += e.x;
    s[1] += e.y;
    s[2] += e.z;
    s[3] += e.w;
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const double v = block_sum<kWaves>(s[q], lds);
    if (threadIdx.x == 0) stats[q] = (float)v;
  }
}

struct PairArgs {
  const int64_t* start;
  const float* weight;
  const float* ref_logp;
  const float* dloss;
  const float2* stat;
  float* dlogp;
  float* rewards;
  float* pair_loss;
  double beta, smoothing;
  int64_t pairs;
};

__device__ __forceinline__ double softplus(double x) { return fmax(x, 0.) + log1p(exp(-fabs(x))); }

// One workgroup per pair: both sums of log ratios, the pair's loss, and the gradient of every log-probability in it.  In float64:
// log ratios are small differences of large numbers, and there are few rows.
template <int DT>
__global__ __launch_bounds__(kThreads) void k_pairs(Logits L, PairArgs a) {
  typedef typename Elem<DT>::raw raw;
  __shared__ double lds[kWaves];
  const int64_t p = blockIdx.x;
  double reward[2];
  int64_t from[2], to[2];
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    const int64_t i = p + side * a.pairs;
    const int64_t f = a.start[i], t = a.start[i + 1];
    from[side] = f < 0 ? 0 : f < L.rows ? f : L.rows;
    to[side] = t < from[side] ? from[side] : t < L.rows ? t : L.rows;
    double s = 0.;
    for (int64_t n = from[side] + threadIdx.x; n < to[side]; n += kThreads) {
      const float w = a.weight[n];
      const int64_t y = L.targets[n];
      if (w == 0.f || y < 0 || y >= L.vocab) continue;
      const float2 st = a.stat[n];
      const float xy = Elem<DT>::widen(static_cast<const raw*>(L.x)[n * L.stride + y]);
      const double logp = ((double)xy - (double)st.x) * (double)L.scale - (double)st.y;
      s += (double)w * (logp - (double)a.ref_logp[n]);
    }
    reward[side] = a.beta * block_sum<kWaves>(s, lds);
  }
  const double h = reward[0] - reward[1];
  const double dh = a.beta * (a.smoothing / (1. + exp(-h)) - (1. - a.smoothing) / (1. + exp(h))) / (double)a.pairs *
                    (a.dloss ? (double)*a.dloss : 1.);
  if (threadIdx.x == 0) {
    a.rewards[p] = (float)reward[0];
    a.rewards[p + a.pairs] = (float)reward[1];
    a.pair_loss[p] = (float)((1. - a.smoothing) * softplus(-h) + a.smoothing * softplus(h));
  }
#pragma unroll
  for (int side = 0; side < 2; ++side)
    for (int64_t n = from[side] + threadIdx.x; n < to[side]; n += kThreads) {
      const float w = a.weight[n];
      a.dlogp[n] = w == 0.f ? 0.f : (float)((side ? -dh : dh) * (double)w);
    }
}

__global__ __launch_bounds__(kThreads) void k_pair_mean(const float* pair_loss, int64_t pairs, float* loss) {
  __shared__ double lds[kWaves];
  double s = 0.;
  for (int64_t p = threadIdx.x; p < pairs; p += kThreads) s += (double)pair_loss[p];
  s = block_sum<kWaves>(s, lds);
  if (threadIdx.x == 0) *loss = (float)(s / (double)pairs);
}

__global__ void k_zero_floats(float* p, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i < n) p[i] = 0.f;
}

constexpr size_t kAlign = 256;
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

int launched() { return hipGetLastError() == hipSuccess ? TGRAD_OK : TGRAD_ERR_HIP; }
bool pending() { return hipPeekAtLastError() != hipSuccess; }

bool float_ptr(const void* p) { return p && (uintptr_t)p % 4 == 0; }
bool float_ptr_or_null(const void* p) { return (uintptr_t)p % 4 == 0; }

int check_logits(const tgrad_logits* l, Logits* out) {
  if (!l) return TGRAD_ERR_INVALID_ARG;
  if (l->dtype != TGRAD_F32 && l->dtype != TGRAD_BF16 && l->dtype != TGRAD_F16) return TGRAD_ERR_INVALID_ARG;
  constexpr int64_t kMost = ((int64_t)1 << 31) - 1;
  if (l->rows < 0 || l->rows > kMost || l->vocab < 1 || l->vocab > kMost || l->row_stride < l->vocab) return TGRAD_ERR_INVALID_ARG;
  if (l->rows > 0 && l->row_stride > (((int64_t)1 << 62) / l->rows)) return TGRAD_ERR_INVALID_ARG;
  if (!(l->temperature > 0.f) || !std::isfinite(l->temperature)) return TGRAD_ERR_INVALID_ARG;
  const double inv = 1. / (double)l->temperature;
  if (!std::isfinite((float)(inv * kLog2e)) || (float)inv == 0.f) return TGRAD_ERR_INVALID_ARG;
  if (l->rows > 0 && (!l->data || !l->targets)) return TGRAD_ERR_INVALID_ARG;
  if ((uintptr_t)l->data % (uintptr_t)real_bytes(l->dtype) || (uintptr_t)l->targets % 8) return TGRAD_ERR_INVALID_ARG;
  *out = Logits{l->data, l->rows, l->row_stride, l->targets, (int)l->vocab, (float)inv, (float)(inv * kLog2e)};
  return TGRAD_OK;
}

int check_gradient(const tgrad_logits* l, const void* dx, int64_t stride) {
  if (stride < l->vocab || (l->rows > 0 && stride > (((int64_t)1 << 62) / l->rows))) return TGRAD_ERR_INVALID_ARG;
  if ((uintptr_t)dx % (uintptr_t)real_bytes(l->dtype)) return TGRAD_ERR_INVALID_ARG;
  if (dx == l->data && stride != l->row_stride) return TGRAD_ERR_INVALID_ARG;
  return TGRAD_OK;
}

template <typename F>
void for_type(int dt, F&& f) {
  if (dt == TGRAD_F32) f(std::integral_constant<int, TGRAD_F32>());
  else if (dt == TGRAD_BF16) f(std::integral_constant<int, TGRAD_BF16>());
  else f(std::integral_constant<int, TGRAD_F16>());
}

// Scratch of the losses.
struct Scratch {
  size_t each, stat, dlogp, pair_loss, bytes;
};
Scratch scratch(int64_t rows, int64_t pairs) {
  Scratch s;
  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t at = o; o += align_up(bytes); return at; };
  s.each = s.stat = take((size_t)rows * (pairs ? sizeof(float2) : sizeof(float4)));
  s.dlogp = take(pairs ? (size_t)rows * sizeof(float) : 0);
  s.pair_loss = take((size_t)pairs * sizeof(float));
  s.bytes = o ? o : kAlign;
  return s;
}

}  // namespace

extern "C" {

int tgrad_token_logprobs(const tgrad_logits* logits, float* logp, float* lse, void* hip_stream) {
  Logits L;
  const int rc = check_logits(logits, &L);
  if (rc != TGRAD_OK) return rc;
  if (!float_ptr_or_null(logp) || !float_ptr_or_null(lse)) return TGRAD_ERR_INVALID_ARG;
  if (pending()) return TGRAD_ERR_HIP;
  if (L.rows == 0 || (!logp && !lse)) return TGRAD_OK;
  for_type(logits->dtype, [&](auto dt) {
    k_logprobs<dt.value><<<dim3((uint32_t)L.rows), dim3(kThreads), 0, static_cast<hipStream_t>(hip_stream)>>>(L, nullptr, logp, lse,
                                                                                                            nullptr);
  });
  return launched();
}

int tgrad_token_logprobs_backward(const tgrad_logits* logits, const float* lse, const float* dlogp, void* dlogits,
                                  int64_t dlogits_stride, void* hip_stream) {
  Logits L;
  int rc = check_logits(logits, &L);
  if (rc != TGRAD_OK) return rc;
  rc = check_gradient(logits, dlogits, dlogits_stride);
  if (rc != TGRAD_OK) return rc;
  if (L.rows > 0 && (!float_ptr(lse) || !float_ptr(dlogp) || !dlogits)) return TGRAD_ERR_INVALID_ARG;
  if (pending()) return TGRAD_ERR_HIP;
  if (L.rows == 0) return TGRAD_OK;
  for_type(logits->dtype, [&](auto dt) {
    k_logprobs_back<dt.value><<<dim3((uint32_t)L.rows), dim3(kThreads), 0, static_cast<hipStream_t>(hip_stream)>>>(
        L, lse, nullptr, dlogp, dlogits, dlogits_stride);
  });
  return launched();
}

int tgrad_loss_query_size(int64_t rows, int64_t pairs, size_t* workspace_bytes) {
  if (!workspace_bytes || rows < 0 || rows >= ((int64_t)1 << 31) || pairs < 0 || pairs >= ((int64_t)1 << 30)) return TGRAD_ERR_INVALID_ARG;
  *workspace_bytes = scratch(rows, pairs).bytes;
  return TGRAD_OK;
}

int tgrad_policy_loss(const tgrad_logits* logits, const tgrad_policy* policy, const float* weight, const float* advantage,
                      const float* old_logp, const float* ref_logp, const float* dloss, void* workspace_dev, float* stats,
                      float* logp, void* dlogits, int64_t dlogits_stride, void* hip_stream) {
  Logits L;
  int rc = check_logits(logits, &L);
  if (rc != TGRAD_OK) return rc;
  if (!policy || !(policy->clip_low >= 0.f && policy->clip_low <= 1.f) || !(policy->clip_high >= 0.f) ||
      !std::isfinite(policy->clip_high) || !std::isfinite(policy->kl_beta))
    return TGRAD_ERR_INVALID_ARG;
  if (!workspace_dev || (uintptr_t)workspace_dev % kAlign || !float_ptr(stats)) return TGRAD_ERR_INVALID_ARG;
  if (L.rows > 0 && (!float_ptr(weight) || !float_ptr(advantage) || !float_ptr(old_logp))) return TGRAD_ERR_INVALID_ARG;
  if (!float_ptr_or_null(ref_logp) || !float_ptr_or_null(dloss) || !float_ptr_or_null(logp)) return TGRAD_ERR_INVALID_ARG;
  if (dlogits) {
    rc = check_gradient(logits, dlogits, dlogits_stride);
    if (rc != TGRAD_OK) return rc;
  }
  if (pending()) return TGRAD_ERR_HIP;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const Scratch sc = scratch(L.rows, 0);
  PolicyArgs a{1.f - policy->clip_low, 1.f + policy->clip_high, policy->kl_beta, weight, advantage, old_logp, ref_logp, dloss,
               reinterpret_cast<float4*>(static_cast<char*>(workspace_dev) + sc.each), logp, dlogits, dlogits_stride};
  if (L.rows > 0)
    for_type(logits->dtype, [&](auto dt) { k_policy<dt.value><<<dim3((uint32_t)L.rows), dim3(kThreads), 0, s>>>(L, a); });
  k_policy_sums<<<dim3(1), dim3(kThreads), 0, s>>>(a.each, L.rows, stats);
  return launched();
}

int tgrad_preference_loss(const tgrad_logits* logits, const tgrad_preference* preference, int64_t pairs,
                          const int64_t* seq_start, const float* weight, const float* ref_logp, const float* dloss,
                          void* workspace_dev, float* loss, float* rewards, float* logp, void* dlogits,
                          int64_t dlogits_stride, void* hip_stream) {
  Logits L;
  int rc = check_logits(logits, &L);
  if (rc != TGRAD_OK) return rc;
  if (!preference || !(preference->beta > 0.f) || !std::isfinite(preference->beta) || !(preference->label_smoothing >= 0.f) ||
      !(preference->label_smoothing <= 0.5f))
    return TGRAD_ERR_INVALID_ARG;
  if (pairs < 1 || pairs >= ((int64_t)1 << 30) || !seq_start || (uintptr_t)seq_start % 8) return TGRAD_ERR_INVALID_ARG;
  if (!workspace_dev || (uintptr_t)workspace_dev % kAlign || !float_ptr(loss) || !float_ptr(rewards)) return TGRAD_ERR_INVALID_ARG;
  if (L.rows > 0 && (!float_ptr(weight) || !float_ptr(ref_logp))) return TGRAD_ERR_INVALID_ARG;
  if (!float_ptr_or_null(dloss) || !float_ptr_or_null(logp)) return TGRAD_ERR_INVALID_ARG;
  if (dlogits) {
    rc = check_gradient(logits, dlogits, dlogits_stride);
    if (rc != TGRAD_OK) return rc;
  }
  if (pending()) return TGRAD_ERR_HIP;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const Scratch sc = scratch(L.rows, pairs);
  char* ws = static_cast<char*>(workspace_dev);
  float2* stat = reinterpret_cast<float2*>(ws + sc.stat);
  float* dlogp = reinterpret_cast<float*>(ws + sc.dlogp);
  float* pair_loss = reinterpret_cast<float*>(ws + sc.pair_loss);
  PairArgs a{seq_start, weight, ref_logp, dloss, stat, dlogp, rewards, pair_loss, preference->beta, preference->label_smoothing, pairs};
  for_type(logits->dtype, [&](auto dt) {
    if (L.rows > 0) {
      // rows that lie in no sequence
      k_zero_floats<<<dim3((uint32_t)((L.rows + 255) / 256)), dim3(256), 0, s>>>(dlogp, L.rows);
      k_logprobs<dt.value><<<dim3((uint32_t)L.rows), dim3(kThreads), 0, s>>>(L, weight, logp, nullptr, stat);
    }
    k_pairs<dt.value><<<dim3((uint32_t)pairs), dim3(kThreads), 0, s>>>(L, a);
    k_pair_mean<<<dim3(1), dim3(kThreads), 0, s>>>(pair_loss, pairs, loss);
    if (dlogits && L.rows > 0)
      k_logprobs_back<dt.value><<<dim3((uint32_t)L.rows), dim3(kThreads), 0, s>>>(L, nullptr, stat, dlogp, dlogits, dlogits_stride);
  });
  return launched();
}

}  // extern "C"

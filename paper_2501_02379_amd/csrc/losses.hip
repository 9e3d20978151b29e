// The loss at the head of a training step, on logits x (rows, vocab): log-probabilities of given tokens, the clipped policy loss
// with a KL term, the preference loss on paired log ratios, and their gradients with respect to the logits.
//
// Both losses depend on a row through logp = z_y - lse, lse = log sum_v exp z_v (z = x / temperature), alone, so the gradient is
// d loss / d logp times (1[v = y] - exp(z_v - lse)) / temperature.  There are some ten operations for every two to eight bytes: memory bounds
// all of it, and what counts is how often a row is read, how many bytes are on their way, and that arithmetic goes on under them.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>
#include <limits>
#include <type_traits>

#include "launch_util.h"
#include "train_common.h"

using namespace tgrad;

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr double kLog2e = 1.4426950408889634;
constexpr float kLn2 = 0.693147180559945f;

struct Logits {
  const void* x;
  int64_t rows, stride;
  const int64_t* targets;
  int64_t first;                          // the row of a launch's first workgroup
  int vocab;
  float temperature;
  float scale;                            // 1 / temperature
  float scale2;                           // log2(e) / temperature
  float high, low;                        // the same in two terms (see Fine)
  double bend;                            // scale2 / (log2(e) / temperature): 1, but for scale2's rounding
  __device__ __forceinline__ double nats() const { return 0.69314718055994531 * (2. - bend); }   // z = x scale2 nats()
};

// 16 bytes of a row.
template <int DT> struct Pack {
  typedef typename Elem<DT>::raw raw;
  static constexpr int N = 16 / sizeof(raw);
  static constexpr uint32_t kLowest = DT == TGRAD_F32 ? 0xFF800000u : DT == TGRAD_BF16 ? 0xFF80FF80u : 0xFC00FC00u;   // -inf
  // LAST: not read again soon
  template <bool LAST>
  static __device__ __forceinline__ Quad load(const raw* p) {
    const QuadAny* q = reinterpret_cast<const QuadAny*>(p);
    return LAST ? __builtin_nontemporal_load(q) : *q;
  }
  static __device__ __forceinline__ void store(raw* p, Quad v) { __builtin_nontemporal_store(v, reinterpret_cast<QuadAny*>(p)); }
  static __device__ __forceinline__ void widen(Quad v, float* f) {
    if constexpr (DT == TGRAD_F32) {
      Four<DT>::widen(v, f);
    } else {
      Four<DT>::widen(Duo{v[0], v[1]}, f);
      Four<DT>::widen(Duo{v[2], v[3]}, f + 4);
    }
  }
  static __device__ __forceinline__ Quad narrow(const float* f) {
    if constexpr (DT == TGRAD_F32) {
      return Four<DT>::narrow(f);
    } else {
      const Duo a = Four<DT>::narrow(f), b = Four<DT>::narrow(f + 4);
      return Quad{a[0], a[1], b[0], b[1]};
    }
  }
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }   // one instruction; 0 below 2^-126

// A running sum of 2^(x scale2 - b), b the largest x scale2 so far, rounded, or -kReach if that is more: one fused multiply-add an
// exponent.  (b is a float32, so its rounding is no error: the sum is relative to that very number.)  -inf, and masks of the type's
// lowest value, add 0; a NaN makes the sum NaN, and so does +inf.  Rows whose maximum lies beyond kReach either way, where an exponent
// would lose its fraction, are summed again (wide).
constexpr float kReach = 1048576.f;
struct alignas(8) Soft {
  float b, s;
};

// scale2 as the sums take it: one float32, or two more that make it up exactly.  Rounded to one it is up to 6e-8 off, and with it every
// exponent, the same way in every row; a sum of many small log ratios, as a preference loss forms it, sees that.  The first of the two
// has 16 bits, so that the second one's part is more than the first one's rounding takes away; it is positive, so that -inf stays -inf.
struct Plain {
  float whole;
  __device__ __forceinline__ float above(float x, float b) const { return fmaf(x, whole, -b); }
};
struct Fine {
  float whole, high, low;
  __device__ __forceinline__ float above(float x, float b) const { return fmaf(x, low, fmaf(x, high, -b)); }
};
template <bool FINE>
__device__ __forceinline__ auto scale_of(const Logits& L) {
  if constexpr (FINE) return Fine{L.scale2, L.high, L.low};
  else return Plain{L.scale2};
}

// The new terms are added up by themselves, four at a time: next to a sum that holds a large one each of the small ones would be rounded
// away, always downwards (-2.5e-8 of a row's sum at T = 0.7 and 3001 entries, -3e-9 this way).
template <int N, typename S>
__device__ __forceinline__ void soft_add(Soft& a, const float* x, S scale) {
  float m = x[0];
#pragma unroll
  for (int k = 1; k < N; ++k) m = fmaxf(m, x[k]);
  const float b = fmaxf(a.b, m * scale.whole);
  constexpr int C = N < 4 ? N : 4;
  float s[C];
#pragma unroll
  for (int k = 0; k < C; ++k) s[k] = exp2_fast(scale.above(x[k], b));
#pragma unroll
  for (int k = C; k < N; ++k) s[k % C] += exp2_fast(scale.above(x[k], b));
#pragma unroll
  for (int k = 1; k < C; ++k) s[0] += s[k];
  a = Soft{b, fmaf(a.s, exp2_fast(a.b - b), s[0])};
}
// Of all T threads, the same in every one.
template <int T>
__device__ __forceinline__ Soft soft_all(Soft a, Soft* lds) {
  float b = a.b;
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) b = fmaxf(b, __shfl_xor(b, d));
  float s = a.s * exp2_fast(a.b - b);
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) s += __shfl_xor(s, d);
  if constexpr (T == kWave) return Soft{b, s};
  if (lane_id() == 0) lds[threadIdx.x / kWave] = Soft{b, s};
  __syncthreads();
  Soft w[T / kWave];
#pragma unroll
  for (int i = 0; i < T / kWave; ++i) w[i] = lds[i];
  b = w[0].b;
#pragma unroll
  for (int i = 1; i < T / kWave; ++i) b = fmaxf(b, w[i].b);
  s = 0.f;
#pragma unroll
  for (int i = 0; i < T / kWave; ++i) s += w[i].s * exp2_fast(w[i].b - b);
  return Soft{b, s};
}

// Sum of a row: of 2^(x scale2 - ref), or, where it is wide, of 2^((x - ref) scale2 - rest), whose exponents are not above 0: the reference
// is the row's maximum, or a given log sum, that of these numbers as its rounding left it.
struct RowSum {
  float ref, s;
  bool wide;
  float rest = 0.f;
  // z_y - lse, lse in units of log2
  __device__ __forceinline__ float above(float x, float scale2) const {
    if (!wide) return fmaf(x, scale2, -ref);
    const float t = fmaf(x - ref, scale2, -rest);
    return t > 0.f ? 0.f : t;             // a NaN stays one
  }
  __device__ __forceinline__ float logp(float xy, float scale2) const { return (above(xy, scale2) - log2f(s)) * kLn2; }
  __device__ __forceinline__ float lse(const Logits& L) const {
    return (float)((wide ? (double)ref * (double)L.scale2 : (double)ref) * L.nats() + (double)(log2f(s) * kLn2));
  }
};

// The whole row again, one element at a time, relative to its maximum: exponents are exact at the maximum whatever its size.
template <int DT, int T, typename S>
__device__ __forceinline__ RowSum wide_sum(const typename Elem<DT>::raw* x, int vocab, S scale, Soft* lds) {
  float m = -INFINITY, s = 0.f;
  for (int i = threadIdx.x; i < vocab; i += T) m = fmaxf(m, Elem<DT>::widen(x[i]));
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
  __syncthreads();
  if (lane_id() == 0) lds[threadIdx.x / kWave].b = m;
  __syncthreads();
  for (int i = 0; i < T / kWave; ++i) m = fmaxf(m, lds[i].b);
  if constexpr (std::is_same<S, Fine>::value) {
    // numbers this large have few values and their exponents few roundings, the same ones in every row: in float64
    double t = 0.;
    const double fine = (double)scale.high + (double)scale.low;
    for (int i = threadIdx.x; i < vocab; i += T) t += exp2(((double)Elem<DT>::widen(x[i]) - (double)m) * fine);
    s = (float)block_sum<T / kWave>(t, reinterpret_cast<double*>(lds));
  } else {
    for (int i = threadIdx.x; i < vocab; i += T) s += exp2_fast((Elem<DT>::widen(x[i]) - m) * scale.whole);
    s = block_sum<T / kWave>(s, &lds->s);
  }
  return RowSum{m, s, true};
}

template <int DT, int T, typename S>
__device__ __forceinline__ RowSum row_sum(Soft a, const typename Elem<DT>::raw* x, int vocab, S scale, Soft* lds) {
  a = soft_all<T>(a, lds);
  if (a.b > -kReach && a.b < kReach) return RowSum{a.b, a.s, false};
  return wide_sum<DT, T>(x, vocab, scale, lds);
}

// A piece in flight.  ODD: rows of two-byte elements that start in the upper half of a four-byte word are read from that word on, five
// words for a piece, and shifted into place where they are used: loads of 16 bytes that are not aligned to 4 take twice as long (4096
// rows of 100003 bf16 numbers, every other row such a one, scored in 175 us, now 128; stores do not mind).  The first and the last word
// of such a row may lie across its ends by one element, which is not used.
template <bool ODD> struct Flight {
  Quad v;
  uint32_t more;
  __device__ __forceinline__ Quad settle() const {
    return Quad{__builtin_amdgcn_alignbit(v[1], v[0], 16), __builtin_amdgcn_alignbit(v[2], v[1], 16), __builtin_amdgcn_alignbit(v[3], v[2], 16),
                __builtin_amdgcn_alignbit(more, v[3], 16)};
  }
};
template <> struct Flight<false> {
  Quad v;
  __device__ __forceinline__ Quad settle() const { return v; }
};

// A row as a workgroup of T threads sees it: `head` elements, `full` pieces of 16 bytes, of which thread t's are t, t + T, ..., and a last
// few elements; those outside the pieces (`odd` of them) belong to the first threads, one each.
// Sums take head = 0: where the row lies in memory has then no part in their order, and they are the same bits at any address.
template <int DT, int T, bool ODD = false>
struct Row {
  typedef Pack<DT> P;
  typedef typename P::raw raw;
  typedef Flight<ODD> F;
  const raw* x;                           // the first piece
  int head, full, odd;
  __device__ __forceinline__ Row(const raw* p, int vocab, int up = 0) {
    head = up < vocab ? up : vocab;
    full = (vocab - head) / P::N;
    odd = vocab - full * P::N;
    x = p + head;
  }
  // elements from p to the next 16-byte boundary
  static __device__ __forceinline__ int to_boundary(const raw* p) { return (int)((0u - (uint32_t)(uintptr_t)p) & 15u) / (int)sizeof(raw); }
  // this thread's odd element, counted from the first piece
  __device__ __forceinline__ int64_t odd_at() const {
    const int t = (int)threadIdx.x;
    return t < head ? t - head : (int64_t)full * P::N + (t - head);
  }
  // U pieces of every thread, from `first` on; past the end: the last one again (masked in add())
  template <int U, bool LAST>
  __device__ __forceinline__ void load(F* q, int first) const {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = first + u * T + (int)threadIdx.x;
      const raw* p = x + (int64_t)(i < full ? i : full - 1) * P::N;
      if constexpr (ODD) {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(p - 1);
        q[u].v = P::template load<LAST>(p - 1);
        q[u].more = w[4];
      } else {
        q[u].v = P::template load<LAST>(p);
      }
    }
    asm volatile("" ::: "memory");        // all of them on their way: the compiler would move each to the branch that uses it
  }
  // two pieces at a time: one step of the running maximum for both
  template <int U, typename S>
  __device__ __forceinline__ void add(Soft& a, F* q, int first, S scale) const {
    static_assert(U % 2 == 0, "pieces are added in pairs");
#pragma unroll
    for (int u = 0; u < U; u += 2) {
      const int at = first + u * T;
      if (at >= full) break;
      float f[2 * P::N];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        Quad v = q[u + k].v = q[u + k].settle();
        if (at + 2 * T > full && at + k * T + (int)threadIdx.x >= full) v = Quad{P::kLowest, P::kLowest, P::kLowest, P::kLowest};
        P::widen(v, f + k * P::N);
      }
      soft_add<2 * P::N>(a, f, scale);
    }
  }
  // pieces first ... end - 1, read and forgotten
  template <int U, bool LAST, typename S>
  __device__ __forceinline__ void stream(Soft& a, int first, int end, S scale) const {
    for (; first < end; first += U * T) {
      F q[U];
      load<U, LAST>(q, first);
      add<U>(a, q, first, scale);
    }
  }
  template <typename S>
  __device__ __forceinline__ void add_odd(Soft& a, S scale) const {
    if ((int)threadIdx.x < odd) {
      const float f = Elem<DT>::widen(x[odd_at()]);
      soft_add<1>(a, &f, scale);
    }
  }
};

// Gradient of a row: -q 2^(x scale2 - ref) with q = d / sum, and d more at the target, d = d loss / d z_y / temperature.
template <int DT, int T, bool ODD = false>
struct RowGradient {
  typedef Pack<DT> P;
  typedef typename P::raw raw;
  typedef Row<DT, T, ODD> R;
  raw* out;                               // where the first piece's gradient goes
  RowSum sum;
  float scale2, q;
  __device__ __forceinline__ RowGradient(raw* o, RowSum r, float scale2_, float d) : out(o), sum(r), scale2(scale2_), q(d / r.s) {}
  __device__ __forceinline__ float at(float x) const { return -q * exp2_fast(sum.above(x, scale2)); }
  __device__ __forceinline__ void piece(Quad v, int i, int full) const {
    float f[P::N];
    P::widen(v, f);
#pragma unroll
    for (int k = 0; k < P::N; ++k) f[k] = -q * exp2_fast(fmaf(f[k], scale2, -sum.ref));
    if (i < full) P::store(out + (int64_t)i * P::N, P::narrow(f));
  }
  // elements first ... end - 1 of a row that was summed wide
  __device__ __forceinline__ void wide(const raw* x, raw* row, int64_t first, int64_t end) const {
    for (int64_t i = first + threadIdx.x; i < end; i += T) row[i] = Elem<DT>::narrow(at(Elem<DT>::widen(x[i])));
  }
  // pieces that add() has settled
  template <int U>
  __device__ __forceinline__ void pieces(const R& r, const typename R::F* v, int first) const {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (first + u * T >= r.full) break;
      piece(v[u].v, first + u * T + (int)threadIdx.x, r.full);
    }
  }
  template <int U>
  __device__ __forceinline__ void stream(const R& r, int first, int end) const {
    for (; first < end; first += U * T) {
      typename R::F v[U];
      r.template load<U, true>(v, first);
#pragma unroll
      for (int u = 0; u < U; ++u) v[u].v = v[u].settle();
      pieces<U>(r, v, first);
    }
  }
  __device__ __forceinline__ void odd(const R& r) const {
    if ((int)threadIdx.x < r.odd) {
      const int64_t i = r.odd_at();
      out[i] = Elem<DT>::narrow(at(Elem<DT>::widen(r.x[i])));
    }
  }
  // Behind everything else, by the thread that wrote this element before: its stores keep their order.
  __device__ __forceinline__ void target(const R& r, int64_t y, float xy, float d) const {
    const int64_t i = y - r.head, behind = i - (int64_t)r.full * P::N;
    const int owner = i < 0 ? (int)y : behind < 0 ? (int)(i / P::N) % T : r.head + (int)behind;
    if ((int)threadIdx.x == owner) out[i] = Elem<DT>::narrow(d + at(xy));
  }
};

template <int DT, int T>
__device__ __forceinline__ void row_zero(typename Elem<DT>::raw* out, int vocab) {
  const Row<DT, T> r(out, vocab, Row<DT, T>::to_boundary(out));
  typename Elem<DT>::raw* body = out + r.head;
  for (int i = threadIdx.x; i < r.full; i += T) Pack<DT>::store(body + (int64_t)i * Pack<DT>::N, Quad{0u, 0u, 0u, 0u});
  if ((int)threadIdx.x < r.odd) body[r.odd_at()] = Elem<DT>::narrow(0.f);
}

// f(true) for a row of two-byte elements that starts in the upper half of a four-byte word, f(false) for any other.
template <int DT, typename F>
__device__ __forceinline__ void with_parity(const typename Elem<DT>::raw* x, F&& f) {
  if constexpr (DT != TGRAD_F32) {
    if ((uintptr_t)x & 2) return f(std::true_type());
  }
  f(std::false_type());
}

// What a preference loss keeps of a row.
struct RowStat {
  double gap;                             // w (logp - ref_logp); 0 for an ignored row
  float ref, s;                           // its sum
  int32_t wide;
};

// AGAIN: the logits are read again soon, by the kernels behind this one in a preference loss, for which stat and dlogp (zero for the
// rows that lie in no sequence) are.  Log ratios are small differences of large numbers, and a reward adds up hundreds of them: the sum
// takes the scale in two terms, and the rest is formed in float64.  (With it 5721 rows of 100003 float16 numbers are scored in 156 us, without
// it in 154; a whole loss on short rows, 9000 bf16 numbers each, takes 2 % longer.)  Elsewhere this is the last read, and the hint for that
// is worth 10 %: 4096 rows of 131072 bf16 numbers, a quarter of them ignored, 136 us with it, 151 without; now 125, 6.4 TB/s.  8 pieces of
// every thread are on their way.
template <int DT, int T, bool AGAIN>
__global__ __launch_bounds__(T) void k_logprobs(Logits L, const float* weight, const float* ref_logp, float* logp, float* lse, RowStat* stat,
                                                float* dlogp) {
  typedef typename Elem<DT>::raw raw;
  __shared__ Soft lds[T / kWave];
  const int64_t n = L.first + blockIdx.x;
  const int64_t y = L.targets[n];
  const bool live = y >= 0 && y < L.vocab && (!weight || weight[n] != 0.f);
  RowSum r{0.f, 1.f, false};
  float xy = 0.f, lp = 0.f, l = 0.f;
  if (live) {
    const raw* x = static_cast<const raw*>(L.x) + n * L.stride;
    xy = Elem<DT>::widen(x[y]);
    with_parity<DT>(x, [&](auto odd) {
      const Row<DT, T, odd.value> row(x, L.vocab);
      const auto scale = scale_of<AGAIN>(L);
      Soft a{-kReach, 0.f};
      row.template stream<8, !AGAIN>(a, 0, row.full, scale);
      row.add_odd(a, scale);
      r = row_sum<DT, T>(a, x, L.vocab, scale, lds);
    });
    if constexpr (!AGAIN) {
      lp = r.logp(xy, L.scale2);
      l = r.lse(L);
    }
  }
  if (threadIdx.x == 0) {
    if constexpr (AGAIN) {
      double gap = 0.;
      if (live) {
        const double scale = (double)L.high + (double)L.low;
        const double above = r.wide ? ((double)xy - (double)r.ref) * scale : (double)xy * scale - (double)r.ref;
        const double p = (above - log2((double)r.s)) / kLog2e;
        gap = (double)weight[n] * (p - (double)ref_logp[n]);
        lp = (float)p;
        if (!r.wide) {                    // the gradient's kernel takes the scale in one term: the reference as that sees it
          const double ref = (double)r.ref * L.bend;
          r.ref = (float)ref;
          r.s *= exp2f((float)(ref - (double)r.ref));
        }
      }
      stat[n] = RowStat{gap, r.ref, r.s, r.wide};
      dlogp[n] = 0.f;
    }
    if (logp) logp[n] = lp;
    if (lse) lse[n] = l;
  }
}

struct PairMean {
  const float* pair_loss;
  int64_t pairs;
  float* loss;
};
template <int T>
__device__ __forceinline__ void pair_mean(const PairMean& a) {
  __shared__ double lds[T / kWave];
  double s = 0.;
  for (int64_t p = threadIdx.x; p < a.pairs; p += T) s += (double)a.pair_loss[p];
  s = block_sum<T / kWave>(s, lds);
  if (threadIdx.x == 0) *a.loss = (float)(s / (double)a.pairs);
}

// stat: what every row's sum was, or null and lse given.  `parts` workgroups of T threads share a row, U pieces a thread and no more: each
// loads, computes and stores once (with a workgroup that walks its row a loss on 5721 rows of 100003 float16 numbers took 563 us, so
// 501; the gradient alone now 321, 6.2 TB/s with what the memory-side cache still has).  Pieces start at 16-byte boundaries of the gradient.  The
// first workgroup forms the mean over `pairs` pairs besides.
template <int DT, int T, int U>
__global__ __launch_bounds__(T) void k_logprobs_back(Logits L, const float* lse, const RowStat* stat, const float* dlogp, void* dx,
                                                     int64_t dstride, int parts, PairMean mean) {
  typedef typename Elem<DT>::raw raw;
  if (blockIdx.x == 0 && mean.pairs > 0) pair_mean<T>(mean);
  const uint32_t row = blockIdx.x / (uint32_t)parts;
  const int part = (int)(blockIdx.x - row * (uint32_t)parts);
  const int64_t n = L.first + row;
  const int64_t y = L.targets[n];
  raw* out = static_cast<raw*>(dx) + n * dstride;
  const float d = dlogp[n] * L.scale;
  const raw* x = static_cast<const raw*>(L.x) + n * L.stride;
  const Row<DT, T> r(x, L.vocab, Row<DT, T>::to_boundary(out));
  const int first = part * U * T;
  if (!(y >= 0 && y < L.vocab) || d == 0.f) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = first + u * T + (int)threadIdx.x;
      if (i < r.full) Pack<DT>::store(out + r.head + (int64_t)i * Pack<DT>::N, Quad{0u, 0u, 0u, 0u});
    }
    if (part == 0 && (int)threadIdx.x < r.odd) out[r.head + r.odd_at()] = Elem<DT>::narrow(0.f);
    return;
  }
  RowSum sum;
  if (stat) {
    sum = RowSum{stat[n].ref, stat[n].s, stat[n].wide != 0};
  } else {                                // a reference near lse, and what its rounding leaves
    const double top = (double)lse[n] * (double)L.temperature;          // exact
    const double l2 = top * (double)L.scale2;
    sum.wide = !(fabs(l2) < (double)kReach);
    if (sum.wide) {
      sum.ref = fminf(fmaxf((float)top, -FLT_MAX), FLT_MAX);
      sum.s = 1.f;
      sum.rest = (float)((top - (double)sum.ref) * (double)L.scale2);
    } else {
      sum.ref = (float)l2;
      sum.s = exp2f((float)(l2 - (double)sum.ref));
    }
  }
  const RowGradient<DT, T> g(out + r.head, sum, L.scale2, d);
  // the target's element: by the thread that writes it (again) behind the others
  const int64_t i = y - r.head;
  const int piece = i >= 0 && i < (int64_t)r.full * Pack<DT>::N ? (int)(i / Pack<DT>::N) : -1;
  const bool here = piece >= 0 ? piece >= first && piece < first + U * T : part == 0;
  const float xy = here ? Elem<DT>::widen(x[y]) : 0.f;
  const bool plain = first < r.full && !sum.wide;
  typename Row<DT, T>::F v[U];
  if (plain) r.template load<U, true>(v, first);
  if constexpr (T > kWave) {
    if (out == x) __syncthreads();                   // the target's logit is read before anything is written
  }
  if (plain) {
    g.template pieces<U>(r, v, first);
  } else if (first < r.full) {
    const int last = first + U * T < r.full ? first + U * T : r.full;
    g.wide(r.x, g.out, (int64_t)first * Pack<DT>::N, (int64_t)last * Pack<DT>::N);
    if constexpr (T > kWave) __syncthreads();        // the target's element is another thread's here
  }
  if (part == 0) g.odd(r);
  if (here) g.target(r, y, xy, d);
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

template <int DT, int T, int NV, bool ODD>
__device__ __forceinline__ void policy_row(const Logits& L, const PolicyArgs& a, int64_t n, int64_t y, float w, const typename Elem<DT>::raw* x,
                                           typename Elem<DT>::raw* out, Soft* lds) {
  constexpr int kStream = 4;              // pieces in flight in the part that does not stay
  typedef Row<DT, T, ODD> R;
  const R r(x, L.vocab);
  const float xy = Elem<DT>::widen(x[y]);
  const float adv = a.advantage[n], old = a.old_logp[n], ref = a.ref_logp ? a.ref_logp[n] : 0.f, scale = a.dloss ? *a.dloss : 1.f;
  Soft run{-kReach, 0.f};
  typename R::F held[NV];
  // a whole number of batches, so that a piece belongs to the same thread whether it stays or not
  const int over = r.full - T * NV;
  const int start = over > 0 ? (over + kStream * T - 1) / (kStream * T) * (kStream * T) : 0;
  const Plain plain{L.scale2};
  r.template stream<kStream, false>(run, 0, start, plain);
  if (start < r.full) {
    r.template load<NV, true>(held, start);
    r.template add<NV>(run, held, start, plain);
  }
  r.add_odd(run, plain);
  const RowSum sum = row_sum<DT, T>(run, x, L.vocab, plain, lds);
  const float logp = sum.logp(xy, L.scale2);
  const float ratio = expf(logp - old);
  // an advantage of 0 takes the row out whatever its ratio, one beyond float32 too (logp - old above 88.7)
  const bool none = adv == 0.f && logp - old < INFINITY;
  const float whole = none ? 0.f : ratio * adv, cut = none ? 0.f : fminf(fmaxf(ratio, a.low), a.high) * adv;
  const bool clipped = cut < whole;
  const float pg = clipped ? -cut : -whole;
  float dlogp = clipped ? 0.f : -whole, kl = 0.f;
  if (a.ref_logp) {
    const float d = ref - logp, e = expm1f(d);
    kl = d < INFINITY ? e - d : d;         // a token of probability 0: infinite
    if (a.kl_beta != 0.f) dlogp -= a.kl_beta * e;
  }
  if (threadIdx.x == 0) {
    const float term = a.kl_beta != 0.f ? pg + a.kl_beta * kl : pg;
    a.each[n] = make_float4(w * term, w * pg, w * kl, clipped ? w : 0.f);
    if (a.logp) a.logp[n] = logp;
  }
  if (!out) return;
  const float d = w * dlogp * scale * L.scale;
  if (d == 0.f) return row_zero<DT, T>(out, L.vocab);
  const RowGradient<DT, T, ODD> g(out, sum, L.scale2, d);
  if (sum.wide) {
    g.wide(x, out, 0, L.vocab);
    if constexpr (T > kWave) __syncthreads();        // the target's element is another thread's here
  } else {
    if (start < r.full) g.template pieces<NV>(r, held, start);
    for (int first = start - kStream * T; first >= 0; first -= kStream * T) g.template stream<kStream>(r, first, first + kStream * T);
    g.odd(r);
  }
  g.target(r, y, xy, d);
}

// One workgroup of T threads per row; the last T NV pieces of 16 bytes stay in registers from the sum to the gradient, what lies
// before them in longer rows is read twice, the second time backwards.  8192 rows of 131072 bf16 numbers, a quarter ignored: 662 us,
// 5.7 TB/s, a copy's rate.  1024 of 200003 float32 numbers: 327 us, 6.2 TB/s with a fifth of the bytes read again (in LDS besides 3 % less,
// but rows of 150000 bf16 numbers 260 instead of 252).  2048 of 50001 bf16 numbers: 75 us, 4.9 TB/s, two rows a compute unit at a time in
// three rounds (four rows of 256 threads 87, one of 1024 90).
template <int DT, int T, int NV>
__global__ __launch_bounds__(T) void k_policy(Logits L, PolicyArgs a) {
  typedef typename Elem<DT>::raw raw;
  __shared__ Soft lds[T / kWave];
  const int64_t n = L.first + blockIdx.x;
  const int64_t y = L.targets[n];
  const float w = a.weight[n];
  raw* out = a.dx ? static_cast<raw*>(a.dx) + n * a.dstride : nullptr;
  if (!(y >= 0 && y < L.vocab && w != 0.f)) {
    if (threadIdx.x == 0) {
      a.each[n] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (a.logp) a.logp[n] = 0.f;
    }
    if (out) row_zero<DT, T>(out, L.vocab);
    return;
  }
  const raw* x = static_cast<const raw*>(L.x) + n * L.stride;
  with_parity<DT>(x, [&](auto odd) { policy_row<DT, T, NV, odd.value>(L, a, n, y, w, x, out, lds); });
}

// One workgroup: the four sums over all rows, in float64.
__global__ __launch_bounds__(1024) void k_policy_sums(const float4* each, int64_t rows, float* stats) {
  __shared__ double lds[16];
  constexpr int U = 8;                    // rows of a thread in flight
  double s[4] = {0., 0., 0., 0.};
  for (int64_t first = threadIdx.x; first < rows; first += U * 1024) {
    float4 e[U];
#pragma unroll
    for (int u = 0; u < U; ++u) e[u] = each[first + u * 1024 < rows ? first + u * 1024 : first];
    asm volatile("" ::: "memory");
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (first + u * 1024 < rows) {
        s[0] += e[u].x;
        s[1] += e[u].y;
        s[2] += e[u].z;
        s[3] += e[u].w;
      }
    }
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const double v = block_sum<16>(s[q], lds);
    if (threadIdx.x == 0) stats[q] = (float)v;
  }
}

struct PairArgs {
  const int64_t* start;
  const float* weight;
  const float* dloss;
  const RowStat* stat;
  float* dlogp;
  float* rewards;
  float* pair_loss;
  double beta, smoothing;
  int64_t pairs;
};

__device__ __forceinline__ double softplus(double x) { return fmax(x, 0.) + log1p(exp(-fabs(x))); }

// One workgroup per pair: both sums of log ratios, in float64, the pair's loss, and the gradient of every log-probability in it.
constexpr int kPairThreads = 512;
__global__ __launch_bounds__(kPairThreads) void k_pairs(int64_t rows, PairArgs a) {
  __shared__ double lds[kPairThreads / kWave];
  constexpr int U = 4;                    // rows of a thread in flight
  const int64_t p = blockIdx.x;
  double sum[2] = {0., 0.};
  int64_t from[2], to[2];
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    const int64_t i = p + side * a.pairs;
    const int64_t f = a.start[i], t = a.start[i + 1];
    from[side] = f < 0 ? 0 : f < rows ? f : rows;
    to[side] = t < from[side] ? from[side] : t < rows ? t : rows;
  }
#pragma unroll
  for (int side = 0; side < 2; ++side)
    for (int64_t n = from[side] + threadIdx.x; n < to[side]; n += U * kPairThreads) {
      double gap[U];
#pragma unroll
      for (int u = 0; u < U; ++u) gap[u] = a.stat[n + u * kPairThreads < to[side] ? n + u * kPairThreads : n].gap;
#pragma unroll
      for (int u = 0; u < U; ++u) sum[side] += n + u * kPairThreads < to[side] ? gap[u] : 0.;
    }
  const double chosen = a.beta * block_sum<kPairThreads / kWave>(sum[0], lds);
  const double rejected = a.beta * block_sum<kPairThreads / kWave>(sum[1], lds);
  const double h = chosen - rejected;
  const double dh = a.beta * (a.smoothing / (1. + exp(-h)) - (1. - a.smoothing) / (1. + exp(h))) / (double)a.pairs *
                    (a.dloss ? (double)*a.dloss : 1.);
  if (threadIdx.x == 0) {
    a.rewards[p] = (float)chosen;
    a.rewards[p + a.pairs] = (float)rejected;
    // without smoothing the second term is not there, also where softplus(h) is infinite (a rejected token of probability 0)
    a.pair_loss[p] = (float)((1. - a.smoothing) * softplus(-h) + (a.smoothing > 0. ? a.smoothing * softplus(h) : 0.));
  }
#pragma unroll
  for (int side = 0; side < 2; ++side)
    for (int64_t n = from[side] + threadIdx.x; n < to[side]; n += kPairThreads) {
      const float w = a.weight[n];
      a.dlogp[n] = w == 0.f ? 0.f : (float)((side ? -dh : dh) * (double)w);
    }
}

__global__ __launch_bounds__(kThreads) void k_pair_mean(PairMean mean) { pair_mean<kThreads>(mean); }

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
  if (l->rows < 0 || l->rows > kMost || l->vocab < 1 || l->vocab > kMost / 2 || l->row_stride < l->vocab) return TGRAD_ERR_INVALID_ARG;
  if (l->rows > 0 && l->row_stride > (((int64_t)1 << 62) / l->rows)) return TGRAD_ERR_INVALID_ARG;
  if (!(l->temperature > 0.f) || !std::isfinite(l->temperature)) return TGRAD_ERR_INVALID_ARG;
  const double inv = 1. / (double)l->temperature;
  if (!std::isfinite((float)(inv * kLog2e)) || (float)inv == 0.f) return TGRAD_ERR_INVALID_ARG;
  if (l->rows > 0 && (!l->data || !l->targets)) return TGRAD_ERR_INVALID_ARG;
  if ((uintptr_t)l->data % (uintptr_t)real_bytes(l->dtype) || (uintptr_t)l->targets % 8) return TGRAD_ERR_INVALID_ARG;
  const double scale = inv * kLog2e;
  float high = (float)scale;
  if ((double)high > scale) high = std::nextafterf(high, 0.f);
  uint32_t bits;
  std::memcpy(&bits, &high, 4);
  bits &= 0xFFFFFF00u;
  std::memcpy(&high, &bits, 4);
  const float low = std::max((float)(scale - (double)high), std::numeric_limits<float>::denorm_min());
  *out = Logits{l->data, l->rows, l->row_stride, l->targets, 0, (int)l->vocab, l->temperature, (float)inv, (float)scale, high, low, (double)(float)scale / scale};
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

// f(first, rows) for parts of the rows whose launches, `groups` workgroups of T threads a row, stay below 2^32 threads.
template <typename F>
void by_rows(const Logits& L, int T, int64_t groups, F&& f) {
  const int64_t most = std::max<int64_t>(1, (((int64_t)1 << 32) - 1) / (T * groups));
  for (int64_t at = 0; at < L.rows; at += most) {
    Logits some = L;
    some.first = at;
    f(some, (uint32_t)(std::min(L.rows - at, most) * groups));
  }
}

// Threads of a row: as many as have no more than 8 pieces each, the number on their way at a time, up to 256 (16384 rows of 3111 bf16
// numbers 20 us with a wavefront each, 38 with 256 threads; of 6111 float16 33 with 128, 46 with 256); 1024 where there are fewer rows
// than compute units (a call behind another, 1024 / 256 threads: 64 rows of 131072 bf16 numbers 10.8 / 14.6 us, one of 131072
// float32 numbers 12.4 / 18.9, 300 rows of 131072 bf16 numbers 23.3 / 21.1; 512 are never better).
template <int DT, bool AGAIN>
void launch_logprobs(hipStream_t s, const Logits& L, const float* weight, const float* ref_logp, float* logp, float* lse, RowStat* stat,
                     float* dlogp) {
  const int pieces = L.vocab / Pack<DT>::N;
  const int T = pieces <= 512 ? 64 : pieces <= 1024 ? 128 : L.rows > compute_units() ? 256 : 1024;
  by_rows(L, T, 1, [&](const Logits& some, uint32_t grid) {
    if (T == 64) k_logprobs<DT, 64, AGAIN><<<dim3(grid), dim3(64), 0, s>>>(some, weight, ref_logp, logp, lse, stat, dlogp);
    else if (T == 128) k_logprobs<DT, 128, AGAIN><<<dim3(grid), dim3(128), 0, s>>>(some, weight, ref_logp, logp, lse, stat, dlogp);
    else if (T == 256) k_logprobs<DT, 256, AGAIN><<<dim3(grid), dim3(256), 0, s>>>(some, weight, ref_logp, logp, lse, stat, dlogp);
    else k_logprobs<DT, 1024, AGAIN><<<dim3(grid), dim3(1024), 0, s>>>(some, weight, ref_logp, logp, lse, stat, dlogp);
  });
}

template <int DT, int T, int U>
void launch_logprobs_back_as(hipStream_t s, const Logits& L, const float* lse, const RowStat* stat, const float* dlogp, void* dx,
                             int64_t dstride, PairMean mean) {
  const int64_t pieces = L.vocab / Pack<DT>::N;
  const int64_t parts = std::max<int64_t>(1, (pieces + U * T - 1) / (U * T));
  by_rows(L, T, parts, [&](const Logits& some, uint32_t grid) {
    k_logprobs_back<DT, T, U><<<dim3(grid), dim3(T), 0, s>>>(some, lse, stat, dlogp, dx, dstride, (int)parts, mean);
    mean.pairs = 0;
  });
}

// One workgroup for a row of up to 2048 pieces, 8 for every thread; parts of 512 pieces of longer ones (a loss on 14403 rows of 3111 bf16
// numbers 51 us with 64 threads of 8 pieces, 57 with parts; 10354 of 12345 float16 109 with 256 of 8, 138 with parts; 5721 of 100003 float16
// 501 in parts of 512 pieces, 512 of 2048).
template <int DT>
void launch_logprobs_back(hipStream_t s, const Logits& L, const float* lse, const RowStat* stat, const float* dlogp, void* dx,
                          int64_t dstride, PairMean mean) {
  const int pieces = L.vocab / Pack<DT>::N;
  if (pieces <= 256) launch_logprobs_back_as<DT, 64, 4>(s, L, lse, stat, dlogp, dx, dstride, mean);
  else if (pieces <= 512) launch_logprobs_back_as<DT, 64, 8>(s, L, lse, stat, dlogp, dx, dstride, mean);
  else if (pieces <= 1024) launch_logprobs_back_as<DT, 128, 8>(s, L, lse, stat, dlogp, dx, dstride, mean);
  else if (pieces <= 2048) launch_logprobs_back_as<DT, 256, 8>(s, L, lse, stat, dlogp, dx, dstride, mean);
  else launch_logprobs_back_as<DT, 256, 2>(s, L, lse, stat, dlogp, dx, dstride, mean);
}

template <int DT, int T, int NV>
void launch_policy_as(hipStream_t s, const Logits& L, const PolicyArgs& a) {
  by_rows(L, T, 1, [&](const Logits& some, uint32_t grid) { k_policy<DT, T, NV><<<dim3(grid), dim3(T), 0, s>>>(some, a); });
}

// The fewest threads whose registers hold the row, but not more than they need: several rows then share a compute unit, and one loads
// while another computes.  (The next larger one, us: 16384 rows of 4096 bf16 numbers 66, with 128 threads 56.5; 4096 of 24000 79, with 512
// threads of 8 pieces 74.7; a call with its sums.)
template <int DT>
void launch_policy(hipStream_t s, const Logits& L, const PolicyArgs& a) {
  const int pieces = L.vocab / Pack<DT>::N;
  if (pieces <= 64 * 4) launch_policy_as<DT, 64, 4>(s, L, a);
  else if (pieces <= 128 * 4) launch_policy_as<DT, 128, 4>(s, L, a);
  else if (pieces <= 256 * 4) launch_policy_as<DT, 256, 4>(s, L, a);
  else if (pieces <= 256 * 8) launch_policy_as<DT, 256, 8>(s, L, a);
  else if (pieces <= 512 * 8) launch_policy_as<DT, 512, 8>(s, L, a);
  else if (pieces <= 512 * 16) launch_policy_as<DT, 512, 16>(s, L, a);
  else launch_policy_as<DT, 1024, 16>(s, L, a);
}

constexpr int64_t kMostPairs = (int64_t)1 << 22;   // a workgroup for each

// Scratch of the losses.
struct Scratch {
  size_t each, stat, dlogp, pair_loss, bytes;
};
Scratch scratch(int64_t rows, int64_t pairs) {
  Scratch s;
  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t at = o; o += align_up(bytes); return at; };
  s.each = s.stat = take((size_t)rows * (pairs ? sizeof(RowStat) : sizeof(float4)));
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
    launch_logprobs<dt.value, false>(static_cast<hipStream_t>(hip_stream), L, nullptr, nullptr, logp, lse, nullptr, nullptr);
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
    launch_logprobs_back<dt.value>(static_cast<hipStream_t>(hip_stream), L, lse, nullptr, dlogp, dlogits, dlogits_stride, PairMean{nullptr, 0, nullptr});
  });
  return launched();
}

int tgrad_loss_query_size(int64_t rows, int64_t pairs, size_t* workspace_bytes) {
  if (!workspace_bytes || rows < 0 || rows >= ((int64_t)1 << 31) || pairs < 0 || pairs >= kMostPairs) return TGRAD_ERR_INVALID_ARG;
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
    for_type(logits->dtype, [&](auto dt) { launch_policy<dt.value>(s, L, a); });
  k_policy_sums<<<dim3(1), dim3(1024), 0, s>>>(a.each, L.rows, stats);
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
  if (pairs < 1 || pairs >= kMostPairs || !seq_start || (uintptr_t)seq_start % 8) return TGRAD_ERR_INVALID_ARG;
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
  RowStat* stat = reinterpret_cast<RowStat*>(ws + sc.stat);
  float* dlogp = reinterpret_cast<float*>(ws + sc.dlogp);
  float* pair_loss = reinterpret_cast<float*>(ws + sc.pair_loss);
  PairArgs a{seq_start, weight, dloss, stat, dlogp, rewards, pair_loss, preference->beta, preference->label_smoothing, pairs};
  const PairMean mean{pair_loss, pairs, loss};
  for_type(logits->dtype, [&](auto dt) {
    if (L.rows > 0) launch_logprobs<dt.value, true>(s, L, weight, ref_logp, logp, nullptr, stat, dlogp);
    k_pairs<<<dim3((uint32_t)pairs), dim3(kPairThreads), 0, s>>>(L.rows, a);
    if (dlogits && L.rows > 0) launch_logprobs_back<dt.value>(s, L, nullptr, stat, dlogp, dlogits, dlogits_stride, mean);
    else k_pair_mean<<<dim3(1), dim3(kThreads), 0, s>>>(mean);
  });
  return launched();
}

}  // extern "C"

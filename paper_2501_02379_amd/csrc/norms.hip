// The norms after and before a block, the gate and the scale of its residual branch, forward and backward:
//   x' = x + alpha gate (norm(b) w_post),  h = norm(x') w_pre.
//
// With n the normed vector and r its factor 1 / sqrt(mean((v - m)^2) + eps), a gradient u with respect to n goes on as
// r (u - n mean(u n) [- mean(u)]).  Forward two reads and two writes a number, backward four and two, for 14 and 26 operations: memory bounds both, so a
// row is read once and kept in registers through its sums.  (Backward up to 8192 columns: see k_block_norm_sums.)
#include "block8.h"

using namespace tgrad;

namespace {

// Sums over a workgroup, the same in every thread; each call has its own `lds`, so that one barrier does.
template <int WAVES>
__device__ __forceinline__ float2 sums_of_block(float2 v, float2* lds) {
  v.x = sum_of_lanes(v.x);
  v.y = sum_of_lanes(v.y);
  if constexpr (WAVES == 1) return v;
  if (lane_id() == 0) lds[threadIdx.x / kWave] = v;
  __syncthreads();
  v = lds[0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) {
    v.x += lds[w].x;
    v.y += lds[w].y;
  }
  return v;
}
template <int WAVES>
__device__ __forceinline__ float sum_of_block(float v, float* lds) {
  v = sum_of_lanes(v);
  if constexpr (WAVES == 1) return v;
  if (lane_id() == 0) lds[threadIdx.x / kWave] = v;
  __syncthreads();
  v = lds[0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) v += lds[w];
  return v;
}

struct Desc {
  const void *post, *pre;
  Mat gate;
  int64_t shared;                         // rows of the matrix to one row of the gate
  int weight_dtype, cols;
  bool centered;
  float scale, eps;
};

// Mean and factor of a row held in registers (numbers beyond its end are 0 there).  The mean is taken off before squares are summed.
template <int T, int NV>
__device__ __forceinline__ float2 stats_of(float (*v)[8], const Desc& d, float (*lds)[T / kWave]) {
  float mean = 0.f;
  if (d.centered) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int k = 0; k < 8; ++k) s += v[i][k];
    mean = sum_of_block<T / kWave>(s, lds[0]) / (float)d.cols;
  }
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int col = (threadIdx.x + i * T) * 8;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float c = col + k < d.cols ? v[i][k] - mean : 0.f;
      s += c * c;
    }
  }
  s = sum_of_block<T / kWave>(s, lds[1]);
  return make_float2(mean, 1.f / sqrtf(s / (float)d.cols + d.eps));
}

// A workgroup a row.  8192^2 bf16: 85 us on what the memory-side cache partly holds, 105 on other buffers every time (537 MB, 5.1 TB/s); 4096 x 5120 with a float32
// stream 42.  (Workgroups that go from row to row with the next row's loads ahead hold twice the registers, and half as many rows a compute unit were
// slower: 65536 x 512 71 us for 45, 2048 x 32768 311 for 125.)
template <int XT, int BT, bool BLOCK, int T, int NV>
__global__ __launch_bounds__(T) void k_block_norm(Desc d, int64_t first, Mat x, Mat block, Mat x_out, Mat h, Codes8 h8, float4* stats) {
  __shared__ float lds[4][T / kWave];
  __shared__ uint32_t lds_top[T / kWave];
  const int64_t row = first + blockIdx.x;
  constexpr int xs = sizeof(typename Elem<XT>::raw), bs = sizeof(typename Elem<BT>::raw);
  Eight<XT> ex[NV];
  float v[NV][8];
  float4 st = make_float4(0.f, 1.f, 0.f, 1.f);
  if constexpr (BLOCK) {
    Eight<BT> eb[NV], eg[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (threadIdx.x + i * T) * 8;
      ex[i].clear();
      eb[i].clear();
      eg[i].clear();
      if (col < d.cols) {
        ex[i].load(x.row(row) + (int64_t)col * xs, d.cols - col);
        eb[i].load(block.row(row) + (int64_t)col * bs, d.cols - col);
        if (d.gate.data) eg[i].load(d.gate.row(row / d.shared) + (int64_t)col * bs, d.cols - col);
      }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) eb[i].get(v[i]);
    if (d.post) {
      const float2 m = stats_of<T, NV>(v, d, lds);
      st.x = m.x;
      st.y = m.y;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (threadIdx.x + i * T) * 8;
      float f[8], w[8], g[8];
      ex[i].get(f);
      eg[i].get(g);
      if (d.post && col < d.cols) load_weights(d.post, d.weight_dtype, col, d.cols - col, w);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        float o = v[i][k];
        if (d.post) o = (o - st.x) * st.y * w[k];
        f[k] += d.scale * (d.gate.data ? g[k] * o : o);
      }
      ex[i].set(f);
      if (col < d.cols) ex[i].store(x_out.row(row) + (int64_t)col * xs, d.cols - col);
    }
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (threadIdx.x + i * T) * 8;
      ex[i].clear();
      if (col < d.cols) ex[i].load(x.row(row) + (int64_t)col * xs, d.cols - col);
    }
  }
  if (d.pre) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (threadIdx.x + i * T) * 8;
      ex[i].get(v[i]);
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (col + k >= d.cols) v[i][k] = 0.f;
    }
    const float2 m = stats_of<T, NV>(v, d, lds + 2);
    st.z = m.x;
    st.w = m.y;
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (threadIdx.x + i * T) * 8;
      float w[8];
      if (col < d.cols) load_weights(d.pre, d.weight_dtype, col, d.cols - col, w);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[i][k] = col + k < d.cols ? (v[i][k] - st.z) * st.w * w[k] : 0.f;
      top = max(top, largest(v[i]));
      if (h.data && col < d.cols) {
        Eight<BT> o;
        o.set(v[i]);
        o.store(h.row(row) + (int64_t)col * bs, d.cols - col);
      }
    }
    if (h8.codes) {
      const Rounding r = rounding_of(largest_of_block<T / kWave>(top, lds_top));
      if (threadIdx.x == 0) h8.scale[row] = r.scale;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int col = (threadIdx.x + i * T) * 8;
        if (col < d.cols) store_codes(h8.codes + row * h8.stride + col, codes_of(v[i], r), d.cols - col);
      }
    }
  }
  if (stats && threadIdx.x == 0) stats[row] = st;
}

// ---- backward ----------------------------------------------------------------------------------------------------------------

// The rows in chunks, a workgroup for each, which adds its rows up column by column in registers.  A chunk lies within one row of the gate
// (`per_gate` chunks to each) or holds several of them whole (per_gate = 1).
struct Chunks {
  int64_t count, rows, per_gate, span;    // span: rows of the matrix to `per_gate` chunks
};

constexpr int kHeldCols = 8192;           // a row that one workgroup holds

Chunks chunks_of(int64_t rows, int64_t cols, int64_t shared) {
  const int64_t most = cols > kHeldCols ? 128 : cols > 4096 ? 256 : cols > 2048 ? 512 : cols > 512 ? 1024 : 4096;
  const int64_t want = std::max<int64_t>(1, (rows + most - 1) / most);
  Chunks c;
  shared = std::min(shared, std::max<int64_t>(rows, 1));
  if (shared > want) {
    c.per_gate = (shared + want - 1) / want;
    c.rows = (shared + c.per_gate - 1) / c.per_gate;
    c.span = shared;
    c.count = (rows + shared - 1) / shared * c.per_gate;
  } else {
    c.rows = want / shared * shared;
    c.per_gate = 1;
    c.span = c.rows;
    c.count = (rows + c.rows - 1) / c.rows;
  }
  return c;
}

struct Back {
  Mat dx_out, dh, x_out, block, dx, dblock;
  const float4* stats;
  float4* sums;                           // of every row, where it is longer than kHeldCols: along and off of both norms
  char* dgate;                            // rows of cols elements of the block's type
  float *dpost, *dpre, *gate_sums;        // [chunks][cols]; gate_sums where a row of the gate has several chunks
  Chunks chunks;
  int64_t rows;
};

// The gradient u = dh w_pre goes on as inv (u - n along - off); see the top.
struct Through {
  float mean, inv, along, off;
  __device__ __forceinline__ float normed(float v) const { return (v - mean) * inv; }
  __device__ __forceinline__ float of(float u, float n) const { return inv * (u - n * along - off); }
};

// A row's units in flight: what one thread has of it.
template <int XT, int BT, bool BLOCK, int T, int NV>
struct RowParts {
  Eight<XT> d[NV], x[NV];
  Eight<BT> h[NV], b[NV], g[NV];
  float4 st;

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      d[i].clear();
      x[i].clear();
      h[i].clear();
      b[i].clear();
      g[i].clear();
    }
    st = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  __device__ __forceinline__ void load(const Desc& q, const Back& a, int64_t row, int col0, bool gate) {
    constexpr int xs = sizeof(typename Elem<XT>::raw), bs = sizeof(typename Elem<BT>::raw);
    st = a.stats[row];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = col0 + (threadIdx.x + i * T) * 8, n = q.cols - col;
      if (n <= 0) continue;
      if (a.dx_out.data) d[i].load(a.dx_out.row(row) + (int64_t)col * xs, n);
      if (q.pre) {
        h[i].load(a.dh.row(row) + (int64_t)col * bs, n);
        x[i].load(a.x_out.row(row) + (int64_t)col * xs, n);
      }
      if constexpr (BLOCK) {
        b[i].load(a.block.row(row) + (int64_t)col * bs, n);
        if (gate) g[i].load(q.gate.row(row / q.shared) + (int64_t)col * bs, n);
      }
    }
  }
};

// One row after another, the next one's loads ahead of this one's sums.  GIVEN: a row's sums are there already, and a workgroup has T * NV * 8 of its columns,
// blockIdx.y says which.  8192^2 bf16: 160 us (805 MB, 5 TB/s); with a row's loads behind the sums of the one before 205.  float32 streams beyond 4096 columns
// spill registers: 4096 x 5120 with a bf16 block 121 us; without the loads ahead 134, by 1024 threads 168, in two passes 143.
template <int XT, int BT, bool BLOCK, int T, int NV, bool GIVEN>
__global__ __launch_bounds__(T) void k_block_norm_back(Desc d, Back a) {
  __shared__ float2 lds[2][2][T / kWave];
  constexpr int xs = sizeof(typename Elem<XT>::raw), bs = sizeof(typename Elem<BT>::raw);
  const int64_t chunk = blockIdx.x, part = chunk % a.chunks.per_gate, base = chunk / a.chunks.per_gate * a.chunks.span;
  const int64_t begin = base + part * a.chunks.rows;
  const int64_t end = min(min(begin + a.chunks.rows, base + a.chunks.span), a.rows);
  const int col0 = GIVEN ? blockIdx.y * (T * NV * 8) : 0;
  const float per = 1.f / (float)d.cols;
  float pre_sum[NV][8], post_sum[NV][8], gate_sum[NV][8], w_pre[NV][8], w_post[NV][8];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int col = col0 + (threadIdx.x + i * T) * 8;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      pre_sum[i][k] = post_sum[i][k] = gate_sum[i][k] = w_pre[i][k] = 0.f;
      w_post[i][k] = 1.f;
    }
    if (d.pre && col < d.cols) load_weights(d.pre, d.weight_dtype, col, d.cols - col, w_pre[i]);
    if (d.post && col < d.cols) load_weights(d.post, d.weight_dtype, col, d.cols - col, w_post[i]);
  }
  RowParts<XT, BT, BLOCK, T, NV> now, next;
  now.clear();
  next.clear();
  if (begin < end) next.load(d, a, begin, col0, d.gate.data != nullptr);
  int which = 0;
  for (int64_t row = begin; row < end; ++row, which ^= 1) {
    now = next;
    const bool gate_ends = row + 1 == end || (row + 1) % d.shared == 0;
    if (row + 1 < end) next.load(d, a, row + 1, col0, d.gate.data && gate_ends);
    float4 given = make_float4(0.f, 0.f, 0.f, 0.f);
    if constexpr (GIVEN) given = a.sums[row];
    Through px = {now.st.z, now.st.w, given.x, given.y}, pb = {now.st.x, now.st.y, given.z, given.w};
    float dx[NV][8];
    if (d.pre) {
      float2 s = make_float2(0.f, 0.f);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        float x[8], u[8];
        now.x[i].get(x);
        now.h[i].get(u);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float n = px.normed(x[k]), g = u[k] * w_pre[i][k];
          s.x += g * n;
          s.y += g;
          pre_sum[i][k] += u[k] * n;
        }
      }
      if constexpr (!GIVEN) {
        s = sums_of_block<T / kWave>(s, lds[which][0]);
        px.along = s.x * per;
        px.off = d.centered ? s.y * per : 0.f;
      }
    }
    float2 s = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = col0 + (threadIdx.x + i * T) * 8;
      float x[8], u[8], b[8], g[8];
      now.d[i].get(dx[i]);
      if (d.pre) {
        now.x[i].get(x);
        now.h[i].get(u);
#pragma unroll
        for (int k = 0; k < 8; ++k) dx[i][k] += px.of(u[k] * w_pre[i][k], px.normed(x[k]));
      }
      if (col < d.cols) {
        Eight<XT> o;
        o.set(dx[i]);
        o.store(a.dx.row(row) + (int64_t)col * xs, d.cols - col);
      }
      if constexpr (BLOCK) {
        now.b[i].get(b);
        now.g[i].get(g);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float q = col + k < d.cols ? d.scale * dx[i][k] : 0.f;
          const float n = d.post ? pb.normed(b[k]) : b[k];
          const float w = d.gate.data ? g[k] : 1.f;
          gate_sum[i][k] += q * n * w_post[i][k];
          post_sum[i][k] += q * w * n;
          const float up = q * w * w_post[i][k];
          s.x += up * n;
          s.y += up;
        }
      }
    }
    if constexpr (BLOCK) {
      if constexpr (!GIVEN) {
        if (d.post) s = sums_of_block<T / kWave>(s, lds[which][1]);
        pb.along = s.x * per;
        pb.off = d.centered ? s.y * per : 0.f;
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int col = col0 + (threadIdx.x + i * T) * 8;
        float b[8], g[8];
        now.b[i].get(b);
        now.g[i].get(g);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float up = d.scale * dx[i][k] * (d.gate.data ? g[k] : 1.f) * w_post[i][k];
          b[k] = d.post ? pb.of(up, pb.normed(b[k])) : up;
        }
        if (col < d.cols) {
          Eight<BT> o;
          o.set(b);
          o.store(a.dblock.row(row) + (int64_t)col * bs, d.cols - col);
        }
      }
      // the last of a gate's rows here: all of them, or this chunk's share
      if (d.gate.data && gate_ends) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int col = col0 + (threadIdx.x + i * T) * 8;
          if (col < d.cols) {
            if (a.chunks.per_gate > 1) {
              Eight<TGRAD_F32> o;
              o.set(gate_sum[i]);
              o.store(reinterpret_cast<char*>(a.gate_sums + chunk * d.cols + col), d.cols - col);
            } else {
              Eight<BT> o;
              o.set(gate_sum[i]);
              o.store(a.dgate + (row / d.shared * d.cols + col) * bs, d.cols - col);
            }
          }
#pragma unroll
          for (int k = 0; k < 8; ++k) gate_sum[i][k] = 0.f;
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int col = col0 + (threadIdx.x + i * T) * 8;
    if (col >= d.cols) continue;
    Eight<TGRAD_F32> o;
    if (a.dpre) {
      o.set(pre_sum[i]);
      o.store(reinterpret_cast<char*>(a.dpre + chunk * d.cols + col), d.cols - col);
    }
    if (a.dpost) {
      o.set(post_sum[i]);
      o.store(reinterpret_cast<char*>(a.dpost + chunk * d.cols + col), d.cols - col);
    }
    if (begin >= end && d.gate.data && a.chunks.per_gate > 1) {     // a chunk without rows
      o.set(gate_sum[i]);
      o.store(reinterpret_cast<char*>(a.gate_sums + chunk * d.cols + col), d.cols - col);
    }
  }
}

// The sums of a row that is longer than kHeldCols, a workgroup a row.  dh and x_out are read twice here and once more by k_block_norm_back, dx_out, block and
// gate once here and once there.  A row has 10 bytes a column, 20 in float32: 32 rows of a die are 2.6 to 21 MB, so that L2 (4 MB a die) holds
// the shortest of them between the readings and the memory-side cache the others.
template <int XT, int BT, bool BLOCK>
__global__ __launch_bounds__(1024) void k_block_norm_sums(Desc d, Back a, int64_t first) {
  constexpr int T = 1024;
  __shared__ float2 lds[2][T / kWave];
  const int64_t row = first + blockIdx.x;
  const float per = 1.f / (float)d.cols;
  const float4 st = a.stats[row];
  Through px = {st.z, st.w, 0.f, 0.f}, pb = {st.x, st.y, 0.f, 0.f};
  RowParts<XT, BT, BLOCK, T, 1> r;
  float2 s = make_float2(0.f, 0.f);
  if (d.pre) {
    for (int col0 = 0; col0 < d.cols; col0 += T * 8) {
      const int col = col0 + threadIdx.x * 8;
      if (col >= d.cols) break;
      float w[8], x[8], u[8];
      r.clear();
      r.load(d, Back{Mat{nullptr, 0}, a.dh, a.x_out, a.block, a.dx, a.dblock, a.stats}, row, col0, false);
      load_weights(d.pre, d.weight_dtype, col, d.cols - col, w);
      r.x[0].get(x);
      r.h[0].get(u);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float g = col + k < d.cols ? u[k] * w[k] : 0.f;
        s.x += g * px.normed(x[k]);
        s.y += g;
      }
    }
    s = sums_of_block<T / kWave>(s, lds[0]);
    px.along = s.x * per;
    px.off = d.centered ? s.y * per : 0.f;
  }
  if constexpr (BLOCK) {
    if (d.post) {
      s = make_float2(0.f, 0.f);
      for (int col0 = 0; col0 < d.cols; col0 += T * 8) {
        const int col = col0 + threadIdx.x * 8;
        if (col >= d.cols) break;
        float w[8], x[8], u[8], dx[8], b[8], g[8];
        r.clear();
        r.load(d, a, row, col0, d.gate.data != nullptr);
        r.d[0].get(dx);
        r.b[0].get(b);
        r.g[0].get(g);
        if (d.pre) {
          load_weights(d.pre, d.weight_dtype, col, d.cols - col, w);
          r.x[0].get(x);
          r.h[0].get(u);
#pragma unroll
          for (int k = 0; k < 8; ++k) dx[k] += px.of(u[k] * w[k], px.normed(x[k]));
        }
        load_weights(d.post, d.weight_dtype, col, d.cols - col, w);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float up = col + k < d.cols ? d.scale * dx[k] * (d.gate.data ? g[k] : 1.f) * w[k] : 0.f;
          s.x += up * pb.normed(b[k]);
          s.y += up;
        }
      }
      s = sums_of_block<T / kWave>(s, lds[1]);
      pb.along = s.x * per;
      pb.off = d.centered ? s.y * per : 0.f;
    }
  }
  if (threadIdx.x == 0) a.sums[row] = make_float4(px.along, px.off, pb.along, pb.off);
}

// out[g][col] = sum over the `per` chunks of g, for up to three results at once.  16 columns and 64 shares of the chunks to a workgroup; shares, then their
// sums in order.
struct SumJob {
  const float* part;
  int64_t per, gates;
  char* out;
  int dt;
};
struct SumJobs {
  SumJob job[3];
};
__global__ __launch_bounds__(1024) void k_chunk_sums(SumJobs jobs, int64_t first, int cols) {
  __shared__ float lds[64][17];
  const int lane = threadIdx.x & 15, share = threadIdx.x >> 4;
  const int col = blockIdx.x * 16 + lane;
  int64_t g = first + blockIdx.y;
  int j = 0;
  while (j < 2 && g >= jobs.job[j].gates) g -= jobs.job[j++].gates;
  const SumJob job = jobs.job[j];
  float s = 0.f;
  if (col < cols) {
    const float* at = job.part + g * job.per * cols + col;
#pragma unroll 8
    for (int64_t c = share; c < job.per; c += 64) s += at[c * cols];
  }
  lds[share][lane] = s;
  __syncthreads();
  if (share == 0 && col < cols) {
    for (int w = 1; w < 64; ++w) s += lds[w][lane];
    const int64_t to = g * cols + col;
    if (job.dt == TGRAD_F32) reinterpret_cast<float*>(job.out)[to] = s;
    else if (job.dt == TGRAD_BF16) reinterpret_cast<uint16_t*>(job.out)[to] = Elem<TGRAD_BF16>::narrow(s);
    else reinterpret_cast<_Float16*>(job.out)[to] = Elem<TGRAD_F16>::narrow(s);
  }
}

void launch_chunk_sums(hipStream_t s, const SumJobs& jobs, int cols) {
  const int64_t all = jobs.job[0].gates + jobs.job[1].gates + jobs.job[2].gates;
  for (int64_t at = 0; at < all; at += 32768)
    k_chunk_sums<<<dim3((cols + 15) / 16, (uint32_t)std::min<int64_t>(all - at, 32768)), dim3(1024), 0, s>>>(jobs, at, cols);
}

// Threads and units of a row, all of them held in registers: 512 threads up to 16384 columns, so that a compute unit has three rows and more in turn (16384 x
// 8192 bf16: 299 us with 1024 threads a row, 229 with 512; 8192 x 16384: 246 and 222); 1024 beyond, whose registers are needed.
template <typename F>
void for_width(int cols, F&& f) {
  const int units = (cols + 7) / 8;
  typedef std::integral_constant<int, 64> t64;
  typedef std::integral_constant<int, 256> t256;
  typedef std::integral_constant<int, 512> t512;
  typedef std::integral_constant<int, 1024> t1024;
  typedef std::integral_constant<int, 1> n1;
  typedef std::integral_constant<int, 2> n2;
  typedef std::integral_constant<int, 4> n4;
  if (units <= 64) f(t64(), n1());
  else if (units <= 256) f(t256(), n1());
  else if (units <= 512) f(t256(), n2());
  else if (units <= 1024) f(t512(), n2());
  else if (units <= 2048) f(t512(), n4());
  else f(t1024(), n4());
}

template <typename F>
void for_width_back(int cols, F&& f) {
  const int units = (cols + 7) / 8;
  typedef std::integral_constant<int, 64> t64;
  typedef std::integral_constant<int, 256> t256;
  typedef std::integral_constant<int, 512> t512;
  typedef std::integral_constant<int, 1> n1;
  typedef std::integral_constant<int, 2> n2;
  if (units <= 64) f(t64(), n1());
  else if (units <= 256) f(t256(), n1());
  else if (units <= 512) f(t512(), n1());
  else f(t512(), n2());
}

// f(type of the stream, type of the block): the same, or a stream in float32.
template <typename F>
void for_types(int xt, int bt, F&& f) {
  typedef std::integral_constant<int, TGRAD_F32> f32;
  for_real(bt, [&](auto b) { xt == TGRAD_F32 ? f(f32(), b) : f(b, b); });
}

bool good(const tgrad_block* d, bool block) {
  if (!d || !is_real(d->weight_dtype) || !std::isfinite(d->scale) || !(d->eps > 0.f) || !std::isfinite(d->eps)) return false;
  if (d->centered != 0 && d->centered != 1) return false;
  if (!block && (d->post_weight || d->gate || !d->pre_weight)) return false;
  const uintptr_t w = (uintptr_t)real_bytes(d->weight_dtype);
  return (uintptr_t)d->post_weight % w == 0 && (uintptr_t)d->pre_weight % w == 0;
}
bool good_gate(const tgrad_block* d, int64_t cols, int bt) {
  if (!d->gate) return true;
  return (uintptr_t)d->gate % (uintptr_t)real_bytes(bt) == 0 && d->rows_per_gate >= 1 && d->gate_stride >= cols && d->gate_stride <= ((int64_t)1 << 28) * 8;
}
Desc describe(const tgrad_block* d, int cols, int bt) {
  const Mat gate{static_cast<char*>(const_cast<void*>(d->gate)), d->gate ? d->gate_stride * real_bytes(bt) : 0};
  return Desc{d->post_weight, d->pre_weight, gate, d->gate ? d->rows_per_gate : 1, d->weight_dtype, cols, d->centered == 1, d->scale, d->eps};
}
bool types_ok(int xt, int bt) { return xt == bt || xt == TGRAD_F32; }

// Scratch of the backward pass.
struct Scratch {
  size_t dpost, dpre, gate, sums, bytes;
};
Scratch scratch_of(const Chunks& c, int64_t rows, int64_t cols) {
  auto aligned = [](size_t n) { return (n + kScratchAlign - 1) / kScratchAlign * kScratchAlign; };
  const size_t each = aligned((size_t)c.count * (size_t)cols * 4);
  Scratch s;
  s.dpost = 0;
  s.dpre = each;
  s.gate = 2 * each;
  s.sums = (c.per_gate > 1 ? 3 : 2) * each;
  s.bytes = s.sums + (cols > kHeldCols ? aligned((size_t)rows * 16) : 0);
  s.bytes = std::max<size_t>(s.bytes, kScratchAlign);
  return s;
}

}  // namespace

extern "C" {

int tgrad_block_norm(const tgrad_block* desc, const tgrad_matrix* x, const tgrad_matrix* block, const tgrad_matrix* x_out,
                     const tgrad_matrix* h, const tgrad_codes* h8, float* stats, void* hip_stream) {
  if (!good(x) || !good(desc, block != nullptr) || (uintptr_t)stats % 16) return TGRAD_ERR_INVALID_ARG;
  const int64_t rows = x->rows, cols = x->cols;
  if (!block != !x_out || (desc->pre_weight ? !h == !h8 : h || h8)) return TGRAD_ERR_INVALID_ARG;
  int bt = x->dtype;
  if (block) {
    if (!good(block) || !good(x_out) || !same_size(block, rows, cols) || !same_size(x_out, rows, cols) || x_out->dtype != x->dtype)
      return TGRAD_ERR_INVALID_ARG;
    bt = block->dtype;
  } else if (h) {
    bt = h->dtype;
  }
  if (h && (!good(h) || !same_size(h, rows, cols) || h->dtype != bt)) return TGRAD_ERR_INVALID_ARG;
  if (h8 && (!good(h8) || !same_size(h8, rows, cols) || h8->group != 0)) return TGRAD_ERR_INVALID_ARG;
  if (!types_ok(x->dtype, bt) || !good_gate(desc, cols, bt)) return TGRAD_ERR_INVALID_ARG;
  if (cols > TGRAD_NORM_MAX_COLS) return TGRAD_ERR_UNSUPPORTED;
  if (pending()) return TGRAD_ERR_HIP;
  if (rows == 0) return TGRAD_OK;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const Desc d = describe(desc, (int)cols, bt);
  const Mat mx = mat(x), mb = mat(block), mo = mat(x_out), mh = mat(h);
  const Codes8 c = codes8(h8);
  float4* st = reinterpret_cast<float4*>(stats);
  for_types(x->dtype, bt, [&](auto xt, auto yt) {
    for_width((int)cols, [&](auto t, auto n) {
      constexpr int XT = decltype(xt)::value, BT = decltype(yt)::value, T = decltype(t)::value, NV = decltype(n)::value;
      rows_in_launches(rows, T, 1, [&](int64_t first, int64_t some) {
        if (block) k_block_norm<XT, BT, true, T, NV><<<dim3((uint32_t)some), dim3(T), 0, s>>>(d, first, mx, mb, mo, mh, c, st);
        else k_block_norm<XT, BT, false, T, NV><<<dim3((uint32_t)some), dim3(T), 0, s>>>(d, first, mx, mb, mo, mh, c, st);
      });
    });
  });
  return launched();
}

int tgrad_block_norm_query_size(int64_t rows, int64_t cols, int64_t rows_per_gate, size_t* workspace_bytes) {
  if (!workspace_bytes || !extents_ok(rows, cols, cols) || rows_per_gate < 1) return TGRAD_ERR_INVALID_ARG;
  if (cols > TGRAD_NORM_MAX_COLS) return TGRAD_ERR_UNSUPPORTED;
  *workspace_bytes = scratch_of(chunks_of(rows, cols, rows_per_gate), rows, cols).bytes;
  return TGRAD_OK;
}

int tgrad_block_norm_backward(const tgrad_block* desc, const tgrad_matrix* dx_out, const tgrad_matrix* dh, const tgrad_matrix* x_out,
                              const tgrad_matrix* block, const float* stats, const tgrad_matrix* dx, const tgrad_matrix* dblock,
                              void* dgate, float* dpost, float* dpre, void* workspace_dev, void* hip_stream) {
  if (!good(x_out) || !good(dx) || !good(desc, block != nullptr)) return TGRAD_ERR_INVALID_ARG;
  const int64_t rows = x_out->rows, cols = x_out->cols;
  const int xt = x_out->dtype, bt = block ? block->dtype : dh ? dh->dtype : xt;
  if (!same_size(dx, rows, cols) || dx->dtype != xt) return TGRAD_ERR_INVALID_ARG;
  if (dx_out && (!good(dx_out) || !same_size(dx_out, rows, cols) || dx_out->dtype != xt || (dx_out->data == dx->data && dx_out->row_stride != dx->row_stride)))
    return TGRAD_ERR_INVALID_ARG;
  if ((dh != nullptr) != (desc->pre_weight != nullptr) || (dh && (!good(dh) || !same_size(dh, rows, cols) || dh->dtype != bt))) return TGRAD_ERR_INVALID_ARG;
  if (!block != !dblock) return TGRAD_ERR_INVALID_ARG;
  if (block && (!good(block) || !good(dblock) || !same_size(block, rows, cols) || !same_size(dblock, rows, cols) || dblock->dtype != bt))
    return TGRAD_ERR_INVALID_ARG;
  if (!types_ok(xt, bt) || !good_gate(desc, cols, bt)) return TGRAD_ERR_INVALID_ARG;
  if ((uintptr_t)stats % 16 || (!stats && rows > 0) || !workspace_dev || (uintptr_t)workspace_dev % kScratchAlign) return TGRAD_ERR_INVALID_ARG;
  if ((dpost != nullptr) != (desc->post_weight != nullptr) || (dpre != nullptr) != (desc->pre_weight != nullptr)) return TGRAD_ERR_INVALID_ARG;
  if ((uintptr_t)dpost % 4 || (uintptr_t)dpre % 4 || (uintptr_t)dgate % (uintptr_t)real_bytes(bt)) return TGRAD_ERR_INVALID_ARG;
  if (rows > 0 && (dgate != nullptr) != (desc->gate != nullptr)) return TGRAD_ERR_INVALID_ARG;
  if (cols > TGRAD_NORM_MAX_COLS) return TGRAD_ERR_UNSUPPORTED;
  if (pending()) return TGRAD_ERR_HIP;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const Desc d = describe(desc, (int)cols, bt);
  const Chunks c = chunks_of(rows, cols, desc->gate ? desc->rows_per_gate : 1);
  const Scratch sc = scratch_of(c, rows, cols);
  char* ws = static_cast<char*>(workspace_dev);
  const bool one = c.count == 1 && rows > 0;            // then the chunk's sums are the results
  Back a;
  a.dx_out = mat(dx_out);
  a.dh = mat(dh);
  a.x_out = mat(x_out);
  a.block = mat(block);
  a.dx = mat(dx);
  a.dblock = mat(dblock);
  a.stats = reinterpret_cast<const float4*>(stats);
  a.sums = reinterpret_cast<float4*>(ws + sc.sums);
  a.dgate = static_cast<char*>(dgate);
  a.dpost = !dpost ? nullptr : one ? dpost : reinterpret_cast<float*>(ws + sc.dpost);
  a.dpre = !dpre ? nullptr : one ? dpre : reinterpret_cast<float*>(ws + sc.dpre);
  a.gate_sums = reinterpret_cast<float*>(ws + sc.gate);
  a.chunks = c;
  a.rows = rows;
  if (rows > 0) {
    for_types(xt, bt, [&](auto x, auto b) {
      constexpr int XT = decltype(x)::value, BT = decltype(b)::value;
      auto run = [&](auto with) {
        constexpr bool BLOCK = decltype(with)::value;
        if (cols > kHeldCols) {
          rows_in_launches(rows, 1024, 1, [&](int64_t first, int64_t some) {
            k_block_norm_sums<XT, BT, BLOCK><<<dim3((uint32_t)some), dim3(1024), 0, s>>>(d, a, first);
          });
          k_block_norm_back<XT, BT, BLOCK, 256, 1, true><<<dim3((uint32_t)c.count, (uint32_t)((cols + 2047) / 2048)), dim3(256), 0, s>>>(d, a);
        } else {
          for_width_back((int)cols, [&](auto t, auto n) {
            constexpr int T = decltype(t)::value, NV = decltype(n)::value;
            k_block_norm_back<XT, BT, BLOCK, T, NV, false><<<dim3((uint32_t)c.count), dim3(T), 0, s>>>(d, a);
          });
        }
      };
      if (block) run(std::true_type());
      else run(std::false_type());
    });
  }
  const int64_t chunks = rows > 0 ? c.count : 0;
  SumJobs jobs = {};
  if (dpost && !one) jobs.job[0] = SumJob{a.dpost, chunks, 1, reinterpret_cast<char*>(dpost), TGRAD_F32};
  if (dpre && !one) jobs.job[1] = SumJob{a.dpre, chunks, 1, reinterpret_cast<char*>(dpre), TGRAD_F32};
  if (rows > 0 && desc->gate && c.per_gate > 1) jobs.job[2] = SumJob{a.gate_sums, c.per_gate, c.count / c.per_gate, a.dgate, bt};
  launch_chunk_sums(s, jobs, (int)cols);
  return launched();
}

}  // extern "C"

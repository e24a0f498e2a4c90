// The kernels of dconv_join and its gradient.  Instantiated per type in
// join_f32.hip, join_f16.hip and join_bf16.hip.
//
// Both are bound by memory (forward 4, backward 6 values moved per element, some
// 20 operations), so a row is read once and stays in registers: TPR threads hold
// EPT elements each, and the row's sums go over the lanes and, past a wave,
// through LDS.  25088 rows of 2048 values in bf16: forward 79 us (5.2 TB/s), backward
// 140 (4.6 TB/s with the runs' sums).  A group of TPR threads walks a run of rows with the vectors (and
// in the backward pass the vectors' sums) in registers and the next row's loads in
// flight.
#pragma once

#include "internal.h"
#include "join.h"
#include "tokens.h"

namespace dconv {

// V elements, 16 bytes of a row; on an element's boundary only (the memory takes
// such accesses as one) where rows are not whole 16-byte pieces.
template <class T, int V, bool WHOLE>
struct alignas(!WHOLE ? sizeof(T) : V * sizeof(T) < 16 ? V * sizeof(T) : 16) Pack {
  T v[V];
};

// How a row lies over TPR threads: thread `me` holds elements
// V (i TPR + me) .. + V - 1 for i < EPT / V.
template <int V_, int TPR_, int EPT_, bool WHOLE_>
struct Row {
  static constexpr int V = V_, TPR = TPR_, EPT = EPT_;
  static constexpr bool WHOLE = WHOLE_;
  static __device__ __forceinline__ int first(int i, int me) { return V * (i * TPR + me); }
};

// A thread's part of a row, as it is in memory.
template <class T, class R>
struct RowPart {
  typedef Pack<T, R::V, R::WHOLE> P;
  P p[R::EPT / R::V];
  __device__ __forceinline__ void load(const T *row, int D, int me) {
#pragma unroll
    for (int i = 0; i < R::EPT / R::V; ++i) {
      const int e = R::first(i, me);
      if (R::WHOLE ? e < D : e + R::V <= D) {
        p[i] = *reinterpret_cast<const P *>(row + e);
      } else if (!R::WHOLE && e < D) {
#pragma unroll
        for (int j = 0; j < R::V; ++j)
          if (e + j < D) p[i].v[j] = row[e + j];
      }
    }
  }
  __device__ __forceinline__ void store(T *row, int D, int me) const {
#pragma unroll
    for (int i = 0; i < R::EPT / R::V; ++i) {
      const int e = R::first(i, me);
      if (R::WHOLE ? e < D : e + R::V <= D) {
        *reinterpret_cast<P *>(row + e) = p[i];
      } else if (!R::WHOLE && e < D) {
#pragma unroll
        for (int j = 0; j < R::V; ++j)
          if (e + j < D) row[e + j] = p[i].v[j];
      }
    }
  }
  __device__ __forceinline__ float get(int k) const { return to_f32(p[k / R::V].v[k % R::V]); }
  __device__ __forceinline__ void set(int k, float x) { p[k / R::V].v[k % R::V] = from_f32<T>(x); }
};

// f(k): for each of the thread's elements that the row has.
template <class R, class F>
__device__ __forceinline__ void each(int D, int me, F f) {
#pragma unroll
  for (int i = 0; i < R::EPT / R::V; ++i)
    if (R::first(i, me) < D) {
#pragma unroll
      for (int j = 0; j < R::V; ++j)
        if (R::WHOLE || R::first(i, me) + j < D) f(i * R::V + j);
    }
}

template <class T, class R>
__device__ __forceinline__ void store_row(T *row, int D, int me, const float (&x)[R::EPT]) {
  RowPart<T, R> p;
#pragma unroll
  for (int k = 0; k < R::EPT; ++k) p.set(k, x[k]);
  p.store(row, D, me);
}

// A vector's part (of type W) in fp32; `absent` where there is none or past the
// row's end.
template <class W, class R>
__device__ __forceinline__ void load_vector(float (&x)[R::EPT], const void *p, int64_t offset, int D, int me,
                                            float absent) {
#pragma unroll
  for (int k = 0; k < R::EPT; ++k) x[k] = absent;
  if (!p) return;
  RowPart<W, R> v;
  v.load((const W *)p + offset, D, me);
  each<R>(D, me, [&](int k) { x[k] = v.get(k); });
}

constexpr int join_block(int TPR) { return TPR > 256 ? TPR : 256; }

// Sums over the TPR threads of a row.  Past a wave: through LDS, in two places
// used in turn, so that one barrier per sum is enough (a wave that writes a place
// again has passed the barrier that every reader of it reached after reading).
template <int TPR>
struct RowSum {
  float *place;
  int turn;
  __device__ __forceinline__ float operator()(float x) {
    if constexpr (TPR <= 64) return lanes_sum<TPR>(x);
    constexpr int kWaves = TPR / 64;
    x = lanes_sum<64>(x);
    float *at = place + (turn ^= kWaves);
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = x;
    wait_lds_barrier();
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) s += at[i];
    return s;
  }
};

// Which rows a group of threads walks: run c of segment s is rows [first, end) of
// the flattened tokens.  All rows of a run share the vectors.
struct JoinRuns {
  int segments, rows;   // rows per segment
  int runs, run_rows;   // runs per segment
};
struct Run {
  int64_t segment, first, end;
};
__device__ __forceinline__ Run run_of(const JoinRuns &r, int64_t id) {
  const int64_t s = id / r.runs, c = id % r.runs;
  Run x;
  x.segment = s;
  x.first = s * r.rows + c * r.run_rows;
  x.end = min(x.first + r.run_rows, (s + 1) * (int64_t)r.rows);
  return x;
}
__device__ __forceinline__ int64_t row_at(const long long *stride, int64_t n, int T) {
  return n / T * stride[0] + n % T * stride[1];
}

template <class T, class W, class R>
__global__ __launch_bounds__(join_block(R::TPR)) void join_forward(const dconv_join_shape sh, const JoinPtrs p,
                                                                const JoinRuns runs) {
  constexpr int TPR = R::TPR, EPT = R::EPT, kPerBlock = join_block(TPR) / TPR;
  __shared__ float place[2 * (TPR / 64 + 1)];
  DCONV_POISON(poison_lds(place, 2 * (TPR / 64 + 1)));
  const int me = threadIdx.x % TPR, D = sh.D;
  const int64_t id = (int64_t)blockIdx.x * kPerBlock + threadIdx.x / TPR;
  if (id >= (int64_t)runs.segments * runs.runs) return;   // whole rows of threads; none past a wave
  const Run run = run_of(runs, id);
  if (run.first >= run.end) return;
  RowSum<TPR> sum = {place, 0};
  const float inv = 1.0f / D;
  const bool layer = sh.norm == DCONV_NORM_LAYER, post = sh.post && p.branch;
  const int64_t b = run.segment;   // the sequence, if a vector is set for each
  float pw[EPT], g[EPT], w[EPT], bias[EPT];
  load_vector<W, R>(pw, post ? p.post_weight : nullptr, sh.per_sample & DCONV_JOIN_POST_WEIGHT ? b * D : 0,
                              D, me, 1.0f);
  load_vector<W, R>(g, p.gate, sh.per_sample & DCONV_JOIN_GATE ? b * D : 0, D, me, 1.0f);
  load_vector<W, R>(w, p.pre_weight, sh.per_sample & DCONV_JOIN_PRE_WEIGHT ? b * D : 0, D, me, 1.0f);
  load_vector<W, R>(bias, p.pre_bias, sh.per_sample & DCONV_JOIN_PRE_BIAS ? b * D : 0, D, me, 0.0f);
#pragma unroll
  for (int k = 0; k < EPT; ++k) g[k] *= sh.branch_scale;

  RowPart<T, R> x, br, x_next, br_next;
  auto load = [&](int64_t n) {
    x_next.load((const T *)p.x + row_at(sh.x_stride, n, sh.T), D, me);
    if (p.branch) br_next.load((const T *)p.branch + row_at(sh.branch_stride, n, sh.T), D, me);
  };
  load(run.first);
  for (int64_t n = run.first; n < run.end; ++n) {
    x = x_next;
    br = br_next;
    if (n + 1 < run.end) load(n + 1);
    float h[EPT] = {}, mb = 0.0f, rb = 1.0f;
    auto all = [&](auto f) { each<R>(D, me, f); };
    // N(z) of the row in z: the mean first, then the squares about it
    auto norm = [&](float (&z)[EPT], float &m, float &r) {
      m = 0.0f;
      float s = 0.0f;
      if (layer) {
        all([&](int k) { s += z[k]; });
        m = sum(s) * inv;
        s = 0.0f;
      }
      all([&](int k) {
        z[k] -= m;
        s = fmaf(z[k], z[k], s);
      });
      r = 1.0f / sqrtf(fmaf(sum(s), inv, sh.eps));
      all([&](int k) { z[k] *= r; });
    };
    if (p.branch) {
      all([&](int k) { h[k] = br.get(k); });
      if (post) norm(h, mb, rb);
      all([&](int k) { h[k] = fmaf(sh.residual_scale, x.get(k), g[k] * (h[k] * pw[k])); });
    } else {
      all([&](int k) { h[k] = sh.residual_scale * x.get(k); });
    }
    if (p.h) store_row<T, R>((T *)p.h + n * D, D, me, h);
    if (!p.y && !p.stats) continue;
    float mh, rh;
    norm(h, mh, rh);
    if (p.y) {
      all([&](int k) { h[k] = fmaf(h[k], w[k], bias[k]); });
      store_row<T, R>((T *)p.y + n * D, D, me, h);
    }
    if (p.stats && me == 0) *reinterpret_cast<float4 *>(p.stats + 4 * n) = make_float4(mb, rb, mh, rh);
  }
}

// dx, dbranch, and each run's sums for the vectors: into the vectors' gradients
// themselves where there is one run to a segment and a segment to a vector, else
// into the workspace, [vector][run][D].
template <class T, class W, class R>
__global__ __launch_bounds__(join_block(R::TPR), R::TPR <= 256 ? (R::EPT == 8 ? 3 : 2) : 1) void join_backward(const dconv_join_shape sh, const JoinPtrs p,
                                                                 const JoinRuns runs, float *partial) {
  constexpr int TPR = R::TPR, EPT = R::EPT, kPerBlock = join_block(TPR) / TPR;
  __shared__ float place[2 * (TPR / 64 + 1)];
  DCONV_POISON(poison_lds(place, 2 * (TPR / 64 + 1)));
  const int me = threadIdx.x % TPR, D = sh.D;
  const int64_t id = (int64_t)blockIdx.x * kPerBlock + threadIdx.x / TPR;
  const int64_t all_runs = (int64_t)runs.segments * runs.runs;
  if (id >= all_runs) return;
  const Run run = run_of(runs, id);
  RowSum<TPR> sum = {place, 0};
  const float inv = 1.0f / D;
  const bool layer = sh.norm == DCONV_NORM_LAYER, post = sh.post && p.branch;
  const int64_t b = run.segment;   // the sequence, if a vector is set for each
  float pw[EPT], g[EPT], w[EPT];
  load_vector<W, R>(pw, post ? p.post_weight : nullptr, sh.per_sample & DCONV_JOIN_POST_WEIGHT ? b * D : 0,
                              D, me, 1.0f);
  load_vector<W, R>(g, p.gate, sh.per_sample & DCONV_JOIN_GATE ? b * D : 0, D, me, 1.0f);
  load_vector<W, R>(w, p.pre_weight, sh.per_sample & DCONV_JOIN_PRE_WEIGHT ? b * D : 0, D, me, 1.0f);
#pragma unroll
  for (int k = 0; k < EPT; ++k) g[k] *= sh.branch_scale;
  float s_pw[EPT] = {}, s_g[EPT] = {}, s_w[EPT] = {}, s_bias[EPT] = {};

  RowPart<T, R> x, br, dh, dy, x_next, br_next, dh_next, dy_next;
  float4 st, st_next;
  auto load = [&](int64_t n) {
    x_next.load((const T *)p.x + row_at(sh.x_stride, n, sh.T), D, me);
    if (p.branch) br_next.load((const T *)p.branch + row_at(sh.branch_stride, n, sh.T), D, me);
    if (p.dh) dh_next.load((const T *)p.dh + row_at(sh.dh_stride, n, sh.T), D, me);
    if (p.dy) dy_next.load((const T *)p.dy + row_at(sh.dy_stride, n, sh.T), D, me);
    st_next = *reinterpret_cast<const float4 *>(p.stats + 4 * n);
  };
  if (run.first < run.end) load(run.first);
  for (int64_t n = run.first; n < run.end; ++n) {
    x = x_next, br = br_next, dh = dh_next, dy = dy_next, st = st_next;
    if (n + 1 < run.end) load(n + 1);
    const float mb = st.x, rb = st.y, mh = st.z, rh = st.w;
    auto all = [&](auto f) { each<R>(D, me, f); };
    float nb[EPT] = {}, gh[EPT] = {};
    if (p.branch) all([&](int k) { nb[k] = post ? (br.get(k) - mb) * rb : br.get(k); });
    if (p.dy) {
      // t = N(h); dH = dh + r_h (dt - mean(dt) - t mean(dt t))
      float t[EPT] = {}, s1 = 0.0f, s2 = 0.0f;
      all([&](int k) {
        const float h = fmaf(sh.residual_scale, x.get(k), p.branch ? g[k] * (nb[k] * pw[k]) : 0.0f);
        const float d = dy.get(k);
        t[k] = (h - mh) * rh;
        s_bias[k] += d;
        s_w[k] = fmaf(d, t[k], s_w[k]);
        gh[k] = d * w[k];
        s1 += gh[k];
        s2 = fmaf(gh[k], t[k], s2);
      });
      s1 = layer ? sum(s1) * inv : 0.0f;
      s2 = sum(s2) * inv;
      all([&](int k) { gh[k] = rh * (gh[k] - s1 - t[k] * s2); });
    }
    if (p.dh) all([&](int k) { gh[k] += dh.get(k); });
    float o[EPT] = {};
    all([&](int k) { o[k] = sh.residual_scale * gh[k]; });
    store_row<T, R>((T *)p.dx + n * D, D, me, o);
    if (!p.branch) continue;
    float q1 = 0.0f, q2 = 0.0f;
    all([&](int k) {
      const float u = gh[k] * nb[k];
      s_pw[k] = fmaf(u, g[k], s_pw[k]);
      s_g[k] = fmaf(u, pw[k], s_g[k]);
      o[k] = gh[k] * g[k] * pw[k];
      q1 += o[k];
      q2 = fmaf(o[k], nb[k], q2);
    });
    if (post) {
      q1 = layer ? sum(q1) * inv : 0.0f;
      q2 = sum(q2) * inv;
      all([&](int k) { o[k] = rb * (o[k] - q1 - nb[k] * q2); });
    }
    store_row<T, R>((T *)p.dbranch + n * D, D, me, o);
  }
#pragma unroll
  for (int k = 0; k < EPT; ++k) s_g[k] *= sh.branch_scale;
  float *out = partial + id * D;
  auto leave = [&](void *to, int bit, const float (&s)[EPT]) {
    if (!to) return;
    if (runs.runs == 1 && (runs.segments == 1 || (sh.per_sample & bit))) {
      store_row<W, R>((W *)to + id * D, D, me, s);
    } else {
      store_row<float, R>(out, D, me, s);
      out += all_runs * D;
    }
  };
  leave(p.dpost_weight, DCONV_JOIN_POST_WEIGHT, s_pw);
  leave(p.dgate, DCONV_JOIN_GATE, s_g);
  leave(p.dpre_weight, DCONV_JOIN_PRE_WEIGHT, s_w);
  leave(p.dpre_bias, DCONV_JOIN_PRE_BIAS, s_bias);
}

// Adds the runs' sums of each vector (blockIdx.z): 64 columns per workgroup, its 16
// waves each every 16th run, then the waves in order.
struct JoinSums {
  const float *partial[4];
  void *out[4];
  int runs[4], segments[4];
};
template <class W>
__global__ __launch_bounds__(1024) void join_runs(const JoinSums sums, int D) {
  __shared__ float part[16][64];
  DCONV_POISON(poison_lds(&part[0][0], 1024));
  const int z = blockIdx.z, runs = sums.runs[z];
  if ((int)blockIdx.y >= sums.segments[z]) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, d = blockIdx.x * 64 + lane;
  const float *from = sums.partial[z] + (int64_t)blockIdx.y * runs * D;
  float s[4] = {};
  if (d < D) {
    int r = wave;
    for (; r + 48 < runs; r += 64)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] += from[(int64_t)(r + 16 * i) * D + d];
    for (; r < runs; r += 16) s[0] += from[(int64_t)r * D + d];
  }
  part[wave][lane] = (s[0] + s[1]) + (s[2] + s[3]);
  __syncthreads();
  if (wave == 0 && d < D) {
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) t += part[i][lane];
    ((W *)sums.out[z])[(int64_t)blockIdx.y * D + d] = from_f32<W>(t);
  }
}

// ---------------------------------------------------------------------------
// Launch
// ---------------------------------------------------------------------------
// f(a Row as a value).
template <class T, class F>
void by_row(const JoinPlan &plan, F f) {
  constexpr int V = 16 / sizeof(T);
  auto at = [&](auto tpr) {
    constexpr int TPR = decltype(tpr)::value;
    if (plan.ept == 8)
      plan.whole ? f(Row<V, TPR, 8, true>()) : f(Row<V, TPR, 8, false>());
    else
      plan.whole ? f(Row<V, TPR, 16, true>()) : f(Row<V, TPR, 16, false>());
  };
  if (plan.tpr == 16) at(std::integral_constant<int, 16>());
  if (plan.tpr == 64) at(std::integral_constant<int, 64>());
  if (plan.tpr == 256) at(std::integral_constant<int, 256>());
  if (plan.tpr == 1024) at(std::integral_constant<int, 1024>());
}

template <class T, class W>
void launch_join(const dconv_join_shape &sh, const JoinPtrs &p, const JoinPlan &plan, float *workspace, bool backward,
                 hipStream_t s) {
  const JoinRuns runs = {plan.segments, plan.rows, plan.runs, plan.run_rows};
  const int64_t all_runs = (int64_t)plan.segments * plan.runs;
  by_row<T>(plan, [&](auto row) {
    typedef decltype(row) R;
    const int per_block = join_block(R::TPR) / R::TPR;
    const dim3 grid((unsigned)((all_runs + per_block - 1) / per_block)), block(join_block(R::TPR));
    if (all_runs == 0) return;
    if (!backward)
      hipLaunchKernelGGL((join_forward<T, W, R>), grid, block, 0, s, sh, p, runs);
    else
      hipLaunchKernelGGL((join_backward<T, W, R>), grid, block, 0, s, sh, p, runs, workspace);
  });
  if (!backward) return;
  const struct { void *out; int bit; } vectors[] = {{p.dpost_weight, DCONV_JOIN_POST_WEIGHT},
                                                    {p.dgate, DCONV_JOIN_GATE},
                                                    {p.dpre_weight, DCONV_JOIN_PRE_WEIGHT},
                                                    {p.dpre_bias, DCONV_JOIN_PRE_BIAS}};
  JoinSums sums = {};
  int n = 0, most = 0;
  for (const auto &g : vectors) {
    const bool per = sh.per_sample & g.bit;
    if (!g.out || (plan.runs == 1 && (plan.segments == 1 || per)) || (per && plan.segments == 0)) continue;
    sums.partial[n] = workspace;
    sums.out[n] = g.out;
    sums.runs[n] = per ? plan.runs : (int)all_runs;
    sums.segments[n] = per ? plan.segments : 1;
    most = sums.segments[n] > most ? sums.segments[n] : most;
    ++n;
    workspace += all_runs * sh.D;
  }
  if (n > 0)
    hipLaunchKernelGGL((join_runs<W>), dim3((sh.D + 63) / 64, most, n), dim3(1024), 0, s, sums, sh.D);
}

}  // namespace dconv

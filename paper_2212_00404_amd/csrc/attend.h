// What the kernels of windowed attention share: which keys a query sees, and
// the plain form of one row, by which the matrix-core kernels are backed.
#pragma once

#include "internal.h"
#include "tokens.h"

namespace dconv {

struct AttendPtrs {
  const void *q, *k, *v, *out, *dout;
  const float *lse;
  const int *lengths, *starts;
  void *o, *dq, *dk, *dv;
  float *lse_out;
};

// Sequence b: its number of keys and the position of its first query.
struct Seq {
  int len;
  int64_t start;
};
__device__ __forceinline__ Seq seq_of(const dconv_attend_shape &sh, const AttendPtrs &p, int b) {
  Seq s;
  s.len = sh.Tk;
  if (p.lengths) s.len = min(max(p.lengths[b], 0), sh.Tk);
  s.start = p.starts ? (int64_t)p.starts[b] : (int64_t)s.len - sh.Tq;
  return s;
}

// Keys [0, first) and [lo, hi) are what a query at position i sees.
struct Span {
  int first, lo, hi;
};
__device__ __forceinline__ Span span_of(const dconv_attend_shape &sh, const Seq &s, int64_t i) {
  Span r = {0, 0, 0};
  if (i < 0) return r;
  r.hi = sh.right < 0 ? s.len : (int)min((int64_t)s.len, i + sh.right + 1);
  r.lo = sh.left < 0 ? 0 : (int)min((int64_t)r.hi, max((int64_t)0, i - sh.left));
  r.first = min(sh.sinks, r.lo);
  return r;
}

// Queries [lo, hi) are those that see key j < length.
struct QuerySpan {
  int lo, hi;
};
__device__ __forceinline__ QuerySpan queries_of(const dconv_attend_shape &sh, const Seq &s, int j) {
  const int64_t from = max((int64_t)0, sh.right < 0 ? (int64_t)0 : (int64_t)j - sh.right) - s.start;
  const int64_t to =
      sh.left < 0 || j < sh.sinks ? (int64_t)sh.Tq : (int64_t)j + sh.left + 1 - s.start;
  QuerySpan r;
  r.lo = (int)min(max(from, (int64_t)0), (int64_t)sh.Tq);
  r.hi = (int)min(max(to, (int64_t)r.lo), (int64_t)sh.Tq);
  return r;
}

constexpr int kAttendMaxD = 256;
constexpr int kRowParts = kAttendMaxD / 64;   // elements of a head per lane

template <class T>
__device__ __forceinline__ const T *row_of(const void *p, const long long *stride, int64_t b, int64_t t,
                                           int64_t h) {
  return (const T *)p + b * stride[0] + t * stride[1] + h * stride[2];
}

template <class T>
__device__ __forceinline__ float row_dot(const T *a, const T *b, int D) {
  float s = 0.0f;
  for (int d = 0; d < D; ++d) s = fmaf(to_f32(a[d]), to_f32(b[d]), s);
  return s;
}

// acc += w * row, each lane its elements lane, lane + 64, ...
template <class A, class T>
__device__ __forceinline__ void row_add(A *acc, float w, const T *row, int D, int lane) {
#pragma unroll
  for (int i = 0; i < kRowParts; ++i)
    if (lane + 64 * i < D) acc[i] = fma((A)w, (A)to_f32(row[lane + 64 * i]), acc[i]);
}

// One query of one head by one wave: 64 keys at a time, a key per lane for the
// products and a part of the head per lane for the sum.  Only visible keys and
// values are read.  The sums are in 64 bits: rows come here whose sum of values,
// before it is divided by that of the weights, is past fp32's largest, and their
// mean is not.
template <class T>
__device__ void attend_row(const dconv_attend_shape &sh, const AttendPtrs &p, int b, int h, int t) {
  const int lane = threadIdx.x & 63, D = sh.D, hk = h / (sh.Hq / sh.Hkv);
  const Seq s = seq_of(sh, p, b);
  const Span see = span_of(sh, s, s.start + t);
  const T *q = row_of<T>(p.q, sh.q_stride, b, t, h);
  float m = -INFINITY;
  double l = 0.0, acc[kRowParts] = {};
  for (int part = 0; part < 2; ++part) {
    const int end = part ? see.hi : see.first;
    for (int j0 = part ? see.lo : 0; j0 < end; j0 += 64) {
      const int j = j0 + lane;
      float x = -INFINITY;
      if (j < end) x = sh.scale * row_dot(q, row_of<T>(p.k, sh.k_stride, b, j, hk), D);
      const float top = fmaxf(m, lanes_max<64>(x));
      // (every score -infinity: exp(x - top) would be NaN)
      const float base = top == -INFINITY ? 0.0f : top;
      const float w = j < end ? expf(x - base) : 0.0f;
      const float keep = expf(m - base);
      m = top;
      l = l * keep + lanes_sum<64>(w);
#pragma unroll
      for (int i = 0; i < kRowParts; ++i) acc[i] *= keep;
      for (int k = 0; k < 64 && j0 + k < end; ++k)
        row_add(acc, __shfl(w, k), row_of<T>(p.v, sh.v_stride, b, j0 + k, hk), D, lane);
    }
  }
  const bool none = see.hi - see.lo + see.first == 0;
  T *o = (T *)p.o + b * sh.out_stride[0] + t * sh.out_stride[1] + h * sh.out_stride[2];
#pragma unroll
  for (int i = 0; i < kRowParts; ++i)
    if (lane + 64 * i < D) o[lane + 64 * i] = from_f32<T>(none ? 0.0f : (float)(acc[i] / l));
  if (p.lse_out && lane == 0)
    p.lse_out[((int64_t)b * sh.Hq + h) * sh.Tq + t] = none ? -INFINITY : m + logf((float)l);
}

// dq of one query of one head by one wave.
template <class T>
__device__ void attend_row_dq(const dconv_attend_shape &sh, const AttendPtrs &p, int b, int h, int t) {
  const int lane = threadIdx.x & 63, D = sh.D, hk = h / (sh.Hq / sh.Hkv);
  const Seq s = seq_of(sh, p, b);
  const Span see = span_of(sh, s, s.start + t);
  const T *q = row_of<T>(p.q, sh.q_stride, b, t, h);
  const T *g = row_of<T>(p.dout, sh.dout_stride, b, t, h);
  const float lse = p.lse[((int64_t)b * sh.Hq + h) * sh.Tq + t];
  const float delta = row_dot(g, row_of<T>(p.out, sh.out_stride, b, t, h), D);
  float acc[kRowParts] = {};
  for (int part = 0; part < 2; ++part) {
    const int end = part ? see.hi : see.first;
    for (int j0 = part ? see.lo : 0; j0 < end; j0 += 64) {
      const int j = j0 + lane;
      float ds = 0.0f;
      if (j < end) {
        const float w = expf(sh.scale * row_dot(q, row_of<T>(p.k, sh.k_stride, b, j, hk), D) - lse);
        ds = sh.scale * w * (row_dot(g, row_of<T>(p.v, sh.v_stride, b, j, hk), D) - delta);
      }
      for (int k = 0; k < 64 && j0 + k < end; ++k)
        row_add(acc, __shfl(ds, k), row_of<T>(p.k, sh.k_stride, b, j0 + k, hk), D, lane);
    }
  }
  T *o = (T *)p.dq + (((int64_t)b * sh.Tq + t) * sh.Hq + h) * D;
#pragma unroll
  for (int i = 0; i < kRowParts; ++i)
    if (lane + 64 * i < D) o[lane + 64 * i] = from_f32<T>(acc[i]);
}

// dk and dv of one key by one wave: 64 queries at a time, for each head of the
// group.
template <class T>
__device__ void attend_row_dkv(const dconv_attend_shape &sh, const AttendPtrs &p, int b, int hk, int j) {
  const int lane = threadIdx.x & 63, D = sh.D, G = sh.Hq / sh.Hkv;
  const Seq s = seq_of(sh, p, b);
  QuerySpan by = {0, 0};
  if (j < s.len) by = queries_of(sh, s, j);
  const T *k = row_of<T>(p.k, sh.k_stride, b, j, hk), *v = row_of<T>(p.v, sh.v_stride, b, j, hk);
  float dk[kRowParts] = {}, dv[kRowParts] = {};
  for (int h = hk * G; h < hk * G + G; ++h)
    for (int t0 = by.lo; t0 < by.hi; t0 += 64) {
      const int t = t0 + lane;
      float w = 0.0f, ds = 0.0f;
      if (t < by.hi) {
        const T *g = row_of<T>(p.dout, sh.dout_stride, b, t, h);
        w = expf(sh.scale * row_dot(row_of<T>(p.q, sh.q_stride, b, t, h), k, D) -
                 p.lse[((int64_t)b * sh.Hq + h) * sh.Tq + t]);
        ds = sh.scale * w *
             (row_dot(g, v, D) - row_dot(g, row_of<T>(p.out, sh.out_stride, b, t, h), D));
      }
      for (int i = 0; i < 64 && t0 + i < by.hi; ++i) {
        row_add(dv, __shfl(w, i), row_of<T>(p.dout, sh.dout_stride, b, t0 + i, h), D, lane);
        row_add(dk, __shfl(ds, i), row_of<T>(p.q, sh.q_stride, b, t0 + i, h), D, lane);
      }
    }
  const int64_t o = (((int64_t)b * sh.Tk + j) * sh.Hkv + hk) * D;
#pragma unroll
  for (int i = 0; i < kRowParts; ++i)
    if (lane + 64 * i < D) {
      ((T *)p.dk)[o + lane + 64 * i] = from_f32<T>(dk[i]);
      ((T *)p.dv)[o + lane + 64 * i] = from_f32<T>(dv[i]);
    }
}

// How a forward call runs: `few` rows with the keys divided over waves and
// `splits` workgroups (attend_split), else 128 rows per workgroup
// (attend_tiles).
struct ForwardPlan {
  bool few, direct, near;
  int dp;              // head size the kernels are built for
  int tiles, splits;   // tiles of rows per key head, parts of the keys
  int64_t workspace;   // bytes
};
constexpr int attend_part_floats(int dp) { return 32 * (2 + dp); }

// Instantiated in attend_f32.hip, attend_f16.hip and attend_bf16.hip.
template <class T>
void launch_attend(const dconv_attend_shape &sh, const AttendPtrs &p, const ForwardPlan &plan, float *workspace,
                   hipStream_t s);

// How a backward call runs (head sizes up to 128): dq by tiles of 128 rows; dk
// and dv of the keys [0, first) by tiles of 32 with the rows divided
// (attend_dkv_split), of the others by tiles of key_groups * 32 (attend_dkv).
constexpr int kGradMaxD = 128;
struct BackwardPlan {
  bool direct, near;
  int dp;
  int row_tiles, key_tiles, key_groups;
  int first, first_tiles, parts;
  int64_t stats_bytes, workspace;
};
// Instantiated in attend_grad_f32.hip, attend_grad_f16.hip and attend_grad_bf16.hip.
template <class T>
void launch_attend_grad(const dconv_attend_shape &sh, const AttendPtrs &p, const BackwardPlan &plan, void *workspace,
                        hipStream_t s);

}  // namespace dconv

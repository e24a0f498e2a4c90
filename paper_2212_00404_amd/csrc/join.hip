// From a block's output to the next block's input (dconv_join): the norm after
// the block, its gate and scales, the residual sum and the norm before the
// next block, and the gradients.
#include <climits>

#include "internal.h"
#include "tokens.h"

#define DCONV_EXPORT extern "C" __attribute__((visibility("default")))

namespace dconv {
namespace {

constexpr int kMaxD = 16384;

struct JoinPtrs {
  const void *branch, *x, *post_weight, *gate, *pre_weight, *pre_bias;
  const void *dh, *dy;
  void *h, *y;
  float *stats;
  void *dbranch, *dx, *dpost_weight, *dgate, *dpre_weight, *dpre_bias;
};

template <class W>
__device__ __forceinline__ float vec(const void *p, const dconv_join_shape &sh, int bit, int b, int d,
                                     float absent) {
  if (!p) return absent;
  return to_f32(((const W *)p)[(sh.per_sample & bit ? (int64_t)b * sh.D : 0) + d]);
}

// Sum over the 256 threads of a workgroup, the same value in every thread.
__device__ __forceinline__ float block_sum(float v, float *red) {
  v = lanes_sum<64>(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

// One workgroup per token, the row of h kept in LDS.
template <class T, class W>
__global__ __launch_bounds__(256) void join_row(const dconv_join_shape sh, const JoinPtrs p) {
  extern __shared__ float row[];
  float *red = row + sh.D;
  const int64_t n = blockIdx.x;
  const int b = (int)(n / sh.T), t = (int)(n % sh.T), D = sh.D;
  const T *x = (const T *)p.x + b * sh.x_stride[0] + t * sh.x_stride[1];
  const T *br = p.branch ? (const T *)p.branch + b * sh.branch_stride[0] + t * sh.branch_stride[1] : nullptr;
  const bool layer = sh.norm == DCONV_NORM_LAYER, post = sh.post && br;
  float mb = 0.0f, rb = 1.0f;
  if (post) {
    float s = 0.0f;
    if (layer) {
      for (int d = threadIdx.x; d < D; d += 256) s += to_f32(br[d]);
      mb = block_sum(s, red) / D;
    }
    s = 0.0f;
    for (int d = threadIdx.x; d < D; d += 256) {
      const float z = to_f32(br[d]) - mb;
      s += z * z;
    }
    rb = 1.0f / sqrtf(block_sum(s, red) / D + sh.eps);
  }
  float s = 0.0f;
  for (int d = threadIdx.x; d < D; d += 256) {
    float h = sh.residual_scale * to_f32(x[d]);
    if (br) {
      float q = to_f32(br[d]);
      if (post) q = (q - mb) * rb * vec<W>(p.post_weight, sh, DCONV_JOIN_POST_WEIGHT, b, d, 1.0f);
      h += sh.branch_scale * vec<W>(p.gate, sh, DCONV_JOIN_GATE, b, d, 1.0f) * q;
    }
    if (p.h) ((T *)p.h)[n * D + d] = from_f32<T>(h);
    row[d] = h;
    s += h;
  }
  if (!p.y && !p.stats) return;
  const float mh = layer ? block_sum(s, red) / D : 0.0f;
  s = 0.0f;
  for (int d = threadIdx.x; d < D; d += 256) s += (row[d] - mh) * (row[d] - mh);
  const float rh = 1.0f / sqrtf(block_sum(s, red) / D + sh.eps);
  if (p.y)
    for (int d = threadIdx.x; d < D; d += 256)
      ((T *)p.y)[n * D + d] =
          from_f32<T>((row[d] - mh) * rh * vec<W>(p.pre_weight, sh, DCONV_JOIN_PRE_WEIGHT, b, d, 1.0f) +
                      vec<W>(p.pre_bias, sh, DCONV_JOIN_PRE_BIAS, b, d, 0.0f));
  if (p.stats && threadIdx.x == 0) {
    p.stats[4 * n] = mb;
    p.stats[4 * n + 1] = rb;
    p.stats[4 * n + 2] = mh;
    p.stats[4 * n + 3] = rh;
  }
}

// h of the forward call, before its rounding, and p = N(branch) * post_weight.
template <class T, class W>
struct JoinRow {
  const dconv_join_shape &sh;
  const JoinPtrs &p;
  int64_t n;
  int b;
  const T *x, *br, *dh, *dy;
  float mb, rb, mh, rh;
  bool post;
  __device__ JoinRow(const dconv_join_shape &sh_, const JoinPtrs &p_, int64_t n_)
      : sh(sh_), p(p_), n(n_), b((int)(n_ / sh_.T)) {
    const int t = (int)(n % sh.T);
    x = (const T *)p.x + b * sh.x_stride[0] + t * sh.x_stride[1];
    br = p.branch ? (const T *)p.branch + b * sh.branch_stride[0] + t * sh.branch_stride[1] : nullptr;
    dh = p.dh ? (const T *)p.dh + b * sh.dh_stride[0] + t * sh.dh_stride[1] : nullptr;
    dy = p.dy ? (const T *)p.dy + b * sh.dy_stride[0] + t * sh.dy_stride[1] : nullptr;
    post = sh.post && br;
    mb = p.stats[4 * n];
    rb = p.stats[4 * n + 1];
    mh = p.stats[4 * n + 2];
    rh = p.stats[4 * n + 3];
  }
  __device__ float normed_branch(int d) const { return post ? (to_f32(br[d]) - mb) * rb : to_f32(br[d]); }
  __device__ float post_weight(int d) const {
    return post ? vec<W>(p.post_weight, sh, DCONV_JOIN_POST_WEIGHT, b, d, 1.0f) : 1.0f;
  }
  __device__ float gate(int d) const { return sh.branch_scale * vec<W>(p.gate, sh, DCONV_JOIN_GATE, b, d, 1.0f); }
  __device__ float normed_h(int d) const {
    float h = sh.residual_scale * to_f32(x[d]);
    if (br) h += gate(d) * (normed_branch(d) * post_weight(d));
    return (h - mh) * rh;
  }
  __device__ float grad_y(int d) const { return dy ? to_f32(dy[d]) : 0.0f; }
  __device__ float grad_t(int d) const {
    return grad_y(d) * vec<W>(p.pre_weight, sh, DCONV_JOIN_PRE_WEIGHT, b, d, 1.0f);
  }
};

// dx and dbranch: one workgroup per token, the row of dH kept in LDS (and in
// the workspace for the sums over tokens).
template <class T, class W>
__global__ __launch_bounds__(256) void join_backward_row(const dconv_join_shape sh, const JoinPtrs p,
                                                         float *grad_h) {
  extern __shared__ float row[];
  float *red = row + sh.D;
  const JoinRow<T, W> r(sh, p, blockIdx.x);
  const int D = sh.D;
  const bool layer = sh.norm == DCONV_NORM_LAYER;
  float s1 = 0.0f, s2 = 0.0f;
  for (int d = threadIdx.x; d < D; d += 256) {
    s1 += r.grad_t(d);
    s2 += r.grad_t(d) * r.normed_h(d);
  }
  s1 = layer ? block_sum(s1, red) / D : 0.0f;
  s2 = block_sum(s2, red) / D;
  float q1 = 0.0f, q2 = 0.0f;
  for (int d = threadIdx.x; d < D; d += 256) {
    float g = r.rh * (r.grad_t(d) - s1 - r.normed_h(d) * s2);
    if (r.dh) g += to_f32(r.dh[d]);
    row[d] = g;
    grad_h[r.n * D + d] = g;
    ((T *)p.dx)[r.n * D + d] = from_f32<T>(sh.residual_scale * g);
    if (r.br) {
      const float dn = g * r.gate(d) * r.post_weight(d);
      q1 += dn;
      q2 += dn * r.normed_branch(d);
    }
  }
  if (!r.br) return;
  q1 = layer ? block_sum(q1, red) / D : 0.0f;
  q2 = block_sum(q2, red) / D;
  for (int d = threadIdx.x; d < D; d += 256) {
    float dn = row[d] * r.gate(d) * r.post_weight(d);
    if (r.post) dn = r.rb * (dn - q1 - r.normed_branch(d) * q2);
    ((T *)p.dbranch)[r.n * D + d] = from_f32<T>(dn);
  }
}

// The gradient of one vector: a thread per element, over its tokens.
template <class T, class W>
__global__ __launch_bounds__(256) void join_backward_vector(const dconv_join_shape sh, const JoinPtrs p,
                                                            const float *grad_h, void *out, int bit) {
  const int d = blockIdx.x * 256 + threadIdx.x;
  if (d >= sh.D) return;
  const bool per = sh.per_sample & bit;
  const int64_t rows = per ? sh.T : (int64_t)sh.B * sh.T;
  const int64_t n0 = blockIdx.y * rows;
  float s = 0.0f;
  for (int64_t n = n0; n < n0 + rows; ++n) {
    const JoinRow<T, W> r(sh, p, n);
    if (bit == DCONV_JOIN_POST_WEIGHT) s += grad_h[n * sh.D + d] * r.gate(d) * r.normed_branch(d);
    if (bit == DCONV_JOIN_GATE)
      s += grad_h[n * sh.D + d] * sh.branch_scale * r.normed_branch(d) * r.post_weight(d);
    if (bit == DCONV_JOIN_PRE_WEIGHT) s += r.grad_y(d) * r.normed_h(d);
    if (bit == DCONV_JOIN_PRE_BIAS) s += r.grad_y(d);
  }
  ((W *)out)[(int64_t)blockIdx.y * sh.D + d] = from_f32<W>(s);
}

template <class T, class W>
hipError_t launch_join(const dconv_join_shape &sh, const JoinPtrs &p, hipStream_t s) {
  hipLaunchKernelGGL((join_row<T, W>), dim3((unsigned)(sh.B * sh.T)), dim3(256),
                     (sh.D + 4) * sizeof(float), s, sh, p);
  return hipGetLastError();
}

template <class T, class W>
hipError_t launch_join_backward(const dconv_join_shape &sh, const JoinPtrs &p, float *ws, hipStream_t s) {
  if (sh.B > 0 && sh.T > 0)
    hipLaunchKernelGGL((join_backward_row<T, W>), dim3((unsigned)(sh.B * sh.T)), dim3(256),
                       (sh.D + 4) * sizeof(float), s, sh, p, ws);
  const struct { void *out; int bit; } v[] = {{p.dpost_weight, DCONV_JOIN_POST_WEIGHT},
                                              {p.dgate, DCONV_JOIN_GATE},
                                              {p.dpre_weight, DCONV_JOIN_PRE_WEIGHT},
                                              {p.dpre_bias, DCONV_JOIN_PRE_BIAS}};
  for (const auto &g : v)
    if (g.out && (sh.B > 0 || !(sh.per_sample & g.bit)))
      hipLaunchKernelGGL((join_backward_vector<T, W>),
                         dim3((sh.D + 255) / 256, sh.per_sample & g.bit ? sh.B : 1), dim3(256), 0, s,
                         sh, p, ws, g.out, g.bit);
  return hipGetLastError();
}

template <class F>
hipError_t by_types(const dconv_join_shape &sh, F f) {
  if (sh.dtype == DCONV_F32) return f((float *)nullptr, (float *)nullptr);
  if (sh.dtype == DCONV_F16)
    return sh.vector_dtype == DCONV_F32 ? f((f16_t *)nullptr, (float *)nullptr)
                                        : f((f16_t *)nullptr, (f16_t *)nullptr);
  return sh.vector_dtype == DCONV_F32 ? f((bf16_t *)nullptr, (float *)nullptr)
                                      : f((bf16_t *)nullptr, (bf16_t *)nullptr);
}

int validate(const dconv_join_shape &sh) {
  if (sh.B < 0 || sh.T < 0 || sh.D < 1 || !element_size(sh.dtype) ||
      (sh.vector_dtype != DCONV_F32 && sh.vector_dtype != sh.dtype) ||
      (sh.norm != DCONV_NORM_RMS && sh.norm != DCONV_NORM_LAYER) || (sh.post & ~1) ||
      (sh.per_sample & ~15) || !(sh.eps >= 0.0f))
    return DCONV_EINVAL;
  if (sh.D > kMaxD || (int64_t)sh.B * sh.T > INT_MAX) return DCONV_ERANGE;
  return DCONV_OK;
}

int64_t workspace(const dconv_join_shape &sh) { return (int64_t)sh.B * sh.T * sh.D * 4; }

}  // namespace
}  // namespace dconv

DCONV_EXPORT int dconv_join(const dconv_join_shape *shape, const void *branch, const void *x,
                            const void *post_weight, const void *gate, const void *pre_weight,
                            const void *pre_bias, void *h, void *y, float *stats, void *stream) {
  using namespace dconv;
  if (!shape) return DCONV_ENULL;
  const int rc = validate(*shape);
  if (rc != DCONV_OK) return rc;
  if ((int64_t)shape->B * shape->T == 0) return DCONV_OK;
  if (!x || (branch && !h) || (!h && !y)) return DCONV_ENULL;
  JoinPtrs p = {};
  p.branch = branch;
  p.x = x;
  p.post_weight = post_weight;
  p.gate = gate;
  p.pre_weight = pre_weight;
  p.pre_bias = pre_bias;
  p.h = h;
  p.y = y;
  p.stats = stats;
  (void)hipGetLastError();  // report this launch only
  const hipError_t e = by_types(*shape, [&](auto *t, auto *w) {
    return launch_join<std::remove_pointer_t<decltype(t)>, std::remove_pointer_t<decltype(w)>>(
        *shape, p, (hipStream_t)stream);
  });
  return e == hipSuccess ? DCONV_OK : DCONV_EHIP;
}

DCONV_EXPORT int dconv_join_workspace(const dconv_join_shape *shape, long long *bytes) {
  if (!shape || !bytes) return DCONV_ENULL;
  const int rc = dconv::validate(*shape);
  if (rc == DCONV_OK) *bytes = dconv::workspace(*shape);
  return rc;
}

DCONV_EXPORT int dconv_join_backward(const dconv_join_shape *shape, const void *dh, const void *dy,
                                     const void *branch, const void *x, const void *post_weight,
                                     const void *gate, const void *pre_weight, const float *stats,
                                     void *dbranch, void *dx, void *dpost_weight, void *dgate,
                                     void *dpre_weight, void *dpre_bias, void *workspace,
                                     long long workspace_bytes, void *stream) {
  using namespace dconv;
  if (!shape) return DCONV_ENULL;
  const int rc = validate(*shape);
  if (rc != DCONV_OK) return rc;
  const bool none = (int64_t)shape->B * shape->T == 0;
  if (!none && (branch == nullptr) != (dbranch == nullptr)) return DCONV_ENULL;
  if ((!none && !branch && (dgate || dpost_weight)) || (!shape->post && dpost_weight))
    return DCONV_EINVAL;
  if ((dpost_weight && !post_weight) || (dgate && !gate) || (dpre_weight && !pre_weight))
    return DCONV_ENULL;
  if (!none && (!x || !stats || !dx || !workspace)) return DCONV_ENULL;
  if (workspace_bytes < dconv::workspace(*shape)) return DCONV_EWORKSPACE;
  JoinPtrs p = {};
  p.branch = branch;
  p.x = x;
  p.post_weight = post_weight;
  p.gate = gate;
  p.pre_weight = pre_weight;
  p.dh = dh;
  p.dy = dy;
  p.stats = const_cast<float *>(stats);
  p.dbranch = dbranch;
  p.dx = dx;
  p.dpost_weight = dpost_weight;
  p.dgate = dgate;
  p.dpre_weight = dpre_weight;
  p.dpre_bias = dpre_bias;
  (void)hipGetLastError();  // report this launch only
  const hipError_t e = by_types(*shape, [&](auto *t, auto *w) {
    return launch_join_backward<std::remove_pointer_t<decltype(t)>, std::remove_pointer_t<decltype(w)>>(
        *shape, p, (float *)workspace, (hipStream_t)stream);
  });
  return e == hipSuccess ? DCONV_OK : DCONV_EHIP;
}

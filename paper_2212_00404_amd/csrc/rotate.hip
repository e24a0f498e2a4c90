// Rotary positions with several axes (dconv_rotate).
#include <climits>

#include "internal.h"
#include "tokens.h"

#define DCONV_EXPORT extern "C" __attribute__((visibility("default")))

namespace dconv {
namespace {

// Threads to aim for: two waves per SIMD.  More of them share their sines with
// fewer heads and load the memory no better: a clip of 25088 tokens, 20 heads of
// 128 in bf16 (257 MB) takes 52.9 us with 256 x 512, 53.2 with 256 x 1024, 56.6
// with 256 x 2048 and 63 with twice that.
constexpr int64_t kThreads = 256 * 512;

// sin and cos of position * freq.  The angle is taken in turns: freq / 2pi as
// the sum of two fp32 values, the product with its rounding error (one fma),
// and the whole turns dropped exactly before anything is rounded, so the
// result is good to fp32's last bits at any position (an angle rounded as a
// whole is off by 6e-8 of its size: 0.004 radians at 65536).  The quarter turns
// are dropped likewise; of the eighth that is left the Taylor series to the 9th
// and 10th power are off by less than 2e-9.
__device__ __forceinline__ void turn_sincos(float position, float freq, float *s, float *c) {
  // (fused, p - rintf(p) would hold the product's rounding error a second time)
#pragma clang fp contract(off)
  constexpr float k_hi = 0.15915494309189535f;                          // 1 / 2pi
  constexpr float k_lo = (float)(0.15915494309189533576888 - (double)0.15915494309189535f);
  const float f_hi = freq * k_hi;
  const float f_lo = fmaf(freq, k_lo, fmaf(freq, k_hi, -f_hi));
  const float p = position * f_hi;
  const float e = fmaf(position, f_lo, fmaf(position, f_hi, -p));
  const float turns = (p - rintf(p)) + e;
  const float quarters = rintf(4.0f * turns);
  const float x = 6.28318530717958648f * fmaf(-0.25f, quarters, turns), y = x * x;
  float a = fmaf(y, 1.0f / 362880, -1.0f / 5040);
  a = fmaf(y, a, 1.0f / 120);
  a = fmaf(y, a, -1.0f / 6);
  a = fmaf(x * y, a, x);
  float b = fmaf(y, -1.0f / 3628800, 1.0f / 40320);
  b = fmaf(y, b, -1.0f / 720);
  b = fmaf(y, b, 1.0f / 24);
  b = fmaf(y, b, -0.5f);
  b = fmaf(y, b, 1.0f);
  const int q = (int)quarters;
  const float u = q & 1 ? b : a, w = q & 1 ? a : b;
  *s = q & 2 ? -u : u;
  *c = (q + 1) & 2 ? -w : w;
}

// V elements; on an element's boundary only (the memory takes such accesses as
// one) where rows are not whole 16-byte pieces.
template <class T, int V, bool WHOLE>
struct alignas(WHOLE ? V * sizeof(T) : sizeof(T)) Pack {
  T v[V];
};
// n of the V elements, all of them in one access.
template <class T, int V, bool WHOLE>
__device__ __forceinline__ Pack<T, V, WHOLE> load_pack(const T *p, int n) {
  Pack<T, V, WHOLE> x;
  if (WHOLE || n >= V) return *reinterpret_cast<const Pack<T, V, WHOLE> *>(p);
#pragma unroll
  for (int i = 0; i < V; ++i) x.v[i] = i < n ? p[i] : from_f32<T>(0.0f);
  return x;
}
template <class T, int V, bool WHOLE>
__device__ __forceinline__ void store_pack(T *p, const Pack<T, V, WHOLE> &x, int n) {
  if (WHOLE || n >= V) {
    *reinterpret_cast<Pack<T, V, WHOLE> *>(p) = x;
    return;
  }
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (i < n) p[i] = x.v[i];
}

// Bound by memory: every element is read and written once.  A thread takes one
// piece of a token (P pairs, or V elements past the pairs), computes its sines and
// cosines once (some 60 instructions a pair) and turns that piece in every
// `split`-th head; neighbouring threads take neighbouring pieces, then heads.
struct Work {
  int pieces, pairs;   // pieces per token, those that hold pairs
  int split;           // threads that share a token's heads
  uint32_t threads;    // per sequence
};

// Pieces of V elements (16 bytes).  WHOLE: on 16-byte boundaries, without a
// remainder in a piece of pairs or past them.
template <class T, bool ADJACENT, bool WHOLE>
__device__ __forceinline__ void rotate_piece(const dconv_rotate_shape &sh, const Work &wk, const T *x,
                                             const float *__restrict__ positions, const float *__restrict__ freq,
                                             const int *__restrict__ axis, T *out, int piece, int h0, int64_t t,
                                             int64_t b) {
  constexpr int V = 16 / sizeof(T), P = ADJACENT ? V / 2 : V;   // pairs per piece
  const T *xr = x + b * sh.x_stride[0] + t * sh.x_stride[1];
  T *yr = out + b * sh.out_stride[0] + t * sh.out_stride[1];

  if (piece >= wk.pairs) {   // past the pairs: copied
    const int e = 2 * sh.R + (piece - wk.pairs) * V, n = sh.D - e;
#pragma unroll 4
    for (int h = h0; h < sh.H; h += wk.split)
      store_pack<T, V, WHOLE>(yr + h * sh.out_stride[2] + e,
                              load_pack<T, V, WHOLE>(xr + h * sh.x_stride[2] + e, n), n);
    return;
  }
  const int r0 = piece * P;
  float s[P], c[P];
  bool turned[P];
#pragma unroll
  for (int k = 0; k < P; ++k) {
    const int r = r0 + k;
    const int a = r < sh.R ? axis[r] : -1;
    s[k] = 0.0f;
    c[k] = 1.0f;
    turned[k] = a >= 0 && a < sh.axes;
    if (turned[k])
      turn_sincos(positions[a * sh.pos_stride[0] + b * sh.pos_stride[1] + t * sh.pos_stride[2]], freq[r], &s[k],
                  &c[k]);
    if (sh.inverse) s[k] = -s[k];
  }
  // (a pair that is not turned is copied: 0 times an infinity is not 0)
  auto turn = [&](int k, T &u, T &w) {
    const float fu = to_f32(u), fw = to_f32(w);
    if (turned[k]) {
      // (which product is fused is written out: the same bits in every variant)
      u = from_f32<T>(fmaf(fu, c[k], -(fw * s[k])));
      w = from_f32<T>(fmaf(fu, s[k], fw * c[k]));
    }
  };
  const int eu = ADJACENT ? 2 * r0 : r0, n = ADJACENT ? 2 * (sh.R - r0) : sh.R - r0;
#pragma unroll 4
  for (int h = h0; h < sh.H; h += wk.split) {
    const T *xh = xr + h * sh.x_stride[2];
    T *yh = yr + h * sh.out_stride[2];
    auto u = load_pack<T, V, WHOLE>(xh + eu, n);
    if constexpr (ADJACENT) {
#pragma unroll
      for (int k = 0; k < P; ++k) turn(k, u.v[2 * k], u.v[2 * k + 1]);
    } else {
      auto w = load_pack<T, V, WHOLE>(xh + eu + sh.R, n);
#pragma unroll
      for (int k = 0; k < P; ++k) turn(k, u.v[k], w.v[k]);
      store_pack<T, V, WHOLE>(yh + eu + sh.R, w, n);
    }
    store_pack<T, V, WHOLE>(yh + eu, u, n);
  }
}

template <class T, bool ADJACENT, bool WHOLE>
__global__ __launch_bounds__(256) void rotate_pieces(const dconv_rotate_shape sh, const Work wk, const T *x,
                                                     const float *__restrict__ positions,
                                                     const float *__restrict__ freq, const int *__restrict__ axis,
                                                     T *out) {
  const uint32_t id = blockIdx.x * 256u + threadIdx.x;
  if (id >= wk.threads) return;
  const uint32_t rest = id / wk.pieces, t = rest / wk.split;
  const int piece = (int)(id - rest * wk.pieces), h0 = (int)(rest - t * wk.split);
  for (int64_t b = blockIdx.y; b < sh.B; b += gridDim.y)
    rotate_piece<T, ADJACENT, WHOLE>(sh, wk, x, positions, freq, axis, out, piece, h0, t, b);
}

template <class T, bool ADJACENT, bool WHOLE>
void launch_pieces(const dconv_rotate_shape &sh, const void *x, const float *positions, const float *freq,
                   const int *axis, void *out, hipStream_t s) {
  constexpr int V = 16 / sizeof(T), P = ADJACENT ? V / 2 : V;
  Work wk;
  wk.pairs = (sh.R + P - 1) / P;
  wk.pieces = wk.pairs + (sh.D - 2 * sh.R + V - 1) / V;
  // Each thread takes as many heads as leave threads enough to fill the chip.
  const int64_t per_head = (int64_t)sh.B * sh.T * wk.pieces;
  const int64_t split = (kThreads + per_head - 1) / per_head;
  wk.split = (int)(split < sh.H ? split : sh.H);
  wk.threads = (uint32_t)((int64_t)sh.T * wk.pieces * wk.split);
  hipLaunchKernelGGL((rotate_pieces<T, ADJACENT, WHOLE>), dim3((wk.threads + 255) / 256, sh.B < 65535 ? sh.B : 65535),
                     dim3(256), 0, s, sh, wk, (const T *)x, positions, freq, axis, (T *)out);
}

template <class T>
hipError_t launch(const dconv_rotate_shape &sh, const void *x, const float *positions, const float *freq,
                  const int *axis, void *out, hipStream_t s) {
  constexpr int V = 16 / sizeof(T);
  bool whole = sh.D % V == 0 && (uintptr_t)x % 16 == 0 && (uintptr_t)out % 16 == 0 &&
               sh.R % (sh.adjacent ? V / 2 : V) == 0;
  for (int i = 0; i < 3; ++i) whole = whole && sh.x_stride[i] % V == 0 && sh.out_stride[i] % V == 0;
  if (whole)
    sh.adjacent ? launch_pieces<T, true, true>(sh, x, positions, freq, axis, out, s)
                : launch_pieces<T, false, true>(sh, x, positions, freq, axis, out, s);
  else
    sh.adjacent ? launch_pieces<T, true, false>(sh, x, positions, freq, axis, out, s)
                : launch_pieces<T, false, false>(sh, x, positions, freq, axis, out, s);
  return hipGetLastError();
}

}  // namespace
}  // namespace dconv

DCONV_EXPORT int dconv_rotate(const dconv_rotate_shape *shape, const void *x,
                              const float *positions, const float *freq, const int *axis,
                              void *out, void *stream) {
  if (!shape) return DCONV_ENULL;
  const dconv_rotate_shape &sh = *shape;
  if (sh.B < 0 || sh.T < 0 || sh.H < 1 || sh.D < 1 || sh.R < 0 || sh.R > sh.D / 2 ||
      sh.axes < 1 || (sh.adjacent & ~1) || (sh.inverse & ~1) || !dconv::element_size(sh.dtype))
    return DCONV_EINVAL;
  // a sequence's pieces, one thread each at most, are counted in 32 bits
  const int64_t pieces = (int64_t)sh.D * dconv::element_size(sh.dtype) / 16 + 3;
  if (sh.H > INT_MAX / sh.D || sh.T > (int64_t)(UINT32_MAX - 255) / (sh.H * pieces)) return DCONV_ERANGE;
  if (sh.B == 0 || sh.T == 0) return DCONV_OK;
  if (!x || !out || (sh.R > 0 && (!positions || !freq || !axis))) return DCONV_ENULL;
  (void)hipGetLastError();  // report this launch only
  const hipStream_t s = (hipStream_t)stream;
  const hipError_t e =
      sh.dtype == DCONV_F32
          ? dconv::launch<float>(sh, x, positions, freq, axis, out, s)
          : sh.dtype == DCONV_F16
                ? dconv::launch<dconv::f16_t>(sh, x, positions, freq, axis, out, s)
                : dconv::launch<dconv::bf16_t>(sh, x, positions, freq, axis, out, s);
  return e == hipSuccess ? DCONV_OK : DCONV_EHIP;
}

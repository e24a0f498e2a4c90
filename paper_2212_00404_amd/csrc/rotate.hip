// Rotary positions with several axes (dconv_rotate).
#include <climits>

#include "internal.h"
#include "tokens.h"

#define DCONV_EXPORT extern "C" __attribute__((visibility("default")))

namespace dconv {
namespace {

// sin and cos of position * freq.  The angle is taken in turns: freq / 2pi as
// the sum of two fp32 values, the product with its rounding error (one fma),
// and the whole turns dropped exactly before anything is rounded, so the
// result is good to fp32's last bits at any position (an angle rounded as a
// whole is off by 6e-8 of its size: 0.004 radians at 65536).
__device__ __forceinline__ void turn_sincos(float position, float freq, float *s, float *c) {
  // (fused, p - rintf(p) would hold the product's rounding error a second time)
#pragma clang fp contract(off)
  constexpr float k_hi = 0.15915494309189535f;                          // 1 / 2pi
  constexpr float k_lo = (float)(0.15915494309189533576888 - (double)0.15915494309189535f);
  const float f_hi = freq * k_hi;
  const float f_lo = fmaf(freq, k_lo, fmaf(freq, k_hi, -f_hi));
  const float p = position * f_hi;
  const float e = fmaf(position, f_lo, fmaf(position, f_hi, -p));
  sincospif(2.0f * ((p - rintf(p)) + e), s, c);
}

// One thread per pair, or per element of the unrotated rest.
template <class T>
__global__ __launch_bounds__(256) void rotate_pairs(const dconv_rotate_shape sh, const T *x,
                                                    const float *__restrict__ positions,
                                                    const float *__restrict__ freq,
                                                    const int *__restrict__ axis, T *out) {
  const int per_head = sh.D - sh.R;
  const int64_t n = (int64_t)sh.B * sh.T * sh.H * per_head;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int r = (int)(i % per_head);
    int64_t k = i / per_head;
    const int h = (int)(k % sh.H);
    k /= sh.H;
    const int t = (int)(k % sh.T);
    const int b = (int)(k / sh.T);
    const T *xr = x + b * sh.x_stride[0] + t * sh.x_stride[1] + h * sh.x_stride[2];
    T *yr = out + b * sh.out_stride[0] + t * sh.out_stride[1] + h * sh.out_stride[2];
    if (r >= sh.R) {
      yr[r + sh.R] = xr[r + sh.R];
      continue;
    }
    const int a = axis[r];
    float s = 0.0f, c = 1.0f;
    if (a >= 0 && a < sh.axes)
      turn_sincos(positions[a * sh.pos_stride[0] + b * sh.pos_stride[1] + t * sh.pos_stride[2]],
                  freq[r], &s, &c);
    if (sh.inverse) s = -s;
    const int iu = sh.adjacent ? 2 * r : r, iw = sh.adjacent ? 2 * r + 1 : r + sh.R;
    const float u = to_f32(xr[iu]), w = to_f32(xr[iw]);
    yr[iu] = from_f32<T>(u * c - w * s);
    yr[iw] = from_f32<T>(u * s + w * c);
  }
}

template <class T>
hipError_t launch(const dconv_rotate_shape &sh, const void *x, const float *positions,
                  const float *freq, const int *axis, void *out, hipStream_t s) {
  const int64_t n = (int64_t)sh.B * sh.T * sh.H * (sh.D - sh.R);
  const int64_t blocks = (n + 255) / 256;
  hipLaunchKernelGGL(rotate_pairs<T>, dim3((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20))),
                     dim3(256), 0, s, sh, (const T *)x, positions, freq, axis, (T *)out);
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
  if (sh.H > INT_MAX / sh.D || (int64_t)sh.B * sh.T > INT64_MAX / sh.H / sh.D / 8)
    return DCONV_ERANGE;
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

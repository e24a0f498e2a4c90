// What the kernels of attention over a cache in pages share: which keys a row
// sees, and the plain form of one row, by which the matrix-core kernels are backed.
#pragma once

#include "cache.h"

namespace dconv {

struct CacheAttendPtrs {
  CachePtrs cache;
  const void *q;
  void *out;
  float *lse;
};

// Keys [0, first) and [lo, hi) are what a query at position i sees.
struct KeySpan {
  int first, lo, hi;
  __device__ __forceinline__ bool none() const { return hi - lo + first == 0; }
};
__device__ __forceinline__ KeySpan keys_seen(const dconv_cache_attend_shape &sh, int len, int i) {
  KeySpan r = {0, 0, 0};
  if (i < 0) return r;
  r.hi = sh.right < 0 ? len : (int)min((int64_t)len, (int64_t)i + sh.right + 1);
  r.lo = sh.left < 0 ? 0 : (int)min((int64_t)r.hi, max((int64_t)0, (int64_t)i - sh.left));
  r.first = min(sh.sinks, r.lo);
  return r;
}

constexpr int kLaneParts = kMostHead / 64;   // elements of a head per lane

// Row `row` (of sequence b, whose rows are s) of head h by one wave: 64 keys at a
// time, a key per lane for the products and a part of the head per lane for the
// sum.  Only seen keys and values of pages that are there are read.  The sums are in
// 64 bits: rows come here whose sum of values, before it is divided by that of the
// weights, is past fp32's largest, and their mean is not.
template <class T, int FORMAT>
__device__ void cache_attend_row(const dconv_cache &c, const dconv_cache_attend_shape &sh, const Batch &t,
                                 const CacheAttendPtrs &p, int b, const Rows &s, int row, int h) {
  const int lane = threadIdx.x & 63, D = c.D, hk = h / (sh.Hq / c.Hkv);
  const KeySpan see = keys_seen(sh, s.len, s.start() + (row - s.row));
  const T *q = static_cast<const T *>(p.q) + row * sh.q_stride[0] + h * sh.q_stride[1];
  auto head = [&](const void *base, const long long *stride, int page, int slot) {
    return static_cast<const char *>(base) +
           place(stride, page, slot, hk) * (FORMAT == DCONV_CACHE_PLAIN ? (int64_t)sizeof(T) : 1);
  };
  auto scales = [&](const uint8_t *base, const long long *stride, int page, int slot) {
    return FORMAT == DCONV_CACHE_PLAIN ? base : base + place(stride, page, slot, hk);
  };
  float m = -INFINITY;
  double l = 0.0, acc[kLaneParts] = {};
  bool any = false;
  for (int part = 0; part < 2; ++part) {
    const int end = part ? see.hi : see.first;
    for (int j0 = part ? see.lo : 0; j0 < end; j0 += 64) {
      const int j = j0 + lane;
      float x = -INFINITY;
      int slot = 0;
      const int page = j < end ? page_of(t, p.cache, b, j, &slot) : -1;
      if (page >= 0) {
        const void *k = head(p.cache.k, c.k_stride, page, slot);
        const uint8_t *ks = scales(p.cache.k_scale, c.k_scale_stride, page, slot);
        float sum = 0.0f;
        for (int d = 0; d < D; ++d) sum = fmaf(to_f32(q[d]), element<T, FORMAT>(k, ks, d), sum);
        x = sh.scale * sum;
      }
      any |= __any(page >= 0);
      const float top = fmaxf(m, lanes_max<64>(x));
      // (every score -infinity: exp(x - top) would be NaN)
      const float base = top == -INFINITY ? 0.0f : top;
      const float w = page >= 0 ? expf(x - base) : 0.0f;
      const float keep = expf(m - base);
      m = top;
      l = l * keep + lanes_sum<64>(w);
#pragma unroll
      for (int i = 0; i < kLaneParts; ++i) acc[i] *= keep;
      for (int k = 0; k < 64 && j0 + k < end; ++k) {
        const int kp = __shfl(page, k), ks = __shfl(slot, k);
        const float kw = __shfl(w, k);
        if (kp < 0) continue;
        const void *v = head(p.cache.v, c.v_stride, kp, ks);
        const uint8_t *vs = scales(p.cache.v_scale, c.v_scale_stride, kp, ks);
#pragma unroll
        for (int i = 0; i < kLaneParts; ++i)
          if (lane + 64 * i < D)
            acc[i] = fma((double)kw, (double)element<T, FORMAT>(v, vs, lane + 64 * i), acc[i]);
      }
    }
  }
  T *o = static_cast<T *>(p.out) + row * sh.out_stride[0] + h * sh.out_stride[1];
#pragma unroll
  for (int i = 0; i < kLaneParts; ++i)
    if (lane + 64 * i < D) o[lane + 64 * i] = from_f32<T>(any ? (float)(acc[i] / l) : 0.0f);
  if (p.lse && lane == 0) p.lse[(int64_t)row * sh.Hq + h] = any ? m + logf((float)l) : -INFINITY;
}

// Rows of one key head that are joined from parts: its sums are those that `parts`
// workgroups from `first` on have left.  Each of them joins a share of the rows, this
// the index-th; two such of every workgroup, as for its parts.
struct CacheJoin {
  int parts, first, index;
  int b, hk, r0, rows;   // rows r0 .. of the key head's
  Rows s;
};

// How a call runs: workgroups for sequences of up to 32 rows of a key head
// (cache_few) and for others (cache_tiles), 0 for a kernel that is not needed.
struct CachePlan {
  int dp;                       // head size the kernels are built for
  bool direct, pieces, near;    // as in CacheTile
  int few, tiles;               // workgroups
  int few_least, tiles_least;   // least work of one, in keys
  int few_whole, tiles_whole;   // items of a sequence's key head, if every workgroup takes one; 0: by work
  int64_t joins_bytes, workspace;
};

// Instantiated in cache_attend_*.hip.
template <class T, int FORMAT>
void launch_cache_attend(const dconv_cache &c, const dconv_cache_attend_shape &sh, const Batch &t,
                         const CacheAttendPtrs &p, const CachePlan &plan, char *workspace, hipStream_t s);

}  // namespace dconv

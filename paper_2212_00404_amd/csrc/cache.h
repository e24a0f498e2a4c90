// What the kernels of a cache in pages share: which token a row is, where a
// token stands, and what its bits stand for.
#pragma once

#include "internal.h"
#include "tokens.h"

namespace dconv {

// Division by a divisor that the host knows, as a product and shifts: with
// s = ceil(log2 d) and m = floor(2^32 (2^s - d) / d) + 1, floor(n / d) is
// (t + ((n - t) >> 1)) >> (s - 1) for t the upper half of m n and every n of 32
// bits (Granlund and Montgomery, "Division by invariant integers using
// multiplication", figure 4.1; d = 1 has s = 0 and shifts by none).
struct FastDiv {
  uint32_t d, m;
  int s1, s2;
  FastDiv() = default;
  explicit FastDiv(uint32_t by) : d(by) {
    int s = 0;
    while (s < 32 && (1ull << s) < by) ++s;
    m = (uint32_t)((((1ull << s) - by) << 32) / by + 1);
    s1 = s < 1 ? s : 1;
    s2 = s < 1 ? 0 : s - 1;
  }
  __device__ __forceinline__ uint32_t div(uint32_t n) const {
    const uint32_t t = __umulhi(m, n);
    return (t + ((n - t) >> s1)) >> s2;
  }
};

struct CachePtrs {
  void *k, *v;
  uint8_t *k_scale, *v_scale;
  const int *table, *lengths, *offsets;
};

// The sequences of a call.
struct Batch {
  int B, N, each;      // each: rows of every sequence without offsets
  int pages, width;    // width: of the table
  int most;            // tokens that a table names
  long long table_stride;
  FastDiv page;
};
inline Batch batch_of(const dconv_cache &c, int B, int N, int width, long long table_stride, const int *offsets) {
  Batch t;
  t.B = B;
  t.N = N;
  t.each = offsets ? 0 : N / B;
  t.pages = c.pages;
  t.width = width;
  t.most = width * c.page_size;
  t.table_stride = table_stride;
  t.page = FastDiv((uint32_t)c.page_size);
  return t;
}

// Rows [row, row + n) of a sequence, its length, and the position of the first.
struct Rows {
  int row, n, len;
  __device__ __forceinline__ int start() const { return len - n; }
};
__device__ __forceinline__ Rows rows_of(const Batch &t, const CachePtrs &p, int b) {
  Rows r;
  r.len = min(max(p.lengths[b], 0), t.most);
  if (p.offsets) {
    r.row = min(max(p.offsets[b], 0), t.N);
    r.n = min(max(p.offsets[b + 1], r.row), t.N) - r.row;
  } else {
    r.row = b * t.each;
    r.n = t.each;
  }
  return r;
}

// The sequence of a row by bisection, -1 if that finds none: where offsets rise, the
// row is then of no sequence.  Where they fall somewhere, it finds one that has the row
// for every row in offsets[0] .. offsets[B] - 1, and for others may miss one.
__device__ __forceinline__ int sequence_of(const Batch &t, const CachePtrs &p, int row) {
  if (!p.offsets) return row / t.each;
  int lo = 0, hi = t.B;   // offsets[lo] <= row < offsets[hi], as far as they rise
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (p.offsets[mid] <= row) lo = mid;
    else hi = mid;
  }
  return row >= p.offsets[lo] && row < p.offsets[lo + 1] ? lo : -1;
}

// The page of token i (0 <= i < most) of sequence b, -1 for none.
__device__ __forceinline__ int page_of(const Batch &t, const CachePtrs &p, int b, int i, int *slot) {
  const uint32_t at = t.page.div((uint32_t)i);
  *slot = i - (int)(at * t.page.d);
  const int page = p.table[b * t.table_stride + at];
  return page >= 0 && page < t.pages ? page : -1;
}

__device__ __forceinline__ int64_t place(const long long *stride, int page, int slot, int head) {
  return page * stride[0] + slot * stride[1] + head * stride[2];
}

// ---------------------------------------------------------------------------
// 8 and 4 bits
// ---------------------------------------------------------------------------
constexpr int kBlock = 32;   // elements of a scale

// A scale as the conversions take it: they use the exponent's bits alone (0 is
// 2^-127, 255 makes NaN).
__device__ __forceinline__ float scale_of(uint32_t s) { return __uint_as_float(s << 23); }

// The largest value of a format's mantissa in the type of the rows.
template <class T, int FORMAT>
__device__ __forceinline__ constexpr float limit() {
  constexpr float top = sizeof(T) == 2 && !__is_same(T, bf16_t) ? 0x1p15f : 0x1p127f;
  return FORMAT == DCONV_CACHE_E4M3 ? 1.875f * top : 1.5f * top;
}

// Two codes as values: pair i of a word.
template <class T, int FORMAT>
__device__ __forceinline__ void decode_pair(uint32_t w, int i, float scale, T *out) {
  if constexpr (FORMAT == DCONV_CACHE_E4M3) {
    if constexpr (__is_same(T, float)) {
      const auto r = i ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, true)
                       : __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, false);
      __builtin_memcpy(out, &r, sizeof(r));
    } else if constexpr (__is_same(T, bf16_t)) {
      const auto r = i ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true)
                       : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
      __builtin_memcpy(out, &r, sizeof(r));
    } else {
      const auto r = i ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, true)
                       : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, false);
      __builtin_memcpy(out, &r, sizeof(r));
    }
  } else {
#define DCONV_PAIRS(name)                                                             \
  const auto r = i == 0   ? __builtin_amdgcn_cvt_scalef32_pk_##name##_fp4(w, scale, 0) \
                 : i == 1 ? __builtin_amdgcn_cvt_scalef32_pk_##name##_fp4(w, scale, 1) \
                 : i == 2 ? __builtin_amdgcn_cvt_scalef32_pk_##name##_fp4(w, scale, 2) \
                          : __builtin_amdgcn_cvt_scalef32_pk_##name##_fp4(w, scale, 3)
    if constexpr (__is_same(T, float)) {
      DCONV_PAIRS(f32);
      __builtin_memcpy(out, &r, sizeof(r));
    } else if constexpr (__is_same(T, bf16_t)) {
      DCONV_PAIRS(bf16);
      __builtin_memcpy(out, &r, sizeof(r));
    } else {
      DCONV_PAIRS(f16);
      __builtin_memcpy(out, &r, sizeof(r));
    }
#undef DCONV_PAIRS
  }
}

template <int FORMAT>
constexpr int codes_per_word() { return FORMAT == DCONV_CACHE_E4M3 ? 4 : 8; }

// Element d of a stored head.
template <class T, int FORMAT>
__device__ __forceinline__ float element(const void *head, const uint8_t *scales, int d) {
  if constexpr (FORMAT == DCONV_CACHE_PLAIN) {
    return to_f32(static_cast<const T *>(head)[d]);
  } else {
    constexpr int kPer = codes_per_word<FORMAT>() / 4;   // elements per byte
    T x[2];
    decode_pair<T, FORMAT>(static_cast<const uint8_t *>(head)[d / kPer], 0, scale_of(scales[d / kBlock]), x);
    return to_f32(x[kPer == 2 ? d & 1 : 0]);
  }
}

template <class F>
void by_format(int format, F f) {
  if (format == DCONV_CACHE_PLAIN) return f(std::integral_constant<int, DCONV_CACHE_PLAIN>());
  if (format == DCONV_CACHE_E4M3) return f(std::integral_constant<int, DCONV_CACHE_E4M3>());
  return f(std::integral_constant<int, DCONV_CACHE_E2M1>());
}

constexpr int kMostHead = 256, kMostHeads = 4096, kMostSequences = 1 << 20;

// What every call on a cache checks.
int validate_cache(const dconv_cache &c);
int batch_range(int B, int N, int width, int page_size);
bool cache_pointers(const dconv_cache &c, const CachePtrs &p);

}  // namespace dconv

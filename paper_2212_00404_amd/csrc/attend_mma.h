// Windowed attention on the matrix cores: fragments, tiles in LDS and the two
// forward kernels.  Instantiated per type in attend_*.hip.
//
// All products are 32 x 32 tiles.  Scores are computed transposed, keys along
// the rows of the tile and queries along its columns: a lane then holds half
// of one query's scores (the other half is 32 lanes away), so the maximum, the
// sum and the rescaling of the softmax are register arithmetic, and the
// probabilities already stand where the next product, values transposed times
// probabilities, takes its second operand from (see Mma).
#pragma once

#include "attend.h"

namespace dconv {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) void *lds_ptr;

// 32 x 32 += (32 x 16) (16 x 32).  Operands: lane l holds row (column) l % 32
// and eight of the 16 inner indices, group l / 32.  Result: register i of lane
// l is column l % 32, row acc_row(i, l / 32) = 8 (i / 4) + 4 (l / 32) + i % 4.
// The inner index has no order of its own: eight result registers 8 s .. 8 s + 7
// serve as a second operand whose inner indices are the rows
// 16 s + 8 (e / 4) + 4 (l / 32) + e % 4, if the first operand is read by the
// same rows (Tile::column).
// fp32 takes eight 32 x 32 x 2 instructions, one per element of the fragment.
template <class T>
struct Mma;
template <>
struct Mma<bf16_t> {
  typedef bf16_t Frag __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x16 mac(Frag a, Frag b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Mma<f16_t> {
  typedef f16_t Frag __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x16 mac(Frag a, Frag b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Mma<float> {
  typedef float Frag __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x16 mac(Frag a, Frag b, f32x16 c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
    return c;
  }
};

__device__ __forceinline__ constexpr int acc_row(int i, int half) { return 8 * (i / 4) + 4 * half + i % 4; }

// Registers 8 s .. 8 s + 7 of a result as an operand.
template <class T>
__device__ __forceinline__ typename Mma<T>::Frag as_operand(const f32x16 &c, int s) {
  typename Mma<T>::Frag f;
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = from_f32<T>(c[8 * s + e]);
  return f;
}

// Rows of DP elements in LDS, in chunks of eight elements that are permuted
// within a row by an exclusive or with bits of the row's number.  LDS serves 256
// bytes, sixteen chunks of 16 bytes, at a time: sixteen consecutive rows of one
// chunk (a row operand), and four rows of four neighbouring chunks (a column
// operand), shall lie on different banks.
template <class T, int DP>
struct Tile {
  typedef typename Mma<T>::Frag Frag;
  static constexpr int kChunks = DP / 8;
  static __device__ __forceinline__ int swizzle(int row) {
    if constexpr (sizeof(T) == 4) return DP % 64 == 0 ? row & 7 : row & 3;
    // rows of 256 bytes begin on one bank; of 128 on two in turn; of 64 and 192 on four
    if constexpr (DP % 128 == 0) return (row & 3) << 2 | (row >> 2 & 3);
    if constexpr (DP % 64 == 0) return (row >> 1 & 1) << 2 | (row >> 2 & 3);
    return row >> 2 & 3;
  }
  static __device__ __forceinline__ int at(int row, int chunk) { return row * DP + (chunk ^ swizzle(row)) * 8; }

  // Elements 16 s + 8 (l / 32) .. + 7 of row r0 + l % 32.
  static __device__ __forceinline__ Frag row(const T *t, int r0, int s, int lane) {
    const T *p = t + at(r0 + (lane & 31), 2 * s + (lane >> 5));
    if constexpr (sizeof(T) == 4) {
      // (two loads of 16 bytes: one of 32, split by the compiler, loses which
      // buffer it reads and waits for the copies into the other one)
      typedef float f32x4 __attribute__((ext_vector_type(4)));
      const f32x4 a = *reinterpret_cast<const f32x4 *>(p), b = *reinterpret_cast<const f32x4 *>(p + 4);
      return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      return *reinterpret_cast<const Frag *>(p);
    }
  }
  // Column 32 c + l % 32 of the rows r0 + 8 (e / 4) + 4 (l / 32) + e % 4
  // (r0 a multiple of 16).
  static __device__ __forceinline__ Frag column(const T *t, int r0, int c, int lane) {
    Frag f;
    if constexpr (sizeof(T) == 2) {
      // a 16-lane group reads four rows of 16 elements, a lane four of a row,
      // and gets four rows of one column
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) s16x4 *lds_s16x4;
      const int r = r0 + 4 * (lane >> 5) + ((lane & 15) >> 2);
      const int chunk = 4 * c + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
      s16x4 v[2];
#pragma unroll
      for (int j = 0; j < 2; ++j)
        v[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_s16x4)(t + at(r + 8 * j, chunk) + 4 * (lane & 1)));
      __builtin_memcpy(&f, v, 16);
    } else {
      const int d = 32 * c + (lane & 31);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = t[at(r0 + 8 * (e / 4) + 4 * (lane >> 5) + e % 4, d >> 3) + (d & 7)];
    }
    return f;
  }

};

// Copies of NR rows of D elements into a Tile by NW waves.
template <class T, int DP, int NR, int NW>
struct Copy {
  static constexpr int kPer = 16 / sizeof(T), kPieces = DP / kPer, kThreads = 64 * NW;
  static constexpr int kCopies = (NR * kPieces + kThreads - 1) / kThreads;   // per wave
  static_assert(NR * kPieces % 64 == 0, "whole waves");
  // Rows between a lane's copies, where they are in the same place of a row.
  static constexpr int kStep = kThreads % (16 * kPieces) == 0 ? kThreads / kPieces : 0;
  uint32_t offset[kStep ? 1 : kCopies];   // of the lane's pieces from the tile's first row, in bytes

  // Row and element of the lane's piece in copy i.  A piece past D repeats the
  // row's first (its products meet zeros).
  static __device__ __forceinline__ int row(int i, int wave, int lane) { return (i * kThreads + 64 * wave + lane) / kPieces; }
  static __device__ __forceinline__ int element(int i, int wave, int lane, int D) {
    const int piece = (i * kThreads + 64 * wave + lane) % kPieces;
    const int e = ((piece * kPer / 8) ^ Tile<T, DP>::swizzle(row(i, wave, lane))) * 8 + piece * kPer % 8;
    return e < D ? e : 0;
  }
  static __device__ __forceinline__ bool has(int i, int wave) {
    return NR * kPieces % kThreads == 0 || i * kThreads + 64 * wave < NR * kPieces;
  }
  static __device__ __forceinline__ T *to(T *lds, int i, int wave) {   // lane l lands 16 l bytes on
    return lds + (i * kThreads + 64 * wave) * kPer;
  }

  // byte_offset(r): of row r from the tile's first, in 32 bits.
  template <class F>
  __device__ __forceinline__ void init(int D, int wave, int lane, F byte_offset) {
#pragma unroll
    for (int i = 0; i < (kStep ? 1 : kCopies); ++i)
      offset[i] = byte_offset(row(i, wave, lane)) + element(i, wave, lane, D) * (uint32_t)sizeof(T);
  }
  // The rows as init has described them, from `first`; row r + kStep is `step`
  // bytes after row r.  One instruction per copy: a scalar base and a 32-bit offset.
  __device__ __forceinline__ void tile(T *lds, const T *first, int64_t step, int wave) const {
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      if (!has(i, wave)) break;
      uint32_t o = offset[kStep ? 0 : i];
      asm volatile("" : "+v"(o));
      const char *base = reinterpret_cast<const char *>(first) + (kStep ? i * step : 0);
      __builtin_amdgcn_global_load_lds(base + o, (lds_ptr)to(lds, i, wave), 16, 0, 0);
    }
  }
  // The same with offsets computed here.
  template <class F>
  static __device__ __forceinline__ void tile_at(T *lds, const T *first, int D, int wave, int lane, F byte_offset) {
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      if (!has(i, wave)) break;
      uint32_t o = byte_offset(row(i, wave, lane)) + element(i, wave, lane, D) * (uint32_t)sizeof(T);
      asm volatile("" : "+v"(o));
      __builtin_amdgcn_global_load_lds(reinterpret_cast<const char *>(first) + o, (lds_ptr)to(lds, i, wave), 16, 0, 0);
    }
  }
  // Any rows: row_start(r) is where row r begins.
  template <class F>
  static __device__ __forceinline__ void rows(T *lds, int D, int wave, int lane, F row_start) {
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      if (!has(i, wave)) break;
      __builtin_amdgcn_global_load_lds(row_start(row(i, wave, lane)) + element(i, wave, lane, D),
                                       (lds_ptr)to(lds, i, wave), 16, 0, 0);
    }
  }
  // Rows that are not whole 16-byte pieces: element by element, zeros past D.
  template <class F>
  static __device__ __forceinline__ void elements(T *lds, int D, int wave, int lane, F row_start) {
    for (int x = 64 * wave + lane; x < NR * DP; x += kThreads) {
      const int r = x / DP, d = x % DP;
      lds[Tile<T, DP>::at(r, d >> 3) + (d & 7)] = d < D ? row_start(r)[d] : from_f32<T>(0.0f);
    }
  }
};

// Eight elements of a row in memory from d on, times `sign`; zeros past D.
template <class T>
__device__ __forceinline__ typename Mma<T>::Frag load_frag(const T *row, int d, int D, bool direct, float sign) {
  typename Mma<T>::Frag f;
  if (direct && d + 8 <= D) {
    __builtin_memcpy(&f, __builtin_assume_aligned(row + d, 4), sizeof(f));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = d + e < D ? row[d + e] : from_f32<T>(0.0f);
  }
  if (sign != 1.0f) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = from_f32<T>(to_f32(f[e]) * sign);
  }
  return f;
}

// Waits until at most N of this wave's copies, and no LDS operation, are on their
// way.  (As an instruction that the compiler knows: it counts copies into LDS too,
// and after a wait it cannot see it would put its own, for all of them, before the
// first read.)
template <int N>
__device__ __forceinline__ void landed() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | 7 << 4 | (N >> 4) << 14);   // vmcnt(N) lgkmcnt(0)
  asm volatile("" ::: "memory");
}

// 2^x.  The instruction gives 0 below 2^-126; fp32 tensors keep such values, for
// 16-bit ones they are far below what a probability is rounded to.
template <class T>
__device__ __forceinline__ float power2(float x) {
  return sizeof(T) == 4 ? exp2f(x) : __builtin_amdgcn_exp2f(x);
}

// The other half of a query's lanes, 32 away.
__device__ __forceinline__ float half_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Keeps a branch a branch: the compiler would otherwise run a rare block's
// arithmetic every time and select.
__device__ __forceinline__ void no_speculation() { asm volatile(""); }

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// f(i, whether acc_row(i, half) lies in [lo, hi)): one subtraction and one
// comparison each.
template <class F>
__device__ __forceinline__ void within(int lo, int hi, int half, F f) {
  const unsigned from = (unsigned)(lo - 4 * half), span = (unsigned)max(hi - lo, 0);
#pragma unroll
  for (int i = 0; i < 16; ++i) f(i, (unsigned)acc_row(i, 0) - from < span);
}

// What the host hands to the tile kernels beside the shape.
struct AttendTile {
  float scale2;   // |scale| / ln 2: the softmax is taken in powers of two
  float sign;     // of the scale, taken into the queries; 0: every score is 0
  bool direct;    // rows can be copied in 16-byte pieces
  bool near;      // and 64 of them span less than 2^31 bytes
  int tiles;      // tiles of rows per key head
  int splits;     // parts of the keys (attend_split)
  float *partial; // their sums
};

// Rows of a group: row r of key head hk is query r / G of head hk * G + r % G, so
// that the heads that share keys share the tiles of them.  The keys that any row
// of a tile sees are numbered v = 0 .. n - 1: the first keys, then the window.
struct Keys {
  int n, first, off;
  __device__ __forceinline__ int key(int v) const { return v < first ? v : v + off; }
};
__device__ __forceinline__ Keys keys_of(const dconv_attend_shape &sh, const Seq &s, int t0, int t1) {
  Keys k = {0, 0, 0};
  if (s.start + t1 < 0) return k;
  const Span a = span_of(sh, s, max((int64_t)0, s.start + t0)), b = span_of(sh, s, s.start + t1);
  k.first = uniform(a.first);
  k.off = uniform(a.lo - a.first);
  k.n = uniform(b.hi - k.off);
  return k;
}
// Tiles of keys and values, in this order, of one key head.
template <class T, int DP, int BN, int NW>
struct KeyTiles {
  Copy<T, DP, BN, NW> ck, cv;
  const T *k, *v;
  int64_t k_stride, v_stride;

  __device__ __forceinline__ KeyTiles(const dconv_attend_shape &sh, const AttendPtrs &p, int b, int hk, int wave,
                                      int lane)
      : k(row_of<T>(p.k, sh.k_stride, b, 0, hk)), v(row_of<T>(p.v, sh.v_stride, b, 0, hk)),
        k_stride(sh.k_stride[1]), v_stride(sh.v_stride[1]) {
    ck.init(sh.D, wave, lane, [&](int r) { return (uint32_t)r * (uint32_t)k_stride * (uint32_t)sizeof(T); });
    cv.init(sh.D, wave, lane, [&](int r) { return (uint32_t)r * (uint32_t)v_stride * (uint32_t)sizeof(T); });
  }
  // Keys v0 .. of the n of `keys`; past the last one it is repeated.
  __device__ __forceinline__ void stage(T *lds, const AttendTile &at, const Keys &keys, int n, int v0, int D, int wave,
                                        int lane) const {
    typedef Copy<T, DP, BN, NW> C;
    if (at.near && v0 + BN <= n && (v0 >= keys.first || keys.off == 0)) {
      const int64_t j = v0 + keys.off;
      ck.tile(lds, k + j * k_stride, C::kStep * k_stride * (int64_t)sizeof(T), wave);
      cv.tile(lds + BN * DP, v + j * v_stride, C::kStep * v_stride * (int64_t)sizeof(T), wave);
      return;
    }
    auto from = [&](const T *base, int64_t stride) {
      return [=](int r) { return base + (int64_t)keys.key(min(v0 + r, n - 1)) * stride; };
    };
    if (at.direct) {
      C::rows(lds, D, wave, lane, from(k, k_stride));
      C::rows(lds + BN * DP, D, wave, lane, from(v, v_stride));
    } else {
      C::elements(lds, D, wave, lane, from(k, k_stride));
      C::elements(lds + BN * DP, D, wave, lane, from(v, v_stride));
    }
  }
};

// Row at position i sees v < hi with v >= lo or v < sinks.
struct RowKeys {
  int lo, hi;
  bool none;
};
__device__ __forceinline__ RowKeys row_keys(const dconv_attend_shape &sh, const Seq &s, const Keys &k, int64_t i) {
  const Span a = span_of(sh, s, i);
  RowKeys r;
  r.none = a.hi - a.lo + a.first == 0;
  r.lo = a.lo - k.off;
  r.hi = r.none ? 0 : a.hi - k.off;
  return r;
}

// What reads LDS and what multiplies stays on its side of this line (vector and
// scalar arithmetic may cross): operands are read well before their products.
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0x2 | 0x4 | 0x400); }

// f(i, whether register i's key, of those from v0 on, is seen by the lane's row).
template <class F>
__device__ __forceinline__ void seen_keys(int v0, const RowKeys &see, int sinks, int lane, F f) {
  const int half = lane >> 5;
  if (v0 >= sinks) {
    within(see.lo - v0, see.hi - v0, half, f);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int v = v0 + acc_row(i, half);
      f(i, v < see.hi && (v >= see.lo || v < sinks));
    }
  }
}

// The running softmax of 32 rows by one wave: each lane half of a row.
template <class T, int DP>
struct Softmax {
  static constexpr int KS = DP / 16, DT = DP / 32;
  typedef typename Mma<T>::Frag Frag;
  f32x16 o[DT];   // o[c][i]: column 32 c + acc_row(i, half) of the row
  float m, l;     // base of the exponentials (in powers of two), this lane's sum

  __device__ __forceinline__ void clear() {
    for (int c = 0; c < DT; ++c) o[c] = f32x16{};
    m = -INFINITY;
    l = 0.0f;
  }

  // 32 scores of each row: keys k0 .. of the tile.
  static __device__ __forceinline__ f32x16 scores(const T *ks, int k0, const Frag (&q)[KS], int lane) {
    f32x16 s = {};
#pragma unroll
    for (int k = 0; k < KS; ++k) s = Mma<T>::mac(Tile<T, DP>::row(ks, k0, k, lane), q[k], s);
    return s;
  }
  // gone: bit k for key v0 + k that nobody sees.
  static __device__ __forceinline__ void mask(f32x16 &s, int v0, const RowKeys &see, int sinks, int lane,
                                              uint32_t gone = 0) {
    seen_keys(v0, see, sinks, lane, [&](int i, bool on) { s[i] = on ? s[i] : -INFINITY; });
    if (gone) {
      no_speculation();
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = gone >> acc_row(i, lane >> 5) & 1 ? -INFINITY : s[i];
    }
  }
  // The base is set kBelow powers of two under the largest score, and follows it only
  // when it is left kLag further behind: sums and probabilities stay below
  // 2^(kBelow + kLag) times their true size, and the rescaling of the result is rare.
  // bf16 and fp32 have range enough for the base to be the largest itself.  An fp16
  // operand is rounded to steps of 2^-24 however small it is: with the base at the
  // largest, a key of 2^-25.5 of its weight would be lost from the result and kept in the
  // sum, 0.28% of all weight for 131072 such keys beside one.  From 2^10 under it steps are
  // 2^-34 of the largest's weight (131072 keys: 2^-18 of it lost at most), and
  // 2^14 leaves two powers of two of fp16's range for the rounding of large scores.
  // The price is a lag of 2^4 instead of 2^8.
  static constexpr float kBelow = __is_same(T, f16_t) ? 10.0f : 0.0f, kLag = __is_same(T, f16_t) ? 4.0f : 8.0f;
  // before(): what has to be added first.
  template <class F>
  __device__ __forceinline__ void follow(const f32x16 &s, float scale2, F before) {
    float top = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
    top = half_max(top) * scale2;
    if (__any(top - m > kBelow + kLag)) {
      before();
      const float to = fmaxf(m, top - kBelow);
      const float keep = to == -INFINITY ? 1.0f : exp2f(m - to);
#pragma unroll
      for (int c = 0; c < DT; ++c) o[c] *= keep;
      l *= keep;
      m = to;
    }
  }
  // Scores to probabilities (times 2^-m), as operands: rounded to the tensors' type,
  // which the matrix instructions take.  Their sum is of the values before that.  (A
  // result is then off by 1.3 times what its own rounding alone leaves: 0.0021 of its
  // size against 0.0016 for the prompt in bf16.  Operands of twice the bits would be
  // twice the products.)
  __device__ __forceinline__ void probabilities(const f32x16 &s, float scale2, Frag (&w)[2]) {
    const float base = m == -INFINITY ? 0.0f : m;
    f32x16 x;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      x[i] = power2<T>(fmaf(s[i], scale2, -base));
      l += x[i];
    }
    w[0] = as_operand<T>(x, 0);
    w[1] = as_operand<T>(x, 1);
  }
  // The result plus the values k0 .. of the tile times their probabilities.
  __device__ __forceinline__ void values(const T *vs, int k0, const Frag (&w)[2], int lane) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int c = 0; c < DT; ++c) o[c] = Mma<T>::mac(Tile<T, DP>::column(vs, k0 + 16 * k, c, lane), w[k], o[c]);
  }

  static __device__ __forceinline__ void load_keys(Frag (&f)[KS], const T *ks, int k0, int lane) {
#pragma unroll
    for (int k = 0; k < KS; ++k) f[k] = Tile<T, DP>::row(ks, k0, k, lane);
  }
  static __device__ __forceinline__ void load_values(Frag (&f)[DT], const T *vs, int k0, int lane) {
#pragma unroll
    for (int c = 0; c < DT; ++c) f[c] = Tile<T, DP>::column(vs, k0, c, lane);
  }
  static __device__ __forceinline__ f32x16 products(const Frag (&f)[KS], const Frag (&q)[KS]) {
    f32x16 s = {};
#pragma unroll
    for (int k = 0; k < KS; ++k) s = Mma<T>::mac(f[k], q[k], s);
    return s;
  }
  __device__ __forceinline__ void weigh(const Frag (&f)[DT], Frag w) {
#pragma unroll
    for (int c = 0; c < DT; ++c) o[c] = Mma<T>::mac(f[c], w, o[c]);
  }

  // Adds 32 keys, v0 .., of the tiles ks, vs.
  __device__ __forceinline__ void add(const T *ks, const T *vs, const Frag (&q)[KS], int v0, const RowKeys &see,
                                      int sinks, float scale2, bool masked, int lane) {
    f32x16 s = scores(ks, 0, q, lane);
    if (masked) mask(s, v0, see, sinks, lane);
    follow(s, scale2, [] {});
    Frag w[2];
    probabilities(s, scale2, w);
    values(vs, 0, w, lane);
  }
  // Adds 64 keys.  The second half's scores are computed beside the first half's
  // probabilities, and the first half's sum beside the second's probabilities: the
  // matrix and the vector unit work at the same time within a wave.
  __device__ __forceinline__ void add_two(const T *ks, const T *vs, const Frag (&q)[KS], int v0, const RowKeys &see,
                                          int sinks, float scale2, bool masked, int lane) {
    Frag w0[2], w1[2];
    if constexpr (DP > 96) {
      // (operands read ahead would not leave registers for two waves per SIMD, and
      // a register that comes back from memory waits for the copies too)
      f32x16 s0 = scores(ks, 0, q, lane);
      if (masked) mask(s0, v0, see, sinks, lane);
      follow(s0, scale2, [] {});
      f32x16 s1 = scores(ks, 32, q, lane);
      probabilities(s0, scale2, w0);
      asm volatile("" ::"v"(w0[0]), "v"(w0[1]));   // here, not after the next branch
      if (masked) mask(s1, v0 + 32, see, sinks, lane);
      follow(s1, scale2, [&] {
        values(vs, 0, w0, lane);
        w0[0] = w0[1] = Frag{};
      });
      values(vs, 0, w0, lane);
      probabilities(s1, scale2, w1);
      values(vs, 32, w1, lane);
      return;
    }
    Frag kf[KS], vf[2][DT];
    load_keys(kf, ks, 0, lane);
    in_order();
    f32x16 s0 = products(kf, q), s1;
    load_keys(kf, ks, 32, lane);
    in_order();
    if (masked) mask(s0, v0, see, sinks, lane);
    follow(s0, scale2, [] {});
    s1 = products(kf, q);
    load_values(vf[0], vs, 0, lane);
    in_order();
    probabilities(s0, scale2, w0);
    asm volatile("" ::"v"(w0[0]), "v"(w0[1]));
    if (masked) mask(s1, v0 + 32, see, sinks, lane);
    follow(s1, scale2, [&] {
      values(vs, 0, w0, lane);
      w0[0] = w0[1] = Frag{};
    });
    load_values(vf[1], vs, 16, lane);
    in_order();
    weigh(vf[0], w0[0]);
    load_values(vf[0], vs, 32, lane);
    in_order();
    weigh(vf[1], w0[1]);
    load_values(vf[1], vs, 48, lane);
    in_order();
    probabilities(s1, scale2, w1);
    weigh(vf[0], w1[0]);
    weigh(vf[1], w1[1]);
  }
};

// log(2) (m + log2(l))
__device__ __forceinline__ float log_sum(float m, float l) { return 0.69314718055994531f * (m + log2f(l)); }

template <class T>
constexpr int forward_keys(int dp) { return dp * (int)sizeof(T) <= 256 ? 64 : 32; }
constexpr int kForwardRows = 128;

// 128 rows per workgroup, 32 per wave; tiles of BN keys and values in two LDS
// buffers, the next one copied while the current one is used.  Registers for two
// workgroups per compute unit (a prompt of 8192 tokens, 32 heads of 128 over 8, window
// 1024, bf16: 295 us with one, 178 with two, 129 GFLOP of seen scores).  There the
// matrix cores run 0.40 of the cycles and vector instructions issue in 0.50 of them;
// leaving out the copies changes nothing, LDS is busy 0.2: what bounds it is vector
// issue beside the products, some 110 instructions and 32 exponentials per 64 keys.
template <class T, int DP>
__global__ __launch_bounds__(256, DP * sizeof(T) <= 256 ? 2 : 1) void attend_tiles(const dconv_attend_shape sh, const AttendPtrs p,
                                                    const AttendTile at) {
  constexpr int BN = forward_keys<T>(DP), KS = DP / 16, DT = DP / 32;
  __shared__ __align__(16) T buf0[2 * BN * DP];
  __shared__ __align__(16) T buf1[2 * BN * DP];
  DCONV_POISON(poison_lds(buf0, 2 * BN * DP); poison_lds(buf1, 2 * BN * DP));
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int id = xcd_remap(blockIdx.x, gridDim.x);
  const int bh = id / at.tiles, b = bh / sh.Hkv, hk = bh % sh.Hkv, G = sh.Hq / sh.Hkv;
  const int r0 = (id % at.tiles) * kForwardRows, rows = sh.Tq * G;
  const Seq seq = seq_of(sh, p, b);
  const Keys keys = keys_of(sh, seq, r0 / G, (min(r0 + kForwardRows, rows) - 1) / G);
  const int n = uniform(keys.n);

  const int r = r0 + 32 * wave + (lane & 31), rr = min(r, rows - 1);
  const int t = rr / G, h = hk * G + rr % G;
  const RowKeys see = row_keys(sh, seq, keys, seq.start + t);
  // the wave's keys: none outside [from, to) but for the first ones, all visible
  // to all rows inside [all_from, all_to)
  int from = see.lo, to = see.hi, all_from = see.lo, all_to = see.hi;
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) {
    from = min(from, __shfl_xor(from, x));
    to = max(to, __shfl_xor(to, x));
    all_from = max(all_from, __shfl_xor(all_from, x));
    all_to = min(all_to, __shfl_xor(all_to, x));
  }
  from = uniform(from), to = uniform(to), all_from = uniform(all_from), all_to = uniform(all_to);

  typename Mma<T>::Frag q[KS];
  const T *qrow = row_of<T>(p.q, sh.q_stride, b, t, h);
#pragma unroll
  for (int k = 0; k < KS; ++k) q[k] = load_frag(qrow, 16 * k + 8 * (lane >> 5), sh.D, at.direct, at.sign);

  const KeyTiles<T, DP, BN, 4> tiles(sh, p, b, hk, wave, lane);
  auto stage = [&](T *buf, int v0) { tiles.stage(buf, at, keys, n, v0, sh.D, wave, lane); };
  Softmax<T, DP> soft;
  soft.clear();
  // keys v0 .. v0 + N - 1 by the wave's rows: none seen, all seen
  auto unseen = [&](int v0, int N) { return v0 >= to || (v0 + N <= from && v0 >= sh.sinks); };
  auto masked = [&](int v0, int N) { return !(v0 + N <= all_to && (v0 >= all_from || v0 + N <= sh.sinks)); };
  auto step = [&](const T *buf, int v0) {
    if constexpr (BN == 64 && sizeof(T) == 2) {
      if (!unseen(v0, BN))
        soft.add_two(buf, buf + BN * DP, q, v0, see, sh.sinks, at.scale2, masked(v0, BN), lane);
    } else {
      // (fp32: a tile's products last long enough by themselves)
#pragma unroll
      for (int k = 0; k < BN; k += 32)
        if (!unseen(v0 + k, 32))
          soft.add(buf + k * DP, buf + (BN + k) * DP, q, v0 + k, see, sh.sinks, at.scale2, masked(v0 + k, 32), lane);
    }
  };
  auto arrived = [&]() {
    landed<0>();
    __syncthreads();
  };
  if (n > 0) stage(buf0, 0);
  for (int v0 = 0; v0 < n; v0 += 2 * BN) {
    arrived();
    if (v0 + BN < n) stage(buf1, v0 + BN);
    step(buf0, v0);
    if (v0 + BN >= n) break;
    arrived();
    if (v0 + 2 * BN < n) stage(buf0, v0 + 2 * BN);
    step(buf1, v0 + BN);
  }

  const float l = half_sum(soft.l), inv = see.none ? 0.0f : 1.0f / l;
  bool bad = false;
#pragma unroll
  for (int c = 0; c < DT; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      soft.o[c][i] = see.none ? 0.0f : soft.o[c][i] * inv;
      bad |= 32 * c + acc_row(i, lane >> 5) < sh.D && !(fabsf(soft.o[c][i]) < INFINITY);
    }
  const unsigned long long any = __ballot(bad && r < rows);
  const unsigned redo = kSumAgain ? (unsigned)(any | (any >> 32)) : 0u;
  if (r < rows && !(redo >> (lane & 31) & 1)) {
    T *o = (T *)p.o + b * sh.out_stride[0] + t * sh.out_stride[1] + h * sh.out_stride[2];
#pragma unroll
    for (int c = 0; c < DT; ++c)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int d = 32 * c + acc_row(i, lane >> 5);
        T x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = from_f32<T>(soft.o[c][i + e]);
        if (at.direct && d + 4 <= sh.D) {
          __builtin_memcpy(__builtin_assume_aligned(o + d, 4), x, sizeof(x));
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (d + e < sh.D) o[d + e] = x[e];
        }
      }
    if (p.lse_out && lane < 32)
      p.lse_out[((int64_t)b * sh.Hq + h) * sh.Tq + t] = see.none ? -INFINITY : log_sum(soft.m, l);
  }
  // A row with a result that is not finite is taken again by the plain form,
  // which reads visible keys and values only: a zero probability times an
  // infinity or NaN that the row does not see has made a NaN here.
  for (unsigned again = redo; again; again &= again - 1) {
    const int x = r0 + 32 * wave + __ffs(again) - 1;
    attend_row<T>(sh, p, b, hk * G + x % G, x / G);
  }
}

// ---------------------------------------------------------------------------
// Few rows: the keys divided over waves and workgroups
// ---------------------------------------------------------------------------
template <class T>
constexpr int split_waves(int dp) { return dp * (int)sizeof(T) <= 256 ? 4 : dp * (int)sizeof(T) <= 512 ? 2 : 1; }

// The result registers of W waves in LDS (in two buffers of W 2 x 32 x DP elements):
// register i of part c of wave w in a row of 64 lanes, 65 floats apart, so that both
// a register's lanes and a result row's elements lie on different banks (rows of
// DP floats, written a row per lane, would put all lanes on one).
template <class T, int DP, int W>
struct WaveSums {
  static constexpr int DT = DP / 32, kWave = DT * 16 * 65, kHalf = (W + 1) / 2;
  static_assert(kHalf * kWave * sizeof(float) <= W * 2 * 32 * DP * sizeof(T), "half the waves fit a buffer");
  T *buf0, *buf1;
  __device__ __forceinline__ float *of(int w) const {
    return reinterpret_cast<float *>(w < kHalf ? buf0 : buf1) + (w < kHalf ? w : w - kHalf) * kWave;
  }
  __device__ __forceinline__ void leave(int w, int lane, const f32x16 (&o)[DT]) const {
    float *to = of(w) + lane;
#pragma unroll
    for (int c = 0; c < DT; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) to[(16 * c + i) * 65] = o[c][i];
  }
  // Element d of column x of the wave's result.
  __device__ __forceinline__ float get(int w, int x, int d) const {
    const int i = (d >> 5) * 16 + (d >> 3 & 3) * 4 + (d & 3);
    return of(w)[i * 65 + (d >> 2 & 1) * 32 + x];
  }
};

// One row's parts joined: lane l gets elements l, l + 64, ... of the result.
// base(i), sum(i) and value(i, d) of part i, not divided by its sum.
template <class T, class M, class L, class V>
__device__ __forceinline__ void join_parts(const dconv_attend_shape &sh, const AttendPtrs &p, int b, int h, int t,
                                           bool none, int parts, M base_of, L sum_of, V value) {
  const int lane = threadIdx.x & 63;
  float m = -INFINITY, l = 0.0f, acc[kRowParts] = {};
  for (int i = 0; i < parts; ++i) m = fmaxf(m, base_of(i));
  const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll 4
  for (int i = 0; i < parts; ++i) {
    const float w = exp2f(base_of(i) - base);
    l += w * sum_of(i);
#pragma unroll
    for (int k = 0; k < kRowParts; ++k)
      if (lane + 64 * k < sh.D) acc[k] = fmaf(w, value(i, lane + 64 * k), acc[k]);
  }
  bool bad = false;
#pragma unroll
  for (int k = 0; k < kRowParts; ++k) {
    acc[k] = none ? 0.0f : acc[k] / l;
    bad |= lane + 64 * k < sh.D && !(fabsf(acc[k]) < INFINITY);
  }
  if (kSumAgain && __any(bad)) {
    attend_row<T>(sh, p, b, h, t);
    return;
  }
  T *o = (T *)p.o + b * sh.out_stride[0] + t * sh.out_stride[1] + h * sh.out_stride[2];
#pragma unroll
  for (int k = 0; k < kRowParts; ++k)
    if (lane + 64 * k < sh.D) o[lane + 64 * k] = from_f32<T>(acc[k]);
  if (p.lse_out && lane == 0)
    p.lse_out[((int64_t)b * sh.Hq + h) * sh.Tq + t] = none ? -INFINITY : log_sum(m, l);
}

// Floats of one part of 32 rows in the workspace: bases, sums, rows.
template <int DP>
constexpr int part_floats() { return attend_part_floats(DP); }

// 32 rows per workgroup; wave w of part s takes tiles of 32 keys by itself, with
// two LDS buffers of its own and no barrier.  Bound by memory where there are keys
// enough: 16 sequences, 8 key heads of 128, 4100 keys each of bf16 caches, 248 MB in
// 44.5 us (5.6 TB/s), one workgroup per compute unit with 64 KB of copies on their way.
template <class T, int DP>
__global__ __launch_bounds__(64 * split_waves<T>(DP), 1) void attend_split(const dconv_attend_shape sh,
                                                                        const AttendPtrs p, const AttendTile at) {
  constexpr int KS = DP / 16, kTile = 32 * DP, W = split_waves<T>(DP);
  __shared__ __align__(16) T buf0[W * 2 * kTile];
  __shared__ __align__(16) T buf1[W * 2 * kTile];
  DCONV_POISON(poison_lds(buf0, W * 2 * kTile); poison_lds(buf1, W * 2 * kTile));
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int part = blockIdx.x % at.splits, id = blockIdx.x / at.splits;
  const int bh = id / at.tiles, b = bh / sh.Hkv, hk = bh % sh.Hkv, G = sh.Hq / sh.Hkv;
  const int r0 = (id % at.tiles) * 32, rows = sh.Tq * G;
  const Seq seq = seq_of(sh, p, b);
  const Keys keys = keys_of(sh, seq, r0 / G, (min(r0 + 32, rows) - 1) / G);
  const int n = uniform(keys.n);
  const int rr = min(r0 + (lane & 31), rows - 1), t = rr / G, h = hk * G + rr % G;
  const RowKeys see = row_keys(sh, seq, keys, seq.start + t);

  typename Mma<T>::Frag q[KS];
  const T *qrow = row_of<T>(p.q, sh.q_stride, b, t, h);
#pragma unroll
  for (int k = 0; k < KS; ++k) q[k] = load_frag(qrow, 16 * k + 8 * (lane >> 5), sh.D, at.direct, at.sign);

  const KeyTiles<T, DP, 32, 1> tiles(sh, p, b, hk, 0, lane);
  auto stage = [&](T *buf, int v0) { tiles.stage(buf + wave * 2 * kTile, at, keys, n, v0, sh.D, 0, lane); };
  Softmax<T, DP> soft;
  soft.clear();
  auto step = [&](const T *buf, int v0) {
    const T *mine = buf + wave * 2 * kTile;
    soft.add(mine, mine + kTile, q, v0, see, sh.sinks, at.scale2, true, lane);
  };
  auto arrived = [&]() { landed<0>(); };
  // tiles part * W + wave, then every (splits * W)-th
  const int stride = 32 * at.splits * W;
  int v0 = 32 * (part * W + wave);
  if (v0 < n) stage(buf0, v0);
  for (; v0 < n; v0 += 2 * stride) {
    arrived();
    if (v0 + stride < n) stage(buf1, v0 + stride);
    step(buf0, v0);
    if (v0 + stride >= n) break;
    arrived();
    if (v0 + 2 * stride < n) stage(buf0, v0 + 2 * stride);
    step(buf1, v0 + stride);
  }
  const float l = half_sum(soft.l);
  // each wave's sums in LDS, in the buffers that all have read
  __shared__ float ml[W][64];
  const WaveSums<T, DP, W> sums = {buf0, buf1};
  __syncthreads();
  sums.leave(wave, lane, soft.o);
  if (lane < 32) {
    ml[wave][lane] = soft.m;
    ml[wave][32 + lane] = l;
  }
  __syncthreads();
  for (int x = wave; x < 32 && r0 + x < rows; x += W) {
    const int tx = (r0 + x) / G, hx = hk * G + (r0 + x) % G;
    if (at.splits == 1) {
      const bool none = row_keys(sh, seq, keys, seq.start + tx).none;
      join_parts<T>(sh, p, b, hx, tx, none, W, [&](int w) { return ml[w][x]; },
                    [&](int w) { return ml[w][32 + x]; }, [&](int w, int d) { return sums.get(w, x, d); });
      continue;
    }
    // the workgroup's part: the waves joined, not divided yet
    float m = -INFINITY, sum = 0.0f;
    for (int w = 0; w < W; ++w) m = fmaxf(m, ml[w][x]);
    const float base = m == -INFINITY ? 0.0f : m;
    float *out = at.partial + (int64_t)blockIdx.x * part_floats<DP>();
    float f[W];
    for (int w = 0; w < W; ++w) {
      f[w] = exp2f(ml[w][x] - base);
      sum += f[w] * ml[w][32 + x];
    }
    for (int d = lane; d < DP; d += 64) {
      float o = 0.0f;
      for (int w = 0; w < W; ++w) o = fmaf(f[w], sums.get(w, x, d), o);
      out[64 + x * DP + d] = o;
    }
    if (lane == 0) {
      out[x] = m;
      out[32 + x] = sum;
    }
  }
}

// A wave per row joins the parts that workgroups left.
template <class T, int DP>
__global__ __launch_bounds__(64) void attend_join(const dconv_attend_shape sh, const AttendPtrs p,
                                                  const AttendTile at) {
  const int G = sh.Hq / sh.Hkv, rows = sh.Tq * G;
  const int r = blockIdx.x % rows, bh = blockIdx.x / rows, b = bh / sh.Hkv, hk = bh % sh.Hkv;
  const Seq seq = seq_of(sh, p, b);
  const Span see = span_of(sh, seq, seq.start + r / G);
  const float *base = at.partial + ((int64_t)bh * at.tiles + r / 32) * at.splits * part_floats<DP>();
  auto part = [&](int i) { return base + (int64_t)i * part_floats<DP>() + (r & 31); };
  join_parts<T>(sh, p, b, hk * G + r % G, r / G, see.hi - see.lo + see.first == 0, at.splits,
                [&](int i) { return part(i)[0]; }, [&](int i) { return part(i)[32]; },
                [&](int i, int d) { return part(i)[64 + (r & 31) * (DP - 1) + d]; });
}

// ---------------------------------------------------------------------------
// Launch
// ---------------------------------------------------------------------------
template <class F>
void by_width(int dp, F f) {
  if (dp == 32) return f(std::integral_constant<int, 32>());
  if (dp == 64) return f(std::integral_constant<int, 64>());
  if (dp == 96) return f(std::integral_constant<int, 96>());
  if (dp == 128) return f(std::integral_constant<int, 128>());
  return f(std::integral_constant<int, 256>());
}

inline AttendTile attend_tile(const dconv_attend_shape &sh, bool direct, bool near) {
  AttendTile at = {};
  at.scale2 = sh.scale == 0.0f ? 1.0f : fabsf(sh.scale) * 1.4426950408889634f;
  at.sign = sh.scale > 0.0f ? 1.0f : sh.scale < 0.0f ? -1.0f : 0.0f;
  at.direct = direct;
  at.near = near;
  return at;
}

template <class T>
void launch_attend(const dconv_attend_shape &sh, const AttendPtrs &p, const ForwardPlan &plan, float *workspace,
                   hipStream_t s) {
  AttendTile at = attend_tile(sh, plan.direct, plan.near);
  at.tiles = plan.tiles;
  at.splits = plan.splits;
  at.partial = workspace;
  by_width(plan.dp, [&](auto dp) {
    constexpr int DP = decltype(dp)::value;
    const unsigned groups = (unsigned)(sh.B * sh.Hkv * plan.tiles);
    if (!plan.few) {
      hipLaunchKernelGGL((attend_tiles<T, DP>), dim3(groups), dim3(256), 0, s, sh, p, at);
      return;
    }
    hipLaunchKernelGGL((attend_split<T, DP>), dim3(groups * plan.splits), dim3(64 * split_waves<T>(DP)), 0, s,
                       sh, p, at);
    if (plan.splits > 1)
      hipLaunchKernelGGL((attend_join<T, DP>), dim3((unsigned)((int64_t)sh.B * sh.Hq * sh.Tq)), dim3(64), 0, s,
                         sh, p, at);
  });
}

}  // namespace dconv

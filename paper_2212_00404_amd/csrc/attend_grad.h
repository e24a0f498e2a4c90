// The gradients of windowed attention on the matrix cores.  Probabilities are
// computed again from the scores and the forward call's sums; with
//   ds = p (dout . v - delta),  delta = dout . out
// the kernels below take four products per tile of scores each (attend_dq one of
// them for delta's rounding).  attend_dq walks the keys for each tile of rows as the forward kernel does, and
// leaves each row's sum and delta for the others; attend_dkv and attend_dkv_split
// walk the rows for each tile of keys.  Nothing is added by atomics: the order
// of every sum is fixed.
#pragma once

#include "attend_mma.h"

namespace dconv {

// A row's sum (in powers of two, less kLift) and its delta, as the workspace holds them.
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

struct GradTile {
  AttendTile a;
  f32x2 *stats;      // [B * Hkv][rows]
  int first;         // keys [0, first) belong to attend_dkv_split, the others to attend_dkv
  int parts;         // parts of the rows (attend_dkv_split)
};

// in_order() for head sizes whose operands fit the registers beside the sums.
template <class T, int DP>
constexpr bool kAhead = DP * sizeof(T) <= 128;
template <class T, int DP>
__device__ __forceinline__ void read_ahead() {
  if constexpr (kAhead<T, DP>) in_order();
}

template <class T>
__device__ __forceinline__ float frag_dot(typename Mma<T>::Frag a, typename Mma<T>::Frag b) {
  float s = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) s = fmaf(to_f32(a[e]), to_f32(b[e]), s);
  return s;
}

// Probabilities and their gradients are operands of the tensors' type.  fp16 has five
// bits of exponent only: a probability is below its normal values from 2^-14 on, a
// gradient, which is as small as dout over the number of keys, for ordinary losses,
// and past its largest value for scaled ones.  So fp16 holds 2^15 times the
// probabilities (they are 1 at most) and a power of two times their gradients, one
// for each column of a tile of scores, that is for each row of dq and each key of dk:
// it begins high enough for any fp16 inputs and falls when a value of the column
// reaches 2, to bring the largest to 1/4 .. 1/2; the sums so far are scaled with it.
// What is rounded below the normal values is then off by less than 2^-23 of the
// column's largest, and the scales lose nothing, as they are powers of two.  Below 2
// the first bit of the exponent is 0, so that one bit of each operand tells.  (It costs
// fp16 1 to 16%, in the branch's moves of sums between register files: 2 x 4096
// queries, 16 heads of 64 over 4, window 512: 132 -> 147 us.)
template <class T>
constexpr bool kScaled = std::is_same<T, f16_t>::value;
template <class T>
constexpr float kLift = kScaled<T> ? 15.0f : 0.0f;   // log2 of the probabilities' scale
constexpr float kUnlift = 0x1p-15f;

struct ColumnScale {
  float up = 0x1p60f;
  // x, scaled by up, as operands, after it has been brought into range.  sums(f):
  // what has been summed up so far, times f.
  template <class T, class F>
  __device__ __forceinline__ void fit(f32x16 &x, typename Mma<T>::Frag (&u)[2], F sums) {
    u[0] = as_operand<T>(x, 0);
    u[1] = as_operand<T>(x, 1);
    uint32_t bits[8], any = 0;
    __builtin_memcpy(bits, u, sizeof(bits));
#pragma unroll
    for (int i = 0; i < 8; ++i) any |= bits[i];
    if (__any((any & 0x40004000u) != 0)) {
      no_speculation();
      float top = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(x[i]));
      top = half_max(top);
      // 2^(-2 - e) for a top of 2^e .. 2^(e + 1), past fp16's largest too; an infinity
      // stays one
      const float f = top >= 1.0f ? __uint_as_float((252u - min(__float_as_uint(top) >> 23, 250u)) << 23) : 1.0f;
      x *= f;
      up *= f;
      sums(f);
      u[0] = as_operand<T>(x, 0);
      u[1] = as_operand<T>(x, 1);
    }
  }
  // What takes the scales out of the sums of the gradients.
  __device__ __forceinline__ float down() const { return kUnlift / up; }
};

// Stores four consecutive elements from column d on.
template <class T>
__device__ __forceinline__ void store4(T *row, int d, int D, bool whole, float a, float b, float c, float e) {
  T x[4] = {from_f32<T>(a), from_f32<T>(b), from_f32<T>(c), from_f32<T>(e)};
  if (whole && d + 4 <= D) {
    __builtin_memcpy(__builtin_assume_aligned(row + d, 4), x, sizeof(x));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (d + i < D) row[d + i] = x[i];
  }
}

// ---------------------------------------------------------------------------
// dq: 61 us for 2 x 4096 queries, 16 heads of 64, window 512, bf16; the matrix cores
// run 0.29 of the cycles and vector instructions issue in 0.47 of them
// ---------------------------------------------------------------------------
template <class T, int DP>
__global__ __launch_bounds__(256, DP * sizeof(T) <= 128 ? 2 : 1) void attend_dq(const dconv_attend_shape sh, const AttendPtrs p, const GradTile gt) {
  constexpr int BN = forward_keys<T>(DP), KS = DP / 16, DT = DP / 32;
  typedef typename Mma<T>::Frag Frag;
  __shared__ __align__(16) T buf0[2 * BN * DP];
  __shared__ __align__(16) T buf1[2 * BN * DP];
  DCONV_POISON(poison_lds(buf0, 2 * BN * DP); poison_lds(buf1, 2 * BN * DP));
  const AttendTile &at = gt.a;
  const int lane = threadIdx.x & 63, half = lane >> 5, wave = uniform(threadIdx.x >> 6);
  const int id = xcd_remap(blockIdx.x, gridDim.x);
  const int bh = id / at.tiles, b = bh / sh.Hkv, hk = bh % sh.Hkv, G = sh.Hq / sh.Hkv;
  const int r0 = (id % at.tiles) * kForwardRows, rows = sh.Tq * G;
  const Seq seq = seq_of(sh, p, b);
  const Keys keys = keys_of(sh, seq, r0 / G, (min(r0 + kForwardRows, rows) - 1) / G);
  const int n = uniform(keys.n);
  const int r = r0 + 32 * wave + (lane & 31), rr = min(r, rows - 1);
  const int t = rr / G, h = hk * G + rr % G;
  const RowKeys see = row_keys(sh, seq, keys, seq.start + t);
  int from = see.lo, to = see.hi, all_from = see.lo, all_to = see.hi;
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) {
    from = min(from, __shfl_xor(from, x));
    to = max(to, __shfl_xor(to, x));
    all_from = max(all_from, __shfl_xor(all_from, x));
    all_to = min(all_to, __shfl_xor(all_to, x));
  }
  from = uniform(from), to = uniform(to), all_from = uniform(all_from), all_to = uniform(all_to);

  const KeyTiles<T, DP, BN, 4> tiles(sh, p, b, hk, wave, lane);
  auto stage = [&](T *buf, int v0) { tiles.stage(buf, at, keys, n, v0, sh.D, wave, lane); };
  if (n > 0) stage(buf0, 0);

  Frag q[KS], g[KS];
  const T *qrow = row_of<T>(p.q, sh.q_stride, b, t, h), *grow = row_of<T>(p.dout, sh.dout_stride, b, t, h);
  const T *orow = row_of<T>(p.out, sh.out_stride, b, t, h);
  float delta = 0.0f;
#pragma unroll
  for (int k = 0; k < KS; ++k) {
    const int d = 16 * k + 8 * half;
    q[k] = load_frag(qrow, d, sh.D, at.direct, at.sign);
    g[k] = load_frag(grow, d, sh.D, at.direct, 1.0f);
    delta += frag_dot<T>(g[k], load_frag(orow, d, sh.D, at.direct, 1.0f));
  }
  delta = half_sum(delta);
  const float lse2 =
      (see.none ? 0.0f : 1.4426950408889634f * p.lse[((int64_t)b * sh.Hq + h) * sh.Tq + t]) - kLift<T>;
  ColumnScale scale;

  // out, rounded to the tensors' type, gives delta to within that rounding of
  // |dout| |out|.  Where a row's weight is on a few keys, dp - delta cancels and
  // that error is much of what is left.  The sum of p (dp - delta) over the keys
  // is how far off it is: it corrects delta for the other kernels and, times the
  // mean key (sum of p k: a fourth product, on operands already loaded), dq.
  f32x16 acc[DT], mean[DT];
  float miss = 0.0f;
#pragma unroll
  for (int c = 0; c < DT; ++c) acc[c] = mean[c] = f32x16{};
  auto columns = [&](Frag(&f)[DT], const T *t, int row) {
#pragma unroll
    for (int c = 0; c < DT; ++c) f[c] = Tile<T, DP>::column(t, row, c, lane);
  };
  // keys v .. v + 31 by the wave's rows: none seen, all seen
  auto unseen = [&](int v) { return v >= to || (v + 32 <= from && v >= sh.sinks); };
  auto all_seen = [&](int v) { return v + 32 <= all_to && (v >= all_from || v + 32 <= sh.sinks); };
  auto step = [&](const T *buf, int v0) {
    const T *ks = buf, *vs = buf + BN * DP;
#pragma unroll
    for (int hb = 0; hb < BN / 32; ++hb) {
      if (unseen(v0 + 32 * hb)) continue;
      const bool masked = !all_seen(v0 + 32 * hb);
      Frag a[KS], x[KS], col[2][DT];
#pragma unroll
      for (int k = 0; k < KS; ++k) a[k] = Tile<T, DP>::row(ks, 32 * hb, k, lane);
#pragma unroll
      for (int k = 0; k < KS; ++k) x[k] = Tile<T, DP>::row(vs, 32 * hb, k, lane);
      read_ahead<T, DP>();
      f32x16 s = {}, dp = {};
#pragma unroll
      for (int k = 0; k < KS; ++k) s = Mma<T>::mac(a[k], q[k], s);
      if constexpr (kAhead<T, DP>) columns(col[0], ks, 32 * hb);
      read_ahead<T, DP>();
#pragma unroll
      for (int k = 0; k < KS; ++k) dp = Mma<T>::mac(x[k], g[k], dp);
      if constexpr (kAhead<T, DP>) columns(col[1], ks, 32 * hb + 16);
      read_ahead<T, DP>();
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[i] = power2<T>(fmaf(s[i], at.scale2, -lse2));
        dp[i] = s[i] * (kScaled<T> ? fmaf(dp[i], scale.up, -delta * scale.up) : dp[i] - delta);
      }
      if (masked) {
        no_speculation();
        seen_keys(v0 + 32 * hb, see, sh.sinks, lane, [&](int i, bool on) {
          s[i] = on ? s[i] : 0.0f;
          dp[i] = on ? dp[i] : 0.0f;
        });
      }
      // (before the branch in fit(), which nothing is moved across)
      if constexpr (kScaled<T> && !kAhead<T, DP>) columns(col[0], ks, 32 * hb);
      const Frag w[2] = {as_operand<T>(s, 0), as_operand<T>(s, 1)};
      Frag u[2];
      if constexpr (kScaled<T>) {
        scale.fit<T>(dp, u, [&](float f) {
#pragma unroll
          for (int c = 0; c < DT; ++c) acc[c] *= f;
          miss *= f;
        });
      } else {
        u[0] = as_operand<T>(dp, 0);
        u[1] = as_operand<T>(dp, 1);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) miss += dp[i];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if constexpr (!kAhead<T, DP>)
          if (!kScaled<T> || k > 0) columns(col[k], ks, 32 * hb + 16 * k);
#pragma unroll
        for (int c = 0; c < DT; ++c) {
          acc[c] = Mma<T>::mac(col[k][c], u[k], acc[c]);
          mean[c] = Mma<T>::mac(col[k][c], w[k], mean[c]);
        }
      }
    }
  };
  auto arrived = [&]() {
    landed<0>();
    __syncthreads();
  };
  for (int v0 = 0; v0 < n; v0 += 2 * BN) {
    arrived();
    if (v0 + BN < n) stage(buf1, v0 + BN);
    step(buf0, v0);
    if (v0 + BN >= n) break;
    arrived();
    if (v0 + 2 * BN < n) stage(buf0, v0 + 2 * BN);
    step(buf1, v0 + BN);
  }

  miss = half_sum(miss);
  if constexpr (kScaled<T>) {
    miss *= scale.down();
#pragma unroll
    for (int c = 0; c < DT; ++c) {
      acc[c] *= scale.down();
      mean[c] *= kUnlift;
    }
  }
  if (half == 0 && r < rows) gt.stats[(int64_t)bh * rows + r] = f32x2{lse2, delta + miss};
  bool bad = false;
#pragma unroll
  for (int c = 0; c < DT; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      acc[c][i] = sh.scale * fmaf(-miss, mean[c][i], acc[c][i]);
      bad |= 32 * c + acc_row(i, half) < sh.D && !(fabsf(acc[c][i]) < INFINITY);
    }
  const unsigned long long any = __ballot(bad && r < rows);
  const unsigned redo = kSumAgain ? (unsigned)(any | (any >> 32)) : 0u;
  if (r < rows && !(redo >> (lane & 31) & 1)) {
    T *o = (T *)p.dq + (((int64_t)b * sh.Tq + t) * sh.Hq + h) * sh.D;
#pragma unroll
    for (int c = 0; c < DT; ++c)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        store4(o, 32 * c + acc_row(i, half), sh.D, at.direct, acc[c][i], acc[c][i + 1], acc[c][i + 2],
               acc[c][i + 3]);
  }
  for (unsigned again = redo; again; again &= again - 1) {
    const int x = r0 + 32 * wave + __ffs(again) - 1;
    attend_row_dq<T>(sh, p, b, hk * G + x % G, x / G);
  }
}

// ---------------------------------------------------------------------------
// dk, dv
// ---------------------------------------------------------------------------
// 32 keys of one wave, a key per column (lane % 32).
template <class T, int DP>
struct KeyGrad {
  static constexpr int KS = DP / 16, DT = DP / 32;
  typedef typename Mma<T>::Frag Frag;
  Frag k[KS], v[KS];
  f32x16 dk[DT], dv[DT];   // dk[c][i]: element 32 c + acc_row(i, half) of the key
  ColumnScale scale;

  __device__ __forceinline__ void load(const dconv_attend_shape &sh, const AttendTile &at, const T *krow,
                                       const T *vrow, int half) {
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      k[s] = load_frag(krow, 16 * s + 8 * half, sh.D, at.direct, at.sign);
      v[s] = load_frag(vrow, 16 * s + 8 * half, sh.D, at.direct, 1.0f);
    }
#pragma unroll
    for (int c = 0; c < DT; ++c) dk[c] = dv[c] = f32x16{};
  }

  // 32 rows r .. of the tiles qs (queries) and gs (dout), their statistics in st;
  // the key is seen by rows [lo, hi).
  __device__ __forceinline__ void add(const T *qs, const T *gs, const f32x2 *st, int r, int lo, int hi, bool masked,
                                      float scale2, int lane) {
    const int half = lane >> 5;
    // operands are read well before their products: LDS answers after some
    // hundred clocks, and two waves per SIMD do not cover that for one another
    Frag a[KS], b[KS], cg[2][DT], cq[2][DT];
#pragma unroll
    for (int x = 0; x < KS; ++x) a[x] = Tile<T, DP>::row(qs, 0, x, lane);
#pragma unroll
    for (int x = 0; x < KS; ++x) b[x] = Tile<T, DP>::row(gs, 0, x, lane);
    read_ahead<T, DP>();
    f32x16 s = {}, dp = {};
#pragma unroll
    for (int x = 0; x < KS; ++x) s = Mma<T>::mac(a[x], k[x], s);
    // (base, delta) of the rows 8 i + 4 half .. + 3
    f32x4 st4[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      st4[2 * i] = *reinterpret_cast<const f32x4 *>(st + 8 * i + 4 * half);
      st4[2 * i + 1] = *reinterpret_cast<const f32x4 *>(st + 8 * i + 4 * half + 2);
    }
    read_ahead<T, DP>();
#pragma unroll
    for (int x = 0; x < KS; ++x) dp = Mma<T>::mac(b[x], v[x], dp);
    if constexpr (kAhead<T, DP>) columns(cg[0], cq[0], gs, qs, 0, lane);
    read_ahead<T, DP>();
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const f32x4 x = st4[i / 4 * 2 + i % 4 / 2];
      s[i] = power2<T>(fmaf(s[i], scale2, -x[i % 2 * 2]));
      dp[i] = (kScaled<T> ? s[i] * scale.up : s[i]) * (dp[i] - x[i % 2 * 2 + 1]);
    }
    if (masked) {
      no_speculation();
      within(lo - r, hi - r, half, [&](int i, bool on) {
        s[i] = on ? s[i] : 0.0f;
        dp[i] = on ? dp[i] : 0.0f;
      });
    }
    if constexpr (kScaled<T> && !kAhead<T, DP>) columns(cg[0], cq[0], gs, qs, 0, lane);
    const Frag w[2] = {as_operand<T>(s, 0), as_operand<T>(s, 1)};
    Frag u[2];
    if constexpr (kScaled<T>) {
      scale.fit<T>(dp, u, [&](float f) {
#pragma unroll
        for (int c = 0; c < DT; ++c) dk[c] *= f;
      });
    } else {
      u[0] = as_operand<T>(dp, 0);
      u[1] = as_operand<T>(dp, 1);
    }
    if constexpr (kAhead<T, DP>) columns(cg[1], cq[1], gs, qs, 16, lane);
    read_ahead<T, DP>();
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      if constexpr (!kAhead<T, DP>)
        if (!kScaled<T> || x > 0) columns(cg[x], cq[x], gs, qs, 16 * x, lane);
#pragma unroll
      for (int c = 0; c < DT; ++c) {
        dv[c] = Mma<T>::mac(cg[x][c], w[x], dv[c]);
        dk[c] = Mma<T>::mac(cq[x][c], u[x], dk[c]);
      }
    }
  }
  // After the last rows: the sums without their scales.
  __device__ __forceinline__ void finish() {
    if constexpr (kScaled<T>) {
#pragma unroll
      for (int c = 0; c < DT; ++c) {
        dk[c] *= scale.down();
        dv[c] *= kUnlift;
      }
    }
  }
  static __device__ __forceinline__ void columns(Frag (&cg)[DT], Frag (&cq)[DT], const T *gs, const T *qs, int r,
                                                 int lane) {
#pragma unroll
    for (int c = 0; c < DT; ++c) {
      cg[c] = Tile<T, DP>::column(gs, r, c, lane);
      cq[c] = Tile<T, DP>::column(qs, r, c, lane);
    }
  }
};

// Rows [lo, hi) that see key j (of those this kernel counts).
struct KeyRows {
  int lo, hi;
};
__device__ __forceinline__ KeyRows key_rows(const dconv_attend_shape &sh, const Seq &s, int j, int from, int end) {
  KeyRows r = {0, 0};
  if (j < from || j >= min(end, s.len)) return r;
  const QuerySpan q = queries_of(sh, s, j);
  const int G = sh.Hq / sh.Hkv;
  r.lo = q.lo * G;
  r.hi = q.hi * G;
  return r;
}

// The rows of a wave's 32 keys: all of them, and those that see every key.
struct TileRows {
  int from, to, all_from, all_to;
};
__device__ __forceinline__ TileRows tile_rows(const KeyRows &k) {
  TileRows t = {k.lo < k.hi ? k.lo : 0x7fffffff, k.hi, k.lo, k.hi};
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) {
    t.from = min(t.from, __shfl_xor(t.from, x));
    t.to = max(t.to, __shfl_xor(t.to, x));
    t.all_from = max(t.all_from, __shfl_xor(t.all_from, x));
    t.all_to = min(t.all_to, __shfl_xor(t.all_to, x));
  }
  t.from = uniform(t.from), t.to = uniform(t.to), t.all_from = uniform(t.all_from), t.all_to = uniform(t.all_to);
  return t;
}

// The statistics of 32 rows r .. into LDS, by one wave (past `to` the last row's).
__device__ __forceinline__ void stage_stats(f32x2 *lds, const f32x2 *stats, int r, int to, int lane) {
  const float *from = reinterpret_cast<const float *>(stats + min(r + (lane >> 1), to - 1)) + (lane & 1);
  __builtin_amdgcn_global_load_lds(from, (lds_ptr)lds, 4, 0, 0);
}

// Tiles of NR rows of queries and dout, in this order, and the rows' statistics.
template <class T, int DP, int NR, int NW>
struct RowTiles {
  typedef Copy<T, DP, NR, NW> C;
  C cq, cg;
  const T *q, *g;
  const f32x2 *stats;
  int G;
  bool near, alike;   // alike: every tile's rows lie as the first one's do

  __device__ __forceinline__ RowTiles(const dconv_attend_shape &sh, const AttendPtrs &p, const GradTile &gt, int b,
                                      int hk, int wave, int lane)
      : q(row_of<T>(p.q, sh.q_stride, b, 0, (int64_t)hk * (sh.Hq / sh.Hkv))),
        g(row_of<T>(p.dout, sh.dout_stride, b, 0, (int64_t)hk * (sh.Hq / sh.Hkv))),
        stats(gt.stats + ((int64_t)b * sh.Hkv + hk) * sh.Tq * (sh.Hq / sh.Hkv)), G(sh.Hq / sh.Hkv) {
    near = gt.a.near && G <= 128;
    // walks begin with the first head of a group
    alike = near && NR % G == 0 && (C::kStep ? C::kStep : NR) % G == 0;
    if (alike) {
      cq.init(sh.D, wave, lane, [&](int r) { return offset(r, 0, sh.q_stride); });
      cg.init(sh.D, wave, lane, [&](int r) { return offset(r, 0, sh.dout_stride); });
    }
  }
  // Of row r of a tile that begins with head g0 of a group, in bytes.  (The
  // quotient by a product: exact while (r + g0) G < 2^16.)
  __device__ __forceinline__ uint32_t offset(int r, int g0, const long long *stride) const {
    const uint32_t v = r + g0, t = v * (65536u / G + 1) >> 16;
    return (t * (uint32_t)stride[1] + (v - t * G) * (uint32_t)stride[2]) * (uint32_t)sizeof(T);
  }
  // Rows r ..; past `to` the last one.
  __device__ __forceinline__ void stage(T *lds, f32x2 *st, const dconv_attend_shape &sh, bool direct, int r, int to,
                                        int wave, int lane) const {
    if (wave < NR / 32) stage_stats(st + 32 * wave, stats, r + 32 * wave, to, lane);
    if (near && r + NR <= to) {
      const int t = r / G, g0 = r - t * G;
      const T *qt = q + t * sh.q_stride[1], *dt = g + t * sh.dout_stride[1];
      if (alike) {
        cq.tile(lds, qt, C::kStep / G * sh.q_stride[1] * (int64_t)sizeof(T), wave);
        cg.tile(lds + NR * DP, dt, C::kStep / G * sh.dout_stride[1] * (int64_t)sizeof(T), wave);
      } else {
        C::tile_at(lds, qt, sh.D, wave, lane, [&](int x) { return offset(x, g0, sh.q_stride); });
        C::tile_at(lds + NR * DP, dt, sh.D, wave, lane, [&](int x) { return offset(x, g0, sh.dout_stride); });
      }
      return;
    }
    auto from = [&](const T *base, const long long *stride) {
      const int64_t by_t = stride[1], by_h = stride[2];
      return [=](int x) {
        const int y = min(r + x, to - 1);
        return base + y / G * by_t + y % G * by_h;
      };
    };
    if (direct) {
      C::rows(lds, sh.D, wave, lane, from(q, sh.q_stride));
      C::rows(lds + NR * DP, sh.D, wave, lane, from(g, sh.dout_stride));
    } else {
      C::elements(lds, sh.D, wave, lane, from(q, sh.q_stride));
      C::elements(lds + NR * DP, sh.D, wave, lane, from(g, sh.dout_stride));
    }
  }
};


// 32 keys per wave and KG key groups of them per workgroup; its waves form RG row
// groups, which take R tiles of 32 rows of queries and dout each per step and are
// added at the end.  Eight waves, so that a workgroup alone on its compute unit has
// two waves per SIMD to fill each other's waits; larger heads leave registers for
// four.  Two tiles per step where LDS has room, as one tile's products are too short
// for the next one's copies.  (2 x 4096 keys, four key heads of 64, window 512, 256
// workgroups, bf16: 92 us with four waves, 75 with eight, 71 with operands read
// ahead, 67 with two tiles per step: the matrix cores run 0.26 of the cycles, the
// waves wait 0.43 of theirs, mostly for LDS and for copies.)  KG = 4 reads the rows
// least often; KG = 2 and 1 make twice and four times the workgroups.
template <class T>
constexpr int row_groups(int dp, int key_groups) {
  const int bytes = dp * (int)sizeof(T);
  if (key_groups == 1) return bytes <= 128 ? 8 : 4;   // (what two LDS buffers hold)
  return (bytes <= 128 ? 8 : 4) / key_groups;
}

template <class T, int DP, int KG, int RG>
__global__ __launch_bounds__(64 * KG * RG) void attend_dkv(const dconv_attend_shape sh, const AttendPtrs p,
                                                           const GradTile gt) {
  constexpr int W = KG * RG, DT = DP / 32;
  constexpr int R = 32 * RG * DP * (int)sizeof(T) <= 8192 ? 2 : 1, BM = 32 * RG * R;
  constexpr int kMerge = KG * (RG - 1) * 1024 * 4 / (int)sizeof(T);   // sums of one 32-column part
  constexpr int kBuf = 2 * BM * DP > kMerge ? 2 * BM * DP : kMerge;
  __shared__ __align__(16) T buf0[kBuf];
  __shared__ __align__(16) T buf1[kBuf];
  __shared__ __align__(16) f32x2 stats0[BM];
  __shared__ __align__(16) f32x2 stats1[BM];
  __shared__ int span[2][KG];
  DCONV_POISON(poison_lds(buf0, kBuf); poison_lds(buf1, kBuf); poison_lds(stats0, BM); poison_lds(stats1, BM));
  const AttendTile &at = gt.a;
  const int lane = threadIdx.x & 63, half = lane >> 5, wave = uniform(threadIdx.x >> 6);
  const int kg = wave % KG, rg = wave / KG;   // key group, row group
  const int id = xcd_remap(blockIdx.x, gridDim.x);
  const int bh = id / at.tiles, b = bh / sh.Hkv, hk = bh % sh.Hkv;
  const int j = (id % at.tiles) * (32 * KG) + 32 * kg + (lane & 31), jj = min(j, sh.Tk - 1);
  const Seq seq = seq_of(sh, p, b);
  const KeyRows see = key_rows(sh, seq, j, gt.first, sh.Tk);
  const TileRows mine = tile_rows(see);
  if (lane == 0 && rg == 0) {
    span[0][kg] = mine.from;
    span[1][kg] = mine.to;
  }
  __syncthreads();
  int from = span[0][0], to = span[1][0];
#pragma unroll
  for (int x = 1; x < KG; ++x) {
    from = min(from, span[0][x]);
    to = max(to, span[1][x]);
  }
  from = uniform(from), to = uniform(to);

  const RowTiles<T, DP, BM, W> tiles(sh, p, gt, b, hk, wave, lane);
  auto stage = [&](T *buf, f32x2 *st, int r) { tiles.stage(buf, st, sh, at.direct, r, to, wave, lane); };
  if (from < to) stage(buf0, stats0, from);
  KeyGrad<T, DP> acc;
  acc.load(sh, at, row_of<T>(p.k, sh.k_stride, b, jj, hk), row_of<T>(p.v, sh.v_stride, b, jj, hk), half);
  auto step = [&](const T *buf, const f32x2 *st, int r) {
#pragma unroll
    for (int x = 0; x < R; ++x) {
      const int row = 32 * (rg * R + x);
      if (r + row >= mine.to || r + row + 32 <= mine.from) continue;
      acc.add(buf + row * DP, buf + (BM + row) * DP, st + row, r + row, see.lo, see.hi,
              !(r + row >= mine.all_from && r + row + 32 <= mine.all_to), at.scale2, lane);
    }
  };
  auto arrived = [&]() {
    landed<0>();
    __syncthreads();
  };
  for (int r = from; r < to; r += 2 * BM) {
    arrived();
    if (r + BM < to) stage(buf1, stats1, r + BM);
    step(buf0, stats0, r);
    if (r + BM >= to) break;
    arrived();
    if (r + 2 * BM < to) stage(buf0, stats0, r + 2 * BM);
    step(buf1, stats1, r + BM);
  }
  acc.finish();
  if constexpr (RG > 1) {
#pragma unroll
    for (int c = 0; c < DT; ++c) {
      __syncthreads();   // every wave is done with what the buffers hold
      if (rg > 0) {
        const int x = ((rg - 1) * KG + kg) * 1024 + lane;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          reinterpret_cast<float *>(buf0)[x + 64 * i] = acc.dk[c][i];
          reinterpret_cast<float *>(buf1)[x + 64 * i] = acc.dv[c][i];
        }
      }
      __syncthreads();
      if (rg == 0) {
#pragma unroll
        for (int g = 0; g < RG - 1; ++g) {
          const int x = (g * KG + kg) * 1024 + lane;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            acc.dk[c][i] += reinterpret_cast<const float *>(buf0)[x + 64 * i];
            acc.dv[c][i] += reinterpret_cast<const float *>(buf1)[x + 64 * i];
          }
        }
      }
    }
    if (rg > 0) return;
  }

  bool bad = false;
#pragma unroll
  for (int c = 0; c < DT; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      acc.dk[c][i] *= sh.scale;
      bad |= 32 * c + acc_row(i, half) < sh.D &&
             !(fabsf(acc.dk[c][i]) < INFINITY && fabsf(acc.dv[c][i]) < INFINITY);
    }
  const bool own = j >= gt.first && j < sh.Tk;
  const unsigned long long any = __ballot(bad && own);
  const unsigned redo = kSumAgain ? (unsigned)(any | (any >> 32)) : 0u;
  if (own && !(redo >> (lane & 31) & 1)) {
    const int64_t o = (((int64_t)b * sh.Tk + j) * sh.Hkv + hk) * sh.D;
#pragma unroll
    for (int c = 0; c < DT; ++c)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int d = 32 * c + acc_row(i, half);
        store4((T *)p.dk + o, d, sh.D, at.direct, acc.dk[c][i], acc.dk[c][i + 1], acc.dk[c][i + 2], acc.dk[c][i + 3]);
        store4((T *)p.dv + o, d, sh.D, at.direct, acc.dv[c][i], acc.dv[c][i + 1], acc.dv[c][i + 2], acc.dv[c][i + 3]);
      }
  }
  for (unsigned again = redo; again; again &= again - 1)
    attend_row_dkv<T>(sh, p, b, hk, (id % at.tiles) * (32 * KG) + 32 * kg + __ffs(again) - 1);
}

// Keys [0, gt.first) in tiles of 32: the first keys, which every row sees.  The rows are divided over the waves, each with two LDS
// buffers of its own, and over gt.parts workgroups, which leave their sums in the
// workspace.  (14.6 us for four first keys and 16384 rows per key head: four tiles of
// rows per wave, each a wait for its copies.)
template <class T, int DP>
__global__ __launch_bounds__(64 * split_waves<T>(DP)) void attend_dkv_split(const dconv_attend_shape sh,
                                                                                 const AttendPtrs p,
                                                                                 const GradTile gt) {
  constexpr int kTile = 32 * DP, W = split_waves<T>(DP);
  __shared__ __align__(16) T buf0[W * 2 * kTile];
  __shared__ __align__(16) T buf1[W * 2 * kTile];
  __shared__ __align__(16) f32x2 stats0[W * 32];
  __shared__ __align__(16) f32x2 stats1[W * 32];
  DCONV_POISON(poison_lds(buf0, W * 2 * kTile); poison_lds(buf1, W * 2 * kTile); poison_lds(stats0, W * 32);
               poison_lds(stats1, W * 32));
  const AttendTile &at = gt.a;
  const int lane = threadIdx.x & 63, half = lane >> 5, wave = uniform(threadIdx.x >> 6);
  const int part = blockIdx.x % gt.parts, id = blockIdx.x / gt.parts;
  const int bh = id / at.tiles, b = bh / sh.Hkv, hk = bh % sh.Hkv;
  const int j0 = (id % at.tiles) * 32, j = j0 + (lane & 31), jj = min(j, sh.Tk - 1);
  const Seq seq = seq_of(sh, p, b);
  const KeyRows see = key_rows(sh, seq, j, 0, gt.first);
  const TileRows mine = tile_rows(see);

  const RowTiles<T, DP, 32, 1> tiles(sh, p, gt, b, hk, 0, lane);
  auto stage = [&](T *buf, f32x2 *st, int r) {
    tiles.stage(buf + wave * 2 * kTile, st + wave * 32, sh, at.direct, r, mine.to, 0, lane);
  };
  KeyGrad<T, DP> acc;
  acc.load(sh, at, row_of<T>(p.k, sh.k_stride, b, jj, hk), row_of<T>(p.v, sh.v_stride, b, jj, hk), half);
  auto step = [&](const T *buf, const f32x2 *st, int r) {
    const T *from = buf + wave * 2 * kTile;
    acc.add(from, from + kTile, st + wave * 32, r, see.lo, see.hi, true, at.scale2, lane);
  };
  auto arrived = [&]() { landed<0>(); };
  const int stride = 32 * gt.parts * W;
  if (mine.from < mine.to) {
    int r = mine.from + 32 * (part * W + wave);
    if (r < mine.to) stage(buf0, stats0, r);
    for (; r < mine.to; r += 2 * stride) {
      arrived();
      if (r + stride < mine.to) stage(buf1, stats1, r + stride);
      step(buf0, stats0, r);
      if (r + stride >= mine.to) break;
      arrived();
      if (r + 2 * stride < mine.to) stage(buf0, stats0, r + 2 * stride);
      step(buf1, stats1, r + stride);
    }
  }
  acc.finish();
  // the waves' sums in LDS: first dk, then dv
  const WaveSums<T, DP, W> sums = {buf0, buf1};
  for (int which = 0; which < 2; ++which) {
    __syncthreads();
    sums.leave(wave, lane, which ? acc.dv : acc.dk);
    __syncthreads();
    float *out = at.partial + ((int64_t)blockIdx.x * 2 + which) * kTile;
    for (int x = threadIdx.x; x < kTile; x += 64 * W) {
      float s = 0.0f;
#pragma unroll
      for (int w = 0; w < W; ++w) s += sums.get(w, x / DP, x % DP);
      out[x] = s;
    }
  }
}

// Four waves per key add the parts, each every fourth, then the waves in order.
template <class T, int DP>
__global__ __launch_bounds__(256) void attend_dkv_join(const dconv_attend_shape sh, const AttendPtrs p,
                                                       const GradTile gt) {
  __shared__ float sum[4][2][DP];
  DCONV_POISON(poison_lds(&sum[0][0][0], 8 * DP));
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, j = blockIdx.x % gt.first, bh = blockIdx.x / gt.first;
  const int b = bh / sh.Hkv, hk = bh % sh.Hkv;
  const float *part = gt.a.partial + ((int64_t)bh * gt.a.tiles + j / 32) * gt.parts * 64 * DP + j % 32 * DP;
#pragma unroll
  for (int d = lane; d < DP; d += 64) {
    float k = 0.0f, v = 0.0f;
#pragma unroll 8
    for (int x = wave; x < gt.parts; x += 4) {
      k += part[(int64_t)x * 64 * DP + d];
      v += part[(int64_t)x * 64 * DP + 32 * DP + d];
    }
    sum[wave][0][d] = k;
    sum[wave][1][d] = v;
  }
  __syncthreads();
  if (wave > 0) return;
  float dk[(DP + 63) / 64], dv[(DP + 63) / 64];
  bool bad = false;
#pragma unroll
  for (int i = 0; i < (DP + 63) / 64; ++i) {
    const int d = lane + 64 * i;
    if (d >= sh.D) continue;
    dk[i] = sh.scale * ((sum[0][0][d] + sum[1][0][d]) + (sum[2][0][d] + sum[3][0][d]));
    dv[i] = (sum[0][1][d] + sum[1][1][d]) + (sum[2][1][d] + sum[3][1][d]);
    bad |= !(fabsf(dk[i]) < INFINITY && fabsf(dv[i]) < INFINITY);
  }
  if (kSumAgain && __any(bad)) {
    attend_row_dkv<T>(sh, p, b, hk, j);
    return;
  }
  const int64_t o = (((int64_t)b * sh.Tk + j) * sh.Hkv + hk) * sh.D;
#pragma unroll
  for (int i = 0; i < (DP + 63) / 64; ++i)
    if (lane + 64 * i < sh.D) {
      ((T *)p.dk)[o + lane + 64 * i] = from_f32<T>(dk[i]);
      ((T *)p.dv)[o + lane + 64 * i] = from_f32<T>(dv[i]);
    }
}

template <class T>
void launch_attend_grad(const dconv_attend_shape &sh, const AttendPtrs &p, const BackwardPlan &plan, void *workspace,
                        hipStream_t s) {
  GradTile gt = {};
  gt.a = attend_tile(sh, plan.direct, plan.near);
  gt.stats = (f32x2 *)workspace;
  gt.a.partial = (float *)((char *)workspace + plan.stats_bytes);
  gt.first = plan.first;
  gt.parts = plan.parts;
  auto launch = [&](auto dp) {
    constexpr int DP = decltype(dp)::value;
    const unsigned heads = (unsigned)(sh.B * sh.Hkv);
    if (plan.row_tiles > 0) {
      gt.a.tiles = plan.row_tiles;
      hipLaunchKernelGGL((attend_dq<T, DP>), dim3(heads * plan.row_tiles), dim3(256), 0, s, sh, p, gt);
    }
    if (plan.first < sh.Tk) {
      gt.a.tiles = plan.key_tiles;
      auto dkv = [&](auto groups) {
        constexpr int KG = decltype(groups)::value, RG = row_groups<T>(DP, KG);
        hipLaunchKernelGGL((attend_dkv<T, DP, KG, RG>), dim3(heads * plan.key_tiles), dim3(64 * KG * RG), 0, s, sh, p,
                           gt);
      };
      if (plan.key_groups == 4) dkv(std::integral_constant<int, 4>());
      if (plan.key_groups == 2) dkv(std::integral_constant<int, 2>());
      if constexpr (DP * sizeof(T) <= 256)
        if (plan.key_groups == 1) dkv(std::integral_constant<int, 1>());
    }
    if (plan.first > 0) {
      gt.a.tiles = plan.first_tiles;
      hipLaunchKernelGGL((attend_dkv_split<T, DP>), dim3(heads * plan.first_tiles * plan.parts),
                         dim3(64 * split_waves<T>(DP)), 0, s, sh, p, gt);
      hipLaunchKernelGGL((attend_dkv_join<T, DP>), dim3(heads * plan.first), dim3(256), 0, s, sh, p, gt);
    }
  };
  if (plan.dp == 32) launch(std::integral_constant<int, 32>());
  if (plan.dp == 64) launch(std::integral_constant<int, 64>());
  if (plan.dp == 96) launch(std::integral_constant<int, 96>());
  if (plan.dp == 128) launch(std::integral_constant<int, 128>());
}

}  // namespace dconv

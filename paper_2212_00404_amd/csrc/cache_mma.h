// Attention over a cache in pages on the matrix cores: the products and the
// running softmax of attend_mma.h over tiles of keys whose places a table gives.
// Instantiated per type and format in cache_attend_*.hip.
#pragma once

#include "attend_mma.h"
#include "cache_attend.h"

namespace dconv {

// What the host hands to the kernels beside the shape.
struct CacheTile {
  float scale2, sign;   // as in AttendTile
  bool direct;          // queries and results in 16-byte pieces
  bool pieces, near;    // rows of a plain cache too (codes: on 4-byte boundaries); a tile's slots span less than 2^31 bytes
  int groups, least;    // workgroups, the least work of one
  int whole;            // tiles per sequence and key head, one for each workgroup; 0: by work
  float *partial;       // two parts of each workgroup's
  CacheJoin *joins;     // and two joins
};

// A kernel's one argument.  What it holds is read from the argument's own memory
// where it is used (fresh), as a hundred scalars that stay in registers through the
// loops over segments would push out those of the loops over keys.
struct CacheCall {
  dconv_cache c;
  dconv_cache_attend_shape sh;
  Batch t;
  CacheAttendPtrs p;
  CacheTile few, tiles;
  template <bool FEW>
  __device__ __forceinline__ const CacheTile &tile() const {
    return FEW ? few : tiles;
  }
};
__device__ __forceinline__ const CacheCall &fresh() {
  typedef const __attribute__((address_space(4))) CacheCall *Arg;
  Arg a = (Arg)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(a));
  return *(const CacheCall *)a;
}

// ---------------------------------------------------------------------------
// The keys of a tile of rows
// ---------------------------------------------------------------------------
// Keys [0, first) and [lo, hi), as tiles of BN that begin on multiples of BN: so a
// tile lies within a page, or consists of whole pages, for every page size that is a
// power of two.
template <int BN>
struct KeyRange {
  int first, lo, hi;
  int front, from, n;   // tiles of the first keys, first tile of the others, tiles
  __device__ __forceinline__ KeyRange(const dconv_cache_attend_shape &sh, int len, int i0, int i1) {
    first = lo = hi = front = from = n = 0;
    if (i1 < 0) return;
    const KeySpan a = keys_seen(sh, len, max(i0, 0)), b = keys_seen(sh, len, i1);
    first = uniform(a.first);
    lo = uniform(a.lo);
    hi = uniform(b.hi);
    front = (first + BN - 1) / BN;
    from = max(front, lo / BN);
    n = front + max(hi > lo ? (hi + BN - 1) / BN - from : 0, 0);
  }
  __device__ __forceinline__ int start(int u) const { return (u < front ? u : u - front + from) * BN; }
  // Key j of the tile from j0 on, or where no row sees it one of the tile that is seen.
  __device__ __forceinline__ int key(int j0, int j) const {
    if (j < first) return j;
    if (j < lo) return lo < j0 + BN ? lo : first - 1;
    return min(j, hi - 1);
  }
  __device__ __forceinline__ bool whole(int j0) const { return (j0 >= lo && j0 + BN <= hi) || j0 + BN <= first; }
};

// Where the keys of a tile are, asked for a tile ahead, as the table's entry comes
// from memory.  ONE: a tile lies within a page, and is found by scalar arithmetic: the
// place of its first key.  Else key l of it in lane l (and l + 32 for 32 keys): the
// places are handed to the lanes that load by exchanges, 75 vector instructions for a
// wave and tile of 64 keys beside some 300 of its arithmetic.
struct Asked {
  int page, slot;
};
struct Found {
  int64_t k, v, ks, vs;   // bytes from the head's base
  uint64_t gone;          // keys without a page, whose places are the first page's
};
template <class T, int FORMAT, int BN, bool ONE>
struct Finder {
  static constexpr int64_t kBytes = FORMAT == DCONV_CACHE_PLAIN ? sizeof(T) : 1;
  const int *table;
  FastDiv page;
  int pages;
  __device__ __forceinline__ Asked ask(const KeyRange<BN> &keys, int j0) const {
    const uint32_t j = (uint32_t)(ONE ? j0 : keys.key(j0, j0 + (int)(threadIdx.x & (BN - 1))));
    const uint32_t at = page.div(j);
    return {table[at], (int)(j - at * page.d)};
  }
  __device__ __forceinline__ Found find(const dconv_cache &c, const Asked &a) const {
    const int entry = ONE ? uniform(a.page) : a.page;
    const bool there = entry >= 0 && entry < pages;
    const int64_t p = there ? entry : 0;
    Found f;
    f.k = (p * c.k_stride[0] + a.slot * c.k_stride[1]) * kBytes;
    f.v = (p * c.v_stride[0] + a.slot * c.v_stride[1]) * kBytes;
    f.ks = f.vs = 0;
    if constexpr (FORMAT != DCONV_CACHE_PLAIN) {
      f.ks = p * c.k_scale_stride[0] + a.slot * c.k_scale_stride[1];
      f.vs = p * c.v_scale_stride[0] + a.slot * c.v_scale_stride[1];
    }
    f.gone = ONE ? (there ? 0 : ~(uint64_t)0) : __ballot(!there);
    return f;
  }
};

__device__ __forceinline__ int64_t from_lane(int64_t x, int lane) {
  const int lo = __shfl((int)x, lane), hi = __shfl((int)(x >> 32), lane);
  return (int64_t)hi << 32 | (uint32_t)lo;
}
__device__ __forceinline__ int64_t from_uniform_lane(int64_t x, int lane) {
  const int lo = __builtin_amdgcn_readlane((int)x, lane), hi = __builtin_amdgcn_readlane((int)(x >> 32), lane);
  return (int64_t)hi << 32 | (uint32_t)lo;
}

// ---------------------------------------------------------------------------
// Tiles of a plain cache: copied into LDS
// ---------------------------------------------------------------------------
template <class T, int DP, int BN, int NW, bool ONE>
struct PlainTiles {
  typedef Copy<T, DP, BN, NW> C;
  static constexpr int kRows = C::kPieces < 64 ? 64 / C::kPieces : 1;   // of one copy of a wave, where they are whole
  static constexpr bool kWhole = 64 % C::kPieces == 0;
  C copy;             // offsets of the lane's pieces: from the tile's first row, or (not ONE) from the copy's
  int64_t stride;     // of slots, in elements

  __device__ __forceinline__ void init(int D, int64_t slot_stride, int wave, int lane) {
    stride = slot_stride;
    if constexpr (ONE || kWhole)
      copy.init(D, wave, lane, [&](int r) {
        return (uint32_t)(ONE ? r : r % kRows) * (uint32_t)slot_stride * (uint32_t)sizeof(T);
      });
  }
  // The tile from key j0 on, whose place is `at` (of its first key, or of the keys in
  // the lanes).  `close`: the rows of a copy stand in one page, and all are seen: a
  // scalar base and a 32-bit offset each.
  __device__ __forceinline__ void stage(T *lds, const char *base, int64_t at, const KeyRange<BN> &keys, int j0,
                                        bool close, bool pieces, int D, int wave, int lane) const {
    if (close) {
      if constexpr (ONE) {
        copy.tile(lds, reinterpret_cast<const T *>(base + at), C::kStep * stride * (int64_t)sizeof(T), wave);
        return;
      } else if constexpr (kWhole) {
#pragma unroll
        for (int i = 0; i < C::kCopies; ++i) {
          if (!C::has(i, wave)) break;
          uint32_t o = copy.offset[C::kStep ? 0 : i];
          asm volatile("" : "+v"(o));
          const char *row = base + from_uniform_lane(at, (i * C::kThreads + 64 * wave) / C::kPieces);
          __builtin_amdgcn_global_load_lds(row + o, (lds_ptr)C::to(lds, i, wave), 16, 0, 0);
        }
        return;
      }
    }
    auto row = [&](int r) {
      if constexpr (ONE)
        return reinterpret_cast<const T *>(base + at) + (keys.key(j0, j0 + r) - j0) * stride;
      else
        return reinterpret_cast<const T *>(base + from_lane(at, r));
    };
    if (pieces) {
      C::rows(lds, D, wave, lane, row);
      return;
    }
    // rows that are no whole pieces: element by element, zeros past D
    for (int x = 64 * wave + lane; x < BN * DP; x += C::kThreads) {
      const int r = x / DP, d = x % DP;
      const T *from = row(r);   // (by all lanes: places are in lanes)
      lds[Tile<T, DP>::at(r, d >> 3) + (d & 7)] = d < D ? from[d] : from_f32<T>(0.0f);
    }
  }
};

// ---------------------------------------------------------------------------
// Tiles of 8 and 4 bits: read into registers a tile ahead, converted into LDS
// ---------------------------------------------------------------------------
// A thread takes blocks of 32 neighbours with their scale: sixteen lanes the same
// block of sixteen rows (whose chunks lie on different banks of LDS), the next sixteen
// the next block of them.  TENSORS: keys and values, or values alone.
template <int WORDS>
struct __attribute__((packed, aligned(1))) RawCodes {
  uint32_t w[WORDS];
};
template <class T, int DP, int BN, int NT, int FORMAT, int TENSORS, bool ONE>
struct CodeTiles {
  static constexpr int kBlocks = DP / kBlock, kTensor = BN * kBlocks, kAll = TENSORS * kTensor;
  static constexpr int kPer = (kAll + NT - 1) / NT, kWords = kBlock / codes_per_word<FORMAT>();
  RawCodes<kWords> raw[kPer];
  uint32_t scale[kPer];

  static __device__ __forceinline__ bool has(int u) { return kAll % NT == 0 || u < kAll; }
  static __device__ __forceinline__ int row_of(int u) { return (u & 15) + u % kTensor / (16 * kBlocks) * 16; }
  static __device__ __forceinline__ int block_of(int u) { return (u >> 4) % kBlocks; }
  // k, v, ks, vs: the head's bases.
  __device__ __forceinline__ void load(const dconv_cache &c, const char *k, const char *v, const uint8_t *ks,
                                       const uint8_t *vs, const Found &f, const KeyRange<BN> &keys, int j0, int D,
                                       int thread) {
    const bool whole = ONE && keys.whole(j0);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int u = has(i * NT + thread) ? i * NT + thread : kAll - 1, row = row_of(u), blk = block_of(u);
      bool value = TENSORS == 1 || u >= kTensor;
      if constexpr (TENSORS == 1 || kTensor % 64 == 0) value = uniform(value);   // a wave's are of one tensor
      const char *from;
      const uint8_t *sfrom;
      if constexpr (ONE) {
        const int r = whole ? row : keys.key(j0, j0 + row) - j0;
        const int rs = (int)(value ? c.v_stride[1] : c.k_stride[1]);
        const int ss = (int)(value ? c.v_scale_stride[1] : c.k_scale_stride[1]);
        from = (value ? v + f.v : k + f.k) + (uint32_t)(r * rs + blk * (kWords * 4));
        sfrom = (value ? vs + f.vs : ks + f.ks) + (uint32_t)(r * ss + blk);
      } else if constexpr (TENSORS == 1 || kTensor % 64 == 0) {
        from = (value ? v : k) + from_lane(value ? f.v : f.k, row) + blk * (kWords * 4);
        sfrom = (value ? vs : ks) + from_lane(value ? f.vs : f.ks, row) + blk;
      } else {
        const int64_t ak = from_lane(f.k, row), av = from_lane(f.v, row), sk = from_lane(f.ks, row),
                      sv = from_lane(f.vs, row);
        from = (value ? v + av : k + ak) + blk * (kWords * 4);
        sfrom = (value ? vs + sv : ks + sk) + blk;
      }
      if (DP <= 128 || blk * kBlock < D) {   // (up to 128 a head is as long as it is padded to)
        raw[i] = *reinterpret_cast<const RawCodes<kWords> *>(from);
        scale[i] = *sfrom;
      } else {
        raw[i] = {};
        scale[i] = 0;
      }
    }
  }
  // (a block past the head's end is zeros: codes 0 times 2^-127)
  __device__ __forceinline__ void store(T *kt, T *vt, int thread) const {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int u = i * NT + thread, row = row_of(u), blk = block_of(u);
      if (!has(u)) break;
      T *to = TENSORS == 1 || u >= kTensor ? vt : kt;
      constexpr int kPairs = codes_per_word<FORMAT>() / 2;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        struct alignas(16) {
          T x[8];
        } y;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          decode_pair<T, FORMAT>(raw[i].w[(4 * j + e) / kPairs], (4 * j + e) % kPairs, scale_of(scale[i]), y.x + 2 * e);
        __builtin_memcpy(__builtin_assume_aligned(to + Tile<T, DP>::at(row, 4 * blk + j), 16), &y, sizeof(y));
      }
    }
  }
};

// The codes of 32 keys, copied into LDS as they are (32 rows by rows' lanes straight
// into registers would touch every row's line with each load) and read as row operands:
// the lane of key l % 32 takes elements 32 b + 16 (l / 32) .. + 15 of every block b, and
// the queries are taken in the same order (order_of), as the inner index has none.
template <class T, int DP, int FORMAT>
struct KeyCodes {
  typedef typename Mma<T>::Frag Frag;
  static constexpr int kBlocks = DP / kBlock, kWords = 16 / codes_per_word<FORMAT>();
  static constexpr int kRow = DP / kBlock * kWords * 8, kPieces = kRow / 16, kAll = 32 * kPieces;
  uint32_t scale[kBlocks];
  static __device__ __forceinline__ int order_of(int k, int half) { return 32 * (k / 2) + 16 * half + 8 * (k & 1); }
  // Pieces are permuted within a row so that sixteen rows' lie on different banks.
  static __device__ __forceinline__ int swizzle(int row) {
    return kPieces == 16 ? row & 15 : kPieces == 8 ? row >> 1 & 7 : kPieces == 4 ? row >> 2 & 3 : kPieces == 2 ? row >> 3 & 1 : 0;
  }
  // row(r): where row r is; scales: those of the lane's row.  `pieces`: rows begin on
  // 4-byte boundaries, which copies into LDS need.
  template <class F>
  __device__ __forceinline__ void load(char *lds, const uint8_t *scales, int D, int lane, bool pieces, F row) {
#pragma unroll
    for (int i = 0; i < (kAll + 63) / 64; ++i) {
      const int x = min(i * 64 + lane, kAll - 1), r = x / kPieces;
      int piece = x % kPieces ^ swizzle(r);
      if (DP > 128 && piece * (kBlock * 16) >= D * kWords * 8) piece = 0;   // (meets queries that are zeros)
      const char *from = row(r) + piece * 16;
      if (pieces) {
        if (kAll % 64 == 0 || i * 64 + lane < kAll)
          __builtin_amdgcn_global_load_lds(from, (lds_ptr)(lds + i * 1024), 16, 0, 0);
      } else {
        const RawCodes<4> w = *reinterpret_cast<const RawCodes<4> *>(from);
        __builtin_memcpy(__builtin_assume_aligned(lds + x * 16, 16), &w, 16);
      }
    }
    if constexpr (kBlocks == 4) {
      const uint32_t w = reinterpret_cast<const RawCodes<1> *>(scales)->w[0];
#pragma unroll
      for (int b = 0; b < 4; ++b) scale[b] = w >> 8 * b & 255;
    } else {
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) scale[b] = DP <= 128 || b * kBlock < D ? scales[b] : 0;
    }
  }
  // The lane's codes, of all blocks.
  __device__ __forceinline__ void read(const char *lds, int lane, RawCodes<kWords> (&raw)[kBlocks]) const {
    const int row = lane & 31, half = lane >> 5;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
      if constexpr (FORMAT == DCONV_CACHE_E4M3)
        __builtin_memcpy(&raw[b], __builtin_assume_aligned(lds + row * kRow + ((2 * b + half) ^ swizzle(row)) * 16, 16), 16);
      else
        __builtin_memcpy(&raw[b], __builtin_assume_aligned(lds + row * kRow + (b ^ swizzle(row)) * 16 + half * 8, 8), 8);
    }
  }
  // Operand k of them.
  __device__ __forceinline__ Frag frag(const RawCodes<kWords> (&raw)[kBlocks], int k) const {
    constexpr int kPairs = codes_per_word<FORMAT>() / 2;
    struct alignas(16) {
      T x[8];
    } y;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      decode_pair<T, FORMAT>(raw[k / 2].w[(4 * (k & 1) + e) / kPairs], (4 * (k & 1) + e) % kPairs,
                             scale_of(scale[k / 2]), y.x + 2 * e);
    Frag f;
    __builtin_memcpy(&f, &y, sizeof(f));
    return f;
  }
};

// ---------------------------------------------------------------------------
// Operands from LDS
// ---------------------------------------------------------------------------
// What Tile::row and Tile::column read, from four numbers of a lane: a chunk's place
// in its row is an exclusive or with constants, so an address is one instruction
// (v_xad) from two of them.  Kept as addresses they would take a sixth of the registers.
template <class T, int DP>
struct Reader {
  typedef typename Mma<T>::Frag Frag;
  static constexpr uint32_t kRow = DP * sizeof(T), kChunk = 8 * sizeof(T);
  uint32_t rx, rb, cx, cb;
  __device__ __forceinline__ explicit Reader(int lane) {
    const int row = lane & 31, half = lane >> 5;
    rb = row * kRow;
    rx = (half ^ Tile<T, DP>::swizzle(row)) * kChunk;
    if constexpr (sizeof(T) == 2) {
      const int r = 4 * half + ((lane & 15) >> 2);
      cb = r * kRow + 4 * (lane & 1) * sizeof(T);
      cx = ((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ Tile<T, DP>::swizzle(r)) * kChunk;
    } else {
      cb = 4 * half * kRow + (lane & 7) * sizeof(T);
      cx = ((row >> 3) ^ Tile<T, DP>::swizzle(4 * half)) * kChunk;
    }
  }
  // (computed again from here on, not kept)
  __device__ __forceinline__ void again() { asm volatile("" : "+v"(rx), "+v"(rb), "+v"(cx), "+v"(cb)); }
  static __device__ __forceinline__ const char *bytes(const T *t) { return reinterpret_cast<const char *>(t); }

  __device__ __forceinline__ Frag row(const T *t, int r0, int k) const {
    const char *p = bytes(t) + ((rx ^ 2 * k * kChunk) + rb) + r0 * kRow;
    if constexpr (sizeof(T) == 4) {
      typedef float f32x4 __attribute__((ext_vector_type(4)));   // (two loads: see Tile::row)
      const f32x4 a = *reinterpret_cast<const f32x4 *>(p), b = *reinterpret_cast<const f32x4 *>(p + 16);
      return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      return *reinterpret_cast<const Frag *>(p);
    }
  }
  __device__ __forceinline__ Frag column(const T *t, int r0, int c) const {
    Frag f;
    if constexpr (sizeof(T) == 2) {
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) s16x4 *lds_s16x4;
      s16x4 v[2];
#pragma unroll
      for (int j = 0; j < 2; ++j)   // (rows 8 further: two chunks further, exclusively or)
        v[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_s16x4)(bytes(t) + ((cx ^ (4 * c ^ 2 * j) * kChunk) + cb) + (r0 + 8 * j) * kRow));
      __builtin_memcpy(&f, v, 16);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        f[e] = *reinterpret_cast<const T *>(bytes(t) + ((cx ^ (4 * c ^ e % 4) * kChunk) + cb) +
                                            (r0 + 8 * (e / 4) + e % 4) * kRow);
    }
    return f;
  }
};

// The running softmax of 32 rows, with operands by a Reader.
template <class T, int DP>
struct CacheSoftmax : Softmax<T, DP> {
  typedef Softmax<T, DP> Base;
  typedef typename Mma<T>::Frag Frag;
  static constexpr int KS = Base::KS, DT = Base::DT;
  using Base::o;

  static __device__ __forceinline__ f32x16 scores(const Reader<T, DP> &rd, const T *ks, int k0, const Frag (&q)[KS]) {
    f32x16 s = {};
    if constexpr (sizeof(T) == 4) {   // two sums: half as many roundings one after another
      f32x16 z = {};
#pragma unroll
      for (int k = 0; k < KS; k += 2) {
        s = Mma<T>::mac(rd.row(ks, k0, k), q[k], s);
        z = Mma<T>::mac(rd.row(ks, k0, k + 1), q[k + 1], z);
      }
      return s + z;
    }
#pragma unroll
    for (int k = 0; k < KS; ++k) s = Mma<T>::mac(rd.row(ks, k0, k), q[k], s);
    return s;
  }
  // (operands are read well before their products, where registers hold them)
  static constexpr bool kReadAhead = KS * sizeof(Frag) <= 128;
  static __device__ __forceinline__ f32x16 scores_ahead(const Reader<T, DP> &rd, const T *ks, const Frag (&q)[KS]) {
    if constexpr (!kReadAhead) return scores(rd, ks, 0, q);
    Frag kf[KS];
    load_keys(rd, kf, ks, 0);
    return Base::products(kf, q);
  }
  __device__ __forceinline__ void values_ahead(const Reader<T, DP> &rd, const T *vs, const Frag (&w)[2]) {
    if constexpr (!kReadAhead) return values(rd, vs, 0, w);
    Frag vf[2][DT];
    load_values(rd, vf[0], vs, 0);
    load_values(rd, vf[1], vs, 16);
    Base::weigh(vf[0], w[0]);
    Base::weigh(vf[1], w[1]);
  }
  __device__ __forceinline__ void values(const Reader<T, DP> &rd, const T *vs, int k0, const Frag (&w)[2]) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int c = 0; c < DT; ++c) o[c] = Mma<T>::mac(rd.column(vs, k0 + 16 * k, c), w[k], o[c]);
  }
  static __device__ __forceinline__ void load_keys(const Reader<T, DP> &rd, Frag (&f)[KS], const T *ks, int k0) {
#pragma unroll
    for (int k = 0; k < KS; ++k) f[k] = rd.row(ks, k0, k);
    in_order();
  }
  static __device__ __forceinline__ void load_values(const Reader<T, DP> &rd, Frag (&f)[DT], const T *vs, int k0) {
#pragma unroll
    for (int c = 0; c < DT; ++c) f[c] = rd.column(vs, k0, c);
    in_order();
  }
  // Adds 32 keys, j0 .., of the tiles ks, vs.
  __device__ __forceinline__ void add(Reader<T, DP> rd, const T *ks, const T *vs, const Frag (&q)[KS], int j0,
                                      const RowKeys &see, int sinks, float scale2, bool masked, int lane,
                                      uint32_t gone) {
    rd.again();
    if constexpr (kReadAhead) {
      Frag kf[KS], vf[2][DT];
      load_keys(rd, kf, ks, 0);
      f32x16 s = Base::products(kf, q);
      load_values(rd, vf[0], vs, 0);
      if (masked) Base::mask(s, j0, see, sinks, lane, gone);
      Base::follow(s, scale2, [] {});
      Frag w[2];
      Base::probabilities(s, scale2, w);
      load_values(rd, vf[1], vs, 16);
      Base::weigh(vf[0], w[0]);
      Base::weigh(vf[1], w[1]);
      return;
    }
    f32x16 s = scores(rd, ks, 0, q);
    if (masked) Base::mask(s, j0, see, sinks, lane, gone);
    Base::follow(s, scale2, [] {});
    Frag w[2];
    Base::probabilities(s, scale2, w);
    values(rd, vs, 0, w);
  }
  // Adds 64 keys, the matrix and the vector unit at the same time (Softmax::add_two).
  __device__ __forceinline__ void add_two(Reader<T, DP> rd, const T *ks, const T *vs, const Frag (&q)[KS], int j0,
                                          const RowKeys &see, int sinks, float scale2, bool masked, int lane,
                                          uint64_t gone) {
    const uint32_t gone0 = (uint32_t)gone, gone1 = (uint32_t)(gone >> 32);
    Frag w0[2], w1[2];
    rd.again();
    Frag kf[KS], vf[2][DT];
    load_keys(rd, kf, ks, 0);
    f32x16 s0 = Base::products(kf, q), s1;
    load_keys(rd, kf, ks, 32);
    if (masked) Base::mask(s0, j0, see, sinks, lane, gone0);
    Base::follow(s0, scale2, [] {});
    s1 = Base::products(kf, q);
    load_values(rd, vf[0], vs, 0);
    Base::probabilities(s0, scale2, w0);
    asm volatile("" ::"v"(w0[0]), "v"(w0[1]));
    if (masked) Base::mask(s1, j0 + 32, see, sinks, lane, gone1);
    Base::follow(s1, scale2, [&] {
      values(rd, vs, 0, w0);
      w0[0] = w0[1] = Frag{};
    });
    load_values(rd, vf[1], vs, 16);
    Base::weigh(vf[0], w0[0]);
    load_values(rd, vf[0], vs, 32);
    Base::weigh(vf[1], w0[1]);
    load_values(rd, vf[1], vs, 48);
    Base::probabilities(s1, scale2, w1);
    Base::weigh(vf[0], w1[0]);
    Base::weigh(vf[1], w1[1]);
  }
};

// ---------------------------------------------------------------------------
// Division of the work
// ---------------------------------------------------------------------------
// An item is a tile of rows of one key head of one sequence; its work is its number
// of keys and a constant.  Lengths are on the device, so every workgroup sums all
// sequences' work and takes an equal share of it, a range of a line on which the
// items stand one behind another: parts of two items, and whole ones between them.
// A wave's lanes take as many sequences each.  Cuts depend on the line alone, so the
// workgroups agree on them, and sums are joined in a fixed order.
constexpr int kFewRows = 32, kTileRows = 128;

template <bool FEW>
struct Work {
  int rows, tiles;          // of a key head
  int64_t base, cap, step;  // work of tile i: min(base + i step, cap) + kFixed
  static constexpr int kFixed = 64;
  __device__ __forceinline__ Work(const dconv_cache_attend_shape &sh, int G, const Rows &s, int most) {
    rows = s.n * G;
    tiles = 0;
    base = cap = step = 0;
    if (s.n <= 0 || s.n > most || (rows <= kFewRows) != FEW) return;
    tiles = FEW ? 1 : (rows + kTileRows - 1) / kTileRows;
    step = FEW ? 0 : max(kTileRows / G, 1);
    const int i0 = s.start(), i1 = i0 + (FEW ? s.n : min(s.n, (int)step)) - 1;
    cap = s.len;
    if (sh.left >= 0)
      cap = min(cap, (int64_t)sh.left + max(sh.right, 0) + 1 + (sh.right < 0 ? s.len : step + s.n * FEW) + sh.sinks);
    if (i1 >= 0) {
      const KeySpan a = keys_seen(sh, s.len, max(i0, 0)), b = keys_seen(sh, s.len, i1);
      base = min((int64_t)a.first + max(b.hi - a.lo, 0), cap);
    }
  }
  __device__ __forceinline__ int64_t of(int i) const { return min(base + i * step, cap) + kFixed; }
  // Work of the tiles before i.
  __device__ __forceinline__ int64_t before(int64_t i) const {
    const int64_t rising = step > 0 ? min(i, (cap - base) / step + 1) : i;
    return i * kFixed + rising * base + step * (rising * (rising - 1) / 2) + (i - rising) * cap;
  }
  // The tile that holds point z < before(tiles).
  __device__ __forceinline__ int at(int64_t z) const {
    int lo = 0, hi = tiles;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (before(mid) <= z) lo = mid;
      else hi = mid;
    }
    return lo;
  }
};

__device__ __forceinline__ int64_t uniform64(int64_t x) {
  return (int64_t)uniform((int)(x >> 32)) << 32 | (uint32_t)uniform((int)x);
}

__device__ __forceinline__ int most_rows(const CacheCall &a) { return a.sh.max_rows > 0 ? a.sh.max_rows : a.t.N; }

// A workgroup's range of the line: it begins `at` work into sequence b.
struct Range {
  int id, b;
  int64_t at, begin, end, share;
};
struct RangeScratch {
  int64_t wave[4], at;
  int b;
};
template <bool FEW, int NT>
__device__ __forceinline__ Range find_range(const CacheCall &a, RangeScratch &lds) {
  const dconv_cache &c = a.c;
  const CacheTile &ct = a.tile<FEW>();
  const dconv_cache_attend_shape &sh = a.sh;
  const Batch &t = a.t;
  const CachePtrs &p = a.p.cache;
  const int tid = threadIdx.x, G = sh.Hq / c.Hkv, most = most_rows(a);
  if (ct.whole > 0) {   // an item
    Range r = {};
    r.id = xcd_remap(blockIdx.x, ct.groups);
    r.b = r.id / (c.Hkv * ct.whole);
    r.end = 1;
    return r;
  }
  const int per = (t.B + NT - 1) / NT, b0 = min(tid * per, t.B), b1 = min(b0 + per, t.B);
  auto work = [&](int b) {
    const Work<FEW> w(sh, G, rows_of(t, p, b), most);
    return w.tiles > 0 ? w.before(w.tiles) * c.Hkv : (int64_t)0;
  };
  int64_t mine = 0;
  for (int b = b0; b < b1; ++b) mine += work(b);
  int64_t upto = mine;   // of the wave's lanes up to this one
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t x = from_lane(upto, (int)(tid & 63) - d);
    if ((tid & 63) >= d) upto += x;
  }
  if ((tid & 63) == 63) lds.wave[tid >> 6] = upto;
  if (tid == 0) lds.b = t.B;
  __syncthreads();
  int64_t total = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    if (w < (tid >> 6)) upto += lds.wave[w];
    total += lds.wave[w];
  }
  Range r;
  r.id = xcd_remap(blockIdx.x, ct.groups);
  r.share = max((total + ct.groups - 1) / ct.groups, (int64_t)ct.least);
  r.begin = r.id * r.share;
  r.end = min(r.begin + r.share, total);
  int64_t from = upto - mine;
  if (r.begin < total && from <= r.begin && r.begin < upto) {
    int b = b0;
    for (;; ++b) {
      const int64_t x = work(b);
      if (r.begin < from + x || b + 1 >= b1) break;
      from += x;
    }
    lds.b = b;
    lds.at = r.begin - from;
  }
  __syncthreads();
  r.b = uniform(lds.b);
  r.at = r.b < t.B ? uniform64(lds.at) : 0;
  r.share = uniform64(r.share);
  r.begin = uniform64(r.begin);
  r.end = uniform64(r.end);
  return r;
}

// A value that the compiler computes again where it is used: what a loop over
// segments would otherwise carry in registers (masks of a head's end, addresses in
// LDS) does not fit them.
__device__ __forceinline__ int again_scalar(int x) {
  asm volatile("" : "+s"(x));
  return x;
}
__device__ __forceinline__ int again_vector(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// A segment of an item: from `pos` to `end` of its work.
struct Segment {
  int b, hk, tile;
  Rows s;
  int64_t pos, end, work, item;   // item: where the item begins on the line
};

// Steps that lie before point pos of an item with `steps` of them.  (Cuts near an
// end go to it: a sliver costs as much as the constant.)
__device__ __forceinline__ int cut(int64_t pos, int64_t work, int steps, int64_t share) {
  if (pos < work && pos <= share / 8) return 0;
  if (work - pos <= share / 8) return steps;
  return (int)(pos * steps / work);
}

// The join of a segment's item, of which the segment's workgroup has a part.
__device__ __forceinline__ CacheJoin join_of(const Range &r, const Segment &g, int steps, int r0, int rows) {
  int first = (int)(g.item / r.share), upto;   // (or one after it, where its cut has gone to the item's beginning)
  while ((upto = cut(min((first + 1) * r.share - g.item, g.work), g.work, steps, r.share)) == 0 && first < r.id) ++first;
  if (upto == steps) return {};                // the first has done all of it: a cut has gone to the item's end
  return {(int)((g.item + g.work - 1) / r.share) - first + 1, first, r.id - first, g.b, g.hk, r0, rows, g.s};
}

// A workgroup's records of joins, until a segment has one.
template <bool FEW>
__device__ __forceinline__ void no_joins(const Range &r) {
  const CacheTile &ct = fresh().tile<FEW>();
  if (threadIdx.x == 0 && ct.whole == 0) ct.joins[2 * r.id].parts = ct.joins[2 * r.id + 1].parts = 0;
}

template <bool FEW, class F>
__device__ __forceinline__ void for_segments(const Range &r, F f) {
  int64_t x = r.begin, at = r.at;
  for (int b = r.b; x < r.end; ++b) {
    const CacheCall &a = fresh();
    if (b >= a.t.B) break;
    const int G = a.sh.Hq / a.c.Hkv, heads = a.c.Hkv;
    Rows s = rows_of(a.t, a.p.cache, b);
    s = {uniform(s.row), uniform(s.n), uniform(s.len)};
    const Work<FEW> w(a.sh, G, s, most_rows(a));
    const int whole = a.tile<FEW>().whole;
    int hk = 0, tile = 0;
    if (whole > 0) {   // one item, as if it were the line
      tile = r.id % whole;
      hk = r.id / whole % heads;
      if (tile >= w.tiles) break;
    }
    if (w.tiles == 0) continue;
    const int64_t head = w.before(w.tiles);
    if (whole == 0 && at > 0) {
      hk = (int)(at / head);
      at -= hk * head;
      tile = w.at(at);
      at -= w.before(tile);
    }
    for (; hk < heads && x < r.end; ++hk, tile = 0)
      for (; tile < w.tiles && x < r.end; ++tile) {
        Segment g = {b, uniform(hk), uniform(tile), s, at, 0, whole > 0 ? 1 : w.of(tile), x - at};
        g.end = min(g.work, at + (r.end - x));
        f(g);
        x += g.end - at;
        at = 0;
      }
  }
}

// Parts of R rows: sums, bases and totals.
template <int R, int DP>
constexpr int cache_part() { return R * (DP + 2); }

// ---------------------------------------------------------------------------
// 128 rows: four waves of 32 share tiles of keys
// ---------------------------------------------------------------------------
// A plain cache's tiles are copied into two LDS buffers in turn, the next while the
// current one is used; codes come a tile ahead into registers and go into the other
// buffer after it.  Chunks of 401 to 512 tokens over up to 8192, 32 heads of 128 over
// 8, bf16: 168 GFLOP of seen scores in 247 us (680 TFLOP/s; matrix cores busy in 0.38 of the
// cycles, vector instructions issuing in 0.42, waves waiting for data in 0.25 of theirs and
// for a unit in 0.31: two waves per SIMD, each a chain of operands, products and
// exponentials, do not fill it), and 24 us for the join of rows that two or three
// workgroups have parts of.
template <class T, int DP, int FORMAT, bool ONE, int LEN>
__device__ __forceinline__ void tiles_body(T (&buf0)[LEN], T (&buf1)[LEN], RangeScratch &scratch) {
  constexpr int BN = forward_keys<T>(DP), KS = DP / 16, DT = DP / 32;
  typedef typename Mma<T>::Frag Frag;
  static_assert(2 * BN * DP <= LEN, "a tile's keys and values");
  const int wave = uniform(threadIdx.x >> 6);
  const Range range = find_range<false, 256>(fresh(), scratch);
  no_joins<false>(range);

  for_segments<false>(range, [&](const Segment &g) {
    const CacheCall &a = fresh();
    const dconv_cache &c = a.c;
    const dconv_cache_attend_shape &sh = a.sh;
    const Batch &t = a.t;
    const CacheAttendPtrs &p = a.p;
    const CacheTile &ct = a.tile<false>();
    const int G = sh.Hq / c.Hkv, sinks = again_scalar(sh.sinks);
    const float scale2 = __int_as_float(again_scalar(__float_as_int(ct.scale2)));
    const int lane = again_vector(threadIdx.x & 63), D = again_scalar(c.D);
    const int rows = g.s.n * G, r0 = g.tile * kTileRows, start = g.s.start();
    const KeyRange<BN> keys(sh, g.s.len, start + r0 / G, start + (min(r0 + kTileRows, rows) - 1) / G);
    const int u0 = uniform(cut(g.pos, g.work, keys.n, range.share)), u1 = uniform(cut(g.end, g.work, keys.n, range.share));
    // nothing of it, and no part of it: all lies before, or after
    if (u0 == u1 && (keys.n == 0 ? g.pos > 0 : u0 == 0)) return;
    const bool complete = u0 == 0 && u1 == keys.n;

    const int r = r0 + 32 * wave + (lane & 31), rr = min(r, rows - 1), row = g.s.row + rr / G, h = g.hk * G + rr % G;
    const KeySpan span = keys_seen(sh, g.s.len, start + rr / G);
    const RowKeys see = {span.lo, span.none() ? 0 : span.hi, span.none()};
    // the wave's keys: none outside [from, to) but for the first ones, all seen by
    // all rows inside [all_from, all_to)
    int from = see.lo, to = see.hi, all_from = see.lo, all_to = see.hi;
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) {
      from = min(from, __shfl_xor(from, x));
      to = max(to, __shfl_xor(to, x));
      all_from = max(all_from, __shfl_xor(all_from, x));
      all_to = min(all_to, __shfl_xor(all_to, x));
    }
    from = uniform(from), to = uniform(to), all_from = uniform(all_from), all_to = uniform(all_to);
    if (r0 + 32 * wave >= rows) to = 0, from = 0x7fffffff;   // a wave without rows sees nothing
    const bool idle = r0 + 32 * wave >= rows;

    Frag q[KS];
    const T *qrow = static_cast<const T *>(p.q) + row * sh.q_stride[0] + h * sh.q_stride[1];
#pragma unroll
    for (int k = 0; k < KS; ++k) q[k] = load_frag(qrow, 16 * k + 8 * (lane >> 5), D, ct.direct, ct.sign);

    const Finder<T, FORMAT, BN, ONE> finder = {p.cache.table + g.b * t.table_stride, t.page, t.pages};
    const int64_t es = Finder<T, FORMAT, BN, ONE>::kBytes;
    const char *kb = static_cast<const char *>(p.cache.k) + g.hk * c.k_stride[2] * es;
    const char *vb = static_cast<const char *>(p.cache.v) + g.hk * c.v_stride[2] * es;
    const Reader<T, DP> rd(lane);
    CacheSoftmax<T, DP> soft;
    soft.clear();
    auto step = [&](const T *buf, int j0, uint64_t gone) {
      auto unseen = [&](int v0, int N) { return idle || v0 >= to || (v0 + N <= from && v0 >= sinks); };
      auto masked = [&](int v0, int N) {
        return gone != 0 || !(v0 + N <= all_to && (v0 >= all_from || v0 + N <= sinks));
      };
      if constexpr (BN == 64 && sizeof(T) == 2 && (FORMAT == DCONV_CACHE_PLAIN || DP <= 64)) {
        if (!unseen(j0, BN))
          soft.add_two(rd, buf, buf + BN * DP, q, j0, see, sinks, scale2, masked(j0, BN), lane, gone);
      } else {
        // (codes of the next tile are on their way to registers: the scores of a second
        // 32 keys would not fit beside them)
#pragma unroll
        for (int k = 0; k < BN; k += 32)
          if (!unseen(j0 + k, 32))
            soft.add(rd, buf + k * DP, buf + (BN + k) * DP, q, j0 + k, see, sinks, scale2, masked(j0 + k, 32), lane,
                     (uint32_t)(gone >> k));
      }
    };
    __syncthreads();   // the segment before is through with the buffers
    if (u0 < u1) {
      Asked asked = finder.ask(keys, keys.start(u0));
      if constexpr (FORMAT == DCONV_CACHE_PLAIN) {
        typedef PlainTiles<T, DP, BN, 4, ONE> Tiles;
        Tiles kt, vt;
        kt.init(D, c.k_stride[1], wave, lane);
        vt.init(D, c.v_stride[1], wave, lane);
        const bool near = ct.near && (ONE || (Tiles::kWhole && t.page.d % Tiles::kRows == 0));
        // stages tile u and asks for the one after it
        auto stage = [&](T *buf, int u) {
          const int j0 = keys.start(u);
          const Found f = finder.find(c, asked);
          const bool close = near && keys.whole(j0);
          kt.stage(buf, kb, f.k, keys, j0, close, ct.pieces, D, wave, lane);
          vt.stage(buf + BN * DP, vb, f.v, keys, j0, close, ct.pieces, D, wave, lane);
          if (u + 1 < u1) asked = finder.ask(keys, keys.start(u + 1));
          return f.gone;
        };
        auto arrived = [&]() {
          landed<0>();
          __syncthreads();
        };
        uint64_t gone0 = stage(buf0, u0), gone1 = 0;
        for (int u = u0; u < u1; u += 2) {
          arrived();
          if (u + 1 < u1) gone1 = stage(buf1, u + 1);
          step(buf0, keys.start(u), gone0);
          if (u + 1 >= u1) break;
          arrived();
          if (u + 2 < u1) gone0 = stage(buf0, u + 2);
          step(buf1, keys.start(u + 1), gone1);
        }
      } else {
        const uint8_t *ksb = p.cache.k_scale + g.hk * c.k_scale_stride[2], *vsb = p.cache.v_scale + g.hk * c.v_scale_stride[2];
        CodeTiles<T, DP, BN, 256, FORMAT, 2, ONE> codes;
        uint64_t next = 0;
        auto load = [&](int u) {
          const Found f = finder.find(c, asked);
          codes.load(c, kb, vb, ksb, vsb, f, keys, keys.start(u), D, threadIdx.x);
          next = f.gone;
          if (u + 1 < u1) asked = finder.ask(keys, keys.start(u + 1));
        };
        load(u0);
        codes.store(buf0, buf0 + BN * DP, threadIdx.x);
        uint64_t gone = next;
        if (u0 + 1 < u1) load(u0 + 1);
        __syncthreads();
        for (int u = u0; u < u1; ++u) {
          T *now = (u - u0) & 1 ? buf1 : buf0, *then = (u - u0) & 1 ? buf0 : buf1;
          step(now, keys.start(u), gone);
          if (u + 1 >= u1) break;
          codes.store(then, then + BN * DP, threadIdx.x);
          gone = next;
          if (u + 2 < u1) load(u + 2);
          __syncthreads();
        }
      }
    }

    const float l = half_sum(soft.l);
    if (!complete) {
      float *part = ct.partial + ((int64_t)range.id * 2 + (u0 == 0)) * cache_part<kTileRows, DP>();
      const int x = 32 * wave + (lane & 31);
#pragma unroll
      for (int k = 0; k < DT; ++k)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const float y[4] = {soft.o[k][i], soft.o[k][i + 1], soft.o[k][i + 2], soft.o[k][i + 3]};
          __builtin_memcpy(__builtin_assume_aligned(part + x * DP + 32 * k + acc_row(i, lane >> 5), 16), y, 16);
        }
      if (lane < 32) {
        part[kTileRows * DP + x] = soft.m;
        part[kTileRows * (DP + 1) + x] = l;
      }
      if (threadIdx.x == 0) fresh().tiles.joins[2 * range.id + (u0 == 0)] = join_of(range, g, keys.n, r0, min(kTileRows, rows - r0));
      return;
    }
    const float inv = see.none ? 0.0f : 1.0f / l;
    bool bad = false;
#pragma unroll
    for (int k = 0; k < DT; ++k)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        soft.o[k][i] = see.none ? 0.0f : soft.o[k][i] * inv;
        bad |= 32 * k + acc_row(i, lane >> 5) < D && !(fabsf(soft.o[k][i]) < INFINITY);
      }
    const unsigned long long any = __ballot(bad && r < rows);
    const unsigned redo = kSumAgain ? (unsigned)(any | (any >> 32)) : 0u;
    if (r < rows && !(redo >> (lane & 31) & 1)) {
      T *o = static_cast<T *>(p.out) + row * sh.out_stride[0] + h * sh.out_stride[1];
#pragma unroll
      for (int k = 0; k < DT; ++k)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const int d = 32 * k + acc_row(i, lane >> 5);
          T x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = from_f32<T>(soft.o[k][i + e]);
          if (ct.direct && d + 4 <= D) {
            __builtin_memcpy(__builtin_assume_aligned(o + d, 4), x, sizeof(x));
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (d + e < D) o[d + e] = x[e];
          }
        }
      if (p.lse && lane < 32) p.lse[(int64_t)row * sh.Hq + h] = see.none ? -INFINITY : log_sum(soft.m, l);
    }
    // A row with a result that is not finite is taken again by the plain form, which
    // reads seen keys and values only: a zero probability times an infinity or NaN
    // that the row does not see has made a NaN here (or it sees no page).
    for (unsigned again = redo; again; again &= again - 1) {
      const int x = r0 + 32 * wave + __ffs(again) - 1;
      const CacheCall &f = fresh();
      cache_attend_row<T, FORMAT>(f.c, f.sh, f.t, f.p, g.b, g.s, g.s.row + x / G, g.hk * G + x % G);
    }
  });
}

// ---------------------------------------------------------------------------
// Up to 32 rows: each wave takes tiles of 32 keys by itself
// ---------------------------------------------------------------------------
// No barrier between tiles.  Bound by memory for a plain cache: 32 sequences of 853 to
// 16384 tokens, 8 key heads of 128, bf16, 1125 MB in 216 us (5.2 TB/s).  A tile of
// codes takes a wave as long for half or a quarter of the bytes: 64 sequences over 4
// key heads in e4m3, 568 MB in 144 us (3.9 TB/s); 131072 tokens, 8 heads, five rows
// each of 4, e2m1, 142 MB in 45 us (3.2 TB/s), the same with all pages in L2.  Reading
// codes two or three tiles ahead gains nothing, for want of registers (568 MB: 162 and 244
// us a call, join and all, beside 151).
template <class T, int DP>
struct FewScratch {
  float ml[split_waves<T>(DP)][64];
  unsigned again;
};
template <class T, int DP, int FORMAT, bool ONE, int LEN>
__device__ __forceinline__ void few_body(T (&kbuf)[LEN], T (&vbuf)[LEN], RangeScratch &scratch, FewScratch<T, DP> &fs) {
  constexpr int KS = DP / 16, DT = DP / 32, BN = 32, kTile = BN * DP, W = split_waves<T>(DP);
  typedef typename Mma<T>::Frag Frag;
  typedef KeyCodes<T, DP, FORMAT == DCONV_CACHE_PLAIN ? DCONV_CACHE_E4M3 : FORMAT> Codes;
  static_assert(W * kTile <= LEN, "a tile of each wave");
  float(&ml)[W][64] = fs.ml;
  unsigned &again = fs.again;
  const int wave = uniform(threadIdx.x >> 6);
  const Range range = find_range<true, 64 * W>(fresh(), scratch);
  no_joins<true>(range);

  for_segments<true>(range, [&](const Segment &g) {
    const CacheCall &a = fresh();
    const dconv_cache &c = a.c;
    const dconv_cache_attend_shape &sh = a.sh;
    const Batch &t = a.t;
    const CacheAttendPtrs &p = a.p;
    const CacheTile &ct = a.tile<true>();
    const int G = sh.Hq / c.Hkv, sinks = again_scalar(sh.sinks);
    const float scale2 = __int_as_float(again_scalar(__float_as_int(ct.scale2)));
    const int lane = again_vector(threadIdx.x & 63), D = again_scalar(c.D);
    const int rows = g.s.n * G, start = g.s.start();
    const KeyRange<BN> keys(sh, g.s.len, start, start + g.s.n - 1);
    const int steps = (keys.n + W - 1) / W;
    const int u0 = uniform(cut(g.pos, g.work, steps, range.share)), u1 = uniform(cut(g.end, g.work, steps, range.share));
    if (u0 == u1 && (steps == 0 ? g.pos > 0 : u0 == 0)) return;
    const bool complete = u0 == 0 && u1 == steps;

    const int r = lane & 31, rr = min(r, rows - 1), row = g.s.row + rr / G, h = g.hk * G + rr % G;
    const KeySpan span = keys_seen(sh, g.s.len, start + rr / G);
    const RowKeys see = {span.lo, span.none() ? 0 : span.hi, span.none()};
    int all_from = see.lo, all_to = see.hi;   // keys that all rows see
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) {
      all_from = max(all_from, __shfl_xor(all_from, x));
      all_to = min(all_to, __shfl_xor(all_to, x));
    }
    all_from = uniform(all_from), all_to = uniform(all_to);
    Frag q[KS];
    const T *qrow = static_cast<const T *>(p.q) + row * sh.q_stride[0] + h * sh.q_stride[1];
#pragma unroll
    for (int k = 0; k < KS; ++k)
      q[k] = load_frag(qrow, FORMAT == DCONV_CACHE_PLAIN ? 16 * k + 8 * (lane >> 5) : Codes::order_of(k, lane >> 5), D,
                       ct.direct, ct.sign);

    const Finder<T, FORMAT, BN, ONE> finder = {p.cache.table + g.b * t.table_stride, t.page, t.pages};
    const int64_t es = Finder<T, FORMAT, BN, ONE>::kBytes;
    const char *kb = static_cast<const char *>(p.cache.k) + g.hk * c.k_stride[2] * es;
    const char *vb = static_cast<const char *>(p.cache.v) + g.hk * c.v_stride[2] * es;
    const Reader<T, DP> reader(lane);
    CacheSoftmax<T, DP> soft;
    soft.clear();
    T *kt = kbuf + wave * kTile, *vt = vbuf + wave * kTile;
    // Scores to probabilities.
    auto weigh = [&](f32x16 &s, int j0, uint32_t gone, Frag(&w)[2]) {
      if (gone != 0 || !(j0 + BN <= all_to && (j0 >= all_from || j0 + BN <= sinks)))
        soft.mask(s, j0, see, sinks, lane, gone);
      soft.follow(s, scale2, [] {});
      soft.probabilities(s, scale2, w);
    };
    // this wave's tiles: u0 W + wave, and every W-th from there
    const int end = min(u1 * W, keys.n);
    int u = u0 * W + wave;
    if (u < end) {
      Asked asked = finder.ask(keys, keys.start(u));
      if constexpr (FORMAT == DCONV_CACHE_PLAIN) {
        // Keys and values have a buffer each, filled again as soon as it is read: a
        // tile is on its way through all of the other's arithmetic.
        typedef PlainTiles<T, DP, BN, 1, ONE> Tiles;
        Tiles ck, cv;
        ck.init(D, c.k_stride[1], 0, lane);
        cv.init(D, c.v_stride[1], 0, lane);
        const bool near = ct.near && (ONE || (Tiles::kWhole && t.page.d % Tiles::kRows == 0));
        Found f = finder.find(c, asked);
        auto stage_keys = [&](int v) {
          const int j0 = keys.start(v);
          ck.stage(kt, kb, f.k, keys, j0, near && keys.whole(j0), ct.pieces, D, 0, lane);
        };
        auto stage_values = [&](int v) {
          const int j0 = keys.start(v);
          cv.stage(vt, vb, f.v, keys, j0, near && keys.whole(j0), ct.pieces, D, 0, lane);
        };
        stage_keys(u);
        if (u + W < end) asked = finder.ask(keys, keys.start(u + W));
        stage_values(u);
        for (; u < end; u += W) {
          const uint32_t gone = (uint32_t)f.gone;
          const bool more = u + W < end;
          Reader<T, DP> rd = reader;
          rd.again();
          landed<Tiles::C::kCopies>();   // the keys; the values may still be on their way
          f32x16 s = soft.scores_ahead(rd, kt, q);
          landed<Tiles::C::kCopies>();   // (read)
          if (more) {
            f = finder.find(c, asked);
            stage_keys(u + W);
          }
          Frag w[2];
          weigh(s, keys.start(u), gone, w);
          if (more) landed<Tiles::C::kCopies>();   // the values; not the next keys
          else landed<0>();
          soft.values_ahead(rd, vt, w);
          if (more) {
            if (u + 2 * W < end) asked = finder.ask(keys, keys.start(u + 2 * W));
            landed<63>();   // (read)
            stage_values(u + W);
          }
        }
      } else {
        // Codes come a tile ahead: keys into LDS, values into registers and from there,
        // converted, into LDS, which turns them.
        const uint8_t *ksb = p.cache.k_scale + g.hk * c.k_scale_stride[2], *vsb = p.cache.v_scale + g.hk * c.v_scale_stride[2];
        Codes kc;
        CodeTiles<T, DP, BN, 64, FORMAT, 1, ONE> vc;
        char *kl = reinterpret_cast<char *>(kt);
        static_assert(32 * Codes::kRow <= kTile * (int)sizeof(T), "the codes of a tile of keys");
        uint32_t next = 0;
        // (past the last tile it comes again: loads under a condition would be waited for
        // one and all, as the compiler cannot count them)
        const int last = u + (end - 1 - u) / W * W;
        auto load = [&](int v) {   // tile v, whose places have been asked for
          const Found f = finder.find(c, asked);
          asked = finder.ask(keys, keys.start(min(v + W, last)));
          const int j0 = keys.start(v);
          const bool whole = keys.whole(j0);
          auto slot = [&](int r) { return (uint32_t)(whole ? r : keys.key(j0, j0 + r) - j0); };
          const uint32_t ks = (uint32_t)c.k_stride[1];
          auto krow = [&](int r) { return ONE ? kb + f.k + slot(r) * ks : kb + from_lane(f.k, r); };
          kc.load(kl, ksb + f.ks + (ONE ? slot(lane & 31) * (uint32_t)c.k_scale_stride[1] : 0), D, lane, ct.pieces, krow);
          vc.load(c, kb, vb, ksb, vsb, f, keys, j0, D, lane);
          next = (uint32_t)f.gone;
        };
        load(u);
        for (; u < end; u += W) {
          Reader<T, DP> rd = reader;
          rd.again();
          const int seen_from = again_vector(lane);
          landed<0>();
          RawCodes<Codes::kWords> raw[DT];
          kc.read(kl, seen_from, raw);
          in_order();
          f32x16 s = {};
          if constexpr (sizeof(T) == 4) {   // (as CacheSoftmax::scores)
            f32x16 z = {};
#pragma unroll
            for (int k = 0; k < KS; k += 2) {
              s = Mma<T>::mac(kc.frag(raw, k), q[k], s);
              z = Mma<T>::mac(kc.frag(raw, k + 1), q[k + 1], z);
            }
            s += z;
          } else {
#pragma unroll
            for (int k = 0; k < KS; ++k) s = Mma<T>::mac(kc.frag(raw, k), q[k], s);
          }
          vc.store(vt, vt, lane);
          const uint32_t gone = next;
          landed<0>();   // (read)
          load(min(u + W, last));
          Frag w[2];
          weigh(s, keys.start(u), gone, w);
          soft.values_ahead(rd, vt, w);
        }
        landed<0>();   // the last copies, of no use
      }
    }

    // the waves' sums, on the largest of their bases; wave k % W adds columns 32 k ..
    const float lw = half_sum(soft.l);
    if (threadIdx.x == 0) again = 0;
    if (lane < 32) {
      ml[wave][lane] = soft.m;
      ml[wave][32 + lane] = lw;
    }
    __syncthreads();   // (and every wave is through with its tiles)
    float m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) m = fmaxf(m, ml[w][r]);
    const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int w = 0; w < W; ++w) l += exp2f(ml[w][r] - base) * ml[w][32 + r];
    const float mine = exp2f(soft.m - base);
    constexpr int kSlots = W * kTile * (int)sizeof(T) / 4096;   // of 16 registers, in each buffer
    auto slot = [&](int k, int w) {   // of wave w's columns 32 k .., w not their owner
      const int i = k * (W - 1) + (w < k % W ? w : w - 1);
      return reinterpret_cast<float *>(i < kSlots ? kbuf : vbuf) + (i < kSlots ? i : i - kSlots) * 1024;
    };
    static_assert(DT * (W - 1) <= 2 * kSlots, "the waves' sums fit the buffers");
#pragma unroll
    for (int k = 0; k < DT; ++k) {
      soft.o[k] *= mine;
      if (k % W == wave) continue;
      float *to = slot(k, wave) + lane;
#pragma unroll
      for (int i = 0; i < 16; ++i) to[64 * i] = soft.o[k][i];
    }
    __syncthreads();
    float *part = ct.partial + ((int64_t)range.id * 2 + (u0 == 0)) * cache_part<kFewRows, DP>();
    const float inv = see.none ? 0.0f : 1.0f / l;
    bool bad = false;
    T *o = static_cast<T *>(p.out) + row * sh.out_stride[0] + h * sh.out_stride[1];
#pragma unroll
    for (int k = 0; k < DT; ++k) {
      if (k % W != wave) continue;
#pragma unroll
      for (int w = 0; w < W; ++w) {   // (this wave's own stands where it stands in the order of all)
        if (w == wave) continue;
        const float *x = slot(k, w) + lane;
#pragma unroll
        for (int i = 0; i < 16; ++i) soft.o[k][i] += x[64 * i];
      }
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int d = 32 * k + acc_row(i, lane >> 5);
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = soft.o[k][i + e];
        if (!complete) {
          __builtin_memcpy(__builtin_assume_aligned(part + r * DP + d, 16), y, 16);
          continue;
        }
        T x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          y[e] = see.none ? 0.0f : y[e] * inv;
          bad |= d + e < D && !(fabsf(y[e]) < INFINITY);
          x[e] = from_f32<T>(y[e]);
        }
        if (r >= rows) continue;
        if (ct.direct && d + 4 <= D) {
          __builtin_memcpy(__builtin_assume_aligned(o + d, 4), x, sizeof(x));
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (d + e < D) o[d + e] = x[e];
        }
      }
    }
    if (!complete) {
      if (wave == 0 && lane < 32) {
        part[kFewRows * DP + lane] = m;
        part[kFewRows * (DP + 1) + lane] = l;
      }
      if (threadIdx.x == 0) fresh().few.joins[2 * range.id + (u0 == 0)] = join_of(range, g, steps, 0, rows);
      __syncthreads();
      return;
    }
    if (p.lse && wave == 0 && lane < rows)
      p.lse[(int64_t)row * sh.Hq + h] = see.none ? -INFINITY : log_sum(m, l);
    const unsigned long long any = __ballot(bad && r < rows);
    if (kSumAgain && any && lane == 0) atomicOr(&again, (unsigned)(any | (any >> 32)));
    __syncthreads();
    // (see cache_tiles; the stores above come first, a row's by this workgroup alone)
    const unsigned redo = again;
    for (int x = wave; x < rows; x += W)
      if (redo >> x & 1) {
        const CacheCall &f = fresh();
        cache_attend_row<T, FORMAT>(f.c, f.sh, f.t, f.p, g.b, g.s, g.s.row + x / G, g.hk * G + x % G);
      }
    __syncthreads();
  });
}

// ---------------------------------------------------------------------------
// The kernels
// ---------------------------------------------------------------------------
template <class T, int DP, int FORMAT, bool ONE>
__global__ __launch_bounds__(64 * split_waves<T>(DP), split_waves<T>(DP) == 4 ? 2 : 1) void cache_few(const CacheCall) {
  constexpr int N = split_waves<T>(DP) * 32 * DP;
  __shared__ __align__(16) T buf0[N];
  __shared__ __align__(16) T buf1[N];
  __shared__ RangeScratch scratch;
  __shared__ FewScratch<T, DP> fs;
  DCONV_POISON(poison_lds(buf0, N); poison_lds(buf1, N));
  few_body<T, DP, FORMAT, ONE>(buf0, buf1, scratch, fs);
}

// Both kinds of sequences by the same workgroups, where they have as many waves: a
// share of the chunks, then one of the single tokens (16 sequences of both: 131 and
// 21 us apart, 144 together, and a launch less).
template <class T, int DP, int FORMAT, bool ONE>
__global__ __launch_bounds__(256, DP * sizeof(T) <= 256 ? 2 : 1) void cache_tiles(const CacheCall) {
  constexpr int N = 2 * forward_keys<T>(DP) * DP;
  __shared__ __align__(16) T buf0[N];
  __shared__ __align__(16) T buf1[N];
  __shared__ RangeScratch scratch;
  DCONV_POISON(poison_lds(buf0, N); poison_lds(buf1, N));
  tiles_body<T, DP, FORMAT, ONE>(buf0, buf1, scratch);
  if constexpr (split_waves<T>(DP) == 4) {
    __shared__ FewScratch<T, DP> fs;
    if (fresh().few.groups == 0) return;
    __syncthreads();   // the tiles are through with the buffers
    few_body<T, DP, FORMAT, ONE>(buf0, buf1, scratch, fs);
  }
}

// ---------------------------------------------------------------------------
// Parts joined
// ---------------------------------------------------------------------------
// A row by as many lanes as it has pieces of four floats (or a power of two), so that
// a wave joins several; and where parts are many beside the rows by eight waves, each
// every eighth part.  Four parts are on their way at a time: what it waits for is memory.  (Waves
// start at some 1.7 per nanosecond: a workgroup for every few rows of every workgroup's
// parts, most of which have nothing to do, took 30 us.)
constexpr int kJoinWaves = 8;
template <int DP>
struct JoinLds {
  float4 o[kJoinWaves][64];
  float ml[kJoinWaves][64][2];
};
template <int DP>
constexpr int join_lanes() { return DP <= 32 ? 8 : DP <= 64 ? 16 : DP <= 128 ? 32 : 64; }
template <class T, int DP, int FORMAT, int R>
__device__ __forceinline__ void join_rows(const dconv_cache &c, const dconv_cache_attend_shape &sh, const Batch &t,
                                          const CacheAttendPtrs &p, const CacheTile &ct, int id, JoinLds<DP> &lds) {
  const CacheJoin j = ct.joins[id];
  if (j.parts == 0) return;
  constexpr int L = join_lanes<DP>(), kRows = 64 / L;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), G = sh.Hq / c.Hkv, d = lane % L * 4;
  const int share = (j.rows + j.parts - 1) / j.parts;
  // the way with fewer loads one after another
  const bool in = d < DP, shared = (share + kRows - 1) / kRows * ((j.parts + 4 * kJoinWaves - 1) / (4 * kJoinWaves)) <
                                   (share + kJoinWaves * kRows - 1) / (kJoinWaves * kRows) * ((j.parts + 3) / 4);
  const int first = shared ? wave : 0, step = shared ? kJoinWaves : 1, rows = shared ? kRows : kJoinWaves * kRows;
  const int from = share * j.index, to = min(from + share, j.rows);
  for (int x0 = from; x0 < to; x0 += rows) {
    const int y = x0 + (shared ? 0 : wave * kRows) + lane / L, x = min(y, j.rows - 1);
    float m = -INFINITY, l = 0.0f;
    float4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int i0 = first; i0 < j.parts; i0 += 4 * step) {
      float pm[4], pl[4];
      float4 po[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        // the first part is its workgroup's second one
        const int i = min(i0 + k * step, j.parts - 1);
        const float *part = ct.partial + ((int64_t)(j.first + i) * 2 + (i == 0)) * cache_part<R, DP>();
        pm[k] = part[R * DP + x];
        pl[k] = part[R * (DP + 1) + x];
        po[k] = in ? *reinterpret_cast<const float4 *>(part + x * DP + d) : float4{};
      }
      float top = m;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (i0 + k * step >= j.parts) pm[k] = -INFINITY, po[k] = float4{}, pl[k] = 0.0f;
        top = fmaxf(top, pm[k]);
      }
      const float base = top == -INFINITY ? 0.0f : top, keep = exp2f(m - base);
      m = top;
      l *= keep;
      acc = {acc.x * keep, acc.y * keep, acc.z * keep, acc.w * keep};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float w = exp2f(pm[k] - base);
        l = fmaf(w, pl[k], l);
        acc = {fmaf(w, po[k].x, acc.x), fmaf(w, po[k].y, acc.y), fmaf(w, po[k].z, acc.z), fmaf(w, po[k].w, acc.w)};
      }
    }
    if (shared) {   // by the first wave, in the waves' order
      lds.o[wave][lane] = acc;
      lds.ml[wave][lane][0] = m;
      lds.ml[wave][lane][1] = l;
      __syncthreads();
      if (wave == 0) {
        const int n = min(j.parts, kJoinWaves);
        float top = -INFINITY;
        for (int w = 0; w < n; ++w) top = fmaxf(top, lds.ml[w][lane][0]);
        const float base = top == -INFINITY ? 0.0f : top;
        m = top;
        l = 0.0f;
        acc = float4{};
#pragma unroll 4
        for (int w = 0; w < n; ++w) {
          const float f = exp2f(lds.ml[w][lane][0] - base);
          const float4 o = lds.o[w][lane];
          l = fmaf(f, lds.ml[w][lane][1], l);
          acc = {fmaf(f, o.x, acc.x), fmaf(f, o.y, acc.y), fmaf(f, o.z, acc.z), fmaf(f, o.w, acc.w)};
        }
      }
      __syncthreads();
      if (wave > 0) continue;
    }
    const int r = j.r0 + x, row = j.s.row + r / G, h = j.hk * G + r % G;
    const bool none = keys_seen(sh, j.s.len, j.s.start() + r / G).none();
    const float sum[4] = {acc.x, acc.y, acc.z, acc.w};
    T out[4];
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float z = none ? 0.0f : sum[e] / l;
      bad |= y < to && d + e < c.D && !(fabsf(z) < INFINITY);
      out[e] = from_f32<T>(z);
    }
    const unsigned long long any = kSumAgain ? __ballot(bad) : 0ull;
    const bool redo = any >> (lane / L * L) & (L == 64 ? ~0ull : (1ull << (L & 63)) - 1);
    if (y < to && !redo) {
      T *o = static_cast<T *>(p.out) + row * sh.out_stride[0] + h * sh.out_stride[1];
      if (ct.direct && d + 4 <= c.D) {
        __builtin_memcpy(__builtin_assume_aligned(o + d, 4), out, sizeof(out));
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (d + e < c.D) o[d + e] = out[e];
      }
      if (p.lse && d == 0) p.lse[(int64_t)row * sh.Hq + h] = none ? -INFINITY : log_sum(m, l);
    }
    for (int k = 0; any && k < kRows; ++k) {   // (not finite: see cache_tiles)
      if (!(any >> (k * L) & (L == 64 ? ~0ull : (1ull << (L & 63)) - 1))) continue;
      const int z = j.r0 + x0 + (shared ? 0 : wave * kRows) + k;
      cache_attend_row<T, FORMAT>(c, sh, t, p, j.b, j.s, j.s.row + z / G, j.hk * G + z % G);
    }
  }
}

template <class T, int DP, int FORMAT>
__global__ __launch_bounds__(64 * kJoinWaves) void cache_join(const dconv_cache c, const dconv_cache_attend_shape sh,
                                                              const Batch t, const CacheAttendPtrs p, const CacheTile few,
                                                              const CacheTile tiles) {
  __shared__ JoinLds<DP> lds;
  for (int i = 0; i < 2; ++i) {
    if (!few.whole && (int)blockIdx.x < few.groups)
      join_rows<T, DP, FORMAT, kFewRows>(c, sh, t, p, few, 2 * blockIdx.x + i, lds);
    if (!tiles.whole && (int)blockIdx.x < tiles.groups)
      join_rows<T, DP, FORMAT, kTileRows>(c, sh, t, p, tiles, 2 * blockIdx.x + i, lds);
  }
}

template <class T, int FORMAT>
void launch_cache_attend(const dconv_cache &c, const dconv_cache_attend_shape &sh, const Batch &t,
                         const CacheAttendPtrs &p, const CachePlan &plan, char *workspace, hipStream_t s) {
  // (fp32's products last so long that it does not matter how a tile is found)
  constexpr bool kScalar = sizeof(T) == 2;
  const AttendTile scale = [&] {
    dconv_attend_shape a = {};
    a.scale = sh.scale;
    return attend_tile(a, false, false);
  }();
  CacheTile few = {scale.scale2, scale.sign, plan.direct, plan.pieces, plan.near, plan.few, plan.few_least,
                   plan.few_whole, nullptr, nullptr};
  CacheTile tiles = few;
  tiles.groups = plan.tiles;
  tiles.least = plan.tiles_least;
  tiles.whole = plan.tiles_whole;
  const int few_joins = plan.few_whole ? 0 : plan.few, tile_joins = plan.tiles_whole ? 0 : plan.tiles;
  few.joins = reinterpret_cast<CacheJoin *>(workspace);
  tiles.joins = few.joins + 2 * few_joins;
  few.partial = reinterpret_cast<float *>(workspace + plan.joins_bytes);
  by_width(plan.dp, [&](auto dp) {
    constexpr int DP = decltype(dp)::value;
    tiles.partial = few.partial + (int64_t)few_joins * 2 * cache_part<kFewRows, DP>();
    const CacheCall call = {c, sh, t, p, few, tiles};
    const bool together = plan.few > 0 && plan.tiles > 0 && split_waves<T>(DP) == 4;
    if (plan.few > 0 && !together) {
      const dim3 block(64 * split_waves<T>(DP));
      if (kScalar && plan.near && c.page_size % 32 == 0)
        hipLaunchKernelGGL((cache_few<T, DP, FORMAT, kScalar>), dim3(plan.few), block, 0, s, call);
      else
        hipLaunchKernelGGL((cache_few<T, DP, FORMAT, false>), dim3(plan.few), block, 0, s, call);
    }
    if (plan.tiles > 0) {
      CacheCall both = call;
      if (!together) both.few.groups = 0;
      if (kScalar && plan.near && c.page_size % forward_keys<T>(DP) == 0)
        hipLaunchKernelGGL((cache_tiles<T, DP, FORMAT, kScalar>), dim3(plan.tiles), dim3(256), 0, s, both);
      else
        hipLaunchKernelGGL((cache_tiles<T, DP, FORMAT, false>), dim3(plan.tiles), dim3(256), 0, s, both);
    }
    const int joins = few_joins > tile_joins ? few_joins : tile_joins;
    if (joins > 0)
      hipLaunchKernelGGL((cache_join<T, DP, FORMAT>), dim3(joins), dim3(64 * kJoinWaves), 0, s, c, sh, t, p, few, tiles);
  });
}

}  // namespace dconv

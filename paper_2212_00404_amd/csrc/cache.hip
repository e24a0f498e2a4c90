// Keys and values into a cache in pages and back (dconv_cache_write,
// dconv_cache_read): validation, kernels and launch.
#include <climits>

#include "cache.h"

#define DCONV_EXPORT extern "C" __attribute__((visibility("default")))

namespace dconv {
namespace {

constexpr int kPiece = 8;          // elements per thread and step
constexpr int kMostRows = 64;      // of a workgroup
constexpr int kNowhere = -1, kNoRow = -2;   // instead of a page

// How a workgroup's steps run over its rows: a row is its keys' pieces, then its
// values'; a head has `pieces` of them.
struct Walk {
  int rows, per_row;       // rows of a workgroup, pieces of a row
  FastDiv by_row, by_head; // per_row, pieces of a head
  long long k_stride[2], v_stride[2];
};

struct RowPtrs {
  void *k, *v;
};

template <class T>
struct __attribute__((packed, aligned(alignof(T)))) Piece {
  T x[kPiece];
};
template <int N>
struct __attribute__((packed, aligned(1))) Codes {
  uint32_t w[N];
};

// The first n elements of a piece (zeros past them).
template <class T>
__device__ __forceinline__ Piece<T> load_piece(const T *p, int n) {
  Piece<T> a;
  if (n == kPiece) return *reinterpret_cast<const Piece<T> *>(p);
#pragma unroll
  for (int e = 0; e < kPiece; ++e) a.x[e] = e < n ? p[e] : from_f32<T>(0.0f);
  return a;
}
template <class T>
__device__ __forceinline__ void store_piece(T *p, const Piece<T> &a, int n) {
  if (n == kPiece) {
    *reinterpret_cast<Piece<T> *>(p) = a;
    return;
  }
#pragma unroll
  for (int e = 0; e < kPiece; ++e)
    if (e < n) p[e] = a.x[e];
}

// Where piece c of the workgroup's is: in the rows, and in the cache.
struct Spot {
  int page, n;             // page or kNowhere, kNoRow; elements
  bool value;
  int64_t row, kept, scale;
};
__device__ __forceinline__ Spot spot_of(const dconv_cache &c, const Walk &w, const int2 *at, int r0, uint32_t x) {
  const uint32_t r = w.by_row.div(x), y = x - r * w.per_row;
  const uint32_t h2 = w.by_head.div(y), d = (y - h2 * w.by_head.d) * kPiece;
  Spot s;
  s.value = h2 >= (uint32_t)c.Hkv;
  const int h = (int)(s.value ? h2 - c.Hkv : h2);
  s.page = at[r].x;
  s.n = min(kPiece, c.D - (int)d);
  const long long *rs = s.value ? w.v_stride : w.k_stride, *ks = s.value ? c.v_stride : c.k_stride,
                  *ss = s.value ? c.v_scale_stride : c.k_scale_stride;
  const int page = max(s.page, 0);
  s.row = (int64_t)(r0 + r) * rs[0] + h * rs[1] + d;
  s.kept = place(ks, page, at[r].y, h);
  s.scale = c.format == DCONV_CACHE_PLAIN ? 0 : place(ss, page, at[r].y, h) + d / kBlock;
  s.kept += c.format == DCONV_CACHE_E2M1 ? d / 2 : d;
  return s;
}

// Pages and slots of a workgroup's rows, into LDS.  Offsets and lengths come there
// first, all at once: looked up one by one in memory they would be a chain of loads
// that miss (17 us for a call whose bytes take 1).
constexpr int kFewSequences = 512;
struct Lookup {
  int offsets[kFewSequences + 1], lengths[kFewSequences];
  int2 at[kMostRows];
  int falls[4];            // of each wave's part of the offsets
  int owner[kMostRows];
};

__device__ __forceinline__ void find_rows(const Batch &t, const CachePtrs &p, int r0, int rows, Lookup &lds) {
  static_assert(kMostRows == 64, "a row for each lane of the first wave");
  const int r = threadIdx.x;
  CachePtrs q = p;
  bool may_fall = p.offsets;   // (unless they are seen not to)
  if (p.offsets && t.B <= kFewSequences) {
    bool falls = false;
    for (int b = threadIdx.x; b <= t.B; b += 256) {
      lds.offsets[b] = p.offsets[b];
      if (b < t.B) {
        lds.lengths[b] = p.lengths[b];
        falls |= p.offsets[b + 1] < p.offsets[b];
      }
    }
    falls = __any(falls);
    if ((threadIdx.x & 63) == 0) lds.falls[threadIdx.x >> 6] = falls;
    __syncthreads();
    may_fall = (lds.falls[0] | lds.falls[1] | lds.falls[2] | lds.falls[3]) != 0;
    q.offsets = lds.offsets;
    q.lengths = lds.lengths;
  }
  int b = r < rows ? sequence_of(t, q, r0 + r) : 0;
  // A row that the bisection has not found is of no sequence, unless offsets fall: then
  // the first sequence that has it, if any.  (Offsets that do not come into LDS are
  // looked through by the workgroups that hold such rows, padding as a rule: 4096
  // sequences and 2048 rows of none take 7 us instead of 5.)
  if (may_fall) {
    if (r < kMostRows) lds.owner[r] = b < 0 ? t.B : -1;
    if (__syncthreads_or(b < 0)) {
#pragma unroll 4
      for (int x = threadIdx.x; x < t.B; x += 256) {
        const int from = max(q.offsets[x], r0), to = min(q.offsets[x + 1], r0 + rows);
        for (int row = from; row < to; ++row) atomicMin(&lds.owner[row - r0], x);
      }
      __syncthreads();
      if (b < 0 && lds.owner[r] < t.B) b = lds.owner[r];
    }
  }
  if (r < rows) {
    int2 s = {kNoRow, 0};
    if (b >= 0) {
      const Rows n = rows_of(t, q, b);
      const int i = n.start() + (r0 + r - n.row);
      s.x = i < 0 || i >= n.len ? kNowhere : page_of(t, p, b, i, &s.y);
    }
    lds.at[r] = s;
  }
  __syncthreads();
}

// Bits of the largest magnitude among the 32 neighbours that four lanes hold.
template <class T>
__device__ __forceinline__ uint32_t block_top(const Piece<T> &x) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < kPiece; ++e) m = max(m, __float_as_uint(to_f32(x.x[e])) & 0x7fffffffu);
  m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xf, 0xf, true));
  return max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xf, 0xf, true));
}

// The exponent of the smallest power of two, from 2^-127 on, that times M is not
// below the magnitude with bits `top`: that of top / M, one more where its mantissa
// is over M's (1.75, 1.5).
template <class T, int FORMAT>
__device__ __forceinline__ uint32_t scale_for(uint32_t top) {
  if (top >= 0x7f800000u) return 255;
  const int a = (int)min(top, __float_as_uint(limit<T, FORMAT>()));
  return max(0, FORMAT == DCONV_CACHE_E4M3 ? ((a + 0x1fffff) >> 23) - 8 : ((a + 0x3fffff) >> 23) - 2);
}

template <class T, int FORMAT>
__device__ __forceinline__ Codes<FORMAT == DCONV_CACHE_E4M3 ? 2 : 1> encode(const Piece<T> &x, uint32_t s) {
  constexpr float kLimit = limit<T, FORMAT>();
  const float scale = scale_of(s == 255 ? 254 : s);
  Codes<FORMAT == DCONV_CACHE_E4M3 ? 2 : 1> out;
  float y[kPiece];
#pragma unroll
  for (int e = 0; e < kPiece; ++e) y[e] = fminf(fmaxf(to_f32(x.x[e]), -kLimit), kLimit);
  if constexpr (FORMAT == DCONV_CACHE_E4M3) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      typedef short s16x2 __attribute__((ext_vector_type(2)));
      s16x2 w = {0, 0};
      w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, y[4 * i], y[4 * i + 1], scale, false);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, y[4 * i + 2], y[4 * i + 3], scale, true);
      __builtin_memcpy(&out.w[i], &w, 4);
    }
  } else {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], scale, 3);
    out.w[0] = w;
  }
  return out;
}

// A thread's pieces, a batch on their way at a time.
// (Writing gains nothing by it: a prompt of 61096 tokens, 8 heads of 128, bf16 into
// e4m3, 379 MB, takes 94 us by one at a time and 111 by four, which leave registers for
// five waves per SIMD; reading 65536 back takes 99 us by four and 103 by one.)
constexpr int kWriteBatch = 1, kReadBatch = 4;

template <class T, int FORMAT>
__global__ __launch_bounds__(256) void cache_write(const dconv_cache c, const Batch t, const CachePtrs p, const Walk w,
                                                   const RowPtrs from) {
  __shared__ Lookup lds;
  const int r0 = blockIdx.x * w.rows, rows = min(w.rows, t.N - r0), n = rows * w.per_row;
  find_rows(t, p, r0, rows, lds);
  for (int x0 = threadIdx.x; x0 < n; x0 += kWriteBatch * 256) {
    Spot s[kWriteBatch];
    Piece<T> a[kWriteBatch] = {};
#pragma unroll
    for (int i = 0; i < kWriteBatch; ++i) {
      s[i].page = kNoRow;
      if (x0 + i * 256 >= n) continue;
      s[i] = spot_of(c, w, lds.at, r0, (uint32_t)(x0 + i * 256));
      if (s[i].page < 0) continue;
      a[i] = load_piece(static_cast<const T *>(s[i].value ? from.v : from.k) + s[i].row, s[i].n);
    }
#pragma unroll
    for (int i = 0; i < kWriteBatch; ++i) {
      if (s[i].page < 0) continue;
      if constexpr (FORMAT == DCONV_CACHE_PLAIN) {
        store_piece(static_cast<T *>(s[i].value ? p.v : p.k) + s[i].kept, a[i], s[i].n);
      } else {
        const uint32_t scale = scale_for<T, FORMAT>(block_top(a[i]));
        const auto code = encode<T, FORMAT>(a[i], scale);
        *reinterpret_cast<decltype(encode<T, FORMAT>(a[i], scale)) *>(
            static_cast<uint8_t *>(s[i].value ? p.v : p.k) + s[i].kept) = code;
        if ((threadIdx.x & 3) == 0) (s[i].value ? p.v_scale : p.k_scale)[s[i].scale] = (uint8_t)scale;
      }
    }
  }
}

template <class T, int FORMAT>
__global__ __launch_bounds__(256) void cache_read(const dconv_cache c, const Batch t, const CachePtrs p, const Walk w,
                                                  const RowPtrs to) {
  constexpr bool kCodes = FORMAT != DCONV_CACHE_PLAIN;
  constexpr int kWords = FORMAT == DCONV_CACHE_E2M1 ? 1 : 2, kPairs = kCodes ? codes_per_word<FORMAT>() / 2 : 2;
  __shared__ Lookup lds;
  const int r0 = blockIdx.x * w.rows, rows = min(w.rows, t.N - r0), n = rows * w.per_row;
  find_rows(t, p, r0, rows, lds);
  for (int x0 = threadIdx.x; x0 < n; x0 += kReadBatch * 256) {
    Spot s[kReadBatch];
    Piece<T> a[kReadBatch] = {};
    Codes<kWords> code[kReadBatch];
    uint32_t scale[kReadBatch];
#pragma unroll
    for (int i = 0; i < kReadBatch; ++i) {
      s[i].page = kNoRow;
      if (x0 + i * 256 >= n) continue;
      s[i] = spot_of(c, w, lds.at, r0, (uint32_t)(x0 + i * 256));
      if (s[i].page < 0) continue;
      const void *kept = s[i].value ? p.v : p.k;
      if constexpr (kCodes) {
        code[i] = *reinterpret_cast<const Codes<kWords> *>(static_cast<const uint8_t *>(kept) + s[i].kept);
        scale[i] = (s[i].value ? p.v_scale : p.k_scale)[s[i].scale];
      } else {
        a[i] = load_piece(static_cast<const T *>(kept) + s[i].kept, s[i].n);
      }
    }
#pragma unroll
    for (int i = 0; i < kReadBatch; ++i) {
      if (s[i].page == kNoRow) continue;
      if constexpr (kCodes) {
        if (s[i].page >= 0) {
#pragma unroll
          for (int e = 0; e < kPiece / 2; ++e)
            decode_pair<T, FORMAT>(code[i].w[e / kPairs], e % kPairs, scale_of(scale[i]), a[i].x + 2 * e);
        }
      }
      store_piece(static_cast<T *>(s[i].value ? to.v : to.k) + s[i].row, a[i], s[i].n);
    }
  }
}

template <class F>
void by_type(int dtype, F f) {
  if (dtype == DCONV_F32) return f((float *)nullptr);
  if (dtype == DCONV_F16) return f((f16_t *)nullptr);
  return f((bf16_t *)nullptr);
}

int validate_rows(const dconv_cache &c, const dconv_cache_rows &r, const int *offsets) {
  const int rc = validate_cache(c);
  if (rc != DCONV_OK) return rc;
  if (r.B < 0 || r.N < 0 || r.table_width < 0 || !element_size(r.dtype)) return DCONV_EINVAL;
  if (c.format == DCONV_CACHE_PLAIN && c.dtype != r.dtype) return DCONV_EINVAL;
  if (!offsets && (r.B == 0 ? r.N > 0 : r.N % r.B != 0)) return DCONV_EINVAL;
  return batch_range(r.B, r.N, r.table_width, c.page_size);
}

// Rows per workgroup: some 2048 pieces, if there are workgroups enough.
Walk walk_of(const dconv_cache &c, const dconv_cache_rows &r) {
  Walk w;
  const int pieces = (c.D + kPiece - 1) / kPiece;
  w.per_row = 2 * c.Hkv * pieces;
  w.by_row = FastDiv((uint32_t)w.per_row);
  w.by_head = FastDiv((uint32_t)pieces);
  const int64_t want = (2048 + w.per_row - 1) / w.per_row, room = ((int64_t)r.N + 1023) / 1024;
  w.rows = (int)(want < room ? want : room);
  w.rows = w.rows < 1 ? 1 : w.rows > kMostRows ? kMostRows : w.rows;
  for (int i = 0; i < 2; ++i) {
    w.k_stride[i] = r.k_stride[i];
    w.v_stride[i] = r.v_stride[i];
  }
  return w;
}

template <bool WRITE>
int move(const dconv_cache *cache, const dconv_cache_rows *rows, const RowPtrs &kv, const CachePtrs &p, void *stream) {
  if (!cache || !rows) return DCONV_ENULL;
  const int rc = validate_rows(*cache, *rows, p.offsets);
  if (rc != DCONV_OK) return rc;
  if (rows->B == 0 || rows->N == 0) return DCONV_OK;
  if (!kv.k || !kv.v || !cache_pointers(*cache, p) || !p.lengths || (rows->table_width > 0 && !p.table))
    return DCONV_ENULL;
  const Batch t = batch_of(*cache, rows->B, rows->N, rows->table_width, rows->table_stride, p.offsets);
  const Walk w = walk_of(*cache, *rows);
  const unsigned grid = (unsigned)(((int64_t)rows->N + w.rows - 1) / w.rows);
  if (grid >= (1ll << 32) / 256) return DCONV_ERANGE;   // a launch has less than 2^32 threads
  (void)hipGetLastError();  // report this launch only
  by_type(rows->dtype, [&](auto *type) {
    using T = std::remove_pointer_t<decltype(type)>;
    by_format(cache->format, [&](auto format) {
      constexpr int FORMAT = decltype(format)::value;
      if constexpr (WRITE)
        hipLaunchKernelGGL((cache_write<T, FORMAT>), dim3(grid), dim3(256), 0, (hipStream_t)stream, *cache, t, p, w, kv);
      else
        hipLaunchKernelGGL((cache_read<T, FORMAT>), dim3(grid), dim3(256), 0, (hipStream_t)stream, *cache, t, p, w, kv);
    });
  });
  return hipGetLastError() == hipSuccess ? DCONV_OK : DCONV_EHIP;
}

}  // namespace

int validate_cache(const dconv_cache &c) {
  if (c.pages < 1 || c.page_size < 1 || c.Hkv < 1 || c.D < 1) return DCONV_EINVAL;
  if (c.format == DCONV_CACHE_PLAIN) {
    if (!element_size(c.dtype)) return DCONV_EINVAL;
  } else if (c.format != DCONV_CACHE_E4M3 && c.format != DCONV_CACHE_E2M1) {
    return DCONV_EINVAL;
  } else if (c.D % kBlock) {
    return DCONV_EUNSUPPORTED;
  }
  if (c.D > kMostHead) return DCONV_EUNSUPPORTED;
  // pieces of a workgroup's rows are counted in 32 bits
  return c.Hkv > kMostHeads ? DCONV_ERANGE : DCONV_OK;
}

bool cache_pointers(const dconv_cache &c, const CachePtrs &p) {
  return p.k && p.v && (c.format == DCONV_CACHE_PLAIN || (p.k_scale && p.v_scale));
}

int batch_range(int B, int N, int width, int page_size) {
  constexpr int64_t kMost = INT_MAX - 65536;
  return B > kMostSequences || N > kMost || (int64_t)width * page_size > kMost ? DCONV_ERANGE : DCONV_OK;
}

}  // namespace dconv

DCONV_EXPORT int dconv_cache_write(const dconv_cache *cache, const dconv_cache_rows *rows, const void *k,
                                   const void *v, void *cache_k, void *cache_v, void *k_scale, void *v_scale,
                                   const int *table, const int *lengths, const int *offsets, void *stream) {
  return dconv::move<true>(cache, rows, {const_cast<void *>(k), const_cast<void *>(v)},
                           {cache_k, cache_v, (uint8_t *)k_scale, (uint8_t *)v_scale, table, lengths, offsets}, stream);
}

DCONV_EXPORT int dconv_cache_read(const dconv_cache *cache, const dconv_cache_rows *rows, const void *cache_k,
                                  const void *cache_v, const void *k_scale, const void *v_scale, const int *table,
                                  const int *lengths, const int *offsets, void *k, void *v, void *stream) {
  return dconv::move<false>(cache, rows, {k, v},
                            {const_cast<void *>(cache_k), const_cast<void *>(cache_v), (uint8_t *)const_cast<void *>(k_scale),
                             (uint8_t *)const_cast<void *>(v_scale), table, lengths, offsets},
                            stream);
}

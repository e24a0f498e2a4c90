// Attention of new tokens over a cache in pages (dconv_cache_attend): validation
// and launch.
#include <climits>
#include <cmath>

#include "cache_attend.h"

#define DCONV_EXPORT extern "C" __attribute__((visibility("default")))

namespace dconv {
namespace {

// One wave per row and head, four per workgroup.
template <class T, int FORMAT>
__global__ __launch_bounds__(256) void cache_attend_rows(const dconv_cache c, const dconv_cache_attend_shape sh,
                                                         const Batch t, const CacheAttendPtrs p) {
  const int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i >= (int64_t)t.N * sh.Hq) return;
  const int row = (int)(i / sh.Hq), h = (int)(i % sh.Hq);
  const int b = sequence_of(t, p.cache, row);
  if (b < 0) return;
  const Rows s = rows_of(t, p.cache, b);
  if (sh.max_rows > 0 && s.n > sh.max_rows) return;
  cache_attend_row<T, FORMAT>(c, sh, t, p, b, s, row, h);
}

template <class F>
void by_type(int dtype, F f) {
  if (dtype == DCONV_F32) return f((float *)nullptr);
  if (dtype == DCONV_F16) return f((f16_t *)nullptr);
  return f((bf16_t *)nullptr);
}

int validate(const dconv_cache &c, const dconv_cache_attend_shape &sh) {
  const int rc = validate_cache(c);
  if (rc != DCONV_OK) return rc;
  if (sh.B < 0 || sh.N < 0 || sh.table_width < 0 || sh.Hq < 1 || sh.Hq % c.Hkv || sh.left < -1 || sh.right < -1 ||
      sh.sinks < 0 || sh.max_rows < 0 || !element_size(sh.dtype) || !std::isfinite(sh.scale))
    return DCONV_EINVAL;
  if (c.format == DCONV_CACHE_PLAIN && c.dtype != sh.dtype) return DCONV_EINVAL;
  if ((int64_t)sh.N * sh.Hq > INT_MAX - 65536) return DCONV_ERANGE;
  return batch_range(sh.B, sh.N, sh.table_width, c.page_size);
}

}  // namespace
}  // namespace dconv

DCONV_EXPORT int dconv_cache_attend_workspace(const dconv_cache *cache, const dconv_cache_attend_shape *shape,
                                              long long *bytes) {
  if (!cache || !shape || !bytes) return DCONV_ENULL;
  const int rc = dconv::validate(*cache, *shape);
  if (rc == DCONV_OK) *bytes = 0;
  return rc;
}

DCONV_EXPORT int dconv_cache_attend(const dconv_cache *cache, const dconv_cache_attend_shape *shape, const void *q,
                                    const void *cache_k, const void *cache_v, const void *k_scale,
                                    const void *v_scale, const int *table, const int *lengths, const int *offsets,
                                    void *out, float *lse, void *workspace, long long workspace_bytes, void *stream) {
  using namespace dconv;
  if (!cache || !shape) return DCONV_ENULL;
  const int rc = validate(*cache, *shape);
  if (rc != DCONV_OK) return rc;
  if (!offsets && (shape->B == 0 ? shape->N > 0 : shape->N % shape->B != 0)) return DCONV_EINVAL;
  if (shape->B == 0 || shape->N == 0) return DCONV_OK;
  CacheAttendPtrs p = {};
  p.cache = {const_cast<void *>(cache_k), const_cast<void *>(cache_v), (uint8_t *)const_cast<void *>(k_scale),
             (uint8_t *)const_cast<void *>(v_scale), table, lengths, offsets};
  p.q = q;
  p.out = out;
  p.lse = lse;
  if (!q || !out || !cache_pointers(*cache, p.cache) || !lengths || (shape->table_width > 0 && !table)) return DCONV_ENULL;
  const Batch t = batch_of(*cache, shape->B, shape->N, shape->table_width, shape->table_stride, offsets);
  const unsigned grid = (unsigned)(((int64_t)shape->N * shape->Hq + 3) / 4);
  (void)hipGetLastError();  // report this launch only
  by_type(shape->dtype, [&](auto *type) {
    using T = std::remove_pointer_t<decltype(type)>;
    by_format(cache->format, [&](auto format) {
      hipLaunchKernelGGL((cache_attend_rows<T, decltype(format)::value>), dim3(grid), dim3(256), 0,
                         (hipStream_t)stream, *cache, *shape, t, p);
    });
  });
  return hipGetLastError() == hipSuccess ? DCONV_OK : DCONV_EHIP;
}

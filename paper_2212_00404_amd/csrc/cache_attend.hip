// Attention of new tokens over a cache in pages (dconv_cache_attend): validation
// and launch.
#include <algorithm>
#include <climits>
#include <cmath>

#include "cache_attend.h"

#define DCONV_EXPORT extern "C" __attribute__((visibility("default")))

namespace dconv {
namespace {

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

// Rows in memory as whole 16-byte pieces on 4-byte boundaries.
bool whole_pieces(const void *p, int D, int es, std::initializer_list<long long> strides) {
  bool whole = D * es % 16 == 0 && (uintptr_t)p % 4 == 0;
  for (long long s : strides) whole = whole && s % (4 / es) == 0;
  return whole;
}

int padded_head(int D) { return D <= 32 ? 32 : D <= 64 ? 64 : D <= 96 ? 96 : D <= 128 ? 128 : 256; }

// `even`: every sequence has max_rows rows.
CachePlan plan_attend(const dconv_cache &c, const dconv_cache_attend_shape &sh, bool even) {
  CachePlan f = {};
  f.dp = padded_head(c.D);
  const int es = element_size(sh.dtype), G = sh.Hq / c.Hkv;
  const int64_t rows = (int64_t)(sh.max_rows > 0 ? sh.max_rows : sh.N) * G, heads = (int64_t)sh.B * c.Hkv;
  const int64_t keys = (int64_t)sh.table_width * c.page_size;
  // Two workgroups per compute unit, where LDS and registers hold them; no more than
  // there is work for.
  auto groups = [](int most, double work, int least) {   // (work may pass 64 bits)
    const double n = std::ceil(work / least);
    return n < 1 ? 1 : n < most ? (int)n : most;
  };
  // (fp32 takes sixteen times as long for the products of as many keys)
  f.few_least = es == 4 ? 128 : 256;
  f.tiles_least = es == 4 ? 96 : 512;
  const int whole = es == 4 ? 256 : 512;
  if (!even || rows <= 32) {
    f.few = groups(f.dp * es <= 256 ? 512 : 256, (double)heads * (double)(keys + 64), f.few_least);
    // tables of a few steps of a workgroup: nothing is divided, and nothing joined
    if (keys <= whole && heads < (1 << 20)) f.few_whole = 1, f.few = (int)heads;
  }
  if (rows > 32) {
    const int64_t tiles = ((int64_t)sh.N * G / 128 + sh.B) * c.Hkv;
    f.tiles = groups(f.dp * es <= 256 ? 512 : 256, (double)tiles * (double)(keys + 64), f.tiles_least);
    const int64_t each = (rows + 127) / 128;
    if (even && keys <= whole && heads * each < (1 << 20)) f.tiles_whole = (int)each, f.tiles = (int)(heads * each);
  }
  // one launch for both kinds (cache_tiles): as many workgroups, and shares of both
  if (f.few > 0 && f.tiles > 0 && f.dp * es <= 256) {
    f.few_whole = 0;
    f.few = f.tiles = std::max(std::min(f.few, 512), f.tiles);
  }
  const int64_t few = f.few_whole ? 0 : f.few, tiles = f.tiles_whole ? 0 : f.tiles;
  f.joins_bytes = ((few + tiles) * 2 * (int64_t)sizeof(CacheJoin) + 15) / 16 * 16;
  f.workspace = f.joins_bytes + (few * 32 + tiles * 128) * 2 * (f.dp + 2) * 4;
  return f;
}

int launch(const dconv_cache &c, const dconv_cache_attend_shape &sh, const Batch &t, const CacheAttendPtrs &p,
           CachePlan &plan, void *workspace, void *stream) {
  const int es = element_size(sh.dtype);
  plan.direct = whole_pieces(p.q, c.D, es, {sh.q_stride[0], sh.q_stride[1]}) &&
                whole_pieces(p.out, c.D, es, {sh.out_stride[0], sh.out_stride[1]});
  if (c.format == DCONV_CACHE_PLAIN) {
    plan.pieces = whole_pieces(p.cache.k, c.D, es, {c.k_stride[0], c.k_stride[1], c.k_stride[2]}) &&
                  whole_pieces(p.cache.v, c.D, es, {c.v_stride[0], c.v_stride[1], c.v_stride[2]});
  } else {
    plan.pieces = whole_pieces(p.cache.k, c.D, 1, {c.k_stride[0], c.k_stride[1], c.k_stride[2]});
  }
  // as many slots as a tile has keys (64) span less than 2^31 bytes
  plan.near = c.format != DCONV_CACHE_PLAIN || plan.pieces;
  const long long far = (1ll << 31) / (c.format == DCONV_CACHE_PLAIN ? es : 1) / 64 - c.D;
  for (long long s : {c.k_stride[1], c.v_stride[1], c.k_scale_stride[1], c.v_scale_stride[1]})
    plan.near = plan.near && s >= 0 && s < far;
  (void)hipGetLastError();  // report this launch only
  by_type(sh.dtype, [&](auto *type) {
    by_format(c.format, [&](auto format) {
      launch_cache_attend<std::remove_pointer_t<decltype(type)>, decltype(format)::value>(
          c, sh, t, p, plan, static_cast<char *>(workspace), (hipStream_t)stream);
    });
  });
  return hipGetLastError() == hipSuccess ? DCONV_OK : DCONV_EHIP;
}

}  // namespace
}  // namespace dconv

DCONV_EXPORT int dconv_cache_attend_workspace(const dconv_cache *cache, const dconv_cache_attend_shape *shape,
                                              long long *bytes) {
  if (!cache || !shape || !bytes) return DCONV_ENULL;
  const int rc = dconv::validate(*cache, *shape);
  if (rc == DCONV_OK) *bytes = shape->B == 0 || shape->N == 0 ? 0 : std::max(dconv::plan_attend(*cache, *shape, false).workspace,
                                        dconv::plan_attend(*cache, *shape, true).workspace);
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
  dconv_cache_attend_shape sh = *shape;
  if (!offsets) sh.max_rows = t.each;
  CachePlan plan = plan_attend(*cache, sh, !offsets);
  if (plan.workspace > 0 && !workspace) return DCONV_ENULL;
  if (workspace_bytes < plan.workspace) return DCONV_EWORKSPACE;
  if ((uintptr_t)workspace % 16 != 0) return DCONV_EINVAL;
  return launch(*cache, sh, t, p, plan, workspace, stream);
}

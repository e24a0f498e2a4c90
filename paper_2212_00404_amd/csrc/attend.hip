// Attention with a sliding window and first keys that stay visible
// (dconv_attend, dconv_attend_backward): validation and launch.
#include <climits>
#include <cmath>

#include "attend.h"

#define DCONV_EXPORT extern "C" __attribute__((visibility("default")))

namespace dconv {
namespace {

// One wave per row, four rows per workgroup.
template <class T, int KIND>
__global__ __launch_bounds__(256) void attend_rows(const dconv_attend_shape sh, const AttendPtrs p,
                                                   const int64_t n, const int heads, const int T_) {
  const int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i >= n) return;
  const int t = (int)(i % T_), h = (int)(i / T_ % heads), b = (int)(i / T_ / heads);
  if constexpr (KIND == 1) attend_row_dq<T>(sh, p, b, h, t);
  if constexpr (KIND == 2) attend_row_dkv<T>(sh, p, b, h, t);
}

template <class T, int KIND>
void rows(const dconv_attend_shape &sh, const AttendPtrs &p, hipStream_t s) {
  const int heads = KIND == 2 ? sh.Hkv : sh.Hq, len = KIND == 2 ? sh.Tk : sh.Tq;
  const int64_t n = (int64_t)sh.B * heads * len;
  if (n > 0)
    hipLaunchKernelGGL((attend_rows<T, KIND>), dim3((unsigned)((n + 3) / 4)), dim3(256), 0, s, sh, p,
                       n, heads, len);
}

template <class F>
void by_type(int dtype, F f) {
  if (dtype == DCONV_F32) return f((float *)nullptr);
  if (dtype == DCONV_F16) return f((f16_t *)nullptr);
  return f((bf16_t *)nullptr);
}

int validate(const dconv_attend_shape &sh) {
  if (sh.B < 0 || sh.Tq < 0 || sh.Tk < 0 || sh.Hq < 1 || sh.Hkv < 1 || sh.Hq % sh.Hkv || sh.D < 1 ||
      sh.left < -1 || sh.right < -1 || sh.sinks < 0 || !element_size(sh.dtype) ||
      !std::isfinite(sh.scale))
    return DCONV_EINVAL;
  if (sh.D > kAttendMaxD) return DCONV_EUNSUPPORTED;
  // rows of queries and of keys are counted in 32 bits, and walked by steps that end
  // past the last one: two strides of at most 32 (a tile) x 4 (waves) x 256 (parts)
  constexpr int kMost = INT_MAX - 2 * 32 * 4 * 256;
  if ((int64_t)sh.B * sh.Hq > INT_MAX / ((int64_t)(sh.Tq > sh.Tk ? sh.Tq : sh.Tk) + 1) || sh.Tk > kMost ||
      (int64_t)sh.Tq * (sh.Hq / sh.Hkv) > kMost)
    return DCONV_ERANGE;
  return DCONV_OK;
}

// Rows in memory as whole 16-byte pieces on 4-byte boundaries (what the copies
// into LDS need).
bool whole_pieces(const void *p, const long long *stride, const dconv_attend_shape &sh) {
  const int es = element_size(sh.dtype), unit = 4 / es;
  return sh.D * es % 16 == 0 && (uintptr_t)p % 4 == 0 && stride[0] % unit == 0 && stride[1] % unit == 0 &&
         stride[2] % unit == 0;
}

// Whether as many rows as a tile has at most (256, of queries) span less than 2^31
// bytes, as rows of one head and as the heads of a group.
bool close_rows(const long long *stride, const dconv_attend_shape &sh) {
  const long long most = (1ll << 31) / element_size(sh.dtype) / 512 / (sh.Hq / sh.Hkv) - sh.D;
  return stride[1] >= 0 && stride[2] >= 0 && stride[1] < most && stride[2] < most;
}

int padded_head(int D) { return D <= 32 ? 32 : D <= 64 ? 64 : D <= 96 ? 96 : D <= 128 ? 128 : 256; }

// The most keys that a tile of `queries` queries sees (lengths are on the device).
int64_t most_keys(const dconv_attend_shape &sh, int queries) {
  int64_t n = sh.Tk;
  if (sh.left >= 0 && sh.right >= 0) {
    const int64_t window = (int64_t)sh.left + sh.right + queries + sh.sinks;
    if (window < n) n = window;
  }
  return n;
}

ForwardPlan plan_forward(const dconv_attend_shape &sh) {
  ForwardPlan f = {};
  f.dp = padded_head(sh.D);
  const int64_t rows = (int64_t)sh.Tq * (sh.Hq / sh.Hkv), heads = (int64_t)sh.B * sh.Hkv;
  // Keys divided over waves and workgroups: up to 32 rows, of which 128-row tiles
  // would be mostly empty (16 sequences x 8 key heads x 32 rows, 4096 keys: 52 us
  // against 85); and long walks of keys by few workgroups (32 workgroups of 128
  // rows over 4096 keys: 35 us against 82).  Shorter walks, or more workgroups, lose
  // more by the second launch than they gain (112 workgroups over 226 keys: 16
  // against 10.5; 64 over 543 keys: 16.7 against 14).
  f.few = rows <= 32 || (heads * ((rows + 31) / 32) <= 128 && most_keys(sh, 128) >= 1024);
  f.tiles = (int)(f.few ? (rows + 31) / 32 : (rows + 127) / 128);
  f.splits = 1;
  if (f.few) {
    const int waves = f.dp * element_size(sh.dtype) <= 256 ? 4 : f.dp * element_size(sh.dtype) <= 512 ? 2 : 1;
    const int64_t groups = heads * f.tiles, room = (256 + groups - 1) / groups;
    const int64_t tiles = (most_keys(sh, 32) + 32 * waves - 1) / (32 * waves);
    f.splits = (int)(room < tiles ? room : tiles);
    if (f.splits < 1) f.splits = 1;
    if (f.splits > 1) f.workspace = groups * f.splits * attend_part_floats(f.dp) * 4;
  }
  return f;
}

// A launch has less than 2^32 threads.
bool launchable(int64_t workgroups, int threads) { return workgroups < (1ll << 32) / threads; }

int forward_range(const dconv_attend_shape &sh) {
  const int64_t rows = (int64_t)sh.Tq * (sh.Hq / sh.Hkv), heads = (int64_t)sh.B * sh.Hkv;
  return launchable(heads * ((rows + 31) / 32), 256) ? DCONV_OK : DCONV_ERANGE;
}

int64_t forward_workspace(const dconv_attend_shape &sh) {
  return sh.B == 0 || sh.Tq == 0 ? 0 : plan_forward(sh).workspace;
}
BackwardPlan plan_backward(const dconv_attend_shape &sh) {
  BackwardPlan f = {};
  f.dp = padded_head(sh.D);
  const int G = sh.Hq / sh.Hkv;
  const int64_t rows = (int64_t)sh.Tq * G, heads = (int64_t)sh.B * sh.Hkv;
  f.row_tiles = (int)((rows + 127) / 128);
  // 128 keys per workgroup where that gives every compute unit one (256 workgroups:
  // 116 us the whole gradient, against 129 with 64 keys each); else 64 where that
  // does; else 32, by four or eight row groups (128 workgroups of 64 keys: 61 us
  // against 72, 72 of them: 72 against 83).  Larger heads have LDS for two row groups
  // only and gain nothing by it (58 us against 52).
  if (heads * ((sh.Tk + 127) / 128) >= 256)
    f.key_groups = 4;
  else
    f.key_groups = heads * ((sh.Tk + 63) / 64) >= 256 || f.dp * element_size(sh.dtype) > 256 ? 2 : 1;
  f.key_tiles = (sh.Tk + 32 * f.key_groups - 1) / (32 * f.key_groups);
  // the keys that every query sees, where that is more than twice what another tile
  // of keys is seen by
  const int64_t window = sh.left < 0 || sh.right < 0 ? sh.Tq : (int64_t)sh.left + sh.right + 32 * f.key_groups;
  f.first = sh.Tq <= 2 * window ? 0 : sh.sinks < sh.Tk ? sh.sinks : sh.Tk;
  f.first_tiles = (f.first + 31) / 32;
  f.parts = 1;
  if (f.first > 0) {
    const int64_t groups = heads * f.first_tiles, room = (256 + groups - 1) / groups;
    const int64_t tiles = (rows + 127) / 128;   // 32 rows for each of four waves
    f.parts = (int)(room < tiles ? room : tiles);
    if (f.parts < 1) f.parts = 1;
  }
  f.stats_bytes = (heads * rows * 8 + 15) / 16 * 16;
  f.workspace = f.stats_bytes + (f.first > 0 ? heads * f.first_tiles * f.parts * 64 * f.dp * 4 : 0);
  return f;
}

int backward_range(const dconv_attend_shape &sh) {
  const int64_t heads = (int64_t)sh.B * sh.Hkv;
  if (sh.D > kGradMaxD)   // attend_rows: a wave per row
    return launchable((int64_t)sh.B * sh.Hq * sh.Tq, 64) && launchable(heads * sh.Tk, 64) ? DCONV_OK : DCONV_ERANGE;
  const BackwardPlan f = plan_backward(sh);
  return launchable(heads * f.row_tiles, 256) && launchable(heads * f.key_tiles, 512) &&
                 launchable(heads * f.first, 256) && launchable(heads * f.first_tiles * f.parts, 256)
             ? DCONV_OK
             : DCONV_ERANGE;
}

int64_t backward_workspace(const dconv_attend_shape &sh) {
  return sh.B == 0 || sh.D > kGradMaxD ? 0 : plan_backward(sh).workspace;
}

}  // namespace
}  // namespace dconv

DCONV_EXPORT int dconv_attend_workspace(const dconv_attend_shape *shape, long long *bytes) {
  if (!shape || !bytes) return DCONV_ENULL;
  int rc = dconv::validate(*shape);
  if (rc == DCONV_OK) rc = dconv::forward_range(*shape);
  if (rc == DCONV_OK) *bytes = dconv::forward_workspace(*shape);
  return rc;
}

DCONV_EXPORT int dconv_attend_backward_workspace(const dconv_attend_shape *shape, long long *bytes) {
  if (!shape || !bytes) return DCONV_ENULL;
  int rc = dconv::validate(*shape);
  if (rc == DCONV_OK) rc = dconv::backward_range(*shape);
  if (rc == DCONV_OK) *bytes = dconv::backward_workspace(*shape);
  return rc;
}

DCONV_EXPORT int dconv_attend(const dconv_attend_shape *shape, const void *q, const void *k,
                              const void *v, const int *lengths, const int *starts, void *out,
                              float *lse, void *workspace, long long workspace_bytes, void *stream) {
  using namespace dconv;
  if (!shape) return DCONV_ENULL;
  int rc = validate(*shape);
  if (rc == DCONV_OK) rc = forward_range(*shape);
  if (rc != DCONV_OK) return rc;
  if (shape->B == 0 || shape->Tq == 0) return DCONV_OK;
  if (!q || !out || (shape->Tk > 0 && (!k || !v))) return DCONV_ENULL;
  const int64_t need = forward_workspace(*shape);
  if (need > 0 && !workspace) return DCONV_ENULL;
  if (workspace_bytes < need) return DCONV_EWORKSPACE;
  if (need > 0 && (uintptr_t)workspace % 16 != 0) return DCONV_EINVAL;
  AttendPtrs p = {};
  p.q = q;
  p.k = k;
  p.v = v;
  p.lengths = lengths;
  p.starts = starts;
  p.o = out;
  p.lse_out = lse;
  ForwardPlan plan = plan_forward(*shape);
  plan.direct = whole_pieces(q, shape->q_stride, *shape) && whole_pieces(k, shape->k_stride, *shape) &&
                whole_pieces(v, shape->v_stride, *shape) && whole_pieces(out, shape->out_stride, *shape);
  plan.near = plan.direct && close_rows(shape->k_stride, *shape) && close_rows(shape->v_stride, *shape);
  (void)hipGetLastError();  // report this launch only
  by_type(shape->dtype, [&](auto *t) {
    launch_attend<std::remove_pointer_t<decltype(t)>>(*shape, p, plan, (float *)workspace, (hipStream_t)stream);
  });
  return hipGetLastError() == hipSuccess ? DCONV_OK : DCONV_EHIP;
}

DCONV_EXPORT int dconv_attend_backward(const dconv_attend_shape *shape, const void *dout,
                                       const void *q, const void *k, const void *v, const void *out,
                                       const float *lse, const int *lengths, const int *starts,
                                       void *dq, void *dk, void *dv, void *workspace,
                                       long long workspace_bytes, void *stream) {
  using namespace dconv;
  if (!shape) return DCONV_ENULL;
  int rc = validate(*shape);
  if (rc == DCONV_OK) rc = backward_range(*shape);
  if (rc != DCONV_OK) return rc;
  if (shape->B == 0) return DCONV_OK;
  if (shape->Tq > 0 && (!dout || !q || !out || !lse || !dq)) return DCONV_ENULL;
  if (shape->Tk > 0 && (!k || !v || !dk || !dv)) return DCONV_ENULL;
  const int64_t need = backward_workspace(*shape);
  if (need > 0 && !workspace) return DCONV_ENULL;
  if (workspace_bytes < need) return DCONV_EWORKSPACE;
  if (need > 0 && (uintptr_t)workspace % 16 != 0) return DCONV_EINVAL;
  AttendPtrs p = {};
  p.q = q;
  p.k = k;
  p.v = v;
  p.out = out;
  p.dout = dout;
  p.lse = lse;
  p.lengths = lengths;
  p.starts = starts;
  p.dq = dq;
  p.dk = dk;
  p.dv = dv;
  BackwardPlan plan = plan_backward(*shape);
  const int64_t flat = (int64_t)shape->D;
  const long long dense[3] = {flat, flat, flat};
  plan.direct = whole_pieces(q, shape->q_stride, *shape) && whole_pieces(k, shape->k_stride, *shape) &&
                whole_pieces(v, shape->v_stride, *shape) && whole_pieces(out, shape->out_stride, *shape) &&
                whole_pieces(dout, shape->dout_stride, *shape) && whole_pieces(dq, dense, *shape) &&
                whole_pieces(dk, dense, *shape) && whole_pieces(dv, dense, *shape);
  plan.near = plan.direct && close_rows(shape->q_stride, *shape) && close_rows(shape->k_stride, *shape) &&
              close_rows(shape->v_stride, *shape) && close_rows(shape->dout_stride, *shape);
  (void)hipGetLastError();  // report this launch only
  by_type(shape->dtype, [&](auto *t) {
    using T = std::remove_pointer_t<decltype(t)>;
    if (shape->D <= kGradMaxD) {
      launch_attend_grad<T>(*shape, p, plan, workspace, (hipStream_t)stream);
      return;
    }
    // larger heads: keys, values and both gradients of a tile do not fit the
    // registers of a wave
    rows<T, 1>(*shape, p, (hipStream_t)stream);
    rows<T, 2>(*shape, p, (hipStream_t)stream);
  });
  return hipGetLastError() == hipSuccess ? DCONV_OK : DCONV_EHIP;
}

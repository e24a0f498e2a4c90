// From a block's output to the next block's input (dconv_join): the norm after
// the block, its gate and scales, the residual sum and the norm before the
// next block, and the gradients.
#include <climits>

#include "internal.h"
#include "join.h"
#include "tokens.h"

#define DCONV_EXPORT extern "C" __attribute__((visibility("default")))

namespace dconv {
namespace {

constexpr int kMaxD = 16384;

template <class T, class W>
hipError_t run(const dconv_join_shape &sh, const JoinPtrs &p, const JoinPlan &plan, void *workspace, bool backward,
               hipStream_t s) {
  (void)hipGetLastError();  // report these launches only
  launch_join<T, W>(sh, p, plan, (float *)workspace, backward, s);
  return hipGetLastError();
}
int run(const dconv_join_shape &sh, const JoinPtrs &p, const JoinPlan &plan, void *workspace, bool backward,
        void *stream) {
  const hipStream_t s = (hipStream_t)stream;
  const bool wide = sh.vector_dtype == DCONV_F32;
  hipError_t e;
  if (sh.dtype == DCONV_F32)
    e = run<float, float>(sh, p, plan, workspace, backward, s);
  else if (sh.dtype == DCONV_F16)
    e = wide ? run<f16_t, float>(sh, p, plan, workspace, backward, s)
             : run<f16_t, f16_t>(sh, p, plan, workspace, backward, s);
  else
    e = wide ? run<bf16_t, float>(sh, p, plan, workspace, backward, s)
             : run<bf16_t, bf16_t>(sh, p, plan, workspace, backward, s);
  return e == hipSuccess ? DCONV_OK : DCONV_EHIP;
}

int validate(const dconv_join_shape &sh) {
  if (sh.B < 0 || sh.T < 0 || sh.D < 1 || !element_size(sh.dtype) ||
      (sh.vector_dtype != DCONV_F32 && sh.vector_dtype != sh.dtype) ||
      (sh.norm != DCONV_NORM_RMS && sh.norm != DCONV_NORM_LAYER) || (sh.post & ~1) ||
      (sh.per_sample & ~15) || !(sh.eps >= 0.0f))
    return DCONV_EINVAL;
  if (sh.D > kMaxD || (int64_t)sh.B * sh.T > INT_MAX) return DCONV_ERANGE;
  // a launch has less than 2^32 threads, a run per sequence at least, of up to 1024
  if (sh.per_sample && sh.B >= 1 << 22) return DCONV_ERANGE;
  return DCONV_OK;
}

// The rows of a call and how they are divided.  Eight elements per thread where
// a workgroup's threads reach that far, else 16.
JoinPlan plan_join(const dconv_join_shape &sh, bool backward) {
  JoinPlan f = {};
  f.tpr = 16;
  f.ept = 8;
  while (f.tpr * f.ept < sh.D) {
    if (f.ept == 8) {
      f.ept = 16;
    } else {
      f.tpr *= 4;
      f.ept = 8;
    }
  }
  // Runs end where a vector changes.
  f.segments = sh.per_sample ? sh.B : 1;
  f.rows = (int)(sh.per_sample ? sh.T : (int64_t)sh.B * sh.T);
  // Threads enough to fill the chip once.  (The backward kernel's registers leave
  // room for 768 threads per compute unit, 512 with 16 elements each; one more
  // workgroup than that and the last ones run alone.)
  const int64_t groups = 256 * (!backward ? 2048 : f.tpr > 256 ? 1024 : f.ept == 8 ? 768 : 512) / f.tpr;
  int64_t runs = f.segments > 0 ? groups / f.segments : 1;
  if (runs > f.rows) runs = f.rows;
  if (runs < 1) runs = 1;
  f.run_rows = (int)((f.rows + runs - 1) / runs);
  if (f.run_rows < 1) f.run_rows = 1;
  f.runs = (int)(((int64_t)f.rows + f.run_rows - 1) / f.run_rows);
  if (f.runs < 1) f.runs = 1;
  return f;
}

int64_t workspace_bytes_of(const dconv_join_shape &sh) {
  const JoinPlan f = plan_join(sh, true);
  return f.runs == 1 && f.segments <= 1 ? 0 : (int64_t)f.segments * f.runs * sh.D * 4 * 4;
}

// Whether every row and vector is whole 16-byte pieces.
struct Alignment {
  bool ok = true;
  void need(const void *p) { ok = ok && (uintptr_t)p % 16 == 0; }
  void rows(const void *p, const long long *stride, int es) {
    if (!p) return;
    need(p);
    ok = ok && stride[0] * es % 16 == 0 && stride[1] * es % 16 == 0;
  }
};
bool whole_pieces(const dconv_join_shape &sh, const JoinPtrs &p) {
  const int es = element_size(sh.dtype);
  Alignment a;
  a.ok = sh.D * es % 16 == 0;
  a.rows(p.branch, sh.branch_stride, es);
  a.rows(p.x, sh.x_stride, es);
  a.rows(p.dh, sh.dh_stride, es);
  a.rows(p.dy, sh.dy_stride, es);
  for (const void *v : {p.post_weight, p.gate, p.pre_weight, p.pre_bias, (const void *)p.dpost_weight,
                        (const void *)p.dgate, (const void *)p.dpre_weight, (const void *)p.dpre_bias})
    a.need(v);
  for (const void *v : {(const void *)p.h, (const void *)p.y, (const void *)p.dbranch, (const void *)p.dx}) a.need(v);
  return a.ok;
}

}  // namespace
}  // namespace dconv

DCONV_EXPORT int dconv_join(const dconv_join_shape *shape, const void *branch, const void *x,
                            const void *post_weight, const void *gate, const void *pre_weight,
                            const void *pre_bias, void *h, void *y, float *stats, void *stream) {
  using namespace dconv;
  if (!shape) return DCONV_ENULL;
  const int rc = validate(*shape);
  if (rc != DCONV_OK) return rc;
  if ((int64_t)shape->B * shape->T == 0) return DCONV_OK;
  if (!x || (branch && !h) || (!h && !y)) return DCONV_ENULL;
  JoinPtrs p = {};
  p.branch = branch;
  p.x = x;
  p.post_weight = post_weight;
  p.gate = gate;
  p.pre_weight = pre_weight;
  p.pre_bias = pre_bias;
  p.h = h;
  p.y = y;
  p.stats = stats;
  if (stats && (uintptr_t)stats % 16 != 0) return DCONV_EINVAL;
  JoinPlan plan = plan_join(*shape, false);
  plan.whole = whole_pieces(*shape, p);
  return run(*shape, p, plan, nullptr, false, stream);
}

DCONV_EXPORT int dconv_join_workspace(const dconv_join_shape *shape, long long *bytes) {
  if (!shape || !bytes) return DCONV_ENULL;
  const int rc = dconv::validate(*shape);
  if (rc == DCONV_OK) *bytes = dconv::workspace_bytes_of(*shape);
  return rc;
}

DCONV_EXPORT int dconv_join_backward(const dconv_join_shape *shape, const void *dh, const void *dy,
                                     const void *branch, const void *x, const void *post_weight,
                                     const void *gate, const void *pre_weight, const float *stats,
                                     void *dbranch, void *dx, void *dpost_weight, void *dgate,
                                     void *dpre_weight, void *dpre_bias, void *workspace,
                                     long long workspace_bytes, void *stream) {
  using namespace dconv;
  if (!shape) return DCONV_ENULL;
  const int rc = validate(*shape);
  if (rc != DCONV_OK) return rc;
  const bool none = (int64_t)shape->B * shape->T == 0;
  if (!none && (branch == nullptr) != (dbranch == nullptr)) return DCONV_ENULL;
  if ((!none && !branch && (dgate || dpost_weight)) || (!shape->post && dpost_weight))
    return DCONV_EINVAL;
  if ((dpost_weight && !post_weight) || (dgate && !gate) || (dpre_weight && !pre_weight))
    return DCONV_ENULL;
  // (without rows too: the sums of none of them are left there)
  const int64_t need = workspace_bytes_of(*shape);
  if ((!none && (!x || !stats || !dx)) || (need > 0 && !workspace)) return DCONV_ENULL;
  if (workspace_bytes < need) return DCONV_EWORKSPACE;
  if (need > 0 && (uintptr_t)workspace % 16 != 0) return DCONV_EINVAL;
  JoinPtrs p = {};
  p.branch = branch;
  p.x = x;
  p.post_weight = post_weight;
  p.gate = gate;
  p.pre_weight = pre_weight;
  p.dh = dh;
  p.dy = dy;
  p.stats = const_cast<float *>(stats);
  p.dbranch = dbranch;
  p.dx = dx;
  p.dpost_weight = dpost_weight;
  p.dgate = dgate;
  p.dpre_weight = dpre_weight;
  p.dpre_bias = dpre_bias;
  if (stats && (uintptr_t)stats % 16 != 0) return DCONV_EINVAL;
  JoinPlan plan = plan_join(*shape, true);
  plan.whole = whole_pieces(*shape, p);
  return run(*shape, p, plan, workspace, true, stream);
}

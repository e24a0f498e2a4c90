// Declarations shared by dconv_join's host side (join.hip) and its kernels.
#pragma once

#include <hip/hip_runtime.h>

#include "dconv.h"

namespace dconv {

struct JoinPtrs {
  const void *branch, *x, *post_weight, *gate, *pre_weight, *pre_bias;
  const void *dh, *dy;
  void *h, *y;
  float *stats;
  void *dbranch, *dx, *dpost_weight, *dgate, *dpre_weight, *dpre_bias;
};

// How a call runs: `tpr` threads per row with `ept` elements each, 16 bytes at a
// time (`whole`: on 16-byte boundaries, without a remainder); the rows as `segments` of `rows`, each walked in
// `runs` of `run_rows`.
struct JoinPlan {
  bool whole;
  int tpr, ept;
  int segments, rows, runs, run_rows;
};

// Instantiated in join_f32.hip, join_f16.hip and join_bf16.hip.
template <class T, class W>
void launch_join(const dconv_join_shape &sh, const JoinPtrs &p, const JoinPlan &plan, float *workspace, bool backward,
                 hipStream_t s);

}  // namespace dconv

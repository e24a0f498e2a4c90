// The matrix-core kernels of windowed attention for one type.
#include "attend_mma.h"

namespace dconv {
template void launch_attend<f16_t>(const dconv_attend_shape &, const AttendPtrs &, const ForwardPlan &, float *,
                                     hipStream_t);
}  // namespace dconv

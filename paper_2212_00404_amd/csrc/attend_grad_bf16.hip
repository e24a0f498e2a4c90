// The matrix-core kernels of windowed attention's gradient for one type.
#include "attend_grad.h"

namespace dconv {
template void launch_attend_grad<bf16_t>(const dconv_attend_shape &, const AttendPtrs &, const BackwardPlan &, void *,
                                           hipStream_t);
}  // namespace dconv

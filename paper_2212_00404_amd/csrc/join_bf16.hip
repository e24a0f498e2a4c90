// The kernels of dconv_join for one type.
#include "join_kernels.h"

namespace dconv {
template void launch_join<bf16_t, float>(const dconv_join_shape &, const JoinPtrs &, const JoinPlan &, float *, bool, hipStream_t);
template void launch_join<bf16_t, bf16_t>(const dconv_join_shape &, const JoinPtrs &, const JoinPlan &, float *, bool, hipStream_t);
}  // namespace dconv

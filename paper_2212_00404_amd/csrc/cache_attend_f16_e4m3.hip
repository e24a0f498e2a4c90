// Attention over a cache in pages for one type and one format.
#include "cache_mma.h"

namespace dconv {
template void launch_cache_attend<f16_t, DCONV_CACHE_E4M3>(const dconv_cache &, const dconv_cache_attend_shape &, const Batch &,
                                          const CacheAttendPtrs &, const CachePlan &, char *, hipStream_t);
}  // namespace dconv

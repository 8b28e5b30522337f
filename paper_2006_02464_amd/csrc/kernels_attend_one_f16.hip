// Attention of one new token over a paged cache, queries in fp16.
#include <algorithm>

#include "attend_one_body.h"

namespace cw {

hipError_t launch_attend_one_f16(const AttendOneArgs &a, hipStream_t s) {
    return a.cache.dtype == DT_E4M3 ? launch_attend_one_typed<f16, true>(a, s) : launch_attend_one_typed<f16, false>(a, s);
}

}  // namespace cw

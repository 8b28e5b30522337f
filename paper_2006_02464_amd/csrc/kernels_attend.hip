// Attention of packed prompts (cw_attend has the definition): which kernel takes it.
#include "attend_common.h"

namespace cw {

hipError_t launch_attend_f16(const AttendArgs &a, hipStream_t s);
hipError_t launch_attend_bf16(const AttendArgs &a, hipStream_t s);

bool attend_fits(const AttendArgs &a) {   // rows and workgroups are counted in 31 bits
    return (int64_t)a.tokens * a.heads + (int64_t)a.sequences * a.kv_heads <= INT32_MAX && attend_workgroups(a) * 64 * kAttendWaves <= kMostThreads;
}

hipError_t launch_attend(const AttendArgs &a, hipStream_t s) { return a.dtype == DT_F16 ? launch_attend_f16(a, s) : launch_attend_bf16(a, s); }

}  // namespace cw

// Attention of one new token over a paged cache (cw_attend_one has the definition): which kernel takes it.
#include "attend_common.h"

namespace cw {

hipError_t launch_attend_one_f16(const AttendOneArgs &a, hipStream_t s);
hipError_t launch_attend_one_bf16(const AttendOneArgs &a, hipStream_t s);

size_t attend_one_workspace_bytes() { return (size_t)32 << 20; }

// Where there are so many items, none is in parts.
bool attend_one_fits(const AttendOneArgs &a) {
    const OneForm f = one_form(a);
    return f.items * 64 * (f.wave_each ? 1 : kOneWaves) <= kMostThreads;
}

hipError_t launch_attend_one(const AttendOneArgs &a, hipStream_t s) { return a.dtype == DT_F16 ? launch_attend_one_f16(a, s) : launch_attend_one_bf16(a, s); }

}  // namespace cw

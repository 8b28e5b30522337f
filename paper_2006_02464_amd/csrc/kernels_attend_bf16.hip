// Attention of packed prompts in bf16.
#include "attend_body.h"

namespace cw {

hipError_t launch_attend_bf16(const AttendArgs &a, hipStream_t s) { return launch_attend_typed<bf16>(a, s); }

}  // namespace cw

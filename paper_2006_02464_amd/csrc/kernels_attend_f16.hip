// Attention of packed prompts in fp16.
#include "attend_body.h"

namespace cw {

hipError_t launch_attend_f16(const AttendArgs &a, hipStream_t s) { return launch_attend_typed<f16>(a, s); }

}  // namespace cw

#include "fc4_body.h"

namespace cw {

template hipError_t launch_fc4_x<X_PLAIN>(const Fc4Args &, const Fc4Plan &, hipStream_t);

}  // namespace cw

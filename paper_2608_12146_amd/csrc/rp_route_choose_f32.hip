// The router's choices on logits of type float.
#include "rp_route_choose.h"

namespace rp {

int choose_f32(const RouteArgs &a, hipStream_t stream) { return choose<float>(a, stream); }

}  // namespace rp

// The router's choices on logits of type _Float16.
#include "rp_route_choose.h"

namespace rp {

int choose_f16(const RouteArgs &a, hipStream_t stream) { return choose<_Float16>(a, stream); }

}  // namespace rp

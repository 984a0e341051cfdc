// The router's choices on logits of type __bf16.
#include "rp_route_choose.h"

namespace rp {

int choose_bf16(const RouteArgs &a, hipStream_t stream) { return choose<__bf16>(a, stream); }

}  // namespace rp

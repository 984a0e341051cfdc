// The gradient for logits of type __bf16.
#include "rp_route_back.h"

namespace rp {

int back_bf16(const BackArgs &a, hipStream_t stream) { return route_back<__bf16>(a, stream); }

}  // namespace rp

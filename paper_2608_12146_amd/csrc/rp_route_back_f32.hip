// The gradient for logits of type float.
#include "rp_route_back.h"

namespace rp {

int back_f32(const BackArgs &a, hipStream_t stream) { return route_back<float>(a, stream); }

}  // namespace rp

// The gradient for logits of type _Float16.
#include "rp_route_back.h"

namespace rp {

int back_f16(const BackArgs &a, hipStream_t stream) { return route_back<_Float16>(a, stream); }

}  // namespace rp

// The router's choices among groups of experts, for logits of one type (rp_route_groups.h).
#include "rp_route_groups.h"

namespace rp {
int choose_groups_f16(const GroupArgs &a, hipStream_t stream) { return choose_groups<_Float16>(a, stream); }
}  // namespace rp

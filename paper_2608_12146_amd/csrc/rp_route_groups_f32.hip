// The router's choices among groups of experts, for logits of one type (rp_route_groups.h).
#include "rp_route_groups.h"

namespace rp {
int choose_groups_f32(const GroupArgs &a, hipStream_t stream) { return choose_groups<float>(a, stream); }
}  // namespace rp

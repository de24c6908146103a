// The router's kernels for many pixels, bf16 logits (sr_route_lanes.h).
#include "sr_route_lanes.h"

namespace srd {
SR_ROUTE_LANES(bf16raw)
}  // namespace srd

// The router's kernels for many pixels, f32 logits (sr_route_lanes.h).
#include "sr_route_lanes.h"

namespace srd {
SR_ROUTE_LANES(float)
}  // namespace srd

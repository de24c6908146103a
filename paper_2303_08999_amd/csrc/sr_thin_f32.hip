// The layers' kernels for many rows and a small weight, f32 (sr_thin.h, sr_thin_grad.h).
#include <type_traits>

#include "sr_thin_grad.h"

namespace srd {
template hipError_t launch_thin<float>(const GemmArgs&, int, hipStream_t);
template hipError_t launch_thin_grad<float>(const ThinGradArgs&, bool, int, hipStream_t);
}  // namespace srd

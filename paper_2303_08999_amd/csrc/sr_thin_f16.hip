// The layers' kernels for many rows and a small weight, f16 (sr_thin.h, sr_thin_grad.h).
#include <type_traits>

#include "sr_thin_grad.h"

namespace srd {
template hipError_t launch_thin<__half>(const GemmArgs&, int, hipStream_t);
template hipError_t launch_thin_grad<__half>(const ThinGradArgs&, bool, int, hipStream_t);
}  // namespace srd

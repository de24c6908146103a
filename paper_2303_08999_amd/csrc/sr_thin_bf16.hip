// The layers' kernels for many rows and a small weight, bf16 (sr_thin.h, sr_thin_grad.h).
#include <type_traits>

#include "sr_thin_grad.h"

namespace srd {
template hipError_t launch_thin<bf16raw>(const GemmArgs&, int, hipStream_t);
template hipError_t launch_thin_grad<bf16raw>(const ThinGradArgs&, bool, int, hipStream_t);
}  // namespace srd

// The layers' products, f32 (sr_gemm.h).
#include <type_traits>

#include "sr_gemm_kernel.h"
#include "sr_skinny.h"

namespace srd {
template hipError_t launch_gemm<float>(const GemmArgs&, int, bool, int, hipStream_t);
template hipError_t launch_pack<float>(const void*, int64_t, int, void*, hipStream_t);
template hipError_t launch_skinny<float>(const GemmArgs&, bool, hipStream_t);
template hipError_t launch_gemm_finish<float>(const GemmArgs&, hipStream_t);
}  // namespace srd

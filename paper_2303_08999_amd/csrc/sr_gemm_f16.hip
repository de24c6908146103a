// The layers' products, f16 (sr_gemm.h).
#include <type_traits>

#include "sr_gemm_kernel.h"
#include "sr_skinny.h"

namespace srd {
template hipError_t launch_gemm<__half>(const GemmArgs&, int, bool, int, hipStream_t);
template hipError_t launch_pack<__half>(const void*, int64_t, int, void*, hipStream_t);
template hipError_t launch_skinny<__half>(const GemmArgs&, bool, hipStream_t);
template hipError_t launch_gemm_finish<__half>(const GemmArgs&, hipStream_t);
}  // namespace srd

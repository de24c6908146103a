// The layers' products, bf16 (sr_gemm.h).
#include <type_traits>

#include "sr_gemm_kernel.h"
#include "sr_skinny.h"

namespace srd {
template hipError_t launch_gemm<bf16raw>(const GemmArgs&, int, bool, int, hipStream_t);
template hipError_t launch_pack<bf16raw>(const void*, int64_t, int, void*, hipStream_t);
template hipError_t launch_skinny<bf16raw>(const GemmArgs&, bool, hipStream_t);
template hipError_t launch_gemm_finish<bf16raw>(const GemmArgs&, hipStream_t);
}  // namespace srd

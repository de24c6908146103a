// Gradient of the list form on the matrix cores, f16 values (sr_list_grad_mfma.h).
#include "sr_list_grad_mfma.h"

namespace srd {
template <> hipError_t launch_list_grad_mfma<__half>(const ListGradArgs& a, int k, int grid, hipStream_t st) {
    return k == 3 ? grad_mfma_k<3, __half>(a, grid, st) : k == 5 ? grad_mfma_k<5, __half>(a, grid, st) : grad_mfma_k<7, __half>(a, grid, st);
}
}  // namespace srd

// Gradient of the list form on the matrix cores, f32 values (sr_list_grad_mfma.h).
#include "sr_list_grad_mfma.h"

namespace srd {
template <> hipError_t launch_list_grad_mfma<float>(const ListGradArgs& a, int k, int grid, hipStream_t st) {
    return k == 3 ? grad_mfma_k<3, float>(a, grid, st) : k == 5 ? grad_mfma_k<5, float>(a, grid, st) : grad_mfma_k<7, float>(a, grid, st);
}
}  // namespace srd

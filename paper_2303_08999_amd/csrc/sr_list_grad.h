// Arguments of the list gradient's kernels (sr_list_grad.hip, sr_list_grad_mfma.h).
#pragma once
#include <stdint.h>

#include "sr_launch.h"
#include "../../include/sr_route.h"

namespace srd {

struct ListGradArgs {
    const void* lr;                  // [N][C][h][w]
    const unsigned char* index;      // [N][T][H][W]
    const void* value;               // [N][T][H][W]
    const float* dict;               // [L][k][k]
    const unsigned char* mask;       // [N][H][W] or null
    const void* dout;                // [N][C][H][W]
    void* dvalue;                    // [N][T][H][W] or null
    double* partial;                 // [workgroups][L][k][k], or null: no gradient of the dictionary
    int N, C, h, w, H, W, s, L, T;
    int io_f16;                      // lr and dout are fp16
    int tiles_x, tiles_y;
    int64_t tiles;
};

constexpr int GRAD_RECORDS = 512;            // workgroups of a call that writes ddict, at most

// Matrix-core kernel: which calls it takes, and the launch (grid: workgroups).
constexpr int GM_TW = 64, GM_TH = 8;         // its tile
bool list_grad_mfma_supported(const ListGradArgs& a, int k);
template <typename TV> hipError_t launch_list_grad_mfma(const ListGradArgs& a, int k, int grid, hipStream_t st);

}  // namespace srd

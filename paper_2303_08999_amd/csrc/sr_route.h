// What the router's kernels share (include/sr_route.h): arguments, where a pixel's logits are, order of logits, narrowing.
#pragma once
#include <stdint.h>

#include "sr_launch.h"
#include "../../include/sr_route.h"

namespace srd {

struct RouteArgs {
    const void* z;                  // logits, any of three orders
    const unsigned char* mask;      // [N][H][W] or null
    unsigned char* index;           // [N][T][H][W]; read by the gradient
    void* value;                    // [N][T][H][W]; the gradient's dvalue (may be null there)
    const long long* counts;        // gradient: L + 1, or null
    const float* dloss;
    void* dz;
    void* partial;                  // balance: records of sums, one a workgroup
    int64_t px, total;              // pixels of an image, of the call
    int64_t lstride;                // from one atom of a pixel to the next, in elements
    int L, T, kind, layout;
    int H, W, h, w, s;              // h, w, s: the order before the pixel-shuffle only
    int records;
};

// Sums of one workgroup (balance): share[L] and counts[L], then lse^2 and M.
struct RouteRecord {
    double* share; unsigned long long* counts; double* squares; unsigned long long* live;
    __host__ __device__ RouteRecord(void* base, int L, int r) {
        share = (double*)base + (size_t)r * (2 * L + 2);
        counts = (unsigned long long*)(share + L);
        squares = (double*)(counts + L);
        live = (unsigned long long*)(squares + 1);
    }
};
constexpr int ROUTE_RECORDS = 1024;      // workgroups of a balance call, at most

// Element offset of atom 0 of pixel i of image n.
__device__ __forceinline__ int64_t logit_base(const RouteArgs& a, int64_t n, int64_t i) {
    if (a.layout == SR_COEFF_PIXEL_MAJOR) return (n * a.px + i) * a.L;
    if (a.layout == SR_COEFF_PLANAR) return n * a.L * a.px + i;
    const int64_t Y = i / a.W;
    const int X = (int)(i - Y * a.W), y = (int)(Y / a.s), x = X / a.s;
    const int sub = (int)(Y - (int64_t)y * a.s) * a.s + (X - x * a.s);
    const int64_t hw = (int64_t)a.h * a.w;
    return (n * a.L * a.s * a.s + sub) * hw + (int64_t)y * a.w + x;
}

// Order-preserving map of logits to unsigned integers: larger logits to larger integers, -0 and +0 to the same one.
__device__ __forceinline__ unsigned logit_order(float z) {
    const unsigned b = __float_as_uint(z + 0.0f);
    return b ^ ((unsigned)((int)b >> 31) | 0x80000000u);
}

__device__ __forceinline__ float logit_log(float s) { return __builtin_amdgcn_logf(s) * 0.693147180559945309417f; }

// One rounding, to the nearest even, from the fp32 value as it is.
__device__ __forceinline__ void st_from_float(bf16raw* p, size_t i, float v) {
    const __bf16 r = (__bf16)v;
    __builtin_memcpy(p + i, &r, 2);
}

// Wavefront sums with a fixed order.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}

// exp(z - m), m the pixel's largest logit, from what exp_origin makes of m.  fp16 logits: one multiply-add, whose rounding
// of m's part is the same for all of a pixel's atoms and cancels (up to 65504 LOG2E 2^-24 = 0.006 in the exponent); the
// other types reach 3e38, where that part would overflow: subtracted first.  A masked logit gives 0, also in a pixel of
// none but masked ones (origin 0).
template <typename TZ> __device__ __forceinline__ float exp_origin(float m) { return m == -INFINITY ? 0.0f : m; }
template <> __device__ __forceinline__ float exp_origin<__half>(float m) { return m == -INFINITY ? 0.0f : logit_shift(m); }
template <typename TZ> __device__ __forceinline__ float exp_from(float z, float o) { return __builtin_amdgcn_exp2f((z - o) * LOG2E); }
template <> __device__ __forceinline__ float exp_from<__half>(float z, float o) { return logit_exp(z, o); }

}  // namespace srd

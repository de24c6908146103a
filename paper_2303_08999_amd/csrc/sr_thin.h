// Products of many rows with a small weight (sr_gemm.h): a pixel's layer of few features, bound by the rows' way through memory.
//
// The weight, turned so that k runs fastest and filled up with zeros, and the bias stay in LDS for the whole launch.  A wavefront takes 32 (or 16)
// rows at a time, loaded straight into the matrix instructions' operands while those before are worked on, and leaves what it made of
// them in LDS as the piece of the output that it is: rows without gaps, stored 16 bytes a lane whatever a row's length is.  Wavefronts wait for
// nobody.  72 outputs of 64 features for the 8.3 million pixels of a 4K frame, fp16: 470 us would be the speed of a copy; the tile kernel takes 654.
#pragma once
#include "sr_gemm.h"

namespace srd {
namespace {

// wavefronts that a SIMD's registers hold
template <int KS, bool GATED> constexpr int thin_waves = KS <= 2 && !GATED ? 4 : 3;

// Bytes of LDS: weight rows (each half filled up to np of them), bias, and a piece of the output for each wavefront
template <typename T> size_t thin_lds(int np, int halves, int steps, int width, int waves, int rows) {
    return (size_t)np * halves * (steps * 64 + 16) + (size_t)np * halves * 4 + (size_t)waves * ((rows * width * sizeof(T) + 15) / 16 * 16);
}

// four values of a row
template <typename T> __device__ __forceinline__ void thin_get4(const T* p, int count, float e[4]) {
    using u32x2u = __attribute__((ext_vector_type(2), aligned(2))) unsigned;
    if (count >= 4) {
        if constexpr (sizeof(T) == 4) {
            const u32x4u v = *(const u32x4u*)p;
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = __uint_as_float(v[i]);
        } else {
            const u32x2u v = *(const u32x2u*)p;
            if constexpr (__is_same(T, __half)) {
                using half4g = __attribute__((ext_vector_type(4))) _Float16;
                using u32x2g = __attribute__((ext_vector_type(2))) unsigned;
                const half4g h = __builtin_bit_cast(half4g, (u32x2g)v);
#pragma unroll
                for (int i = 0; i < 4; ++i) e[i] = (float)h[i];
            } else {
#pragma unroll
                for (int i = 0; i < 2; ++i) e[2 * i] = __uint_as_float(v[i] << 16), e[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) e[i] = i < count ? gm_get(p + i) : 0.0f;
    }
}
// ... into the piece of the output; count: of them there
template <typename T, bool FOURS> __device__ __forceinline__ void thin_put4(T* p, int count, const float v[4]) {
    if constexpr (FOURS) {                                 // rows are multiples of four values: all four are there, or none, and aligned
        if (count <= 0) return;
        if constexpr (sizeof(T) == 4) {
            *(f32x4g*)p = f32x4g{v[0], v[1], v[2], v[3]};
        } else if constexpr (__is_same(T, __half)) {
            using half4g = __attribute__((ext_vector_type(4))) _Float16;
            *(half4g*)p = half4g{(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3]};
        } else {
            using bf4g = __attribute__((ext_vector_type(4))) __bf16;
            *(bf4g*)p = bf4g{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < count) gm_put(p + i, v[i]);
    }
}

// KS steps of 64 bytes of k.  NG tiles of 16 columns at a time, of each half.
template <typename T, int KS, int NG, int RF, bool GATED, bool FOURS>
__global__ __launch_bounds__(256, (thin_waves<KS, GATED>)) void k_thin(const GemmArgs g, const int rc, const int np) {
    constexpr int E = 16 / sizeof(T), H = GATED ? 2 : 1, SB = KS * 64 + 16, THIN_ROWS = 16 * RF, U = (NG * RF + 1) / 2;
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    float* const bias = (float*)(lds + (size_t)np * H * SB);
    const int width = g.n;
    const int patch_bytes = (THIN_ROWS * width * (int)sizeof(T) + 15) / 16 * 16;
    T* const patch = (T*)(lds + (size_t)np * H * (SB + 4) + wave * patch_bytes);

    if (rc) {                                              // [k][n] in memory
        for (int i = threadIdx.x; i < np * KS * 4 * E; i += blockDim.x) {
            const int k = i / np, n = i - k * np;
            T v;
            __builtin_memset(&v, 0, sizeof v);
            if (k < g.k && n < g.n) v = ((const T*)g.b)[(int64_t)k * g.ldb + n];
            *(T*)(lds + n * SB + k * (int)sizeof(T)) = v;
        }
    } else {
        for (int i = threadIdx.x; i < np * H * KS * 4; i += blockDim.x) {
            const int row = i / (KS * 4), p = i - row * (KS * 4), h = row >= np, n = h ? row - np : row;
            *(u32x4g*)(lds + row * SB + p * 16) = gm_piece((const T*)g.b + (int64_t)(n + h * g.half) * g.ldb + p * E, n < g.n ? g.k - p * E : 0);
        }
    }
    for (int i = threadIdx.x; i < np * H; i += blockDim.x) {
        const int h = i >= np, n = h ? i - np : i;
        bias[i] = g.bias && n < g.n ? gm_get((const T*)g.bias + n + h * g.half) : 0.0f;
    }
    __syncthreads();

    const int r = lane % 16, q = lane / 16;
    const int64_t end = (int64_t)g.m * g.lda;              // elements of A
    const int blocks = (g.m + THIN_ROWS - 1) / THIN_ROWS, step = gridDim.x * waves;
    u32x4g now[RF][KS], next[RF][KS];
    auto load = [&](int block, u32x4g (&v)[RF][KS]) {
#pragma unroll
        for (int f = 0; f < RF; ++f) {
            const int row = block * THIN_ROWS + f * 16 + r;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const int k = (s * 4 + q) * E;
                const int64_t at = (int64_t)row * g.lda + k;
                // a whole piece wherever one is, though the next row may begin in it; what is not this row's becomes zero
                const bool in = row < g.m && k < g.k;
                if (in && at + E <= end) v[f][s] = *(const u32x4u*)((const T*)g.a + at);
                else v[f][s] = gm_piece((const T*)g.a + at, in ? g.k - k : 0);
            }
        }
    };
    auto cut = [&](u32x4g (&v)[RF][KS]) {
        if (g.k == KS * 4 * E) return;
#pragma unroll
        for (int f = 0; f < RF; ++f)
#pragma unroll
            for (int s = 0; s < KS; ++s) v[f][s] = gm_cut<T>(v[f][s], g.k - (s * 4 + q) * E);
    };
    // What is added comes as the piece that the output leaves as, and through the same place in LDS.
    int block = blockIdx.x * waves + wave;
    if (block < blocks) load(block, next);
    for (; block < blocks; block += step) {
#pragma unroll
        for (int f = 0; f < RF; ++f)
#pragma unroll
            for (int s = 0; s < KS; ++s) now[f][s] = next[f][s];
        cut(now);
        if (block + step < blocks) load(block + step, next);
        const int row0 = block * THIN_ROWS, rows = g.m - row0 < THIN_ROWS ? g.m - row0 : THIN_ROWS, count = rows * width;
        if (g.extra) {
            const T* const in = (const T*)g.extra + (int64_t)row0 * width;
            for (int i = lane * E; i < count; i += 4 * 64 * E) {
                u32x4g v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = gm_piece(in + i + j * 64 * E, count - i - j * 64 * E);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (i + j * 64 * E < count) *(u32x4g*)(patch + i + j * 64 * E) = v[j];
            }
            __builtin_amdgcn_wave_barrier();
        }
        for (int n0 = 0; n0 < g.n; n0 += NG * 16) {
            // [NG][RF][4 columns] as rows of 8
            float z[U][8], u[U][8], e[U][8];
            if constexpr (NG * RF == 1) {
#pragma unroll
                for (int i = 4; i < 8; ++i) z[0][i] = u[0][i] = e[0][i] = 0.0f;
            }
#pragma unroll
            for (int j = 0; j < NG; ++j)
#pragma unroll
                for (int f = 0; f < RF; ++f) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) e[(j * RF + f) / 2][(j * RF + f) % 2 * 4 + i] = 0.0f;
                    const int n = n0 + j * 16 + q * 4;
                    if (g.extra && n < g.n) thin_get4(patch + (f * 16 + r) * width + n, g.n - n, e[(j * RF + f) / 2] + (j * RF + f) % 2 * 4);
                }
            f32x4g acc[H][NG][RF];
#pragma unroll
            for (int h = 0; h < H; ++h)
#pragma unroll
                for (int j = 0; j < NG; ++j)
#pragma unroll
                    for (int f = 0; f < RF; ++f) acc[h][j][f] = *(const f32x4g*)(bias + h * np + n0 + j * 16 + q * 4);
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int h = 0; h < H; ++h)
#pragma unroll
                    for (int j = 0; j < NG; ++j) {
                        const u32x4g b = *(const u32x4g*)(lds + (h * np + n0 + j * 16 + r) * SB + (s * 4 + q) * 16);
#pragma unroll
                        for (int f = 0; f < RF; ++f) gm_mul<T, 16>(acc[h][j][f], b, now[f][s]);
                    }
#pragma unroll
            for (int j = 0; j < NG; ++j)
#pragma unroll
                for (int f = 0; f < RF; ++f)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        z[(j * RF + f) / 2][(j * RF + f) % 2 * 4 + i] = acc[0][j][f][i];
                        if constexpr (GATED) u[(j * RF + f) / 2][(j * RF + f) % 2 * 4 + i] = acc[H - 1][j][f][i];
                    }
            gm_forward<GATED, U>(g.act, z, u, e);
#pragma unroll
            for (int j = 0; j < NG; ++j)
#pragma unroll
                for (int f = 0; f < RF; ++f) {
                    const int n = n0 + j * 16 + q * 4;
                    T* const p = patch + (f * 16 + r) * width + n;
                    thin_put4<T, FOURS>(p, g.n - n, z[(j * RF + f) / 2] + (j * RF + f) % 2 * 4);
                }
        }
        __builtin_amdgcn_wave_barrier();
        T* const out = (T*)g.out + (int64_t)row0 * width;
        for (int i = lane * E; i < count; i += 64 * E) {
            if (i + E <= count) {
                *(u32x4u*)(out + i) = *(const u32x4g*)(patch + i);
            } else {
                for (int j = i; j < count; ++j) out[j] = patch[j];
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

template <typename T, int KS, int NG, int RF, bool GATED>
hipError_t start_thin(const GemmArgs& g, bool rc, int np, int waves, size_t lds, hipStream_t st) {
    const int64_t blocks = ((int64_t)g.m + 16 * RF - 1) / (16 * RF), groups = (blocks + waves - 1) / waves;
    // as many workgroups as the compute units hold at once, by LDS and by registers
    int per = (int)((160 * 1024) / lds);
    if (per * waves > 4 * thin_waves<KS, GATED>) per = 4 * thin_waves<KS, GATED> / waves;
    const int64_t most = (int64_t)per * 256;
    const int grid = (int)(groups < most ? groups : most);
    if (g.n % 4 == 0) k_thin<T, KS, NG, RF, GATED, true><<<grid, waves * 64, lds, st>>>(g, rc, np);
    else k_thin<T, KS, NG, RF, GATED, false><<<grid, waves * 64, lds, st>>>(g, rc, np);
    return hipGetLastError();
}

}  // namespace

template <typename T>
hipError_t launch_thin(const GemmArgs& g, int layout, hipStream_t st) {
    const bool gated = g.mode == GEMM_GATED;
    const ThinShape s = thin_shape(g.n, g.k, sizeof(T), gated);
    if (!s.waves || !(gated || g.mode == GEMM_STORE)) return hipErrorInvalidValue;
    const size_t lds = thin_lds<T>(s.np, gated ? 2 : 1, s.steps, g.n, s.waves, s.rows);
    const bool rc = layout == GEMM_KC_RC;
    auto go = [&](auto ks) {
        constexpr int KS = decltype(ks)::value;
        auto start = [&](auto ng, auto rf) {
            constexpr int NG = decltype(ng)::value, RF = decltype(rf)::value;
            return gated ? start_thin<T, KS, NG, RF, true>(g, rc, s.np, s.waves, lds, st) : start_thin<T, KS, NG, RF, false>(g, rc, s.np, s.waves, lds, st);
        };
        constexpr std::integral_constant<int, 1> one{};
        constexpr std::integral_constant<int, 2> two{};
        if (s.rows == 16) return s.group == 1 ? start(one, one) : start(two, one);
        return s.group == 1 ? start(one, two) : start(two, two);
    };
    switch (s.steps) {
    case 1: return go(std::integral_constant<int, 1>{});
    case 2: return go(std::integral_constant<int, 2>{});
    case 3: return go(std::integral_constant<int, 3>{});
    default: return go(std::integral_constant<int, 4>{});
    }
}

}  // namespace srd

// The gradient of a small layer under many rows in one pass over them (sr_layer.hip): x and dy are read once, dx is written once, dz is never
// stored, and what the rows add to dW and db stays in registers until a workgroup has no more of them.
//
// A workgroup takes 64 rows at a time, loaded while the 64 before are worked on.  Its four wavefronts make dz = dy act'(z) and dx = dz W of 16
// rows each from LDS, then share out the 16 x 16 tiles of dW, whose operands the LDS reads turn as in sr_gemm.h.  The
// weight stays in LDS, both ways round where z is made anew.  Bound by the rows' way through memory: 2 C + O values a row, where separate products
// read dz twice and x once or twice more (1080p, 72 of 64 bfloat16: 829 MB).
#pragma once
#include "sr_gemm_kernel.h"
#include "sr_thin.h"

namespace srd {
namespace {

constexpr int TG_ROWS = 64;

// 16 columns from `col` of a tile in LDS whose rows are k: the fragment of one matrix step, 64 / sizeof(T) of them
template <typename T> __device__ __forceinline__ u32x4g turned_frag(const char* tile, int stride, int step, int col, int lane) {
    if constexpr (sizeof(T) == 2) {
        const int g = lane / 16, i = lane % 16;
        const char* p = tile + (step * 32 + 8 * g + i / 4) * stride + (col + i % 4 * 4) * 2;
        using u2 = __attribute__((ext_vector_type(2))) unsigned;
        const u2 a = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4g*)p));
        const u2 b = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4g*)(p + 4 * stride)));
        return u32x4g{a[0], a[1], b[0], b[1]};
    } else {
        const char* p = tile + (step * 16 + lane / 16 * 4) * stride + (col + lane % 16) * 4;
        u32x4g v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = *(const unsigned*)(p + j * stride);
        return v;
    }
}

// NT: tiles of 16 of C; MW: tiles of 16 of dz's columns a wavefront has; Z: z is made anew
template <typename T, int NT, int MW, bool GATED, bool Z>
__global__ __launch_bounds__(256, 2) void k_thin_grad(const ThinGradArgs a) {
    constexpr int E = 16 / sizeof(T), ES = sizeof(T), KM = 64 / ES, RS = TG_ROWS / KM;
    constexpr int NX = (TG_ROWS * NT * 16 / E + 255) / 256, ND = (TG_ROWS * MW * 64 / (GATED ? 2 : 1) / E + 255) / 256;
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane % 16, q = lane / 16;
    const int wide = GATED ? 2 * a.o : a.o;
    const ThinGradShape s = thin_grad_shape(a.c, a.o, ES, GATED, Z);
    char* const wt = lds;                                  // [c][wide]
    char* const wz = lds + s.wz;                           // [wide][c]
    char* const dz = lds + s.dz;                           // [row][wide]; dy first where there is no gate
    // 16-bit types: what dz's rounding left off, for all three sums (2^-17 and better instead of 2^-9, fp16 2^-12)
    constexpr bool LO = Z && sizeof(T) == 2;
    char* const dl = lds + s.lo;
    char* const xs = lds + s.x;                            // [row][c]
    char* const dys = lds + (GATED ? s.dy : s.dz);         // [row][o]
    float* const bias = (float*)(lds + s.bias);
    const int dy_stride = GATED ? s.dy_stride : s.dz_stride;

    // What is no value of the tiles stays zero: their rows' ends are never written again.
    for (int i = threadIdx.x; i < s.bytes / 16; i += 256) ((u32x4g*)lds)[i] = u32x4g{0, 0, 0, 0};
    __syncthreads();
    for (int i = threadIdx.x; i < wide * a.c; i += 256) {
        const int o = i / a.c, c = i - o * a.c;
        const T v = ((const T*)a.w)[i];
        *(T*)(wt + c * s.dz_stride + o * ES) = v;
        if constexpr (Z) *(T*)(wz + o * s.x_stride + c * ES) = v;
    }
    if (Z && a.bias)
        for (int i = threadIdx.x; i < wide; i += 256) bias[i] = gm_get((const T*)a.bias + i);

    f32x4g acc[MW][NT], sum[MW];
#pragma unroll
    for (int i = 0; i < MW; ++i) {
        sum[i] = f32x4g{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = f32x4g{0.0f, 0.0f, 0.0f, 0.0f};
    }

    u32x4g vx[NX], vd[ND];
    const int xp = a.c / E, dp = a.o / E;                  // pieces of a row
    auto load = [&](int64_t block) {
        const int64_t row0 = block * TG_ROWS;
        const int rows = a.rows - row0 < TG_ROWS ? (int)(a.rows - row0) : TG_ROWS;
        const u32x4g* const x = (const u32x4g*)((const T*)a.x + row0 * a.c);
        const u32x4g* const d = (const u32x4g*)((const T*)a.dy + row0 * a.o);
#pragma unroll
        for (int i = 0; i < NX; ++i) {
            const int p = i * 256 + threadIdx.x;
            vx[i] = p < rows * xp ? x[p] : u32x4g{0, 0, 0, 0};
        }
#pragma unroll
        for (int i = 0; i < ND; ++i) {
            const int p = i * 256 + threadIdx.x;
            vd[i] = p < rows * dp ? d[p] : u32x4g{0, 0, 0, 0};
        }
    };
    auto park = [&] {
#pragma unroll
        for (int i = 0; i < NX; ++i) {
            const int p = i * 256 + threadIdx.x, row = p / xp;
            if (row < TG_ROWS) *(u32x4g*)(xs + row * s.x_stride + (p - row * xp) * 16) = vx[i];
        }
#pragma unroll
        for (int i = 0; i < ND; ++i) {
            const int p = i * 256 + threadIdx.x, row = p / dp;
            if (row < TG_ROWS) *(u32x4g*)(dys + row * dy_stride + (p - row * dp) * 16) = vd[i];
        }
    };

    int64_t block = blockIdx.x;
    const int64_t blocks = (a.rows + TG_ROWS - 1) / TG_ROWS;
    if (block < blocks) load(block);
    for (; block < blocks; block += gridDim.x) {
        __syncthreads();                                   // the tiles of the block before are read
        park();
        if (block + gridDim.x < blocks) load(block + gridDim.x);
        __syncthreads();
        const int mine = wave * 16 + r;                    // this lane's row in dz and dx
        if constexpr (Z) {
            for (int n = 0; n < a.o; n += 16) {
                f32x4g zg = *(const f32x4g*)(bias + n + 4 * q), zu = zg;
                if constexpr (GATED) zu = *(const f32x4g*)(bias + a.o + n + 4 * q);
                for (int k = 0; k < s.x_steps; ++k) {
                    const u32x4g x = *(const u32x4g*)(xs + mine * s.x_stride + (k * 4 + q) * 16);
                    gm_mul<T, 16>(zg, *(const u32x4g*)(wz + (n + r) * s.x_stride + (k * 4 + q) * 16), x);
                    if constexpr (GATED) gm_mul<T, 16>(zu, *(const u32x4g*)(wz + (a.o + n + r) * s.x_stride + (k * 4 + q) * 16), x);
                }
                if (n + 4 * q < a.o) {                     // o is a multiple of four
                    float z[1][8], u[1][8], e[1][8];
                    T* const p = (T*)(dz + mine * s.dz_stride) + n + 4 * q;
                    const T* const d = (const T*)(dys + mine * dy_stride) + n + 4 * q;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        z[0][i] = zg[i], u[0][i] = zu[i], e[0][i] = gm_get(d + i);
                        z[0][4 + i] = u[0][4 + i] = e[0][4 + i] = 0.0f;
                    }
                    GemmArgs g;
                    g.mode = GATED ? GEMM_GATED_SLOPE : GEMM_SLOPE;
                    g.act = a.act;
                    gm_finish<GATED, 1>(g, z, u, e);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        gm_put(p + i, z[0][i]);
                        if constexpr (LO) gm_put((T*)(dl + ((char*)(p + i) - dz)), gm_rest<T>(z[0][i]));
                        if constexpr (GATED) {
                            gm_put(p + a.o + i, u[0][i]);
                            if constexpr (LO) gm_put((T*)(dl + ((char*)(p + a.o + i) - dz)), gm_rest<T>(u[0][i]));
                        }
                    }
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
        if (a.dx) {
            f32x4g d[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j) d[j] = f32x4g{0.0f, 0.0f, 0.0f, 0.0f};
            for (int k = 0; k < s.dz_steps; ++k) {
                const u32x4g f = *(const u32x4g*)(dz + mine * s.dz_stride + (k * 4 + q) * 16);
                u32x4g fl;
                if constexpr (LO) fl = *(const u32x4g*)(dl + mine * s.dz_stride + (k * 4 + q) * 16);
#pragma unroll
                for (int j = 0; j < NT; ++j)
                    if (j * 16 < a.c) {
                        const u32x4g w = *(const u32x4g*)(wt + (j * 16 + r) * s.dz_stride + (k * 4 + q) * 16);
                        gm_mul<T, 16>(d[j], w, f);
                        if constexpr (LO) gm_mul<T, 16>(d[j], w, fl);
                    }
            }
            const int64_t row = block * TG_ROWS + mine;
            if (row < a.rows) {
                T* const out = (T*)a.dx + row * a.c + 4 * q;
#pragma unroll
                for (int j = 0; j < NT; ++j)
                    if (j * 16 + 4 * q < a.c) {
                        const float v[4] = {d[j][0], d[j][1], d[j][2], d[j][3]};
                        thin_put4<T, true>(out + j * 16, 4, v);
                    }
            }
        }
        if (Z) __syncthreads();                            // everyone's dz
        if (a.partial || a.sums) {
#pragma unroll
            for (int k = 0; k < RS; ++k) {
                u32x4g fx[NT];
#pragma unroll
                for (int j = 0; j < NT; ++j)
                    if (j * 16 < a.c) fx[j] = turned_frag<T>(xs, s.x_stride, k, j * 16, lane);
#pragma unroll
                for (int i = 0; i < MW; ++i) {
                    const int m = (i * 4 + wave) * 16;
                    if (m < wide) {                        // uniform
                        const u32x4g f = turned_frag<T>(dz, s.dz_stride, k, m, lane);
#pragma unroll
                        for (int j = 0; j < NT; ++j)
                            if (j * 16 < a.c) gm_mul<T, 16>(acc[i][j], fx[j], f);
                        constexpr unsigned one = sizeof(T) == 4 ? 0x3f800000u : __is_same(T, __half) ? 0x3c003c00u : 0x3f803f80u;
                        gm_mul<T, 16>(sum[i], u32x4g{one, one, one, one}, f);
                        if constexpr (LO) {
                            const u32x4g fl = turned_frag<T>(dl, s.dz_stride, k, m, lane);
#pragma unroll
                            for (int j = 0; j < NT; ++j)
                                if (j * 16 < a.c) gm_mul<T, 16>(acc[i][j], fx[j], fl);
                            gm_mul<T, 16>(sum[i], u32x4g{one, one, one, one}, fl);
                        }
                    }
                }
            }
        }
    }
    // [workgroup][wide][c] and [workgroup][wide]; a lane has one column of dz
#pragma unroll
    for (int i = 0; i < MW; ++i) {
        const int m = (i * 4 + wave) * 16 + r;
        if (m < wide) {
            if (a.partial) {
                float* const p = a.partial + ((int64_t)blockIdx.x * wide + m) * a.c + 4 * q;
#pragma unroll
                for (int j = 0; j < NT; ++j)
                    if (j * 16 + 4 * q < a.c) *(f32x4g*)(p + j * 16) = acc[i][j];
            }
            if (a.sums && q == 0) a.sums[(int64_t)blockIdx.x * wide + m] = sum[i][0];
        }
    }
}

template <typename T, bool GATED, bool Z>
hipError_t pick_thin_grad(const ThinGradArgs& a, int grid, hipStream_t st) {
    const int wide = GATED ? 2 * a.o : a.o;
    const ThinGradShape s = thin_grad_shape(a.c, a.o, sizeof(T), GATED, Z);
    auto go = [&](auto nt, auto mw) {
        k_thin_grad<T, decltype(nt)::value, decltype(mw)::value, GATED, Z><<<grid, 256, s.bytes, st>>>(a);
        return hipGetLastError();
    };
    auto rows = [&](auto nt) {
        if (wide <= 64) return go(nt, std::integral_constant<int, 1>{});
        if constexpr (decltype(nt)::value < 8) {
            if (wide > 128) return go(nt, std::integral_constant<int, 4>{});
        }
        return go(nt, std::integral_constant<int, 2>{});
    };
    if (a.c <= 32) return rows(std::integral_constant<int, 2>{});
    if (a.c <= 64) return rows(std::integral_constant<int, 4>{});
    return rows(std::integral_constant<int, 8>{});
}

}  // namespace

template <typename T>
hipError_t launch_thin_grad(const ThinGradArgs& a, bool gated, int grid, hipStream_t st) {
    if (gated) return pick_thin_grad<T, true, true>(a, grid, st);
    return a.act == SR_ACT_NONE ? pick_thin_grad<T, false, false>(a, grid, st) : pick_thin_grad<T, false, true>(a, grid, st);
}

}  // namespace srd

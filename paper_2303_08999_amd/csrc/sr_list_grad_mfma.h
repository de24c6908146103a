// Gradient of the per-pixel list form on the matrix cores: lists of up to 16 entries, up to 128 atoms, one or three channels.
//
// Both gradients are products with E, the gradient of a pixel's filter (k^2 numbers a pixel):
//     responses  R[l][i] = sum_j D[l][j] E[j][i]       of which a pixel's listed ones are its dvalue
//     ddict      G[l][j] = sum_i Phi[l][i] E[j][i]     Phi the lists as dense columns
// v_mfma_f32_16x16x32_f16 serves both: for R the sum runs over the taps, so lane (q, n) forms taps 8 q .. 8 q + 7 of pixel n of a
// group of 16, which is the operand as it lies in its registers; for G it runs over the 32 pixels of a unit, so E goes through LDS
// as [tap][pixel], the lists are scattered into a dense [atom][pixel] array that is all zero between uses, and R goes through LDS
// for its gather.  All of that is a wavefront's own scratch: no barrier but around the up-sampled tile.
//
// Precision: fp16 products with fp32 sums.  E is scaled pixel by pixel by a power of two (to 2^14 .. 2^15) and split in two fp16
// numbers, 22 bits; D likewise with one power of two; R takes the three products that matter.  For G the pixels of a unit share
// the largest one's power of two (parts below 2^-38 of it are lost), fp16 values enter as they are, fp32 ones split as well; a
// unit's sums are added in fp32, unscaled, and handed on in double after at most 4096 pixels of a wavefront.
#pragma once
#include "sr_list_grad.h"

namespace srd {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef unsigned u32x4v __attribute__((ext_vector_type(4)));
// LDS scratch is read under other types than it is written
typedef float4v __attribute__((may_alias)) lds_f4;
typedef float __attribute__((may_alias)) lds_f;
typedef u32x4v __attribute__((may_alias)) lds_u4;
typedef unsigned __attribute__((may_alias)) lds_u;
typedef unsigned short __attribute__((may_alias)) lds_h;

template <int K, int LP, int CM, typename TV>
struct GradCfg {
    static constexpr int KK = K * K, R = (K - 1) / 2, NS = (KK + 31) / 32, NT = (KK + 15) / 16, MT = LP / 16;
    static constexpr int UW = GM_TW + K - 1, UH = GM_TH + K - 1;
    static constexpr int MAXLRX = (UW - 1) / 2 + 5, MAXLRY = (UH - 1) / 2 + 5;       // scale >= 2
    static constexpr int UN = CM * UH * UW;                                            // and one zero behind
    static constexpr int VN = CM * UH * MAXLRX;
    static constexpr bool SPLIT = sizeof(TV) == 4;                                     // values in two parts
    static constexpr int PP = 40;                  // pitch of Phi in halves: 16 rows' 16-byte pieces fall on all 64 banks
    static constexpr int EP = 36;                  // pitch of [tap][pixel] in words, likewise
    static constexpr int RP = LP + 4;              // pitch of a pixel's responses, likewise
    static constexpr int PHI_B = LP * PP * 2 * (SPLIT ? 2 : 1);
    static constexpr int ER_B = 32 * NS * EP * 4 > 16 * RP * 4 ? 32 * NS * EP * 4 : 16 * RP * 4;
    static constexpr int WAVE_B = PHI_B + ER_B;
    static constexpr int WPE = K == 7 || LP > 80 ? 1 : 2;                              // wavefronts per SIMD (registers)
    static_assert(CM * MAXLRY * MAXLRX <= UN, "the LR rows fit where the tile goes");
};

__device__ __forceinline__ void wave_lds_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
// 2^n for an exponent field (n + 127), kept where fp32 has it
__device__ __forceinline__ float pow2_field(int field) { return __uint_as_float((unsigned)clampi(field, 1, 254) << 23); }
// exponent field of a magnitude, from 15 on: its reciprocal scale below stays a number
__device__ __forceinline__ int exponent_field(float m) { return clampi((int)(__float_as_uint(m) >> 23), 15, 254); }

// x and y scaled into fp16's range -> words (high part, low part)
__device__ __forceinline__ void split_pair(float x, float y, unsigned& hi, unsigned& lo) {
    const auto h = __builtin_amdgcn_cvt_pkrtz(x, y);
    const auto l = __builtin_amdgcn_cvt_pkrtz(x - (float)h[0], y - (float)h[1]);
    __builtin_memcpy(&hi, &h, 4);
    __builtin_memcpy(&lo, &l, 4);
}

template <int K, int LP, int CM, typename TV>
__global__ __launch_bounds__(256, (GradCfg<K, LP, CM, TV>::WPE))
void k_list_grad_mfma(const ListGradArgs a) {
    using F = GradCfg<K, LP, CM, TV>;
    constexpr int KK = F::KK, R = F::R, NS = F::NS, NT = F::NT, MT = F::MT, UW = F::UW, UH = F::UH, MAXLRX = F::MAXLRX, MAXLRY = F::MAXLRY;
    __shared__ float U[F::UN + 4];                   // up-sampled tile, then a zero; before that, in its place, the LR footprint
    __shared__ float V[F::VN];
    __shared__ float4 xw[UW], yw[UH];
    __shared__ int xb[UW], yb[UH];
    __shared__ __align__(16) unsigned char scratch[4][F::WAVE_B];
    __shared__ float dmax[4];

    const int tid = threadIdx.x, lane = tid & 63, q = lane >> 4, n = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    unsigned char* const phi = scratch[wave];
    unsigned char* const er = scratch[wave] + F::PHI_B;
    const size_t plane = (size_t)a.H * a.W;
    const unsigned lmax = (unsigned)a.L - 1u;

    // ---- the dictionary as operands of R: lane (q, n) has atom 16 mt + n, taps 32 s + 8 q and on, times 2^14 / its largest exponent
    float big = 0.0f;
    for (int e = tid; e < a.L * KK; e += 256) big = fmaxf(big, fabsf(a.dict[e]));
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) big = fmaxf(big, __shfl_xor(big, d));
    if (lane == 0) dmax[wave] = big;
    for (int e = lane; e < F::PHI_B / 16; e += 64) ((lds_u4*)phi)[e] = (u32x4v){0, 0, 0, 0};
    if (tid < 4) U[F::UN + tid] = 0.0f;
    __syncthreads();
    const int dx = exponent_field(fmaxf(fmaxf(dmax[0], dmax[1]), fmaxf(dmax[2], dmax[3])));
    const float dscale = pow2_field(268 - dx), dback = pow2_field(dx - 14);
    u32x4v Dh[MT][NS], Dl[MT][NS];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const int l = 16 * mt + n;
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int j = 32 * s + 8 * q + i;
                v[i] = l < a.L && j < KK ? a.dict[l * KK + j] * dscale : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                unsigned hi, lo;
                split_pair(v[2 * i], v[2 * i + 1], hi, lo);
                Dh[mt][s][i] = hi, Dl[mt][s][i] = lo;
            }
        }
    // where a lane's taps are in the tile, from its pixel's corner (the zero behind the tile: a tap that is none)
    int tap[NS][8];
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int j = 32 * s + 8 * q + i;
            tap[s][i] = j < KK ? j / K * UW + j % K : -1;
        }
    float4v G[MT][NT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int t = 0; t < NT; ++t) G[mt][t] = (float4v){0, 0, 0, 0};
    double* const rec = a.partial ? a.partial + (size_t)blockIdx.x * a.L * KK : nullptr;
    bool first = true;
    int held = 0;

    // hands the sums on: the wavefronts one after the other, through their scratch (G is 16 x 16 tiles: lane (q, n) has atoms 4 q ..
    // 4 q + 3 of tap n)
    auto hand_on = [&]() {
#pragma unroll 1
        for (int w = 0; w < 4; ++w) {
            if (wave == w) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int l = 16 * mt + 4 * q + r, j = 16 * t + n;
                            if (l < a.L && j < KK) {
                                double* at = rec + l * KK + j;
                                *at = (first && w == 0 ? 0.0 : *at) + (double)G[mt][t][r];
                            }
                            G[mt][t][r] = 0.0f;
                        }
            }
            __syncthreads();
        }
        first = false;
    };

    for (int64_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
        const int im = (int)(tile / ((int64_t)a.tiles_x * a.tiles_y));
        const int in = (int)(tile - (int64_t)im * a.tiles_x * a.tiles_y);
        const int Y0 = in / a.tiles_x * GM_TH, X0 = in % a.tiles_x * GM_TW;
        // ---- stage 1, all channels together
        const TileOrigin o = tile_origin(Y0, X0, R, UH, UW, a.H, a.W, a.s);
        __syncthreads();                             // the last tile has been used
        build_taps<UW, MAXLRX, 256>(X0, R, a.W, a.s, o.lx0, xw, xb, tid);
        build_taps<UH, MAXLRY, 256>(Y0, R, a.H, a.s, o.ly0, yw, yb, tid);
#pragma unroll
        for (int c = 0; c < CM; ++c) {
            const size_t pl = ((size_t)im * CM + c) * (size_t)a.h * a.w;
            if (a.io_f16) load_lr_tile<__half, MAXLRY, MAXLRX, 256>((const __half*)a.lr + pl, a.h, a.w, o, U + c * MAXLRY * MAXLRX, tid);
            else load_lr_tile<float, MAXLRY, MAXLRX, 256>((const float*)a.lr + pl, a.h, a.w, o, U + c * MAXLRY * MAXLRX, tid);
        }
        __syncthreads();
#pragma unroll
        for (int c = 0; c < CM; ++c) vpass<MAXLRX, UH, 256>(U + c * MAXLRY * MAXLRX, V + c * UH * MAXLRX, yw, yb, tid);
        __syncthreads();
#pragma unroll
        for (int c = 0; c < CM; ++c)
            hpass<MAXLRX, UW, UH, 256>(V + c * UH * MAXLRX, xw, xb, tid, [&](int yy, int xx, float v) { U[(c * UH + yy) * UW + xx] = v; });
        __syncthreads();

        // ---- a wavefront's units: 32 pixels of a row, two groups of 16
#pragma unroll 1
        for (int u = 0; u < GM_TH * 2 / 4; ++u) {
            const int ty = wave * (GM_TH / 4) + u / 2, Y = Y0 + ty, x0 = u % 2 * 32;
            if (Y >= a.H || X0 + x0 >= a.W) continue;
            unsigned idx[2][4];
            TV val[2][4];
            float dy[2][CM];
            bool on[2], inside[2];
            size_t at[2];
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const int X = X0 + x0 + 16 * g + n;
                inside[g] = X < a.W;
                at[g] = (size_t)Y * a.W + (inside[g] ? X : 0);
                on[g] = inside[g] && (!a.mask || a.mask[(size_t)im * plane + at[g]] != 0);
#pragma unroll
                for (int c = 0; c < CM; ++c) {
                    const size_t e = ((size_t)im * CM + c) * plane + at[g];
                    dy[g][c] = !on[g] ? 0.0f : a.io_f16 ? ld_as_float((const __half*)a.dout, e) : ((const float*)a.dout)[e];
                }
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (4 * r < a.T) {
                        const int t = 4 * r + q;
                        const size_t e = ((size_t)im * a.T + (t < a.T ? t : 0)) * plane + at[g];
                        const unsigned l = inside[g] ? (unsigned)a.index[e] : 0u;
                        idx[g][r] = l < lmax ? l : lmax;
                        val[g][r] = on[g] && t < a.T ? ((const TV*)a.value)[e] : (TV)0.0f;
                    }
            }
            unsigned word[2][NS][8];                 // E as (high, low) halves, of the pixel's own scale
            int ex[2];
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                float E[NS][8];
#pragma unroll
                for (int s = 0; s < NS; ++s)
#pragma unroll
                    for (int i = 0; i < 8; ++i) E[s][i] = 0.0f;
#pragma unroll
                for (int c = 0; c < CM; ++c) {
                    const float* const corner = U + (c * UH + ty) * UW + x0 + 16 * g + n;
#pragma unroll
                    for (int s = 0; s < NS; ++s)
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float* p = tap[s][i] < 0 ? U + F::UN : corner + tap[s][i];
                            E[s][i] = fmaf(dy[g][c], *p, E[s][i]);
                        }
                }
                float m = 0.0f;
#pragma unroll
                for (int s = 0; s < NS; ++s)
#pragma unroll
                    for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(E[s][i]));
                m = fmaxf(m, __shfl_xor(m, 16));
                m = fmaxf(m, __shfl_xor(m, 32));
                ex[g] = exponent_field(m);
                const float sc = pow2_field(268 - ex[g]);
                u32x4v Eh[NS], El[NS];
#pragma unroll
                for (int s = 0; s < NS; ++s)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        unsigned hi, lo;
                        split_pair(E[s][2 * i] * sc, E[s][2 * i + 1] * sc, hi, lo);
                        Eh[s][i] = hi, El[s][i] = lo;
                        word[g][s][2 * i] = (hi & 0xffffu) | (lo << 16);
                        word[g][s][2 * i + 1] = (hi >> 16) | (lo & 0xffff0000u);
                    }
                if (a.dvalue) {
                    wave_lds_fence();
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        float4v r = {0, 0, 0, 0};
#pragma unroll
                        for (int s = 0; s < NS; ++s) {
                            const half8 dh = __builtin_bit_cast(half8, Dh[mt][s]), dl = __builtin_bit_cast(half8, Dl[mt][s]);
                            const half8 eh = __builtin_bit_cast(half8, Eh[s]), el = __builtin_bit_cast(half8, El[s]);
                            r = __builtin_amdgcn_mfma_f32_16x16x32_f16(dl, eh, r, 0, 0, 0);
                            r = __builtin_amdgcn_mfma_f32_16x16x32_f16(dh, el, r, 0, 0, 0);
                            r = __builtin_amdgcn_mfma_f32_16x16x32_f16(dh, eh, r, 0, 0, 0);
                        }
                        *(lds_f4*)(er + 4 * (n * F::RP + 16 * mt + 4 * q)) = r;
                    }
                    wave_lds_fence();
                    const float back = pow2_field(ex[g] - 14);
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (4 * r < a.T) {
                            const int t = 4 * r + q;
                            const float v = *(lds_f*)(er + 4 * (n * F::RP + idx[g][r])) * back * dback;
                            if (inside[g] && t < a.T) st_from_float((TV*)a.dvalue, ((size_t)im * a.T + t) * plane + at[g], on[g] ? v : 0.0f);
                        }
                }
            }
            if (rec) {
                // the unit's scale, its values' scale; E to [tap][pixel], the lists to [atom][pixel]
                int es = max(ex[0], ex[1]);
#pragma unroll
                for (int d = 8; d > 0; d >>= 1) es = max(es, __shfl_xor(es, d));
                float vback = 1.0f, vsc = 1.0f;
                if (F::SPLIT) {
                    float m = 0.0f;
#pragma unroll
                    for (int g = 0; g < 2; ++g)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (4 * r < a.T) m = fmaxf(m, fabsf((float)val[g][r]));
#pragma unroll
                    for (int d = 32; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
                    const int vx = exponent_field(m);
                    vsc = pow2_field(268 - vx);
                    vback = pow2_field(vx - 14);
                }
                wave_lds_fence();
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const _Float16 f = (_Float16)pow2_field(127 + ex[g] - es);
                    const half2v ff = {f, f};
#pragma unroll
                    for (int s = 0; s < NS; ++s)
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const half2v v = __builtin_bit_cast(half2v, word[g][s][i]) * ff;
                            *(lds_u*)(er + 4 * ((32 * s + 8 * q + i) * F::EP + 16 * g + n)) = __builtin_bit_cast(unsigned, v);
                        }
                }
                wave_lds_fence();
                half8 eh[NT], el[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const lds_u4* p = (const lds_u4*)(er + 4 * ((16 * t + n) * F::EP + 8 * q));
                    const u32x4v w0 = p[0], w1 = p[1];
                    u32x4v h, l;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        h[i] = __builtin_amdgcn_perm(w0[2 * i + 1], w0[2 * i], 0x05040100u);
                        l[i] = __builtin_amdgcn_perm(w0[2 * i + 1], w0[2 * i], 0x07060302u);
                        h[2 + i] = __builtin_amdgcn_perm(w1[2 * i + 1], w1[2 * i], 0x05040100u);
                        l[2 + i] = __builtin_amdgcn_perm(w1[2 * i + 1], w1[2 * i], 0x07060302u);
                    }
                    eh[t] = __builtin_bit_cast(half8, h), el[t] = __builtin_bit_cast(half8, l);
                }
                const float back = pow2_field(es - 14) * vback;
                // Entries into the dense columns.  An atom that a pixel lists twice has one place there: every entry writes its number, those that
                // find another's wait for the next pass (lists as the router makes them: one pass).
                unsigned left = 0;
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (4 * r + q < a.T) left |= 0x11u << r;
#pragma unroll 1
                do {
#pragma unroll
                    for (int g = 0; g < 2; ++g)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (left >> (4 * g + r) & 1) *(lds_h*)(phi + 2 * (idx[g][r] * F::PP + 16 * g + n)) = (unsigned short)(4 * r + q + 1);
                    wave_lds_fence();
                    unsigned mine = 0;
#pragma unroll
                    for (int g = 0; g < 2; ++g)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if ((left >> (4 * g + r) & 1) && *(lds_h*)(phi + 2 * (idx[g][r] * F::PP + 16 * g + n)) == 4 * r + q + 1) mine |= 1u << (4 * g + r);
                    wave_lds_fence();
#pragma unroll
                    for (int g = 0; g < 2; ++g)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (mine >> (4 * g + r) & 1) {
                                unsigned char* p = phi + 2 * (idx[g][r] * F::PP + 16 * g + n);
                                if (F::SPLIT) {
                                    unsigned hi, lo;
                                    split_pair((float)val[g][r] * vsc, 0.0f, hi, lo);
                                    *(lds_h*)p = (unsigned short)hi;
                                    *(lds_h*)(p + LP * F::PP * 2) = (unsigned short)lo;
                                } else {
                                    unsigned short h;
                                    __builtin_memcpy(&h, &val[g][r], 2);
                                    *(lds_h*)p = h;
                                }
                            }
                    left &= ~mine;
                    wave_lds_fence();
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        const half8 p0 = __builtin_bit_cast(half8, *(const lds_u4*)(phi + 2 * ((16 * mt + n) * F::PP + 8 * q)));
                        half8 p1;
                        if (F::SPLIT) p1 = __builtin_bit_cast(half8, *(const lds_u4*)(phi + 2 * ((LP + 16 * mt + n) * F::PP + 8 * q)));
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            float4v r = {0, 0, 0, 0};
                            if (F::SPLIT) r = __builtin_amdgcn_mfma_f32_16x16x32_f16(p1, eh[t], r, 0, 0, 0);
                            r = __builtin_amdgcn_mfma_f32_16x16x32_f16(p0, el[t], r, 0, 0, 0);
                            r = __builtin_amdgcn_mfma_f32_16x16x32_f16(p0, eh[t], r, 0, 0, 0);
#pragma unroll
                            for (int i = 0; i < 4; ++i) G[mt][t][i] = fmaf(r[i], back, G[mt][t][i]);
                        }
                    }
                    wave_lds_fence();
#pragma unroll
                    for (int g = 0; g < 2; ++g)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (mine >> (4 * g + r) & 1) {
                                unsigned char* p = phi + 2 * (idx[g][r] * F::PP + 16 * g + n);
                                *(lds_h*)p = 0;
                                if (F::SPLIT) *(lds_h*)(p + LP * F::PP * 2) = 0;
                            }
                    wave_lds_fence();
                } while (__any(left));
            }
        }
        if (rec && ++held == 4096 / (GM_TW * GM_TH / 4)) {
            held = 0;
            hand_on();
        }
    }
    if (rec) hand_on();
}

template <int K, int LP, int CM, typename TV>
static hipError_t grad_mfma_one(const ListGradArgs& a, int grid, hipStream_t st) {
    k_list_grad_mfma<K, LP, CM, TV><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}
template <int K, typename TV>
static hipError_t grad_mfma_k(const ListGradArgs& a, int grid, hipStream_t st) {
    if (a.L <= 80) return a.C == 1 ? grad_mfma_one<K, 80, 1, TV>(a, grid, st) : grad_mfma_one<K, 80, 3, TV>(a, grid, st);
    return a.C == 1 ? grad_mfma_one<K, 128, 1, TV>(a, grid, st) : grad_mfma_one<K, 128, 3, TV>(a, grid, st);
}

}  // namespace srd

// Products of very many rows whose weight fits the registers of a compute unit (sr_gemm.h): 16-bit types, and fp32 as three bfloat16 parts; rows on 16-byte pieces, or on
// four bytes.
//
// A workgroup has a compute unit to itself and keeps the whole weight in registers as matrix operands, a wavefront NT tiles of 16 columns for all
// k.  Rows come to LDS a block at a time, straight from memory, while the block before is worked on; every wavefront reads them as the other operand.  So
// a tile has no beginning and no end of its own, which is what rows of few features spend their time on in the tile kernel.  Tiles of columns are
// dealt in pairs so that a lane holds 8 neighbouring columns of a row, which go to memory from there.  What a wavefront has made is stored
// behind the next wait for rows, so that no wait is for stores just begun; a register that did not fit would be read again behind the rows on
// their way, so each form takes only what fits (1048576 rows of 512 to 128, bfloat16: 430 us with three of them outside, 254 without).
//
// Bound by memory: 1048576 rows of 128 to 256, bfloat16, 184 us, of 136 to 200 202 us, gated 128 to 256 230 us; the tile kernel 221, 360, 426.  fp32, of 64 to 512
// 545 us, of 100 to 200 506 us; the tile kernel 805, 667.
#pragma once
#include "sr_gemm.h"

namespace srd {
namespace {

using lds_void_r = __attribute__((address_space(3))) void*;
using lds_s4r = __attribute__((address_space(3))) s16x4g;

// STORE or GATED; the same with something to add; SLOPE or GATED_SLOPE; STORE of a weight stored [k][n]
enum { ROWS_FORWARD = 0, ROWS_EXTRA = 1, ROWS_SLOPE = 2, ROWS_TURNED = 3 };

// 8 values of a row as they are stored
template <typename T> struct Held { u32x4g v[sizeof(T) / 2]; };
template <typename T> __device__ __forceinline__ Held<T> rows_pack(const float v[8]) {
    if constexpr (sizeof(T) == 4) {
        return {__builtin_bit_cast(u32x4g, f32x4g{v[0], v[1], v[2], v[3]}), __builtin_bit_cast(u32x4g, f32x4g{v[4], v[5], v[6], v[7]})};
    } else if constexpr (__is_same(T, __half)) {
        return {__builtin_bit_cast(u32x4g, half8g{(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3], (_Float16)v[4], (_Float16)v[5], (_Float16)v[6], (_Float16)v[7]})};
    } else {
        return {__builtin_bit_cast(u32x4g, bf8g{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3], (__bf16)v[4], (__bf16)v[5], (__bf16)v[6], (__bf16)v[7]})};
    }
}
template <typename T> __device__ __forceinline__ void rows_store(T* p, int count, const Held<T>& h) {
    if (count >= 8) {
#pragma unroll
        for (int j = 0; j < (int)sizeof(T) / 2; ++j) *(u32x4u*)(p + j * (16 / sizeof(T))) = h.v[j];
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) ((unsigned*)p)[i] = h.v[i / 4][i % 4];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) ((unsigned short*)p)[i] = (unsigned short)((unsigned)h.v[0][i / 2] >> (i % 2 * 16));
    }
}
// 8 k of a row or a column as a matrix operand: fp32 in its three parts
template <typename T> using RowsFrag = std::conditional_t<sizeof(T) == 4, Split8, u32x4g>;
template <typename T> __device__ __forceinline__ RowsFrag<T> rows_frag(u32x4g lo, u32x4g hi) {
    if constexpr (sizeof(T) == 4) return gm_split(lo, hi);
    else return lo;
}

// KS: steps of 32 k whose weights are held; KIND: see above.  wn x wr wavefronts: groups of columns, groups of rows; subs: of 32 wr rows, in a block.
template <typename T, int KS, int NT, bool GATED, int KIND>
__global__ __launch_bounds__(512, 2) void k_rows(const GemmArgs g, const int wn, const int wr, const int subs) {
    constexpr int E = 16 / sizeof(T), PS = 32 / E, V = sizeof(T) / 2;      // values of a piece of 16 bytes; pieces of a step, of 8 k
    constexpr bool EXTRA = KIND == ROWS_EXTRA || KIND == ROWS_SLOPE;
    constexpr int H = GATED ? 2 : 1, RF = 2, NP = NT / 2, OUTS = GATED && KIND == ROWS_SLOPE ? 2 : 1;
    __shared__ __align__(1024) char lds[2 * ROWS_STAGE];
    __shared__ __align__(16) float bias[H * 8 * NT * 16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = wn * wr;
    const int r = lane % 16, q = lane / 16, wc = wave % wn, rg = wave / wn;
    const int np = wn * NT * 16, n0 = wc * NT * 16;
    const int steps = (g.k + 31) / 32, pieces = (g.k + E - 1) / E;         // of a row
    const int stride = steps * 32 * (int)sizeof(T);

    // Rows in LDS: pieces of 16 bytes, those of a row exchanged so that 8 rows at one k lie in different banks.
    const auto turn = [&](int row) { return stride & 64 ? row >> 1 & 3 : row & 7; };
    const int block_rows = 32 * wr * subs, blocks = g.m / block_rows + (g.m % block_rows != 0), loads = block_rows * stride / 1024;
    const unsigned per_row = (1 << 20) / (PS * steps) + 1;                 // x * per_row >> 20 = x / (PS steps) for x < 4096
    const bool whole = (uintptr_t)g.a % 16 == 0 && g.lda % E == 0;         // else rows come by 4 bytes
    const auto fetch = [&](int block, char* to) {
        const int row0 = block * block_rows, last = g.m - 1 - row0;
        const char* const from = (const char*)g.a + (int64_t)row0 * g.lda * (int)sizeof(T);
        // what is behind a row or the last row is read in their place, and taken out when it is used or not stored (the moves: see the tile kernel's loads)
        if (whole) {
            for (int i = wave; i < loads; i += waves) {
                const int x = i * 64 + lane, row = (int)(x * per_row >> 20);
                int p = (x - row * PS * steps) ^ turn(row);
                if (p >= pieces) p = pieces - 1;
                const unsigned off = (unsigned)(row < last ? row : last) * (unsigned)(g.lda * (int)sizeof(T)) + p * 16;
                uint64_t at;
                unsigned m0;
                asm volatile("s_mov_b32 %1, %4\n\ts_mov_b64 %0, %3\n\tglobal_load_lds_dwordx4 %2, %0" : "=&s"(at), "=&{m0}"(m0) : "v"(off), "s"(from), "s"((unsigned)(uintptr_t)(lds_void_r)(to + i * 1024)) : "memory");
            }
        } else {
            const int fours = (g.k * (int)sizeof(T) + 3) / 4;
            for (int i = wave; i < 4 * loads; i += waves) {
                const int x = i * 16 + lane / 4, row = (int)(x * per_row >> 20);
                int p = ((x - row * PS * steps) ^ turn(row)) * 4 + lane % 4;
                if (p >= fours) p = fours - 1;
                const unsigned off = (unsigned)(row < last ? row : last) * (unsigned)(g.lda * (int)sizeof(T)) + p * 4;
                uint64_t at;
                unsigned m0;
                asm volatile("s_mov_b32 %1, %4\n\ts_mov_b64 %0, %3\n\tglobal_load_lds_dword %2, %0" : "=&s"(at), "=&{m0}"(m0) : "v"(off), "s"(from), "s"((unsigned)(uintptr_t)(lds_void_r)(to + i * 256)) : "memory");
            }
        }
    };
    if (KIND != ROWS_TURNED) fetch(blockIdx.x, lds);

    // the weight: tile t of a wavefront has columns 32 (t / 2) + 4 (t % 2) + {0-3, 8-11, 16-19, 24-27} of its own
    RowsFrag<T> w[H][NT][KS];
    if constexpr (KIND == ROWS_TURNED) {
        // by way of LDS, as many steps at a time as it holds, turned when they are read
        const int ws = np * (int)sizeof(T) + 16, at_once = 2 * ROWS_STAGE / (32 * ws);
        int left = 0;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            if (s < steps) {
                if (!left) {
                    left = at_once;
                    __syncthreads();
                    const int count = (steps - s < left ? steps - s : left) * 32;
                    for (int i = threadIdx.x; i < count * (np / E); i += waves * 64) {
                        const int k = i / (np / E), p = i - k * (np / E);
                        *(u32x4g*)(lds + k * ws + p * 16) = gm_piece((const T*)g.b + (int64_t)(s * 32 + k) * g.ldb + p * E, s * 32 + k < g.k ? g.n - p * E : 0);
                    }
                    __syncthreads();
                }
                const char* const from = lds + (at_once - left--) * 32 * ws;
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const int col = n0 + t / 2 * 32 + t % 2 * 4;
                    if constexpr (sizeof(T) == 4) {
                        const char* const p = from + 8 * q * ws + (col + r / 4 * 8 + r % 4) * 4;
                        u32x4g lo, hi;
#pragma unroll
                        for (int j = 0; j < 4; ++j) lo[j] = *(const unsigned*)(p + j * ws), hi[j] = *(const unsigned*)(p + (4 + j) * ws);
                        w[0][t][s] = rows_frag<T>(lo, hi);
                    } else {
                        const char* const p = from + (8 * q + r / 4) * ws + (col + r % 4 * 8) * 2;
                        using u2 = __attribute__((ext_vector_type(2))) unsigned;
                        const u2 a = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4r*)p));
                        const u2 b = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4r*)(p + 4 * ws)));
                        w[0][t][s] = rows_frag<T>(u32x4g{a[0], a[1], b[0], b[1]}, u32x4g{});
                    }
                }
            }
        }
        __syncthreads();
    } else {
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int n = n0 + t / 2 * 32 + t % 2 * 4 + r / 4 * 8 + r % 4;
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    const int k = s * 32 + q * 8;
                    const T* const p = (const T*)g.b + (int64_t)(n + h * g.half) * g.ldb + k;
                    const int count = n < g.n ? g.k - k : 0;
                    w[h][t][s] = rows_frag<T>(gm_piece(p, count), V == 2 ? gm_piece(p + E, count - E) : u32x4g{});
                }
            }
    }
    for (int i = threadIdx.x; i < H * np; i += waves * 64) {
        const int h = i >= np, n = h ? i - np : i;
        bias[i] = g.bias && n < g.n ? gm_get((const T*)g.bias + n + h * g.half) : 0.0f;
    }

    const int width = GATED ? 2 * g.half : g.half;                         // of a row of sums
    const int rest = g.k - (steps - 1) * 32 - q * 8;                       // of k, in this lane's piece of the last step
    const bool cut = g.k % 32 != 0;
    int64_t held_row = -1;                                                 // uniform: first row of what is still to be stored
    Held<T> held[OUTS][NP][RF];
    const auto store = [&] {
        if (held_row < 0) return;
#pragma unroll
        for (int f = 0; f < RF; ++f) {
            const int64_t m = held_row + f * 16 + r;
            if (m >= g.m) continue;
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                const int col = n0 + p * 32 + q * 8;
                T* const out = (T*)g.out + m * g.ld_out + col;
                rows_store<T>(out, g.n - col, held[0][p][f]);
                if constexpr (OUTS == 2) rows_store<T>(out + g.half, g.n - col, held[1][p][f]);
            }
        }
    };
    Raw8<T> extra[EXTRA ? NP : 1][RF];
    const auto ask = [&](int64_t row) {
#pragma unroll
        for (int f = 0; f < RF; ++f)
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                const int64_t m = row + f * 16 + r;
                const int col = n0 + p * 32 + q * 8;
                extra[p][f].get((const T*)g.extra + m * g.ld_extra + col, m < g.m ? g.n - col : 0);
            }
    };
    float sums[OUTS][KIND == ROWS_SLOPE ? NP : 1][8];
#pragma unroll
    for (int o = 0; o < OUTS; ++o)
#pragma unroll
        for (int p = 0; p < (KIND == ROWS_SLOPE ? NP : 1); ++p)
#pragma unroll
            for (int i = 0; i < 8; ++i) sums[o][p][i] = 0.0f;

    if (KIND == ROWS_TURNED) fetch(blockIdx.x, lds);
    if constexpr (EXTRA) ask((int64_t)blockIdx.x * block_rows + rg * 32);
    int stage = 0;
    for (int block = blockIdx.x; block < blocks; block += gridDim.x) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __syncthreads();                                                   // this block is there, and nobody reads the one before any more
        if (block + (int)gridDim.x < blocks) fetch(block + gridDim.x, lds + (stage ^ 1) * ROWS_STAGE);
        const char* const a = lds + stage * ROWS_STAGE;
        for (int sub = 0; sub < subs; ++sub) {
            store();
            const int first = (sub * wr + rg) * 32;
            const int64_t row = (int64_t)block * block_rows + first;
            f32x4g acc[H][NT][RF];
#pragma unroll
            for (int h = 0; h < H; ++h)
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int f = 0; f < RF; ++f) acc[h][t][f] = *(const f32x4g*)(bias + h * np + n0 + t / 2 * 32 + t % 2 * 4 + q * 8);
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                if (s < steps) {
                    u32x4g x[RF][V];
#pragma unroll
                    for (int f = 0; f < RF; ++f) {
                        const int at = first + f * 16 + r;
#pragma unroll
                        for (int j = 0; j < V; ++j) x[f][j] = *(const u32x4g*)(a + at * stride + ((s * PS + q * V + j ^ turn(at)) << 4));
                    }
                    if (cut && s == steps - 1) {
#pragma unroll
                        for (int f = 0; f < RF; ++f)
#pragma unroll
                            for (int j = 0; j < V; ++j) x[f][j] = gm_cut<T>(x[f][j], rest - j * E);
                    }
                    RowsFrag<T> xf[RF];
#pragma unroll
                    for (int f = 0; f < RF; ++f) xf[f] = rows_frag<T>(x[f][0], x[f][V - 1]);
#pragma unroll
                    for (int part = 0; part < (V == 2 ? 6 : 1); ++part)
#pragma unroll
                        for (int h = 0; h < H; ++h)
#pragma unroll
                            for (int t = 0; t < NT; ++t)
#pragma unroll
                                for (int f = 0; f < RF; ++f) {
                                    if constexpr (V == 2) gm_mul_part<16>(acc[h][t][f], w[h][t][s], xf[f], part);
                                    else gm_mul<T, 16>(acc[h][t][f], w[h][t][s], xf[f]);
                                }
                }
            }
            held_row = row;
#pragma unroll
            for (int f = 0; f < RF; ++f)
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                    float z[1][8], u[1][8], e[1][8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        z[0][i] = acc[0][2 * p + i / 4][f][i % 4];
                        u[0][i] = GATED ? acc[H - 1][2 * p + i / 4][f][i % 4] : 0.0f;
                        e[0][i] = 0.0f;
                    }
                    if constexpr (EXTRA) extra[p][f].values(e[0]);
                    gm_finish<GATED, 1>(g, z, u, e);
                    held[0][p][f] = rows_pack<T>(z[0]);
                    if constexpr (OUTS == 2) held[1][p][f] = rows_pack<T>(u[0]);
                    if constexpr (KIND == ROWS_SLOPE)
                        if (row + f * 16 + r < g.m) {
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                sums[0][p][i] += z[0][i];
                                if constexpr (OUTS == 2) sums[1][p][i] += u[0][i];
                            }
                        }
                }
            if constexpr (EXTRA) ask(sub + 1 < subs ? row + 32 * wr : (int64_t)(block + gridDim.x) * block_rows + rg * 32);
        }
        stage ^= 1;
    }
    store();
    if constexpr (KIND == ROWS_SLOPE) {
        if (!g.sums) return;
#pragma unroll
        for (int o = 0; o < OUTS; ++o)
#pragma unroll
            for (int p = 0; p < NP; ++p) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int d = 1; d < 16; d <<= 1) sums[o][p][i] += __shfl_xor(sums[o][p][i], d);
                const int col = n0 + p * 32 + q * 8;
                if (r == 0) gm_put_some(g.sums + ((int64_t)blockIdx.x * wr + rg) * width + o * g.half + col, g.n - col, sums[o][p]);
            }
    }
}

// tiles x steps x halves that fill half of the registers; and that fit beside what is added or multiplied and the sums of dz
template <typename T> constexpr int ROWS_FRAGS = sizeof(T) == 4 ? 8 : 32;
template <typename T> constexpr int ROWS_EXTRA_FRAGS = sizeof(T) == 4 ? 8 : 16;
template <typename T, int KS, int NT, bool GATED, int KIND>
hipError_t start_rows(const GemmArgs& g, const RowsShape& s, hipStream_t st) {
    for (int from = 0; from < g.n; from += s.cols) {
        GemmArgs c = g;
        c.n = g.n - from < s.cols ? g.n - from : s.cols;
        c.b = (const T*)g.b + from * (KIND == ROWS_TURNED ? 1 : g.ldb);
        if (g.bias) c.bias = (const T*)g.bias + from;
        if (g.extra) c.extra = (const T*)g.extra + from;
        if (g.sums) c.sums = g.sums + from;
        c.out = (T*)g.out + from;
        k_rows<T, KS, NT, GATED, KIND><<<s.grid, s.wn * s.wr * 64, 0, st>>>(c, s.wn, s.wr, s.subs);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

template <typename T>
hipError_t launch_rows(const GemmArgs& g, int layout, hipStream_t st) {
    const bool gated = g.mode == GEMM_GATED || g.mode == GEMM_GATED_SLOPE;
    const RowsShape s = rows_shape(g.m, g.n, g.k, sizeof(T), gated, g.extra);
    if (!s.grid) return hipErrorInvalidValue;
    constexpr int MOST = ROWS_FRAGS<T>;
    auto go = [&](auto ks, auto nt) -> hipError_t {
        constexpr int KS = decltype(ks)::value, NT = decltype(nt)::value;
        constexpr bool EXTRAS = KS * NT <= ROWS_EXTRA_FRAGS<T> && (sizeof(T) == 2 || NT == 2);
        if (gated) {
            if constexpr (NT == 2 && KS * NT * 2 <= MOST)
                if (g.mode == GEMM_GATED) return start_rows<T, KS, NT, true, ROWS_FORWARD>(g, s, st);
            if constexpr (NT == 2 && KS * NT * 2 <= ROWS_EXTRA_FRAGS<T>)
                if (g.mode == GEMM_GATED_SLOPE) return start_rows<T, KS, NT, true, ROWS_SLOPE>(g, s, st);
            return hipErrorInvalidValue;
        }
        if (g.mode == GEMM_SLOPE) {
            if constexpr (EXTRAS) return start_rows<T, KS, NT, false, ROWS_SLOPE>(g, s, st);
            return hipErrorInvalidValue;
        }
        if (g.extra) {
            if constexpr (EXTRAS) return start_rows<T, KS, NT, false, ROWS_EXTRA>(g, s, st);
            return hipErrorInvalidValue;
        }
        return layout == GEMM_KC_RC ? start_rows<T, KS, NT, false, ROWS_TURNED>(g, s, st) : start_rows<T, KS, NT, false, ROWS_FORWARD>(g, s, st);
    };
    constexpr std::integral_constant<int, 2> two{};
    constexpr std::integral_constant<int, 4> four{};
    constexpr std::integral_constant<int, 8> eight{};
    constexpr std::integral_constant<int, 16> sixteen{};
    if constexpr (sizeof(T) == 4) {
        if (s.tiles == 4) return go(two, four);
        return s.steps == 2 ? go(two, two) : go(four, two);
    } else {
        if (s.tiles == 4) return s.steps == 4 ? go(four, four) : go(eight, four);
        return s.steps == 4 ? go(four, two) : s.steps == 8 ? go(eight, two) : go(sixteen, two);
    }
}

}  // namespace srd

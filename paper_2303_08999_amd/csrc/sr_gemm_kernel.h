// The tile kernel of sr_gemm.h and its launch, instantiated once for each type (sr_gemm_*.hip).
#pragma once
#include "sr_gemm.h"

namespace srd {
namespace {

using gl_void = const __attribute__((address_space(1))) void*;
using lds_void = __attribute__((address_space(3))) void*;
using lds_u4g = __attribute__((address_space(3))) u32x4g;
using lds_f4g = __attribute__((address_space(3))) f32x4g;
using lds_s4g = __attribute__((address_space(3))) s16x4g;
using lds_floatg = __attribute__((address_space(3))) float;

// MT: rows of a matrix instruction.  A wavefront makes WM x WN.
template <int TILE> struct GemmShape;
template <> struct GemmShape<0> { static constexpr int BM = 64, BN = 64, WM = 32, WN = 32, MT = 16, OCC = 3; };
template <> struct GemmShape<1> { static constexpr int BM = 128, BN = 128, WM = 64, WN = 64, MT = 32, OCC = 2; };
template <> struct GemmShape<2> { static constexpr int BM = 256, BN = 256, WM = 128, WN = 64, MT = 32, OCC = 2; };

// One operand's part in LDS: R rows, 128 bytes of k.
template <typename T, int R, int NW, bool RC, int MT>
struct Operand {
    static constexpr int E = 16 / sizeof(T), BK = 128 / sizeof(T), BYTES = R * 128, LOADS = BYTES / 1024 / NW;
    static constexpr int RB = R * sizeof(T);              // bytes of a k in LDS (RC)
    static constexpr int CB = 16 * sizeof(T);             // bytes of a chunk of 16 rows

    // What the chunks of a k are exchanged by.  16-bit types: a turning read takes 4 k of one chunk with 16 lanes; fp32: the lanes
    // read one row each, 32 / MT... 4 rows of k apart.
    static __device__ __forceinline__ int turn(int k) {
        if constexpr (sizeof(T) == 2) return R >= 128 ? (k & 3) | (k >> 3 & 1) << 2 : k & 3;
        else return MT == 32 ? (k >> 2 & 1) << 1 : k >> 2 & 3;
    }

    const char* base[LOADS];    // uniform: of the first row (KC) or k (RC) that load i takes
    int off[LOADS];             // of this lane from it, bytes
    int place;                  // KC: k of its piece; RC: k of the lane within the load
    int row[RC ? LOADS : 1];    // RC: first of its piece's rows, from the tile's first

    // Row r of the tile is row `row_of(r)` of the stored matrix, and none is past `last`.
    template <typename RowOf>
    __device__ __forceinline__ void init(const void* p, int64_t ld, int row0, int rows, int wave, int lane, int k0, bool aligned, RowOf row_of) {
        const char* q = (const char*)p;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int pos = (i * NW + wave) * 1024;
            if constexpr (!RC) {
                const int r = pos / 128 + lane / 8;
                const int first = row_of(pos / 128), mine = row_of(r);
                const int piece = (lane & 7) ^ (lane / 8);                   // a load's first row is a multiple of 8
                base[i] = q + ((int64_t)first * ld + k0) * (int)sizeof(T);
                off[i] = (int)((mine - first) * ld) * (int)sizeof(T) + piece * 16;
                place = piece * E;
            } else {
                const int k = (pos + lane * 16) / RB, k1 = pos / RB, slot = (pos + lane * 16) % RB;
                const int chunk = (slot / CB) ^ turn(k);
                int r = chunk * 16 + (slot % CB) / (int)sizeof(T);
                row[i] = r;
                if (aligned) r = row0 + r < rows ? r : (rows - 1) / E * E - row0;      // what is past the last row is not stored
                base[i] = q + ((int64_t)(k0 + k1) * ld + row0) * (int)sizeof(T);
                off[i] = (int)((k - k1) * ld + r) * (int)sizeof(T);
                if (i == 0) place = k;
            }
        }
    }
    __device__ __forceinline__ void advance(int64_t bytes) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) base[i] += bytes;
    }
    // Straight to LDS; the whole of it is there.
    __device__ __forceinline__ void fetch(char* lds, int wave) const {
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            __builtin_amdgcn_global_load_lds((gl_void)(base[i] + (unsigned)off[i]), (lds_void)(lds + (i * NW + wave) * 1024), 16, 0, 0);
    }
    // By way of registers: `k` values of k are left, rows behind the last are zeros where pieces may be cut
    __device__ __forceinline__ void load(u32x4g v[LOADS], int k, int row0, int rows, bool aligned) const {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            int count;
            if constexpr (!RC) {
                count = k - place;
            } else {
                const int at = place + i * (NW * 1024 / RB);
                count = at >= k ? 0 : aligned ? E : rows - row0 - row[i];
            }
            if (aligned) v[i] = gm_cut<T>(count > 0 ? *(const u32x4g*)(base[i] + off[i]) : u32x4g{0, 0, 0, 0}, count);
            else v[i] = gm_piece((const T*)(base[i] + off[i]), count);
        }
    }
    __device__ __forceinline__ void park(char* lds, int wave, int lane, const u32x4g v[LOADS]) const {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) *(u32x4g*)(lds + (i * NW + wave) * 1024 + lane * 16) = v[i];
    }
};

// Fragments of F x MT rows from row w0 of an operand in LDS.
template <typename T, int R, bool RC, int MT, int F>
struct Reader {
    static constexpr int PIECES = 64 / MT;                // of k, in a matrix step
    int at[RC ? F : 1];
    __device__ __forceinline__ Reader(int w0, int lane) {
        if constexpr (!RC) {
            const int r = lane % MT;
            at[0] = (w0 + r) * 128 + ((lane / MT ^ (r & 7)) << 4);
        } else if constexpr (sizeof(T) == 2) {
            const int g = lane / 16, i = lane % 16;
            const int k = (MT == 32 ? 8 * (g >> 1) : 8 * g) + i / 4;
#pragma unroll
            for (int f = 0; f < F; ++f) {
                const int chunk = (w0 + f * MT) / 16 + (MT == 32 ? g & 1 : 0);
                at[f] = k * R * 2 + ((chunk ^ Operand<T, R, 1, true, MT>::turn(k)) << 5) + (i % 4) * 8;
            }
        } else {
            const int k = lane / MT * 4;
#pragma unroll
            for (int f = 0; f < F; ++f) {
                const int r = w0 + f * MT + lane % MT;
                at[f] = k * R * 4 + ((r / 16 ^ Operand<T, R, 1, true, MT>::turn(k)) << 6) + r % 16 * 4;
            }
        }
    }
    __device__ __forceinline__ u32x4g operator()(const char* lds, int f, int step) const {
        if constexpr (!RC) {
            return *(const u32x4g*)(lds + (at[0] ^ step * PIECES * 16) + f * MT * 128);
        } else if constexpr (sizeof(T) == 2) {
            const char* p = lds + at[f] + step * (PIECES * 8) * R * 2;
            // rows of k + 4 have the same two lowest bits of k, and bit 3 of it: the same turn
            const s16x4g lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4g*)p);
            const s16x4g hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4g*)(p + 4 * R * 2));
            using u2 = __attribute__((ext_vector_type(2))) unsigned;
            const u2 a = __builtin_bit_cast(u2, lo), b = __builtin_bit_cast(u2, hi);
            return u32x4g{a[0], a[1], b[0], b[1]};
        } else {
            const char* p = lds + at[f] + step * (PIECES * 4) * R * 4;
            u32x4g v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = *(const unsigned*)(p + j * R * 4);
            return v;
        }
    }
};

template <typename T, int LAYOUT, bool GATED, bool ALIGNED, int TILE>
__global__ __launch_bounds__(GemmShape<TILE>::BM / GemmShape<TILE>::WM * (GemmShape<TILE>::BN / GemmShape<TILE>::WN) * 64, GemmShape<TILE>::OCC)
void k_gemm(const GemmArgs g) {
    using S = GemmShape<TILE>;
    constexpr int BM = S::BM, BN = S::BN, WM = S::WM, WN = S::WN, MT = S::MT;
    constexpr int NWN = BN / WN, NW = BM / WM * NWN, FM = WM / MT, FN = WN / MT;
    constexpr bool ARC = LAYOUT == GEMM_RC_RC, BRC = LAYOUT != GEMM_KC_KC;
    using OpA = Operand<T, BM, NW, ARC, MT>;
    using OpB = Operand<T, BN, NW, BRC, MT>;
    constexpr int BK = OpA::BK, STEPS = 8 * MT / 64;
    constexpr int PATCH = 32 * (WN + 4) * 4;              // a wavefront's part of the way out
    constexpr int STAGE = OpA::BYTES + OpB::BYTES, LDS = 2 * STAGE > NW * PATCH ? 2 * STAGE : NW * PATCH;
    __shared__ __align__(1024) char lds[LDS];
    using Acc = typename AccOf<MT>::type;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Workgroups go to the eight XCDs in turn: each XCD gets neighbouring tiles, groups of 8 tile rows by all tile columns, whose
    // operands its L2 then holds.
    int tile, split;
    {
        const int tiles = g.tiles_m * g.tiles_n, all = tiles * g.splits, id = blockIdx.x;
        const int share = all >> 3, rest = all & 7, x = id & 7;
        const int t = x * share + (x < rest ? x : rest) + (id >> 3);
        split = t / tiles;
        tile = t - split * tiles;
    }
    const int group = tile / (8 * g.tiles_n), in_group = tile - group * 8 * g.tiles_n;
    const int height = g.tiles_m - group * 8 < 8 ? g.tiles_m - group * 8 : 8;
    const int tm = group * 8 + in_group % height, tn = in_group / height;
    const int m0 = tm * BM, n0 = tn * (GATED ? BN / 2 : BN);
    const int k0 = split * g.ksplit, kn = g.k - k0 < g.ksplit ? g.k - k0 : g.ksplit;

    OpA oa;
    OpB ob;
    oa.init(g.a, g.lda, m0, g.m, wave, lane, k0, ALIGNED, [&](int r) { return m0 + r < g.m ? m0 + r : g.m - 1; });
    // gated: every MT rows of the first half are followed by the same MT of the second
    ob.init(g.b, g.ldb, n0, g.n, wave, lane, k0, ALIGNED, [&](int r) {
        const int c = n0 + (GATED ? r / (2 * MT) * MT + r % MT : r);
        return (c < g.n ? c : g.n - 1) + (GATED && (r & MT) ? g.half : 0);
    });
    const int64_t step_a = (ARC ? g.lda * BK : (int64_t)BK) * (int)sizeof(T), step_b = (BRC ? g.ldb * BK : (int64_t)BK) * (int)sizeof(T);

    const int wm = wave / NWN * WM, wn = wave % NWN * WN;
    const Reader<T, BM, ARC, MT, FM> ra(wm, lane);
    const Reader<T, BN, BRC, MT, FN> rb(wn, lane);
    Acc acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = Acc(0.0f);
    float sum[ARC ? FM : 1];
#pragma unroll
    for (int i = 0; i < (ARC ? FM : 1); ++i) sum[i] = 0.0f;

    auto multiply = [&](const char* s, bool sums) {
#pragma unroll
        for (int step = 0; step < STEPS; ++step) {
            u32x4g fa[FM], fb[FN];
#pragma unroll
            for (int i = 0; i < FM; ++i) fa[i] = ra(s, i, step);
#pragma unroll
            for (int j = 0; j < FN; ++j) fb[j] = rb(s + OpA::BYTES, j, step);
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) gm_mul<T, MT>(acc[i][j], fb[j], fa[i]);
            if constexpr (ARC)
                if (sums)
#pragma unroll
                    for (int i = 0; i < FM; ++i) sum[i] += gm_sum_piece<T>(fa[i]);
        }
    };

    const bool sums = ARC && tn == 0 && wn == 0 && (g.sums || g.sums_out);
    const int full = kn / BK, tail = kn - full * BK;
    auto loop = [&](auto with) {
        constexpr bool SUMS = decltype(with)::value;
        if constexpr (ALIGNED) {
            // the cut tile first, by way of registers; then the others, each fetched while the one before is multiplied
            int buf = 0, left = full;
            if (tail) {
                u32x4g va[OpA::LOADS], vb[OpB::LOADS];
                oa.advance(step_a * full);
                ob.advance(step_b * full);
                oa.load(va, tail, m0, g.m, true);
                ob.load(vb, tail, n0, g.n, true);
                oa.park(lds, wave, lane, va);
                ob.park(lds + OpA::BYTES, wave, lane, vb);
                oa.advance(-step_a * full);
                ob.advance(-step_b * full);
            } else if (left) {
                oa.fetch(lds, wave);
                ob.fetch(lds + OpA::BYTES, wave);
                oa.advance(step_a);
                ob.advance(step_b);
                --left;
            }
            for (int t = full + (tail ? 1 : 0); t > 0; --t) {
                __builtin_amdgcn_s_waitcnt(0);           // this wavefront's part of the tile is in LDS
                __syncthreads();                         // everyone's is, and nobody reads the other buffer any more
                char* const other = lds + (buf ^ 1) * STAGE;
                if (left > 0) {
                    oa.fetch(other, wave);
                    ob.fetch(other + OpA::BYTES, wave);
                    oa.advance(step_a);
                    ob.advance(step_b);
                    --left;
                }
                multiply(lds + buf * STAGE, SUMS);
                buf ^= 1;
            }
        } else {
            const int tiles = full + (tail ? 1 : 0);
            u32x4g va[OpA::LOADS], vb[OpB::LOADS];
            auto load = [&](int t) {
                oa.load(va, kn - t * BK, m0, g.m, false);
                ob.load(vb, kn - t * BK, n0, g.n, false);
                oa.advance(step_a);
                ob.advance(step_b);
            };
            auto park = [&](int t) {
                char* const s = lds + (t & 1) * STAGE;
                oa.park(s, wave, lane, va);
                ob.park(s + OpA::BYTES, wave, lane, vb);
            };
            if (tiles) load(0), park(0);
            for (int t = 0; t < tiles; ++t) {
                __syncthreads();
                if (t + 1 < tiles) load(t + 1);
                multiply(lds + (t & 1) * STAGE, SUMS);
                if (t + 1 < tiles) park(t + 1);
            }
        }
    };
    if constexpr (ARC) {
        if (sums) loop(std::true_type{});
        else loop(std::false_type{});
    } else {
        loop(std::false_type{});
    }
    __syncthreads();

    if constexpr (ARC) {
        if (sums) {                                       // over the lanes that hold other k of the same rows
#pragma unroll
            for (int i = 0; i < FM; ++i) {
#pragma unroll
                for (int d = 32; d >= MT; d >>= 1) sum[i] += __shfl_xor(sum[i], d);
                const int m = m0 + wm + i * MT + lane;
                if (lane < MT && m < g.m) {
                    if (g.sums) g.sums[(int64_t)split * g.m + m] = sum[i];
                    else gm_put((T*)g.sums_out + m, sum[i]);
                }
            }
        }
    }

    if (g.mode == GEMM_PARTIAL ? !g.partial : !g.out) return;

    // The way out: 32 rows of the wavefront's part at a time, lane by lane 8 columns of a row.
    constexpr int STRIDE = WN + 4, OUT = GATED ? WN / 2 : WN, LR = OUT / 8, RI = 64 / LR, PF = 32 / MT;
    float* const patch = (float*)(lds + wave * PATCH);
    const int lc = lane % LR * 8, lr = lane / LR;
    // in the patch a wavefront's columns come as MT of the first half, MT of the second
    const int pc = GATED ? lc / MT * 2 * MT + lc % MT : lc;
    const int col = n0 + (GATED ? wn / 2 : wn) + lc;
    float bz[8], bu[8];
    if (g.mode != GEMM_PARTIAL) gm_bias8<T>(g, col, GATED, bz, bu);
#pragma unroll
    for (int p = 0; p < FM / PF; ++p) {
#pragma unroll
        for (int q = 0; q < PF; ++q)
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                const Acc c = acc[p * PF + q][j];
                float* const w = patch + (q * MT + lane % MT) * STRIDE + j * MT + lane / MT * 4;
                if constexpr (MT == 32) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) *(f32x4g*)(w + 8 * r) = f32x4g{c[4 * r], c[4 * r + 1], c[4 * r + 2], c[4 * r + 3]};
                } else {
                    *(f32x4g*)w = c;
                }
            }
        __builtin_amdgcn_wave_barrier();
#pragma unroll 1
        for (int it = 0; it < 32 / RI; ++it) {
            const int r = it * RI + lr, m = m0 + wm + p * 32 + r;
            float z[8], u[8];
            *(f32x4g*)z = *(const f32x4g*)(patch + r * STRIDE + pc);
            *(f32x4g*)(z + 4) = *(const f32x4g*)(patch + r * STRIDE + pc + 4);
            if constexpr (GATED) {
                *(f32x4g*)u = *(const f32x4g*)(patch + r * STRIDE + pc + MT);
                *(f32x4g*)(u + 4) = *(const f32x4g*)(patch + r * STRIDE + pc + MT + 4);
            }
            if (m < g.m && col < g.n) {
                if (g.mode == GEMM_PARTIAL) gm_put_some(g.partial + ((int64_t)split * g.m + m) * g.n + col, g.n - col, z);
                else gm_finish8<T>(g, m, col, z, u, bz, bu);
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

template <typename T, int LAYOUT, bool GATED, bool ALIGNED, int TILE>
hipError_t start_gemm(const GemmArgs& g, hipStream_t st) {
    using S = GemmShape<TILE>;
    const int64_t blocks = (int64_t)g.tiles_m * g.tiles_n * g.splits;
    if (blocks < 1 || blocks > 0x7fffffff) return hipErrorInvalidValue;
    k_gemm<T, LAYOUT, GATED, ALIGNED, TILE><<<(int)blocks, S::BM / S::WM * (S::BN / S::WN) * 64, 0, st>>>(g);
    return hipGetLastError();
}
template <typename T, int LAYOUT, bool GATED>
hipError_t pick_gemm(const GemmArgs& g, bool aligned, int tile, hipStream_t st) {
    if (!aligned) return tile == 0 ? start_gemm<T, LAYOUT, GATED, false, 0>(g, st) : start_gemm<T, LAYOUT, GATED, false, 1>(g, st);
    return tile == 0 ? start_gemm<T, LAYOUT, GATED, true, 0>(g, st)
         : tile == 1 ? start_gemm<T, LAYOUT, GATED, true, 1>(g, st) : start_gemm<T, LAYOUT, GATED, true, 2>(g, st);
}

}  // namespace

template <typename T>
hipError_t launch_gemm(const GemmArgs& g, int layout, bool aligned, int tile, hipStream_t st) {
    const bool gated = g.mode == GEMM_GATED || g.mode == GEMM_GATED_SLOPE;
    if (layout == GEMM_KC_KC) return gated ? pick_gemm<T, GEMM_KC_KC, true>(g, aligned, tile, st) : pick_gemm<T, GEMM_KC_KC, false>(g, aligned, tile, st);
    if (layout == GEMM_KC_RC) return pick_gemm<T, GEMM_KC_RC, false>(g, aligned, tile, st);
    return pick_gemm<T, GEMM_RC_RC, false>(g, aligned, tile, st);
}

}  // namespace srd

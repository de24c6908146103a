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

// MT: rows of a matrix instruction.  A wavefront makes WM x WN; the matrix instructions read (WM + WN) / (WM WN) of a tile's values from LDS, so that
// 64 x 64 need more of it than it gives, 128 x 128 three quarters.  PIPE: the loop for one wavefront a SIMD.
template <int TILE, typename T> struct GemmShape;
template <typename T> struct GemmShape<0, T> { static constexpr int BM = 64, BN = 64, WM = 32, WN = 32, MT = 16, OCC = 3; static constexpr bool PIPE = false; };
template <typename T> struct GemmShape<1, T> { static constexpr int BM = 128, BN = 128, WM = 64, WN = 64, MT = 32, OCC = 2; static constexpr bool PIPE = false; };
template <typename T> struct GemmShape<2, T> { static constexpr int BM = 256, BN = 128, WM = 128, WN = 64, MT = sizeof(T) == 2 ? 16 : 32, OCC = 1; static constexpr bool PIPE = true; };
// 16-bit types: instructions of 16 rows (8192^3, fp16: 801 us, of 32 rows 876).  fp32 multiplies its three parts in instructions of 32 rows; the smallest tile
// stays with fp32 instructions, where a wavefront has two parts to make for each product (4096^3: 954 us, by parts 1016).
template <typename T> struct GemmShape<3, T> { static constexpr int BM = 256, BN = 256, WM = 128, WN = 128, MT = sizeof(T) == 2 ? 16 : 32, OCC = 1; static constexpr bool PIPE = true; };

template <int TILE, typename T>
constexpr int gemm_threads = GemmShape<TILE, T>::BM / GemmShape<TILE, T>::WM * (GemmShape<TILE, T>::BN / GemmShape<TILE, T>::WN) * 64;

// What this wavefront has sent to LDS is there, then what all of them have, and all of them have read what they asked for.
__device__ __forceinline__ void landed() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __syncthreads();
}

// One operand's part in LDS: R rows, 128 bytes of k.
template <typename T, int R, int NW, bool RC, int MT, bool GATED = false>
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

    const char* base;           // uniform: of the tile's first row and k
    int64_t second;             // gated: from there to the same row of the second half, bytes
    unsigned off[LOADS];        // of this lane's piece of load i from it, bytes (KC: at most 256 rows of 2^17 values)
    int place;                  // KC: k of its piece; RC: k of the lane within load 0
    int row[RC ? LOADS : 1];    // RC: first of its piece's rows, from the tile's first

    // Row r of the tile is row `row0 + row_of(r)` of the stored matrix (KC), which is there.
    template <typename RowOf>
    __device__ __forceinline__ void init(const void* p, int64_t ld, int row0, int rows, int wave, int lane, int k0, bool aligned, int64_t half, RowOf row_of) {
        second = half * ld * (int)sizeof(T);
        base = (const char*)p + (RC ? (int64_t)k0 * ld + row0 : (int64_t)row0 * ld + k0) * (int)sizeof(T);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int pos = (i * NW + wave) * 1024 + lane * 16;
            if constexpr (!RC) {
                const int r = pos / 128, piece = (lane & 7) ^ (r & 7);
                off[i] = (unsigned)row_of(r) * (unsigned)(ld * (int)sizeof(T)) + piece * 16;
                if (i == 0) place = piece * E;
            } else {
                const int k = pos / RB, slot = pos % RB;
                const int chunk = (slot / CB) ^ turn(k);
                int r = chunk * 16 + (slot % CB) / (int)sizeof(T);
                row[i] = r;
                if (aligned) r = row0 + r < rows ? r : (rows - 1) / E * E - row0;      // what is past the last row is not stored
                off[i] = ((unsigned)k * (unsigned)ld + (unsigned)r) * (unsigned)sizeof(T);
                if (i == 0) place = k;
            }
        }
    }
    __device__ __forceinline__ void advance(int64_t bytes) { base += bytes; }
    // gated: whether load i takes rows of the second half (a load's 8 rows are of one)
    static __device__ __forceinline__ bool other(int i, int wave) { return GATED && ((i * NW + wave) * 8 / MT & 1); }
    __device__ __forceinline__ const char* from(int i, int wave) const { return GATED && other(i, wave) ? base + second : base; }
    // Straight to LDS; the whole of it is there.  Written out, because the compiler lets every turning LDS read wait for all loads to LDS that it
    // knows of, whatever they write: landed() is what waits for these.  The instruction takes the place from m0, a wait state behind its writing; the move of the base
    // is that state.  Both moves are scalar and in here, so that no vector instruction has just written what the load reads (it would need five states, which
    // the compiler counts for its own instructions only).
    __device__ __forceinline__ void fetch(char* lds, int wave, int i) const {
        uint64_t at;
        unsigned m0;
        asm volatile("s_mov_b32 %1, %4\n\ts_mov_b64 %0, %3\n\tglobal_load_lds_dwordx4 %2, %0"
                     : "=&s"(at), "=&{m0}"(m0) : "v"(off[i]), "s"(from(i, wave)), "s"((unsigned)(uintptr_t)(lds_void)(lds + (i * NW + wave) * 1024)) : "memory");
    }
    __device__ __forceinline__ void fetch(char* lds, int wave) const {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) fetch(lds, wave, i);
    }
    // fp32 off 16-byte pieces: by 4 bytes, their places worked out anew each time (four times as many registers would not be there).  row_of: as for init;
    // last: of the rows, from the tile's first (RC).
    template <typename RowOf>
    __device__ __forceinline__ void fetch_fours(char* lds, int wave, int lane, int64_t ld, int last, RowOf row_of) const {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const uint64_t p = (uint64_t)from(i, wave);
            const uint64_t uniform = (uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(p >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)p);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int pos = (i * NW + wave) * 1024 + j * 256 + lane * 4;
                unsigned at;
                if constexpr (!RC) {
                    const int r = pos / 128;
                    at = (unsigned)row_of(r) * (unsigned)(ld * 4) + (((pos % 128 / 16) ^ (r & 7)) << 4) + pos % 16;
                } else {
                    const int k = pos / RB, slot = pos % RB, r = ((slot / CB) ^ turn(k)) * 16 + slot % CB / 4;
                    at = ((unsigned)k * (unsigned)ld + (unsigned)(r < last ? r : last)) * 4;
                }
                uint64_t base_at;
                unsigned m0;
                asm volatile("s_mov_b32 %1, %4\n\ts_mov_b64 %0, %3\n\tglobal_load_lds_dword %2, %0"
                             : "=&s"(base_at), "=&{m0}"(m0) : "v"(at), "s"(uniform), "s"((unsigned)(uintptr_t)(lds_void)(lds + (i * NW + wave) * 1024 + j * 256)) : "memory");
            }
        }
    }
    // By way of registers: `k` values of k are left, rows behind the last are zeros where pieces may be cut
    __device__ __forceinline__ void load(u32x4g v[LOADS], int wave, int k, int row0, int rows, bool aligned) const {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            int count;
            if constexpr (!RC) {
                count = k - place;
            } else {
                const int at = place + i * (NW * 1024 / RB);
                count = at >= k ? 0 : aligned ? E : rows - row0 - row[i];
            }
            const char* const p = from(i, wave) + off[i];
            if (aligned) v[i] = gm_cut<T>(count > 0 ? *(const u32x4g*)p : u32x4g{0, 0, 0, 0}, count);
            else v[i] = gm_piece((const T*)p, count);
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

// ALIGN: how operands come to LDS
enum { BY_REGISTERS = 0, BY_PIECES = 1, BY_FOURS = 2 };
template <typename T, int LAYOUT, bool GATED, int ALIGN, int TILE>
__global__ __launch_bounds__((gemm_threads<TILE, T>), (GemmShape<TILE, T>::OCC))
void k_gemm(const GemmArgs g) {
    using S = GemmShape<TILE, T>;
    constexpr int BM = S::BM, BN = S::BN, WM = S::WM, WN = S::WN, MT = S::MT;
    constexpr int NWN = BN / WN, NW = BM / WM * NWN, FM = WM / MT, FN = WN / MT;
    constexpr bool ARC = LAYOUT == GEMM_RC_RC, BRC = LAYOUT != GEMM_KC_KC;
    using OpA = Operand<T, BM, NW, ARC, MT>;
    using OpB = Operand<T, BN, NW, BRC, MT, GATED>;
    constexpr int BK = OpA::BK, STEPS = 8 * MT / 64;
    constexpr int PR = S::PIPE ? 64 : 32, STRIDE = WN + 4, PATCH = PR * STRIDE * 4;      // a wavefront's part of the way out: rows, bytes
    static_assert(BM / WM == 2, "rows of the output's sums");
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
    const auto row_a = [&](int r) { return m0 + r < g.m ? r : g.m - 1 - m0; };
    // gated: every MT rows of the first half are followed by the same MT of the second
    const auto row_b = [&](int r) {
        const int c = GATED ? r / (2 * MT) * MT + r % MT : r;
        return n0 + c < g.n ? c : g.n - 1 - n0;
    };
    oa.init(g.a, g.lda, m0, g.m, wave, lane, k0, ALIGN == BY_PIECES, 0, row_a);
    ob.init(g.b, g.ldb, n0, g.n, wave, lane, k0, ALIGN == BY_PIECES, g.half, row_b);
    const auto fetch_both = [&](char* to) {
        if constexpr (ALIGN == BY_FOURS) {
            oa.fetch_fours(to, wave, lane, g.lda, g.m - 1 - m0, row_a);
            ob.fetch_fours(to + OpA::BYTES, wave, lane, g.ldb, g.n - 1 - n0, row_b);
        } else {
            oa.fetch(to, wave);
            ob.fetch(to + OpA::BYTES, wave);
        }
    };
    const int64_t step_a = (ARC ? g.lda * BK : (int64_t)BK) * (int)sizeof(T), step_b = (BRC ? g.ldb * BK : (int64_t)BK) * (int)sizeof(T);

    const int wm = wave / NWN * WM, wn = wave % NWN * WN;
    const Reader<T, BM, ARC, MT, FM> ra(wm, lane);
    const Reader<T, BN, BRC, MT, FN> rb(wn, lane);
    Acc acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = Acc(0.0f);
    // Sums of A over k (dz over the rows): by a matrix instruction with ones (every n the same), or, where that has no registers left and for
    // fp32, by each lane for its k between the matrix instructions
    constexpr bool ONES = sizeof(T) == 2 && !S::PIPE;
    using Sum = std::conditional_t<ONES, Acc, float>;
    Sum sum[ARC ? FM : 1];
#pragma unroll
    for (int i = 0; i < (ARC ? FM : 1); ++i) sum[i] = Sum(0.0f);
    auto add_sum = [&](int i, u32x4g f) {
        constexpr unsigned one = __is_same(T, __half) ? 0x3c003c00u : 0x3f803f80u;
        if constexpr (ONES) {
            gm_mul<T, MT>(sum[i], u32x4g{one, one, one, one}, f);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[i] = gm_sum<T>(f[j], sum[i]);
        }
    };

    auto multiply = [&](const char* s, bool sums) {
        if constexpr (sizeof(T) == 4 && MT == 32) {
#pragma unroll
            for (int step = 0; step < STEPS; step += 2) {
                Split8 fa[FM], fb[FN];
#pragma unroll
                for (int i = 0; i < FM; ++i) {
                    const u32x4g lo = ra(s, i, step), hi = ra(s, i, step + 1);
                    if constexpr (ARC)
                        if (sums) add_sum(i, lo), add_sum(i, hi);
                    fa[i] = gm_split(lo, hi);
                }
#pragma unroll
                for (int j = 0; j < FN; ++j) fb[j] = gm_split(rb(s + OpA::BYTES, j, step), rb(s + OpA::BYTES, j, step + 1));
#pragma unroll
                for (int part = 0; part < 6; ++part)
#pragma unroll
                    for (int i = 0; i < FM; ++i)
#pragma unroll
                        for (int j = 0; j < FN; ++j) gm_mul_part<MT>(acc[i][j], fb[j], fa[i], part);
            }
            return;
        }
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
                    for (int i = 0; i < FM; ++i) add_sum(i, fa[i]);
        }
    };

    const bool sums = ARC && tn == 0 && wn == 0 && (g.sums || g.sums_out);
    const int full = kn / BK, tail = kn - full * BK;
    auto loop = [&](auto with) {
        constexpr bool SUMS = decltype(with)::value;
        if constexpr (ALIGN != BY_REGISTERS) {
            // the cut tile first, by way of registers; then the others, each fetched while the one before is multiplied
            int buf = 0, left = full;
            if (tail) {
                u32x4g va[OpA::LOADS], vb[OpB::LOADS];
                oa.advance(step_a * full);
                ob.advance(step_b * full);
                oa.load(va, wave, tail, m0, g.m, ALIGN == BY_PIECES);
                ob.load(vb, wave, tail, n0, g.n, ALIGN == BY_PIECES);
                oa.park(lds, wave, lane, va);
                ob.park(lds + OpA::BYTES, wave, lane, vb);
                oa.advance(-step_a * full);
                ob.advance(-step_b * full);
            } else if (left) {
                fetch_both(lds);
                oa.advance(step_a);
                ob.advance(step_b);
                --left;
            }
            if constexpr (S::PIPE) {
                // One wavefront a SIMD: while the matrix instructions of a step go on it reads the fragments of the next.  In a tile's last step everyone has read all of it: the tile behind the next may overwrite
                // it, and the next one, started a tile's time before, is there.
                static_assert(STEPS >= 2 && STEPS % 2 == 0, "fragments of two steps in turn");
                constexpr int NM = FM * FN, NR = FM + FN, NL = OpA::LOADS + OpB::LOADS;
                auto fetch = [&](char* s, int q) {
                    if (q < OpA::LOADS) oa.fetch(s, wave, q);
                    else ob.fetch(s + OpA::BYTES, wave, q - OpA::LOADS);
                };
                auto advance = [&] {
                    oa.advance(step_a);
                    ob.advance(step_b);
                };
                auto none = [](int) {};
                if constexpr (sizeof(T) == 4) {
                    // Two steps at once, as three parts; their values are read while those of the two before are multiplied.
                    constexpr int DOUBLE = STEPS / 2, ALL = 6 * NM;
                    u32x4g fa[FM][2], fb[FN][2];
                    auto read = [&](const char* s, int pair, int q) {
                        if (q < 2 * FM) fa[q / 2][q % 2] = ra(s, q / 2, 2 * pair + q % 2);
                        else fb[q / 2 - FM][q % 2] = rb(s + OpA::BYTES, q / 2 - FM, 2 * pair + q % 2);
                    };
                    auto step = [&](const char* s, int next, auto load) {
                        Split8 pa[FM], pb[FN];
#pragma unroll
                        for (int i = 0; i < FM; ++i) {
                            if constexpr (SUMS) add_sum(i, fa[i][0]), add_sum(i, fa[i][1]);
                            pa[i] = gm_split(fa[i][0], fa[i][1]);
                        }
#pragma unroll
                        for (int j = 0; j < FN; ++j) pb[j] = gm_split(fb[j][0], fb[j][1]);
                        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                        for (int q = 0; q < ALL; ++q) {
                            gm_mul_part<MT>(acc[q % NM / FN][q % FN], pb[q % FN], pa[q % NM / FN], q / NM);
                            const int r0 = 4 * q * NR / ALL, r1 = 4 * (q + 1) * NR / ALL, l0 = q * NL / ALL, l1 = (q + 1) * NL / ALL;
                            if ((r1 > r0 && r0 < 2 * NR) || l1 > l0) {
                                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                                for (int r = r0; r < r1; ++r)
                                    if (r < 2 * NR) read(s, next, r);
#pragma unroll
                                for (int l = l0; l < l1; ++l) load(l);
                                __builtin_amdgcn_sched_barrier(0);
                            }
                        }
                    };
                    auto tile = [&](auto later) {
                        char *const now = lds + buf * STAGE, *const next = lds + (buf ^ 1) * STAGE;
#pragma unroll
                        for (int i = 0; i + 1 < DOUBLE; ++i) step(now, i + 1, none);
                        landed();
                        step(next, 0, [&](int q) {
                            if constexpr (decltype(later)::value) fetch(now, q);
                        });
                        advance();
                        buf ^= 1;
                    };
                    landed();
                    if (full + (tail ? 1 : 0) > 0) {
#pragma unroll
                        for (int q = 0; q < 2 * NR; ++q) read(lds, 0, q);
                        if (left > 0) {
#pragma unroll
                            for (int q = 0; q < NL; ++q) fetch(lds + STAGE, q);
                            advance();
                            for (; left > 1; --left) tile(std::true_type{});
                            tile(std::false_type{});
                        }
                        tile(std::false_type{});
                    }
                    return;
                }
                u32x4g fa[2][FM], fb[2][FN];
                auto read = [&](int into, const char* s, int step, int q) {
                    if (q < FM) fa[into][q] = ra(s, q, step);
                    else fb[into][q - FM] = rb(s + OpA::BYTES, q - FM, step);
                };
                // The reads in the first half of a step, so that they are there when it ends; the loads all through it: one in every fourth instruction of
                // 16 rows, 8192^3 767 us; in every second 791; half of them in the step after 827.
                auto step = [&](int now, const char* s, int next, auto load) {
#pragma unroll
                    for (int q = 0; q < NM; ++q) {
                        gm_mul<T, MT>(acc[q / FN][q % FN], fb[now][q % FN], fa[now][q / FN]);
                        if constexpr (SUMS) {
#pragma unroll
                            for (int d = q * 4 * FM / NM; d < (q + 1) * 4 * FM / NM; ++d) sum[d / 4] = gm_sum<T>(fa[now][d / 4][d % 4], sum[d / 4]);
                        }
                        const int r0 = 2 * q * NR / NM, r1 = 2 * (q + 1) * NR / NM, l0 = q * NL / NM, l1 = (q + 1) * NL / NM;
                        if ((r1 > r0 && r0 < NR) || l1 > l0) {
                            __builtin_amdgcn_sched_barrier(0);       // this order is kept
#pragma unroll
                            for (int r = r0; r < r1; ++r)
                                if (r < NR) read(now ^ 1, s, next, r);
#pragma unroll
                            for (int l = l0; l < l1; ++l) load(l);
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    }
                };
                // `later`: the tile behind the next is still to be fetched
                auto tile = [&](auto later) {
                    char *const now = lds + buf * STAGE, *const next = lds + (buf ^ 1) * STAGE;
#pragma unroll
                    for (int i = 0; i + 1 < STEPS; ++i) step(i & 1, now, i + 1, none);
                    landed();
                    step(1, next, 0, [&](int q) {
                        if constexpr (decltype(later)::value) fetch(now, q);
                    });
                    advance();
                    buf ^= 1;
                };
                landed();
                if (full + (tail ? 1 : 0) > 0) {
#pragma unroll
                    for (int q = 0; q < NR; ++q) read(0, lds, 0, q);
                    if (left > 0) {
#pragma unroll
                        for (int q = 0; q < NL; ++q) fetch(lds + STAGE, q);
                        advance();
                        for (; left > 1; --left) tile(std::true_type{});
                        tile(std::false_type{});
                    }
                    tile(std::false_type{});
                }
            } else
            for (int t = full + (tail ? 1 : 0); t > 0; --t) {
                landed();                                // everyone's part of the tile is in LDS, and nobody reads the other buffer any more
                char* const other = lds + (buf ^ 1) * STAGE;
                if (left > 0) {
                    fetch_both(other);
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
                oa.load(va, wave, kn - t * BK, m0, g.m, false);
                ob.load(vb, wave, kn - t * BK, n0, g.n, false);
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
    const char* const a0 = oa.base;
    const char* const b0 = ob.base;
    for (int part = 0;; ++part) {
        if constexpr (ARC) {
            if (sums) loop(std::true_type{});
            else loop(std::false_type{});
        } else {
            loop(std::false_type{});
        }
        __syncthreads();
        if (S::PIPE || sizeof(T) == 4 || LAYOUT == GEMM_KC_KC || part || !g.a_lo) break;
        oa.base = a0 + g.a_lo * (int)sizeof(T);            // A's second part
        ob.base = b0;
    }

    if constexpr (ARC) {
        if (sums) {
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                float v;
                if constexpr (ONES) {
                    v = sum[i][0];
                } else {
                    v = sum[i];                            // over the lanes that hold other k of the same rows
#pragma unroll
                    for (int d = 32; d >= MT; d >>= 1) v += __shfl_xor(v, d);
                }
                const int m = m0 + wm + i * MT + lane;
                if (lane < MT && m < g.m) {
                    if (g.sums) g.sums[(int64_t)split * g.m + m] = v;
                    else gm_put((T*)g.sums_out + m, v);
                }
            }
        }
    }

    if (g.mode == GEMM_PARTIAL ? !g.partial : !g.out) return;

    // The way out: PR rows of the wavefront's part at a time, a lane 8 columns of U rows, what is to be added to them or multiplied with on its way
    // while the U rows before are finished.
    constexpr int OUT = GATED ? WN / 2 : WN, LR = OUT / 8, RI = 64 / LR, PF = PR / MT, U = PR / RI < 4 ? PR / RI : 4, CHUNKS = PR / RI / U;
    float* const patch = (float*)(lds + wave * PATCH);
    const int lc = lane % LR * 8, lr = lane / LR;
    // in the patch a wavefront's columns come as MT of the first half, MT of the second
    const int pc = GATED ? lc / MT * 2 * MT + lc % MT : lc;
    const int col = n0 + (GATED ? wn / 2 : wn) + lc, count = g.n - col;
    const int row = m0 + wm + lr;
    const bool extra = g.extra && g.mode != GEMM_PARTIAL;
    Raw8<T> next[U];
    auto ask = [&](int c) {
#pragma unroll
        for (int r = 0; r < U; ++r) {
            const int m = row + (c * U + r) * RI;
            next[r].get((const T*)g.extra + (int64_t)m * g.ld_extra + col, m < g.m ? count : 0);
        }
    };
    if (extra) ask(0);
    // sums of dz over the rows (db), on the way: beside dW's matrix instructions they cost the workgroups that take them a sixth (8192 rows of 2048 to
    // 4096: 14 us of 146)
    constexpr bool SLOPES = LAYOUT == GEMM_KC_KC;
    float sz[8], su[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sz[i] = su[i] = 0.0f;
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
        for (int c = 0; c < CHUNKS; ++c) {
            float z[U][8], u[U][8], e[U][8];
#pragma unroll
            for (int r = 0; r < U; ++r) {
                const float* const s = patch + ((c * U + r) * RI + lr) * STRIDE + pc;
                *(f32x4g*)z[r] = *(const f32x4g*)s;
                *(f32x4g*)(z[r] + 4) = *(const f32x4g*)(s + 4);
                if constexpr (GATED) {
                    *(f32x4g*)u[r] = *(const f32x4g*)(s + MT);
                    *(f32x4g*)(u[r] + 4) = *(const f32x4g*)(s + MT + 4);
                }
            }
            const int first = row + (p * CHUNKS + c) * U * RI;
            if (g.mode == GEMM_PARTIAL) {
#pragma unroll
                for (int r = 0; r < U; ++r)
                    if (first + r * RI < g.m && count > 0) gm_put_some(g.partial + ((int64_t)split * g.m + first + r * RI) * g.n + col, count, z[r]);
                continue;
            }
            if (extra) {
#pragma unroll
                for (int r = 0; r < U; ++r) next[r].values(e[r]);
                if (p * CHUNKS + c + 1 < FM / PF * CHUNKS) ask(p * CHUNKS + c + 1);
            } else {
#pragma unroll
                for (int r = 0; r < U; ++r)
#pragma unroll
                    for (int i = 0; i < 8; ++i) e[r][i] = 0.0f;
            }
#pragma unroll
            for (int r = 0; r < U; ++r)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    z[r][i] += bz[i];
                    if constexpr (GATED) u[r][i] += bu[i];
                }
            gm_finish<GATED, U>(g, z, u, e);
#pragma unroll
            for (int r = 0; r < U; ++r) {
                const int m = first + r * RI;
                if (m < g.m && count > 0) {
                    if (SLOPES && g.sums) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            sz[i] += z[r][i];
                            if constexpr (GATED) su[i] += u[r][i];
                        }
                    }
                    T* const out = (T*)g.out + (int64_t)m * g.ld_out + col;
                    const int64_t lo = S::PIPE ? 0 : g.out_lo;
                    gm_put_parts(out, lo, count, z[r]);
                    if (GATED && g.mode == GEMM_GATED_SLOPE) gm_put_parts(out + g.half, lo, count, u[r]);
                }
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
    if (SLOPES && g.sums && g.mode != GEMM_PARTIAL) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int d = LR; d < 64; d <<= 1) {
                sz[i] += __shfl_xor(sz[i], d);
                if constexpr (GATED) su[i] += __shfl_xor(su[i], d);
            }
        if (lr == 0 && count > 0) {
            float* const s = g.sums + (int64_t)(2 * tm + wm / WM) * (GATED ? 2 * (int64_t)g.half : g.n) + col;
            gm_put_some(s, count, sz);
            if (GATED) gm_put_some(s + g.half, count, su);
        }
    }
}

template <typename T, int LAYOUT, bool GATED, int ALIGN, int TILE>
hipError_t start_gemm(const GemmArgs& g, hipStream_t st) {
    const int64_t blocks = (int64_t)g.tiles_m * g.tiles_n * g.splits;
    if (blocks < 1 || blocks > 0x7fffffff) return hipErrorInvalidValue;
    k_gemm<T, LAYOUT, GATED, ALIGN, TILE><<<(int)blocks, gemm_threads<TILE, T>, 0, st>>>(g);
    return hipGetLastError();
}
template <typename T, int LAYOUT, bool GATED>
hipError_t pick_gemm(const GemmArgs& g, bool aligned, int tile, hipStream_t st) {
    // fp32 is on 4 bytes wherever it is
    constexpr int OFF = sizeof(T) == 4 ? BY_FOURS : BY_REGISTERS;
    if (!aligned) return tile == 0 ? start_gemm<T, LAYOUT, GATED, OFF, 0>(g, st) : start_gemm<T, LAYOUT, GATED, OFF, 1>(g, st);
    if (tile == 0) return start_gemm<T, LAYOUT, GATED, BY_PIECES, 0>(g, st);
    if (tile == 1) return start_gemm<T, LAYOUT, GATED, BY_PIECES, 1>(g, st);
    return tile == 2 ? start_gemm<T, LAYOUT, GATED, BY_PIECES, 2>(g, st) : start_gemm<T, LAYOUT, GATED, BY_PIECES, 3>(g, st);
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

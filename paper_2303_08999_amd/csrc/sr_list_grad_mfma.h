// Gradient of the per-pixel list form on the matrix cores: lists of up to 16 entries, up to 128 atoms, one or three channels.
//
// Both gradients are products with E, the gradient of a pixel's filter (k^2 numbers a pixel):
//     responses  R[l][i] = sum_j D[l][j] E[j][i]       of which a pixel's listed ones are its dvalue
//     ddict      G[l][j] = sum_i Phi[l][i] E[j][i]     Phi the lists as dense columns
// v_mfma_f32_16x16x32_f16 serves both: for R the sum runs over the taps, so lane (q, n) forms taps 8 q .. 8 q + 7 of pixel n of a
// group of 16, which is the operand as it lies in its registers; for G it runs over the 32 pixels of a unit, so E goes through LDS
// and comes back turned, the lists are scattered into a dense [atom][pixel] array that is all zero between uses, and R goes through LDS
// for its gather.  All of that is a wavefront's own scratch: no barrier but around the up-sampled tile.
//
// Precision: fp16 products with fp32 sums.  E is scaled pixel by pixel by a power of two (to 2^14 .. 2^15) and split in two fp16
// numbers, each the nearest: 2^-23 is left.  D likewise, atom by atom; R takes three products, and leaves out the low parts' (2^-22 of a
// term at most, 2^-24.6 as the operands fall: dvalue of a crop is off by 4.9e-8 of its norm, 4.7e-8 with the fourth, which takes a 4K frame
// 9 us; summed in fp32 8.6e-8).
// For G the pixels of a unit share the largest one's power of two (or up to four times that).  Those that are 2^16 and more below it, whose
// lower parts fp16 would cut off, take it less whole steps of 2^16 and are added after the others, in a product of their own for each
// distance: an atom that quiet pixels alone name has its bits, down to 2^-100 of the run's largest E.  (4K frame of 8 entries of 72 in fp16:
// 422 us, 417 without it; 750 where every unit has one such pixel, 1030 where it has two distances of them, 720 where every unit has an atom
// listed twice, which goes the same way: what the frequent case takes of registers went first.)
// fp16 values enter as they are and the sums stay in the matrix instructions.  fp32 ones are split as well, the low part kept 2^11 higher, under
// one power of two: those that are 2^28 and more below the largest wait likewise (softmax lists of logits of deviation 8, where most units have
// such a value: a 4K frame 814 -> 1540 us); a unit's sums are added unscaled.  Both are fp32, and handed on in double after at most 4096
// pixels of a wavefront.
// The matrix instructions cut off below: their sums are a little too low, whatever the sign, which adds up over a frame where the gradients
// cancel.  So every other wavefront sums -E, in a workgroup and from one workgroup to the next (in images of two rows a tile has one
// wavefront's work; without it fp32 values' ddict is off by 2.2e-6 of its norm there): a 4K frame's is off by 4.3e-7 to 5.3e-7, 1.4e-6 without.
//
// Loops: all lanes of a wavefront take the same number of turns, with what is beyond the end done twice or set aside, and nothing that
// differs between lanes is kept in a register across a loop that some lanes leave early.  This is for safety, not for speed: where this
// kernel's registers run out the compiler (ROCm 7.2) copies values to accumulation registers, and it has put such copies at the exit of a
// loop that lanes left one by one, before it switched the lanes on again.  Nothing was copied, and what was read back as an address later
// was not one: a memory fault, with more than 80 atoms.
//
// What bounds it: none of memory (438 MB of a 4K frame of 8 entries, 89 us), vector ALU (188 us), LDS (204 us, of which 58 bank conflicts of the
// gather and the scatter, whose rows are the lists') and matrix cores (84 us) alone: 422 us with 2 wavefronts per SIMD, whose registers
// (235) and LDS (81 KB a workgroup) leave no room for a third.  A unit's chain through LDS and the matrix cores is four round trips
// long.  One wavefront per SIMD where the registers end: 7x7 atoms, more than 80 atoms, fp32 values (a
// 1080p frame of 16 entries of 128 atoms of 7x7 484 us; 8 entries of 72 in fp32 227 us, in fp16 129).
#pragma once
#include "sr_list_grad.h"

namespace srd {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef unsigned u32x4v __attribute__((ext_vector_type(4)));
// LDS scratch is read under other types than it is written
typedef float4v __attribute__((may_alias)) lds_f4;
typedef float __attribute__((may_alias)) lds_f;
typedef u32x4v __attribute__((may_alias)) lds_u4;
typedef unsigned __attribute__((may_alias)) lds_u;
typedef unsigned short __attribute__((may_alias)) lds_h;
typedef short short4v __attribute__((ext_vector_type(4)));
typedef short4v __attribute__((address_space(3), may_alias))* lds_turned;

template <int K, int LP, int CM, int TQ, typename TV>
struct GradCfg {
    static constexpr int KK = K * K, R = (K - 1) / 2, MT = LP / 16;
    // Taps in the operands' places (s, q, i), of which 8 q + i is the place in a sum over 32: lanes q have row 4 s + q of the patch, so
    // that the four groups of 16 lanes read four rows of the tile, 16 banks apart; 5x5 atoms have their fifth row in two places more.
    static constexpr int NS = (K + 2) / 4, NI = K == 5 ? 7 : K, NT = 2 * NS;
    static constexpr int UW = GM_TW + K - 1, UH = GM_TH + K - 1, UP = 80;             // the tile, its pitch (16 modulo 64)
    static constexpr int MAXLRX = (UW - 1) / 2 + 5, MAXLRY = (UH - 1) / 2 + 5;       // scale >= 2
    static constexpr int UN = CM * UH * UP, VN = CM * UH * MAXLRX;
    static constexpr bool SPLIT = sizeof(TV) == 4;                                     // values in two parts
    static constexpr int PP = 40;                  // pitch of Phi in halves: 16 rows' 16-byte pieces fall on all 64 banks
    static constexpr int EP = 64 * NS + 16;        // pitch of a pixel's taps in bytes, likewise
    static constexpr int RP = LP + 4;              // pitch of a pixel's responses, likewise
    static constexpr int PHI_ROWS = LP + 1;        // the last one takes what is not to be added
    static constexpr int PHI_B = PHI_ROWS * PP * 2 * (SPLIT ? 2 : 1);
    static constexpr int R_B = 16 * RP * 4;        // responses of a group
    // Groups whose responses are formed together: two hide each other's latency, one takes fewer registers and less scratch.
    static constexpr int RG = (K == 7 && LP > 80) || (TQ == 4 && LP <= 80 && !SPLIT) ? 1 : 2;
    static constexpr int ER_0 = 2 * 32 * EP > RG * R_B ? 2 * 32 * EP : RG * R_B;
    static constexpr int ER_B = ER_0 > VN * 4 ? ER_0 : (VN * 4 + 15) / 16 * 16;
    static constexpr int WAVE_B = PHI_B + ER_B;
    static constexpr bool DL = K == 7 && LP > 80 && !SPLIT;                            // D's operands in LDS, not in 128 registers
    // Two fp16 numbers hold 2^14 .. 2^15 down to 2^-25: a number that is less than this many powers of two below keeps fp32's half step.
    static constexpr int STEP = 16;
    static constexpr int VSTEP = 28;               // ... of a value, whose low part is kept 2^11 higher
    static constexpr bool ACC = !SPLIT;            // G is summed by the matrix instructions, under one power of two
    static constexpr int WPE = K == 7 || LP > 80 || SPLIT ? 1 : 2;                     // wavefronts per SIMD (registers, LDS)
    static_assert(LP * 16 * 4 <= ER_B && CM * MAXLRY * MAXLRX <= UN && VN * 4 <= ER_B && MAXLRX <= 64 && 3 * UW <= 256, "stage 1 fits where it goes");
    // the tap at a place, or -1
    static __device__ __forceinline__ int tap(int s, int q, int i) {
        const int row = 4 * s + q;
        if (i < K) return row < K ? row * K + i : -1;
        if (K == 5 && i == 5) return 20 + q;
        return K == 5 && i == 6 && q == 0 ? 24 : -1;
    }
};

__device__ __forceinline__ void wave_lds_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
// The largest of a row of 16 lanes, in all of them; over the four rows of a wavefront.
template <int CTRL> __device__ __forceinline__ int row_turned(int v) { return __builtin_amdgcn_update_dpp(v, v, CTRL, 0xf, 0xf, false); }
__device__ __forceinline__ int row_max(int v) {
    v = max(v, row_turned<0x128>(v));                // row_ror 8, 4, 2, 1
    v = max(v, row_turned<0x124>(v));
    v = max(v, row_turned<0x122>(v));
    return max(v, row_turned<0x121>(v));
}
__device__ __forceinline__ int wave_min(int v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v = min(v, __shfl_xor(v, d));
    return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ float rows_max(float v) {
    const unsigned u = __float_as_uint(v);           // magnitudes: their order is that of their bits
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const unsigned b = max(a[0], a[1]);
    const auto c = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    return __uint_as_float(max(c[0], c[1]));
}
// 2^n for an exponent field (n + 127), kept where fp32 has it
__device__ __forceinline__ float pow2_field(int field) { return __uint_as_float((unsigned)clampi(field, 1, 254) << 23); }
// exponent field of a magnitude, from 15 on: its reciprocal scale below stays a number
__device__ __forceinline__ int exponent_field(float m) { return clampi((int)(__float_as_uint(m) >> 23), 15, 254); }

// x and y, times sc into fp16's range -> words (high part, low part), each the nearest: both together are off by 2^-23 at most; sc is a
// power of two
__device__ __forceinline__ half2v nearest_pair(float x, float y) { return __builtin_convertvector((float2v){x, y}, half2v); }
__device__ __forceinline__ void split_pair(float x, float y, float sc, unsigned& hi, unsigned& lo) {
    const half2v h = nearest_pair(x * sc, y * sc);
    hi = __builtin_bit_cast(unsigned, h);
    lo = __builtin_bit_cast(unsigned, nearest_pair(fmaf(x, sc, -(float)h[0]), fmaf(y, sc, -(float)h[1])));
}

// x, times sc into fp16's range -> a word: the high part, and the low part times 2^11, which has the same exponents
__device__ __forceinline__ unsigned split_value(float x, float sc) {
    const _Float16 h = (_Float16)(x * sc);
    return __builtin_bit_cast(unsigned, nearest_pair(x * sc, fmaf(x, sc, -(float)h) * 2048.0f));
}

// A stored value's bits, and the value
template <typename T> struct Bits { typedef unsigned short type; };
template <> struct Bits<float> { typedef unsigned type; };
__device__ __forceinline__ float from_bits(unsigned b, const __half*) { return __half2float(__ushort_as_half((unsigned short)b)); }
__device__ __forceinline__ float from_bits(unsigned b, const float*) { return __uint_as_float(b); }

// What a unit needs of memory, as it is stored, requested one unit ahead.
template <int CM, int TQ> struct GradFetch {
    unsigned dy[2][CM], idx[2][TQ], val[2][TQ], on[2];
};

template <int K, int LP, int CM, int TQ, typename TV, typename TIO>
__global__ __launch_bounds__(256, (GradCfg<K, LP, CM, TQ, TV>::WPE))
void k_list_grad_mfma(const ListGradArgs a) {
    using F = GradCfg<K, LP, CM, TQ, TV>;
    constexpr int KK = F::KK, R = F::R, NS = F::NS, NI = F::NI, NT = F::NT, MT = F::MT, UW = F::UW, UH = F::UH, UP = F::UP;
    constexpr int MAXLRX = F::MAXLRX, MAXLRY = F::MAXLRY;
    constexpr int UNITS = GM_TH * 2 / 4;             // of a wavefront in a tile
    constexpr unsigned VB = sizeof(TV), IB = sizeof(TIO);
    typedef typename Bits<TIO>::type io_bits;
    typedef typename Bits<TV>::type value_bits;
    __shared__ float U[F::UN];                       // up-sampled tile; before that, in its place, the LR footprint
    __shared__ float4 yw[UH];                        // a tile's rows: weights, first LR row
    __shared__ int yb[UH];
    __shared__ __align__(16) unsigned char scratch[4][F::WAVE_B];
    __shared__ int dback[LP];                        // of an atom: what undoes its power of two, and what is common to every pixel's
    __shared__ u32x4v Dsh[F::DL ? 2 * MT * NS * 64 : 1];

    const int tid = threadIdx.x, lane = tid & 63, q = lane >> 4, n = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    unsigned char* const phi = scratch[wave];
    unsigned char* const er = scratch[wave] + F::PHI_B;
    float* const V = (float*)(scratch[0] + F::PHI_B);      // after the vertical pass
    const int64_t plane = (int64_t)a.H * a.W;
    const unsigned lmax = (unsigned)a.L - 1u;

    // ---- the dictionary as operands of R: lane (q, n) has atom 16 mt + n, taps 32 s + 8 q and on, the atom times a power of two (to
    // 2^14 .. 2^15)
    for (int e = 0; e < F::PHI_B / 16; e += 64) ((lds_u4*)phi)[min(e + lane, F::PHI_B / 16 - 1)] = (u32x4v){0, 0, 0, 0};
    u32x4v Dh[F::DL ? 1 : MT][NS], Dl[F::DL ? 1 : MT][NS];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        if (F::DL && (mt & 3) != wave) continue;
        const int l = 16 * mt + n;
        float v[NS][8], big = 0.0f;
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int j = F::tap(s, q, i);
                v[s][i] = l < a.L && j >= 0 ? a.dict[l * KK + j] : 0.0f;
                big = fmaxf(big, fabsf(v[s][i]));
            }
        const int dx = exponent_field(rows_max(big));
        const float dscale = pow2_field(268 - dx);
        dback[l] = dx - 2 * (127 + 14);              // (the four lanes of an atom write the same)
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            u32x4v dh, dl;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                unsigned hi, lo;
                split_pair(v[s][2 * i], v[s][2 * i + 1], dscale, hi, lo);
                dh[i] = hi, dl[i] = lo;
            }
            if (F::DL) Dsh[F::DL ? 2 * (mt * NS + s) * 64 + lane : 0] = dh, Dsh[F::DL ? (2 * (mt * NS + s) + 1) * 64 + lane : 0] = dl;
            else Dh[F::DL ? 0 : mt][s] = dh, Dl[F::DL ? 0 : mt][s] = dl;
        }
    }
    // where a lane's taps are in the tile, from the wavefront's first row on, in bytes (places without one: the patch's last tap; their
    // responses meet zeros of D, their columns of G are not handed on)
    int tap[NS][NI];
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int j = F::tap(s, q, i) < 0 ? KK - 1 : F::tap(s, q, i);
            tap[s][i] = 4 * ((wave * (GM_TH / 4) + j / K) * UP + j % K + n);
        }
    float4v G[MT][NT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int t = 0; t < NT; ++t) G[mt][t] = (float4v){0, 0, 0, 0};
    // every other wavefront sums -E, of its workgroup and of those that are at the same rows of the tiles
    const float turn = (wave ^ blockIdx.x) & 1 ? -1.0f : 1.0f;
    double* const rec = a.partial ? a.partial + (size_t)blockIdx.x * a.L * KK : nullptr;
    bool first = true;
    int held = 0, scale = 15, top = 15;              // G times 2^(scale - 14) is the sum (ACC); the largest scale that this G has had

    struct Tile { int im, Y0, X0; int64_t list, image; };   // (elements before its lists, before its dout)
    auto tile_at = [&](unsigned t) -> Tile {
        const unsigned per = (unsigned)a.tiles_x * (unsigned)a.tiles_y, im = t / per, in = t - im * per, ty = in / (unsigned)a.tiles_x;
        return {(int)im, (int)ty * GM_TH, (int)(in - ty * (unsigned)a.tiles_x) * GM_TW, (int64_t)im * a.T * plane, (int64_t)im * CM * plane};
    };
    // Requests a unit: lane (q, n) has of pixel n of either group the entries 4 r + q.  Every address is one of the tensors'; what is outside of
    // the image or the list is set aside when it is used.  An image's lists and its dout lie within 32-bit offsets.
    // (No branch in here, and every load widened where it is made: a value that is first touched in another block is waited for there.)
    const unsigned pl = (unsigned)plane, unmasked = a.mask ? 0u : 1u;
    unsigned entry[TQ];
#pragma unroll
    for (int r = 0; r < TQ; ++r) entry[r] = (unsigned)min(4 * r + q, a.T - 1) * pl;
    auto fetch = [&](GradFetch<CM, TQ>& f, const Tile& t, int u) {
        const int Y = min(t.Y0 + wave * (GM_TH / 4) + u / 2, a.H - 1), X = min(t.X0 + u % 2 * 32, a.W - 1);
        const unsigned at = (unsigned)Y * (unsigned)a.W + (unsigned)X;     // the same for the whole wavefront
        const unsigned char* const index = a.index + t.list;
        const char* const value = (const char*)a.value + t.list * VB;
        const char* const dout = (const char*)a.dout + t.image * IB;
        const unsigned char* const mask = a.mask ? a.mask + t.im * plane : index;      // without one: some byte, made 1 below
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const unsigned x = at + (unsigned)min(16 * g + n, a.W - 1 - X);
            f.on[g] = mask[x];
#pragma unroll
            for (int c = 0; c < CM; ++c) f.dy[g][c] = *(const io_bits*)(dout + (unsigned)c * (pl * IB) + x * IB);
#pragma unroll
            for (int r = 0; r < TQ; ++r) {
                const unsigned e = entry[r] + x;
                f.idx[g][r] = index[e];
                f.val[g][r] = *(const value_bits*)(value + e * VB);
            }
        }
    };

    // Requests a tile's LR rows, every fourth one a wavefront's, a tile ahead.  (An image's channels lie within 32-bit offsets.)
    constexpr int LRI = (MAXLRY + 3) / 4, VI = (UH + 3) / 4;
    const int lane_x = min(lane, MAXLRX - 1);
    unsigned lrv[CM][LRI];
    auto fetch_lr = [&](const Tile& t) {
        const TileOrigin o = tile_origin(t.Y0, t.X0, R, UH, UW, a.H, a.W, a.s);
        const unsigned x = (unsigned)clampi(o.lx0 + lane_x, 0, a.w - 1), lp = (unsigned)a.h * (unsigned)a.w;
        unsigned row[LRI];
#pragma unroll
        for (int i = 0; i < LRI; ++i) row[i] = (unsigned)clampi(o.ly0 + min(wave + 4 * i, MAXLRY - 1), 0, a.h - 1) * (unsigned)a.w;
        const char* const lr = (const char*)a.lr + (int64_t)t.im * CM * lp * IB;
#pragma unroll
        for (int c = 0; c < CM; ++c)
#pragma unroll
            for (int i = 0; i < LRI; ++i) lrv[c][i] = *(const io_bits*)(lr + ((unsigned)c * lp + row[i]) * IB + x * IB);
    };

    const unsigned tiles = (unsigned)a.tiles;
    unsigned tile = blockIdx.x;
    GradFetch<CM, TQ> next;
    Tile tn = tile_at(tile);
    fetch_lr(tn);
    fetch(next, tn, 0);
    for (; tile < tiles; tile += gridDim.x) {
        const Tile tl = tn;
        const bool last = tile + gridDim.x >= tiles;
        if (!last) tn = tile_at(tile + gridDim.x);
        // ---- stage 1 of all channels, the values of sr_device.h; every loop has the same number of turns for all lanes (see Loops above).  LR rows and rows
        // after the vertical pass are a wavefront's each, columns of the tile a thread's, whose weights stay in registers.
        const TileOrigin o = tile_origin(tl.Y0, tl.X0, R, UH, UW, a.H, a.W, a.s);
        __syncthreads();                             // the last tile has been used
        if (tid < UH) {
            int m;
            const int f = src_floor(clampi(tl.Y0 + tid - R, 0, a.H - 1), a.s, m);
            float wt[4];
            keys_weights(m, a.s, wt);
            yw[tid] = make_float4(wt[0], wt[1], wt[2], wt[3]);
            yb[tid] = clampi(f - 1 - o.ly0, 0, MAXLRY - 4);
        }
#pragma unroll
        for (int c = 0; c < CM; ++c)
#pragma unroll
            for (int i = 0; i < LRI; ++i) {
                U[(c * MAXLRY + min(wave + 4 * i, MAXLRY - 1)) * MAXLRX + lane_x] = from_bits(lrv[c][i], (const TIO*)nullptr);
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < VI; ++i) {
            const int yy = min(wave + 4 * i, UH - 1);
            const float4 w4 = yw[yy];
            const float wt[4] = {w4.x, w4.y, w4.z, w4.w};
            const float* r = U + yb[yy] * MAXLRX + lane_x;
#pragma unroll
            for (int c = 0; c < CM; ++c, r += MAXLRY * MAXLRX)
                V[(c * UH + yy) * MAXLRX + lane_x] = dot4(wt, r[0], r[MAXLRX], r[2 * MAXLRX], r[3 * MAXLRX]);
        }
        __syncthreads();
        {
            const int col = min(tid, 3 * UW - 1), third = col / UW, xx = col - third * UW;
            int m;
            const int f = src_floor(clampi(tl.X0 + xx - R, 0, a.W - 1), a.s, m);
            float wt[4];
            keys_weights(m, a.s, wt);
            const float* r = V + third * MAXLRX + clampi(f - 1 - o.lx0, 0, MAXLRX - 4);
            float* to = U + third * UP + xx;
#pragma unroll 4
            for (int i = 0; i < CM * UH / 3; ++i, r += 3 * MAXLRX, to += 3 * UP) *to = dot4(wt, r[0], r[1], r[2], r[3]);
            if (CM * UH % 3 && third < CM * UH % 3) *to = dot4(wt, r[0], r[1], r[2], r[3]);
        }
        __syncthreads();


        // ---- a wavefront's units: 32 pixels of a row, two groups of 16
#pragma unroll 1
        for (int u = 0; u < UNITS; ++u) {
            const int Y = tl.Y0 + wave * (GM_TH / 4) + u / 2, x0 = u % 2 * 32;
            GradFetch<CM, TQ> f = next;
            if (u + 1 < UNITS || !last) fetch(next, u + 1 < UNITS ? tl : tn, (u + 1) % UNITS);
            if (u == 1 && !last) fetch_lr(tn);       // (not before the first unit, which would wait for these rows as well)
            if (Y >= a.H || tl.X0 + x0 >= a.W) continue;
            const char* const Ub = (const char*)U + 4 * (u / 2 * UP + x0);
            // Entries go into the dense columns.  An atom that a pixel lists twice has one place there: every entry writes its number, those
            // that find another's wait for a later pass (lists as the router makes them: one pass).  The array is all zero between uses.
            bool inside[2], on[2];
            int cur[2][TQ];
            unsigned seen[2][TQ];
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                inside[g] = tl.X0 + x0 + 16 * g + n < a.W;
                on[g] = inside[g] && (f.on[g] | unmasked) != 0;
#pragma unroll
                for (int r = 0; r < TQ; ++r) {
                    f.idx[g][r] = f.idx[g][r] < lmax ? f.idx[g][r] : lmax;
                    f.val[g][r] = on[g] ? f.val[g][r] : 0u;
                    cur[g][r] = 2 * ((4 * r + q < a.T ? (int)f.idx[g][r] : LP) * F::PP + 16 * g + n);
                    if (rec) *(lds_h*)(phi + cur[g][r]) = (unsigned short)(4 * r + q + 1);
                }
            }
            if (rec) {
                wave_lds_fence();
#pragma unroll
                for (int g = 0; g < 2; ++g)
#pragma unroll
                    for (int r = 0; r < TQ; ++r) seen[g][r] = *(lds_h*)(phi + cur[g][r]);
            }
            u32x4v Eh[2][NS], El[2][NS];             // E of the pixel's own scale, high and low parts
            int ex[2];                               // 0: all of it is 0
#pragma unroll
            for (int g0 = 0; g0 < 2; g0 += F::RG) {
#pragma unroll
                for (int g = g0; g < g0 + F::RG; ++g) {
                    float dy[CM];
#pragma unroll
                    for (int c = 0; c < CM; ++c) {
                        dy[c] = on[g] ? from_bits(f.dy[g][c], (const TIO*)nullptr) : 0.0f;
                    }
                    float E[NS][8], m = 0.0f;
#pragma unroll
                    for (int s = 0; s < NS; ++s) {
#pragma unroll
                        for (int i = 0; i < NI; ++i) {
                            const char* p = Ub + tap[s][i];
                            float e = dy[0] * *(const float*)(p + 64 * g);
#pragma unroll
                            for (int c = 1; c < CM; ++c) e = fmaf(dy[c], *(const float*)(p + 64 * g + 4 * c * UH * UP), e);
                            E[s][i] = e;
                            m = fmaxf(m, fabsf(e));
                        }
#pragma unroll
                        for (int i = NI; i < 8; ++i) E[s][i] = 0.0f;
                    }
                    m = rows_max(m);
                    ex[g] = m > 0.0f ? exponent_field(m) : 0;
                    const float sc = pow2_field(268 - ex[g]);
#pragma unroll
                    for (int s = 0; s < NS; ++s)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            unsigned hi = 0, lo = 0;
                            if (2 * i < NI) split_pair(E[s][2 * i], E[s][2 * i + 1], sc, hi, lo);
                            Eh[g][s][i] = hi, El[g][s][i] = lo;
                        }
                }
                if (a.dvalue) {
#pragma unroll
                    for (int g = g0; g < g0 + F::RG; ++g)
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
                            float4v r = {0, 0, 0, 0};
#pragma unroll
                            for (int s = 0; s < NS; ++s) {
                                const half8 dh = __builtin_bit_cast(half8, F::DL ? Dsh[F::DL ? 2 * (mt * NS + s) * 64 + lane : 0] : Dh[F::DL ? 0 : mt][s]);
                                const half8 dl = __builtin_bit_cast(half8, F::DL ? Dsh[F::DL ? (2 * (mt * NS + s) + 1) * 64 + lane : 0] : Dl[F::DL ? 0 : mt][s]);
                                const half8 eh = __builtin_bit_cast(half8, Eh[g][s]), el = __builtin_bit_cast(half8, El[g][s]);
                                r = __builtin_amdgcn_mfma_f32_16x16x32_f16(dl, eh, r, 0, 0, 0);
                                r = __builtin_amdgcn_mfma_f32_16x16x32_f16(dh, el, r, 0, 0, 0);
                                r = __builtin_amdgcn_mfma_f32_16x16x32_f16(dh, eh, r, 0, 0, 0);
                            }
                            *(lds_f4*)(er + (g - g0) * F::R_B + 4 * (n * F::RP + 16 * mt + 4 * q)) = r;
                        }
                    wave_lds_fence();
#pragma unroll
                    for (int g = g0; g < g0 + F::RG; ++g) {
                        // both powers of two undone at once: a response has a place in fp32 where one of them alone would lead out of it
                        float v[TQ];
#pragma unroll
                        for (int r = 0; r < TQ; ++r)
                            v[r] = __builtin_ldexpf(*(lds_f*)(er + (g - g0) * F::R_B + 4 * (n * F::RP + f.idx[g][r])), ex[g] + dback[f.idx[g][r]]);
                        if (inside[g]) {
                            char* const to = (char*)a.dvalue + tl.list * VB;
                            const unsigned x = (unsigned)Y * (unsigned)a.W + (unsigned)(tl.X0 + x0 + 16 * g + n);
#pragma unroll
                            for (int r = 0; r < TQ; ++r)
                                if (4 * r + q < a.T) st_from_float((TV*)(to + (entry[r] + x) * VB), 0, on[g] ? v[r] : 0.0f);
                        }
                    }
                    wave_lds_fence();
                }
            }
            if (rec) {
                // the unit's scale, its values' scale; E to [pixel][place], high parts, then low ones
                int es = row_max(max(ex[0], ex[1]));
                if (F::ACC) {
                    // G's own power of two: at most four times the unit's, or G changes to the double of it; never below 2^-64 of
                    // the largest that it has had: under that one it holds less than 2^(15 + 16) times the 2^16 entries of a run,
                    // 2^111 under the smallest
                    es = __builtin_amdgcn_readfirstlane(es);
                    if (es > scale || (es > 0 && es < scale - 2 && scale > top - 64)) {
                        const int to = max(min(es + 1, 254), top - 64), by = scale - to;
                        top = max(top, to);
                        const float f1 = pow2_field(127 + by / 2), f2 = pow2_field(127 + by - by / 2);
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                            for (int t = 0; t < NT; ++t)
#pragma unroll
                                for (int i = 0; i < 4; ++i) G[mt][t][i] = G[mt][t][i] * f1 * f2;
                        scale = to;
                    }
                    es = scale;
                }
                float vback = 1.0f;
                int below[2];
                int vx = 0, behind = 0;                  // the values' power of two; is there one whole steps below it?
                unsigned val[2][TQ];
                if (F::SPLIT) {
                    float m = 0.0f;
#pragma unroll
                    for (int g = 0; g < 2; ++g)
#pragma unroll
                        for (int r = 0; r < TQ; ++r)
                            if (4 * r + q < a.T) m = fmaxf(m, fabsf(__uint_as_float(f.val[g][r])));
                    m = rows_max(__int_as_float(row_max(__float_as_int(m))));
                    vx = exponent_field(m);
                    const float vsc = pow2_field(268 - vx), least = pow2_field(vx - F::VSTEP + 1);
                    vback = pow2_field(vx - 14);
#pragma unroll
                    for (int g = 0; g < 2; ++g)
#pragma unroll
                        for (int r = 0; r < TQ; ++r) {
                            const float v = __uint_as_float(f.val[g][r]);
                            behind |= fabsf(v) < least && v != 0.0f;
                            val[g][r] = split_value(v, vsc);
                        }
                }
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    // a pixel that is n whole steps below the unit's power of two: n steps less, which are made up for when its entries are
                    // added, after the other ones'
                    below[g] = ex[g] > 0 ? ((es - ex[g]) & -F::STEP) : 0;
                    const _Float16 fs = (_Float16)(turn * pow2_field(127 + ex[g] - es + below[g]));
                    const half2v ff = {fs, fs};
#pragma unroll
                    for (int s = 0; s < NS; ++s) {
                        u32x4v h, l;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            h[i] = __builtin_bit_cast(unsigned, __builtin_bit_cast(half2v, (unsigned)Eh[g][s][i]) * ff);
                            l[i] = __builtin_bit_cast(unsigned, __builtin_bit_cast(half2v, (unsigned)El[g][s][i]) * ff);
                        }
                        unsigned char* const p = er + (16 * g + n) * F::EP + 64 * s + 16 * q;
                        *(lds_u4*)p = h;
                        *(lds_u4*)(p + 32 * F::EP) = l;
                    }
#pragma unroll
                    for (int r = 0; r < TQ; ++r)
                        if (!F::SPLIT) val[g][r] = f.val[g][r];
                }
                wave_lds_fence();
                // ... and back turned: of the 16 places t, four pixels' rows at a time, lane n gets its place's column; lane (q, n) has pixels
                // 8 q .. 8 q + 7 of place 16 t + n then
                int column = (8 * q + n / 4) * F::EP + 8 * (n % 4);
                auto turned = [&](int t, half8& high, half8& low) {
                    short4v v[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        v[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_turned)(er + column + 32 * t + 4 * F::EP * (i % 2) + 32 * F::EP * (i / 2)));
                    high = __builtin_bit_cast(half8, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
                    low = __builtin_bit_cast(half8, __builtin_shufflevector(v[2], v[3], 0, 1, 2, 3, 4, 5, 6, 7));
                };
                half8 eh[NT], el[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) turned(t, eh[t], el[t]);
                const float back = turn * pow2_field(es - 14) * vback;
                // Entries to their places, one of those that share one; what has none yet stays in `cur`
                int put[2][TQ];
                auto scatter = [&] {
#pragma unroll
                    for (int g = 0; g < 2; ++g)
#pragma unroll
                        for (int r = 0; r < TQ; ++r) {
                            const int aside = 2 * (LP * F::PP + 16 * g + n);
                            const bool mine = seen[g][r] == (unsigned)(4 * r + q + 1);
                            put[g][r] = mine ? cur[g][r] : aside;
                            cur[g][r] = mine ? aside : cur[g][r];
                            *(lds_h*)(phi + put[g][r]) = (unsigned short)val[g][r];
                            if (F::SPLIT) *(lds_h*)(phi + F::PHI_ROWS * F::PP * 2 + put[g][r]) = (unsigned short)(val[g][r] >> 16);
                        }
                    wave_lds_fence();
                };
                // how far an entry is behind: its pixel's E, its value
                auto value_steps = [&](int g, int r) -> int {
                    const float v = fabsf(__uint_as_float(f.val[g][r]));
                    return F::SPLIT && v != 0.0f && 4 * r + q < a.T ? (vx - exponent_field(v)) / F::VSTEP * F::VSTEP : 0;
                };
                auto steps = [&](int g, int r) -> int { return below[g] + value_steps(g, r); };
                auto left = [&]() -> bool {
                    bool more = false;
#pragma unroll
                    for (int g = 0; g < 2; ++g)
#pragma unroll
                        for (int r = 0; r < TQ; ++r) more = more || cur[g][r] != 2 * (LP * F::PP + 16 * g + n);
                    return __any(more);
                };
                auto clear = [&] {
                    wave_lds_fence();
#pragma unroll
                    for (int g = 0; g < 2; ++g)
#pragma unroll
                        for (int r = 0; r < TQ; ++r) {
                            *(lds_h*)(phi + put[g][r]) = 0;
                            if (F::SPLIT) *(lds_h*)(phi + F::PHI_ROWS * F::PP * 2 + put[g][r]) = 0;
                        }
                    wave_lds_fence();
                };
                auto operand = [&](int mt, int part) -> half8 {
                    return __builtin_bit_cast(half8, *(const lds_u4*)(phi + 2 * ((part * F::PHI_ROWS + 16 * mt + n) * F::PP + 8 * q)));
                };
                auto product = [&](half8 p0, half8 p1, half8 high, half8 low, float4v r) -> float4v {
                    // (values' low parts are 2^11 higher than they are; of E, beside those, what is left 2^11 lower is enough)
                    if (F::SPLIT) r = __builtin_amdgcn_mfma_f32_16x16x32_f16(p1, high * (_Float16)0x1p-11f, r, 0, 0, 0);
                    r = __builtin_amdgcn_mfma_f32_16x16x32_f16(p0, low, r, 0, 0, 0);
                    return __builtin_amdgcn_mfma_f32_16x16x32_f16(p0, high, r, 0, 0, 0);
                };
                scatter();
                if (__any(below[0] | below[1] | behind)) {       // what is below the rest: not yet
#pragma unroll
                    for (int g = 0; g < 2; ++g)
#pragma unroll
                        for (int r = 0; r < TQ; ++r) {
                            const int aside = 2 * (LP * F::PP + 16 * g + n), out = steps(g, r) ? put[g][r] : aside;
                            *(lds_h*)(phi + out) = 0;
                            if (F::SPLIT) *(lds_h*)(phi + F::PHI_ROWS * F::PP * 2 + out) = 0;
                            cur[g][r] = out != aside ? out : cur[g][r];
                        }
                    wave_lds_fence();
                }
                bool more = left();
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    const half8 p0 = operand(mt, 0), p1 = F::SPLIT ? operand(mt, 1) : p0;
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const float4v r = product(p0, p1, eh[t], el[t], F::ACC ? G[mt][t] : (float4v){0, 0, 0, 0});
                        if (F::ACC) G[mt][t] = r;
                        else
#pragma unroll
                            for (int i = 0; i < 4; ++i) G[mt][t][i] = fmaf(r[i], back, G[mt][t][i]);
                    }
                }
                clear();
                // What is left, if anything: what is below the rest, the nearest first, and atoms listed twice.  Every turn adds an entry: of
                // those that it is for all write their numbers, and one of each place finds its own.
                while (more) {
                    int less = 1 << 20;
#pragma unroll
                    for (int g = 0; g < 2; ++g)
#pragma unroll
                        for (int r = 0; r < TQ; ++r) less = cur[g][r] != 2 * (LP * F::PP + 16 * g + n) ? min(less, steps(g, r)) : less;
                    less = wave_min(less);
#pragma unroll
                    for (int g = 0; g < 2; ++g)
#pragma unroll
                        for (int r = 0; r < TQ; ++r)
                            *(lds_h*)(phi + (steps(g, r) == less ? cur[g][r] : 2 * (LP * F::PP + 16 * g + n))) = (unsigned short)(4 * r + q + 1);
                    wave_lds_fence();
#pragma unroll
                    for (int g = 0; g < 2; ++g)
#pragma unroll
                        for (int r = 0; r < TQ; ++r) seen[g][r] = *(lds_h*)(phi + cur[g][r]);
                    wave_lds_fence();
                    if (F::SPLIT)
#pragma unroll
                        for (int g = 0; g < 2; ++g)
#pragma unroll
                            for (int r = 0; r < TQ; ++r) val[g][r] = split_value(__uint_as_float(f.val[g][r]), pow2_field(268 - vx + value_steps(g, r)));
                    scatter();
                    more = left();
                    asm volatile("" : "+v"(column));         // (hidden: E is read again; kept, it would take registers of every unit)
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        __builtin_amdgcn_sched_barrier(0);   // (one product at a time, for the same reason)
                        half8 high, low;
                        turned(t, high, low);
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
                            __builtin_amdgcn_sched_barrier(0);
                            const float4v r = product(operand(mt, 0), F::SPLIT ? operand(mt, 1) : high, high, low, (float4v){0, 0, 0, 0});
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const float v = __builtin_ldexpf(r[i], -less);
                                // (atoms 4 q + i of the tile times one: the matrix instructions' registers are theirs alone)
                                if (F::ACC) G[mt][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(n == 4 * q + i ? 1.0f : 0.0f, v, G[mt][t], 0, 0, 0);
                                else G[mt][t][i] = fmaf(v, back, G[mt][t][i]);
                            }
                        }
                    }
                    clear();
                }
            }
        }
        // ---- the wavefronts' sums to the record, 16 places of all atoms at a time, through the scratch (G is 16 x 16 tiles: lane (q, n) has
        // atoms 4 q .. 4 q + 3 of place n)
        if (rec && (++held == 4096 / (GM_TW * GM_TH / 4) || last)) {
            held = 0;
            const float back = F::ACC ? turn * pow2_field(scale - 14) : 1.0f;
            scale = top = 15;                        // G is 0 again: the next run's sums owe nothing to this one's
            int id = tid;                            // (hidden: no address of a record is worth a register for the whole tile)
            asm volatile("" : "+v"(id));
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                __syncthreads();
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        *(lds_f*)(er + 4 * ((16 * mt + 4 * q + r) * 16 + n)) = G[mt][t][r] * back;
                        G[mt][t][r] = 0.0f;
                    }
                __syncthreads();
                double was[MT];
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const int l = 16 * i + id / 16, place = 16 * t + id % 16, j = F::tap(place / 32, place / 8 % 4, place % 8);
                    was[i] = !first && l < a.L && j >= 0 ? rec[l * KK + j] : 0.0;
                }
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const int l = 16 * i + id / 16, place = 16 * t + id % 16, j = F::tap(place / 32, place / 8 % 4, place % 8);
                    double v = was[i];
#pragma unroll
                    for (int w = 0; w < 4; ++w) v += (double)*(lds_f*)(scratch[w] + F::PHI_B + 4 * (256 * i + id));
                    if (l < a.L && j >= 0) rec[l * KK + j] = v;
                }
            }
            first = false;
        }
    }
}

template <int K, int LP, int CM, typename TV, typename TIO>
static hipError_t grad_mfma_one(const ListGradArgs& a, int grid, hipStream_t st) {
    if (a.T <= 8) k_list_grad_mfma<K, LP, CM, 2, TV, TIO><<<grid, 256, 0, st>>>(a);
    else k_list_grad_mfma<K, LP, CM, 4, TV, TIO><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}
template <int K, typename TV, typename TIO>
static hipError_t grad_mfma_io(const ListGradArgs& a, int grid, hipStream_t st) {
    if (a.L <= 80) return a.C == 1 ? grad_mfma_one<K, 80, 1, TV, TIO>(a, grid, st) : grad_mfma_one<K, 80, 3, TV, TIO>(a, grid, st);
    return a.C == 1 ? grad_mfma_one<K, 128, 1, TV, TIO>(a, grid, st) : grad_mfma_one<K, 128, 3, TV, TIO>(a, grid, st);
}
template <int K, typename TV>
static hipError_t grad_mfma_k(const ListGradArgs& a, int grid, hipStream_t st) {
    return a.io_f16 ? grad_mfma_io<K, TV, __half>(a, grid, st) : grad_mfma_io<K, TV, float>(a, grid, st);
}

}  // namespace srd

// Products for the layers of include/sr_layer.h: C[m][n] = sum_k A(m, k) B(n, k) on the matrix cores, with what a layer does to C
// before it is stored.
//
// Operands of one type, fp32, fp16 or bfloat16; sums in fp32.  An operand is stored with k running fastest (KC: a layer's rows and
// its weight in the forward product) or with the other index running fastest (RC: the weight in dx = dz W, both in dW = dz^T x).
// A workgroup makes a BM x BN tile of C.  128 bytes of k (64 values, 32 of fp32) of both operands go to LDS at a time, two buffers in
// turn: while one is multiplied the next is under way, straight from memory to LDS (16-bit rows that are no pieces of 16 bytes: by way of registers).  RC operands are turned by the LDS
// reads (16-bit types) or read value by value (fp32, whose matrix instructions are slow enough for that).
//
// LDS: KC as [row][8 pieces of 16 bytes], piece p of row r in place p ^ (r & 7), so that the 16 or 32 rows a read takes at one k lie in
// different banks; RC as [k][row], its chunks of 16 rows exchanged by some bits of k for the same reason.
//
// The matrix instructions get B as their first operand: a lane then holds consecutive n of one m, and the tile goes through LDS
// once more, 32 rows of a wavefront's part at a time, to be finished and stored in pieces of 8 values of a row.
#pragma once
#include <stdint.h>

#include "sr_launch.h"
#include "../../include/sr_layer.h"

namespace srd {

using u32x4g = __attribute__((ext_vector_type(4))) unsigned;
using u32x4u = __attribute__((ext_vector_type(4), aligned(2))) unsigned;      // in memory, at any element
using f32x4g = __attribute__((ext_vector_type(4))) float;
using f32x16g = __attribute__((ext_vector_type(16))) float;
using half8g = __attribute__((ext_vector_type(8))) _Float16;
using bf8g = __attribute__((ext_vector_type(8))) __bf16;
using s16x4g = __attribute__((ext_vector_type(4))) short;

enum { GEMM_KC_KC = 0, GEMM_KC_RC = 1, GEMM_RC_RC = 2 };          // A, B
// What is done to C: z = C + bias
enum {
    GEMM_STORE = 0,        // out = act(z) + extra
    GEMM_SLOPE = 1,        // out = extra act'(z)
    GEMM_GATED = 2,        // out = act(z_gate) z_up
    GEMM_GATED_SLOPE = 3,  // out[n] = extra z_up act'(z_gate), out[half + n] = extra act(z_gate)
    GEMM_PARTIAL = 4       // C itself, fp32, to partial[split]
};

struct GemmArgs {
    const void* a;
    const void* b;
    int64_t lda, ldb;          // elements from one row of the stored matrix to the next
    int m, n, k;               // n: of C; for the gated forms of their halves
    int half;                  // gated forms: row of B where the second half starts
    int tiles_m, tiles_n, splits;
    int ksplit;                // of k a split takes, a multiple of 128 bytes of it
    int mode, act;
    const void* bias;          // [n], or null
    const void* extra;         // residual or dy, [m][ld_extra], or null
    void* out;
    int64_t ld_extra, ld_out;
    float* partial;            // [splits][m][n]
    float* sums;               // RC_RC: [splits][m] sums of A over k, or null; SLOPE, GATED_SLOPE: [2 tiles_m][outputs] sums of the output over m, or null
    void* sums_out;            // RC_RC of one split: sums of A, [m] in the operands' type; and where launch_gemm_finish puts them
    int sum_rows;              // of sums, for launch_gemm_finish (0: splits)
    float* exact;              // SLOPE, GATED_SLOPE by the kernel for few rows or of split sums: [m][outputs], the output before its rounding, or null
    int64_t out_lo;            // SLOPE, GATED_SLOPE: 0, or elements from `out` to where goes what its rounding leaves off (tiles 0 and 1)
    int64_t a_lo;              // KC_RC, RC_RC: 0, or elements from A to a second matrix that is added to it (tiles 0 and 1)
};

// Tiles: 0: 64 x 64, 1: 128 x 128, 2: 256 x 128, 3: 256 x 256 (2 and 3: operands on 16-byte pieces only).
template <typename T> hipError_t launch_gemm(const GemmArgs& g, int layout, bool aligned, int tile, hipStream_t st);
inline int gemm_tile_rows(int tile) { return tile < 2 ? 64 << tile : 256; }
inline int gemm_tile_cols(int tile) { return tile < 1 ? 64 : tile < 3 ? 128 : 256; }

// z of the split sums, and what the epilogue would have done: elements [m][n], sums over the splits in double
template <typename T> hipError_t launch_gemm_finish(const GemmArgs& g, hipStream_t st);
// Rows of `cols` elements at any address to rows of whole 16-byte pieces, zeros behind the last element
template <typename T> hipError_t launch_pack(const void* from, int64_t rows, int cols, void* to, hipStream_t st);
// Few rows: one pass over the weights (layout KC_KC, every mode but PARTIAL).  Each of its workgroups reads all rows: 2048 to 2048, in a graph, bfloat16 1 row 4.4 us, 16
// 5.7, 48 9.9, 64 11.2, of tiles 65 rows 9.6; fp32 7.5, 10.5, 21.6, 24.3, of tiles 16.4; gated, 1024 to 2816, 64 rows 8.4 and 19.6, of tiles 7.0 and 22.0.
template <typename T> hipError_t launch_skinny(const GemmArgs& g, bool aligned, hipStream_t st);
constexpr int SKINNY_ROWS = 64;
// Many rows, a small weight (layouts KC_KC and KC_RC, modes STORE and GATED; rows of the output and of what is added without gaps): what a launch is made of, waves = 0 if
// the case is none for it.  outputs: that a wavefront is to have room for, of 1 that it takes.  rows: that a wavefront takes at a time; group: tiles of 16 columns (of each half) that are made at a time; np: columns of a
// half in LDS; steps: of 64 bytes of k.  With fewer than 12 wavefronts on a compute unit the rows' way through memory is not hidden (500 000 rows of
// 128 to 128, bfloat16, 6 wavefronts: 70 us, the tile kernel 47).
struct ThinShape { int np, steps, waves, group, rows; };
inline ThinShape thin_shape(int64_t n, int64_t k, size_t es, bool gated, int outputs = 1) {
    const int64_t group = n <= 16 ? 1 : 2, np = (n + 16 * group - 1) / (16 * group) * (16 * group), steps = (k * (int64_t)es + 63) / 64;
    if (steps < 1 || steps > 4 || n > 512) return {0, 0, 0, 0, 0};
    for (int rows = 32; rows >= 16; rows /= 2) {
        const int64_t patch = (rows * outputs * n * (int64_t)es + 15) / 16 * 16;
        const int64_t bytes = np * (gated ? 2 : 1) * (steps * 64 + 20) + 4 * patch;
        if (bytes <= 65536 && 163840 / bytes >= 3) return {(int)np, (int)steps, 4, (int)group, rows};
    }
    return {0, 0, 0, 0, 0};
}
template <typename T> hipError_t launch_thin(const GemmArgs& g, int layout, hipStream_t st);

// Very many rows on four bytes, a weight that registers hold (layouts KC_KC and KC_RC, every mode but PARTIAL, no second parts): what
// it is made of, grid = 0 if the case is none for it.  `launches` of up to `cols` columns, one after another; wn groups of `tiles` tiles of 16 columns, times
// wr of rows, are the wavefronts; steps: of 32 k that the kernel has registers for; subs: of 32 wr rows, in a block of rows.
constexpr int ROWS_STAGE = 65536;                    // bytes of a block of rows
struct RowsShape { int grid, launches, cols, wn, wr, tiles, steps, subs; };
inline RowsShape rows_shape(int64_t m, int64_t n, int64_t k, size_t es, bool gated, bool extra) {
    if (n < 1 || k < 1) return {};
    RowsShape s = {};
    const int64_t steps = (k + 31) / 32;
    // tiles x steps x halves: 32 (fp32: 8, of three parts) fill half of the registers; beside what is added or multiplied there is room for half of that
    if (es == 4) {
        if (!gated && !extra && steps <= 2) s.tiles = 4;
        else if (steps <= (gated ? 2 : 4)) s.tiles = 2;
        else return {};
        s.steps = steps <= 2 ? 2 : 4;
    } else {
        if (!gated && steps <= (extra ? 4 : 8)) s.tiles = 4;
        else if (steps <= (gated ? extra ? 4 : 8 : extra ? 8 : 16)) s.tiles = 2;
        else return {};
        s.steps = steps <= 4 ? 4 : steps <= 8 ? 8 : 16;
    }
    const int64_t most_cols = s.tiles * 128, group = s.tiles * 16;
    s.launches = (int)((n + most_cols - 1) / most_cols);
    s.cols = (int)(((n + s.launches - 1) / s.launches + group - 1) / group * group);
    if (s.launches == 1) s.cols = (int)n;
    s.wn = (int)((s.cols + group - 1) / group);
    s.wr = s.wn <= 1 ? 8 : s.wn <= 2 ? 4 : s.wn <= 4 ? 2 : 1;
    const int64_t sub = 32 * s.wr;
    // as few rows a workgroup as there can be, in blocks as large as there can be, but four of them
    int64_t least = 0, most = ROWS_STAGE / (sub * steps * 32 * (int64_t)es);
    if (most > 1 && most > m / (4 * 256 * sub)) most = m / (4 * 256 * sub) > 1 ? m / (4 * 256 * sub) : 1;
    for (int64_t c = most; c >= 1; --c) {
        const int64_t blocks = (m + sub * c - 1) / (sub * c), each = (blocks + 255) / 256 * c;
        if (!s.subs || each < least) least = each, s.subs = (int)c, s.grid = (int)(blocks < 256 ? blocks : 256);
    }
    return s.subs ? s : RowsShape{};
}
template <typename T> hipError_t launch_rows(const GemmArgs& g, int layout, hipStream_t st);

// A small layer's whole gradient in one pass over many rows (everything on 16-byte pieces; c and o multiples of a piece).
struct ThinGradArgs {
    const void *x, *w, *bias, *dy;
    void* dx;                  // or null
    float *partial, *sums;     // [workgroups][wide][c], [workgroups][wide], or null
    int64_t rows;
    int c, o, act;
};
// Its LDS: strides of the rows of the tiles (an odd number of 16-byte pieces), steps of 64 bytes in a row, where the tiles are; bytes = 0 if the case
// is none for it.
struct ThinGradShape { int dz_stride, x_stride, dy_stride, dz_steps, x_steps, wz, dz, lo, x, dy, bias, bytes; };
__host__ __device__ inline ThinGradShape thin_grad_shape(int c, int o, int es, bool gated, bool z) {
    ThinGradShape s = {};
    const int e = 16 / es, wide = gated ? 2 * o : o;
    if (c > 128 || wide > (c > 64 ? 128 : 256) || c % e || o % e) return s;      // dW's tiles have to fit the registers
    s.dz_steps = (wide * es + 63) / 64;
    s.x_steps = (c * es + 63) / 64;
    s.dz_stride = s.dz_steps * 64 + 16;
    s.x_stride = s.x_steps * 64 + 16;
    s.dy_stride = (o * es + 31) / 32 * 32 + 16;
    const int c16 = (c + 15) / 16 * 16, w16 = (wide + 15) / 16 * 16;
    s.wz = c16 * s.dz_stride;
    s.dz = s.wz + (z ? (w16 + (gated ? 16 : 0)) * s.x_stride : 0);
    s.lo = s.dz + 64 * s.dz_stride;
    s.x = s.lo + (z && es == 2 ? 64 * s.dz_stride : 0);
    s.dy = s.x + 64 * s.x_stride;
    s.bias = s.dy + (gated ? 64 * s.dy_stride : 0);
    s.bytes = s.bias + (z ? (w16 + 16) * 4 : 0);
    if (s.bytes > 65536) s.bytes = 0;
    return s;
}
template <typename T> hipError_t launch_thin_grad(const ThinGradArgs& a, bool gated, int grid, hipStream_t st);

// ---- values ---------------------------------------------------------------------------------------------------------
__device__ __forceinline__ float act_exp(float z) { return __builtin_amdgcn_exp2f(z * LOG2E); }
__device__ __forceinline__ float sigmoid_of(float z) { return __builtin_amdgcn_rcpf(1.0f + act_exp(-z)); }
// The normal distribution's integral up to z, and its density without 1 / sqrt(2 pi), by Abramowitz and Stegun 7.1.26: with x = |z| / sqrt 2, t =
// 1 / (1 + p x), erfc(x) = (a1 t + ... + a5 t^5) exp(-x^2) within 1.5e-7.  A third of the time of erff, and the exponential is the density.
__device__ __forceinline__ float normal_cdf(float z, float& density) {
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(z), 0.3275911f * 0.70710678118654752440f, 1.0f));
    density = __builtin_amdgcn_exp2f(z * z * (-0.5f * LOG2E));
    const float q = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 0.5f * 1.061405429f, 0.5f * -1.453152027f), 0.5f * 1.421413741f), 0.5f * -0.284496736f), 0.5f * 0.254829592f) * density;
    return z < 0.0f ? q : 1.0f - q;
}
template <int U, typename F> __device__ __forceinline__ void each8(float (&z)[U][8], F f) {
#pragma unroll
    for (int r = 0; r < U; ++r)
#pragma unroll
        for (int i = 0; i < 8; ++i) f(z[r][i], r, i);
}
// z to act(z); the branches are uniform
template <int U> __device__ __forceinline__ void act8(int act, float (&z)[U][8]) {
    if (act == SR_ACT_RELU) {
        each8<U>(z, [](float& v, int, int) { v = v <= 0.0f ? 0.0f : v; });              // NaN stays
    } else if (act == SR_ACT_GELU) {
        each8<U>(z, [](float& v, int, int) { float d; v *= normal_cdf(v, d); });
    } else if (act == SR_ACT_SILU) {
        each8<U>(z, [](float& v, int, int) { v *= sigmoid_of(v); });
    } else if (act == SR_ACT_SIGMOID) {
        each8<U>(z, [](float& v, int, int) { v = sigmoid_of(v); });
    }
}
// z to act'(z), and the values
template <int U> __device__ __forceinline__ void slope8(int act, float (&z)[U][8], float (&value)[U][8]) {
    if (act == SR_ACT_RELU) {
        each8<U>(z, [&](float& v, int r, int i) { value[r][i] = v <= 0.0f ? 0.0f : v, v = v > 0.0f ? 1.0f : 0.0f; });
    } else if (act == SR_ACT_GELU) {
        each8<U>(z, [&](float& v, int r, int i) {
            float d;
            const float c = normal_cdf(v, d);
            value[r][i] = v * c;
            v = fmaf(v * 0.39894228040143267794f, d, c);
        });
    } else if (act == SR_ACT_SILU) {
        each8<U>(z, [&](float& v, int r, int i) {
            const float s = sigmoid_of(v);
            value[r][i] = v * s;
            v = s * fmaf(v, 1.0f - s, 1.0f);
        });
    } else if (act == SR_ACT_SIGMOID) {
        each8<U>(z, [&](float& v, int r, int i) {
            const float s = sigmoid_of(v);
            value[r][i] = s;
            v = s * (1.0f - s);
        });
    } else {
        each8<U>(z, [&](float& v, int r, int i) { value[r][i] = v, v = 1.0f; });
    }
}

__device__ __forceinline__ float gm_get(const float* p) { return *p; }
__device__ __forceinline__ float gm_get(const __half* p) { return (float)*(const _Float16*)p; }
__device__ __forceinline__ float gm_get(const bf16raw* p) { return __uint_as_float((unsigned)p->bits << 16); }
__device__ __forceinline__ void gm_put(float* p, float v) { *p = v; }
__device__ __forceinline__ void gm_put(__half* p, float v) { *(_Float16*)p = (_Float16)v; }
__device__ __forceinline__ void gm_put(bf16raw* p, float v) { *(__bf16*)p = (__bf16)v; }

__device__ __forceinline__ void gm_get8(const float* p, float v[8]) {
    const u32x4u a = ((const u32x4u*)p)[0], b = ((const u32x4u*)p)[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(a[i]), v[4 + i] = __uint_as_float(b[i]);
}
__device__ __forceinline__ void gm_get8(const __half* p, float v[8]) {
    const half8g a = __builtin_bit_cast(half8g, (u32x4g)*(const u32x4u*)p);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)a[i];
}
__device__ __forceinline__ void gm_get8(const bf16raw* p, float v[8]) {
    const u32x4g a = *(const u32x4u*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(a[i] << 16), v[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
}
__device__ __forceinline__ void gm_put8(float* p, const float v[8]) {
    u32x4u a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = __float_as_uint(v[i]), b[i] = __float_as_uint(v[4 + i]);
    ((u32x4u*)p)[0] = a;
    ((u32x4u*)p)[1] = b;
}
__device__ __forceinline__ void gm_put8(__half* p, const float v[8]) {
    half8g a;
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = (_Float16)v[i];
    *(u32x4u*)p = __builtin_bit_cast(u32x4g, a);
}
__device__ __forceinline__ void gm_put8(bf16raw* p, const float v[8]) {
    bf8g a;
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = (__bf16)v[i];
    *(u32x4u*)p = __builtin_bit_cast(u32x4g, a);
}
// as many of 8 as there are
template <typename T> __device__ __forceinline__ void gm_get_some(const T* p, int count, float v[8]) {
    if (count >= 8) {
        gm_get8(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < count ? gm_get(p + i) : 0.0f;
    }
}
template <typename T> __device__ __forceinline__ void gm_put_some(T* p, int count, const float v[8]) {
    if (count >= 8) {
        gm_put8(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) gm_put(p + i, v[i]);
    }
}

// 16 bytes of a row of which `count` elements are there (0 or less: none), zeros behind them
template <typename T> __device__ __forceinline__ u32x4g gm_piece(const T* p, int count) {
    constexpr int E = 16 / sizeof(T);
    if (count >= E) return *(const u32x4u*)p;
    u32x4g v = {0, 0, 0, 0};
    if (count > 0) {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (i < count) {
                if constexpr (sizeof(T) == 4) v[i] = ((const unsigned*)p)[i];
                else v[i / 2] |= (unsigned)((const unsigned short*)p)[i] << 16 * (i % 2);
            }
    }
    return v;
}

// The first `count` elements of a piece that is there, but may end in what is not the row's
template <typename T> __device__ __forceinline__ u32x4g gm_cut(u32x4g v, int count) {
    constexpr int E = 16 / sizeof(T);
    if (count < E)
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (i >= count) {
                if constexpr (sizeof(T) == 4) v[i] = 0;
                else v[i / 2] &= i % 2 ? 0x0000ffffu : 0xffff0000u;
            }
    return v;
}

// One step of k on a pair of 16-byte fragments: MT = 32: 32 x 32, 2 pieces of k; MT = 16: 16 x 16, 4 pieces.
template <int MT> struct AccOf { typedef f32x16g type; };
template <> struct AccOf<16> { typedef f32x4g type; };
template <typename T, int MT> __device__ __forceinline__ void gm_mul(typename AccOf<MT>::type& c, u32x4g a, u32x4g b) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (MT == 32) c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[j]), __uint_as_float(b[j]), c, 0, 0, 0);
            else c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[j]), __uint_as_float(b[j]), c, 0, 0, 0);
        }
    } else if constexpr (__is_same(T, __half)) {
        if constexpr (MT == 32) c = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8g, a), __builtin_bit_cast(half8g, b), c, 0, 0, 0);
        else c = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8g, a), __builtin_bit_cast(half8g, b), c, 0, 0, 0);
    } else {
        if constexpr (MT == 32) c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8g, a), __builtin_bit_cast(bf8g, b), c, 0, 0, 0);
        else c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8g, a), __builtin_bit_cast(bf8g, b), c, 0, 0, 0);
    }
}
// fp32 on the bfloat16 matrix instructions, sixteen times as fast as the fp32 ones: eight values as the sum of three bfloat16 numbers each, x = h + m + l
// exactly (8 bits are rounded off to the nearest twice, what is left has 8), and of the nine products of two such sums the six large ones; the other
// three come to 2^-24 of x y at most.  Summed in fp32 like the others.  What rounds beyond bfloat16's largest number has that as its h (an infinity there would make NaN of numbers from
// 0x1.ffp127 on; 4096^3: 655 us without, 677 with it).  Below 2^-110 the parts end at bfloat16's smallest number, 2^-133: a value is held to
// 2^-134.  Two of these a value and three conversions a pair: a third of the matrix instructions' time where a wavefront makes 64 x 64.  4096^3: 145
// TFLOP/s by fp32 instructions, 203 so.
constexpr float BF16_MOST = 0x1.fep127f;
struct Split8 { u32x4g h, m, l; };
__device__ __forceinline__ Split8 gm_split(u32x4g a, u32x4g b) {
    using bf2g = __attribute__((ext_vector_type(2))) __bf16;
    Split8 s;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float x = __uint_as_float((unsigned)(i < 2 ? a[2 * i] : b[2 * i - 4])), y = __uint_as_float((unsigned)(i < 2 ? a[2 * i + 1] : b[2 * i - 3]));
        const float hx = __builtin_amdgcn_fmed3f(x, -BF16_MOST, BF16_MOST), hy = __builtin_amdgcn_fmed3f(y, -BF16_MOST, BF16_MOST);
        const unsigned h = __builtin_bit_cast(unsigned, bf2g{(__bf16)hx, (__bf16)hy});
        x -= __uint_as_float(h << 16), y -= __uint_as_float(h & 0xffff0000u);
        const unsigned m = __builtin_bit_cast(unsigned, bf2g{(__bf16)x, (__bf16)y});
        x -= __uint_as_float(m << 16), y -= __uint_as_float(m & 0xffff0000u);
        s.h[i] = h;
        s.m[i] = m;
        s.l[i] = __builtin_bit_cast(unsigned, bf2g{(__bf16)x, (__bf16)y});
    }
    return s;
}
// the six products, the small ones first
template <int MT> __device__ __forceinline__ void gm_mul_part(typename AccOf<MT>::type& c, const Split8& a, const Split8& b, int part) {
    const u32x4g x = part == 0 ? a.l : part == 2 || part == 3 ? a.m : a.h, y = part == 1 ? b.l : part == 2 || part == 4 ? b.m : b.h;
    gm_mul<bf16raw, MT>(c, x, y);
}
// `sum` and the one or two values in 32 bits of a fragment: a dot product with ones, summed in fp32.  (By conversions and additions, four instructions
// instead of one, the workgroups that sum were the last ones: 8192 rows of 2048 to 4096, dW 129 us without, 149 with them.)
template <typename T> __device__ __forceinline__ float gm_sum(unsigned v, float sum) {
    if constexpr (sizeof(T) == 4) {
        return sum + __uint_as_float(v);
    } else if constexpr (__is_same(T, __half)) {
        using half2g = __attribute__((ext_vector_type(2))) _Float16;
        return __builtin_amdgcn_fdot2(__builtin_bit_cast(half2g, v), half2g{(_Float16)1.0f, (_Float16)1.0f}, sum, false);
    } else {
        using bf2g = __attribute__((ext_vector_type(2))) __bf16;
        return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf2g, v), bf2g{(__bf16)1.0f, (__bf16)1.0f}, sum, false);
    }
}
template <typename T>
__device__ __forceinline__ void gm_bias8(const GemmArgs& g, int col, bool gated, float bz[8], float bu[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) bz[i] = bu[i] = 0.0f;
    if (!g.bias || col >= g.n) return;
    gm_get_some((const T*)g.bias + col, g.n - col, bz);
    if (gated) gm_get_some((const T*)g.bias + g.half + col, g.n - col, bu);
}

// 8 values of a row as they are stored, of which `count` are there
template <typename T> struct Raw8 {
    u32x4g v[sizeof(T) / 2];
    __device__ __forceinline__ void get(const T* p, int count) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) v[i] = gm_piece(p + i * (16 / sizeof(T)), count - i * (int)(16 / sizeof(T)));
    }
    __device__ __forceinline__ void values(float e[8]) const {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (sizeof(T) == 4) {
                    e[4 * i + j] = __uint_as_float(v[i][j]);
                } else if constexpr (__is_same(T, __half)) {
                    using half2g = __attribute__((ext_vector_type(2))) _Float16;
                    const half2g h = __builtin_bit_cast(half2g, (unsigned)v[i][j]);
                    e[2 * j] = (float)h[0], e[2 * j + 1] = (float)h[1];
                } else {
                    e[2 * j] = __uint_as_float(v[i][j] << 16), e[2 * j + 1] = __uint_as_float(v[i][j] & 0xffff0000u);
                }
            }
    }
};

// What the rounding of v to T left off; of a value beyond T nothing, so that its infinity stays one.
template <typename T> __device__ __forceinline__ float gm_rest(float v) {
    T t;
    gm_put(&t, v);
    const float f = gm_get(&t);
    return fabsf(f) == INFINITY ? 0.0f : v - f;
}
// 8 columns of a row of an output before its rounding, and of its second half
template <bool GATED> __device__ __forceinline__ void gm_put_exact(const GemmArgs& g, int64_t row, int col, const float z[8], const float u[8]) {
    if (!g.exact) return;
    float* const p = g.exact + row * (GATED ? 2 * (int64_t)g.half : g.n) + col;
    gm_put_some(p, g.n - col, z);
    if constexpr (GATED) gm_put_some(p + g.half, g.n - col, u);
}
// 8 values of an output that comes in two parts
template <typename T> __device__ __forceinline__ void gm_put_parts(T* p, int64_t lo, int count, const float v[8]) {
    gm_put_some(p, count, v);
    if (sizeof(T) == 2 && lo) {
        float rest[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) rest[i] = gm_rest<T>(v[i]);
        gm_put_some(p + lo, count, rest);
    }
}

// What a layer does to 8 U values of z, outputs in its place; e: of `extra`.  For the gated forms u is the same columns of the second half, and
// becomes the second output.
template <bool GATED, int U>
__device__ __forceinline__ void gm_forward(int act, float (&z)[U][8], const float (&u)[U][8], const float (&e)[U][8]) {
    act8<U>(act, z);
#pragma unroll
    for (int r = 0; r < U; ++r)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (GATED) z[r][i] *= u[r][i];
            else z[r][i] += e[r][i];
        }
}
template <bool GATED, int U>
__device__ __forceinline__ void gm_finish(const GemmArgs& g, float (&z)[U][8], float (&u)[U][8], const float (&e)[U][8]) {
    if (g.mode == (GATED ? GEMM_GATED : GEMM_STORE)) {
        gm_forward<GATED, U>(g.act, z, u, e);
    } else {
        float value[U][8];
        slope8<U>(g.act, z, value);
#pragma unroll
        for (int r = 0; r < U; ++r)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (GATED) {
                    z[r][i] *= e[r][i] * u[r][i];
                    u[r][i] = e[r][i] * value[r][i];
                } else {
                    z[r][i] *= e[r][i];
                }
            }
    }
}
// The same for 8 columns from `col` on of row `row`, with the loads and the stores
template <typename T, bool GATED>
__device__ __forceinline__ void gm_finish8(const GemmArgs& g, int64_t row, int col, float (&z)[1][8], float (&u)[1][8]) {
    const int count = g.n - col;
    float e[1][8], bz[8], bu[8];
    gm_bias8<T>(g, col, GATED, bz, bu);
#pragma unroll
    for (int i = 0; i < 8; ++i) e[0][i] = 0.0f;
    if (g.extra) gm_get_some((const T*)g.extra + row * g.ld_extra + col, count, e[0]);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        z[0][i] += bz[i];
        if constexpr (GATED) u[0][i] += bu[i];
    }
    gm_finish<GATED, 1>(g, z, u, e);
    gm_put_exact<GATED>(g, row, col, z[0], u[0]);
    T* const out = (T*)g.out + row * g.ld_out + col;
    gm_put_parts(out, g.out_lo, count, z[0]);
    if (GATED && g.mode == GEMM_GATED_SLOPE) gm_put_parts(out + g.half, g.out_lo, count, u[0]);
}
}  // namespace srd

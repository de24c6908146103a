// Products of few rows with a weight (sr_gemm.h), the sums of split products and of dz, and copies on 16-byte pieces.
#pragma once
#include "sr_gemm.h"

namespace srd {
namespace {

constexpr int SKW = 8;             // wavefronts of a workgroup

// Up to 16 RF rows.  A workgroup makes 16 columns (of both halves, where there are two) and reads their weights once: straight from memory
// into the matrix instructions' first operand, a lane 16 bytes of one of the 16 rows, so that four lanes take 64 bytes of a row together.  Its
// eight wavefronts take every eighth step of k and add up in LDS.  Bound by the weights' way from memory and, for small ones, by the launch.
template <typename T, bool GATED, int RF, bool ALIGNED>
__global__ __launch_bounds__(SKW * 64) void k_skinny(const GemmArgs g) {
    constexpr int E = 16 / sizeof(T), H = GATED ? 2 : 1, AHEAD = RF > 2 ? 2 : RF > 1 || GATED ? 4 : 8;
    __shared__ __align__(16) float sh[SKW * H * RF * 256];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = blockIdx.x * 16, r = lane % 16;
    const int kc = lane / 16 * E;
    const T* pb[H];
    const T* pa[RF];
    {
        const int n = n0 + r < g.n ? n0 + r : g.n - 1;
#pragma unroll
        for (int h = 0; h < H; ++h) pb[h] = (const T*)g.b + (int64_t)(n + h * g.half) * g.ldb + kc;
#pragma unroll
        for (int f = 0; f < RF; ++f) pa[f] = (const T*)g.a + (int64_t)(16 * f + r < g.m ? 16 * f + r : g.m - 1) * g.lda + kc;
    }
    // What finishes 8 columns of a row is asked for first, by the lane that will finish them.
    const int fm = threadIdx.x / 2, fc = threadIdx.x % 2 * 8, col = n0 + fc;
    const bool finishes = threadIdx.x < 32 * RF && fm < g.m && col < g.n;
    Raw8<T> bias[H], extra;
    if (finishes) {
#pragma unroll
        for (int h = 0; h < H; ++h)
            if (g.bias) bias[h].get((const T*)g.bias + h * g.half + col, g.n - col);
        if (g.extra) extra.get((const T*)g.extra + fm * g.ld_extra + col, g.n - col);
    }
    f32x4g acc[H][RF];
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
        for (int f = 0; f < RF; ++f) acc[h][f] = f32x4g{0.0f, 0.0f, 0.0f, 0.0f};
    auto piece = [&](const T* p, int k) -> u32x4g {
        if constexpr (ALIGNED) return kc + k < g.k ? *(const u32x4g*)(p + k) : u32x4g{0, 0, 0, 0};
        else return gm_piece(p + k, g.k - kc - k);
    };
    for (int k = wave * 4 * E; k < g.k; k += SKW * 4 * E * AHEAD) {
        u32x4g vb[AHEAD][H], va[AHEAD][RF];
#pragma unroll
        for (int s = 0; s < AHEAD; ++s) {
            const int at = k + s * SKW * 4 * E;
#pragma unroll
            for (int h = 0; h < H; ++h) vb[s][h] = piece(pb[h], at);
#pragma unroll
            for (int f = 0; f < RF; ++f) va[s][f] = piece(pa[f], at);
        }
#pragma unroll
        for (int s = 0; s < AHEAD; ++s)
#pragma unroll
            for (int h = 0; h < H; ++h)
#pragma unroll
                for (int f = 0; f < RF; ++f) gm_mul<T, 16>(acc[h][f], vb[s][h], va[s][f]);
    }
    // [wave][half][row][16 columns]
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
        for (int f = 0; f < RF; ++f) *(f32x4g*)(sh + ((wave * H + h) * RF * 16 + f * 16 + r) * 16 + lane / 16 * 4) = acc[h][f];
    __syncthreads();
    for (int i = threadIdx.x; i < H * RF * 256; i += SKW * 64) {
        float s = sh[i];
#pragma unroll
        for (int w = 1; w < SKW; ++w) s += sh[w * H * RF * 256 + i];
        sh[i] = s;                                         // read by this thread alone
    }
    __syncthreads();
    if (!finishes) return;
    float z[1][8], u[1][8], e[1][8], add[H][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        z[0][i] = sh[fm * 16 + fc + i];
        u[0][i] = GATED ? sh[RF * 256 + fm * 16 + fc + i] : 0.0f;
        e[0][i] = 0.0f;
    }
    if (g.bias) {
#pragma unroll
        for (int h = 0; h < H; ++h) bias[h].values(add[h]);
#pragma unroll
        for (int i = 0; i < 8; ++i) z[0][i] += add[0][i], u[0][i] += add[H - 1][i];
    }
    if (g.extra) extra.values(e[0]);
    gm_finish<GATED, 1>(g, z, u, e);
    gm_put_exact<GATED>(g, fm, col, z[0], u[0]);
    T* const out = (T*)g.out + fm * g.ld_out + col;
    gm_put_parts(out, g.out_lo, g.n - col, z[0]);
    if (GATED && g.mode == GEMM_GATED_SLOPE) gm_put_parts(out + g.half, g.out_lo, g.n - col, u[0]);
}

// 8 columns of a row for a group of SL threads, each every SL-th split, in double; what follows is as in the tile kernel.  Behind the rows of C
// come the octets of `sums` (rows of g.m values), stored as they are.
struct FinishArgs {
    GemmArgs g;
    int width;                 // of a row of partial: n, or 2 half
    int octets;                // of a row of C
    int64_t all;               // octets of C
    int sum_rows;
    int64_t sum_step;          // values from one row of sums to the next
};
template <typename T, int SL>
__global__ __launch_bounds__(256) void k_gemm_finish(const FinishArgs f) {
    const GemmArgs& g = f.g;
    constexpr int PER = 256 / SL;
    __shared__ double sh[SL > 1 ? 16 * 256 : 1];           // [16 values][SL][PER]
    const int slot = threadIdx.x % PER, slice = threadIdx.x / PER;
    const int64_t o = (int64_t)blockIdx.x * PER + slot;
    const bool in_sums = o >= f.all;
    const int64_t row = in_sums ? 0 : o / f.octets;
    const int col = (int)(in_sums ? o - f.all : o - row * f.octets) * 8;
    const bool gated = !in_sums && (g.mode == GEMM_GATED || g.mode == GEMM_GATED_SLOPE);
    const int count = (in_sums ? g.m : g.n) - col;
    const bool any = count > 0 && (!in_sums || g.sums);
    const float* const p = in_sums ? g.sums + col : g.partial + row * f.width + col;
    const int64_t step = in_sums ? f.sum_step : (int64_t)g.m * f.width;
    double zd[8], ud[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) zd[i] = ud[i] = 0.0;
    if (any) {
#pragma unroll 8
        for (int s = slice; s < (in_sums ? f.sum_rows : g.splits); s += SL) {
            float v[8];
            gm_get_some(p + s * step, count, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) zd[i] += (double)v[i];
            if (gated) {
                gm_get_some(p + s * step + g.half, count, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) ud[i] += (double)v[i];
            }
        }
    }
    if constexpr (SL > 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) sh[(i * SL + slice) * PER + slot] = zd[i], sh[((8 + i) * SL + slice) * PER + slot] = ud[i];
        __syncthreads();
        if (threadIdx.x < 16 * PER) {                      // a value of a slot each, over the slices
            double* const v = sh + threadIdx.x / PER * 256 + threadIdx.x % PER;
            double sum = v[0];
#pragma unroll 8
            for (int i = 1; i < SL; ++i) sum += v[i * PER];
            v[0] = sum;
        }
        __syncthreads();
        if (slice == 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) zd[i] = sh[i * 256 + slot], ud[i] = sh[(8 + i) * 256 + slot];
        }
    }
    if (!any || slice != 0) return;
    float z[1][8], u[1][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) z[0][i] = (float)zd[i], u[0][i] = (float)ud[i];
    if (in_sums) gm_put_some((T*)g.sums_out + col, count, z[0]);
    else if (gated) gm_finish8<T, true>(g, row, col, z, u);
    else gm_finish8<T, false>(g, row, col, z, u);
}

// Sums of many rows: each workgroup adds up `chunk` of them, 64 columns of each, into the first of these, for k_gemm_finish to add those.  Its
// threads for few columns would take the rows one behind another (gradient of 8294400 rows of 27 to 121, bfloat16: 3755 us, so 3205).
__global__ __launch_bounds__(256) void k_fold(float* sums, int rows, int width, int chunk) {
    __shared__ double sh[256];
    const int col = blockIdx.x * 64 + (threadIdx.x & 63), first = blockIdx.y * chunk, end = rows - first < chunk ? rows : first + chunk;
    double s = 0.0;
    if (col < width) {
#pragma unroll 8
        for (int r = first + (threadIdx.x >> 6); r < end; r += 4) s += (double)sums[(int64_t)r * width + col];
    }
    sh[threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.x < 64 && col < width) sums[(int64_t)first * width + col] = (float)(sh[threadIdx.x] + sh[64 + threadIdx.x] + sh[128 + threadIdx.x] + sh[192 + threadIdx.x]);
}

// A workgroup takes `per` rows of `pieces` each, a thread a piece at a time: bound by memory, read and written once.
template <typename T>
__global__ __launch_bounds__(256) void k_pack(const T* from, int64_t rows, int cols, u32x4g* to, int pieces, int per) {
    constexpr int E = 16 / sizeof(T);
    const int64_t row0 = (int64_t)blockIdx.x * per;
    const int all = (int)(rows - row0 < per ? rows - row0 : per) * pieces;
    for (int i = threadIdx.x; i < all; i += 256) {
        const int row = i / pieces, p = i - row * pieces;
        to[row0 * pieces + i] = gm_piece(from + (row0 + row) * cols + p * E, cols - p * E);
    }
}

template <typename T, bool GATED, int RF>
hipError_t start_skinny(const GemmArgs& g, bool aligned, hipStream_t st) {
    const int blocks = (g.n + 15) / 16;
    if (aligned) k_skinny<T, GATED, RF, true><<<blocks, SKW * 64, 0, st>>>(g);
    else k_skinny<T, GATED, RF, false><<<blocks, SKW * 64, 0, st>>>(g);
    return hipGetLastError();
}

constexpr int FOLD_FROM = 512;
template <typename T>
void start_finish(const FinishArgs& f, int64_t octets, int splits, hipStream_t st) {
    // so many slices that a thread's loads are all under way at once (512 splits of 72 x 64: 11.4 us in 16 slices)
    if (splits <= 8) k_gemm_finish<T, 1><<<(int)((octets + 255) / 256), 256, 0, st>>>(f);
    else if (splits <= 128) k_gemm_finish<T, 16><<<(int)((octets + 15) / 16), 256, 0, st>>>(f);
    else k_gemm_finish<T, 64><<<(int)((octets + 3) / 4), 256, 0, st>>>(f);
}

}  // namespace

template <typename T>
hipError_t launch_pack(const void* from, int64_t rows, int cols, void* to, hipStream_t st) {
    constexpr int E = 16 / sizeof(T);
    const int pieces = (cols + E - 1) / E, per = pieces < 1024 ? 1024 / pieces : 1;
    k_pack<T><<<(int)((rows + per - 1) / per), 256, 0, st>>>((const T*)from, rows, cols, (u32x4g*)to, pieces, per);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_skinny(const GemmArgs& g, bool aligned, hipStream_t st) {
    if (g.mode == GEMM_GATED || g.mode == GEMM_GATED_SLOPE)
        return g.m <= 16 ? start_skinny<T, true, 1>(g, aligned, st) : g.m <= 32 ? start_skinny<T, true, 2>(g, aligned, st) : start_skinny<T, true, 4>(g, aligned, st);
    return g.m <= 16 ? start_skinny<T, false, 1>(g, aligned, st) : g.m <= 32 ? start_skinny<T, false, 2>(g, aligned, st) : start_skinny<T, false, 4>(g, aligned, st);
}

template <typename T>
hipError_t launch_gemm_finish(const GemmArgs& g, hipStream_t st) {
    FinishArgs f;
    f.g = g;
    const bool gated = g.mode == GEMM_GATED || g.mode == GEMM_GATED_SLOPE;
    f.width = gated ? 2 * g.half : g.n;
    f.octets = (g.n + 7) / 8;
    f.all = (int64_t)(g.partial ? g.m : 0) * f.octets;
    f.sum_rows = g.sum_rows ? g.sum_rows : g.splits;
    f.sum_step = g.m;
    if (g.sums && g.sum_rows > FOLD_FROM) {
        const int most = g.sum_rows > 16384 ? 256 : 64, chunk = (g.sum_rows + most - 1) / most;
        f.sum_rows = (g.sum_rows + chunk - 1) / chunk;
        f.sum_step = (int64_t)g.m * chunk;
        k_fold<<<dim3((g.m + 63) / 64, f.sum_rows), 256, 0, st>>>(g.sums, g.sum_rows, g.m, chunk);
    }
    // The rows of C share the launch with the sums, whose few threads may take as long as a launch for their rows; more of those have one of their own.
    if (g.partial && g.sums && f.sum_rows > g.splits && f.sum_rows > 64) {
        FinishArgs c = f;
        c.g.sums = nullptr;
        start_finish<T>(c, f.all, g.splits, st);
        f.all = 0;
        f.g.partial = nullptr;
        start_finish<T>(f, (g.m + 7) / 8, f.sum_rows, st);
    } else {
        start_finish<T>(f, f.all + (g.sums ? (g.m + 7) / 8 : 0), g.partial ? g.splits : f.sum_rows, st);
    }
    return hipGetLastError();
}

}  // namespace srd

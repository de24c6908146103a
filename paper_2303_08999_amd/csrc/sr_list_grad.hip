// Gradient of the per-pixel list form (sr_dict_assemble_list) with respect to its values and to the dictionary
// (include/sr_route.h).  The image is y_ic = F_i . B_ic with F_i = sum_t v_t D[idx_t], so with E_i = sum_c dy_ic B_ic
//
//     dv_t = D[idx_t] . E_i          dD[l] = sum over the entries that name l of v_t E_i
//
// E is formed tile by tile (stage 1 as in every kernel) and never leaves the workgroup.
//
// Here: checks, and the kernel that takes every case: a thread forms a pixel's E and the products of its entries, a
// wavefront adds the entries of every fourth atom to the tile's dD, a tap per lane, in the order of the pixels: 256 times the entries,
// one after the other, for every tile.  It is what the matrix-core kernel has no form for (list_grad_mfma_supported), and far slower: a 1080p
// frame of 8 entries, 5x5, fp16, 129 atoms 3.0 ms (128 atoms there 0.25), 2 or 4 channels of 72 atoms 3.0 ms (3 channels 0.13), 17 entries
// 6.5 ms (16 entries 0.17), 16 entries of 129 atoms of 7x7 11.7 ms (128 atoms 0.49).
#include <string.h>

#include "sr_list_grad.h"

namespace srd {
namespace {

constexpr int GTW = 64, GTH = 4, GNT = GTW * GTH;
constexpr int FLUSH = 16;                    // tiles (of 256 pixels) whose sums are held in fp32

template <typename TV, typename TIO, int K>
__global__ __launch_bounds__(GNT) void k_list_grad(const ListGradArgs a) {
    constexpr int KK = K * K, R = (K - 1) / 2;
    constexpr int UW = GTW + K - 1, UH = GTH + K - 1;
    constexpr int MAXLRY = (UH - 1) / 2 + 5, MAXLRX = (UW - 1) / 2 + 5;     // scale >= 2
    constexpr int TC = 8;                            // entries looked at together
    extern __shared__ float dyn[];
    float* El = dyn;                                 // [GNT][KK]: the tile's E (KK is odd: no bank conflicts either way)
    float* acc = dyn + GNT * KK;                     // [L][KK]: dD of the last tiles
    __shared__ float lrT[MAXLRY * MAXLRX];
    __shared__ float V[UH * MAXLRX];
    __shared__ float U[UH * UW];
    __shared__ float4 xw[UW], yw[UH];
    __shared__ int xb[UW], yb[UH];
    __shared__ unsigned char si[TC][GNT];
    __shared__ float sv[TC][GNT];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int tx = tid % GTW, ty = tid / GTW;
    const size_t plane = (size_t)a.H * a.W;
    const unsigned lmax = (unsigned)a.L - 1u;
    const int sums = a.L * KK;
    double* rec = a.partial ? a.partial + (size_t)blockIdx.x * sums : nullptr;
    if (rec)
        for (int e = tid; e < sums; e += GNT) acc[e] = 0.0f, rec[e] = 0.0;
    int held = 0;

    for (int64_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
        const int n = (int)(tile / ((int64_t)a.tiles_x * a.tiles_y));
        const int in = (int)(tile - (int64_t)n * a.tiles_x * a.tiles_y);
        const int Y0 = in / a.tiles_x * GTH, X0 = in % a.tiles_x * GTW;
        const int Y = Y0 + ty, X = X0 + tx;
        const bool inside = Y < a.H && X < a.W;
        const size_t at = (size_t)Y * a.W + X;
        const bool on = inside && (!a.mask || a.mask[(size_t)n * plane + at] != 0);

        float E[KK];
#pragma unroll
        for (int j = 0; j < KK; ++j) E[j] = 0.0f;
        const TileOrigin o = tile_origin(Y0, X0, R, UH, UW, a.H, a.W, a.s);
        __syncthreads();
        build_taps<UW, MAXLRX, GNT>(X0, R, a.W, a.s, o.lx0, xw, xb, tid);
        build_taps<UH, MAXLRY, GNT>(Y0, R, a.H, a.s, o.ly0, yw, yb, tid);
        for (int c = 0; c < a.C; ++c) {
            const size_t pl = (size_t)n * a.C + c;
            load_lr_tile<TIO, MAXLRY, MAXLRX, GNT>((const TIO*)a.lr + pl * (size_t)a.h * a.w, a.h, a.w, o, lrT, tid);
            __syncthreads();
            vpass<MAXLRX, UH, GNT>(lrT, V, yw, yb, tid);
            __syncthreads();
            hpass<MAXLRX, UW, UH, GNT>(V, xw, xb, tid, [&](int yy, int xx, float v) { U[yy * UW + xx] = v; });
            __syncthreads();
            const float dy = on ? ld_as_float((const TIO*)a.dout, pl * plane + at) : 0.0f;
#pragma unroll
            for (int j = 0; j < KK; ++j) E[j] = fmaf(dy, U[(ty + j / K) * UW + tx + j % K], E[j]);
        }
#pragma unroll
        for (int j = 0; j < KK; ++j) El[tid * KK + j] = E[j];

        for (int t0 = 0; t0 < a.T; t0 += TC) {
            const int tn = a.T - t0 < TC ? a.T - t0 : TC;
            __syncthreads();                         // E is there; the entries before these have been used
            for (int t = 0; t < tn; ++t) {
                const size_t e = ((size_t)n * a.T + t0 + t) * plane + at;
                unsigned l = inside ? (unsigned)a.index[e] : 0u;
                l = l < lmax ? l : lmax;             // an index not below L never reaches outside the tables
                si[t][tid] = (unsigned char)l;
                sv[t][tid] = on ? ld_as_float((const TV*)a.value, e) : 0.0f;
                if (a.dvalue && inside) {
                    const float* d = a.dict + (size_t)l * KK;
                    float dot = 0.0f;
#pragma unroll
                    for (int j = 0; j < KK; ++j) dot = fmaf(d[j], E[j], dot);
                    st_from_float((TV*)a.dvalue, e, on ? dot : 0.0f);
                }
            }
            __syncthreads();
            if (rec)
                for (int p = 0; p < GNT; ++p) {
                    const float e = lane < KK ? El[p * KK + lane] : 0.0f;
                    for (int t = 0; t < tn; ++t) {
                        const int l = si[t][p];
                        if ((l & 3) == wave && lane < KK) acc[l * KK + lane] = fmaf(sv[t][p], e, acc[l * KK + lane]);
                    }
                }
        }
        if (rec && ++held == FLUSH) {
            held = 0;
            __syncthreads();
            for (int e = tid; e < sums; e += GNT) rec[e] += acc[e], acc[e] = 0.0f;
        }
    }
    if (rec) {
        __syncthreads();
        for (int e = tid; e < sums; e += GNT) rec[e] += acc[e];
    }
}

// ddict = the workgroups' sums, in their order: 16 values a workgroup, 16 runs of records each, eight records' loads under way at a time
// (32 values, one record after the other, took 19 us of 512 records).
constexpr int DNT = 256, DVAL = 16, DRUNS = DNT / DVAL, DAHEAD = 8;
__global__ __launch_bounds__(DNT) void k_list_grad_finish(const double* partial, int records, int sums, float* ddict) {
    __shared__ double sh[DNT];
    const int tid = threadIdx.x, g = tid / DVAL, e = blockIdx.x * DVAL + tid % DVAL;
    const int run = (records + DRUNS - 1) / DRUNS, end = min(records, (g + 1) * run);
    double s = 0.0;
    if (e < sums)
        for (int r0 = g * run; r0 < end; r0 += DAHEAD) {
            double v[DAHEAD];
#pragma unroll
            for (int i = 0; i < DAHEAD; ++i) v[i] = partial[(size_t)min(r0 + i, end - 1) * sums + e];
#pragma unroll
            for (int i = 0; i < DAHEAD; ++i)
                if (r0 + i < end) s += v[i];
        }
    sh[tid] = s;
    __syncthreads();
    if (g == 0 && e < sums) {
        for (int k = 1; k < DRUNS; ++k) s += sh[k * DVAL + tid];
        ddict[e] = (float)s;
    }
}

template <typename TV, typename TIO, int K>
hipError_t launch_one(const ListGradArgs& a, int grid, hipStream_t st) {
    const size_t lds = ((size_t)GNT + (a.partial ? a.L : 0)) * K * K * sizeof(float);
    if (lds > 48 * 1024) {
        const hipError_t e = hipFuncSetAttribute((const void*)k_list_grad<TV, TIO, K>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    k_list_grad<TV, TIO, K><<<grid, GNT, lds, st>>>(a);
    return hipGetLastError();
}
template <typename TV, typename TIO>
hipError_t launch_k(const ListGradArgs& a, int k, int grid, hipStream_t st) {
    return k == 3 ? launch_one<TV, TIO, 3>(a, grid, st) : k == 5 ? launch_one<TV, TIO, 5>(a, grid, st) : launch_one<TV, TIO, 7>(a, grid, st);
}

size_t grad_esize(sr_dtype d) { return d == SR_F32 ? 4 : (d == SR_U8 ? 1 : 2); }
size_t tensor_bytes(const sr_tensor* t) { return (size_t)t->n * t->c * t->h * t->w * grad_esize(t->dtype); }
bool overlap(const void* p, size_t np, const void* q, size_t nq) {
    const uintptr_t a0 = (uintptr_t)p, b0 = (uintptr_t)q;
    return p && q && np && nq && a0 < b0 + nq && b0 < a0 + np;
}

}  // namespace

bool list_grad_mfma_supported(const ListGradArgs& a, int k) {
    (void)k;
    // an image's lists and its dout lie within 32-bit offsets, as bytes of fp32
    return a.T <= 16 && a.L <= 128 && (a.C == 1 || a.C == 3) && (int64_t)a.H * a.W * (a.T > 3 ? a.T : 3) < (int64_t)1 << 30 &&
           (int64_t)a.N * ((a.W + GM_TW - 1) / GM_TW) * ((a.H + GM_TH - 1) / GM_TH) < (int64_t)1 << 30;
}

}  // namespace srd

using namespace srd;

extern "C" __attribute__((visibility("default")))
size_t sr_dict_assemble_list_grad_workspace_bytes(int L, int k) {
    return L < 1 || L > SR_MAX_ATOMS || (k != 3 && k != 5 && k != 7) ? 0 : (size_t)GRAD_RECORDS * L * k * k * 8;
}

extern "C" __attribute__((visibility("default")))
int sr_dict_assemble_list_grad(const sr_tensor* lr, const sr_tensor* index, const sr_tensor* value, const sr_tensor* dict,
                               int L, int k, int scale, int channels, int entries, const sr_tensor* mask,
                               const sr_tensor* dout, sr_tensor* dvalue, sr_tensor* ddict,
                               void* workspace, size_t workspace_bytes, void* stream) {
    if (!lr || !index || !value || !dict || !dout || (!dvalue && !ddict)) return SR_ERR_NULL;
    if ((lr->dtype != SR_F32 && lr->dtype != SR_F16) || dout->dtype != lr->dtype || index->dtype != SR_U8 ||
        (value->dtype != SR_F32 && value->dtype != SR_F16) || dict->dtype != SR_F32 || (mask && mask->dtype != SR_U8) ||
        (dvalue && dvalue->dtype != value->dtype) || (ddict && ddict->dtype != SR_F32)) return SR_ERR_UNSUPPORTED;
    for (const sr_tensor* t : {lr, index, value, dict, mask, dout, (const sr_tensor*)dvalue, (const sr_tensor*)ddict})
        if (t && (t->n < 0 || t->c < 0 || t->h < 0 || t->w < 0)) return SR_ERR_SHAPE;
    if ((k != 3 && k != 5 && k != 7) || scale < 2 || scale > 4 || L < 1 || L > SR_MAX_ATOMS || channels < 1 ||
        channels > SR_MAX_CHANNELS || entries < 1 || entries > SR_MAX_ATOMS) return SR_ERR_UNSUPPORTED;
    const int64_t H = (int64_t)lr->h * scale, W = (int64_t)lr->w * scale;
    if (lr->c != channels || dout->c != channels || index->c != entries || value->c != entries || (mask && mask->c != 1) ||
        (dvalue && dvalue->c != entries)) return SR_ERR_SHAPE;
    for (const sr_tensor* t : {index, value, mask, dout, (const sr_tensor*)dvalue})
        if (t && (t->n != lr->n || t->h != H || t->w != W)) return SR_ERR_SHAPE;
    for (const sr_tensor* t : {dict, (const sr_tensor*)ddict})
        if (t && (t->n != 1 || t->c != L || t->h != k || t->w != k)) return SR_ERR_SHAPE;
    if (lr->n > 65535 || H > 4 * 65535 || W > (1 << 20)) return SR_ERR_UNSUPPORTED;
    const bool empty = lr->n == 0 || lr->h == 0 || lr->w == 0;
    if (!dict->data || (ddict && !ddict->data)) return SR_ERR_NULL;
    if (!empty && (!lr->data || !index->data || !value->data || !dout->data || (mask && !mask->data) || (dvalue && !dvalue->data)))
        return SR_ERR_NULL;
    for (const sr_tensor* t : {lr, value, dict, dout, (const sr_tensor*)dvalue, (const sr_tensor*)ddict})
        if (t && (uintptr_t)t->data % grad_esize(t->dtype)) return SR_ERR_ALIGN;
    const size_t need = sr_dict_assemble_list_grad_workspace_bytes(L, k);
    if (ddict && (!workspace || workspace_bytes < need)) return SR_ERR_SHAPE;
    if (ddict && (uintptr_t)workspace % 16) return SR_ERR_ALIGN;
    {
        struct Span { const void* p; size_t n; };
        const Span out[] = {{dvalue ? dvalue->data : nullptr, dvalue ? tensor_bytes(dvalue) : 0},
                            {ddict ? ddict->data : nullptr, ddict ? tensor_bytes(ddict) : 0}, {ddict ? workspace : nullptr, need}};
        for (int i = 0; i < 3; ++i) {
            for (const sr_tensor* t : {lr, index, value, dict, mask, dout})
                if (t && overlap(out[i].p, out[i].n, t->data, tensor_bytes(t))) return SR_ERR_ALIAS;
            for (int j = 0; j < i; ++j)
                if (overlap(out[i].p, out[i].n, out[j].p, out[j].n)) return SR_ERR_ALIAS;
        }
    }
    const hipStream_t st = (hipStream_t)stream;
    hipError_t e = hipSuccess;
    int records = 0;
    if (!empty) {
        ListGradArgs a;
        memset(&a, 0, sizeof(a));
        a.lr = lr->data; a.index = (const unsigned char*)index->data; a.value = value->data; a.dict = (const float*)dict->data;
        a.mask = mask ? (const unsigned char*)mask->data : nullptr;
        a.dout = dout->data; a.dvalue = dvalue ? dvalue->data : nullptr; a.partial = ddict ? (double*)workspace : nullptr;
        a.N = lr->n; a.C = channels; a.h = lr->h; a.w = lr->w; a.H = (int)H; a.W = (int)W; a.s = scale; a.L = L; a.T = entries;
        a.io_f16 = lr->dtype == SR_F16;
        const bool mfma = list_grad_mfma_supported(a, k);
        const int tw = mfma ? GM_TW : GTW, th = mfma ? GM_TH : GTH;
        a.tiles_x = (a.W + tw - 1) / tw; a.tiles_y = (a.H + th - 1) / th;
        a.tiles = (int64_t)a.N * a.tiles_x * a.tiles_y;
        const int most = mfma ? 2 * compute_units() : (ddict ? GRAD_RECORDS : 4 * compute_units());
        const int limit = most < GRAD_RECORDS || !ddict ? most : GRAD_RECORDS;
        const int grid = (int)(a.tiles < limit ? a.tiles : limit);
        records = grid;
        if (mfma)
            e = value->dtype == SR_F16 ? launch_list_grad_mfma<__half>(a, k, grid, st) : launch_list_grad_mfma<float>(a, k, grid, st);
        else if (value->dtype == SR_F16)
            e = lr->dtype == SR_F16 ? launch_k<__half, __half>(a, k, grid, st) : launch_k<__half, float>(a, k, grid, st);
        else
            e = lr->dtype == SR_F16 ? launch_k<float, __half>(a, k, grid, st) : launch_k<float, float>(a, k, grid, st);
    }
    if (e == hipSuccess && ddict) {
        const int sums = L * k * k;
        k_list_grad_finish<<<(sums + DVAL - 1) / DVAL, DNT, 0, st>>>((const double*)workspace, records, sums, (float*)ddict->data);
        e = hipGetLastError();
    }
    return e == hipSuccess ? SR_OK : SR_ERR_LAUNCH;
}

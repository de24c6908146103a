// The norm of all gradients, and clipping (include/sr_layer.h, sr_grad_clip).
//
// The tensors' addresses travel in the kernels' arguments, so that a call can be captured and nothing is kept between calls; a launch takes
// up to CLIP_TENSORS of them.  First pass: the tensors are cut into chunks of 16-byte pieces, workgroup b takes chunks b, b + grid, ... and
// leaves the sum of its squares, in double.  Second pass: every workgroup adds these sums up in the same order, and scales its chunks, the
// last ones first: what the first pass read last is what the caches still hold.  Bound by memory: read twice, written once.
#include <math.h>
#include <stdint.h>

#include "sr_gemm.h"

namespace srd {
namespace {

constexpr int CLIP_TENSORS = 128, CLIP_RECORDS = 2048, CNT = 256;
constexpr int CHUNK_PIECES = CNT * 8;          // 32 KB

struct ClipArgs {
    const void* in[CLIP_TENSORS];
    void* out[CLIP_TENSORS];
    int64_t count[CLIP_TENSORS];               // elements
    int chunk[CLIP_TENSORS + 1];               // a tensor's first chunk
    unsigned char type[CLIP_TENSORS];
    int tensors, first, records;               // first: of this launch's records; records: of all launches (second pass)
    int pieces;                                // of a chunk
    double* partial;
    double most;
    float* norm;
    int tells;                                 // this launch's first workgroup writes the norm
};
static_assert(sizeof(ClipArgs) <= 4096, "kernel arguments");

// A chunk's part of a tensor of T: elements before the first 16-byte boundary belong to the first chunk, those behind the last to the last.
struct Part { int64_t head, body, from, to, count; };       // head elements, pieces in all, this chunk's pieces, elements in all
template <typename T> __device__ __forceinline__ Part part_of(const void* p, int64_t count, int chunk, int pieces) {
    constexpr int E = 16 / sizeof(T);
    Part r;
    int64_t head = ((16 - ((uintptr_t)p & 15)) & 15) / sizeof(T);
    r.head = head < count ? head : count;
    r.body = (count - r.head) / E;
    r.from = (int64_t)chunk * pieces;
    r.to = r.from + pieces < r.body ? r.from + pieces : r.body;
    r.count = count;
    return r;
}
// f(element) for what is no whole piece, if this chunk has it
template <typename T, typename F> __device__ __forceinline__ void edges(const Part& r, int pieces, F f) {
    constexpr int E = 16 / sizeof(T);
    if (r.from == 0 && (int64_t)threadIdx.x < r.head) f((int64_t)threadIdx.x);
    const int64_t tail = r.head + r.body * E;
    if (r.from + pieces >= r.body && (r.from < r.body || r.from == 0) && tail + (int64_t)threadIdx.x < r.count) f(tail + threadIdx.x);
}

// The last tensor that begins at or before the chunk: a lane looks at two, all at once (a search by halves waits for memory seven times).
__device__ __forceinline__ int tensor_of(const ClipArgs& a, int chunk) {
    static_assert(CLIP_TENSORS == 128, "two a lane");
    const int lane = threadIdx.x & 63;
    const bool lo = lane < a.tensors && a.chunk[lane] <= chunk, hi = 64 + lane < a.tensors && a.chunk[64 + lane] <= chunk;
    return __builtin_amdgcn_readfirstlane(__popcll(__ballot(lo)) + __popcll(__ballot(hi)) - 1);
}

template <typename T> __device__ __forceinline__ void unpack(u32x4g v, float x[16 / sizeof(T)]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            x[i] = __uint_as_float(v[i]);
        } else if constexpr (__is_same(T, __half)) {
            using half2g = __attribute__((ext_vector_type(2))) _Float16;
            const half2g h = __builtin_bit_cast(half2g, (unsigned)v[i]);
            x[2 * i] = (float)h[0], x[2 * i + 1] = (float)h[1];
        } else {
            x[2 * i] = __uint_as_float(v[i] << 16), x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
        }
    }
}

// A thread's pieces of a chunk from `at` on, BATCH of them, all under way at once; what is behind the chunk's last is 0
constexpr int BATCH = 8;
template <typename T> __device__ __forceinline__ void ask(const void* p, const Part& r, int64_t at, u32x4g w[BATCH]) {
    const u32x4g* const v = (const u32x4g*)((const T*)p + r.head) + at + threadIdx.x;
#pragma unroll
    for (int j = 0; j < BATCH; ++j) w[j] = at + threadIdx.x + j * CNT < r.to ? v[j * CNT] : u32x4g{0, 0, 0, 0};
}

template <typename T> __device__ __forceinline__ double squares(const void* p, int64_t count, int chunk, int pieces) {
    constexpr int E = 16 / sizeof(T);
    const Part r = part_of<T>(p, count, chunk, pieces);
    const T* const q = (const T*)p;
    double s = 0.0;
    for (int64_t at = r.from; at < r.to; at += BATCH * CNT) {
        u32x4g w[BATCH];
        ask<T>(p, r, at, w);
#pragma unroll
        for (int j = 0; j < BATCH; ++j) {
            float x[E];
            unpack<T>(w[j], x);
#pragma unroll
            for (int e = 0; e < E; ++e) s = fma((double)x[e], (double)x[e], s);
        }
    }
    edges<T>(r, pieces, [&](int64_t e) { const double x = gm_get(q + e); s = fma(x, x, s); });
    return s;
}

// first: the first BATCH pieces of each thread are in w already
template <typename T> __device__ __forceinline__ void scale(const void* p, void* o, int64_t count, int chunk, int pieces, float f, bool first, u32x4g w[BATCH]) {
    constexpr int E = 16 / sizeof(T);
    const Part r = part_of<T>(p, count, chunk, pieces);
    const T* const q = (const T*)p;
    T* const d = (T*)o;
    for (int64_t at = r.from; at < r.to; at += BATCH * CNT) {
        if (!first) ask<T>(p, r, at, w);
        first = false;
#pragma unroll
        for (int j = 0; j < BATCH; ++j) {
            const int64_t i = at + threadIdx.x + j * CNT;
            float x[E];
            unpack<T>(w[j], x);
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] *= f;
            if (i >= r.to) continue;
            if constexpr (sizeof(T) == 4) {
                u32x4u y;
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = __float_as_uint(x[e]);
                *(u32x4u*)(d + r.head + i * E) = y;
            } else {
                gm_put8(d + r.head + i * E, x);
            }
        }
    }
    edges<T>(r, pieces, [&](int64_t e) { gm_put(d + e, gm_get(q + e) * f); });
}

// The workgroup's sum, in every thread
__device__ __forceinline__ double block_sum(double s) {
    __shared__ double sh[CNT / 64];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int w = 0; w < CNT / 64; ++w) s += sh[w];
    return s;
}

__global__ __launch_bounds__(CNT) void k_clip_squares(const ClipArgs a) {
    double s = 0.0;
    for (int c = blockIdx.x; c < a.chunk[a.tensors]; c += gridDim.x) {
        const int t = tensor_of(a, c), at = c - a.chunk[t];
        if (a.type[t] == SR_F32) s += squares<float>(a.in[t], a.count[t], at, a.pieces);
        else if (a.type[t] == SR_F16) s += squares<__half>(a.in[t], a.count[t], at, a.pieces);
        else s += squares<bf16raw>(a.in[t], a.count[t], at, a.pieces);
    }
    s = block_sum(s);
    if (threadIdx.x == 0) a.partial[a.first + blockIdx.x] = s;
}

__global__ __launch_bounds__(CNT) void k_clip_scale(const ClipArgs a) {
    // the first chunk's pieces are on their way while the sums are added up
    u32x4g w[BATCH];
    const int last = a.chunk[a.tensors] - 1 - (int)blockIdx.x;
    if (last >= 0) {
        const int t = tensor_of(a, last), at = last - a.chunk[t];
        if (a.type[t] == SR_F32) {
            const Part r = part_of<float>(a.in[t], a.count[t], at, a.pieces);
            ask<float>(a.in[t], r, r.from, w);
        } else {
            const Part r = part_of<__half>(a.in[t], a.count[t], at, a.pieces);
            ask<__half>(a.in[t], r, r.from, w);
        }
    }
    double s = 0.0;
    for (int i = threadIdx.x; i < a.records; i += CNT) s += a.partial[i];
    const double norm = sqrt(block_sum(s));
    const float factor = norm > a.most && norm < INFINITY ? (float)(a.most / norm) : 1.0f;
    if (a.tells && blockIdx.x == 0 && threadIdx.x == 0) a.norm[0] = (float)norm, a.norm[1] = factor;
    for (int c = last; c >= 0; c -= gridDim.x) {
        const int t = tensor_of(a, c), at = c - a.chunk[t];
        if (factor == 1.0f && a.out[t] == a.in[t]) continue;
        if (a.type[t] == SR_F32) scale<float>(a.in[t], a.out[t], a.count[t], at, a.pieces, factor, c == last, w);
        else if (a.type[t] == SR_F16) scale<__half>(a.in[t], a.out[t], a.count[t], at, a.pieces, factor, c == last, w);
        else scale<bf16raw>(a.in[t], a.out[t], a.count[t], at, a.pieces, factor, c == last, w);
    }
}

size_t esize_of(int d) { return d == SR_F32 ? 4 : 2; }
size_t count_of(const sr_tensor& t) { return (size_t)t.n * t.c * t.h * t.w; }

struct Range { uintptr_t from, to; int tensor; };              // tensor: of outs; -1 - i: gradient i
// Ranges by address (heap sort: nothing is allocated)
void sort_ranges(Range* r, int n) {
    auto sift = [&](int i, int end) {
        const Range x = r[i];
        for (int c; (c = 2 * i + 1) < end; i = c) {
            if (c + 1 < end && r[c].from < r[c + 1].from) ++c;
            if (x.from >= r[c].from) break;
            r[i] = r[c];
        }
        r[i] = x;
    };
    for (int i = n / 2 - 1; i >= 0; --i) sift(i, n);
    for (int e = n - 1; e > 0; --e) {
        const Range x = r[0];
        r[0] = r[e];
        r[e] = x;
        sift(0, e);
    }
}
int clip_launches(int tensors) { return (tensors + CLIP_TENSORS - 1) / CLIP_TENSORS; }

}  // namespace
}  // namespace srd

using namespace srd;

extern "C" __attribute__((visibility("default")))
size_t sr_grad_clip_workspace_bytes(int tensors) {
    return tensors < 1 || tensors > SR_MAX_GRADS ? 0 : (size_t)clip_launches(tensors) * CLIP_RECORDS * sizeof(double);
}

extern "C" __attribute__((visibility("default")))
int sr_grad_clip(const sr_tensor* grads, const sr_tensor* outs, int tensors, double max_norm, float* norm,
                 void* workspace, size_t workspace_bytes, void* stream) {
    if (!grads || !norm) return SR_ERR_NULL;
    if (tensors < 1 || tensors > SR_MAX_GRADS || !(max_norm >= 0.0)) return SR_ERR_UNSUPPORTED;
    const size_t need = sr_grad_clip_workspace_bytes(tensors);
    for (int i = 0; i < tensors; ++i) {
        const sr_tensor& g = grads[i];
        if (g.dtype != SR_F32 && g.dtype != SR_F16 && g.dtype != SR_BF16) return SR_ERR_UNSUPPORTED;
        if (g.n < 0 || g.c < 0 || g.h < 0 || g.w < 0) return SR_ERR_SHAPE;
        // 2^40 elements: chunks are numbered in 32 bits
        const double all = (double)g.n * g.c * g.h * g.w;
        if (all > 1099511627776.0) return SR_ERR_UNSUPPORTED;
        const bool any = all > 0.0;
        if (any && !g.data) return SR_ERR_NULL;
        if (any && (uintptr_t)g.data % esize_of(g.dtype)) return SR_ERR_ALIGN;
        if (outs) {
            const sr_tensor& o = outs[i];
            if (o.dtype != g.dtype) return SR_ERR_UNSUPPORTED;
            if (o.n != g.n || o.c != g.c || o.h != g.h || o.w != g.w) return SR_ERR_SHAPE;
            if (any && !o.data) return SR_ERR_NULL;
            if (any && (uintptr_t)o.data % esize_of(g.dtype)) return SR_ERR_ALIGN;
        }
    }
    if (!workspace || workspace_bytes < need) return SR_ERR_SHAPE;
    if ((uintptr_t)workspace % 16 || (uintptr_t)norm % 4) return SR_ERR_ALIGN;
    {
        // Everything that is read or written by address; an output may meet nothing but its own gradient, which it has to cover exactly, and
        // gradients may meet one another.
        Range r[2 * SR_MAX_GRADS + 2];
        int n = 0;
        for (int i = 0; i < tensors; ++i) {
            const size_t bytes = count_of(grads[i]) * esize_of(grads[i].dtype);
            if (!bytes) continue;
            const uintptr_t g = (uintptr_t)grads[i].data, o = outs ? (uintptr_t)outs[i].data : g;
            if (o == g && outs) r[n++] = Range{o, o + bytes, i};
            else {
                r[n++] = Range{g, g + bytes, -1 - i};
                if (outs) r[n++] = Range{o, o + bytes, i};
            }
        }
        r[n++] = Range{(uintptr_t)norm, (uintptr_t)norm + 8, SR_MAX_GRADS};
        r[n++] = Range{(uintptr_t)workspace, (uintptr_t)workspace + need, SR_MAX_GRADS};
        sort_ranges(r, n);
        uintptr_t read_to = 0, written_to = 0;
        for (int i = 0; i < n; ++i) {
            const bool written = r[i].tensor >= 0;
            if (r[i].from < written_to || (written && r[i].from < read_to)) return SR_ERR_ALIAS;
            uintptr_t& to = written ? written_to : read_to;
            if (r[i].to > to) to = r[i].to;
        }
    }
    const int launches = clip_launches(tensors);
    hipStream_t st = (hipStream_t)stream;
    hipError_t e = hipSuccess;
    int records = 0, grids[(SR_MAX_GRADS + CLIP_TENSORS - 1) / CLIP_TENSORS];
    // launch l: tensors l * CLIP_TENSORS on
    auto fill = [&](ClipArgs& a, int l) {
        const int from = l * CLIP_TENSORS, n = tensors - from < CLIP_TENSORS ? tensors - from : CLIP_TENSORS;
        a.tensors = n;
        double all = 0.0;
        for (int i = 0; i < n; ++i) all += (double)count_of(grads[from + i]) * (double)esize_of(grads[from + i].dtype);
        a.pieces = CHUNK_PIECES;
        while ((double)a.pieces * 16.0 * 1e6 < all) a.pieces *= 2;      // chunk numbers stay far below 32 bits
        int chunk = 0;
        for (int i = 0; i < n; ++i) {
            const sr_tensor& g = grads[from + i];
            a.in[i] = g.data;
            a.out[i] = outs ? outs[from + i].data : nullptr;
            a.count[i] = (int64_t)count_of(g);
            a.type[i] = (unsigned char)g.dtype;
            a.chunk[i] = chunk;
            const int64_t pieces = (a.count[i] * (int64_t)esize_of(g.dtype) + 15) / 16;
            chunk += (int)((pieces + a.pieces - 1) / a.pieces);
        }
        a.chunk[n] = chunk;
        a.partial = (double*)workspace;
        a.most = max_norm;
        a.norm = norm;
    };
    ClipArgs a;
    for (int l = 0; l < launches && e == hipSuccess; ++l) {
        fill(a, l);
        const int chunks = a.chunk[a.tensors];
        grids[l] = chunks < 1 ? 1 : chunks < CLIP_RECORDS / launches ? chunks : CLIP_RECORDS / launches > 256 ? CLIP_RECORDS / launches : chunks < 256 ? chunks : 256;
        a.first = records;
        a.records = a.tells = 0;
        records += grids[l];
        k_clip_squares<<<grids[l], CNT, 0, st>>>(a);
        e = hipGetLastError();
    }
    for (int l = launches - 1; l >= 0 && e == hipSuccess; --l) {
        if (launches > 1) fill(a, l);
        a.records = records;
        a.tells = l == launches - 1;
        int grid = grids[l];
        if (!outs) {                                       // the norm alone
            if (!a.tells) continue;
            a.tensors = 0;
            a.chunk[0] = 0;
            grid = 1;
        }
        k_clip_scale<<<grid, CNT, 0, st>>>(a);
        e = hipGetLastError();
    }
    return e == hipSuccess ? SR_OK : SR_ERR_LAUNCH;
}

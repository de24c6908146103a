// The router's kernels for many pixels: one to four lanes (G) hold a pixel's logits in registers, eight atoms at a time.
//
// Selection: a sorted list of TC keys per lane; a new key x moves into it with one median each, a_i' = med3(a_{i-1}, x, a_i).
// A key of a 16-bit logit is one 32-bit integer, the logit's order above and the atom (lower ones first) below; fp32 logits
// keep the atom beside the key (med3, a compare and two selects for each place).  The lists of a pixel's G lanes are merged as
// bitonic sequences.  The softmax runs over the same registers once the largest logit is known: one pass over memory.
#pragma once
#include "sr_route.h"

namespace srd {

constexpr int LCH = 9;                   // chunks of 8 atoms that a lane holds: 72 atoms, times G

// What the lanes of a pixel walk: images of ipx pixels, each with its logits lstride apart (the order before the pixel-shuffle is
// s * s such images for every frame: one for each place under an LR pixel).
struct LaneArgs {
    RouteArgs r;
    int64_t ipx, tiles_per_image, tiles;
    int vec;                             // pixel-major rows of whole, aligned 16-byte pieces
    int half_value;                      // values (dvalue) are fp16, else fp32
};

__device__ __forceinline__ int med3i(int a, int b, int c) {
    int d;
    asm("v_med3_i32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
    return d;
}
__device__ __forceinline__ unsigned med3u(unsigned a, unsigned b, unsigned c) {
    unsigned d;
    asm("v_med3_u32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
    return d;
}

typedef short short2v __attribute__((ext_vector_type(2)));

// Eight logits as they are stored: 16-bit ones two in a word.
template <typename TZ> struct Chunk {                        // __half, bf16raw
    static constexpr int WORDS = 4;
    unsigned w[4];
    // atom 0 at `at + off` (`at` the same for the whole wavefront), the next `stride` bytes on; the first n of them
    template <bool ALL> __device__ __forceinline__ void load(const char* at, unsigned off, int64_t stride, int n) {
        unsigned v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j, at += stride) v[j] = ALL || j < n ? (unsigned)*(const unsigned short*)(at + off) : 0u;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = v[2 * j] | (v[2 * j + 1] << 16);
    }
    __device__ __forceinline__ void load_vec(const char* at, unsigned off) {
        const uint4 v = *(const uint4*)(at + off);
        w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    }
    __device__ __forceinline__ float get(int j) const;
    // signed order of the two logits of a word: negative ones mirrored, so that -0 is +0
    __device__ __forceinline__ unsigned order2(int i) const {
        short2v b, t, s;
        __builtin_memcpy(&b, &w[i], 4);
        s = b >> 15;
        t = (short)-32768 - b;
        const short2v o = (t & s) | (b & ~s);
        unsigned u;
        __builtin_memcpy(&u, &o, 4);
        return u;
    }
};
template <> __device__ __forceinline__ float Chunk<__half>::get(int j) const {
    __half h[2];
    __builtin_memcpy(h, &w[j / 2], 4);
    return __half2float(h[j & 1]);
}
template <> __device__ __forceinline__ float Chunk<bf16raw>::get(int j) const {
    return __uint_as_float(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
}
template <> struct Chunk<float> {
    static constexpr int WORDS = 8;
    float w[8];
    template <bool ALL> __device__ __forceinline__ void load(const char* at, unsigned off, int64_t stride, int n) {
#pragma unroll
        for (int j = 0; j < 8; ++j, at += stride) w[j] = ALL || j < n ? *(const float*)(at + off) : 0.0f;
    }
    __device__ __forceinline__ void load_vec(const char* at, unsigned off) {
        const float4 a = *(const float4*)(at + off), b = *(const float4*)(at + off + 16);
        w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
    }
    __device__ __forceinline__ float get(int j) const { return w[j]; }
};

// The largest keys so far.  `at` is a number below 256 that grows with the atom, the same for every lane of the wavefront
// (chunk and place in it); atoms_of turns it into the atom before lists of several lanes meet.
template <typename TZ, int TC> struct TopList {              // 16-bit logits
    int k[TC];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < TC; ++i) k[i] = (int)0x80000000;
    }
    __device__ __forceinline__ void put(int x) {
#pragma unroll
        for (int i = TC - 1; i > 0; --i) k[i] = med3i(k[i - 1], x, k[i]);
        k[0] = x > k[0] ? x : k[0];
    }
    template <bool ALL> __device__ __forceinline__ void insert(const Chunk<TZ>& c, int at, int n) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned o = c.order2(i);
            const int lo = (int)((o << 16) | (unsigned)(256 - (at + 2 * i))), hi = (int)((o & 0xffff0000u) | (unsigned)(255 - (at + 2 * i)));
            put(ALL || 2 * i < n ? lo : (int)0x80000000);
            put(ALL || 2 * i + 1 < n ? hi : (int)0x80000000);
        }
    }
    __device__ __forceinline__ int at(int t) const { return 256 - (k[t] & 0xffff); }
    __device__ __forceinline__ void set_at(int t, int l) {      // places without an atom stay below every key
        k[t] = k[t] == (int)0x80000000 ? k[t] : (k[t] & (int)0xffff0000) | (256 - l);
    }
    __device__ __forceinline__ float logit(int t) const {
        const int o = k[t] >> 16, b = o < 0 ? -32768 - o : o;
        Chunk<TZ> c;
        c.w[0] = (unsigned)b & 0xffffu;
        return c.get(0);
    }
    __device__ __forceinline__ void merge(int d) {
        int o[TC];
#pragma unroll
        for (int i = 0; i < TC; ++i) o[i] = __shfl_xor(k[i], d);
#pragma unroll
        for (int i = 0; i < TC; ++i) k[i] = k[i] > o[TC - 1 - i] ? k[i] : o[TC - 1 - i];
#pragma unroll
        for (int h = TC / 2; h > 0; h >>= 1)
#pragma unroll
            for (int i = 0; i < TC; ++i)
                if ((i & h) == 0) {
                    const int a = k[i], b = k[i + h];
                    k[i] = a > b ? a : b;
                    k[i + h] = a > b ? b : a;
                }
    }
};
template <int TC> struct TopList<float, TC> {
    unsigned k[TC];                      // 0: no atom yet (an atom's key is at least 1)
    int id[TC];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < TC; ++i) k[i] = 0, id[i] = 0;
    }
    __device__ __forceinline__ void put(unsigned x, int l) {
        bool c[TC];
#pragma unroll
        for (int i = 0; i < TC; ++i) c[i] = x > k[i];
#pragma unroll
        for (int i = TC - 1; i > 0; --i) {
            id[i] = c[i - 1] ? id[i - 1] : (c[i] ? l : id[i]);
            k[i] = med3u(k[i - 1], x, k[i]);
        }
        id[0] = c[0] ? l : id[0];
        k[0] = c[0] ? x : k[0];
    }
    template <bool ALL> __device__ __forceinline__ void insert(const Chunk<float>& c, int at, int n) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const unsigned o = logit_order(c.w[j]);
            put(ALL || j < n ? (o > 1u ? o : 1u) : 0u, at + j);
        }
    }
    __device__ __forceinline__ int at(int t) const { return id[t]; }
    __device__ __forceinline__ void set_at(int t, int l) { id[t] = l; }
    __device__ __forceinline__ float logit(int t) const {
        return __uint_as_float(k[t] & 0x80000000u ? k[t] ^ 0x80000000u : ~k[t]);
    }
    // larger keys first, of equal ones the lower atom; places without an atom last
    static __device__ __forceinline__ bool before(unsigned a, int ia, unsigned b, int ib) { return a > b || (a == b && ia < ib); }
    __device__ __forceinline__ void merge(int d) {
        unsigned o[TC];
        int oid[TC];
#pragma unroll
        for (int i = 0; i < TC; ++i) o[i] = __shfl_xor(k[i], d), oid[i] = __shfl_xor(id[i], d);
#pragma unroll
        for (int i = 0; i < TC; ++i)
            if (before(o[TC - 1 - i], oid[TC - 1 - i], k[i], id[i])) k[i] = o[TC - 1 - i], id[i] = oid[TC - 1 - i];
#pragma unroll
        for (int h = TC / 2; h > 0; h >>= 1)
#pragma unroll
            for (int i = 0; i < TC; ++i)
                if ((i & h) == 0) {
                    const unsigned a = k[i], b = k[i + h];
                    const int ia = id[i], ib = id[i + h];
                    const bool sw = before(b, ib, a, ia);
                    k[i] = sw ? b : a, id[i] = sw ? ib : ia;
                    k[i + h] = sw ? a : b, id[i + h] = sw ? ia : ib;
                }
    }
};

// The pixel of a lane: where its logits, its list and its mask are.
struct LanePixel {
    bool inside;
    int g;
    const char* at;                      // logits: atom 0 of the tile's first pixel, the same for the whole wavefront,
    unsigned off;                        // ... and from there to the lane's first atom, in bytes
    int64_t out, mask;                   // entry 0 in the [N][T][H][W] tensors; the pixel in [N][H][W]
};
template <typename TZ, int G>
__device__ __forceinline__ LanePixel lane_pixel(const LaneArgs& a, int64_t tile, int lane) {
    constexpr int P = 64 / G;            // pixels of a wavefront; a pixel's lanes are P apart, but next to one another where rows of
                                         // logits are contiguous
    const RouteArgs& r = a.r;
    const bool pm = r.layout == SR_COEFF_PIXEL_MAJOR;
    LanePixel p;
    p.g = G == 1 ? 0 : (pm ? lane % G : lane / P);
    const int q = G == 1 ? lane : (pm ? lane / G : lane % P);
    const int64_t m = tile / a.tiles_per_image, i0 = (tile - m * a.tiles_per_image) * P, i = i0 + q;
    p.inside = i < a.ipx;
    p.off = (unsigned)sizeof(TZ) * (unsigned)((pm ? q * r.L : q) + p.g * 8 * r.lstride);
    if (r.layout == SR_COEFF_PRE_SHUFFLE) {
        const int ss = r.s * r.s;
        const int64_t n = m / ss;
        const int sub = (int)(m - n * ss);
        const int64_t y = i / r.w;
        const int x = (int)(i - y * r.w);
        const int64_t at = (y * r.s + sub / r.s) * r.W + (int64_t)x * r.s + sub % r.s;
        p.at = (const char*)r.z + sizeof(TZ) * ((n * r.L * ss + sub) * a.ipx + i0);
        p.out = n * r.T * r.px + at;
        p.mask = n * r.px + at;
    } else {
        p.at = (const char*)r.z + sizeof(TZ) * (pm ? (m * a.ipx + i0) * r.L : m * r.L * a.ipx + i0);
        p.out = m * r.T * r.px + i;
        p.mask = m * r.px + i;
    }
    return p;
}

// Loads the lane's atoms, (c G + g) 8 and on in chunk c.  L and the stride are hidden from the compiler, which would otherwise
// keep the offsets of all planes and the comparisons of all chunks in registers from tile to tile (hundreds of spills).
template <typename TZ, int G>
__device__ __forceinline__ void load_chunks(Chunk<TZ> (&z)[LCH], const LaneArgs& a, const LanePixel& p, int L) {
    int64_t stride = a.r.lstride * (int64_t)sizeof(TZ);
    asm volatile("" : "+s"(stride));
    const char* at = p.at;
#pragma unroll
    for (int c = 0; c < LCH; ++c, at += stride * (8 * G)) {
        const int n = L - (c * G + p.g) * 8;
        if (c * G * 8 < L) {
            if (a.vec) {
                if (n > 0) z[c].load_vec(at, p.off);
            } else if ((c + 1) * G * 8 <= L) {
                z[c].template load<true>(at, p.off, stride, 8);
            } else {
                z[c].template load<false>(at, p.off, stride, n);
            }
        }
    }
}

// Sum over the lanes of a wavefront that hold the same chunk (g), in every lane.
template <int G, typename T> __device__ __forceinline__ T pixels_sum(T v, bool pm) {
    if (G == 1 || !pm) {
#pragma unroll
        for (int d = 64 / G / 2; d > 0; d >>= 1) v += __shfl_xor(v, d);
    } else {
#pragma unroll
        for (int d = 32; d >= G; d >>= 1) v += __shfl_xor(v, d);
    }
    return v;
}
template <int G> __device__ __forceinline__ float lanes_sum(float v, int step) {
#pragma unroll
    for (int d = 1; d < G; d <<= 1) v += __shfl_xor(v, d * step);
    return v;
}
template <int G> __device__ __forceinline__ float lanes_max(float v, int step) {
#pragma unroll
    for (int d = 1; d < G; d <<= 1) v = fmaxf(v, __shfl_xor(v, d * step));
    return v;
}

constexpr int LNT = 256, LWAVES = LNT / 64;

template <typename TZ, int TC, int G, bool STATS>
__global__ __launch_bounds__(LNT, STATS ? 2 : 4) void k_route_lanes(const LaneArgs a) {
    const RouteArgs& r = a.r;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool pm = r.layout == SR_COEFF_PIXEL_MAJOR;
    const int step = pm ? 1 : 64 / G;    // from one of a pixel's lanes to the next
    __shared__ unsigned bins[STATS ? LWAVES * SR_MAX_ATOMS : 1];
    float share[STATS ? LCH * 8 : 1];
    unsigned live = 0;
    double sq = 0.0;
    if (STATS) {
#pragma unroll
        for (int j = 0; j < LCH * 8; ++j) share[j] = 0.0f;
        for (int l = threadIdx.x; l < LWAVES * SR_MAX_ATOMS; l += LNT) bins[l] = 0;
        __syncthreads();
    }
    for (int64_t tile = (int64_t)blockIdx.x * LWAVES + wave; tile < a.tiles; tile += (int64_t)gridDim.x * LWAVES) {
        const LanePixel p = lane_pixel<TZ, G>(a, tile, lane);
        if (!p.inside) continue;
        if (r.mask && r.mask[p.mask] == 0) {
            for (int t = p.g; t < r.T; t += G) {
                r.index[p.out + t * r.px] = (unsigned char)t;
                if (a.half_value) st_from_float((__half*)r.value, p.out + t * r.px, 0.0f);
                else st_from_float((float*)r.value, p.out + t * r.px, 0.0f);
            }
            continue;
        }
        int L = r.L;
        int64_t px = r.px;
        asm volatile("" : "+s"(L), "+s"(px));
        Chunk<TZ> z[LCH];
        load_chunks<TZ, G>(z, a, p, L);
        TopList<TZ, TC> top;
        top.clear();
#pragma unroll
        for (int c = 0; c < LCH; ++c) {
            if ((c + 1) * G * 8 <= L) top.template insert<true>(z[c], 8 * c, 8);
            else if (c * G * 8 < L) top.template insert<false>(z[c], 8 * c, L - (c * G + p.g) * 8);
        }
        if (G > 1) {
#pragma unroll
            for (int t = 0; t < TC; ++t) {
                const int q = top.at(t);                     // chunk and place -> atom
                top.set_at(t, ((q >> 3) * G + p.g) * 8 + (q & 7));
            }
#pragma unroll
            for (int d = 1; d < G; d <<= 1) top.merge(d * step);
        }
        __builtin_amdgcn_sched_barrier(0);                   // nothing of the softmax before: its registers are the list's
        const float m = top.logit(0);
        const float o = exp_origin<TZ>(m);
        float whole = 0.0f, s = 0.0f;
        float e[STATS ? LCH * 8 : 1];
        if (STATS || r.kind == SR_ROUTE_SOFTMAX) {
#pragma unroll
            for (int c = 0; c < LCH; ++c) {
                const bool all = (c + 1) * G * 8 <= L;
                const int n = L - (c * G + p.g) * 8;
                if (c * G * 8 < L)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        float x = exp_from<TZ>(z[c].get(j), o);
                        if (!all && j >= n) x = 0.0f;
                        s += x;
                        if (STATS) e[STATS ? c * 8 + j : 0] = x;
                    }
            }
            s = lanes_sum<G>(s, step);
            whole = s;
        }
        float v[TC];
#pragma unroll
        for (int t = 0; t < TC; ++t) v[t] = r.kind == SR_ROUTE_VALUES ? top.logit(t) : exp_from<TZ>(top.logit(t), o);
        if (r.kind == SR_ROUTE_CHOSEN) {
            whole = 0.0f;
#pragma unroll
            for (int t = 0; t < TC; ++t) whole += t < r.T ? v[t] : 0.0f;
        }
        const float inv = r.kind == SR_ROUTE_VALUES ? 1.0f : (whole > 0.0f || whole != whole ? 1.0f / whole : 0.0f);
#pragma unroll
        for (int t = 0; t < TC; ++t)
            if (t < r.T && (G == 1 || t % G == p.g)) {
                const int64_t at = p.out + t * px;
                r.index[at] = (unsigned char)top.at(t);
                if (a.half_value) st_from_float((__half*)r.value, at, v[t] * inv);
                else st_from_float((float*)r.value, at, v[t] * inv);
                if (STATS && top.logit(t) != -INFINITY) atomicAdd(&bins[wave * SR_MAX_ATOMS + top.at(t)], 1u);
            }
        if (STATS && m != -INFINITY) {
            const float is = 1.0f / s, lse = m + logit_log(s);
#pragma unroll
            for (int c = 0; c < LCH; ++c)
                if (c * G * 8 < L)
#pragma unroll
                    for (int j = 0; j < 8; ++j) share[STATS ? c * 8 + j : 0] = fmaf(e[STATS ? c * 8 + j : 0], is, share[STATS ? c * 8 + j : 0]);
            if (p.g == 0) {
                sq = fma((double)lse, (double)lse, sq);
                ++live;
            }
        }
    }
    if (!STATS) return;
    // over the wavefront's lanes in fp32, over the wavefronts in double, one after the other
    __shared__ double sum[STATS ? SR_MAX_ATOMS + 32 : 1], sh_sq;
    __shared__ unsigned sh_live;
    const int g = G == 1 ? 0 : (pm ? lane % G : lane / (64 / G));
    const bool first = pm ? lane < G : lane % (64 / G) == 0;
    sq = pixels_sum<1>(sq, pm);
    live = pixels_sum<1>(live, pm);
#pragma unroll
    for (int c = 0; c < LCH; ++c)
        if (c * G * 8 < r.L)
#pragma unroll
            for (int j = 0; j < 8; ++j) share[STATS ? c * 8 + j : 0] = pixels_sum<G>(share[STATS ? c * 8 + j : 0], pm);
    for (int w = 0; w < LWAVES; ++w) {
        if (wave == w) {
            if (first)
#pragma unroll
                for (int c = 0; c < LCH; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int l = (c * G + g) * 8 + j;
                        if (l < r.L) sum[l] = (w ? sum[l] : 0.0) + share[STATS ? c * 8 + j : 0];
                    }
            if (lane == 0) {
                sh_sq = (w ? sh_sq : 0.0) + sq;
                sh_live = (w ? sh_live : 0u) + live;
            }
        }
        __syncthreads();
    }
    const RouteRecord rec(r.partial, r.L, blockIdx.x);
    for (int l = threadIdx.x; l < r.L; l += LNT) {
        rec.share[l] = sum[l];
        unsigned n = 0;
        for (int w = 0; w < LWAVES; ++w) n += bins[w * SR_MAX_ATOMS + l];
        rec.counts[l] = n;
    }
    if (threadIdx.x == 0) *rec.squares = sh_sq, *rec.live = sh_live;
}

// The gradient.  A pixel's entries are scattered into a row of LDS per lane ([atom], 16-byte pieces without bank conflicts:
// the pitch of 76 words puts 16 lanes' pieces on 64 banks) and read back beside its logits.
constexpr int DNT = 128, DWAVES = DNT / 64, DPITCH = LCH * 8 + 4;
constexpr unsigned NOT_LISTED = 0x7fc5a5a5u;                 // a NaN that no computation gives

template <typename TZ, int G, int KIND, bool LOSS>
__global__ __launch_bounds__(DNT, 2) void k_route_grad_lanes(const LaneArgs a) {
    const RouteArgs& r = a.r;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int step = r.layout == SR_COEFF_PIXEL_MAJOR ? 1 : 64 / G;
    __shared__ float4 gl[DWAVES][64][DPITCH / 4];
    __shared__ float4 fl[LOSS ? (LCH * 8 * G) / 4 : 1];
    const float none = KIND == SR_ROUTE_CHOSEN ? __uint_as_float(NOT_LISTED) : 0.0f;
    float* own = (float*)gl[wave][lane];
#pragma unroll
    for (int q = 0; q < LCH * 2; ++q) gl[wave][lane][q] = make_float4(none, none, none, none);
    float w0 = 0.0f, w1 = 0.0f;
    if (LOSS) {
        const double M = (double)r.counts[r.L], inv = M > 0.0 ? 1.0 / M : 0.0;
        w0 = (float)(r.dloss[0] * (double)r.L * inv);
        w1 = (float)(r.dloss[1] * 2.0 * inv);
        for (int l = threadIdx.x; l < LCH * 8 * G; l += DNT) ((float*)fl)[l] = l < r.L ? (float)((double)r.counts[l] * inv / r.T) : 0.0f;
        __syncthreads();
    }
    for (int64_t tile = (int64_t)blockIdx.x * DWAVES + wave; tile < a.tiles; tile += (int64_t)gridDim.x * DWAVES) {
        const LanePixel p = lane_pixel<TZ, G>(a, tile, lane);
        if (!p.inside) continue;
        const bool on = !r.mask || r.mask[p.mask] != 0;
        int L = r.L;
        int64_t px = r.px, stride = r.lstride * (int64_t)sizeof(TZ);
        asm volatile("" : "+s"(L), "+s"(px), "+s"(stride));
        float e[LCH * 8], m = -INFINITY, s = 0.0f, scale = 0.0f, tilt = 0.0f, pull = 0.0f;
        if (on && KIND != SR_ROUTE_VALUES) {
            Chunk<TZ> z[LCH];
            load_chunks<TZ, G>(z, a, p, L);
#pragma unroll
            for (int c = 0; c < LCH; ++c)
                if (c * G * 8 < L)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        float x = z[c].get(j);
                        if ((c + 1) * G * 8 > L && j >= L - (c * G + p.g) * 8) x = -INFINITY;
                        e[c * 8 + j] = x;
                        m = fmaxf(m, x);
                    }
        }
        // every lane of the pixel takes the entries of its own atoms
        if (on && r.value)
            for (int t = 0; t < r.T; ++t) {
                const int l = r.index[p.out + t * px];
                const float v = a.half_value ? ld_as_float((const __half*)r.value, p.out + t * px) : ld_as_float((const float*)r.value, p.out + t * px);
                const int c = (l >> 3) / G;
                if (l < L && (G == 1 || (l >> 3) % G == p.g)) own[c * 8 + (l & 7)] = v;
            }
        float mine = 0.0f, sum_q = 0.0f, qg = 0.0f, fp = 0.0f;
        if (on && KIND != SR_ROUTE_VALUES) {
            m = lanes_max<G>(m, step);
            const float o = exp_origin<TZ>(m);
#pragma unroll
            for (int c = 0; c < LCH; ++c)
                if (c * G * 8 < L)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float4 G4 = gl[wave][lane][c * 2 + h];
                        float4 f4 = make_float4(0, 0, 0, 0);
                        if (LOSS) f4 = fl[(c * G + p.g) * 2 + h];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float x = exp_from<TZ>(e[c * 8 + 4 * h + j], o), gv = ((const float*)&G4)[j];
                            e[c * 8 + 4 * h + j] = x;
                            s += x;
                            if (KIND == SR_ROUTE_CHOSEN) {
                                const bool is = __float_as_uint(gv) != NOT_LISTED;
                                sum_q += is ? x : 0.0f;
                                qg = is ? fmaf(x, gv, qg) : qg;
                            } else {
                                qg = fmaf(x, gv, qg);
                            }
                            if (LOSS) fp = fmaf(x, ((const float*)&f4)[j], fp);
                        }
                    }
            s = lanes_sum<G>(s, step);
            qg = lanes_sum<G>(qg, step);
            if (LOSS) fp = lanes_sum<G>(fp, step);
            if (KIND == SR_ROUTE_CHOSEN) sum_q = lanes_sum<G>(sum_q, step);
            const bool live = m != -INFINITY;
            const float is = live ? 1.0f / s : 0.0f;
            scale = KIND == SR_ROUTE_CHOSEN ? (live && sum_q > 0.0f ? 1.0f / sum_q : 0.0f) : is;
            pull = qg * scale;
            if (LOSS) {
                const float lse = live ? m + logit_log(s) : 0.0f;
                mine = is;
                tilt = fmaf(w1, lse, -w0 * (fp * is));
            }
        }
        char* to = (char*)r.dz + (p.at - (const char*)r.z);
#pragma unroll
        for (int c = 0; c < LCH; ++c, to += stride * (8 * G))
            if (c * G * 8 < L) {
                const int n = L - (c * G + p.g) * 8;
                float d[8];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float4 G4 = gl[wave][lane][c * 2 + h];
                    float4 f4 = make_float4(0, 0, 0, 0);
                    if (LOSS) f4 = fl[(c * G + p.g) * 2 + h];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float x = e[c * 8 + 4 * h + j], gv = ((const float*)&G4)[j];
                        float y;
                        if (KIND == SR_ROUTE_VALUES) {
                            y = gv;
                        } else {
                            y = x * scale * (gv - pull);
                            if (KIND == SR_ROUTE_CHOSEN) y = __float_as_uint(gv) != NOT_LISTED ? y : 0.0f;
                            if (LOSS) y = fmaf(x * mine, fmaf(w0, ((const float*)&f4)[j], tilt), y);
                        }
                        d[4 * h + j] = on ? y : 0.0f;
                    }
                }
                if (a.vec) {
                    if (n > 0) {
                        TZ st[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) st_from_float(st, j, d[j]);
#pragma unroll
                        for (int q = 0; q < (int)sizeof(TZ) / 2; ++q) {
                            uint4 u;
                            __builtin_memcpy(&u, (const char*)st + 16 * q, 16);
                            *(uint4*)(to + p.off + 16 * q) = u;
                        }
                    }
                } else if ((c + 1) * G * 8 <= L) {
                    char* q = to;
#pragma unroll
                    for (int j = 0; j < 8; ++j, q += stride) st_from_float((TZ*)(q + p.off), 0, d[j]);
                } else {
                    char* q = to;
#pragma unroll
                    for (int j = 0; j < 8; ++j, q += stride)
                        if (j < n) st_from_float((TZ*)(q + p.off), 0, d[j]);
                }
            }
        if (on && r.value)
            for (int t = 0; t < r.T; ++t) {
                const int l = r.index[p.out + t * px], c = (l >> 3) / G;
                if (l < L && (G == 1 || (l >> 3) % G == p.g)) own[c * 8 + (l & 7)] = none;
            }
    }
}

// Host side.  One instantiation file per type of logits.
template <typename TZ> hipError_t route_lanes(const LaneArgs& a, int G, bool stats, int grid, hipStream_t st);
template <typename TZ> hipError_t route_grad_lanes(const LaneArgs& a, int G, int grid, hipStream_t st);

#define SR_ROUTE_LANES(TZ)                                                                                                         \
    template <int TC, int G> static hipError_t route_tc(const LaneArgs& a, bool stats, int grid, hipStream_t st) {                 \
        if (stats) k_route_lanes<TZ, TC, G, true><<<grid, LNT, 0, st>>>(a);                                                        \
        else k_route_lanes<TZ, TC, G, false><<<grid, LNT, 0, st>>>(a);                                                             \
        return hipGetLastError();                                                                                                  \
    }                                                                                                                              \
    template <int G> static hipError_t route_g(const LaneArgs& a, bool stats, int grid, hipStream_t st) {                          \
        return a.r.T <= 4 ? route_tc<4, G>(a, stats, grid, st) : a.r.T <= 8 ? route_tc<8, G>(a, stats, grid, st) : route_tc<16, G>(a, stats, grid, st); \
    }                                                                                                                              \
    template <> hipError_t route_lanes<TZ>(const LaneArgs& a, int G, bool stats, int grid, hipStream_t st) {                       \
        return G == 1 ? route_g<1>(a, stats, grid, st) : G == 2 ? route_g<2>(a, stats, grid, st) : route_g<4>(a, stats, grid, st); \
    }                                                                                                                              \
    template <int G, int KIND> static hipError_t grad_k(const LaneArgs& a, int grid, hipStream_t st) {                             \
        if (a.r.counts) k_route_grad_lanes<TZ, G, KIND, KIND != SR_ROUTE_VALUES><<<grid, DNT, 0, st>>>(a);                         \
        else k_route_grad_lanes<TZ, G, KIND, false><<<grid, DNT, 0, st>>>(a);                                                      \
        return hipGetLastError();                                                                                                  \
    }                                                                                                                              \
    template <int G> static hipError_t grad_g(const LaneArgs& a, int grid, hipStream_t st) {                                       \
        return a.r.kind == SR_ROUTE_SOFTMAX ? grad_k<G, SR_ROUTE_SOFTMAX>(a, grid, st)                                             \
             : a.r.kind == SR_ROUTE_CHOSEN ? grad_k<G, SR_ROUTE_CHOSEN>(a, grid, st) : grad_k<G, SR_ROUTE_VALUES>(a, grid, st);    \
    }                                                                                                                              \
    template <> hipError_t route_grad_lanes<TZ>(const LaneArgs& a, int G, int grid, hipStream_t st) {                              \
        return G == 1 ? grad_g<1>(a, grid, st) : G == 2 ? grad_g<2>(a, grid, st) : grad_g<4>(a, grid, st);                         \
    }

}  // namespace srd

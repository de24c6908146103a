// The router's kernels for many pixels: one to four lanes (G) hold a pixel's logits in registers, eight atoms at a time.
//
// Selection: a sorted list of TC keys per lane; a new key x moves into it with one median each, a_i' = med3(a_{i-1}, x, a_i).
// A key of a 16-bit logit is one 32-bit integer, the logit's order above and the atom (lower ones first) below; fp32 logits
// keep the atom beside the key (med3, a compare and two selects for each place).  The lists of a pixel's G lanes are merged as
// bitonic sequences.  The softmax runs over the same registers once the largest logit is known: one pass over memory.
#pragma once
#include <type_traits>

#include "sr_route.h"

namespace srd {

// A pointer that is the same for the whole wavefront, kept in scalar registers from here on: what is added to it per lane stays apart, as the
// 32-bit offset of a load or store.
#define SR_GLOBAL __attribute__((address_space(1)))
typedef char SR_GLOBAL* gptr;
__device__ __forceinline__ gptr scalar(gptr p) {
    asm("" : "+s"(p));
    return p;
}
template <typename T> __device__ __forceinline__ T gload(gptr at, unsigned off) { return *(const T SR_GLOBAL*)(at + off); }
template <typename T> __device__ __forceinline__ void gstore(gptr at, unsigned off, T v) { *(T SR_GLOBAL*)(at + off) = v; }

// ... and that offset, made 64 bits wide only where it is used (widened once for a whole tile it takes an addition per access)
__device__ __forceinline__ unsigned lane_offset(unsigned off) {
    asm("" : "+v"(off));
    return off;
}

constexpr int LCH = 9;                   // most chunks of 8 atoms that a lane holds: 72 atoms, times G

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

// A result as it is stored
template <typename TZ> struct Stored { typedef unsigned short type; };
template <> struct Stored<float> { typedef float type; };
template <typename TZ> __device__ __forceinline__ typename Stored<TZ>::type as_stored(float v) {
    TZ t;
    typename Stored<TZ>::type u;
    st_from_float(&t, 0, v);
    __builtin_memcpy(&u, &t, sizeof(t));
    return u;
}

typedef short short2v __attribute__((ext_vector_type(2)));
typedef unsigned vec4u __attribute__((ext_vector_type(4)));
typedef float vec4f __attribute__((ext_vector_type(4)));

// Eight logits as they are stored: those of a contiguous row (VEC) 16 bytes at a time, 16-bit ones two in a word; else one in a
// register, where its load puts it: nothing is done to a load's result before all of a tile's loads are under way.
template <typename TZ, bool VEC> struct Chunk {              // __half, bf16raw
    unsigned w[VEC ? 4 : 8];
    __device__ __forceinline__ void load(int j, gptr at, unsigned off) { w[VEC ? 0 : j] = gload<unsigned short>(at, off); }
    __device__ __forceinline__ void load_row(gptr at, unsigned off) {
        const vec4u v = gload<vec4u>(at, off);
        w[0] = v[0], w[1] = v[1], w[2] = v[2], w[3] = v[3];
    }
    __device__ __forceinline__ unsigned pair(int i) const { return VEC ? w[i] : w[VEC ? 0 : 2 * i] | (w[VEC ? 0 : 2 * i + 1] << 16); }
    __device__ __forceinline__ unsigned bits(int j) const { return VEC ? (j & 1 ? w[j / 2] >> 16 : w[j / 2] & 0xffffu) : w[VEC ? 0 : j]; }
    static __device__ __forceinline__ float widen(unsigned b, const __half*) { return __half2float(__ushort_as_half((unsigned short)b)); }
    static __device__ __forceinline__ float widen(unsigned b, const bf16raw*) { return __uint_as_float(b << 16); }
    __device__ __forceinline__ float get(int j) const { return widen(bits(j), (const TZ*)nullptr); }
    // signed order of the two logits of a pair: negative ones mirrored, so that -0 is +0
    __device__ __forceinline__ unsigned order2(int i) const {
        const unsigned p = pair(i);
        short2v b, t, s;
        __builtin_memcpy(&b, &p, 4);
        s = b >> 15;
        t = (short)-32768 - b;
        const short2v o = (t & s) | (b & ~s);
        unsigned u;
        __builtin_memcpy(&u, &o, 4);
        return u;
    }
};
template <bool VEC> struct Chunk<float, VEC> {
    float w[8];
    __device__ __forceinline__ void load(int j, gptr at, unsigned off) { w[j] = gload<float>(at, off); }
    __device__ __forceinline__ void load_row(gptr at, unsigned off) {
        const vec4f a = gload<vec4f>(at, off), b = gload<vec4f>(at, off + 16);
        w[0] = a[0], w[1] = a[1], w[2] = a[2], w[3] = a[3], w[4] = b[0], w[5] = b[1], w[6] = b[2], w[7] = b[3];
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
    template <bool ALL, bool VEC> __device__ __forceinline__ void insert(const Chunk<TZ, VEC>& c, int at, int n) {   // the first n are atoms
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
        return Chunk<TZ, false>::widen((unsigned)b & 0xffffu, (const TZ*)nullptr);
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
#pragma unroll
        for (int i = 0; i < TC; ++i) asm("" : "+v"(id[i]));  // (one key's selects are not to be mixed with the next one's)
    }
    template <bool ALL, bool VEC> __device__ __forceinline__ void insert(const Chunk<float, VEC>& c, int at, int n) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const unsigned o = logit_order(c.w[j]);
            __builtin_amdgcn_sched_barrier(0);               // one key at a time: each takes as many masks as there are places
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

// Loads the lane's NC chunks: atoms (c G + g) 8 and on in chunk c.  FULL: all of them are there (L = 8 G NC); else places beyond the last atom
// get some atom's logit, never an address beyond it, and are set aside when they are used.  There is no branch: all loads of a tile are under way
// before the first is waited for.  The stride is hidden from the compiler, which would keep the offsets of all planes from tile to tile.
template <typename TZ, int G, bool VEC, int NC, bool FULL>
__device__ __forceinline__ void load_chunks(Chunk<TZ, VEC> (&z)[NC], const LaneArgs& a, const LanePixel& p, int L) {
    int64_t stride = a.r.lstride * (int64_t)sizeof(TZ);
    asm volatile("" : "+s"(stride));
    gptr at = scalar((gptr)p.at);
    if (VEC) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int l = (c * G + p.g) * 8;
            z[c].load_row(at, p.off + (unsigned)sizeof(TZ) * (unsigned)((FULL || l < L ? l : 0) - p.g * 8));
        }
    } else if (G == 1) {
        const unsigned off = lane_offset(p.off);
#pragma unroll
        for (int l = 0; l < 8 * NC; ++l) {
            z[l / 8].load(l % 8, at, off);
            at = scalar(at + (FULL || l + 1 < L ? stride : 0));
        }
    } else {
        const int last = (L - 1) / (8 * G);          // the last chunk that any lane has atoms in
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            // the lane's plane of the chunk, or the last atom's; from there on as long as there are atoms.  Offsets have 32 bits and no
            // sign: they start at a plane that is there, at or after the chunk's first (which `at` points to), and only grow.  Taken back from beyond
            // the last atom to before that plane, one would stand for 4 GB more: a memory fault.
            const int l = (min(c, last) * G + p.g) * 8;
            unsigned off = p.off - (unsigned)max(l - (L - 1), 0) * (unsigned)stride;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                z[c].load(j, at, lane_offset(off));
                off += FULL || l + j + 1 < L ? (unsigned)stride : 0u;
            }
            at = scalar(at + (FULL || c < last ? stride * (8 * G) : 0));
        }
    }
}

// Sum over the lanes of a wavefront that hold the same atoms, without LDS: turns within rows of 16 lanes, then rows exchanged.
template <int CTRL> __device__ __forceinline__ float row_turned(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
template <int G> __device__ __forceinline__ float pixels_sum(float v, bool pm) {
    if (G == 1 || !pm) v += row_turned<0x121>(v), v += row_turned<0x122>(v);     // row_ror 1, 2
    v += row_turned<0x124>(v);
    v += row_turned<0x128>(v);
    if (G == 1 || pm) {
        const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
        const auto c = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(c[0]) + __uint_as_float(c[1]);
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

// What bounds it: with 72 fp16 logits a 4K frame moves 1.39 GB, 284 us at a large copy's 4.9 TB/s, and takes 1323 vector instructions a
// wavefront of 64 pixels (8 medians a logit; 279 us if nothing else ran): 314 to 330 us.  A median per place of the list is what one lane can do a key in;
// lists kept apart by wavefront (k_route_wave) take a reduction over 64 lanes per entry.
// The losses keep every atom's share in a register as well, 2 wavefronts per SIMD instead of 4: 2.1 Mpixel of bfloat16 logits 102 us and 8 for the
// last sum, of 66 us that its bytes take.
// Workgroups: with the losses one a CU, so that few records are left to be added up (512 of them took 13 us).
constexpr int lanes_threads(bool stats) { return stats ? 512 : 256; }

template <typename TZ, int TC, int G, bool VEC, int NC, bool FULL, bool STATS>
__global__ __launch_bounds__(lanes_threads(STATS), STATS ? 2 : 4) void k_route_lanes(const LaneArgs a) {
    constexpr int LNT = lanes_threads(STATS), LWAVES = LNT / 64;
    const RouteArgs& r = a.r;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool pm = r.layout == SR_COEFF_PIXEL_MAJOR;
    const int step = pm ? 1 : 64 / G;    // from one of a pixel's lanes to the next
    __shared__ unsigned bins[STATS ? LWAVES * SR_MAX_ATOMS : 1];
    __shared__ double part[STATS ? LWAVES : 1][STATS ? G * NC * 8 : 1];
    __shared__ float part_run[STATS ? LWAVES : 1][STATS ? G * NC * 8 : 1];
    const int g = G == 1 ? 0 : (pm ? lane % G : lane / (64 / G));
    float share[STATS ? NC * 8 : 1];
    unsigned live = 0;
    int run = 0;
    double sq = 0.0;
    if (STATS) {
#pragma unroll
        for (int j = 0; j < NC * 8; ++j) share[j] = 0.0f;
        for (int l = threadIdx.x; l < LWAVES * SR_MAX_ATOMS; l += LNT) bins[l] = 0;
        for (int l = lane; l < G * NC * 8; l += 64) part[wave][l] = 0.0;
        __syncthreads();
    }
    // the lanes' shares are added up in fp32, each the sum of RUN tiles at most, and to what the wavefront has in double
    constexpr int RUN = 64;
    auto keep_shares = [&] {
        const bool first = pm ? lane < G : lane % (64 / G) == 0;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float v = pixels_sum<G>(share[STATS ? c * 8 + j : 0], pm);
                if (first) part_run[STATS ? wave : 0][STATS ? (c * G + g) * 8 + j : 0] = v;
                share[STATS ? c * 8 + j : 0] = 0.0f;
            }
        asm volatile("" ::: "memory");                       // (a wavefront's LDS accesses keep their order)
        for (int l = lane; l < G * NC * 8; l += 64) part[STATS ? wave : 0][STATS ? l : 0] += (double)part_run[STATS ? wave : 0][STATS ? l : 0];
        asm volatile("" ::: "memory");
    };
    for (int64_t tile = (int64_t)blockIdx.x * LWAVES + wave; tile < a.tiles; tile += (int64_t)gridDim.x * LWAVES) {
        if (STATS && ++run > RUN) {
            keep_shares();
            run = 1;
        }
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
        Chunk<TZ, VEC> z[NC];
        load_chunks<TZ, G, VEC, NC, FULL>(z, a, p, L);
        TopList<TZ, TC> top;
        top.clear();
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            __builtin_amdgcn_sched_barrier(0);
            top.template insert<FULL, VEC>(z[c], 8 * c, L - (c * G + p.g) * 8);
        }
        asm volatile("" : "+s"(L));          // (its comparisons are made again below: 72 masks are too many to keep)
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
        float e[STATS ? NC * 8 : 1];
        if (STATS || r.kind == SR_ROUTE_SOFTMAX) {
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float x = exp_from<TZ>(z[c].get(j), o);
                    if (!FULL) x = j < L - (c * G + p.g) * 8 ? x : 0.0f;
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
            for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) share[STATS ? c * 8 + j : 0] = fmaf(e[STATS ? c * 8 + j : 0], is, share[STATS ? c * 8 + j : 0]);
            if (p.g == 0) {
                sq = fma((double)lse, (double)lse, sq);
                ++live;
            }
        }
    }
    if (!STATS) return;
    keep_shares();
    __shared__ double part_sq[LWAVES];
    __shared__ unsigned part_live[LWAVES];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sq += __shfl_xor(sq, d), live += __shfl_xor(live, d);
    if (lane == 0) part_sq[wave] = sq, part_live[wave] = live;
    __syncthreads();
    const RouteRecord rec(r.partial, r.L, blockIdx.x);
    for (int l = threadIdx.x; l < r.L; l += LNT) {
        double v = 0.0;
        unsigned n = 0;
        for (int w = 0; w < LWAVES; ++w) v += part[STATS ? w : 0][STATS ? l : 0], n += bins[w * SR_MAX_ATOMS + l];
        rec.share[l] = v;
        rec.counts[l] = n;
    }
    if (threadIdx.x == 0) {
        double v = 0.0;
        unsigned long long n = 0;
        for (int w = 0; w < LWAVES; ++w) v += part_sq[w], n += part_live[w];
        *rec.squares = v;
        *rec.live = n;
    }
}

// The gradient.  Which entry names an atom is a byte per atom in LDS, a row for every lane (all zero between tiles; the pitch of 19
// words is free of bank conflicts); the entries' gradients are a table beside it, entry 0 the zero of atoms that are not listed.
// 7 KB a wavefront and 110 registers: four wavefronts per SIMD hide the latency of a tile's loads (with the gradients themselves
// scattered, 20 KB, it was two, and 1247 us instead of 557 for a 4K frame of 72 fp16 logits: 2.59 GB, 528 us at a large copy's 4.9 TB/s).
constexpr int DNT = 256, DWAVES = DNT / 64;

template <typename TZ, int G, bool VEC, int NC, bool FULL, int TT, int KIND, bool LOSS>
__global__ __launch_bounds__(DNT, 4) void k_route_grad_lanes(const LaneArgs a) {
    const RouteArgs& r = a.r;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int step = r.layout == SR_COEFF_PIXEL_MAJOR ? 1 : 64 / G;
    __shared__ unsigned map[DWAVES][64 * (NC * 8 + 4) / 4];
    __shared__ float table[DWAVES][(TT + 1) * 64];
    __shared__ float4 fl[LOSS ? (NC * 8 * G) / 4 : 1];
    unsigned* const row = map[wave] + lane * ((NC * 8 + 4) / 4);
    float* const tab = table[wave];
#pragma unroll
    for (int q = 0; q < NC * 2; ++q) row[q] = 0;
    tab[lane] = 0.0f;
    float w0 = 0.0f, w1 = 0.0f;
    if (LOSS) {
        const double M = (double)r.counts[r.L], inv = M > 0.0 ? 1.0 / M : 0.0;
        w0 = (float)(r.dloss[0] * (double)r.L * inv);
        w1 = (float)(r.dloss[1] * 2.0 * inv);
        for (int l = threadIdx.x; l < NC * 8 * G; l += DNT) ((float*)fl)[l] = l < r.L ? (float)((double)r.counts[l] * inv / r.T) : 0.0f;
        __syncthreads();
    }
    // the table's address of the entry that names place j (0 .. 3) of a word of the row
    const unsigned lane4 = 4u * (unsigned)lane;
    auto entry = [&](unsigned word, int j) -> unsigned { return __builtin_amdgcn_perm(word, lane4, 0x0c0c0000u | (unsigned)(4 + j) << 8); };
    for (int64_t tile = (int64_t)blockIdx.x * DWAVES + wave; tile < a.tiles; tile += (int64_t)gridDim.x * DWAVES) {
        const LanePixel p = lane_pixel<TZ, G>(a, tile, lane);
        if (!p.inside) continue;
        int L = r.L;
        int64_t px = r.px, stride = r.lstride * (int64_t)sizeof(TZ);
        asm volatile("" : "+s"(L), "+s"(px), "+s"(stride));
        gptr to = scalar((gptr)r.dz + (p.at - (const char*)r.z));
        // writes a chunk of the lane: n atoms of it are there
        auto write = [&](gptr q, int n, const float (&d)[8]) {
            const unsigned off = lane_offset(p.off);
            if (VEC) {
                if (FULL || n > 0) {
                    TZ st[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) st_from_float(st, j, d[j]);
#pragma unroll
                    for (int k = 0; k < (int)sizeof(TZ) / 2; ++k) {
                        vec4u u;
                        __builtin_memcpy(&u, (const char*)st + 16 * k, 16);
                        gstore(q, off + 16 * k, u);
                    }
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j, q = scalar(q + stride))
                    if (FULL || j < n) gstore(q, off, as_stored<TZ>(d[j]));
            }
        };
        if (r.mask && r.mask[p.mask] == 0) {
            const float zero[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
            for (int c = 0; c * G * 8 < L; ++c, to = scalar(to + stride * (8 * G))) write(to, L - (c * G + p.g) * 8, zero);
            continue;
        }
        int at[TT];                          // the place in the lane's row of an entry, or -1
        if (r.value) {
#pragma unroll
            for (int t = 0; t < TT; ++t)
                if (t < r.T) {
                    const int l = r.index[p.out + t * px];
                    tab[64 * (t + 1) + lane] = a.half_value ? ld_as_float((const __half*)r.value, p.out + t * px) : ld_as_float((const float*)r.value, p.out + t * px);
                    const int c = (l >> 3) / G;
                    at[t] = l < L && (G == 1 || (l >> 3) % G == p.g) ? c * 8 + (l & 7) : -1;
                    if (at[t] >= 0) ((unsigned char*)row)[at[t]] = (unsigned char)(t + 1);
                }
        }
        float e[NC * 8], scale = 0.0f, tilt = 0.0f, pull = 0.0f, mine = 0.0f;
        if (KIND != SR_ROUTE_VALUES) {
            float m = -INFINITY;
            {
                Chunk<TZ, VEC> z[NC];
                load_chunks<TZ, G, VEC, NC, FULL>(z, a, p, L);
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        float x = z[c].get(j);
                        if (!FULL) x = j < L - (c * G + p.g) * 8 ? x : -INFINITY;
                        e[c * 8 + j] = x;
                        m = fmaxf(m, x);
                    }
            }
            m = lanes_max<G>(m, step);
            const float o = exp_origin<TZ>(m);
            float s = 0.0f, sum_q = 0.0f, qg = 0.0f, fp = 0.0f;
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        __builtin_amdgcn_sched_barrier(0);
                        const unsigned word = row[c * 2 + h];
                        float4 f4 = make_float4(0, 0, 0, 0);
                        if (LOSS) f4 = fl[(c * G + p.g) * 2 + h];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const unsigned en = entry(word, j);
                            const float x = exp_from<TZ>(e[c * 8 + 4 * h + j], o), gv = *(const float*)((const char*)tab + en);
                            e[c * 8 + 4 * h + j] = x;
                            s += x;
                            if (KIND == SR_ROUTE_CHOSEN) {
                                sum_q += en >= 256u ? x : 0.0f;
                                qg = en >= 256u ? fmaf(x, gv, qg) : qg;
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
        int again = 0;                       // (hidden: the rows are read again; kept, what they said would take another 144 registers)
        asm volatile("" : "+v"(again));
#pragma unroll
        for (int c = 0; c < NC; ++c, to = scalar(to + stride * (8 * G)))
            if (FULL || c * G * 8 < L) {
                __builtin_amdgcn_sched_barrier(0);
                float d[8];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const unsigned word = row[c * 2 + h + again];
                    float4 f4 = make_float4(0, 0, 0, 0);
                    if (LOSS) f4 = fl[(c * G + p.g) * 2 + h + again];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const unsigned en = entry(word, j);
                        const float gv = *(const float*)((const char*)(tab + again) + en);
                        float y = gv;
                        if (KIND != SR_ROUTE_VALUES) {
                            const float x = e[c * 8 + 4 * h + j];
                            y = x * scale * (gv - pull);
                            if (KIND == SR_ROUTE_CHOSEN) y = en >= 256u ? y : 0.0f;
                            if (LOSS) y = fmaf(x * mine, fmaf(w0, ((const float*)&f4)[j], tilt), y);
                        }
                        d[4 * h + j] = y;
                    }
                }
                write(to, L - (c * G + p.g) * 8, d);
            }
        if (r.value) {
#pragma unroll
            for (int t = 0; t < TT; ++t)
                if (t < r.T && at[t] >= 0) ((unsigned char*)row)[at[t]] = 0;
        }
    }
}

// Host side.  One instantiation file per type of logits.
template <typename TZ> hipError_t route_lanes(const LaneArgs& a, int G, bool stats, int grid, hipStream_t st);
template <typename TZ> hipError_t route_grad_lanes(const LaneArgs& a, int G, int grid, hipStream_t st);

// Which instantiation: lanes of a pixel, rows of logits or planes, chunks of a lane.  Places without an atom cost a load and an insert as well:
// 8 Mpixel of 27 fp32 logits take 235 us in 6 chunks and 324 in 9, 70 000 pixels of 121 in four lanes' 4 chunks 12.6 us and 22.9 in 9.
#define SR_ROUTE_FORMS(F)                                                                                                          \
    if (a.vec) return a.r.L <= 64 ? F(4, true, 2, false) : a.r.L <= 128 ? F(4, true, 4, false) : F(4, true, LCH, false);            \
    if (G > 1) return a.r.L <= 128 ? F(4, false, 4, false) : F(4, false, LCH, false);                                               \
    return a.r.L == 8 * LCH ? F(1, false, LCH, true) : a.r.L <= 24 ? F(1, false, 3, false)                                          \
         : a.r.L <= 48 ? F(1, false, 6, false) : F(1, false, LCH, false);

#define SR_ROUTE_LANES(TZ)                                                                                                         \
    template <int G, bool VEC, int NC, bool FULL> static hipError_t route_one(const LaneArgs& a, bool stats, int grid, hipStream_t st) { \
        if (a.r.T <= 4) {                                                                                                          \
            if (stats) k_route_lanes<TZ, 4, G, VEC, NC, FULL, true><<<grid, lanes_threads(true), 0, st>>>(a);                   \
            else k_route_lanes<TZ, 4, G, VEC, NC, FULL, false><<<grid, lanes_threads(false), 0, st>>>(a);                       \
        } else if (a.r.T <= 8) {                                                                                                   \
            if (stats) k_route_lanes<TZ, 8, G, VEC, NC, FULL, true><<<grid, lanes_threads(true), 0, st>>>(a);                   \
            else k_route_lanes<TZ, 8, G, VEC, NC, FULL, false><<<grid, lanes_threads(false), 0, st>>>(a);                       \
        } else {                                                                                                                   \
            if (stats) k_route_lanes<TZ, 16, G, VEC, NC, FULL, true><<<grid, lanes_threads(true), 0, st>>>(a);                  \
            else k_route_lanes<TZ, 16, G, VEC, NC, FULL, false><<<grid, lanes_threads(false), 0, st>>>(a);                      \
        }                                                                                                                          \
        return hipGetLastError();                                                                                                  \
    }                                                                                                                              \
    template <int G, bool VEC, int NC, bool FULL, int KIND> static hipError_t grad_kind(const LaneArgs& a, int grid, hipStream_t st) { \
        constexpr bool loss = KIND != SR_ROUTE_VALUES;                                                                             \
        if (a.r.T <= 8) {                                                                                                          \
            if (a.r.counts) k_route_grad_lanes<TZ, G, VEC, NC, FULL, 8, KIND, loss><<<grid, DNT, 0, st>>>(a);                      \
            else k_route_grad_lanes<TZ, G, VEC, NC, FULL, 8, KIND, false><<<grid, DNT, 0, st>>>(a);                                \
        } else {                                                                                                                   \
            if (a.r.counts) k_route_grad_lanes<TZ, G, VEC, NC, FULL, 16, KIND, loss><<<grid, DNT, 0, st>>>(a);                     \
            else k_route_grad_lanes<TZ, G, VEC, NC, FULL, 16, KIND, false><<<grid, DNT, 0, st>>>(a);                               \
        }                                                                                                                          \
        return hipGetLastError();                                                                                                  \
    }                                                                                                                              \
    template <int G, bool VEC, int NC, bool FULL> static hipError_t grad_one(const LaneArgs& a, int grid, hipStream_t st) {        \
        return a.r.kind == SR_ROUTE_SOFTMAX ? grad_kind<G, VEC, NC, FULL, SR_ROUTE_SOFTMAX>(a, grid, st)                           \
             : a.r.kind == SR_ROUTE_CHOSEN ? grad_kind<G, VEC, NC, FULL, SR_ROUTE_CHOSEN>(a, grid, st)                             \
                                           : grad_kind<G, VEC, NC, FULL, SR_ROUTE_VALUES>(a, grid, st);                            \
    }                                                                                                                              \
    template <> hipError_t route_lanes<TZ>(const LaneArgs& a, int G, bool stats, int grid, hipStream_t st) {                       \
        auto f = [&](auto g, auto v, auto n, auto w) { return route_one<g.value, v.value, n.value, w.value>(a, stats, grid, st); }; \
        SR_ROUTE_FORMS(SR_ROUTE_FORM)                                                                                              \
    }                                                                                                                              \
    template <> hipError_t route_grad_lanes<TZ>(const LaneArgs& a, int G, int grid, hipStream_t st) {                              \
        auto f = [&](auto g, auto v, auto n, auto w) { return grad_one<g.value, v.value, n.value, w.value>(a, grid, st); };        \
        SR_ROUTE_FORMS(SR_ROUTE_FORM)                                                                                              \
    }
#define SR_ROUTE_FORM(g, v, n, w) \
    f(std::integral_constant<int, g>{}, std::bool_constant<v>{}, std::integral_constant<int, n>{}, std::bool_constant<w>{})

}  // namespace srd

// The router: per-pixel lists from logits, the atoms' load and losses, and the gradient (include/sr_route.h).
//
// Here: checks, and the kernels that take every case, a wavefront for a pixel: a lane holds every 64th atom, the largest is
// found `entries` times over by a reduction of 64-bit keys (order of the logit, then the lower atom): fast for few pixels (lanes_from), and
// what is there for lists of more than 16 entries: a 1080p frame of 72 fp16 logits 5.5 ms for 17 entries (16 entries on the lanes 0.13),
// with the losses 6.0 (0.19), gradient 5.6 (0.19).
#include <stdint.h>

#include "sr_route_lanes.h"

namespace srd {
namespace {

constexpr int RNT = 256, RWAVES = RNT / 64, RMAXJ = SR_MAX_ATOMS / 64;

__device__ __forceinline__ unsigned long long wave_max_key(unsigned long long k) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        const unsigned long long o = __shfl_xor(k, d);
        k = o > k ? o : k;
    }
    return k;
}

template <typename TZ, typename TV, bool STATS>
__global__ __launch_bounds__(RNT) void k_route_wave(const RouteArgs a) {
    __shared__ double sh_share[STATS ? SR_MAX_ATOMS : 1], sh_sq;
    __shared__ unsigned sh_count[STATS ? SR_MAX_ATOMS : 1], sh_live;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float share[RMAXJ];
    double dshare[RMAXJ];
    unsigned count[RMAXJ], live = 0;
    double sq = 0.0;                     // a square may pass fp32's range where the mean does not
#pragma unroll
    for (int j = 0; j < RMAXJ; ++j) share[j] = 0.0f, dshare[j] = 0.0, count[j] = 0;
    int run = 0;
    for (int64_t g = (int64_t)blockIdx.x * RWAVES + wave; g < a.total; g += (int64_t)gridDim.x * RWAVES) {
        const int64_t n = g / a.px, i = g - n * a.px;
        const int64_t out0 = n * a.T * a.px + i;
        if (a.mask && a.mask[g] == 0) {
            for (int t = lane; t < a.T; t += 64) {
                a.index[out0 + t * a.px] = (unsigned char)t;
                st_from_float((TV*)a.value, out0 + t * a.px, 0.0f);
            }
            continue;
        }
        const int64_t base = logit_base(a, n, i);
        float z[RMAXJ];
        unsigned long long key[RMAXJ];
        float m = -INFINITY;
#pragma unroll
        for (int j = 0; j < RMAXJ; ++j) {
            const int l = lane + 64 * j;
            z[j] = l < a.L ? ld_as_float((const TZ*)a.z, base + l * a.lstride) : -INFINITY;
            // the lower 32 bits are never 0: a key of an atom is above 0, which marks those that are gone
            key[j] = l < a.L ? ((unsigned long long)logit_order(z[j]) << 32) | (unsigned)(~l) : 0;
            m = fmaxf(m, z[j]);
        }
        m = wave_max(m);
        const float o = exp_origin<TZ>(m);
        float e[RMAXJ], s = 0.0f;
#pragma unroll
        for (int j = 0; j < RMAXJ; ++j) s += e[j] = exp_from<TZ>(z[j], o);
        s = wave_sum(s);

        unsigned at[RMAXJ];             // entry t is kept by lane t % 64 in slot t / 64
        float top[RMAXJ];
        float chosen = 0.0f;
#pragma unroll
        for (int q = 0; q < RMAXJ; ++q) {
            at[q] = 0;
            top[q] = 0.0f;
            const int tn = a.T - 64 * q < 64 ? a.T - 64 * q : 64;
            for (int t = 0; t < tn; ++t) {
                unsigned long long k = key[0];
#pragma unroll
                for (int j = 1; j < RMAXJ; ++j) k = key[j] > k ? key[j] : k;
                k = wave_max_key(k);
                const int l = (int)(~(unsigned)k);
                float zv = 0.0f;
#pragma unroll
                for (int j = 0; j < RMAXJ; ++j)
                    if (l == lane + 64 * j) {
                        key[j] = 0;
                        zv = z[j];
                        if (STATS && z[j] != -INFINITY) ++count[j];
                    }
                zv = __shfl(zv, l & 63);
                if (lane == t) at[q] = l, top[q] = zv;
            }
            if (a.kind == SR_ROUTE_CHOSEN) chosen += lane < tn ? exp_from<TZ>(top[q], o) : 0.0f;
        }
        if (a.kind == SR_ROUTE_CHOSEN) chosen = wave_sum(chosen);
        const float whole = a.kind == SR_ROUTE_CHOSEN ? chosen : s;
        const float inv = whole > 0.0f || whole != whole ? 1.0f / whole : 0.0f;
#pragma unroll
        for (int q = 0; q < RMAXJ; ++q) {
            const int t = lane + 64 * q;
            if (t < a.T) {
                a.index[out0 + t * a.px] = (unsigned char)at[q];
                st_from_float((TV*)a.value, out0 + t * a.px, a.kind == SR_ROUTE_VALUES ? top[q] : exp_from<TZ>(top[q], o) * inv);
            }
        }
        if (STATS && m != -INFINITY) {
            const float is = 1.0f / s, lse = m + logit_log(s);
#pragma unroll
            for (int j = 0; j < RMAXJ; ++j) share[j] = fmaf(e[j], is, share[j]);
            sq = fma((double)lse, (double)lse, sq);
            ++live;
            if (++run == 64) {
                run = 0;
#pragma unroll
                for (int j = 0; j < RMAXJ; ++j) dshare[j] += share[j], share[j] = 0.0f;
            }
        }
    }
    if (!STATS) return;
    // the four wavefronts' sums, one after the other
    const RouteRecord r(a.partial, a.L, blockIdx.x);
    for (int w = 0; w < RWAVES; ++w) {
        if (wave == w) {
#pragma unroll
            for (int j = 0; j < RMAXJ; ++j) {
                const int l = lane + 64 * j;
                sh_share[l] = (w ? sh_share[l] : 0.0) + (dshare[j] + share[j]);
                sh_count[l] = (w ? sh_count[l] : 0u) + count[j];
            }
            if (lane == 0) {
                sh_sq = (w ? sh_sq : 0.0) + sq;
                sh_live = (w ? sh_live : 0u) + live;
            }
        }
        __syncthreads();
    }
    for (int l = threadIdx.x; l < a.L; l += RNT) r.share[l] = sh_share[l], r.counts[l] = sh_count[l];
    if (threadIdx.x == 0) *r.squares = sh_sq, *r.live = sh_live;
}

// The workgroups' sums, and the losses from them: one workgroup, a fixed order.  Latencies are what it takes: a thread has AHEAD records'
// loads under way at a time, at most 20 (registers: two 64-bit words each, 16 wavefronts on a CU).  launch_finish shares a thread's records
// out evenly over as few rounds as that leaves.  (131 072 fp16 pixels, the whole call, us, with 8, with 19 whatever the call, so: 16 atoms 16.6, 17.4,
// 16.0; 40 atoms 20.1, 20.3, 19.4; 72 atoms 22.9, 21.7, 22.1; 128 atoms 36.7, 38.3, 37.0; 256 atoms 61.5, 64.6, 62.2.)
constexpr int FNT = 1024;
template <int AHEAD>
__global__ __launch_bounds__(FNT) void k_route_finish(const void* partial, int records, int L, int T,
                                                      long long* counts, float* share, float* loss) {
    __shared__ double sh_s[FNT];
    __shared__ unsigned long long sh_c[FNT];
    __shared__ double sh_sq[FNT / 64], sh_f[SR_MAX_ATOMS / 64];
    __shared__ unsigned long long sh_m[FNT / 64];
    const int tid = threadIdx.x, groups = FNT / L, g = tid / L, l = tid - g * L;
    double q = 0.0;
    unsigned long long m = 0;
    static_assert(ROUTE_RECORDS <= FNT, "a record a thread");
    if (tid < records) {
        const RouteRecord rec((void*)partial, L, tid);
        q = *rec.squares;
        m = *rec.live;
    }
    double s = 0.0;
    unsigned long long c = 0;
    if (g < groups)
        for (int r0 = g; r0 < records; r0 += AHEAD * groups) {
            double v[AHEAD];
            unsigned long long n[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int r = r0 + i * groups;
                const RouteRecord rec((void*)partial, L, r < records ? r : r0);
                v[i] = rec.share[l];
                n[i] = rec.counts[l];
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
                if (r0 + i * groups < records) s += v[i], c += n[i];
        }
    sh_s[tid] = s;
    sh_c[tid] = c;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) q += __shfl_xor(q, d), m += __shfl_xor(m, d);
    if ((tid & 63) == 0) sh_sq[tid >> 6] = q, sh_m[tid >> 6] = m;
    __syncthreads();
    q = 0.0;
    m = 0;
#pragma unroll
    for (int w = 0; w < FNT / 64; ++w) q += sh_sq[w], m += sh_m[w];
    const double inv = m ? 1.0 / (double)m : 0.0;
    double fp = 0.0;
    if (tid < L) {
        s = 0.0;
        c = 0;
        for (int k = 0; k < groups; ++k) s += sh_s[k * L + tid], c += sh_c[k * L + tid];
        counts[tid] = (long long)c;
        share[tid] = (float)(s * inv);
        fp = (double)c * inv / T * (s * inv);
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) fp += __shfl_xor(fp, d);
    if ((tid & 63) == 0 && tid < SR_MAX_ATOMS) sh_f[tid >> 6] = fp;
    __syncthreads();
    if (tid == 0) {
        fp = 0.0;
        for (int w = 0; w < SR_MAX_ATOMS / 64; ++w) fp += sh_f[w];
        counts[L] = (long long)m;
        loss[0] = (float)(L * fp);
        loss[1] = (float)(q * inv);
    }
}

template <typename TZ, typename TV>
__global__ __launch_bounds__(RNT) void k_route_grad_wave(const RouteArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const bool softmax = a.kind == SR_ROUTE_SOFTMAX;
    float f[RMAXJ], w0 = 0.0f, w1 = 0.0f;
#pragma unroll
    for (int j = 0; j < RMAXJ; ++j) f[j] = 0.0f;
    if (a.counts) {
        const double M = (double)a.counts[a.L], inv = M > 0.0 ? 1.0 / M : 0.0;
        w0 = (float)(a.dloss[0] * (double)a.L * inv);
        w1 = (float)(a.dloss[1] * 2.0 * inv);
#pragma unroll
        for (int j = 0; j < RMAXJ; ++j)
            if (lane + 64 * j < a.L) f[j] = (float)((double)a.counts[lane + 64 * j] * inv / a.T);
    }
    for (int64_t g = (int64_t)blockIdx.x * RWAVES + wave; g < a.total; g += (int64_t)gridDim.x * RWAVES) {
        const int64_t n = g / a.px, i = g - n * a.px;
        const int64_t in0 = n * a.T * a.px + i, base = logit_base(a, n, i);
        const bool on = !a.mask || a.mask[g] != 0;
        float z[RMAXJ], e[RMAXJ], G[RMAXJ], m = -INFINITY;
        bool listed[RMAXJ];
#pragma unroll
        for (int j = 0; j < RMAXJ; ++j) {
            const int l = lane + 64 * j;
            z[j] = on && l < a.L && a.kind != SR_ROUTE_VALUES ? ld_as_float((const TZ*)a.z, base + l * a.lstride) : -INFINITY;
            m = fmaxf(m, z[j]);
            G[j] = 0.0f;
            listed[j] = false;
        }
        m = wave_max(m);
        const float o = exp_origin<TZ>(m);
        if (on && a.value)
            for (int t = 0; t < a.T; ++t) {
                const int l = a.index[in0 + t * a.px];
                const float v = ld_as_float((const TV*)a.value, in0 + t * a.px);
#pragma unroll
                for (int j = 0; j < RMAXJ; ++j)
                    if (l == lane + 64 * j) G[j] += v, listed[j] = true;
            }
        float s = 0.0f, sq = 0.0f, qG = 0.0f, fp = 0.0f;
#pragma unroll
        for (int j = 0; j < RMAXJ; ++j) {
            e[j] = exp_from<TZ>(z[j], o);
            s += e[j];
            const float q = softmax || listed[j] ? e[j] : 0.0f;
            sq += q;
            qG = fmaf(q, G[j], qG);
            fp = fmaf(e[j], f[j], fp);
        }
        s = wave_sum(s);
        sq = wave_sum(sq);
        qG = wave_sum(qG);
        fp = wave_sum(fp);
        const bool live = m != -INFINITY;
        const float is = live ? 1.0f / s : 0.0f, iq = live && sq > 0.0f ? 1.0f / sq : 0.0f;
        const float lse = live ? m + logit_log(s) : 0.0f;
        qG *= iq;
        fp *= is;
#pragma unroll
        for (int j = 0; j < RMAXJ; ++j) {
            const int l = lane + 64 * j;
            if (l >= a.L) continue;
            float d;
            if (a.kind == SR_ROUTE_VALUES) {
                d = G[j];
            } else {
                d = softmax || listed[j] ? e[j] * iq * (G[j] - qG) : 0.0f;
                if (a.counts) d = fmaf(e[j] * is, fmaf(w0, f[j] - fp, w1 * lse), d);
                if (z[j] == -INFINITY) d = 0.0f;
            }
            st_from_float((TZ*)a.dz, base + l * a.lstride, d);
        }
    }
}

void launch_finish(const void* partial, int records, int L, int T, long long* counts, float* share, float* loss, hipStream_t st) {
    const int groups = FNT / L, each = (records + groups - 1) / groups, rounds = (each + 19) / 20, ahead = rounds ? (each + rounds - 1) / rounds : 0;
    auto go = [&](auto n) { k_route_finish<decltype(n)::value><<<1, FNT, 0, st>>>(partial, records, L, T, counts, share, loss); };
    if (ahead <= 4) go(std::integral_constant<int, 4>{});
    else if (ahead <= 8) go(std::integral_constant<int, 8>{});
    else if (ahead <= 12) go(std::integral_constant<int, 12>{});
    else if (ahead <= 16) go(std::integral_constant<int, 16>{});
    else go(std::integral_constant<int, 20>{});
}

size_t route_esize(sr_dtype d) { return d == SR_F32 ? 4 : (d == SR_U8 ? 1 : 2); }

bool route_overlap(const void* p, size_t np, const void* q, size_t nq) {
    const uintptr_t a0 = (uintptr_t)p, b0 = (uintptr_t)q;
    return p && q && np && nq && a0 < b0 + nq && b0 < a0 + np;
}

size_t tensor_bytes(const sr_tensor* t) { return (size_t)t->n * t->c * t->h * t->w * route_esize(t->dtype); }

// Checks that the three calls share; fills what they share of the arguments.  `list`: index and value or dvalue (null: none).
int route_args(RouteArgs& a, bool& empty, const sr_tensor* coeff, int L, int scale, int entries, int kind, int layout,
               const sr_tensor* mask, const sr_tensor* index, const sr_tensor* value) {
    if (!coeff || !index) return SR_ERR_NULL;
    if ((coeff->dtype != SR_F32 && coeff->dtype != SR_F16 && coeff->dtype != SR_BF16) || index->dtype != SR_U8 ||
        (value && value->dtype != SR_F32 && value->dtype != SR_F16) || (mask && mask->dtype != SR_U8)) return SR_ERR_UNSUPPORTED;
    if (kind < SR_ROUTE_SOFTMAX || kind > SR_ROUTE_VALUES) return SR_ERR_UNSUPPORTED;
    if (layout != SR_COEFF_PLANAR && layout != SR_COEFF_PRE_SHUFFLE && layout != SR_COEFF_PIXEL_MAJOR) return SR_ERR_UNSUPPORTED;
    const bool pre = layout == SR_COEFF_PRE_SHUFFLE;
    if (L < 1 || L > SR_MAX_ATOMS || entries < 1 || entries > L || (pre && (scale < 2 || scale > 4))) return SR_ERR_UNSUPPORTED;
    for (const sr_tensor* t : {coeff, index, value, mask})
        if (t && (t->n < 0 || t->c < 0 || t->h < 0 || t->w < 0)) return SR_ERR_SHAPE;
    const int64_t H = (int64_t)coeff->h * (pre ? scale : 1), W = (int64_t)coeff->w * (pre ? scale : 1);
    if ((int64_t)coeff->c != (int64_t)L * (pre ? scale * scale : 1)) return SR_ERR_SHAPE;
    for (const sr_tensor* t : {index, value, mask})
        if (t && (t->n != coeff->n || t->h != H || t->w != W)) return SR_ERR_SHAPE;
    if (index->c != entries || (value && value->c != entries) || (mask && mask->c != 1)) return SR_ERR_SHAPE;
    if (coeff->n > 65535 || H > 4 * 65535 || W > (1 << 20)) return SR_ERR_UNSUPPORTED;
    empty = coeff->n == 0 || H == 0 || W == 0;
    if (!empty) {
        if (!coeff->data || !index->data || (value && !value->data) || (mask && !mask->data)) return SR_ERR_NULL;
        if ((uintptr_t)coeff->data % route_esize(coeff->dtype) || (value && (uintptr_t)value->data % route_esize(value->dtype)))
            return SR_ERR_ALIGN;
    }
    a = RouteArgs{};
    a.z = coeff->data;
    a.mask = mask ? (const unsigned char*)mask->data : nullptr;
    a.index = (unsigned char*)index->data;
    a.value = value ? value->data : nullptr;
    a.px = H * W;
    a.total = coeff->n * a.px;
    a.L = L; a.T = entries; a.kind = kind; a.layout = layout;
    a.H = (int)H; a.W = (int)W; a.h = coeff->h; a.w = coeff->w; a.s = pre ? scale : 1;
    a.lstride = layout == SR_COEFF_PIXEL_MAJOR ? 1 : (pre ? (int64_t)scale * scale * coeff->h * coeff->w : a.px);
    return SR_OK;
}

int blocks_for(int64_t waves, int most) {
    const int64_t need = (waves + RWAVES - 1) / RWAVES;
    return (int)(need < most ? need : most);
}

template <bool STATS>
hipError_t launch_route(const RouteArgs& a, sr_dtype z, sr_dtype v, int grid, hipStream_t st) {
    const bool half = v == SR_F16;
    if (z == SR_F32) {
        if (half) k_route_wave<float, __half, STATS><<<grid, RNT, 0, st>>>(a);
        else k_route_wave<float, float, STATS><<<grid, RNT, 0, st>>>(a);
    } else if (z == SR_F16) {
        if (half) k_route_wave<__half, __half, STATS><<<grid, RNT, 0, st>>>(a);
        else k_route_wave<__half, float, STATS><<<grid, RNT, 0, st>>>(a);
    } else {
        if (half) k_route_wave<bf16raw, __half, STATS><<<grid, RNT, 0, st>>>(a);
        else k_route_wave<bf16raw, float, STATS><<<grid, RNT, 0, st>>>(a);
    }
    return hipGetLastError();
}

hipError_t launch_route_grad(const RouteArgs& a, sr_dtype z, sr_dtype v, int grid, hipStream_t st) {
    const bool half = v == SR_F16;
    if (z == SR_F32) {
        if (half) k_route_grad_wave<float, __half><<<grid, RNT, 0, st>>>(a);
        else k_route_grad_wave<float, float><<<grid, RNT, 0, st>>>(a);
    } else if (z == SR_F16) {
        if (half) k_route_grad_wave<__half, __half><<<grid, RNT, 0, st>>>(a);
        else k_route_grad_wave<__half, float><<<grid, RNT, 0, st>>>(a);
    } else {
        if (half) k_route_grad_wave<bf16raw, __half><<<grid, RNT, 0, st>>>(a);
        else k_route_grad_wave<bf16raw, float><<<grid, RNT, 0, st>>>(a);
    }
    return hipGetLastError();
}

// The kernels for many pixels (sr_route_lanes.h): lists of at most 16 entries, a pixel's logits within 32-bit offsets of one another.
// A lane goes through its atoms one after the other, whatever the number of pixels, a wavefront for a pixel takes as long as there are
// pixels; they meet (72 to 256 atoms, fp32 and bfloat16, us a wavefront / lanes): lists 4096 pixels 9.1 / 9.5 and 9.2 / 12.1; with the
// losses 1024 pixels 17.2 / 21.0, 2048 pixels 21.9 / 21.1 and 43 / 26; gradient 4096 pixels 8.7 / 8.5, 256 atoms 8192 pixels 12.9 / 12.7
// and 13.1 / 19.6.  Lists come from the same kernel with and without the losses, so that both calls give the same bits: 2048 pixels costs
// the lists 2.5 us there and spares the losses 17.
// Rows of up to 72 atoms that are aligned 16-byte pieces, eight atoms or four a load, bfloat16, 1 and 1024 of them: 72 atoms 5.3 / 4.6 and
// 6.3 / 4.8, losses 10.6 / 11.8 and 15.6 / 16.2; 8 atoms 5.2 / 3.9 and 6.2 / 4.1, losses 13.0 / 12.2 and 17.8 / 13.9 (fp32 rows of 8 to 64,
// 5.3 / 5.3 and 6.2 / 5.7; of 72, 5.3 / 7.1 and 6.3 / 7.4).  Rows off those pieces, an atom a load, 1024 of them, fp32: 8 atoms 6.2 / 8.1, losses 17.8 / 19.9; 72 atoms
// 6.3 / 8.6 and 15.6 / 20.8: as planes.
int64_t lanes_from(const RouteArgs& r, bool vec, bool gradient) {
    if (gradient) return r.L > 128 ? 8192 : 4096;
    return vec && r.L <= 8 * LCH ? 1 : 2048;
}
int lanes_of(LaneArgs& a, const RouteArgs& r, sr_dtype z, sr_dtype v, const void* dz, bool gradient) {
    const bool pm = r.layout == SR_COEFF_PIXEL_MAJOR, pre = r.layout == SR_COEFF_PRE_SHUFFLE;
    const int64_t es = (int64_t)route_esize(z);
    const int G = pm || r.L > 8 * LCH ? 4 : 1;
    const bool vec = pm && r.L % 8 == 0 && (uintptr_t)r.z % 16 == 0 && (uintptr_t)dz % 16 == 0;
    if (r.T > 16 || r.total < lanes_from(r, vec, gradient)) return 0;
    if (G > 1 && 32 * r.lstride * es >= (int64_t)1 << 32) return 0;
    a.r = r;
    a.ipx = pre ? (int64_t)r.h * r.w : r.px;
    a.tiles_per_image = (a.ipx + 64 / G - 1) / (64 / G);
    a.tiles = r.total / a.ipx * a.tiles_per_image;
    a.vec = vec;
    a.half_value = v == SR_F16;
    return G;
}
hipError_t launch_lanes(const LaneArgs& a, sr_dtype z, int G, bool stats, int grid, hipStream_t st) {
    return z == SR_F32 ? route_lanes<float>(a, G, stats, grid, st) : z == SR_F16 ? route_lanes<__half>(a, G, stats, grid, st)
                                                                                 : route_lanes<bf16raw>(a, G, stats, grid, st);
}
int grid_for(int64_t tiles, int waves, int64_t most) {
    const int64_t need = (tiles + waves - 1) / waves;
    return (int)(need < most ? need : most);
}

// The outputs of a call (bytes, null where there is none) against its inputs and one another.
struct Span { const void* p; size_t n; };
template <int NO, int NI>
bool any_overlap(const Span (&out)[NO], const Span (&in)[NI]) {
    for (int i = 0; i < NO; ++i) {
        for (int j = 0; j < NI; ++j)
            if (route_overlap(out[i].p, out[i].n, in[j].p, in[j].n)) return true;
        for (int j = 0; j < i; ++j)
            if (route_overlap(out[i].p, out[i].n, out[j].p, out[j].n)) return true;
    }
    return false;
}
Span span(const sr_tensor* t) { return t ? Span{t->data, tensor_bytes(t)} : Span{nullptr, 0}; }

}  // namespace
}  // namespace srd

using namespace srd;

extern "C" __attribute__((visibility("default")))
int sr_list_route(const sr_tensor* coeff, int L, int scale, int entries, int kind, int coeff_layout,
                  const sr_tensor* mask, sr_tensor* index, sr_tensor* value, void* stream) {
    RouteArgs a;
    bool empty;
    if (!value) return SR_ERR_NULL;
    const int st = route_args(a, empty, coeff, L, scale, entries, kind, coeff_layout, mask, index, value);
    if (st != SR_OK || empty) return st;
    const Span out[] = {span(index), span(value)}, in[] = {span(coeff), span(mask)};
    if (any_overlap(out, in)) return SR_ERR_ALIAS;
    LaneArgs m;
    const int G = lanes_of(m, a, coeff->dtype, value->dtype, nullptr, false);
    const hipError_t e = G ? launch_lanes(m, coeff->dtype, G, false, grid_for(m.tiles, lanes_threads(false) / 64, 1 << 20), (hipStream_t)stream)
                           : launch_route<false>(a, coeff->dtype, value->dtype, blocks_for(a.total, 8 * compute_units()), (hipStream_t)stream);
    return e == hipSuccess ? SR_OK : SR_ERR_LAUNCH;
}

extern "C" __attribute__((visibility("default")))
size_t sr_list_route_workspace_bytes(int L) {
    return L < 1 || L > SR_MAX_ATOMS ? 0 : (size_t)ROUTE_RECORDS * (2 * L + 2) * 8;
}

extern "C" __attribute__((visibility("default")))
int sr_list_route_balance(const sr_tensor* coeff, int L, int scale, int entries, int kind, int coeff_layout,
                          const sr_tensor* mask, sr_tensor* index, sr_tensor* value,
                          long long* counts, float* share, float* loss,
                          void* workspace, size_t workspace_bytes, void* stream) {
    RouteArgs a;
    bool empty;
    if (!value || !counts || !share || !loss) return SR_ERR_NULL;
    const int st = route_args(a, empty, coeff, L, scale, entries, kind, coeff_layout, mask, index, value);
    if (st != SR_OK) return st;
    if (kind == SR_ROUTE_VALUES) return SR_ERR_UNSUPPORTED;
    if (!workspace || workspace_bytes < sr_list_route_workspace_bytes(L)) return SR_ERR_SHAPE;
    if ((uintptr_t)workspace % 16 || (uintptr_t)counts % 8 || (uintptr_t)share % 4 || (uintptr_t)loss % 4) return SR_ERR_ALIGN;
    const Span out[] = {span(index), span(value), {counts, (size_t)(L + 1) * 8}, {share, (size_t)L * 4}, {loss, 8},
                        {workspace, sr_list_route_workspace_bytes(L)}};
    const Span in[] = {span(coeff), span(mask)};
    if (any_overlap(out, in)) return SR_ERR_ALIAS;
    hipError_t e = hipSuccess;
    if (!empty) {
        a.partial = workspace;
        LaneArgs m;
        const int G = lanes_of(m, a, coeff->dtype, value->dtype, nullptr, false);
        a.records = G ? grid_for(m.tiles, lanes_threads(true) / 64, compute_units() < ROUTE_RECORDS ? compute_units() : ROUTE_RECORDS) : blocks_for(a.total, ROUTE_RECORDS);
        e = G ? launch_lanes(m, coeff->dtype, G, true, a.records, (hipStream_t)stream)
              : launch_route<true>(a, coeff->dtype, value->dtype, a.records, (hipStream_t)stream);
    }
    if (e == hipSuccess) {
        launch_finish(workspace, empty ? 0 : a.records, L, entries, counts, share, loss, (hipStream_t)stream);
        e = hipGetLastError();
    }
    return e == hipSuccess ? SR_OK : SR_ERR_LAUNCH;
}

extern "C" __attribute__((visibility("default")))
int sr_list_route_grad(const sr_tensor* coeff, const sr_tensor* index, const sr_tensor* dvalue,
                       int L, int scale, int entries, int kind, int coeff_layout, const sr_tensor* mask,
                       const long long* counts, const float* dloss, sr_tensor* dcoeff, void* stream) {
    RouteArgs a;
    bool empty;
    if (!dcoeff) return SR_ERR_NULL;
    const int st = route_args(a, empty, coeff, L, scale, entries, kind, coeff_layout, mask, index, dvalue);
    if (st != SR_OK) return st;
    if (!counts != !dloss) return SR_ERR_NULL;
    if (dcoeff->dtype != coeff->dtype || (kind == SR_ROUTE_VALUES && counts)) return SR_ERR_UNSUPPORTED;
    if (dcoeff->n != coeff->n || dcoeff->c != coeff->c || dcoeff->h != coeff->h || dcoeff->w != coeff->w) return SR_ERR_SHAPE;
    if (empty) return SR_OK;
    if (!dcoeff->data) return SR_ERR_NULL;
    if ((uintptr_t)dcoeff->data % route_esize(dcoeff->dtype) || (uintptr_t)counts % 8 || (uintptr_t)dloss % 4) return SR_ERR_ALIGN;
    const Span out[] = {span(dcoeff)};
    const Span in[] = {span(coeff), span(mask), span(index), span(dvalue), {counts, (size_t)(L + 1) * 8}, {dloss, 8}};
    if (any_overlap(out, in)) return SR_ERR_ALIAS;
    a.counts = counts;
    a.dloss = dloss;
    a.dz = dcoeff->data;
    const sr_dtype vd = dvalue ? dvalue->dtype : SR_F32;
    LaneArgs m;
    const int G = lanes_of(m, a, coeff->dtype, vd, a.dz, true);
    hipError_t e;
    if (!G) {
        e = launch_route_grad(a, coeff->dtype, vd, blocks_for(a.total, 8 * compute_units()), (hipStream_t)stream);
    } else {
        const int grid = grid_for(m.tiles, DWAVES, 4 * compute_units());
        e = coeff->dtype == SR_F32 ? route_grad_lanes<float>(m, G, grid, (hipStream_t)stream)
          : coeff->dtype == SR_F16 ? route_grad_lanes<__half>(m, G, grid, (hipStream_t)stream)
                                   : route_grad_lanes<bf16raw>(m, G, grid, (hipStream_t)stream);
    }
    return e == hipSuccess ? SR_OK : SR_ERR_LAUNCH;
}

// Layers and their gradients (include/sr_layer.h): checks, which kernels a call is made of, and their workspace.
//
// A gradient is three products: z made anew, with dz = dy act'(z) as its epilogue, stored in the workspace; dx = dz W; dW = dz^T x.  db comes from sums that the
// first leaves on its way out, or from the workgroups of dW's first column of tiles, which sum dz beside it.  Without an activation dy is dz.
#include <stdint.h>
#include <type_traits>

#include "sr_gemm.h"

namespace srd {
namespace {

constexpr int GPU_CUS = 256;                 // of a gfx950 in one partition; the plan is the same wherever the sizes are asked for

size_t layer_esize(int d) { return d == SR_F32 ? 4 : 2; }
bool layer_type(int d) { return d == SR_F32 || d == SR_F16 || d == SR_BF16; }
bool layer_act(int a) { return a >= SR_ACT_NONE && a <= SR_ACT_SIGMOID; }
bool features(int64_t c) { return c >= 1 && c <= SR_MAX_FEATURES; }
constexpr long long MOST_ROWS = 0x7fffffffLL - 256;

size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

struct Span { const void* p; size_t n; };
size_t bytes_of(const sr_tensor* t) { return (size_t)t->n * t->c * t->h * t->w * layer_esize(t->dtype); }
Span span(const sr_tensor* t) { return t ? Span{t->data, bytes_of(t)} : Span{nullptr, 0}; }
bool overlap(const Span& a, const Span& b) {
    const uintptr_t p = (uintptr_t)a.p, q = (uintptr_t)b.p;
    return a.p && b.p && a.n && b.n && p < q + b.n && q < p + a.n;
}
template <int NO, int NI>
bool any_overlap(const Span (&out)[NO], const Span (&in)[NI]) {
    for (int i = 0; i < NO; ++i) {
        for (int j = 0; j < NI; ++j)
            if (overlap(out[i], in[j])) return true;
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return true;
    }
    return false;
}

int64_t rows_of(const sr_tensor* t) { return (int64_t)t->n * t->h * t->w; }

struct Layer {
    int64_t rows;
    int in, out, wide, dtype;
    bool gated;
};

// How one product is cut: tile (or the kernel for few rows, or for a small weight), splits of k, and what the tiles should take.
constexpr int SKINNY = -1, THIN = -2;
struct Cut { int tile, splits, ksplit; double us; bool rows; };       // rows: by launch_rows where A's rows are at multiples of four bytes

// Microseconds of c workgroups of a tile on each compute unit, each with `steps` of 128 bytes of k: what one alone takes a step, what each takes
// where `share` of them keep a unit busy, and what a round of them takes beside that.  Measured with 1, 2, 4 and 8 workgroups a unit and k
// from 64 to 8192.
double tile_time(int tile, int64_t c, int64_t steps, size_t es) {
    static const double alone[2][4] = {{0.30, 0.58, 0.79, 1.28}, {0.62, 1.58, 2.67, 4.77}}, full[2][4] = {{0.19, 0.485, 0.79, 1.28}, {0.47, 1.46, 2.67, 4.77}};
    static const double round[4] = {3.0, 5.0, 9.0, 13.0};
    static const int share[4] = {4, 2, 1, 1};
    const int f = es == 4;
    const int64_t whole = c / share[tile], rest = c % share[tile];
    double us = (double)whole * (share[tile] * full[f][tile] * (double)steps + round[tile]);
    if (rest) us += (rest * full[f][tile] > alone[f][tile] ? rest * full[f][tile] : alone[f][tile]) * (double)steps + round[tile];
    return us;
}
// From here on rows with a weight that fits go to the kernel for them; where that takes 16 at a time (500 000 of 128 to 128, bfloat16: 58 us, tiles 47), only
// if the rows are no 16-byte pieces, which the tile kernels read by way of registers (351 576 of 27 to 121, fp32: 55 us, tiles 65).
constexpr int64_t THIN_FROM = 4096;
// A gated block goes there where LDS has room for its output, or, if its products take longer than its rows' way (rows of more than 192 bytes, fp32 64) or its
// output's rows meet in the same banks of LDS (16 bits, multiples of 256 bytes), for twice that: bfloat16, 400 000 rows of 32 to 120 30 us, by other kernels 38, of 64
// to 72 23 and 38; but of 32 to 128 57 and 35, 12 000 of 128 to 64 8.5 and 7.2; fp32, 400 000 of 16 to 64 33 and 41, but of 32 to 64 48 and 41.
int thin_room(int64_t n, int64_t k, size_t es, bool gated) {
    return gated && (k * (int64_t)es > (es == 2 ? 192 : 64) || (es == 2 && n * (int64_t)es % 256 == 0)) ? 2 : 1;
}
// From so many outputs on (of a launch; more where there is more to read, or several) the kernel that holds the weight is worth its start (bfloat16, 65536 rows
// of 64 to 512: 21 us, tiles 25, of 256 to 256 26 and 22; 1048576 rows of 64 to 512: 231 and 415, of 136 to 200 202 and 360).  Each launch reads the
// rows again (bfloat16, 131072 rows of 256 to 1024 in four launches, gradient: 446 us, tiles 427; fp32, 351576 rows of 64 to 1024 in two: 564 and 505).
// fp32 of more than 64 features splits more values than it multiplies (351576 rows of 128 to 256: 200 us, tiles 196; 1048576: 530 and 581; all fp32 figures here are some 4 %
// more on both sides since h is kept finite).
// A residual, of which the plan knows nothing, can halve a launch's columns: up to as many launches as there may be without one (bfloat16, 131072 rows
// of 256 to 2048: 460 us in eight, tiles 380; of 136 to 1024 206 in four, tiles 227; fp32, 1048576 rows of 64 to 512 1003 in two, tiles 1213).
constexpr double ROWS_FROM = 26e6;
constexpr int ROWS_LAUNCHES = 4;
// A launch has less than 2^32 threads, 256 a tile: 2^31 rows of few columns need larger tiles than the smallest.
constexpr int64_t LAUNCH_TILES = 1 << 24;
// The cut that should take least.  Split sums cost a launch and their way, written and read in fp32, at 8 bytes a ps through the
// caches, at 4.5 past them.
Cut cut_of(int64_t m, int64_t n, int64_t k, size_t es, int layout, bool gated, bool thin = true, bool rows = true, bool slope = false, int tiles_up_to = 4) {
    const int64_t bk = 128 / (int64_t)es, steps = (k + bk - 1) / bk;
    if (layout == GEMM_KC_KC && m <= SKINNY_ROWS) return {SKINNY, 1, 0, 0.0, false};
    if (thin && layout != GEMM_RC_RC && m >= THIN_FROM) {
        const ThinShape s = thin_shape(n, k, es, gated, thin_room(n, k, es, gated));
        if (s.waves && (s.rows == 32 || k * (int64_t)es % 16)) return {THIN, 1, 0, 0.0, false};
    }
    const int64_t nn = gated ? 2 * n : n;
    Cut best = {0, 1, 0, 0.0, false};
    double least = 1e300;
    for (int tile = 0; tile < tiles_up_to; ++tile) {
        const int64_t tiles = ((m + gemm_tile_rows(tile) - 1) / gemm_tile_rows(tile)) * ((nn + gemm_tile_cols(tile) - 1) / gemm_tile_cols(tile));
        if (tiles >= LAUNCH_TILES && tile < 3) continue;
        auto look = [&](int64_t splits) {
            if (splits > steps / 2) splits = steps / 2;
            if (splits > 1024) splits = 1024;
            if (splits < 1) splits = 1;
            const int64_t each = steps ? (steps + splits - 1) / splits : 0;
            splits = steps ? (steps + each - 1) / each : 1;
            double us = tile_time(tile, (tiles * splits + GPU_CUS - 1) / GPU_CUS, each, es);
            const double mb = 8e-6 * (double)splits * (double)m * (double)nn;
            if (splits > 1) us += 3.0 + mb / (mb < 128.0 ? 8.0 : 4.5);
            if (us < least) least = us, best = Cut{tile, (int)splits, (int)(each * bk), us, false};
        };
        for (int s = 1; s <= 8; ++s) look(s);
        for (int c = 1; c <= 8 && tiles; ++c) look(c * GPU_CUS / tiles);
    }
    if (rows && layout != GEMM_RC_RC && best.splits == 1) {
        const RowsShape s = rows_shape(m, n, k, es, gated, slope);
        const double cols = gated ? 2.0 * s.cols : s.cols;
        const int most = es == 2 ? slope ? 2 : ROWS_LAUNCHES : gated && !slope ? ROWS_LAUNCHES : 1;
        const double from = ROWS_FROM * (k > cols ? (double)k / cols : 1.0) * (s.launches > 1 ? 2.0 : 1.0) * (es == 4 && k > 64 ? 4.0 : 1.0);
        best.rows = s.grid && s.launches <= most && (double)m * cols >= from;
    }
    return best;
}

// Scratch of a split product: its partial results, and (dW) its partial sums of dz
size_t partial_bytes(const Cut& c, int64_t m, int64_t width) { return c.splits > 1 ? up256((size_t)c.splits * m * width * 4) : 0; }

template <typename F> hipError_t by_type(int d, F f) {
    return d == SR_F32 ? f((float*)nullptr) : d == SR_F16 ? f((__half*)nullptr) : f((bf16raw*)nullptr);
}

// Scratch for the sums of dz over the rows that the product which makes it leaves: two of them for each row of tiles, of 128 rows where the operands are
// off 16-byte pieces; one for each group of rows of a workgroup that holds the weight; where the product is split or of few rows, dz itself in fp32
bool leaves_rows(const Cut& c) { return c.tile == SKINNY || c.splits > 1; }
size_t slope_sum_bytes(const Cut& c, const Layer& l) {
    if (leaves_rows(c)) return up256((size_t)l.rows * l.wide * 4);
    const int64_t rows = gemm_tile_rows(c.tile > 1 ? 1 : c.tile);
    int64_t all = 2 * ((l.rows + rows - 1) / rows);
    if (c.rows) {
        const RowsShape s = rows_shape(l.rows, l.out, l.in, layer_esize(l.dtype), l.gated, true);
        if (all < (int64_t)s.grid * s.wr) all = (int64_t)s.grid * s.wr;
    }
    return up256((size_t)all * l.wide * 4);
}

// One product, split or not.  g: operands, sizes, mode and what the epilogue needs.  `ws`: partial_bytes of scratch (and, for RC_RC with sums_out but
// no sums, of those).  A forward product with g.sums says in *sum_rows how many rows of them it leaves.
hipError_t product(GemmArgs g, const Cut& c, int dtype, int layout, void* ws, hipStream_t st, int* sum_rows = nullptr) {
    const size_t es = layer_esize(dtype);
    const bool gated = g.mode == GEMM_GATED || g.mode == GEMM_GATED_SLOPE;
    const bool aligned = (uintptr_t)g.a % 16 == 0 && (uintptr_t)g.b % 16 == 0 && g.lda * es % 16 == 0 && g.ldb * es % 16 == 0;
    g.splits = c.splits;
    g.ksplit = c.ksplit ? c.ksplit : g.k;
    if (sum_rows && leaves_rows(c)) {
        g.exact = g.sums;
        g.sums = nullptr;
        *sum_rows = g.m;
    }
    return by_type(dtype, [&](auto t) -> hipError_t {
        using T = std::remove_pointer_t<decltype(t)>;
        if (c.tile == SKINNY) return launch_skinny<T>(g, aligned, st);
        if (c.tile == THIN) return launch_thin<T>(g, layout, st);
        if (c.rows && (uintptr_t)g.a % 4 == 0 && g.lda * es % 4 == 0) {
            const RowsShape r = rows_shape(g.m, g.n, g.k, es, gated, g.extra);
            if (r.grid && r.launches <= ROWS_LAUNCHES) {
                if (sum_rows) *sum_rows = r.grid * r.wr;
                return launch_rows<T>(g, layout, st);
            }
        }
        int tile = c.tile;
        if ((!aligned || g.a_lo || g.out_lo) && tile > 1) tile = 1;
        const int rows = gemm_tile_rows(tile), cols = gemm_tile_cols(tile);
        const int64_t width = gated ? 2 * (int64_t)g.n : g.n;
        g.tiles_m = (g.m + rows - 1) / rows;
        g.tiles_n = g.out ? (int)((width + cols - 1) / cols) : 1;      // without: the sums of dz alone
        if (g.sums && sum_rows) *sum_rows = 2 * g.tiles_m;
        GemmArgs p = g;
        if (g.splits > 1) {
            p.mode = GEMM_PARTIAL;
            p.n = (int)width;
            p.partial = g.partial = g.out ? (float*)ws : nullptr;
        }
        if (layout == GEMM_RC_RC) {
            if (g.sums) p.sums = nullptr, p.sums_out = nullptr;        // there already: only to be added up
            else if (g.sums_out && g.splits > 1) p.sums = g.sums = (float*)((char*)ws + partial_bytes(c, g.m, width));
        }
        if (layout != GEMM_RC_RC || g.out || !g.sum_rows) {
            const hipError_t e = launch_gemm<T>(p, layout, aligned, tile, st);
            if (e != hipSuccess) return e;
        }
        return g.partial || (layout == GEMM_RC_RC && g.sums) ? launch_gemm_finish<T>(g, st) : hipSuccess;
    });
}

// Rows on 16-byte pieces: dz, and copies of tensors that are not, where the products gain more than the copies take.  16-bit types: the tile kernels read other rows by way
// of registers and take 2.2 times as long (gradient of 16207 rows of 1754 to 1183, gated, fp16: 1087 us, so 508).  fp32 goes to LDS by 4 bytes (500 rows of 333 to 555: 16
// us, by registers 21); copies have the larger tiles to gain.
int64_t whole_row(const Layer& l, int64_t cols) { const int64_t e = 16 / (int64_t)layer_esize(l.dtype); return (cols + e - 1) / e * e; }
bool whole(const Layer& l, int64_t cols) { return whole_row(l, cols) == cols; }
size_t copy_bytes(const Layer& l, int64_t rows, int64_t cols) { return up256((size_t)rows * whole_row(l, cols) * layer_esize(l.dtype)); }
constexpr int TILES_OFF_PIECES = 2;
constexpr double OFF_PIECES = 1.1;          // what these take there, of what tile_time says (8192 rows of 4095 to 4097, fp32: 1817 us, with copies 1713)
bool copies_pay(double gain, size_t bytes, int copies) { return gain > 4.0 * copies + 2.0 * (double)bytes / 4.5e6; }
hipError_t copy_rows(const Layer& l, const void* from, int64_t rows, int cols, void* to, hipStream_t st) {
    return by_type(l.dtype, [&](auto t) { return launch_pack<std::remove_pointer_t<decltype(t)>>(from, rows, cols, to, st); });
}

// A forward call: its product, and whether x and the weight are copied first; its scratch.
struct ForwardPlan { Cut z; size_t x, w, need; };
ForwardPlan forward_plan(const Layer& l) {
    ForwardPlan p = {};
    const size_t es = layer_esize(l.dtype);
    p.z = cut_of(l.rows, l.out, l.in, es, GEMM_KC_KC, l.gated);
    if (p.z.tile >= 0 && !whole(l, l.in) && !(p.z.rows && es == 4)) {
        const size_t x = copy_bytes(l, l.rows, l.in), w = copy_bytes(l, l.wide, l.in);
        const Cut off = es == 4 ? cut_of(l.rows, l.out, l.in, es, GEMM_KC_KC, l.gated, true, false, false, TILES_OFF_PIECES) : p.z;
        if (copies_pay(es == 4 ? OFF_PIECES * off.us - p.z.us : 1.2 * p.z.us, x + w, 2)) p.x = x, p.w = w;
        else p.z = off;
    }
    p.need = p.x + p.w + partial_bytes(p.z, l.rows, l.wide);
    return p;
}

// 16-bit types: up to so many operations a product, dz goes on as two numbers, which hold it to 2^-17 or better: twice the matrix instructions in two products that
// are launches' time.  Beyond, it is rounded once, which adds 2^-9 (fp16: 2^-12) of each value in random directions to sums over many: a gradient's error in norm
// is 1.4 times that of its own rounding.  db is summed before that rounding.
constexpr double TWO_PARTS_UP_TO = 2e9;

// How a gradient is made.  pass: the workgroups of the one pass that makes all of it, for a small layer whose tensors allow it, or 0.  Else three products, z, dx and
// dweight; parts: numbers that dz is stored as (0: dy is dz); slopes: db comes from sums that z's product leaves.  Scratch: copies of x, the
// weight and dy on 16-byte pieces where they pay, dz, those sums, and what the products take.
struct GradPlan { Cut z, x, w; int pass, parts; bool slopes; size_t copy_x, copy_w, copy_dy, dz, sums, need; };
GradPlan grad_plan(const Layer& l, int act) {
    const size_t es = layer_esize(l.dtype);
    const bool again = l.gated || act != SR_ACT_NONE;
    GradPlan p = {};
    if (l.rows >= THIN_FROM && thin_grad_shape(l.in, l.out, (int)es, l.gated, again).bytes) {
        const int64_t blocks = (l.rows + 63) / 64;
        p.pass = (int)(blocks < 2 * GPU_CUS ? blocks : 2 * GPU_CUS);
    }
    if (again) p.parts = es == 2 && 2.0 * (double)l.rows * l.in * l.wide <= TWO_PARTS_UP_TO ? 2 : 1;
    const bool free = p.parts < 2;                         // of second parts: any kernel
    auto cut = [&](int tiles) {
        p.x = cut_of(l.rows, l.in, l.wide, es, GEMM_KC_RC, false, free, free, false, tiles);
        p.w = cut_of(l.wide, l.in, l.rows, es, GEMM_RC_RC, false, false, false, false, tiles);
        if (again) p.z = cut_of(l.rows, l.out, l.in, es, GEMM_KC_KC, l.gated, false, free, true, tiles);
        return p.z.us + p.x.us + p.w.us;
    };
    size_t copies[3] = {whole(l, l.in) ? 0 : copy_bytes(l, l.rows, l.in), whole(l, l.in) ? 0 : copy_bytes(l, l.wide, l.in),
                        again || whole(l, l.out) ? 0 : copy_bytes(l, l.rows, l.out)};
    const size_t copied = copies[0] + copies[1] + copies[2];
    double us = cut(4);
    if (l.rows && copied) {
        const double off = es == 4 ? cut(TILES_OFF_PIECES) : 0.0;
        if (copies_pay(es == 4 ? OFF_PIECES * off - us : 1.2 * us, copied, 3)) {
            p.copy_x = copies[0], p.copy_w = copies[1], p.copy_dy = copies[2];
            if (es == 4) us = cut(4);
        }
    }
    size_t most = 0;
    if (again) {
        // fp32 loses nothing on the way; there it is only that the large tiles' sums beside dW cost their workgroups a sixth
        p.slopes = es == 2 ? p.parts == 1 : !leaves_rows(p.z) && p.w.tile >= 2;
        p.dz = up256((size_t)p.parts * l.rows * whole_row(l, l.wide) * es);
        p.sums = p.slopes ? slope_sum_bytes(p.z, l) : 0;
        most = partial_bytes(p.z, l.rows, l.wide);
    }
    const size_t x = partial_bytes(p.x, l.rows, l.in);
    const size_t w = partial_bytes(p.w, l.wide, l.in) + (p.w.splits > 1 ? up256((size_t)p.w.splits * l.wide * 4) : 0);
    if (x > most) most = x;
    if (w > most) most = w;
    p.need = p.copy_x + p.copy_w + p.copy_dy + p.dz + p.sums + most;
    const size_t pass = up256((size_t)p.pass * l.wide * l.in * 4) + up256((size_t)p.pass * l.wide * 4);
    if (pass > p.need) p.need = pass;
    return p;
}

bool layer_sizes(Layer& l, long long rows, int in, int out, int dtype, bool gated) {
    if (rows < 0 || rows > MOST_ROWS || !features(in) || !features(out) || !layer_type(dtype)) return false;
    l = Layer{rows, in, out, gated ? 2 * out : out, dtype, gated};
    return true;
}

bool is_matrix(const sr_tensor* t, int rows, int cols) { return t->n == 1 && t->c == 1 && t->h == rows && t->w == cols; }
bool same_rows(const sr_tensor* t, const sr_tensor* x) { return t->n == x->n && t->h == x->h && t->w == x->w; }

// What all four calls check.  `y` is the forward call's output or dy; rest: further tensors with the rows of x and y's features (or null).
int layer_args(Layer& l, const sr_tensor* x, const sr_tensor* weight, const sr_tensor* bias, int act, const sr_tensor* y,
               const sr_tensor* residual, bool gated) {
    if (!x || !weight || !y) return SR_ERR_NULL;
    if (!layer_type(x->dtype) || !layer_act(act)) return SR_ERR_UNSUPPORTED;
    for (const sr_tensor* t : {weight, bias, y, residual})
        if (t && t->dtype != x->dtype) return SR_ERR_UNSUPPORTED;
    for (const sr_tensor* t : {x, weight, bias, y, residual})
        if (t && (t->n < 0 || t->c < 0 || t->h < 0 || t->w < 0)) return SR_ERR_SHAPE;
    if (!features(x->c) || !features(y->c)) return SR_ERR_UNSUPPORTED;
    if ((int64_t)x->n * x->h > MOST_ROWS || (int64_t)x->n * x->h * x->w > MOST_ROWS) return SR_ERR_UNSUPPORTED;
    layer_sizes(l, rows_of(x), x->c, y->c, x->dtype, gated);
    if (!is_matrix(weight, l.wide, l.in) || (bias && !is_matrix(bias, 1, l.wide)) || !same_rows(y, x)) return SR_ERR_SHAPE;
    if (residual && (!same_rows(residual, x) || residual->c != y->c)) return SR_ERR_SHAPE;
    const size_t es = layer_esize(l.dtype);
    for (const sr_tensor* t : {weight, bias}) {
        if (t && !t->data) return SR_ERR_NULL;
        if (t && (uintptr_t)t->data % es) return SR_ERR_ALIGN;
    }
    if (l.rows)
        for (const sr_tensor* t : {x, y, residual}) {
            if (t && !t->data) return SR_ERR_NULL;
            if (t && (uintptr_t)t->data % es) return SR_ERR_ALIGN;
        }
    return SR_OK;
}
int scratch_args(const void* workspace, size_t bytes, size_t need) {
    if (need && (!workspace || bytes < need)) return SR_ERR_SHAPE;
    return need && (uintptr_t)workspace % 16 ? SR_ERR_ALIGN : SR_OK;
}

GemmArgs forward_args(const Layer& l, const sr_tensor* x, const sr_tensor* weight, const sr_tensor* bias, int act) {
    GemmArgs g = {};
    g.a = x->data;
    g.b = weight->data;
    g.lda = g.ldb = l.in;
    g.m = (int)l.rows;
    g.n = g.half = l.out;
    g.k = l.in;
    g.act = act;
    g.bias = bias ? bias->data : nullptr;
    g.ld_extra = g.ld_out = l.out;
    return g;
}

int forward(const sr_tensor* x, const sr_tensor* weight, const sr_tensor* bias, int act, const sr_tensor* residual, sr_tensor* y, bool gated,
            void* workspace, size_t workspace_bytes, void* stream) {
    Layer l;
    int st = layer_args(l, x, weight, bias, act, y, residual, gated);
    if (st != SR_OK) return st;
    const ForwardPlan plan = forward_plan(l);
    const size_t need = plan.need;
    st = scratch_args(workspace, workspace_bytes, need);
    if (st != SR_OK) return st;
    const Span out[] = {span(y), {need ? workspace : nullptr, need}}, in[] = {span(x), span(weight), span(bias), span(residual)};
    if (any_overlap(out, in)) return SR_ERR_ALIAS;
    if (!l.rows) return SR_OK;
    GemmArgs g = forward_args(l, x, weight, bias, act);
    g.mode = gated ? GEMM_GATED : GEMM_STORE;
    g.extra = residual ? residual->data : nullptr;
    g.out = y->data;
    hipStream_t s = (hipStream_t)stream;
    hipError_t e = hipSuccess;
    if (plan.x) {
        char* const copy = (char*)workspace;
        e = copy_rows(l, x->data, l.rows, l.in, copy, s);
        if (e == hipSuccess) e = copy_rows(l, weight->data, l.wide, l.in, copy + plan.x, s);
        g.a = copy;
        g.b = copy + plan.x;
        g.lda = g.ldb = whole_row(l, l.in);
    }
    if (e == hipSuccess) e = product(g, plan.z, l.dtype, GEMM_KC_KC, (char*)workspace + plan.x + plan.w, s);
    return e == hipSuccess ? SR_OK : SR_ERR_LAUNCH;
}

int gradient(const sr_tensor* x, const sr_tensor* weight, const sr_tensor* bias, int act, const sr_tensor* dy,
             sr_tensor* dx, sr_tensor* dweight, sr_tensor* dbias, bool gated, void* workspace, size_t workspace_bytes, void* stream) {
    Layer l;
    int st = layer_args(l, x, weight, bias, act, dy, nullptr, gated);
    if (st != SR_OK) return st;
    if (!dx && !dweight && !dbias) return SR_ERR_NULL;
    for (const sr_tensor* t : {dx, dweight, dbias})
        if (t && t->dtype != x->dtype) return SR_ERR_UNSUPPORTED;
    if ((dx && (!same_rows(dx, x) || dx->c != x->c)) || (dweight && !is_matrix(dweight, l.wide, l.in)) || (dbias && !is_matrix(dbias, 1, l.wide)))
        return SR_ERR_SHAPE;
    const size_t es = layer_esize(l.dtype);
    for (const sr_tensor* t : {l.rows ? dx : nullptr, dweight, dbias}) {
        if (t && !t->data) return SR_ERR_NULL;
        if (t && (uintptr_t)t->data % es) return SR_ERR_ALIGN;
    }
    const GradPlan plan = grad_plan(l, act);
    const size_t need = plan.need;
    st = scratch_args(workspace, workspace_bytes, need);
    if (st != SR_OK) return st;
    const Span out[] = {span(dx), span(dweight), span(dbias), {need ? workspace : nullptr, need}};
    const Span in[] = {span(x), span(weight), span(bias), span(dy)};
    if (any_overlap(out, in)) return SR_ERR_ALIAS;

    hipStream_t s = (hipStream_t)stream;
    uintptr_t at = 0;
    for (const sr_tensor* t : {x, weight, dy, (const sr_tensor*)dx}) at |= t ? (uintptr_t)t->data : 0;
    if (plan.pass && at % 16 == 0) {
        ThinGradArgs a = {x->data, weight->data, bias ? bias->data : nullptr, dy->data, dx ? dx->data : nullptr, nullptr, nullptr, l.rows, l.in, l.out, act};
        if (dweight) a.partial = (float*)workspace;
        if (dbias) a.sums = (float*)((char*)workspace + up256((size_t)plan.pass * l.wide * l.in * 4));
        GemmArgs g = {};
        g.m = l.wide;
        g.n = l.in;
        g.splits = plan.pass;
        g.mode = GEMM_STORE;
        g.out = dweight ? dweight->data : nullptr;
        g.ld_out = l.in;
        g.sums_out = dbias ? dbias->data : nullptr;
        g.partial = a.partial;
        g.sums = a.sums;
        const hipError_t e = by_type(l.dtype, [&](auto t) -> hipError_t {
            using T = std::remove_pointer_t<decltype(t)>;
            const hipError_t first = launch_thin_grad<T>(a, gated, plan.pass, s);
            return first != hipSuccess || !(dweight || dbias) ? first : launch_gemm_finish<T>(g, s);
        });
        return e == hipSuccess ? SR_OK : SR_ERR_LAUNCH;
    }
    char* at_ws = (char*)workspace;
    auto take = [&](size_t bytes) { char* const p = at_ws; at_ws += bytes; return p; };
    const void *xa = x->data, *wa = weight->data, *z = dy->data;
    int64_t ldx = l.in, ldz = l.out, lo = 0;
    hipError_t e = hipSuccess;
    if (plan.copy_x) {
        char *const cx = take(plan.copy_x), *const cw = take(plan.copy_w);
        e = copy_rows(l, xa, l.rows, l.in, cx, s);
        if (e == hipSuccess) e = copy_rows(l, wa, l.wide, l.in, cw, s);
        xa = cx;
        wa = cw;
        ldx = whole_row(l, l.in);
    }
    if (plan.copy_dy) {
        char* const cd = take(plan.copy_dy);
        if (e == hipSuccess) e = copy_rows(l, z, l.rows, l.out, cd, s);
        z = cd;
        ldz = whole_row(l, l.out);
    }
    char* const dz = take(plan.dz);
    float* const slopes = plan.slopes ? (float*)take(plan.sums) : nullptr;
    void* const rest = at_ws;
    int slope_rows = 0;
    if (plan.parts && e == hipSuccess) {
        GemmArgs g = forward_args(l, x, weight, bias, act);
        g.a = xa;
        g.b = wa;
        g.lda = g.ldb = ldx;
        g.mode = gated ? GEMM_GATED_SLOPE : GEMM_SLOPE;
        g.extra = dy->data;
        g.out = dz;
        g.ld_out = ldz = whole_row(l, l.wide);
        g.out_lo = lo = plan.parts == 2 ? l.rows * ldz : 0;
        if (dbias) g.sums = slopes;
        z = dz;
        if (l.rows) e = product(g, plan.z, l.dtype, GEMM_KC_KC, rest, s, g.sums ? &slope_rows : nullptr);
    }
    if (dx && l.rows && e == hipSuccess) {
        GemmArgs g = {};
        g.a = z;
        g.lda = ldz;
        g.a_lo = lo;
        g.b = wa;
        g.ldb = ldx;
        g.m = (int)l.rows;
        g.n = l.in;
        g.k = l.wide;
        g.mode = GEMM_STORE;
        g.out = dx->data;
        g.ld_out = l.in;
        e = product(g, plan.x, l.dtype, GEMM_KC_RC, rest, s);
    }
    if ((dweight || dbias) && e == hipSuccess) {
        GemmArgs g = {};
        g.a = z;
        g.lda = ldz;
        g.a_lo = lo;
        g.b = xa;
        g.ldb = ldx;
        g.m = l.wide;
        g.n = l.in;
        g.k = (int)l.rows;
        g.mode = GEMM_STORE;
        g.out = dweight ? dweight->data : nullptr;
        g.ld_out = l.in;
        g.sums_out = dbias ? dbias->data : nullptr;
        if (slope_rows) g.sums = slopes, g.sum_rows = slope_rows;
        e = product(g, plan.w, l.dtype, GEMM_RC_RC, rest, s);
    }
    return e == hipSuccess ? SR_OK : SR_ERR_LAUNCH;
}

}  // namespace
}  // namespace srd

using namespace srd;

extern "C" __attribute__((visibility("default")))
size_t sr_layer_linear_workspace_bytes(long long rows, int in, int out, int dtype) {
    Layer l;
    return layer_sizes(l, rows, in, out, dtype, false) ? forward_plan(l).need : 0;
}

extern "C" __attribute__((visibility("default")))
int sr_layer_linear(const sr_tensor* x, const sr_tensor* weight, const sr_tensor* bias, int act, const sr_tensor* residual,
                    sr_tensor* y, void* workspace, size_t workspace_bytes, void* stream) {
    return forward(x, weight, bias, act, residual, y, false, workspace, workspace_bytes, stream);
}

extern "C" __attribute__((visibility("default")))
size_t sr_layer_linear_grad_workspace_bytes(long long rows, int in, int out, int dtype, int act) {
    Layer l;
    return layer_act(act) && layer_sizes(l, rows, in, out, dtype, false) ? grad_plan(l, act).need : 0;
}

extern "C" __attribute__((visibility("default")))
int sr_layer_linear_grad(const sr_tensor* x, const sr_tensor* weight, const sr_tensor* bias, int act, const sr_tensor* dy,
                         sr_tensor* dx, sr_tensor* dweight, sr_tensor* dbias,
                         void* workspace, size_t workspace_bytes, void* stream) {
    return gradient(x, weight, bias, act, dy, dx, dweight, dbias, false, workspace, workspace_bytes, stream);
}

extern "C" __attribute__((visibility("default")))
size_t sr_layer_gated_workspace_bytes(long long rows, int in, int out, int dtype) {
    Layer l;
    return layer_sizes(l, rows, in, out, dtype, true) ? forward_plan(l).need : 0;
}

extern "C" __attribute__((visibility("default")))
int sr_layer_gated(const sr_tensor* x, const sr_tensor* weight, const sr_tensor* bias, int act, sr_tensor* y,
                   void* workspace, size_t workspace_bytes, void* stream) {
    return forward(x, weight, bias, act, nullptr, y, true, workspace, workspace_bytes, stream);
}

extern "C" __attribute__((visibility("default")))
size_t sr_layer_gated_grad_workspace_bytes(long long rows, int in, int out, int dtype) {
    Layer l;
    return layer_sizes(l, rows, in, out, dtype, true) ? grad_plan(l, SR_ACT_NONE).need : 0;
}

extern "C" __attribute__((visibility("default")))
int sr_layer_gated_grad(const sr_tensor* x, const sr_tensor* weight, const sr_tensor* bias, int act, const sr_tensor* dy,
                        sr_tensor* dx, sr_tensor* dweight, sr_tensor* dbias,
                        void* workspace, size_t workspace_bytes, void* stream) {
    return gradient(x, weight, bias, act, dy, dx, dweight, dbias, true, workspace, workspace_bytes, stream);
}

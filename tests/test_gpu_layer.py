"""Layers over rows and their gradients through the C ABI against the 64-bit oracle on the same stored values.

Tolerances, u = 2^-24.  Products of the stored values are exact for 16-bit types and rounded once (u) for fp32.  A matrix
instruction adds 16 products (fp32: 2) to a sum; whatever it does inside, each of its partial sums is taken to be off by 2 u of the
sum of magnitudes M, so K products are within steps(K) = (K / 4 + 16) u M, fp32: (2 K + 16) u M; sums split over workgroups only have
fewer steps.  Activations: the exponential's argument is rounded twice and its constant once, 1.733 |z| u, the instruction adds 2 u, sum,
quotient and product one each: (1.75 |z| + 8) u relative; erf is within 4 u of 1, so gelu is within 4 u |z|, its slope adds the exponential's
z^2 / 2: (4 + 2 z^2 exp(-z^2 / 2)) u in all is below 8 u (|z| + 1).  One bound for all of them: a value is within u (1.75 |z| + 8) (|value| + |z| + 1), a
slope the same with |slope| + 1.  Slopes are below 1.13, second derivatives below 0.8: z's own error counts that much.  A rounding to type t is off by
eps_t / 2 of the value, or half of t's smallest step."""
import ctypes
import math

import pytest
import torch

import paper_2303_08999_amd as sr
from oracle import layer_oracle as lo

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SMALLEST = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}


class Guarded:
    """A tensor between two strips of NaN that a call must neither use nor touch."""

    def __init__(self, shape, dtype, shift=0, fill=None):
        numel = math.prod(shape)
        self.raw = torch.full((numel + 1024,), float("nan"), device=DEV, dtype=dtype)
        self.lo, self.hi = 512 + shift, 512 + shift + numel
        self.t = self.raw[self.lo:self.hi].view(shape)
        if fill is not None:
            self.t.copy_(fill)

    def check(self):
        assert self.raw[:self.lo].isnan().all() and self.raw[self.hi:].isnan().all(), "written outside of the tensor"


def half_step(t, v):
    return torch.finfo(DT[t]).eps / 2 * v.abs() + SMALLEST[t] / 2


def steps(t, K):
    return ((2 * K if t == "f32" else K / 4) + 16) * U


def inputs(P, C, O, t, gated, seed, bias=True, residual=False):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device=DEV)
    wide = 2 * O if gated else O
    d = {"x": r(P, C), "w": r(wide, C) / math.sqrt(C), "b": r(wide) / 2 if bias else None, "dy": r(P, O) / 8,
         "res": r(P, O) if residual else None}
    return {k: None if v is None else v.to(DT[t]) for k, v in d.items()}


def wide64(d):
    return {k: None if v is None else v.double() for k, v in d.items()}


def z_error(t, e):
    """z and what it may be off by."""
    C = e["x"].shape[1]
    z = lo.affine(e["x"], e["w"], e["b"])
    M = lo.affine(e["x"].abs(), e["w"].abs(), None if e["b"] is None else e["b"].abs())
    return z, steps(t, C) * M


def act_error(z, v):
    return U * (1.75 * z.abs() + 8) * (v.abs() + z.abs() + 1)


def forward_bound(t, e, kind, gated):
    z, ez = z_error(t, e)
    if gated:
        (g, u), (eg, eu) = z.chunk(2, 1), ez.chunk(2, 1)
        v = lo.act(kind, g)
        want = v * u
        ev = 1.13 * eg + act_error(g, v)
        err = ev * u.abs() + (v.abs() + ev) * eu + 2 * U * want.abs()
    else:
        v = lo.act(kind, z)
        err = 1.13 * ez + (act_error(z, v) if kind else 0)
        want = v
        if e["res"] is not None:
            want = v + e["res"]
            err = err + U * want.abs()
    return want, err + half_step(t, want.abs() + err)


def slope_error(kind, z, ez):
    s = lo.slope(kind, z)
    if kind == lo.NONE:
        return s, torch.zeros_like(z)
    err = 0.8 * ez + U * (1.75 * z.abs() + 8) * (s.abs() + 1)
    if kind == lo.RELU:
        err = torch.where(z.abs() <= ez, torch.ones_like(z), torch.zeros_like(z))
    return s, err


def dz_bound(t, e, kind, gated):
    if not gated and kind == lo.NONE:
        return e["dy"], torch.zeros_like(e["dy"])
    z, ez = z_error(t, e)
    dy = e["dy"]
    if gated:
        (g, u), (eg, eu) = z.chunk(2, 1), ez.chunk(2, 1)
        s, es = slope_error(kind, g, eg)
        v = lo.act(kind, g)
        ev = 1.13 * eg + (act_error(g, v) if kind else 0)
        want = torch.cat([dy * u * s, dy * v], 1)
        err = torch.cat([dy.abs() * (u.abs() * es + eu * (s.abs() + es)), dy.abs() * ev], 1) + 3 * U * want.abs()
    else:
        s, es = slope_error(kind, z, ez)
        want = dy * s
        err = dy.abs() * es + U * want.abs()
    return want, err + half_step(t, want.abs() + err)


def behind_bound(t, e, dz, edz):
    x, w = e["x"], e["w"]
    out = []
    for want, err, mag, K in ((dz @ w, edz @ w.abs(), dz.abs() @ w.abs(), w.shape[0]),
                              (dz.t() @ x, edz.t() @ x.abs(), dz.abs().t() @ x.abs(), x.shape[0]),
                              (dz.sum(0), edz.sum(0), dz.abs().sum(0), x.shape[0])):
        err = err + (2 * K + 16 if want.dim() == 1 else steps(t, K) / U) * U * (mag + err)
        out.append((want, err + half_step(t, want.abs() + err)))
    return out


def compare(what, got, want, bound):
    got = got.double()
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float(((got - want).abs() / bound).max()):.2f} of the bound"


def run_forward(d, t, kind, gated, shift=0):
    P, O = d["dy"].shape
    dev = {k: None if v is None else Guarded(v.shape, v.dtype, shift, v) for k, v in d.items()}
    y = Guarded((P, O), DT[t], shift)
    get = lambda k: dev[k] and dev[k].t
    if gated:
        sr.sr_layer_gated(get("x"), get("w"), get("b"), kind, y.t)
    else:
        sr.sr_layer_linear(get("x"), get("w"), get("b"), kind, get("res"), y.t)
    torch.cuda.synchronize()
    for v in (*dev.values(), y):
        if v is not None:
            v.check()
    return y.t


def run_grad(d, t, kind, gated, shift=0, want=(True, True, True)):
    dev = {k: None if v is None else Guarded(v.shape, v.dtype, shift, v) for k, v in d.items()}
    wide = d["w"].shape[0]
    out = [Guarded(s, DT[t], shift) if on else None for s, on in zip((d["x"].shape, d["w"].shape, (wide,)), want)]
    get = lambda k: dev[k] and dev[k].t
    call = sr.sr_layer_gated_grad if gated else sr.sr_layer_linear_grad
    call(get("x"), get("w"), get("b"), kind, get("dy"), *(o and o.t for o in out))
    torch.cuda.synchronize()
    for v in (*dev.values(), *out):
        if v is not None:
            v.check()
    return [o and o.t for o in out]


def check_forward(P, C, O, t, kind, gated, seed=1, bias=True, residual=False, shift=0, spoil=None):
    d = inputs(P, C, O, t, gated, seed, bias, residual)
    if spoil:
        spoil(d)
    want, bound = forward_bound(t, wide64(d), kind, gated)
    compare("y", run_forward(d, t, kind, gated, shift), want, bound)


def check_grad(P, C, O, t, kind, gated, seed=1, bias=True, shift=0, spoil=None):
    d = inputs(P, C, O, t, gated, seed, bias)
    if spoil:
        spoil(d)
    e = wide64(d)
    bounds = behind_bound(t, e, *dz_bound(t, e, kind, gated))
    got = run_grad(d, t, kind, gated, shift)
    for name, g, (want, bound) in zip(("dx", "dweight", "dbias"), got, bounds):
        compare(name, g, want, bound)
    return d, got


# rows from one to several tiles, features below, at and above what a load, a matrix step and a tile hold
SHAPES = [(1, 1, 1), (1, 8, 8), (1, 2048, 33), (3, 5, 7), (16, 64, 72), (17, 72, 64), (33, 40, 130), (64, 129, 31), (65, 64, 64), (100, 27, 121),
          (127, 136, 40), (128, 64, 128), (129, 128, 129), (200, 1000, 264), (257, 200, 257), (300, 65, 1), (1000, 72, 96), (515, 1536, 520),
          (4099, 64, 72), (90, 4100, 65), (2049, 8, 16)]


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "P%dC%dO%d" % s)
@pytest.mark.parametrize("gated", [False, True], ids=["linear", "gated"])
def test_forward(gated, shape, t):
    kind = (shape[0] + shape[1]) % 5
    check_forward(*shape, t, kind, gated, seed=sum(shape), bias=shape[0] % 2 == 1, residual=not gated and shape[1] % 2 == 0)


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "P%dC%dO%d" % s)
@pytest.mark.parametrize("gated", [False, True], ids=["linear", "gated"])
def test_gradients(gated, shape, t):
    check_grad(*shape, t, (shape[0] + shape[2]) % 5, gated, seed=sum(shape), bias=shape[0] % 2 == 1)


@pytest.mark.parametrize("kind", range(5))
@pytest.mark.parametrize("gated", [False, True], ids=["linear", "gated"])
@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_every_activation(t, gated, kind):
    check_forward(150, 72, 88, t, kind, gated)
    check_forward(20, 72, 88, t, kind, gated)
    check_grad(150, 72, 88, t, kind, gated)


@pytest.mark.parametrize("shift", [1, 4, 7])
@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("gated", [False, True], ids=["linear", "gated"])
def test_addresses_off_16_bytes(gated, t, shift):
    """The header promises any address that is aligned to an element."""
    for P in (9, 140, 300):
        check_forward(P, 64, 72, t, lo.GELU, gated, shift=shift, residual=not gated)
        check_grad(P, 64, 72, t, lo.SILU, gated, shift=shift)


@pytest.mark.parametrize("shape,t", [((16400, 520, 264), "bf16"), ((8200, 264, 1030), "f16"), ((3000, 1032, 776), "f32"), ((70000, 40, 24), "bf16"),
                                     ((66000, 64, 72), "f32"), ((2100, 2056, 2568), "f16")], ids=str)
@pytest.mark.parametrize("gated", [False, True], ids=["linear", "gated"])
def test_large_tiles_and_long_sums(gated, shape, t):
    check_forward(*shape, t, lo.SILU, gated, residual=not gated)
    check_grad(*shape, t, lo.GELU if not gated else lo.SILU, gated)
    if not gated:
        check_grad(*shape, t, lo.NONE, gated)


# a small weight under many rows: every number of 64-byte steps of a row, rows that are no pieces of 16 bytes, outputs that are no fours
THIN = [(4096, 1, 1), (4097, 27, 121), (5003, 64, 72), (4100, 31, 33), (9999, 128, 4), (4111, 8, 130), (6000, 33, 64), (4127, 100, 5), (4128, 72, 64), (20001, 16, 31),
        (4099, 127, 63), (131077, 12, 20), (4160, 72, 40), (4097, 128, 128), (4100, 80, 8), (5000, 8, 248), (33333, 64, 64), (4223, 40, 120), (4100, 24, 300), (4500, 65, 200)]


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", THIN, ids=lambda s: "P%dC%dO%d" % s)
@pytest.mark.parametrize("gated", [False, True], ids=["linear", "gated"])
def test_many_rows_and_a_small_weight(gated, shape, t):
    P, C, O = shape
    for kind, shift in ((lo.NONE, 0), (P % 4 + 1, P % 3)):
        check_forward(P, C, O, t, kind, gated, bias=kind > 0, residual=not gated, shift=shift)
        check_grad(P, C, O, t, kind, gated, bias=kind > 0, shift=shift)


@pytest.mark.parametrize("gated", [False, True], ids=["linear", "gated"])
def test_a_row_of_nan_among_many(gated):
    for C, O in ((27, 121), (64, 72), (100, 5)):
        d = inputs(4200, C, O, "f32", gated, 5)
        clean = run_forward(d, "f32", lo.SILU, gated).clone()
        for row in (0, 777, 4199):
            d["x"][row] = float("nan")
        y = run_forward(d, "f32", lo.SILU, gated)
        rows = torch.ones(4200, dtype=torch.bool, device=DEV)
        rows[0] = rows[777] = rows[4199] = False
        assert torch.equal(y[rows], clean[rows]) and y[~rows].isnan().all()


def test_what_is_not_asked_for_is_not_written_and_changes_nothing():
    for gated in (False, True):
        for shape in ((70, 40, 24), (5000, 72, 64), (7, 64, 9)):
            d = inputs(*shape, "f16", gated, 3)
            every = run_grad(d, "f16", lo.SILU, gated)
            for want in ((True, False, False), (False, True, False), (False, False, True), (True, False, True), (True, True, False)):
                for a, b in zip(run_grad(d, "f16", lo.SILU, gated, want=want), every):
                    assert a is None or torch.equal(a, b)


def test_no_rows():
    for gated in (False, True):
        d = inputs(0, 40, 24, "bf16", gated, 1)
        assert run_forward(d, "bf16", lo.GELU, gated).shape == (0, 24)
        dx, dw, db = run_grad(d, "bf16", lo.GELU, gated)
        assert dx.shape == (0, 40) and (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("gated", [False, True], ids=["linear", "gated"])
@pytest.mark.parametrize("P,C", [(9, 100), (200, 100), (200, 128), (700, 2000)])
def test_infinities_and_nan_stay_in_their_rows(gated, P, C):
    """A row's NaN reaches that row of y alone; of a padded K or a clamped row nothing gets anywhere."""
    for t in ("f32", "bf16"):
        d = inputs(P, C, 70, t, gated, 5)
        clean = run_forward(d, t, lo.SILU, gated).clone()
        d["x"][3, C - 1] = float("nan")
        d["x"][P - 1, 0] = float("inf")
        y = run_forward(d, t, lo.SILU, gated)
        rows = torch.ones(P, dtype=torch.bool, device=DEV)
        rows[3] = rows[P - 1] = False
        assert torch.equal(y[rows], clean[rows]) and y[3].isnan().all()
        d["w"][5] = float("nan")                                     # ... and a weight's row that column
        y = run_forward(d, t, lo.SILU, gated)
        cols = torch.arange(70, device=DEV) != 5
        assert torch.equal(y[rows][:, cols], clean[rows][:, cols]) and y[:, 5].isnan().all()


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
def test_large_and_small_values(t):
    """Saturated activations, and gradients as small as the type holds."""
    def spoil(d):
        d["x"] *= 30
    for kind in range(5):
        check_forward(90, 64, 40, t, kind, False, spoil=spoil)
        check_grad(90, 64, 40, t, kind, False, spoil=spoil)

    def faint(d):
        d["dy"] *= 2.0 ** -16 if t == "f16" else 2.0 ** -80
    check_grad(90, 64, 40, t, lo.GELU, False, spoil=faint)
    check_grad(90, 64, 40, t, lo.SILU, True, spoil=faint)


@pytest.mark.parametrize("shape", [(8200, 264, 1032), (16400, 2048, 4096)], ids=str)
@pytest.mark.parametrize("t", ["f16", "bf16"])
def test_faint_gradients_of_large_layers(t, shape):
    """fp16 gradients that are subnormal numbers, in the products and in the sums beside them."""
    def faint(d):
        d["dy"] *= 2.0 ** -16 if t == "f16" else 2.0 ** -100
    check_grad(*shape, t, lo.NONE, False, spoil=faint)


@pytest.mark.parametrize("shape,parts", [((500, 64, 72), 2), ((33, 520, 40), 2), ((5000, 64, 72), 2), ((4100, 24, 16), 2), ((900, 1000, 1030), 2), ((3000, 1032, 776), 1),
                                         ((9000, 256, 512), 1)], ids=str)
@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("gated", [False, True], ids=["linear", "gated"])
def test_errors_of_gradients_in_norm(gated, t, shape, parts):
    """In norm: the error of an exact result's rounding, and, where z's gradient goes through the type, as much again in random directions (1.41 in all; the
    bias's gradient is summed before).  Where it goes in two parts, nothing is added.  A fifth of each is left for what a few hundred
    values scatter."""
    d = inputs(*shape, t, gated, 31)
    e = wide64(d)
    dz = (lo.gated_dz if gated else lo.linear_dz)(e["x"], e["w"], e["b"], lo.GELU, e["dy"])
    if 2 * shape[0] * shape[1] * d["w"].shape[0] > 2e9:
        parts = 1
    for name, got, want in zip(("dx", "dweight", "dbias"), run_grad(d, t, lo.GELU, gated), lo.behind_dz(e["x"], e["w"], dz)):
        rounding = (want.to(DT[t]).double() - want).norm()
        assert (got.double() - want).norm() <= (1.2 if parts == 2 or name == "dbias" else 1.7) * rounding, name


def test_runs_give_the_same_bits():
    for shape in ((3000, 72, 64), (40, 520, 33), (9000, 256, 256)):
        for gated in (False, True):
            d = inputs(*shape, "bf16", gated, 8)
            a, b = run_forward(d, "bf16", lo.GELU, gated), run_forward(d, "bf16", lo.GELU, gated)
            assert torch.equal(a, b)
            for x, y in zip(run_grad(d, "bf16", lo.GELU, gated), run_grad(d, "bf16", lo.GELU, gated)):
                assert torch.equal(x, y)


def test_images_as_rows():
    """[N][H][W][C] is what its rows are."""
    d = inputs(2 * 5 * 7, 24, 40, "f16", False, 4)
    y, y4 = torch.empty(70, 40, device=DEV, dtype=torch.float16), torch.empty(2, 5, 7, 40, device=DEV, dtype=torch.float16)
    sr.sr_layer_linear(d["x"], d["w"], d["b"], lo.RELU, None, y)
    sr.sr_layer_linear(d["x"].view(2, 5, 7, 24), d["w"], d["b"], lo.RELU, None, y4)
    assert torch.equal(y.view(2, 5, 7, 40), y4)


def test_other_streams_and_captured_graphs():
    """On a stream of the caller's; captured with workspaces of their own and replayed with other work in between."""
    P, C, O = 3000, 136, 72
    d = inputs(P, C, O, "bf16", True, 6)
    want = [run_forward(d, "bf16", lo.SILU, True)] + run_grad(d, "bf16", lo.SILU, True)
    outs = [torch.zeros_like(v) for v in want]
    ws = torch.empty(sr.sr_layer_gated_grad_workspace_bytes(P, C, O, torch.bfloat16), device=DEV, dtype=torch.uint8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    sr.sr_layer_gated(d["x"], d["w"], d["b"], lo.SILU, outs[0], stream=side)
    sr.sr_layer_gated_grad(d["x"], d["w"], d["b"], lo.SILU, d["dy"], *outs[1:], workspace=ws, stream=side.cuda_stream)
    side.synchronize()
    for a, b in zip(outs, want):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sr.sr_layer_gated(d["x"], d["w"], d["b"], lo.SILU, outs[0])
        sr.sr_layer_gated_grad(d["x"], d["w"], d["b"], lo.SILU, d["dy"], *outs[1:], workspace=ws)
    for i in range(4):
        for o in outs:
            o.zero_()
        ws.fill_(255)                                                # what is there before a call is meaningless
        d["x"].mul_(1.0 if i % 2 else -1.0)
        graph.replay()
        torch.cuda.synchronize()
        now = [run_forward(d, "bf16", lo.SILU, True)] + run_grad(d, "bf16", lo.SILU, True)
        for a, b in zip(outs, now):
            assert torch.equal(a, b), f"replay {i}"


@pytest.mark.parametrize("P,C,O", [((1 << 25) + 77, 128, 8), ((1 << 23) + 33, 520, 24)], ids=["small_weight", "tiles"])
def test_more_elements_than_32_bits_count(P, C, O):
    """x has more than 2^32 elements; all rows but a few, some of them the last, are zeros."""
    assert P * C > 1 << 32
    g = torch.Generator(device=DEV).manual_seed(3)
    at = torch.tensor([0, 1, 4095, P // 2, P - 130, P - 2, P - 1], device=DEV)
    x = torch.zeros((P, C), device=DEV, dtype=torch.bfloat16)
    x[at] = torch.randn((7, C), generator=g, device=DEV).bfloat16()
    w, b = (torch.randn((O, C), generator=g, device=DEV) / 16).bfloat16(), torch.randn(O, generator=g, device=DEV).bfloat16()
    y = torch.empty((P, O), device=DEV, dtype=torch.bfloat16)
    sr.sr_layer_linear(x, w, b, lo.NONE, None, y)
    few = {"x": x[at], "w": w, "b": b, "dy": torch.zeros((7, O), device=DEV), "res": None}
    want, bound = forward_bound("bf16", wide64(few), lo.NONE, False)
    compare("y", y[at], want, bound)
    assert torch.equal(y[2:4095], b.expand(4093, O)) and torch.equal(y[P - 129:P - 2], b.expand(127, O))
    dy = torch.zeros((P, O), device=DEV, dtype=torch.bfloat16)
    dy[at] = torch.randn((7, O), generator=g, device=DEV).bfloat16()
    dx, dw, db = torch.full_like(x, 3.0), torch.empty_like(w), torch.empty_like(b)
    sr.sr_layer_linear_grad(x, w, b, lo.NONE, dy, dx, dw, db)
    few["dy"] = dy[at]
    e = wide64(few)
    for name, got, (want, bound) in zip(("dx", "dweight", "dbias"), (dx[at], dw, db), behind_bound("bf16", e, e["dy"], torch.zeros_like(e["dy"]))):
        compare(name, got, want, bound)
    assert not dx[2:4095].any() and not dx[P - 129:P - 2].any() and int((dx != 0).any(1).sum()) == 7


# features that are no 16-byte pieces, in products long enough for copies that are
@pytest.mark.parametrize("shape,t", [((2500, 1021, 2053), "bf16"), ((3000, 1754, 1183), "f16"), ((1500, 777, 1030), "f32"), ((9000, 1032, 777), "bf16"), ((8200, 2047, 2049), "f32")], ids=str)
@pytest.mark.parametrize("gated", [False, True], ids=["linear", "gated"])
def test_copies_on_whole_pieces(gated, shape, t):
    P, C, O = shape
    if C % 8 and t != "f32":                                      # which the tile kernels read as it is
        need = sr.sr_layer_gated_workspace_bytes if gated else sr.sr_layer_linear_workspace_bytes
        assert need(P, C, O, DT[t]) >= P * C * DT[t].itemsize
    for kind, shift in ((lo.NONE, 0), (lo.SILU, 1)):
        check_forward(*shape, t, kind, gated, residual=not gated, shift=shift)
        check_grad(*shape, t, kind, gated, shift=shift)


@pytest.mark.parametrize("shape,t", [((66000, 136, 200), "bf16"), ((140000, 27, 121), "f16"), ((1200001, 17, 9), "bf16"), ((90000, 520, 264), "f32")], ids=str)
@pytest.mark.parametrize("gated", [False, True], ids=["linear", "gated"])
def test_bias_gradients_of_very_many_rows(gated, shape, t):
    """The sums that every row of tiles leaves are so many that they are added up in two steps."""
    check_grad(*shape, t, lo.GELU, gated)


# so many outputs that the kernel which holds the weight takes them: k that ends inside a step, widths that are no pieces, several launches
HELD = [(65600, 64, 410), (131100, 40, 200), (131075, 136, 201), (70001, 250, 400), (262200, 264, 120), (140000, 8, 264), (110000, 72, 1030), (300000, 512, 100), (56000, 512, 500), (70000, 130, 391),
        (211111, 100, 255), (430001, 120, 62), (900000, 24, 40), (351576, 27, 121), (131080, 59, 300)]


@pytest.mark.parametrize("shape", HELD, ids=lambda s: "P%dC%dO%d" % s)
@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("gated", [False, True], ids=["linear", "gated"])
def test_very_many_rows(gated, shape, t):
    kind = shape[0] % 4 + 1
    check_forward(*shape, t, kind, gated)
    check_forward(*shape, t, lo.NONE, gated, bias=False, residual=not gated, shift=(2, 8, 1)[shape[1] % 3])
    check_grad(*shape, t, kind, gated, shift=(0, 3, 2)[shape[1] % 3])
    check_grad(*shape, t, lo.NONE, gated)


@pytest.mark.parametrize("gated", [False, True], ids=["linear", "gated"])
@pytest.mark.parametrize("t,C", [("bf16", 40), ("bf16", 72), ("bf16", 132), ("bf16", 264), ("f32", 40), ("f32", 59), ("f32", 101)])
def test_rows_of_nan_among_very_many(gated, t, C):
    P, O = 131080, 256 if gated else 264
    d = inputs(P, C, O, t, gated, 5)
    clean = run_forward(d, t, lo.SILU, gated).clone()
    at = torch.tensor([0, 63, 777, 65536, P - 2], device=DEV)
    d["x"][at] = float("nan")
    y = run_forward(d, t, lo.SILU, gated)
    rows = torch.ones(P, dtype=torch.bool, device=DEV)
    rows[at] = False
    assert torch.equal(y[rows], clean[rows]) and y[~rows].isnan().all()
    d["x"].zero_()
    clean = run_grad(d, t, lo.NONE, gated, want=(True, False, False))[0].clone()
    d["dy"][at] = float("nan")
    dx = run_grad(d, t, lo.NONE, gated, want=(True, False, False))[0]
    assert torch.equal(dx[rows], clean[rows]) and dx[~rows].isnan().all()


# one of each way that a call is made: few rows, tiles, split sums, small weights, one pass, dz in two parts or one, copies
WAYS = [(7, 2048, 33), (64, 129, 31), (300, 64, 72), (1000, 1000, 264), (5000, 64, 72), (5000, 31, 33), (2500, 1021, 1030), (90, 4100, 65), (9000, 256, 512), (70000, 136, 40), (66000, 72, 520)]


@pytest.mark.parametrize("shape", WAYS, ids=lambda s: "P%dC%dO%d" % s)
@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("gated", [False, True], ids=["linear", "gated"])
def test_a_workspace_of_the_size_asked_for_and_no_more(gated, t, shape):
    """What is in it before does not matter, and what is around it stays."""
    P, C, O = shape
    d = inputs(*shape, t, gated, 12)
    y, grads = run_forward(d, t, lo.SILU, gated), run_grad(d, t, lo.SILU, gated)
    out = [torch.empty_like(v) for v in (y, *grads)]
    if gated:
        sizes = sr.sr_layer_gated_workspace_bytes(P, C, O, DT[t]), sr.sr_layer_gated_grad_workspace_bytes(P, C, O, DT[t])
    else:
        sizes = sr.sr_layer_linear_workspace_bytes(P, C, O, DT[t]), sr.sr_layer_linear_grad_workspace_bytes(P, C, O, DT[t], lo.SILU)
    room = [torch.full((n + 8192,), 255, device=DEV, dtype=torch.uint8) for n in sizes]
    ws = [r[4096:4096 + n] if n else None for r, n in zip(room, sizes)]
    if gated:
        sr.sr_layer_gated(d["x"], d["w"], d["b"], lo.SILU, out[0], workspace=ws[0])
        sr.sr_layer_gated_grad(d["x"], d["w"], d["b"], lo.SILU, d["dy"], *out[1:], workspace=ws[1])
    else:
        sr.sr_layer_linear(d["x"], d["w"], d["b"], lo.SILU, None, out[0], workspace=ws[0])
        sr.sr_layer_linear_grad(d["x"], d["w"], d["b"], lo.SILU, d["dy"], *out[1:], workspace=ws[1])
    torch.cuda.synchronize()
    for a, b in zip(out, (y, *grads)):
        assert torch.equal(a, b)
    for r, n in zip(room, sizes):
        assert (r[:4096] == 255).all() and (r[4096 + n:] == 255).all()


@pytest.mark.parametrize("shape", WAYS, ids=lambda s: "P%dC%dO%d" % s)
def test_every_way_at_once_on_two_streams_and_replayed(shape):
    """Two streams with a workspace each, at the same time; the same calls from a graph, with eager ones between its replays."""
    P, C, O = shape
    sets = [inputs(*shape, "bf16", gated, 40 + gated) for gated in (False, True)]
    want = [[run_forward(d, "bf16", lo.GELU, gated), *run_grad(d, "bf16", lo.GELU, gated)] for gated, d in enumerate(sets)]
    outs = [[torch.empty_like(v) for v in w] for w in want]
    streams = [torch.cuda.Stream() for _ in sets]
    grad_bytes = (sr.sr_layer_linear_grad_workspace_bytes(P, C, O, torch.bfloat16, lo.GELU), sr.sr_layer_gated_grad_workspace_bytes(P, C, O, torch.bfloat16))
    forward_bytes = (sr.sr_layer_linear_workspace_bytes(P, C, O, torch.bfloat16), sr.sr_layer_gated_workspace_bytes(P, C, O, torch.bfloat16))
    ws = [torch.empty(max(a, b, 16), device=DEV, dtype=torch.uint8) for a, b in zip(grad_bytes, forward_bytes)]

    def both(streams):
        for gated, d in enumerate(sets):
            o = outs[gated]
            if gated:
                sr.sr_layer_gated(d["x"], d["w"], d["b"], lo.GELU, o[0], workspace=ws[1], stream=streams[1])
                sr.sr_layer_gated_grad(d["x"], d["w"], d["b"], lo.GELU, d["dy"], *o[1:], workspace=ws[1], stream=streams[1])
            else:
                sr.sr_layer_linear(d["x"], d["w"], d["b"], lo.GELU, None, o[0], workspace=ws[0], stream=streams[0])
                sr.sr_layer_linear_grad(d["x"], d["w"], d["b"], lo.GELU, d["dy"], *o[1:], workspace=ws[0], stream=streams[0])

    def same(what):
        torch.cuda.synchronize()
        for w, o in zip(want, outs):
            for name, a, b in zip(("y", "dx", "dweight", "dbias"), w, o):
                assert torch.equal(a, b), (what, name)
                b.zero_()
        torch.cuda.synchronize()

    torch.cuda.synchronize()
    for i in range(3):
        both(streams)
    same("two streams")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both((None, None))
    for i in range(3):
        for w in ws:
            w.fill_(255)
        graph.replay()
        same(f"replay {i}")
        both(streams)
        same("between replays")


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("P", [7, 300, 5000, 40000])
@pytest.mark.parametrize("gated", [False, True], ids=["linear", "gated"])
def test_gradients_beyond_the_type_are_infinite(gated, P, t):
    """z's gradient may leave the type between two products: an infinity then, whose row and column it stays in, and no NaN where its
    product with a weight or a feature is none."""
    C, O, row, n = 64, 72, P - 2, 5
    d = inputs(P, C, O, t, gated, 17)
    d["b"].zero_()
    d["w"][:, 0] = 0
    d["w"][n::O, 0] = 1
    d["x"][row] = 2.0 ** -9
    d["x"][row, 0] = 1.5
    big = torch.finfo(DT[t]).max
    d["dy"][row, n] = big                                        # times gelu'(1.5) = 1.128, and for the gate another 1.5
    dx, dw, db = run_grad(d, t, lo.GELU, gated)
    other = torch.arange(P, device=DEV) != row
    assert dx[other].isfinite().all()
    if gated:                                                    # du = dy gelu(1.5) is infinite as well: where the signs of the two weights differ, NaN
        a, b = d["w"][n].float(), d["w"][O + n].float()
        sure = a * b > 0
        assert (dx[row][sure].float() == ((a + b) * math.inf)[sure]).all()
    else:
        a = d["w"][n].float()
        assert (dx[row][a != 0].float() == (a * math.inf)[a != 0]).all()
    rows = torch.zeros(dw.shape[0], dtype=torch.bool, device=DEV)
    rows[n::O] = True
    assert dw[~rows].isfinite().all() and (dw[rows].float() == math.inf).all()
    assert db[~rows].isfinite().all() and (db[rows].float() == math.inf).all()


@pytest.mark.parametrize("P", [(1 << 30) + 77, (1 << 31) - 300])
def test_more_rows_than_a_launch_of_small_tiles_has(P):
    at = torch.tensor([0, 1, 4095, P // 2, P - 130, P - 2, P - 1], device=DEV)
    g = torch.Generator(device=DEV).manual_seed(3)
    x = torch.zeros((P, 1), device=DEV, dtype=torch.bfloat16)
    x[at] = torch.randn((7, 1), generator=g, device=DEV).bfloat16()
    w, b = torch.full((1, 1), 0.75, device=DEV).bfloat16(), torch.full((1,), 0.5, device=DEV).bfloat16()
    dy = torch.zeros((P, 1), device=DEV, dtype=torch.bfloat16)
    dy[at] = torch.randn((7, 1), generator=g, device=DEV).bfloat16()
    e = wide64({"x": x[at], "w": w, "b": b, "dy": dy[at], "res": None})
    y = torch.empty_like(x)
    sr.sr_layer_linear(x, w, b, lo.SILU, None, y)
    want, bound = forward_bound("bf16", e, lo.SILU, False)
    compare("y", y[at], want, bound)
    dx, dw, db = torch.full_like(x, 3.0), torch.empty_like(w), torch.empty_like(b)
    sr.sr_layer_linear_grad(x, w, b, lo.SILU, dy, dx, dw, db)
    for name, got, (want, bound) in zip(("dx", "dweight", "dbias"), (dx[at], dw, db), behind_bound("bf16", e, *dz_bound("bf16", e, lo.SILU, False))):
        compare(name, got, want, bound)
    assert int((dx != 0).sum()) == 7


def test_the_bounds_tell_mistakes_apart():
    """Each of these mistakes, made in the oracle, leaves the bound that the kernels keep."""
    d = inputs(300, 72, 88, "bf16", False, 21, residual=True)
    y = run_forward(d, "bf16", lo.GELU, False).double()
    e = wide64(d)
    want, bound = forward_bound("bf16", e, lo.GELU, False)
    z = lo.affine(e["x"], e["w"], e["b"])
    mistakes = {"no bias": lo.act(lo.GELU, z - e["b"]) + e["res"], "residual inside": lo.act(lo.GELU, z + e["res"]), "no residual": lo.act(lo.GELU, z),
                "silu": lo.act(lo.SILU, z) + e["res"],
                "a k less": lo.act(lo.GELU, z - e["x"][:, -1:] * e["w"][:, -1]) + e["res"], "rows shifted": want.roll(1, 0), "columns shifted": want.roll(1, 1)}
    assert ((y - want).abs() <= bound).all()
    for name, wrong in mistakes.items():
        assert not ((y - wrong).abs() <= bound).all(), name
    d = inputs(300, 72, 88, "bf16", True, 22)
    e = wide64(d)
    dx, dw, db = (v.double() for v in run_grad(d, "bf16", lo.SILU, True))
    dz, edz = dz_bound("bf16", e, lo.SILU, True)
    bounds = [b for _, b in behind_bound("bf16", e, dz, edz)]
    g, u = lo.affine(e["x"], e["w"], e["b"]).chunk(2, 1)
    dg, du = dz.chunk(2, 1)
    mistakes = {"halves exchanged": torch.cat([du, dg], 1), "value for slope": torch.cat([e["dy"] * u * lo.act(lo.SILU, g), du], 1),
                "no product": torch.cat([e["dy"] * lo.slope(lo.SILU, g), du], 1), "a row less": torch.cat([dz[:-1], torch.zeros_like(dz[:1])])}
    for name, wrong in mistakes.items():
        wx, ww, wb = lo.behind_dz(e["x"], e["w"], wrong)
        assert not (((dx - wx).abs() <= bounds[0]).all() and ((dw - ww).abs() <= bounds[1]).all() and ((db - wb).abs() <= bounds[2]).all()), name


# fp32 by each kernel: few rows, fp32 instructions, tiles of three bfloat16 parts on 16-byte pieces and off them, a small weight, a weight that is held
RANGE = [(40, 512, 64), (200, 64, 72), (2048, 512, 2048), (4096, 1024, 4096), (3000, 1021, 1030), (4200, 64, 72), (131080, 40, 264), (131080, 59, 300)]


@pytest.mark.parametrize("shape", RANGE, ids=lambda s: "P%dC%dO%d" % s)
def test_the_largest_fp32_values(shape):
    """Numbers up to the largest there is times small ones are finite.  A row has one value, so an element is one product: the one rounding of an fp32
    instruction, or six products of parts, each added with 2 u of the sum, and 2^-24 for the parts left out: 14 u in all.  The gate's two
    products count both, and one rounding."""
    P, C, O = shape
    g = torch.Generator(device=DEV).manual_seed(9)
    sign = lambda *s: torch.randint(0, 2, s, generator=g, device=DEV) * 2 - 1
    big = lambda n: (torch.randint(0x7f7f8000, 0x7f800000, (n,), generator=g, device=DEV, dtype=torch.int32).view(torch.float32) * sign(n)).float()
    part = lambda *s: (torch.rand(s, generator=g, device=DEV) / 4 + 0.25) * sign(*s)
    rows, k = torch.arange(P, device=DEV), torch.arange(P, device=DEV) % C
    x, w = torch.zeros(P, C, device=DEV), part(O, C)
    x[rows, k] = big(P)
    x[0, 0], x[P - 1, k[P - 1]] = torch.finfo(torch.float32).max, torch.finfo(torch.float32).min
    y = torch.empty(P, O, device=DEV)
    sr.sr_layer_linear(x, w, None, lo.NONE, None, y)
    want = x[rows, k].double()[:, None] * w.double().t()[k]
    compare("y", y, want, 14 * U * want.abs())
    both = torch.cat([w * 2.0 ** -60, part(O, C) * 2.0 ** -100])
    sr.sr_layer_gated(x, both, None, lo.NONE, y)
    want = want * 2.0 ** -60 * (x[rows, k].double()[:, None] * both[O:].double().t()[k])
    compare("gated", y, want, 30 * U * want.abs())
    n = min(P, O)
    dy, x = torch.zeros(P, O, device=DEV), part(P, C)
    dy[rows[:n], rows[:n]] = big(n)
    dx, dw, db = torch.empty(P, C, device=DEV), torch.empty(O, C, device=DEV), torch.empty(O, device=DEV)
    sr.sr_layer_linear_grad(x, w, None, lo.NONE, dy, dx, dw, db)
    d = dy[rows[:n], rows[:n]]
    for name, got, other in (("dx", dx, w), ("dweight", dw, x)):
        want = d.double()[:, None] * other[:n].double()
        compare(name, got[:n], want, 14 * U * want.abs())
        assert not got[n:].any()
    assert torch.equal(db[:n], d) and not db[n:].any()


@pytest.mark.parametrize("shape", RANGE, ids=lambda s: "P%dC%dO%d" % s)
def test_the_smallest_fp32_values(shape):
    """Numbers down to the smallest there is times large ones: 14 u as above, and half of bfloat16's smallest number, 2^-134, of the other factor."""
    P, C, O = shape
    g = torch.Generator(device=DEV).manual_seed(10)
    rows, k = torch.arange(P, device=DEV), torch.arange(P, device=DEV) % C
    part = lambda *s: torch.rand(s, generator=g, device=DEV) + 1
    small = (part(P).double() * 2.0 ** -(100 + rows % 50).double()).float()
    assert float(small.min()) < 2.0 ** -(97 + min(P, 50)) and float(small.max()) > 2.0 ** -100
    x, w, y = torch.zeros(P, C, device=DEV), part(O, C) * 2.0 ** 90, torch.empty(P, O, device=DEV)
    x[rows, k] = small
    sr.sr_layer_linear(x, w, None, lo.NONE, None, y)
    other = w.double().t()[k]
    want = small.double()[:, None] * other
    compare("y", y, want, 14 * U * want.abs() + 2.0 ** -134 * other)
    n = min(P, O)
    dy, x = torch.zeros(P, O, device=DEV), part(P, C) * 2.0 ** 90
    dy[rows[:n], rows[:n]] = small[:n]
    dx, dw, db = torch.empty(P, C, device=DEV), torch.empty(O, C, device=DEV), torch.empty(O, device=DEV)
    sr.sr_layer_linear_grad(x, w, None, lo.NONE, dy, dx, dw, db)
    for name, got, other in (("dx", dx, w), ("dweight", dw, x)):
        want = small[:n].double()[:, None] * other[:n].double()
        compare(name, got[:n], want, 14 * U * want.abs() + 2.0 ** -134 * other[:n].double())
        assert not got[n:].any()
    assert torch.equal(db[:n], small[:n]) and not db[n:].any()


# products of which z's is split, and z of few rows
@pytest.mark.parametrize("shape", [(64, 4096, 4096), (256, 4096, 4096), (512, 4096, 1024), (33, 4104, 8200), (250, 4099, 2052)], ids=str)
@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("gated", [False, True], ids=["linear", "gated"])
def test_bias_gradients_of_few_rows_are_summed_before_their_rounding(gated, t, shape):
    """Where z's gradient is rounded once, the bias's gradient is the exact sum of what it was before, rounded: the error in norm of that rounding,
    and a fifth for scatter."""
    d = inputs(*shape, t, gated, 33)
    assert 2 * shape[0] * shape[1] * d["w"].shape[0] > 2e9
    e = wide64(d)
    dz = (lo.gated_dz if gated else lo.linear_dz)(e["x"], e["w"], e["b"], lo.GELU, e["dy"])
    want = dz.sum(0)
    every = run_grad(d, t, lo.GELU, gated)
    rounding = (want.to(DT[t]).double() - want).norm()
    assert (every[2].double() - want).norm() <= 1.2 * rounding
    for name, got, exact in zip(("dx", "dweight"), every, lo.behind_dz(e["x"], e["w"], dz)):
        assert (got.double() - exact).norm() <= 1.7 * (exact.to(DT[t]).double() - exact).norm(), name
    for ask in ((True, False, False), (False, True, False), (False, False, True)):
        for a, b in zip(run_grad(d, t, lo.GELU, gated, want=ask), every):
            assert a is None or torch.equal(a, b)


@pytest.mark.parametrize("shape", [(64, 4096, 4096), (250, 4099, 2052)], ids=str)
def test_the_workspace_of_few_rows_and_its_replays(shape):
    for gated in (False, True):
        test_a_workspace_of_the_size_asked_for_and_no_more(gated, "bf16", shape)
    test_every_way_at_once_on_two_streams_and_replayed(shape)


class KernelNode(ctypes.Structure):
    _fields_ = [("block", ctypes.c_uint * 3), ("extra", ctypes.c_void_p), ("func", ctypes.c_void_p), ("grid", ctypes.c_uint * 3), ("args", ctypes.c_void_p),
                ("shared", ctypes.c_uint)]


def launches(call):
    """The kernels that a call is made of: the nodes of its graph, as it launches them."""
    hip = ctypes.CDLL("libamdhip64.so")
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()
    count = ctypes.c_size_t()
    assert hip.hipGraphGetNodes(ctypes.c_void_p(graph.raw_cuda_graph()), None, ctypes.byref(count)) == 0
    nodes, kernels = (ctypes.c_void_p * count.value)(), (KernelNode * count.value)()
    assert hip.hipGraphGetNodes(ctypes.c_void_p(graph.raw_cuda_graph()), nodes, ctypes.byref(count)) == 0
    for node, kernel in zip(nodes, kernels):
        assert hip.hipGraphKernelNodeGetParams(ctypes.c_void_p(node), ctypes.byref(kernel)) == 0
    return list(kernels)


def test_a_residual_does_not_multiply_the_launches():
    """The kernel that holds the weight reads the rows again in each launch: there are four at most, with a residual as well."""
    shape = (104000, 256, 2048)
    for t in ("f16", "bf16"):
        for residual in (False, True):
            d = inputs(*shape, t, False, 19, residual=residual)
            y = torch.empty(shape[0], shape[2], device=DEV, dtype=DT[t])
            assert 1 <= len(launches(lambda: sr.sr_layer_linear(d["x"], d["w"], d["b"], lo.GELU, d["res"], y))) <= 4
            rows = torch.arange(0, shape[0], 37, device=DEV)
            some = {k: v if v is None or v.shape[0] != shape[0] else v[rows] for k, v in d.items()}
            compare("y", y[rows], *forward_bound(t, wide64(some), lo.GELU, False))


@pytest.mark.parametrize("C,O,t,small", [(64, 72, "bf16", True), (48, 96, "f16", True), (32, 120, "bf16", True), (96, 64, "f16", True), (16, 64, "f32", True), (12, 48, "f32", True), (64, 64, "bf16", True),
                                         (32, 128, "bf16", False), (128, 64, "f16", False), (48, 48, "f32", False), (64, 200, "bf16", False)], ids=str)
def test_gated_blocks_of_many_rows_go_to_the_kernel_for_a_small_weight(C, O, t, small):
    """... where its LDS has room for the weight and one output: what is asked for is what is launched.  It is the only one of a forward call
    whose LDS is given at the launch."""
    for P in (4100, 20011):
        d = inputs(P, C, O, t, True, 23)
        y = torch.empty(P, O, device=DEV, dtype=DT[t])
        kernels = launches(lambda: sr.sr_layer_gated(d["x"], d["w"], d["b"], lo.SILU, y))
        assert all((k.shared > 0) == small for k in kernels) and (len(kernels) == 1 or not small)
        check_forward(P, C, O, t, lo.SILU, True, shift=P % 2)


def tail_bounds(z):
    """gelu and its slope as the kernels' formula has them, in 64 bits, and what fp32 may be off of that.  erfc(x) = P(t) exp(-x^2), t = 1 / (1 + p x),
    x = |z| / sqrt 2, P = a1 t + ... + a5 t^5 by Abramowitz and Stegun 7.1.26.  t: the constant, the sum and two for the reciprocal, 4 u; P: each of five
    steps rounds once, the constants and t's error to the fifth power come in, 5 + 1 + 20 = 26 u of the sum of magnitudes S.  exp: its argument is rounded three times, 3 u of
    z^2 / 2, the instruction 2 u.  Products with it and z three more.  Where z > 0, 1 - P rounds once more."""
    a = (0.254829592, -0.284496736, 1.421413741, -1.453152027, 1.061405429)
    t, d = 1 / (1 + 0.3275911 * math.sqrt(0.5) * z.abs()), torch.exp(-z * z / 2)
    P = sum(c * t ** (i + 1) for i, c in enumerate(a))
    S = sum(abs(c) * t ** (i + 1) for i, c in enumerate(a))
    q = P * d / 2
    cdf = torch.where(z < 0, q, 1 - q)
    e = S * d / 2 * (26 + 1.5 * z * z + 4) * U + torch.where(z < 0, torch.zeros_like(z), 2 * U * cdf)
    bell = z.abs() * d / math.sqrt(2 * math.pi)
    slope = cdf + torch.sign(z) * bell
    return (z * cdf, z.abs() * e + U * (z * cdf).abs()), (slope, e + bell * (1.5 * z * z + 6) * U + 2 * U * slope.abs())


@pytest.mark.parametrize("P", [37, 2000, 5000], ids=["few rows", "tiles", "small weight"])
def test_activations_in_their_tails(P):
    """By themselves, z being a feature times one: gelu as its formula, and that within 0.75e-7 |z|; silu and sigmoid within (1.75 |z| + 8) u of themselves."""
    C = O = 8
    z = torch.linspace(-12, 12, P * C, device=DEV).view(P, C)
    w, y, dx = torch.eye(C, device=DEV), torch.empty(P, C, device=DEV), torch.empty(P, C, device=DEV)
    v = z.double()
    (want, bound), (want_slope, slope_bound) = tail_bounds(v)
    assert ((want - lo.act(lo.GELU, v)).abs() <= 0.75e-7 * v.abs()).all()
    sr.sr_layer_linear(z, w, None, lo.GELU, None, y)
    compare("gelu", y, want, bound)
    sr.sr_layer_linear_grad(z, w, None, lo.GELU, torch.ones_like(z), dx, None, None)
    compare("slope", dx, want_slope, slope_bound)
    for name, wrong in {"nothing": torch.zeros_like(want), "1 + erf in fp32": z.double() * 0.5 * (1 + torch.erf(z * math.sqrt(0.5))).double(), "half of it": want / 2}.items():
        tail = (v < -4) & (v > -6)
        assert ((wrong - y.double()).abs() > bound)[tail].any(), name
    z = z * 6
    v = z.double()
    for kind in (lo.SILU, lo.SIGMOID):
        sr.sr_layer_linear(z, w, None, kind, None, y)
        want = lo.act(kind, v)
        compare("silu or sigmoid", y, want, U * (1.75 * v.abs() + 8) * want.abs() + 2.0 ** -126)


@pytest.mark.parametrize("shape", [(40, 4096, 256), (300, 4096, 264), (2048, 4096, 2048), (4096, 1024, 4096), (3000, 2045, 1030), (8200, 2047, 2049), (66000, 64, 72), (131080, 64, 264), (131080, 100, 264)],
                         ids=str)
@pytest.mark.parametrize("one_sign", [True, False], ids=["one_sign", "both"])
def test_errors_of_fp32_in_norm(shape, one_sign):
    """A product of K terms is at most n = K / 2 sums one after the other (two products a fp32 instruction; six parts of 16 an instruction are fewer), the i-th of them i / n of
    the whole where all have one sign.  Roundings to nearest add up like sqrt(n / 3) of them at most, each below u; in norm that is below u sqrt(K / 2), with the result's own
    rounding, u, beside it.  Sums that were cut off would be off by n / 2 steps of 2 u / 2 each: 1024 u for 45 at K = 4096.  Operands of both signs make smaller partial
    sums of a smaller whole, and stay below that as well.  dbias: one more sum a row, K of them."""
    P, C, O = shape
    g = torch.Generator(device=DEV).manual_seed(41)
    make = lambda *s: torch.rand(s, generator=g, device=DEV) if one_sign else torch.randn(s, generator=g, device=DEV)
    x, w, dy, y = make(P, C), make(O, C), make(P, O), torch.empty(P, O, device=DEV)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(O, device=DEV)
    sr.sr_layer_linear(x, w, None, lo.NONE, None, y)
    sr.sr_layer_linear_grad(x, w, None, lo.NONE, dy, dx, dw, db)
    exact = lo.behind_dz(x.double(), w.double(), dy.double())
    for name, got, want, n in zip(("y", "dx", "dweight", "dbias"), (y, dx, dw, db), (lo.affine(x.double(), w.double(), None), *exact), (C / 2, O / 2, P / 2, P)):
        off = got.double() - want
        assert off.norm() <= U * (math.sqrt(n) + 1) * want.norm(), name
        if one_sign:
            assert abs(float((off / want).mean())) <= U * (math.sqrt(n) + 1) / 4, (name, "the same way everywhere")

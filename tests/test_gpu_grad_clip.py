"""The norm of all gradients and clipping through the C ABI against the 64-bit oracle.

Tolerances, u = 2^-24: squares and sums are in double (their error is below 2^-40 of the norm), the norm and the factor are rounded to fp32 once
each (u); an output is g times the rounded factor, rounded to fp32 (u) and to its type (eps / 2, or half of its smallest step)."""
import math

import pytest
import torch

import paper_2303_08999_amd as sr
from oracle import layer_oracle as lo
from test_gpu_layer import DT, SMALLEST, U, Guarded

pytestmark = pytest.mark.gpu
DEV = "cuda"


def make(sizes, types, seed=1, scale=1.0, shift=0):
    g = torch.Generator().manual_seed(seed)
    return [Guarded(s, DT[types[i % len(types)]], shift, (torch.randn(s, generator=g) * scale).to(DT[types[i % len(types)]]))
            for i, s in enumerate(sizes)]


def check(sizes, types, most, seed=1, scale=1.0, shift=0, out_shift=None, grads=None):
    grads = grads or make(sizes, types, seed, scale, shift)
    host = [g.t.cpu() for g in grads]
    want, norm, factor = lo.clip([h.double() for h in host], most)
    outs = [Guarded(g.t.shape, g.t.dtype, shift if out_shift is None else out_shift) for g in grads]
    stats = Guarded((2,), torch.float32)
    sr.sr_grad_clip([g.t for g in grads], [o.t for o in outs], most, stats.t)
    torch.cuda.synchronize()
    for v in (*grads, *outs, stats):
        v.check()
    got = stats.t.double().cpu()
    assert abs(float(got[0]) - norm) <= 2 * U * norm + SMALLEST["f32"] and abs(float(got[1]) - factor) <= 2 * U * factor + SMALLEST["f32"], (got, norm, factor)
    for i, (g, h, o, w) in enumerate(zip(grads, host, outs, want)):
        assert torch.equal(g.t.cpu(), h), "an input changed"
        t = types[i % len(types)]
        err = 3 * U * w.abs()
        bound = err + torch.finfo(DT[t]).eps / 2 * (w.abs() + err) + SMALLEST[t] / 2 + SMALLEST["f32"]
        diff = (o.t.cpu().double() - w).abs()
        assert (diff <= bound).all(), f"tensor {i}: worst {float((diff / bound).max()):.2f} of the bound"
        if factor == 1.0:
            assert torch.equal(o.t.cpu(), h)
    # in place: the same bits; the norm alone: the same norm
    alone = torch.empty(2, device=DEV)
    inplace = [g.t for g in grads]
    sr.sr_grad_clip(inplace, None, most, alone)
    assert torch.equal(alone, stats.t)
    sr.sr_grad_clip(inplace, inplace, most, alone)
    torch.cuda.synchronize()
    assert torch.equal(alone, stats.t)
    for g, o in zip(grads, outs):
        g.check()
        assert torch.equal(g.t, o.t)


SIZES = [
    [(1,)], [(7,)], [(8,), (1,)], [(0,), (3,), (0, 5)], [(2048 * 8,)], [(2048 * 8 + 1,), (2048 * 4,)], [(2048 * 4 - 1,), (2048 * 4 + 3,), (2048 * 8 - 5,)],
    [(72, 5, 5), (72, 64), (72,), (64, 27), (64,)], [(100003,), (17,), (65537,), (2,)], [(3, 5, 7, 11, 2)], [(1 << 21,), (5,)],
]


@pytest.mark.parametrize("types", [["f32"], ["f16"], ["bf16"], ["f32", "bf16", "f16"]], ids="-".join)
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "x".join(str(math.prod(v)) for v in s))
def test_clipping(sizes, types):
    total = math.sqrt(sum(math.prod(s) for s in sizes))
    check(sizes, types, total / 3)
    check(sizes, types, total * 3, seed=2)


@pytest.mark.parametrize("shift,out_shift", [(1, 1), (3, 3), (0, 1), (5, 2)])
@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
def test_addresses_off_16_bytes(t, shift, out_shift):
    check([(1,), (3,), (2048 * 8,), (40001,), (9,)], [t], 1.0, shift=shift, out_shift=out_shift)


@pytest.mark.parametrize("count", [127, 128, 129, 300, 1000])
def test_many_tensors(count):
    check([(1 + (i * 37) % 301,) for i in range(count)], ["f32", "bf16"], 5.0)


def test_one_buffer_cut_into_tensors():
    """A bucket: tensors one behind the other, at any alignment."""
    flat = torch.randn(100000, device=DEV).to(torch.bfloat16)
    cuts = [0, 1, 3, 1000, 1001, 33333, 99999, 100000]
    grads = [flat[a:b] for a, b in zip(cuts, cuts[1:])]
    out = torch.empty_like(flat)
    stats, whole = torch.empty(2, device=DEV), torch.empty(2, device=DEV)
    sr.sr_grad_clip(grads, [out[a:b] for a, b in zip(cuts, cuts[1:])], 2.0, stats)
    again = torch.empty_like(flat)
    sr.sr_grad_clip([flat], [again], 2.0, whole)
    norm = float(flat.double().norm())
    assert abs(float(stats[0]) - norm) <= 2 * U * norm and abs(float(whole[0]) - norm) <= 2 * U * norm
    want = flat.double() * (2.0 / norm)
    for o in (out, again):
        assert ((o.double() - want).abs() <= (2.0 ** -8 + 4 * U) * want.abs() + 2.0 ** -133).all()


@pytest.mark.parametrize("t,scale", [("f32", 1e30), ("f32", 1e-30), ("f32", 2.0 ** -140), ("bf16", 1e35), ("bf16", 1e-35), ("f16", 2.0 ** -20)])
def test_values_whose_squares_have_no_place_in_fp32(t, scale):
    check([(3000,), (70,)], [t], 10.0 * scale, scale=scale)
    check([(3000,), (70,)], [t], 1000.0 * scale, scale=scale)


def test_zero_norm_and_zero_most():
    z = [torch.zeros(1000, device=DEV), torch.zeros(3, device=DEV, dtype=torch.float16)]
    stats = torch.empty(2, device=DEV)
    sr.sr_grad_clip(z, z, 0.0, stats)
    assert stats.tolist() == [0.0, 1.0] and not z[0].any()
    one = [torch.ones(1000, device=DEV)]
    sr.sr_grad_clip(one, one, 0.0, stats)
    assert float(stats[1]) == 0.0 and not one[0].any()
    inf = [torch.ones(100, device=DEV)]
    sr.sr_grad_clip(inf, inf, float("inf"), stats)
    assert stats.tolist() == [10.0, 1.0] and (inf[0] == 1).all()


@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_gradients_that_are_not_finite_are_left(bad):
    for t in (torch.float32, torch.float16, torch.bfloat16):
        g = [torch.randn(5000, device=DEV).to(t), torch.randn(77, device=DEV).to(t)]
        g[1][76] = bad
        out = [torch.zeros_like(v) for v in g]
        stats = torch.empty(2, device=DEV)
        sr.sr_grad_clip(g, out, 1e-3, stats)
        assert not math.isfinite(float(stats[0])) and float(stats[1]) == 1.0
        for a, b in zip(g, out):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_no_elements_at_all():
    g = [torch.empty(0, device=DEV), torch.empty((3, 0), device=DEV, dtype=torch.bfloat16)]
    stats = torch.full((2,), 9.0, device=DEV)
    sr.sr_grad_clip(g, g, 1.0, stats)
    assert stats.tolist() == [0.0, 1.0]


def test_the_same_tensor_twice_counts_twice():
    g = torch.full((16,), 3.0, device=DEV)
    stats = torch.empty(2, device=DEV)
    sr.sr_grad_clip([g, g], None, 1.0, stats)
    assert abs(float(stats[0]) - math.sqrt(288.0)) <= 2 * U * 17


def test_orders_of_axes():
    """Stored without gaps in any order of the axes; an output in another order is refused."""
    a = torch.randn(4, 6, 5, 3, device=DEV).to(memory_format=torch.channels_last)
    b = torch.randn(8, 9, device=DEV).t()
    out = [torch.empty_like(a), torch.empty_like(b)]
    stats = torch.empty(2, device=DEV)
    sr.sr_grad_clip([a, b], out, 1.0, stats)
    want, _, _ = lo.clip([a.double(), b.double()], 1.0)
    for o, w in zip(out, want):
        assert ((o.double() - w).abs() <= 4 * U * w.abs()).all()
    with pytest.raises(ValueError, match="another order"):
        sr.sr_grad_clip([a, b], [torch.empty(a.shape, device=DEV), out[1]], 1.0, stats)
    with pytest.raises(ValueError, match="gaps"):
        sr.sr_grad_clip([a[:, :, ::2]], None, 1.0, stats)


def test_lists_kept_streams_and_graphs():
    g = [torch.randn(n, device=DEV) for n in (40000, 3, 555)]
    out = [torch.empty_like(v) for v in g]
    grads, outs, stats = sr.sr_tensor_list(g), sr.sr_tensor_list(out), torch.empty(2, device=DEV)
    ws = torch.empty(sr.sr_grad_clip_workspace_bytes(3), device=DEV, dtype=torch.uint8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    sr.sr_grad_clip(grads, outs, 1.0, stats, workspace=ws, stream=side)
    side.synchronize()
    first = [o.clone() for o in out]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sr.sr_grad_clip(grads, outs, 1.0, stats, workspace=ws)
    for i in range(4):
        for o in out:
            o.zero_()
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for o, f in zip(out, first):
            assert torch.equal(o, f), f"replay {i}"
        g[0].add_(1.0)
        sr.sr_grad_clip(g, out, 1.0, stats)
        first = [o.clone() for o in out]


@pytest.mark.parametrize("shape,t", [(((1 << 32) + 5,), "bf16"), (((1 << 31) + 3,), "f16"), ((1 << 32,), "bf16"), ((3, 1 << 31), "f16"), ((1 << 16, (1 << 16) + 1, 1, 1, 1), "bf16")],
                         ids=lambda v: "x".join(map(str, v)) if isinstance(v, tuple) else v)
def test_a_tensor_of_more_elements_than_32_bits_count(shape, t):
    """A bucket beyond 2^31 and 2^32 elements beside a small tensor; all values but a few, some of them the last, are zeros."""
    big, small = torch.zeros(shape, device=DEV, dtype=DT[t]), torch.tensor([2.0, -4.0], device=DEV)
    flat, n = big.view(-1), big.numel()
    at = torch.tensor(sorted({0, 7, (1 << 30) - 1, 1 << 30, (1 << 31) - 1, min(1 << 31, n - 3), n // 2 + 1, n - 2, n - 1}), device=DEV)
    flat[at] = torch.arange(1, len(at) + 1, device=DEV).to(DT[t])
    values = flat[at].double()
    norm = math.sqrt(float((values ** 2).sum()) + 20.0)
    stats = torch.empty(2, device=DEV)
    grads = sr.sr_tensor_list([big, small])
    ws = torch.empty(sr.sr_grad_clip_workspace_bytes(grads.count), device=DEV, dtype=torch.uint8)
    sr.sr_grad_clip(grads, grads, norm / 4, stats, workspace=ws)
    torch.cuda.synchronize()
    assert abs(float(stats[0]) - norm) <= 2 * U * norm and abs(float(stats[1]) - 0.25) <= 2 * U
    # the quarter of a small whole number is one of the type's, but for the factor's own rounding
    assert ((flat[at].double() - values / 4).abs() <= (torch.finfo(DT[t]).eps / 2 + 4 * U) * values).all()
    assert ((small.double() - torch.tensor([0.5, -1.0], device=DEV)).abs() <= 4 * U).all()
    assert int(torch.count_nonzero(flat)) == len(at)
    if len(shape) == 1 and n % (1 << 30):
        with pytest.raises(ValueError, match="another size"):
            sr.sr_grad_clip(grads, [flat[:1 << 30], small], 1.0, stats)


@pytest.mark.parametrize("most", [1.0, 1e30, 1e38, 2e39])
def test_a_norm_beyond_fp32(most):
    """Written as infinity; the factor is that of the norm itself, in fp32, whose smallest step 2^-149 it has where it is subnormal."""
    g = [torch.full((100,), 3e38, device=DEV), torch.full((7,), -1e38, device=DEV, dtype=torch.bfloat16)]
    outs, stats = [torch.empty_like(v) for v in g], torch.empty(2, device=DEV)
    want, norm, factor = lo.clip([v.double() for v in g], most)
    assert norm > torch.finfo(torch.float32).max and factor < 1
    sr.sr_grad_clip(g, outs, most, stats)
    assert float(stats[0]) == math.inf and abs(float(stats[1]) - factor) <= 2 * U * factor + 2.0 ** -150
    for v, o, w, eps in zip(g, outs, want, (U, 2.0 ** -8)):
        assert ((o.double() - w).abs() <= (3 * U + eps) * w.abs() + 2.0 ** -150 * v.double().abs()).all()

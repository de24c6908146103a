"""The 64-bit oracle of the layers against autograd, against differences, and against values worked out by hand."""
import math

import pytest
import torch

from oracle import layer_oracle as lo

F = torch.nn.functional
LIBRARY = {lo.NONE: lambda z: z, lo.RELU: F.relu, lo.GELU: F.gelu, lo.SILU: F.silu, lo.SIGMOID: torch.sigmoid}


def draw(P, C, O, seed, wide=1):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)
    return r(P, C), r(wide * O, C) / math.sqrt(C), r(wide * O), r(P, O), r(P, O)


@pytest.mark.parametrize("kind", range(5))
def test_activations_and_slopes(kind):
    z = torch.cat([torch.linspace(-9, 9, 361, dtype=torch.float64), torch.tensor([-700.0, 700.0], dtype=torch.float64)]).requires_grad_()
    y = LIBRARY[kind](z)
    assert torch.allclose(lo.act(kind, z), y, rtol=1e-13, atol=1e-300)
    d, = torch.autograd.grad(y.sum(), z)
    assert torch.allclose(lo.slope(kind, z), d, rtol=1e-11, atol=1e-16)
    away = z.detach()[(z.abs() > 0.01) & (z.abs() < 10)]
    h = 1e-5
    assert torch.allclose((lo.act(kind, away + h) - lo.act(kind, away - h)) / (2 * h), lo.slope(kind, away), rtol=1e-7, atol=1e-9)


def test_activations_at_hand_made_points():
    z = torch.tensor([0.0, math.log(3.0)], dtype=torch.float64)
    assert lo.act(lo.SIGMOID, z).tolist() == pytest.approx([0.5, 0.75])
    assert lo.slope(lo.SIGMOID, z).tolist() == pytest.approx([0.25, 0.1875])
    assert lo.act(lo.SILU, z).tolist() == pytest.approx([0.0, 0.75 * math.log(3.0)])
    assert lo.slope(lo.SILU, z).tolist() == pytest.approx([0.5, 0.75 + 0.1875 * math.log(3.0)])
    assert lo.slope(lo.RELU, torch.tensor([-1.0, 0.0, 1.0])).tolist() == [0.0, 0.0, 1.0]
    one = torch.tensor([1.0], dtype=torch.float64)
    assert float(lo.act(lo.GELU, one)) == pytest.approx(0.8413447460685429)
    assert float(lo.slope(lo.GELU, one)) == pytest.approx(0.8413447460685429 + 0.24197072451914337)


@pytest.mark.parametrize("kind", range(5))
@pytest.mark.parametrize("gated", [False, True])
def test_gradients(kind, gated):
    x, w, b, dy, res = draw(7, 5, 6, kind + 10 * gated, 2 if gated else 1)
    for t in (x, w, b):
        t.requires_grad_()
    z = F.linear(x, w, b)
    y = LIBRARY[kind](z[:, :6]) * z[:, 6:] if gated else LIBRARY[kind](z) + res
    assert torch.allclose(lo.gated(x, w, b, kind) if gated else lo.linear(x, w, b, kind, res), y, rtol=1e-12, atol=1e-14)
    want = torch.autograd.grad((y * dy).sum(), (x, w, b))
    x, w, b = x.detach(), w.detach(), b.detach()
    dz = (lo.gated_dz if gated else lo.linear_dz)(x, w, b, kind, dy)
    got = lo.behind_dz(x, w, dz)
    for g, t in zip(got, want):
        assert torch.allclose(g, t, rtol=1e-11, atol=1e-13)
    # ... and differences along a direction
    gen = torch.Generator().manual_seed(99)
    vx, vw, vb = (torch.randn(t.shape, generator=gen, dtype=torch.float64) for t in (x, w, b))
    f = lambda h: float(((lo.gated if gated else lo.linear)(x + h * vx, w + h * vw, b + h * vb, kind) * dy).sum())
    along = float((got[0] * vx).sum() + (got[1] * vw).sum() + (got[2] * vb).sum())
    assert (f(1e-5) - f(-1e-5)) / 2e-5 == pytest.approx(along, rel=1e-6, abs=1e-7)


def test_clip():
    g = [torch.tensor([3.0], dtype=torch.float64), torch.tensor([[0.0, -4.0]], dtype=torch.float64)]
    out, norm, factor = lo.clip(g, 2.5)
    assert norm == 5.0 and factor == 0.5 and out[1].tolist() == [[0.0, -2.0]]
    assert lo.clip(g, 5.0)[2] == 1.0 and lo.clip(g, math.inf)[2] == 1.0
    bad = [g[0], torch.tensor([math.inf])]
    out, norm, factor = lo.clip(bad, 1.0)
    assert norm == math.inf and factor == 1.0 and out[0].tolist() == [3.0]

"""The router, the balance losses and their gradient through the C ABI against the 64-bit oracle on the same stored logits.

Tolerances, in units of u = 2^-24 (half a step of fp32).  An exponential exp2((z - m) LOG2E): the argument x is
rounded twice, 2 |x| u, the constant's own rounding adds |x| u / 2 at most, all of it times ln 2 in the result: 1.733 |x| u; the instruction
adds 2 u.  (fp16 logits: exp2(z LOG2E + o), o the same for a pixel's atoms, so that its rounding cancels in every quotient: less.)
A sum of n positive terms adds n u, the quotient 3 u.  So a probability is within (L + 1.75 X + 8) u of itself, X = the largest |z - m| / ln 2 of the pixel; results below 2^-126
become 0.  A rounding to type t adds finfo(t).eps / 2 of the value, or half of t's smallest step.
lse = m + ln s: nm's rounding, |m| / ln 2 u, times ln 2; the sum's (L + X) u; the logarithm's 3 u (|ln s| + 1); the addition's
u |lse|.  A gradient is a sum of at most five products of such numbers: three times a probability's error, relative to the sum
of its terms' magnitudes, and lse's own part."""
import math

import pytest
import torch

import paper_2303_08999_amd as sr
from oracle import route_oracle as ro

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
INF = float("inf")
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SMALLEST = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}
PLANAR, PRE, PM = sr.SR_COEFF_PLANAR, sr.SR_COEFF_PRE_SHUFFLE, sr.SR_COEFF_PIXEL_MAJOR


def stored(planar, layout, scale):
    if layout == PM:
        return planar.permute(0, 2, 3, 1).contiguous()
    return torch.nn.functional.pixel_unshuffle(planar, scale).contiguous() if layout == PRE else planar.contiguous()


def planar(t, layout, scale):
    if layout == PM:
        return t.permute(0, 3, 1, 2)
    return torch.nn.functional.pixel_shuffle(t, scale) if layout == PRE else t


def logits(n, L, H, W, dtype, seed, spread=1.5, special=True):
    """Gaussian logits of the stored type, ties among them; with `special`, masked atoms, pixels of none but masked atoms, the
    type's lowest value, and both zeros."""
    g = torch.Generator().manual_seed(seed)
    z = (torch.randn((n, L, H, W), generator=g) * spread).to(DT[dtype])
    if special:
        pick = torch.rand((n, 1, H, W), generator=g)
        z = torch.where((torch.rand(z.shape, generator=g) < 0.5) & (pick < 0.2), torch.full_like(z, -INF), z)
        z = torch.where((pick > 0.2) & (pick < 0.3), torch.full_like(z, -INF), z)
        z = torch.where((torch.rand(z.shape, generator=g) < 0.8) & (pick > 0.3) & (pick < 0.4), torch.full_like(z, torch.finfo(DT[dtype]).min), z)
        z = torch.where((torch.rand(z.shape, generator=g) < 0.6) & (pick > 0.4) & (pick < 0.5), torch.zeros_like(z), z)
        z = torch.where((torch.rand(z.shape, generator=g) < 0.3) & (pick > 0.4) & (pick < 0.5), -torch.zeros_like(z), z)
    return z


def make_mask(n, H, W, seed):
    g = torch.Generator().manual_seed(seed)
    return ((torch.rand((n, 1, H, W), generator=g) < 0.7) * torch.randint(1, 256, (n, 1, H, W), generator=g)).to(torch.uint8)


def probability_error(z):
    """(L + 1.75 X + 8) u of every pixel; a masked atom's distance does not count, nor one that no exponential is left of."""
    m = z.amax(1, keepdim=True)
    x = torch.where(torch.isneginf(z), torch.zeros_like(z), (m - z) / math.log(2.0)).clamp(max=160.0)
    return (z.shape[1] + 1.75 * x.amax(1, keepdim=True) + 8) * U


def lse_error(z):
    m = z.amax(1, keepdim=True)
    m = torch.where(torch.isneginf(m), torch.zeros_like(m), m)
    ln_s = (ro.lse(z) - m).abs()
    return (2 * m.abs() + ro.lse(z).abs()) * U + probability_error(z) + 3 * U * (ln_s + 1)


class Guarded:
    """A tensor between two strips that a call must not touch."""

    def __init__(self, shape, dtype, shift=0):
        numel = math.prod(shape)
        self.raw = torch.full((numel + 512,), 77, device=DEV, dtype=dtype)
        self.t = self.raw[256 + shift:256 + shift + numel].view(shape)
        self.lo, self.hi = 256 + shift, 256 + shift + numel

    def check(self):
        assert (self.raw[:self.lo] == 77).all() and (self.raw[self.hi:] == 77).all(), "written outside of the tensor"


def check_all(n, L, H, W, T, zd, vd, kind, layout, scale=2, masked=False, seed=1, spread=1.5, special=True, shift=0):
    z0 = logits(n, L, H, W, zd, seed, spread, special)
    mask = make_mask(n, H, W, seed + 1) if masked else None
    z = z0.double()
    coeff = Guarded(stored(z0, layout, scale).shape, DT[zd], shift)
    coeff.t.copy_(stored(z0, layout, scale))
    dmask = None if mask is None else mask.to(DEV)
    index, value = Guarded((n, T, H, W), torch.uint8, shift), Guarded((n, T, H, W), DT[vd], shift)
    sr.sr_list_route(coeff.t, L, scale, T, kind, layout, dmask, index.t, value.t)
    torch.cuda.synchronize()
    index.check(), value.check()
    want_index, want = ro.route(z, T, kind, mask)
    got_index = index.t.cpu().long()
    assert torch.equal(got_index, want_index), f"{int((got_index != want_index).sum())} indices differ"
    err = (value.t.cpu().double() - want).abs()
    rel = 0.0 if kind == sr.SR_ROUTE_VALUES else probability_error(z)
    stored_rel = torch.finfo(DT[vd]).eps / 2
    bound = want.abs() * (rel + stored_rel) + SMALLEST[vd] / 2 + 2.0 ** -125
    if kind == sr.SR_ROUTE_VALUES:
        over = want.abs() > torch.finfo(DT[vd]).max * (1 + stored_rel / 2)      # no value of that type: infinity
        err = torch.where(over, (value.t.cpu().double() != want.sign() * INF).double(), err)
    assert (torch.nan_to_num(err, nan=INF) <= bound).all() or (kind == sr.SR_ROUTE_VALUES and torch.equal(value.t.cpu(), want.to(DT[vd]))), \
        f"values: worst {float((err / bound).max()):.2f} of the bound"

    counts = dloss = None
    if kind != sr.SR_ROUTE_VALUES:
        i2, v2 = torch.empty_like(index.t), torch.empty_like(value.t)
        counts, share, loss = Guarded((L + 1,), torch.int64), Guarded((L,), torch.float32), Guarded((2,), torch.float32)
        sr.sr_list_route_balance(coeff.t, L, scale, T, kind, layout, dmask, i2, v2, counts.t, share.t, loss.t)
        torch.cuda.synchronize()
        counts.check(), share.check(), loss.check()
        assert torch.equal(i2, index.t) and torch.equal(v2, value.t), "the lists with and without the losses"
        c, s, ls = ro.balance(z, T, mask)
        assert torch.equal(counts.t.cpu(), c)
        on = ro.live(z, mask)
        worst = float((probability_error(z) * on).max()) + 513 * U
        assert ((share.t.cpu().double() - s).abs() <= s * worst + 2.0 ** -125).all()
        assert abs(float(loss.t[0]) - float(ls[0])) <= float(ls[0]) * (worst + 2 * U)
        l, d = ro.lse(z), lse_error(z)
        slack = (torch.where(on, (2 * l.abs() + d) * d, torch.zeros_like(l)).sum() / max(int(on.sum()), 1)) + ls[1] * 514 * U
        if float(ls[1]) > torch.finfo(torch.float32).max * (1 + U):      # the type's lowest value, squared: no fp32 number
            assert float(loss.t[1]) == INF
        else:
            assert abs(float(loss.t[1]) - float(ls[1])) <= float(slack) + 2.0 ** -125
        counts = counts.t

    # gradient: of the values alone, with the losses, of the losses alone
    g = torch.Generator().manual_seed(seed + 2)
    dvalue = torch.randn((n, T, H, W), generator=g).to(DT[vd])
    modes = [(True, False)] if counts is None else [(True, False), (True, True), (False, True)]
    for with_value, with_loss in modes:
        dloss = torch.tensor([0.37, -0.011]) * (n * H * W) if with_loss else None
        dz = Guarded(coeff.t.shape, DT[zd], shift)
        sr.sr_list_route_grad(coeff.t, index.t, dvalue.to(DEV) if with_value else None, L, scale, T, kind, layout, dmask,
                              counts if with_loss else None, None if dloss is None else dloss.to(DEV), dz.t)
        torch.cuda.synchronize()
        dz.check(), coeff.check()
        want, size = ro.route_grad(z, want_index, kind, dvalue.double() if with_value else None,
                                   counts.cpu() if with_loss else None, dloss, mask)
        got = planar(dz.t, layout, scale).cpu().double()
        bound = 3 * size * (0.0 if kind == sr.SR_ROUTE_VALUES else probability_error(z)) + SMALLEST[zd] / 2 + 2.0 ** -120
        if with_loss:
            bound = bound + abs(2 * float(dloss[1])) / max(int(counts[L]), 1) * ro.softmax(z) * lse_error(z)
        if kind != sr.SR_ROUTE_VALUES and with_value:                    # a probability that fp32 has no number for
            bound = bound + 2.0 ** -125 * float(dvalue.double().abs().max()) * T
        bound = bound + want.abs() * torch.finfo(DT[zd]).eps / 2
        err = (got - want).abs()
        err = torch.where(want.abs() > torch.finfo(DT[zd]).max, torch.zeros_like(err), err)
        assert (torch.nan_to_num(err, nan=INF) <= bound).all(), f"gradient {with_value, with_loss}: worst {float((err / bound).max()):.2f} of the bound"
        if masked:
            assert (planar(dz.t, layout, scale).cpu()[(mask == 0).expand(-1, L, -1, -1)] == 0).all()


SOFT, CHOSEN, VALUES = sr.SR_ROUTE_SOFTMAX, sr.SR_ROUTE_CHOSEN, sr.SR_ROUTE_VALUES
SHAPES = [
    # (n, L, H, W, entries, layout, scale, masked)
    (1, 72, 1, 1, 8, PM, 1, False),          # one token
    (1, 72, 1, 1, 8, PLANAR, 1, False),
    (1, 1, 3, 5, 1, PLANAR, 1, True),        # one atom
    (1, 256, 1, 3, 8, PM, 1, False),         # the most atoms
    (2, 256, 5, 13, 16, PLANAR, 1, True),
    (1, 17, 9, 11, 17, PLANAR, 1, False),    # every atom listed
    (1, 70, 2, 3, 70, PM, 1, True),          # more entries than lanes
    (1, 256, 1, 2, 256, PM, 1, False),
    (3, 64, 1, 67, 2, PM, 1, True),          # rows of tokens, padded
    (1, 128, 1, 130, 4, PM, 1, False),
    (2, 73, 7, 9, 3, PM, 1, True),           # rows of 73 logits: no two aligned alike
    (1, 72, 24, 36, 8, PRE, 2, False),       # before the pixel-shuffle
    (2, 40, 9, 15, 5, PRE, 3, True),
    (1, 72, 8, 20, 7, PRE, 4, False),
    (1, 72, 31, 67, 8, PLANAR, 1, False),    # several wavefronts, an odd number of pixels
    (2, 72, 33, 64, 1, PLANAR, 1, True),
    (1, 24, 40, 70, 4, PLANAR, 1, False),
    (1, 144, 16, 34, 8, PLANAR, 1, True),
    (1, 9, 50, 50, 9, PLANAR, 1, False),
    (1, 32, 1, 700, 6, PM, 1, True),
    (1, 200, 1, 150, 12, PM, 1, False),
]


@pytest.mark.parametrize("types", [("f32", "f32"), ("f16", "f16"), ("bf16", "f32"), ("f32", "f16"), ("bf16", "f16"), ("f16", "f32")], ids=lambda t: "-".join(t))
@pytest.mark.parametrize("kind", [SOFT, CHOSEN, VALUES], ids=["softmax", "chosen", "values"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "n%dL%d_%dx%d_T%d_o%ds%d%s" % (s[:7] + ("m" if s[7] else "",)))
def test_lists_losses_and_gradients(shape, kind, types):
    n, L, H, W, T, layout, scale, masked = shape
    check_all(n, L, H, W, T, *types, kind, layout, scale, masked, seed=L * 7 + W)


# enough pixels for the kernels with one to four lanes a pixel
MANY = [
    # (n, L, H, W, entries, layout, scale, masked)
    (1, 72, 61, 69, 8, PLANAR, 1, False),
    (2, 72, 40, 53, 5, PLANAR, 1, True),
    (1, 72, 4100, 1, 16, PLANAR, 1, False),
    (1, 71, 63, 66, 1, PLANAR, 1, True),
    (1, 1, 70, 60, 1, PLANAR, 1, False),
    (1, 9, 64, 65, 9, PLANAR, 1, True),
    (1, 16, 66, 67, 16, PLANAR, 1, False),
    (1, 24, 64, 67, 4, PLANAR, 1, True),
    (1, 25, 64, 67, 4, PLANAR, 1, False),
    (1, 73, 61, 69, 8, PLANAR, 1, False),        # four lanes a pixel
    (1, 96, 64, 66, 16, PLANAR, 1, True),
    (1, 128, 67, 62, 4, PLANAR, 1, False),
    (2, 145, 45, 92, 8, PLANAR, 1, True),
    (1, 256, 83, 99, 12, PLANAR, 1, False),
    (1, 72, 64, 66, 8, PRE, 2, True),
    (2, 40, 60, 39, 3, PRE, 3, False),
    (1, 100, 72, 60, 8, PRE, 4, True),
    (1, 72, 1, 4111, 8, PM, 1, False),           # tokens: aligned rows
    (3, 64, 1, 1401, 2, PM, 1, True),
    (1, 256, 1, 8209, 8, PM, 1, False),
    (1, 120, 1, 4099, 16, PM, 1, True),
    (1, 73, 1, 4177, 4, PM, 1, True),            # rows that are not
    (1, 12, 1, 4150, 12, PM, 1, False),          # ... of fp32, whole 16-byte pieces but no whole eight atoms
    (2, 8, 50, 41, 3, PM, 1, True),
    (1, 5, 1, 4160, 5, PM, 1, False),
    (1, 200, 1, 8255, 16, PM, 1, False),
    (1, 72, 60, 72, 17, PLANAR, 1, False),       # a list longer than they take
]


@pytest.mark.parametrize("types", [("f32", "f32"), ("f16", "f16"), ("bf16", "f32"), ("f16", "f32")], ids=lambda t: "-".join(t))
@pytest.mark.parametrize("kind", [SOFT, CHOSEN, VALUES], ids=["softmax", "chosen", "values"])
@pytest.mark.parametrize("shape", MANY, ids=lambda s: "n%dL%d_%dx%d_T%d_o%ds%d%s" % (s[:7] + ("m" if s[7] else "",)))
def test_many_pixels(shape, kind, types):
    n, L, H, W, T, layout, scale, masked = shape
    check_all(n, L, H, W, T, *types, kind, layout, scale, masked, seed=L * 5 + W)


@pytest.mark.parametrize("zd,vd", [("f16", "f16"), ("f32", "f16"), ("bf16", "f32")])
@pytest.mark.parametrize("layout,L", [(PLANAR, 72), (PM, 72), (PM, 64), (PRE, 72), (PLANAR, 100)])
def test_many_pixels_at_odd_addresses(layout, L, zd, vd):
    for shift in (1, 4):
        check_all(1, L, 62, 70, 8, zd, vd, SOFT, layout, 2, True, seed=8, shift=shift)


@pytest.mark.parametrize("spread", [0.0, 30.0, 300.0])
@pytest.mark.parametrize("kind", [SOFT, CHOSEN])
def test_flat_and_steep_logits(kind, spread):
    """All logits alike: the first atoms win, every value is 1/L; far apart: all but one vanish."""
    check_all(1, 72, 12, 33, 8, "f32", "f32", kind, PLANAR, seed=3, spread=spread, special=False)
    check_all(1, 72, 12, 33, 8, "bf16", "f16", kind, PM, seed=4, spread=spread, special=False)
    check_all(1, 72, 64, 65, 8, "f32", "f32", kind, PLANAR, seed=5, spread=spread, special=False)
    check_all(1, 128, 64, 65, 8, "bf16", "f16", kind, PM, seed=6, spread=spread, special=False)


@pytest.mark.parametrize("zd,vd", [("f16", "f16"), ("f32", "f16"), ("bf16", "f32")])
@pytest.mark.parametrize("layout", [PLANAR, PM, PRE])
def test_tensors_at_odd_addresses(layout, zd, vd):
    for shift in (1, 3):
        check_all(1, 72, 18, 66, 8, zd, vd, SOFT, layout, 2, True, seed=8, shift=shift)


def test_random_shapes():
    g = torch.Generator().manual_seed(20230318)
    pick = lambda *v: v[int(torch.randint(len(v), (1,), generator=g))]
    num = lambda lo, hi: int(torch.randint(lo, hi + 1, (1,), generator=g))
    for at in range(40):
        L = pick(72, num(1, 40), num(65, 130), num(131, 256))
        T = min(L, pick(1, 2, 4, 8, num(1, 16), num(1, 20)))
        layout = pick(PLANAR, PLANAR, PM, PRE)
        s = pick(2, 3, 4) if layout == PRE else 1
        h, w = (num(1, 12), num(1, 40)) if at % 2 else (num(20, 30), num(150, 170) * (3 if L > 128 else 1))
        args = (pick(1, 1, 2), L, h * s, w * s, T, pick("f32", "f16", "bf16"), pick("f32", "f16"), pick(SOFT, CHOSEN, VALUES), layout, s, pick(True, False))
        print(at, args, flush=True)
        check_all(*args, seed=1000 + at)


def test_padding_is_not_looked_at():
    """NaN and infinities in masked pixels: values 0, atoms 0, 1, ...; nothing of them in losses and gradients."""
    for layout, L, H in ((PLANAR, 72, 9), (PLANAR, 200, 9), (PM, 72, 9), (PM, 200, 9), (PLANAR, 72, 110), (PLANAR, 200, 210), (PM, 72, 110), (PM, 200, 210)):
        z = logits(2, L, H, 21, "f32", 5, special=False)
        mask = make_mask(2, H, 21, 6)
        dirty = torch.where(mask == 0, torch.tensor([float("nan"), INF, -INF])[torch.arange(z.numel()) % 3].view(z.shape), z)
        got = []
        for t in (z, dirty):
            c = stored(t, layout, 1).to(DEV)
            index, value = torch.empty((2, 8, H, 21), device=DEV, dtype=torch.uint8), torch.empty((2, 8, H, 21), device=DEV)
            counts, share, loss = torch.empty(L + 1, device=DEV, dtype=torch.int64), torch.empty(L, device=DEV), torch.empty(2, device=DEV)
            sr.sr_list_route_balance(c, L, 1, 8, SOFT, layout, mask.to(DEV), index, value, counts, share, loss)
            dz = torch.empty_like(c)
            dv = torch.randn(value.shape, generator=torch.Generator().manual_seed(9)).to(DEV)
            sr.sr_list_route_grad(c, index, dv, L, 1, 8, SOFT, layout, mask.to(DEV), counts, loss, dz)
            got.append((index, value, counts, share, loss, dz))
        for a, b in zip(*got):
            assert torch.equal(a, b)


def test_nan_and_infinite_logits_still_list_different_atoms():
    for L, layout, px in ((72, PLANAR, 300), (72, PM, 3), (200, PLANAR, 200), (40, PM, 500), (72, PLANAR, 4500), (200, PLANAR, 8300), (40, PM, 4200)):
        z = logits(1, L, 1, px, "f32", 11, special=False)
        g = torch.Generator().manual_seed(12)
        for bad in (float("nan"), INF, -INF, -float("nan")):
            z = torch.where(torch.rand(z.shape, generator=g) < 0.15, torch.tensor(bad), z)
        for zd in ("f32", "f16", "bf16"):
            c = stored(z.to(DT[zd]), layout, 1).to(DEV)
            index, value = torch.empty((1, 8, 1, px), device=DEV, dtype=torch.uint8), torch.empty((1, 8, 1, px), device=DEV)
            sr.sr_list_route(c, L, 1, 8, SOFT, layout, None, index, value)
            i = index.cpu().long()
            assert (i < L).all() and (torch.sort(i, dim=1).values.diff(dim=1) > 0).all()


def test_no_live_pixel_and_empty_calls():
    L, T = 72, 8
    z = torch.full((1, L, 5, 70), -INF, device=DEV)
    index, value = torch.empty((1, T, 5, 70), device=DEV, dtype=torch.uint8), torch.empty((1, T, 5, 70), device=DEV)
    for coeff, i, v in ((z, index, value), (z[:0], index[:0], value[:0])):
        counts, share, loss = torch.full((L + 1,), 5, device=DEV), torch.full((L,), 5.0, device=DEV), torch.full((2,), 5.0, device=DEV)
        sr.sr_list_route_balance(coeff, L, 1, T, SOFT, PLANAR, None, i, v, counts, share, loss)
        torch.cuda.synchronize()
        assert not counts.any() and not share.any() and not loss.any()
    dz = torch.ones_like(z)
    sr.sr_list_route_grad(z, index, value, L, 1, T, SOFT, PLANAR, None, counts, loss, dz)
    torch.cuda.synchronize()
    assert not value.any() and not dz.any() and (index == torch.arange(T, device=DEV, dtype=torch.uint8).view(1, T, 1, 1)).all()


def test_gradient_with_foreign_lists():
    """Atoms listed twice or not below L: unspecified values at that pixel, the others as they are."""
    for layout, W in ((PLANAR, 300), (PM, 4), (PLANAR, 2500), (PM, 2500)):
        z = logits(1, 72, 2, W, "f32", 21, special=False)
        index, _ = ro.route(z.double(), 8, SOFT)
        dv = torch.randn((1, 8, 2, W), generator=torch.Generator().manual_seed(3))
        out = []
        for spoil in (False, True):
            i = index.clone().to(torch.uint8)
            if spoil:
                i[:, 1, 0], i[:, 2, 0] = i[:, 0, 0], 255
            dz = Guarded(stored(z, layout, 1).shape, torch.float32)
            sr.sr_list_route_grad(stored(z, layout, 1).to(DEV), i.to(DEV), dv.to(DEV), 72, 1, 8, SOFT, layout, None, None, None, dz.t)
            torch.cuda.synchronize()
            dz.check()
            out.append(planar(dz.t, layout, 1))
        assert torch.equal(out[0][:, :, 1], out[1][:, :, 1])


def chain(wl, z, lr, D, dout, dloss, T, kind, bufs):
    """A training step's own part: lists and losses, the image, and the gradients back to the logits and the dictionary."""
    index, value, counts, share, loss, out, dvalue, ddict, dz, ws0, ws1 = bufs
    n, L, H, W = z.shape
    sr.sr_list_route_balance(z, L, 1, T, kind, PLANAR, None, index, value, counts, share, loss, workspace=ws0)
    sr.sr_dict_assemble_list(lr, index, value, D, L, 5, wl, 3, T, out)
    sr.sr_dict_assemble_list_grad(lr, index, value, D, L, 5, wl, 3, T, None, dout, dvalue, ddict, workspace=ws1)
    sr.sr_list_route_grad(z, index, dvalue, L, 1, T, kind, PLANAR, None, counts, dloss, dz)


def chain_buffers(z, T, scale, vd):
    n, L, H, W = z.shape
    e = lambda *s, dtype=torch.float32: torch.empty(s, device=DEV, dtype=dtype)
    return (e(n, T, H, W, dtype=torch.uint8), e(n, T, H, W, dtype=vd), e(L + 1, dtype=torch.int64), e(L), e(2), e(n, 3, H, W),
            e(n, T, H, W, dtype=vd), e(L, 5, 5), torch.empty_like(z), e(sr.sr_list_route_workspace_bytes(L), dtype=torch.uint8),
            e(sr.sr_dict_assemble_list_grad_workspace_bytes(L, 5), dtype=torch.uint8))


def chain_inputs(seed, n=1, L=24, h=9, w=19, s=2, zd=torch.float32):
    g = torch.Generator().manual_seed(seed)
    z = (torch.randn((n, L, h * s, w * s), generator=g)).to(zd).to(DEV)
    return (z, torch.rand((n, 3, h, w), generator=g).to(DEV), torch.randn((L, 5, 5), generator=g).to(DEV) / 5,
            torch.randn((n, 3, h * s, w * s), generator=g).to(DEV), torch.tensor([3.0, 0.2], device=DEV))


@pytest.mark.parametrize("kind", [SOFT, CHOSEN])
def test_a_training_step_from_logits_to_gradients(oracle, kind):
    """The chain against the 64-bit chain.  fp32 values: the values' error (48 u here, 24 atoms) enters the image's gradient
    once, the responses' (25 taps, 3 channels and the split operands: 76 u of the magnitudes) the logits' gradient."""
    T = 4
    z, lr, D, dout, dloss = chain_inputs(31)
    bufs = chain_buffers(z, T, 2, torch.float32)
    chain(2, z, lr, D, dout, dloss, T, kind, bufs)
    torch.cuda.synchronize()
    index, value, counts, share, loss, out, dvalue, ddict, dz = (b.cpu() for b in bufs[:9])
    zz, up = z.cpu().double(), torch.from_numpy(oracle.bicubic(lr.cpu().numpy(), 2)).double()
    wi, wv = ro.route(zz, T, kind)
    c, s, l = ro.balance(zz, T)
    assert torch.equal(index.long(), wi) and torch.equal(counts, c)
    dv, dd, _ = ro.list_grad(up, wi, wv, D.cpu().double(), dout.cpu().double())
    want, size = ro.route_grad(zz, wi, kind, dv, c, dloss.cpu())
    mag, _, _ = ro.list_grad(torch.full_like(up, 1.6), wi, wv, D.cpu().double().abs(), dout.cpu().double().abs())
    assert ((dvalue.double() - dv).abs() <= 76 * U * mag).all()
    _, dmag, _ = ro.list_grad(torch.full_like(up, 1.6), wi, wv, D.cpu().double(), dout.cpu().double().abs())
    assert ((ddict.double() - dd).abs() <= (76 + 48 + 684) * U * dmag).all()          # 18 x 38 pixels in one run
    _, size2 = ro.route_grad(zz, wi, kind, mag, None, None)
    assert ((dz.double() - want).abs() <= 3 * probability_error(zz) * size + 2 * 76 * U * size2 + 4 * U * size2 + 2.0 ** -100).all()


def test_calls_replay_inside_a_captured_graph():
    """The whole chain, captured; replays on other inputs with eager work between, each against eager calls."""
    T, kind = 8, SOFT
    first = chain_inputs(40, L=72, h=40, w=33, zd=torch.float16)
    held = [t.clone() for t in first]
    bufs, eager = chain_buffers(first[0], T, 2, torch.float16), chain_buffers(first[0], T, 2, torch.float16)
    chain(2, *held, T, kind, bufs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain(2, *held, T, kind, bufs)
    for rep in range(4):
        fresh = chain_inputs(41 + rep, L=72, h=40, w=33, zd=torch.float16)
        for a, b in zip(held, fresh):
            a.copy_(b)
        for b in bufs:
            b.fill_(3)
        graph.replay()
        chain(2, *fresh, T, kind, eager)
        torch.cuda.synchronize()
        for a, b in zip(bufs[:9], eager[:9]):
            assert torch.equal(a, b), f"replay {rep}"


def test_another_stream_and_repeated_calls_give_the_same_bits():
    T, kind = 8, CHOSEN
    ins = chain_inputs(50, n=2, L=72, h=64, w=80)
    bufs = [chain_buffers(ins[0], T, 2, torch.float32) for _ in range(3)]
    chain(2, *ins, T, kind, bufs[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain(2, *ins, T, kind, bufs[1])
    chain(2, *ins, T, kind, bufs[2])                             # beside it, with scratch of its own
    torch.cuda.synchronize()
    for a, b, c in zip(*[b[:9] for b in bufs]):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_long_sums():
    """More pixels than any run in fp32: shares and counts of half a million pixels, with the lists of all of them."""
    L, T, H, W = 72, 8, 500, 1001
    g = torch.Generator(device=DEV).manual_seed(77)
    z = torch.randn((1, L, H, W), device=DEV, generator=g).half()
    index, value = torch.empty((1, T, H, W), device=DEV, dtype=torch.uint8), torch.empty((1, T, H, W), device=DEV)
    counts, share, loss = torch.empty(L + 1, device=DEV, dtype=torch.int64), torch.empty(L, device=DEV), torch.empty(2, device=DEV)
    sr.sr_list_route_balance(z, L, 1, T, SOFT, PLANAR, None, index, value, counts, share, loss)
    p = torch.softmax(z.double(), 1)
    s = p.mean(dim=(0, 2, 3))
    order = torch.sort(z.float(), dim=1, descending=True, stable=True).indices[:, :T]
    assert torch.equal(index.long(), order)
    assert torch.equal(counts[:L], torch.bincount(order.reshape(-1), minlength=L)) and int(counts[L]) == H * W
    worst = (L + 1.75 * 16 + 8 + 513) * U
    assert ((share.double() - s).abs() <= s * worst).all()
    v = p.gather(1, order)
    assert ((value.double() - v).abs() <= v * (L + 1.75 * 16 + 8) * U).all()
    lse = torch.logsumexp(z.double(), 1)
    assert abs(float(loss[1]) - float((lse * lse).mean())) <= float((lse * lse).mean()) * (514 + 150) * U


@pytest.mark.parametrize("layout,L,H,W", [(PM, 16, 31, 100_003), (PLANAR, 9, 9, 1_000_011)], ids=["rows", "planes"])
def test_sums_over_many_runs(layout, L, H, W):
    """More tiles for every wavefront than one run in fp32 takes (64, then the 64 lanes: 70 additions one after the other)."""
    T = 2
    g = torch.Generator(device=DEV).manual_seed(78)
    z = torch.randn((1, H, W, L) if layout == PM else (1, L, H, W), device=DEV, generator=g).bfloat16()
    mask = (torch.rand((1, 1, H, W), device=DEV, generator=g) < 0.9).byte()
    index, value = torch.empty((1, T, H, W), device=DEV, dtype=torch.uint8), torch.empty((1, T, H, W), device=DEV)
    counts, share, loss = torch.empty(L + 1, device=DEV, dtype=torch.int64), torch.empty(L, device=DEV), torch.empty(2, device=DEV)
    sr.sr_list_route_balance(z, L, 1, T, SOFT, layout, mask, index, value, counts, share, loss)
    on = mask.reshape(-1) != 0
    rows = (z.reshape(-1, L) if layout == PM else z.reshape(L, -1).t())[on].float()
    order = torch.sort(rows, dim=1, descending=True, stable=True).indices[:, :T]
    assert torch.equal(index.reshape(T, -1).t()[on].long(), order)
    assert torch.equal(counts[:L], torch.bincount(order.reshape(-1), minlength=L)) and int(counts[L]) == rows.shape[0]
    s = torch.zeros(L, device=DEV, dtype=torch.float64)
    sq = 0.0
    for part in rows.split(1 << 20):
        s += torch.softmax(part.double(), 1).sum(0)
        sq += float((torch.logsumexp(part.double(), 1) ** 2).sum())
    s, sq = s / rows.shape[0], sq / rows.shape[0]
    assert ((share.double() - s).abs() <= s * (L + 1.75 * 16 + 8 + 71) * U).all()
    assert abs(float(loss[1]) - sq) <= sq * (1 + 150) * U


def test_scratch_made_by_a_call_belongs_to_its_stream(monkeypatch):
    """(Else the current stream may still write to that memory, or get it again before the call has run.)"""
    L, T, k, h, w, s = 16, 4, 3, 20, 30, 2
    g = torch.Generator(device=DEV).manual_seed(79)
    z, lr = torch.randn((1, L, h * s, w * s), device=DEV, generator=g), torch.rand((1, 3, h, w), device=DEV, generator=g)
    D, dout = torch.randn((L, k, k), device=DEV, generator=g), torch.randn((1, 3, h * s, w * s), device=DEV, generator=g)
    index, value = torch.empty((1, T, h * s, w * s), device=DEV, dtype=torch.uint8), torch.empty((1, T, h * s, w * s), device=DEV)
    outs = []
    side, make, made = torch.cuda.Stream(), torch.empty, []
    for stream in (None, side, side.cuda_stream):
        counts, share, loss = torch.empty(L + 1, device=DEV, dtype=torch.int64), torch.empty(L, device=DEV), torch.empty(2, device=DEV)
        dv, dd = torch.empty_like(value), torch.empty_like(D)
        torch.cuda.synchronize()
        with monkeypatch.context() as m:
            m.setattr(torch, "empty", lambda *a, **kw: (made.append(torch.cuda.current_stream().cuda_stream), make(*a, **kw))[1])
            sr.sr_list_route_balance(z, L, 1, T, SOFT, PLANAR, None, index, value, counts, share, loss, stream=stream)
            sr.sr_dict_assemble_list_grad(lr, index, value, D, L, k, s, 3, T, None, dout, dv, dd, stream=stream)
        torch.cuda.synchronize()
        outs.append((counts, share, loss, dv, dd))
    assert made == [torch.cuda.current_stream().cuda_stream] * 2 + [side.cuda_stream] * 4
    for o in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(outs[0], o))

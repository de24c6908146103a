"""Gradient of the per-pixel list form through the C ABI against the 64-bit oracle on the same stored tensors.

Tolerances, u = 2^-24.  E is a sum of C products, each of an up-sampled value within 10 u of |U| <= A max|lr| (A = 1.5625: the
interpolator's weights add up to at most 1.25 along an axis, in magnitude), so within (C + 12) u of its terms' magnitudes.  A
response adds k^2 u in fp32; where the operands of matrix-core products are split in two fp16 numbers, 2^-22 of each and the
product of the lower parts, 12 u in all.  ddict: a run of n entries in fp32 adds n u, n at most 4096 pixels'."""
import pytest
import torch

import paper_2303_08999_amd as sr
from oracle import route_oracle as ro
from test_gpu_route import Guarded, make_mask

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
A = 1.5625
DT = {"f32": torch.float32, "f16": torch.float16}


def inputs(n, C, h, w, s, L, k, T, vd, io, seed, gain=1.0):
    g = torch.Generator().manual_seed(seed)
    H, W = h * s, w * s
    order = torch.rand((n, L, H, W), generator=g).topk(T, dim=1).indices
    value = (torch.rand((n, T, H, W), generator=g) - 0.2).to(DT[vd])
    value = torch.where(torch.rand(value.shape, generator=g) < 0.1, torch.zeros_like(value), value)
    return {"lr": torch.rand((n, C, h, w), generator=g).to(DT[io]), "index": order.to(torch.uint8), "value": value,
            "dict": torch.randn((L, k, k), generator=g) / k, "dout": (torch.randn((n, C, H, W), generator=g) * gain).to(DT[io])}


def run(d, s, mask=None, want=(True, True), shift=0, workspace=None):
    n, C = d["lr"].shape[:2]
    L, k, T = d["dict"].shape[0], d["dict"].shape[-1], d["index"].shape[1]
    dev = {}
    for name, t in d.items():
        dev[name] = Guarded(t.shape, t.dtype, shift)
        dev[name].t.copy_(t)
    dv = Guarded(d["value"].shape, d["value"].dtype, shift) if want[0] else None
    dd = Guarded(d["dict"].shape, torch.float32, shift) if want[1] else None
    sr.sr_dict_assemble_list_grad(dev["lr"].t, dev["index"].t, dev["value"].t, dev["dict"].t, L, k, s, C, T,
                                  None if mask is None else mask.to(DEV), dev["dout"].t, dv and dv.t, dd and dd.t, workspace=workspace)
    torch.cuda.synchronize()
    for x in list(dev.values()) + [dv, dd]:
        if x is not None:
            x.check()
    return dv and dv.t.cpu(), dd and dd.t.cpu()


def check(oracle, n, C, h, w, s, L, k, T, vd, io, masked=False, seed=1, gain=1.0, shift=0, spoil=None):
    d = inputs(n, C, h, w, s, L, k, T, vd, io, seed, gain)
    if spoil:
        spoil(d)
    mask = make_mask(n, h * s, w * s, seed + 1) if masked else None
    up = torch.from_numpy(oracle.bicubic(d["lr"].numpy(), s)).double()
    index = d["index"].long().clamp(max=L - 1)
    D, dout, value = d["dict"].double(), d["dout"].double(), d["value"].double()
    wv, wd, named = ro.list_grad(up, index, value, D, dout, mask)
    top = torch.full_like(up, A * float(d["lr"].double().abs().max()))
    mag, _, _ = ro.list_grad(top, index, value, D.abs(), dout.abs(), mask)
    _, dmag, _ = ro.list_grad(top, index, value.abs(), D, dout.abs(), mask)
    bv = (C + 12 + k * k + 12) * U * mag + wv.abs() * torch.finfo(DT[vd]).eps / 2 + (2.0 ** -25 if vd == "f16" else 2.0 ** -140)
    bd = (C + 12 + 12 + named.clamp(max=4096).view(L, 1, 1)) * U * dmag + U * wd.abs() + 2.0 ** -140
    dv, dd = run(d, s, mask, shift=shift)
    assert ((dv.double() - wv).abs() <= bv).all(), f"dvalue: worst {float(((dv.double() - wv).abs() / bv).max()):.2f} of the bound"
    assert ((dd.double() - wd).abs() <= bd).all(), f"ddict: worst {float(((dd.double() - wd).abs() / bd).max()):.2f} of the bound"
    if masked:
        assert (dv[(mask == 0).expand(-1, T, -1, -1)] == 0).all()
    only_v, only_d = run(d, s, mask, (True, False), shift)[0], run(d, s, mask, (False, True), shift)[1]
    assert torch.equal(only_v, dv) and torch.equal(only_d, dd)
    return d


CASES = [
    # (N, C, h, w, scale, L, k, T, value, image, masked)
    (1, 1, 1, 1, 2, 1, 3, 1, "f32", "f32", False),       # four pixels, one atom
    (1, 3, 1, 1, 4, 72, 5, 8, "f16", "f32", False),
    (1, 3, 37, 64, 4, 72, 5, 8, "f16", "f32", False),
    (2, 3, 25, 48, 4, 72, 5, 8, "f16", "f16", True),
    (1, 3, 20, 33, 2, 72, 5, 5, "f16", "f32", True),
    (1, 3, 29, 44, 3, 80, 5, 16, "f16", "f32", False),
    (1, 3, 30, 40, 4, 128, 5, 7, "f16", "f32", False),
    (1, 1, 19, 23, 2, 40, 3, 4, "f32", "f32", False),
    (3, 2, 9, 70, 4, 128, 7, 16, "f16", "f16", True),
    (1, 3, 17, 30, 4, 100, 7, 12, "f16", "f32", False),
    (1, 16, 7, 5, 2, 17, 5, 1, "f32", "f16", False),
    (1, 3, 13, 21, 3, 72, 5, 8, "f32", "f32", True),
    (1, 3, 30, 130, 2, 256, 7, 3, "f32", "f32", False),  # the largest dictionary
    (1, 3, 11, 20, 4, 72, 5, 17, "f16", "f32", False),   # more entries than a matrix-core form of the list takes
    (1, 1, 6, 6, 2, 200, 3, 200, "f32", "f32", True),    # every atom listed
    (1, 3, 40, 50, 3, 16, 3, 2, "f16", "f32", False),
    (1, 4, 12, 33, 2, 72, 5, 8, "f16", "f32", False),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "N%dC%dh%dw%ds%dL%dk%dT%d%s%s%s" % (c[:10] + ("m" if c[10] else "",)))
def test_gradients_against_the_oracle(oracle, case):
    check(oracle, *case, seed=sum(case[:8]))


@pytest.mark.parametrize("gain", [2.0 ** -26, 2.0 ** -14, 2.0 ** 12])
@pytest.mark.parametrize("k,vd", [(5, "f16"), (3, "f32"), (7, "f16")])
def test_small_and_large_gradients_of_the_image(oracle, k, vd, gain):
    """A mean over a frame sends 1e-7 back, a scaled loss 1e3; with fp16 values a response then has its type's range."""
    if vd == "f16":
        gain = max(gain, 2.0 ** -14) if gain < 1 else 2.0 ** 8
    check(oracle, 1, 3, 12, 40, 4, 72, k, 8, vd, "f32", seed=5, gain=gain)


def test_gradients_of_very_different_sizes_in_one_image(oracle):
    """A few pixels send back a million times what the rest does: the rest keeps its precision relative to its own tile row's
    share of ddict only, its dvalue to its own magnitudes."""
    def spoil(d):
        d["dout"] *= 2.0 ** -20
        d["dout"][..., 7, 11] *= 2.0 ** 20
    d = inputs(1, 3, 16, 40, 4, 72, 5, 8, "f32", "f32", 9)
    spoil(d)
    check(oracle, 1, 3, 16, 40, 4, 72, 5, 8, "f32", "f32", seed=9, spoil=spoil)


@pytest.mark.parametrize("k,L,vd", [(5, 72, "f16"), (3, 40, "f16"), (7, 100, "f16"), (5, 72, "f32")])
@pytest.mark.parametrize("small", [0.0, 2.0 ** -60])
def test_runs_of_pixels_that_send_back_nothing_or_little(oracle, k, L, vd, small):
    """Every other run of 32 pixels has a gradient of (nearly) 0 beside large ones, and atoms of its own: the power of two that a
    wavefront's sums are held under goes down and up again, and the sums with it."""
    def spoil(d):
        x = torch.arange(d["dout"].shape[3]) // 32 % 2 == 1
        d["dout"][..., x] *= small
        d["dout"][:, :, 5:8] *= small
        half = L // 2
        d["index"] = torch.where(x, d["index"] % half, d["index"] % (L - half) + half).to(torch.uint8)
    check(oracle, 1, 3, 20, 48, 4, L, k, 8, vd, "f32", seed=21, gain=256.0, spoil=spoil)


@pytest.mark.parametrize("vd", ["f16", "f32"])
def test_an_atom_listed_twice_gets_both_terms_and_large_indices_stay_inside(oracle, vd):
    def twice(d):
        d["index"][:, 3] = d["index"][:, 0]
        d["index"][:, 5, :4] = 255
    check(oracle, 1, 3, 11, 37, 4, 72, 5, 8, vd, "f32", seed=13, spoil=twice)


@pytest.mark.parametrize("vd", ["f16", "f32"])
def test_tensors_at_odd_addresses(oracle, vd):
    for shift in (1, 3):
        check(oracle, 1, 3, 13, 36, 4, 72, 5, 6, vd, "f16", True, seed=14, shift=shift)


def test_random_shapes(oracle):
    g = torch.Generator().manual_seed(2303)
    pick = lambda *v: v[int(torch.randint(len(v), (1,), generator=g))]
    num = lambda lo, hi: int(torch.randint(lo, hi + 1, (1,), generator=g))
    for at in range(30):
        L = pick(72, 72, num(1, 40), num(73, 128), num(129, 256))
        args = (pick(1, 1, 2), pick(1, 3, 3, num(1, 5)), num(1, 24), num(1, 40), pick(2, 3, 4), L, pick(3, 5, 5, 7),
                min(L, pick(1, 4, 8, num(1, 16), num(1, 20))), pick("f16", "f16", "f32"), pick("f32", "f16"), pick(True, False))
        print(at, args, flush=True)
        check(oracle, *args, seed=3000 + at)


def test_padding_is_not_looked_at(oracle):
    d = inputs(1, 3, 9, 30, 4, 72, 5, 8, "f16", "f32", 17)
    mask = make_mask(1, 36, 120, 18)
    clean = run(d, 4, mask)
    off = (mask == 0)
    d["dout"] = torch.where(off, torch.full_like(d["dout"], float("nan")), d["dout"])
    d["value"] = torch.where(off, torch.full_like(d["value"], float("inf")), d["value"])
    for a, b in zip(clean, run(d, 4, mask)):
        assert torch.equal(a, b)


def test_empty_calls_write_zeros():
    d = inputs(1, 3, 4, 4, 2, 72, 5, 8, "f16", "f32", 19)
    e = {name: (t if name == "dict" else t[:0]) for name, t in d.items()}
    dd = torch.full((72, 5, 5), 7.0, device=DEV)
    sr.sr_dict_assemble_list_grad(*(e[x].to(DEV) for x in ("lr", "index", "value", "dict")), 72, 5, 2, 3, 8, None, e["dout"].to(DEV), None, dd)
    torch.cuda.synchronize()
    assert not dd.any()


def test_a_frame_of_many_tiles(oracle):
    """A 1080p frame: every workgroup walks many tiles and hands its sums on several times.  Errors in ddict do not add up."""
    n, C, h, w, s, L, k, T = 1, 3, 270, 480, 4, 72, 5, 8
    g = torch.Generator(device=DEV).manual_seed(3)
    H, W = h * s, w * s
    index = torch.rand((n, L, H, W), device=DEV, generator=g).topk(T, dim=1).indices
    value = torch.rand((n, T, H, W), device=DEV, generator=g).half()
    lr, D = torch.rand((n, C, h, w), device=DEV, generator=g), torch.randn((L, k, k), device=DEV, generator=g) / k
    dout = torch.randn((n, C, H, W), device=DEV, generator=g)
    dv, dd = torch.empty_like(value), torch.empty_like(D)
    sr.sr_dict_assemble_list_grad(lr, index.to(torch.uint8), value, D, L, k, s, C, T, None, dout, dv, dd)
    again_v, again_d = torch.empty_like(value), torch.empty_like(D)
    sr.sr_dict_assemble_list_grad(lr, index.to(torch.uint8), value, D, L, k, s, C, T, None, dout, again_v, again_d)
    torch.cuda.synchronize()
    assert torch.equal(dv, again_v) and torch.equal(dd, again_d), "the result changes from run to run"
    up = torch.from_numpy(oracle.bicubic(lr.cpu().numpy(), s)).to(DEV).double()
    pad = torch.nn.functional.pad(up, (2, 2, 2, 2), mode="replicate")
    E = torch.stack([(pad[:, :, i // k:i // k + H, i % k:i % k + W] * dout.double()).sum(1) for i in range(k * k)], 1).reshape(k * k, -1)
    phi = torch.zeros((L, H * W), device=DEV, dtype=torch.float64).scatter_add_(0, index.reshape(T, -1), value.double().reshape(T, -1))
    want = phi @ E.t().contiguous()
    size = phi @ (A * dout.double().abs().sum(1).reshape(-1, 1)).expand(-1, k * k).contiguous()
    # runs of 4096 pixels at most, an atom named by every ninth: 456 terms a run on average
    assert ((dd.double().reshape(L, -1) - want).abs() <= (C + 24 + 600) * U * size).all()
    assert float((dd.double().reshape(L, -1) - want).norm() / want.norm()) <= 4e-6
    response = (D.reshape(L, -1).double() @ E).gather(0, index.reshape(T, -1))
    assert float((dv.double().reshape(T, -1) - response).norm() / response.norm()) <= 2.0 ** -11


@pytest.mark.parametrize("k,T,vd", [(3, 3, "f32"), (5, 8, "f16")])
def test_errors_do_not_add_up_where_the_gradients_cancel(oracle, k, T, vd):
    """Gradients of either sign over 900 000 pixels: the sum is a thousandth of its terms' magnitudes, an error of one sign in every
    product would be as large.  E and the values have 22 bits, what is left out of their product is 2^-22 of it, the fp32 sums
    of a run round 16 times by 2^-24: each at random beside the terms, so that the sum keeps 4 x 2^-22."""
    n, C, h, w, s, L = 3, 3, 101, 179, 4, 72
    g = torch.Generator(device=DEV).manual_seed(52)
    H, W = h * s, w * s
    value, index = torch.rand((n, L, H, W), device=DEV, generator=g).topk(T, dim=1)
    value = (value / value.sum(1, keepdim=True)).to(DT[vd])
    lr, D = torch.rand((n, C, h, w), device=DEV, generator=g), torch.randn((L, k, k), device=DEV, generator=g) / k
    dout = torch.randn((n, C, H, W), device=DEV, generator=g) / 64
    dd = torch.empty_like(D)
    sr.sr_dict_assemble_list_grad(lr, index.to(torch.uint8), value, D, L, k, s, C, T, None, dout, None, dd)
    r = k // 2
    pad = torch.nn.functional.pad(torch.from_numpy(oracle.bicubic(lr.cpu().numpy(), s)).to(DEV).double(), (r, r, r, r), mode="replicate")
    want = torch.zeros((L, k * k), device=DEV, dtype=torch.float64)
    for b in range(n):
        E = torch.stack([(pad[b, :, i // k:i // k + H, i % k:i % k + W] * dout[b].double()).sum(0) for i in range(k * k)], 0).reshape(k * k, -1)
        phi = torch.zeros((L, H * W), device=DEV, dtype=torch.float64).scatter_add_(0, index[b].reshape(T, -1), value[b].double().reshape(T, -1))
        want += phi @ E.t().contiguous()
    assert float((dd.double().reshape(L, -1) - want).norm() / want.norm()) <= 4 * 2.0 ** -22

"""Gradient of the per-pixel list form where operands differ in size, against the 64-bit oracle: bounds as in test_gpu_list_grad.py, an atom's
ddict against the magnitudes of its own terms, a response against its own atom's."""
import pytest
import torch

import paper_2303_08999_amd as sr
from test_gpu_list_grad import DEV, DT, U, check, run

pytestmark = pytest.mark.gpu


def test_a_run_of_pixels_owes_nothing_to_the_run_before():
    """A wavefront hands its sums on after 4096 pixels.  Those of the next ones send back 2^-95 of what the first did, to an atom of their
    own, and all of them alike: they keep their bits.  (An image of ones has E = dout in every place; weights of scale 2 are exact.)"""
    grid = min(512, 2 * torch.cuda.get_device_properties(0).multi_processor_count)
    first, W = 32 * 8 * grid, 64                             # rows of 64 pixels: a tile of 8 of them a workgroup, 32 times over
    H = first + 2 * 8 * grid
    g = torch.Generator(device=DEV).manual_seed(1)
    lr = torch.ones((1, 1, H // 2, W // 2), device=DEV)
    dout = torch.ones((1, 1, H, W), device=DEV)
    dout[:, :, first:] = 2.0 ** -95 * (1 + torch.rand((1, 1, H - first, W), device=DEV, generator=g))
    index = torch.zeros((1, 1, H, W), device=DEV, dtype=torch.uint8)
    index[:, :, first:] = 1
    dd = torch.empty((2, 3, 3), device=DEV)
    sr.sr_dict_assemble_list_grad(lr, index, torch.ones((1, 1, H, W), device=DEV, dtype=torch.float16),
                                  torch.ones((2, 3, 3), device=DEV), 2, 3, 2, 1, 1, None, dout, None, dd)
    want = torch.stack([dout[0, 0, :first].double().sum(), dout[0, 0, first:].double().sum()]).view(2, 1, 1).expand(2, 3, 3)
    assert ((dd.double() - want).abs() <= (1 + 24 + 4096) * U * want).all()


@pytest.mark.parametrize("C,k,L", [(1, 5, 72), (3, 3, 40), (1, 7, 100)])
def test_gradients_near_the_top_of_the_type(oracle, C, k, L):
    """An image's gradient of 2^112 and small atoms: responses have a place in fp32, and so has everything on the way to them."""
    def spoil(d):
        d["dict"] *= 2.0 ** -7
    check(oracle, 1, C, 10, 33, 2, L, k, 8, "f32", "f32", seed=31, gain=2.0 ** 112, spoil=spoil)


@pytest.mark.parametrize("C,k,L,T", [(3, 5, 72, 8), (1, 3, 40, 4), (1, 7, 100, 12), (3, 5, 128, 3)])
def test_weak_atoms_beside_strong_ones(oracle, C, k, L, T):
    """Atoms of a dictionary that is being learnt start at nothing: a response has its precision beside its own atom, not the largest."""
    def spoil(d):
        d["dict"] *= 2.0 ** -(9.0 * (torch.arange(L) % 8)).view(L, 1, 1)
    check(oracle, 1, C, 13, 37, 2, L, k, T, "f32", "f32", seed=33, spoil=spoil)


def apart(d, groups, part):
    """Lists of different atoms; pixels (and entries) of a part have atoms that no other part has."""
    L, (n, T, H, W) = d["dict"].shape[0], d["index"].shape
    size = L // groups
    t, y, x = torch.arange(T).view(T, 1, 1), torch.arange(H).view(H, 1), torch.arange(W)
    d["index"] = (part * size + (t + 3 * y + 5 * x) % size).expand(n, T, H, W).to(torch.uint8).contiguous()


@pytest.mark.parametrize("ratios", [(2.0 ** -24,), (2.0 ** -26, 2.0 ** -32, 2.0 ** -70), (2.0 ** -12, 2.0 ** -15, 2.0 ** -18), (2.0 ** -95,)],
                         ids=["24", "26_32_70", "12_15_18", "95"])
@pytest.mark.parametrize("C,k,L,T,vd", [(3, 5, 72, 8, "f16"), (3, 5, 72, 8, "f32"), (1, 3, 40, 4, "f16"), (1, 3, 40, 9, "f32"),
                                        (3, 7, 128, 16, "f16"), (3, 7, 100, 12, "f32"), (1, 5, 128, 5, "f16")])
def test_quiet_pixels_among_loud_ones(oracle, C, k, L, T, vd, ratios):
    """Single pixels send back next to nothing beside their neighbours, to atoms that nobody else names."""
    def spoil(d):
        part = torch.zeros(d["dout"].shape[3], dtype=torch.long)
        for i, r in enumerate(ratios):
            part[5 + 7 * i::32] = i + 1
            d["dout"][..., 5 + 7 * i::32] *= r
        apart(d, len(ratios) + 1, part)
    check(oracle, 1, C, 20, 50, 2, L, k, T, vd, "f32", seed=41, gain=16.0, spoil=spoil)


@pytest.mark.parametrize("vd", ["f16", "f32"])
def test_quiet_pixels_that_list_an_atom_twice(oracle, vd):
    def spoil(d):
        part = torch.zeros(d["dout"].shape[3], dtype=torch.long)
        for i, r in enumerate((2.0 ** -26, 2.0 ** -50)):
            part[5 + 7 * i::32] = i + 1
            d["dout"][..., 5 + 7 * i::32] *= r
        apart(d, 3, part)
        d["index"][:, 3] = d["index"][:, 0]
        d["index"][:, 5, ::2] = d["index"][:, 0, ::2]
    check(oracle, 1, 3, 20, 50, 2, 72, 5, 8, vd, "f32", seed=43, spoil=spoil)


@pytest.mark.parametrize("quiet", [False, True])
@pytest.mark.parametrize("C,k,L,T", [(3, 5, 72, 8), (1, 3, 80, 16), (3, 7, 128, 8)])
def test_small_values_beside_large_ones(oracle, C, k, L, T, quiet):
    """A steep softmax's list: each place holds a small part of the place before, and has atoms of its own."""
    def spoil(d):
        d["value"] = d["value"].abs() + 0.1
        d["value"] *= 2.0 ** -(90.0 * torch.arange(T) / (T - 1)).view(1, T, 1, 1)
        apart(d, T, torch.arange(T).view(T, 1, 1))
        if quiet:
            d["dout"][..., 3::5] *= 2.0 ** -20
            d["dout"][..., 4::32] = 0
    check(oracle, 1, C, 20, 50, 2, L, k, T, "f32", "f32", seed=47, spoil=spoil)


def test_an_atom_listed_twice_with_values_of_very_different_sizes(oracle):
    def spoil(d):
        d["index"][:, 4:] = d["index"][:, :4]
        d["value"][:, 4:] *= 2.0 ** -50
        d["value"][:, 2:4] = 0
    check(oracle, 1, 3, 20, 50, 2, 72, 5, 8, "f32", "f32", seed=53, spoil=spoil)


@pytest.mark.parametrize("k", [3, 5, 7])
def test_products_of_two_numbers(k):
    """An image of ones (E = dout in every place), atoms of one tap, atoms named once: every result is one product.  Of either operand
    two fp16 numbers hold all but 2^-23, 2 u; the product of the low parts, 2^-11 each, may be left out: 4 u; a matrix instruction's sum
    rounds by 2 u at most, of which the last is all that counts: 10 u.  With fp32 values ddict has the same, E beside the low part
    of a value, 2^-11, within 2^-13: 1 u, and a rounding at the end: 12 u.  fp16 values are whole: 5 u."""
    L, h, w, T = 128, 16, 40, 2
    H, W = 2 * h, 2 * w
    for seed in range(4):
        g = torch.Generator().manual_seed(70 + seed)
        sign = lambda shape: torch.randint(0, 2, shape, generator=g) * 2 - 1
        D = torch.zeros((L, k * k))
        D[torch.arange(L), torch.arange(L) * 7 % (k * k)] = (1 + torch.rand(L, generator=g)) * sign((L,))
        index = ((torch.arange(H * W) * 5).view(1, 1, H, W) + torch.arange(T).view(1, T, 1, 1) * 64) % L
        d = {"lr": torch.ones((1, 1, h, w)), "index": index.to(torch.uint8), "dict": D.view(L, k, k),
             "dout": (1 + torch.rand((1, 1, H, W), generator=g)) * sign((1, 1, H, W))}
        for vd in ("f32", "f16"):
            value = ((1 + torch.rand((1, T, H, W), generator=g)) * sign((1, T, H, W)))
            once = torch.zeros((1, T, H, W))
            once.view(T, -1)[0, torch.arange(L) * 13 + seed] = 1       # 13 is prime to L: one pixel for every atom
            d["value"] = (value * once).to(torch.float16 if vd == "f16" else torch.float32)
            dv, dd = run(d, 2)
            tap = D.sum(1).double()[index]
            want = tap * d["dout"].double()
            if vd == "f32":
                assert float(((dv.double() - want).abs() / want.abs()).max()) <= 10 * U
            want = torch.zeros(L, dtype=torch.float64).scatter_add_(0, index.reshape(-1), (d["value"].double() * d["dout"].double()).reshape(-1))
            assert (want != 0).all()
            err = (dd.double().view(L, -1) - want.view(L, 1)).abs() / want.abs().view(L, 1)
            assert float(err.max()) <= (12 if vd == "f32" else 5) * U, vd


@pytest.mark.parametrize("C,k,L,T,vd", [(3, 5, 72, 8, "f16"), (1, 3, 40, 16, "f32"), (3, 7, 128, 16, "f16"), (1, 7, 90, 5, "f32")])
def test_one_atom_in_every_place_of_a_list(oracle, C, k, L, T, vd):
    """Some pixels list one atom alone, some two in turn; quiet pixels, pixels of zeros and padding among them."""
    def spoil(d):
        d["index"][:] = torch.where(torch.arange(d["index"].shape[3]) % 3 == 0, d["index"][:, :1], d["index"])
        d["index"][:, 2::2, ::3] = d["index"][:, :1, ::3]
        d["dout"][..., 4::32] *= 2.0 ** -30
        d["dout"][..., 9::32] = 0
    check(oracle, 1, C, 20, 50, 2, L, k, T, vd, "f32", True, seed=59, spoil=spoil)


@pytest.mark.parametrize("C,k,L,T", [(3, 5, 72, 8), (1, 3, 40, 4), (3, 7, 128, 16)])
def test_small_fp16_values_beside_large_ones(oracle, C, k, L, T):
    """Down to fp16's subnormal numbers, which are taken as they are: each place of a list has atoms of its own."""
    def spoil(d):
        d["value"] = ((d["value"].float().abs() + 0.1) * 2.0 ** -(22.0 * torch.arange(T) / (T - 1)).view(1, T, 1, 1)).half()
        apart(d, T, torch.arange(T).view(T, 1, 1))
    check(oracle, 1, C, 20, 50, 2, L, k, T, "f16", "f32", seed=61, spoil=spoil)


@pytest.mark.parametrize("k,vd", [(3, "f32"), (5, "f16"), (5, "f32"), (7, "f32")])
def test_gradients_near_the_bottom_of_the_type(oracle, k, vd):
    """An image's gradient of 2^-118: results keep their bits down to where fp32 ends (fp16 values: dvalue is 0, ddict is not)."""
    check(oracle, 1, 3, 10, 33, 2, 72, k, 8, vd, "f32", seed=67, gain=2.0 ** -118)


@pytest.mark.parametrize("n,w,k,T,vd", [(1, 450000, 3, 3, "f32"), (1, 450000, 5, 8, "f16"), (400, 600, 5, 8, "f16")])
def test_errors_do_not_add_up_in_images_of_two_rows(oracle, n, w, k, T, vd):
    """As test_errors_do_not_add_up_where_the_gradients_cancel has it, 900 000 pixels and 4 x 2^-22 of the norm, but of a tile's rows two
    are there, one wavefront's."""
    C, s, L, H, W = 1, 2, 72, 2, 2 * w
    g = torch.Generator(device=DEV).manual_seed(1)
    value, index = torch.rand((n, L, H, W), device=DEV, generator=g).topk(T, dim=1)
    value = (value / value.sum(1, keepdim=True)).to(DT[vd])
    lr, D = torch.rand((n, C, 1, w), device=DEV, generator=g), torch.randn((L, k, k), device=DEV, generator=g) / k
    dout = torch.randn((n, C, H, W), device=DEV, generator=g) / 64
    dd = torch.empty_like(D)
    sr.sr_dict_assemble_list_grad(lr, index.to(torch.uint8), value, D, L, k, s, C, T, None, dout, None, dd)
    r = k // 2
    pad = torch.nn.functional.pad(torch.from_numpy(oracle.bicubic(lr.cpu().numpy(), s)).to(DEV).double(), (r, r, r, r), mode="replicate")
    E = torch.stack([(pad[:, :, i // k:i // k + H, i % k:i % k + W] * dout.double()).sum(1) for i in range(k * k)], 0).reshape(k * k, -1)
    phi = torch.zeros((L, n * H * W), device=DEV, dtype=torch.float64)
    phi.scatter_add_(0, index.permute(1, 0, 2, 3).reshape(T, -1), value.double().permute(1, 0, 2, 3).reshape(T, -1))
    want = phi @ E.t().contiguous()
    assert float((dd.double().reshape(L, -1) - want).norm() / want.norm()) <= 4 * 2.0 ** -22

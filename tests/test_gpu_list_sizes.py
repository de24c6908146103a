"""The router and the list form's gradient where offsets come close to 32 bits, and on a 4K frame: what a sample of pixels and sums in 64 bits
on the GPU say.  (Sizes: the largest that the kernels with 32-bit offsets take, and the next that they leave to the others.)"""
import pytest
import torch

import paper_2303_08999_amd as sr
from test_gpu_list_grad import A, U

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dt,H", [(torch.float16, 8191), (torch.float16, 8192), (torch.float32, 4095)])
def test_router_of_planes_up_to_4_gb_apart(dt, H):
    """32 planes of fp16 logits are just below 2^32 bytes at 8191 rows of 8192, and 2^32 at 8192; of fp32 ones at 4095.  73 atoms: four lanes a
    pixel, the last of them beyond the atoms."""
    L, T, W = 73, 2, 8192
    z = torch.empty((1, L, H, W), device=DEV, dtype=dt)
    g = torch.Generator(device=DEV).manual_seed(7)
    for l in range(L):
        z[0, l] = torch.randn((H, W), device=DEV, generator=g)
    index, value = torch.empty((1, T, H, W), device=DEV, dtype=torch.uint8), torch.empty((1, T, H, W), device=DEV)
    sr.sr_list_route(z, L, 1, T, sr.SR_ROUTE_SOFTMAX, sr.SR_COEFF_PLANAR, None, index, value)
    dvalue, dz = torch.randn((1, T, H, W), device=DEV, generator=g), torch.empty_like(z)
    sr.sr_list_route_grad(z, index, dvalue, L, 1, T, sr.SR_ROUTE_SOFTMAX, sr.SR_COEFF_PLANAR, None, None, None, dz)
    torch.cuda.synchronize()
    for rows in (slice(0, 8), slice(H // 2 - 4, H // 2 + 4), slice(H - 8, H)):
        x = z[0, :, rows].double()
        order = torch.sort(x, dim=0, descending=True, stable=True).indices[:T]
        assert torch.equal(index[0, :, rows].long(), order)
        p = torch.softmax(x, 0)
        want = p.gather(0, order)
        # (73 + 1.75 x + 8) u, x at most 12 / ln 2 for 73 Gaussian numbers of 67 million pixels
        assert ((value[0, :, rows].double() - want).abs() <= 120 * U * want).all()
        G = torch.zeros_like(x).scatter_(0, order, dvalue[0, :, rows].double())
        want = p * (G - (p * G).sum(0))
        size = p * (G.abs() + (p * G.abs()).sum(0))
        step = torch.finfo(dt).eps / 2 * want.abs() + (2.0 ** -25 if dt == torch.float16 else 0.0)
        assert ((dz[0, :, rows].double() - want).abs() <= 360 * U * size + step).all()


@pytest.mark.parametrize("H", [8190, 8192])
@pytest.mark.parametrize("vd", [torch.float32, torch.float16])
def test_list_gradient_of_lists_up_to_4_gb(H, vd):
    """16 entries of 8190 rows of 8192 pixels are just below 2^30; 8192 rows are the kernel's that takes every case.  An image of ones has E = dout in every place, so that ddict is a weighted count of the atoms and dvalue an atom's sum times dout."""
    T, L, k, W = 16, 8, 3, 8192
    g = torch.Generator(device=DEV).manual_seed(9)
    s = 2
    lr = torch.ones((1, 1, H // s, W // s), device=DEV)
    D = torch.randn((L, k, k), device=DEV, generator=g)
    dout = torch.randn((1, 1, H, W), device=DEV, generator=g)
    index, value = torch.empty((1, T, H, W), device=DEV, dtype=torch.uint8), torch.empty((1, T, H, W), device=DEV, dtype=vd)
    want, size = torch.zeros(L, device=DEV, dtype=torch.float64), torch.zeros(L, device=DEV, dtype=torch.float64)
    for t in range(T):
        atoms = (torch.arange(L, device=DEV) * 3 + t * 5) % L                  # of every L pixels that follow one another
        index[0, t] = atoms.repeat(W // L)
        value[0, t] = torch.rand((H, W), device=DEV, generator=g)
        w = value[0, t].double() * dout[0, 0].double()
        want[atoms] += w.view(-1, L).sum(0)
        size[atoms] += w.abs().view(-1, L).sum(0)
    dvalue, ddict = torch.empty_like(value), torch.empty_like(D)
    sr.sr_dict_assemble_list_grad(lr, index, value, D, L, k, s, 1, T, None, dout, dvalue, ddict)
    torch.cuda.synchronize()
    # 2 entries of a list name an atom: 8192 terms a run
    assert ((ddict.double().view(L, -1) - want.view(L, 1)).abs() <= (25 + 8192) * U * size.view(L, 1)).all()
    sums, mags = D.double().sum((1, 2)), D.double().abs().sum((1, 2))
    for rows in (slice(0, 4), slice(H // 2, H // 2 + 4), slice(H - 4, H)):
        at, e = index[0, :, rows].long(), dout[0, :, rows].double()
        off = (dvalue[0, :, rows].double() - sums[at] * e).abs()
        assert (off <= (25 + 9) * U * mags[at] * e.abs() + torch.finfo(vd).eps / 2 * (sums[at] * e).abs() + 2.0 ** -25).all()


def test_list_gradient_of_a_4k_frame(oracle):
    """A 4K frame of 8 entries of 72."""
    C, h, w, s, L, k, T = 3, 540, 960, 4, 72, 5, 8
    g = torch.Generator(device=DEV).manual_seed(4)
    H, W = h * s, w * s
    value, index = torch.rand((1, L, H, W), device=DEV, generator=g).topk(T, dim=1)
    value = (value / value.sum(1, keepdim=True)).half()
    lr, D = torch.rand((1, C, h, w), device=DEV, generator=g), torch.randn((L, k, k), device=DEV, generator=g) / k
    dout = torch.randn((1, C, H, W), device=DEV, generator=g)
    dv, dd = torch.empty_like(value), torch.empty_like(D)
    sr.sr_dict_assemble_list_grad(lr, index.to(torch.uint8), value, D, L, k, s, C, T, None, dout, dv, dd)
    up = torch.from_numpy(oracle.bicubic(lr.cpu().numpy(), s)).to(DEV).double()
    pad = torch.nn.functional.pad(up, (2, 2, 2, 2), mode="replicate")
    want, size = torch.zeros((L, k * k), device=DEV, dtype=torch.float64), torch.zeros((L, 1), device=DEV, dtype=torch.float64)
    for y in range(0, H, 240):
        E = torch.stack([(pad[:, :, y + i // k:y + i // k + 240, i % k:i % k + W] * dout[:, :, y:y + 240].double()).sum(1) for i in range(k * k)], 1)
        E = E.reshape(k * k, -1)
        at, v = index[:, :, y:y + 240].reshape(T, -1), value[:, :, y:y + 240].double().reshape(T, -1)
        phi = torch.zeros((L, 240 * W), device=DEV, dtype=torch.float64).scatter_add_(0, at, v)
        want += phi @ E.t().contiguous()
        size += phi @ (A * dout[:, :, y:y + 240].double().abs().sum(1).reshape(-1, 1))
        response = (D.reshape(L, -1).double() @ E).gather(0, at)
        off = (dv[:, :, y:y + 240].double().reshape(T, -1) - response).abs()
        mag = (D.reshape(L, -1).double().abs() @ E.abs()).gather(0, at)
        top = A * dout[:, :, y:y + 240].double().abs().sum(1).reshape(1, -1) * D.double().abs().sum((1, 2))[at]
        assert (off <= (C + 12 + k * k + 12) * U * torch.maximum(mag, top) + 2.0 ** -11 * response.abs() + 2.0 ** -25).all()
    # an atom is named by every ninth pixel: 456 terms a run on average
    assert ((dd.double().reshape(L, -1) - want).abs() <= (C + 24 + 600) * U * size).all()
    assert float((dd.double().reshape(L, -1) - want).norm() / want.norm()) <= 4e-6

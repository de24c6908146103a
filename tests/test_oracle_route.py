"""The 64-bit router: its definitions at hand-checked pixels, its gradients against central differences."""
import pytest
import torch

from oracle import route_oracle as ro

INF = float("inf")


def pixels(rows):
    """[pixels][L] -> [1][L][1][pixels]"""
    return torch.tensor(rows, dtype=torch.float64).t().reshape(1, len(rows[0]), 1, len(rows))


def test_ties_masks_and_empty_rows():
    z = pixels([[1.0, 2.0, 2.0, 0.0], [-INF, -INF, 3.0, -INF], [-INF] * 4, [0.0, -0.0, -1.0, 0.0]])
    index, value = ro.route(z, 3, ro.SOFTMAX)
    assert index[0, :, 0].t().tolist() == [[1, 2, 0], [2, 0, 1], [0, 1, 2], [0, 1, 3]]
    assert value[0, :, 0, 1].tolist() == [1.0, 0.0, 0.0] and value[0, :, 0, 2].tolist() == [0.0, 0.0, 0.0]
    _, chosen = ro.route(z, 3, ro.CHOSEN)
    assert torch.allclose(chosen[0, :, 0, 3], torch.full((3,), 1 / 3, dtype=torch.float64))
    counts, share, loss = ro.balance(z, 3)
    assert counts.tolist() == [2, 2, 2, 1, 3]                  # the empty pixel and the masked atoms are not counted
    assert abs(float(share.sum()) - 1.0) < 1e-12


def test_even_load_has_loss_one():
    z = pixels([[5.0 if l == i else 0.0 for l in range(6)] for i in range(6)])
    assert abs(float(ro.balance(z, 1)[2][0]) - 1.0) < 1e-12


@pytest.mark.parametrize("kind", [ro.SOFTMAX, ro.CHOSEN, ro.VALUES])
@pytest.mark.parametrize("masked", [False, True])
def test_gradient_against_differences(kind, masked):
    g = torch.Generator().manual_seed(5)
    z = torch.randn((2, 7, 2, 3), generator=g, dtype=torch.float64)
    if kind != ro.VALUES:
        z[0, 2, 1, 1] = -INF
    mask = (torch.rand((2, 1, 2, 3), generator=g) < 0.6).to(torch.uint8) if masked else None
    index = ro.order(z, 3)
    dv = torch.randn((2, 3, 2, 3), generator=g, dtype=torch.float64)
    counts, _, _ = ro.balance(z, 3, mask)
    dloss = torch.tensor([0.7, -0.3], dtype=torch.float64)
    counts, dloss = (None, None) if kind == ro.VALUES else (counts, dloss)
    dz, _ = ro.route_grad(z, index, kind, dv, counts, dloss, mask)
    h = 1e-5
    for at in range(z.numel()):
        up, down = z.clone(), z.clone()
        up.view(-1)[at] += h
        down.view(-1)[at] -= h
        diff = (ro.losses(up, index, kind, dv, counts, dloss, mask) - ro.losses(down, index, kind, dv, counts, dloss, mask)) / (2 * h)
        # third derivatives of these sums are of order one: h^2, and 2^-53 of the sum over h
        assert abs(float(diff - dz.view(-1)[at])) < 1e-8


def test_list_gradient_against_differences():
    g = torch.Generator().manual_seed(6)
    up = torch.rand((2, 2, 3, 4), generator=g, dtype=torch.float64)
    D = torch.randn((5, 3, 3), generator=g, dtype=torch.float64)
    index = torch.stack([torch.randperm(5, generator=g)[:3] for _ in range(24)]).reshape(2, 3, 4, 3).permute(0, 3, 1, 2).contiguous()
    value, dout = torch.randn((2, 3, 3, 4), generator=g, dtype=torch.float64), torch.randn((2, 2, 3, 4), generator=g, dtype=torch.float64)

    def image(v, d):
        pad = torch.nn.functional.pad(up, (1, 1, 1, 1), mode="replicate")
        F = (v[..., None] * d.reshape(5, 9)[index]).sum(1)                              # [n][H][W][9]
        win = torch.stack([pad[:, :, i // 3:i // 3 + 3, i % 3:i % 3 + 4] for i in range(9)], -1)
        return (win * F[:, None]).sum(-1)

    dv, dd, named = ro.list_grad(up, index, value, D, dout)
    assert int(named.sum()) == index.numel()
    h = 1e-4                                                    # the image is bilinear: differences are exact but for rounding
    for at in range(value.numel()):
        e = torch.zeros_like(value)
        e.view(-1)[at] = h
        diff = ((image(value + e, D) - image(value - e, D)) * dout).sum() / (2 * h)
        assert abs(float(diff - dv.reshape(-1)[at])) < 1e-10
    for at in range(D.numel()):
        e = torch.zeros_like(D)
        e.view(-1)[at] = h
        diff = ((image(value, D + e) - image(value, D - e)) * dout).sum() / (2 * h)
        assert abs(float(diff - dd.reshape(-1)[at])) < 1e-10

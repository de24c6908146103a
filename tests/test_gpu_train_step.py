"""A training step of the coefficient network's last layers through the C ABI: gated block, head, router with its losses, the list form's image,
and all gradients back to features and weights, clipped; against the same step differentiated by torch in 64 bits, the lists' atoms being
constants; and captured into a graph.

Tolerance: fp32 throughout; each of the chain's sums has at most 4608 terms (768 pixels' neighbourhoods, 5 x 5 taps, 72 atoms), so that no
gradient is off by more than a few thousand u = 2^-24 of its terms' magnitudes.  2^-10 of the largest value of each tensor is more than
ten times that; a wrong term is of the size of the tensor's values."""
import numpy as np
import pytest
import torch

import paper_2303_08999_amd as sr
from oracle import layer_oracle as lo

pytestmark = pytest.mark.gpu
DEV = "cuda"
N, C3, h, w, s, L, k, T, C, F = 1, 3, 12, 16, 2, 72, 5, 4, 24, 40
H, W = h * s, w * s


def step(d, ws, out):
    """The calls of one step; everything is written into `out`."""
    PM, SM = sr.SR_COEFF_PIXEL_MAJOR, sr.SR_ROUTE_SOFTMAX
    sr.sr_layer_gated(d["x"], d["wg"], d["bg"], sr.SR_ACT_SILU, out["hidden"])
    sr.sr_layer_linear(out["hidden"], d["wh"], d["bh"], sr.SR_ACT_NONE, None, out["logits"])
    sr.sr_list_route_balance(out["logits"], L, 1, T, SM, PM, None, out["index"], out["value"], out["counts"], out["share"], out["loss"],
                             workspace=ws["route"])
    sr.sr_dict_assemble_list(d["lr"], out["index"], out["value"], d["dict"], L, k, s, C3, T, out["image"])
    sr.sr_dict_assemble_list_grad(d["lr"], out["index"], out["value"], d["dict"], L, k, s, C3, T, None, d["dout"], out["dvalue"], out["ddict"],
                                  workspace=ws["list"])
    sr.sr_list_route_grad(out["logits"], out["index"], out["dvalue"], L, 1, T, SM, PM, None, out["counts"], d["dloss"], out["dlogits"])
    sr.sr_layer_linear_grad(out["hidden"], d["wh"], d["bh"], sr.SR_ACT_NONE, out["dlogits"], out["dhidden"], out["dwh"], out["dbh"],
                            workspace=ws["head"])
    sr.sr_layer_gated_grad(d["x"], d["wg"], d["bg"], sr.SR_ACT_SILU, out["dhidden"], out["dx"], out["dwg"], out["dbg"], workspace=ws["gated"])
    grads = [out[n] for n in ("ddict", "dwh", "dbh", "dwg", "dbg")]
    sr.sr_grad_clip(grads, [out["c" + n] for n in ("ddict", "dwh", "dbh", "dwg", "dbg")], d["most"], out["norm"], workspace=ws["clip"])


def make():
    g = torch.Generator().manual_seed(11)
    r = lambda *shape: torch.randn(shape, generator=g)
    d = {"x": r(N, H, W, C), "wg": r(2 * F, C) / C ** 0.5, "bg": r(2 * F) / 8, "wh": r(L, F) / F ** 0.5, "bh": r(L) / 8,
         "lr": torch.rand((N, C3, h, w), generator=g), "dict": r(L, k, k) / k, "dout": r(N, C3, H, W) / 32, "dloss": torch.tensor([0.5, 0.25])}
    d = {n: v.to(DEV) for n, v in d.items()}
    d["most"] = 0.25
    e = lambda *shape, t=torch.float32: torch.full(shape, 9, device=DEV, dtype=t)
    out = {"hidden": e(N, H, W, F), "logits": e(N, H, W, L), "index": e(N, T, H, W, t=torch.uint8), "value": e(N, T, H, W),
           "counts": e(L + 1, t=torch.int64), "share": e(L), "loss": e(2), "image": e(N, C3, H, W), "dvalue": e(N, T, H, W),
           "ddict": e(L, k, k), "dlogits": e(N, H, W, L), "dhidden": e(N, H, W, F), "dwh": e(L, F), "dbh": e(L), "dx": e(N, H, W, C),
           "dwg": e(2 * F, C), "dbg": e(2 * F), "norm": e(2)}
    for n in ("ddict", "dwh", "dbh", "dwg", "dbg"):
        out["c" + n] = torch.empty_like(out[n])
    f = torch.float32
    sizes = {"route": sr.sr_list_route_workspace_bytes(L), "list": sr.sr_dict_assemble_list_grad_workspace_bytes(L, k),
             "head": sr.sr_layer_linear_grad_workspace_bytes(N * H * W, F, L, f, sr.SR_ACT_NONE),
             "gated": sr.sr_layer_gated_grad_workspace_bytes(N * H * W, C, F, f), "clip": sr.sr_grad_clip_workspace_bytes(5)}
    ws = {n: torch.empty(v, device=DEV, dtype=torch.uint8) for n, v in sizes.items()}
    return d, ws, out


def reference(oracle, d, out):
    """The step's gradients by torch in 64 bits."""
    leaf = {n: d[n].cpu().double().requires_grad_() for n in ("x", "wg", "bg", "wh", "bh", "dict")}
    hidden = lo.gated(leaf["x"].reshape(-1, C), leaf["wg"], leaf["bg"], lo.SILU)
    z = lo.linear(hidden, leaf["wh"], leaf["bh"], lo.NONE)
    index = out["index"].cpu().long()[0].reshape(T, -1).t()
    p = torch.softmax(z, 1)
    value = p.gather(1, index)
    up = torch.from_numpy(np.asarray(oracle.bicubic(d["lr"].cpu().numpy(), s))).double()
    pad = torch.nn.functional.pad(up, (k // 2,) * 4, mode="replicate")
    patches = torch.nn.functional.unfold(pad, k).reshape(C3, k * k, H * W)                # [c][tap][pixel]
    filters = (value[:, :, None] * leaf["dict"].reshape(L, k * k)[index]).sum(1)          # [pixel][tap]
    image = torch.einsum("ctp,pt->cp", patches, filters)
    M = H * W
    counts = out["counts"].cpu().double()
    balance = L * (counts[:L] / (M * T) * p.mean(0)).sum()
    lse2 = (torch.logsumexp(z, 1) ** 2).mean()
    total = (image * d["dout"].cpu().double().reshape(C3, -1)).sum() + 0.5 * balance + 0.25 * lse2
    grads = dict(zip(leaf, torch.autograd.grad(total, list(leaf.values()))))
    assert torch.allclose(out["image"].cpu().double().reshape(C3, -1), image.detach(), rtol=0, atol=2e-5 * max(1.0, float(image.detach().abs().max())))
    return grads


def test_a_training_step(oracle):
    d, ws, out = make()
    step(d, ws, out)
    torch.cuda.synchronize()
    order = out["logits"].double().sort(dim=3, descending=True, stable=True).indices[..., :T].permute(0, 3, 1, 2)
    assert torch.equal(out["index"].long(), order)
    grads = reference(oracle, d, out)
    for name, of in (("dx", "x"), ("dwg", "wg"), ("dbg", "bg"), ("dwh", "wh"), ("dbh", "bh"), ("ddict", "dict")):
        want = grads[of]
        err = float((out[name].cpu().double() - want).abs().max())
        assert err <= 2.0 ** -10 * float(want.abs().max()), f"{name}: {err} of {float(want.abs().max())}"
    norm = float(sum((out[n].double() ** 2).sum() for n in ("ddict", "dwh", "dbh", "dwg", "dbg")).sqrt())
    assert norm > d["most"] and abs(float(out["norm"][0]) - norm) <= 1e-6 * norm
    clipped = float(sum((out["c" + n].double() ** 2).sum() for n in ("ddict", "dwh", "dbh", "dwg", "dbg")).sqrt())
    assert abs(clipped - d["most"]) <= 1e-6 * d["most"]


def test_a_step_captured_into_a_graph():
    """Replayed with other features each time, an eager step of the same tensors between the replays."""
    d, ws, out = make()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(d, ws, out)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(d, ws, out)
    first = d["x"].clone()
    _, eager_ws, eager = make()
    for i in range(4):
        d["x"].copy_(first * (1 + i))
        for v in out.values():
            v.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        step(d, eager_ws, eager)
        torch.cuda.synchronize()
        for n in out:
            assert torch.equal(out[n], eager[n]), f"replay {i}: {n}"

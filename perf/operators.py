"""Per-pixel lists, made and trained: what is timed, and the same in plain torch.

A coefficient network hands over L logits for every HR pixel (or for every token: a pixel-major tensor of one row); the
router keeps the `entries` largest as (atom, value) lists, which sr_dict_assemble_list takes; training adds the balance of
the atoms' load and the gradients of both steps.  Four operators: `route` (the lists), `balance` (the lists with the atoms'
counts and the two losses), `route_grad` (gradient of the lists' values and of both losses with respect to the logits) and
`list_grad` (gradient of the list form's image with respect to the lists' values and to the dictionary).

A case is a dict of plain values; `prepare` makes what the caller holds before the call, `run` is the call (or, where
`own` is false, the same in elementary torch operations), `exact` the outputs in 64 bits, the gradients by differentiating
the forward formula.  Sizes are those of the paper's Table I, a 4K frame, images of odd sizes and rows of tokens.
"""
import math

import numpy as np
import torch
import torch.nn.functional as F

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}


def _route(op, n, h, w, scale, L, entries, coeff, value, kind, layout="planar", mask=False):
    return {"op": op, "n": n, "h": h, "w": w, "scale": scale, "L": L, "entries": entries, "coeff": coeff, "value": value,
            "kind": kind, "layout": layout, "mask": mask}


def _list_grad(n, c, h, w, scale, L, k, entries, value, image, mask=False):
    return {"op": "list_grad", "n": n, "c": c, "h": h, "w": w, "scale": scale, "L": L, "k": k, "entries": entries,
            "value": value, "image": image, "mask": mask}


def listed():
    def named(name, case):
        return dict(case, name=name)

    return [
        # one token in a serving loop: nothing but the launch counts
        named("route_token_bf16", _route("route", 1, 1, 1, 1, 72, 8, "bf16", "f32", "chosen", "pixel_major")),
        # Table I's 180 x 320 to 720p, an fp32 network: the lists of one frame
        named("route_720p_f32", _route("route", 1, 180, 320, 4, 72, 8, "f32", "f16", "softmax")),
        # the 4K frame with the whole dictionary, fp16 logits
        named("route_4k_f16", _route("route", 1, 540, 960, 4, 72, 8, "f16", "f16", "softmax")),
        # a long row of tokens over the most atoms there can be, channels-last
        named("route_tokens_bf16", _route("route", 1, 1, 50001, 1, 256, 8, "bf16", "f32", "chosen", "pixel_major")),
        # a training photo of odd size, padded in its batch
        named("balance_odd_photo_f32", _route("balance", 2, 171, 257, 2, 72, 5, "f32", "f32", "softmax", "planar", True)),
        # 1080p at x2 straight from the last convolution of a bfloat16 network
        named("balance_1080p_bf16", _route("balance", 1, 540, 960, 2, 72, 4, "bf16", "f16", "chosen", "pre_shuffle")),
        # the smallest training crops
        named("route_grad_crop_f32", _route("route_grad", 1, 64, 64, 2, 72, 8, "f32", "f32", "softmax")),
        # the 4K frame's logits in training
        named("route_grad_4k_f16", _route("route_grad", 1, 540, 960, 4, 72, 8, "f16", "f16", "softmax")),
        # a batch of tokens in training, channels-last, padded
        named("route_grad_tokens_bf16", _route("route_grad", 4, 1, 8191, 1, 128, 4, "bf16", "f32", "chosen", "pixel_major", True)),
        # a luminance crop
        named("list_grad_crop_f32", _list_grad(1, 1, 64, 64, 2, 72, 5, 8, "f32", "f32")),
        # the 4K frame's lists in training
        named("list_grad_4k_f16", _list_grad(1, 3, 540, 960, 4, 72, 5, 8, "f16", "f32")),
        # a 1080p video frame in fp16 throughout, the large dictionary, padded
        named("list_grad_k7_f16", _list_grad(1, 3, 270, 480, 4, 128, 7, 16, "f16", "f16", True)),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["route", "balance", "route_grad", "list_grad"])
    L = rng.choice([72, 72, rng.randint(16, 128), rng.randint(16, 256)])
    entries = min(L, rng.choice([1, 2, 4, 8, 8, rng.randint(1, 16)]))
    value = rng.choice(["f32", "f16"])
    mask = rng.random() < 0.3
    scale = rng.choice([2, 3, 4])
    most = 3840 * 2160 * 72
    if op == "list_grad":
        k = rng.choice([3, 5, 5, 5, 7])
        L = min(L, 128)
        c = rng.choice([1, 3, 3])
        pixels = log(64 * 64, most // max(72, L * k * k // 25))
    else:
        coeff = rng.choice(["f32", "f16", "bf16"])
        kind = rng.choice(["softmax", "chosen"])
        layout = rng.choice(["planar", "planar", "pixel_major", "pre_shuffle"])
        if layout == "pixel_major":                             # tokens
            return _route(op, rng.randint(1, 4), 1, log(1, 60000), 1, L, entries, coeff, value, kind, layout, mask)
        pixels = log(64 * 64, most * 2 // (L * BYTES[coeff]))
    n = rng.choice([1, 1, 2, 3]) if pixels > 100000 else 1
    aspect = rng.uniform(0.6, 2.4)                              # width over height
    h = max(16, int(math.sqrt(pixels / n / aspect) / scale))
    w = max(16, int(h * aspect))
    if rng.random() < 0.5:                                      # half of the frames have widths that are multiples of 8
        w = (w + 7) // 8 * 8
        h = max(16, h * 15 // 16)
    if op == "list_grad":
        return _list_grad(n, c, h, w, scale, L, k, min(entries, L), value, rng.choice(["f32", "f32", "f16"]), mask)
    return _route(op, n, h, w, scale, L, entries, coeff, value, kind, layout, mask)


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _dictionary(L, k, seed):
    """Gaussian filters of all shapes, each with sum 1; every other one sharpened."""
    rng = np.random.Generator(np.random.PCG64(seed))
    yy, xx = np.mgrid[0:k, 0:k].astype(np.float64) - (k - 1) / 2.0
    atoms = np.empty((L, k, k))
    for l in range(L):
        sx, sy, theta, gain = rng.uniform(0.5, 2.5), rng.uniform(0.5, 2.5), rng.uniform(0.0, math.pi), rng.uniform(0.5, 2.0)
        u, v = math.cos(theta) * xx + math.sin(theta) * yy, -math.sin(theta) * xx + math.cos(theta) * yy
        a = np.exp(-0.5 * ((u / sx) ** 2 + (v / sy) ** 2))
        a /= a.sum()
        if l % 2:
            b = np.exp(-0.5 * (xx * xx + yy * yy) / 9.0)
            a = (1.0 + gain) * a - gain * b / b.sum()
        atoms[l] = a
    return torch.from_numpy(atoms.astype(np.float32)).cuda()


def _mask(case, H, W):
    """Frames of unequal sizes in one batch: what lies right of and below a frame is padding."""
    if not case["mask"]:
        return None
    m = torch.zeros((case["n"], 1, H, W), device="cuda", dtype=torch.uint8)
    for b in range(case["n"]):
        m[b, :, :max(1, H - (b + 1) * H // 9), :max(1, W - (b + 2) * W // 11)] = 1
    return m


def _shape(case):
    return case["n"], case["h"] * case["scale"], case["w"] * case["scale"]


def _inputs(case, seed):
    """What a call reads: the same tensors for `run` and for `exact`."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    n, H, W = _shape(case)
    L, T, s = case["L"], case["entries"], case["scale"]
    vt = DTYPES[case["value"]]
    d = {"mask": _mask(case, H, W)}
    if case["op"] == "list_grad":
        score = torch.rand((n, L, H, W), generator=g, device="cuda", dtype=torch.float32)
        value, index = torch.topk(score, T, dim=1)              # different atoms, decreasing values
        d["index"] = index.to(torch.uint8)
        d["value"] = (value / value.sum(1, keepdim=True)).to(vt)
        it = DTYPES[case["image"]]
        d["lr"] = torch.rand((n, case["c"], case["h"], case["w"]), generator=g, device="cuda").to(it)
        d["dict"] = _dictionary(L, case["k"], seed)
        # the gradient that a scaled loss sends back, of the image's type
        d["dout"] = (torch.randn((n, case["c"], H, W), generator=g, device="cuda") / 64).to(it)
        if d["mask"] is not None:
            d["dout"] = d["dout"] * d["mask"].to(it)
        return d
    ct = DTYPES[case["coeff"]]
    shape = {"planar": (n, L, H, W), "pixel_major": (n, H, W, L), "pre_shuffle": (n, L * s * s, case["h"], case["w"])}
    z = torch.empty(shape[case["layout"]], device="cuda", dtype=ct)
    rows = max(1, (1 << 28) // z[0, 0].numel())
    for b in range(n):
        for at in range(0, z.shape[1], rows):
            part = z[b, at:at + rows]
            part.copy_(torch.randn(part.shape, generator=g, device="cuda") * 1.5)
    d["coeff"] = z
    if case["op"] == "route_grad":
        zp = _planar(case, z)
        order = torch.sort(zp.float(), dim=1, descending=True, stable=True).indices[:, :T]
        d["index"] = order.to(torch.uint8).contiguous()
        d["dvalue"] = (torch.randn((n, T, H, W), generator=g, device="cuda") / 16).to(vt)
        on = torch.ones((n, 1, H, W), device="cuda", dtype=torch.int64) if d["mask"] is None else d["mask"].long()
        counts = torch.zeros(L + 1, device="cuda", dtype=torch.int64)
        counts.index_add_(0, order.reshape(-1), on.expand(-1, T, -1, -1).reshape(-1))
        counts[L] = on.sum()
        d["counts"] = counts
        # weights of the two losses against the image's, both scaled with the loss: of the size of the rest
        d["dloss"] = torch.tensor([0.01, 0.001], device="cuda") * float(n * H * W)
    return d


def prepare(case, seed):
    state = _inputs(case, seed)
    state["case"] = case
    n, H, W = _shape(case)
    L, T = case["L"], case["entries"]
    if case["op"] in ("route", "balance"):
        state["index"] = torch.empty((n, T, H, W), device="cuda", dtype=torch.uint8)
        state["value"] = torch.empty((n, T, H, W), device="cuda", dtype=DTYPES[case["value"]])
    if case["op"] == "balance":
        state["counts"] = torch.empty(L + 1, device="cuda", dtype=torch.int64)
        state["share"] = torch.empty(L, device="cuda")
        state["loss"] = torch.empty(2, device="cuda")
    if case["op"] == "route_grad":
        state["dcoeff"] = torch.empty_like(state["coeff"])
    if case["op"] == "list_grad":
        state["dvalue"] = torch.empty_like(state["value"])
        state["ddict"] = torch.empty_like(state["dict"])
    return state


# ---- the plain form -------------------------------------------------------------------------------------------------
def _planar(case, coeff):
    """[n][L][H][W] from any of the three orders."""
    if case["layout"] == "pixel_major":
        return coeff.permute(0, 3, 1, 2)
    if case["layout"] == "pre_shuffle":
        return F.pixel_shuffle(coeff, case["scale"])
    return coeff


def _stored(case, planar):
    """The inverse of _planar, in the type of the logits."""
    planar = planar.to(DTYPES[case["coeff"]])
    if case["layout"] == "pixel_major":
        return planar.permute(0, 2, 3, 1).contiguous()
    if case["layout"] == "pre_shuffle":
        return F.pixel_unshuffle(planar, case["scale"])
    return planar


def _softmax(z):
    e = torch.exp(z - z.amax(1, keepdim=True))
    return e / e.sum(1, keepdim=True)


def _plain_route(state):
    case, mask = state["case"], state["mask"]
    L, T = case["L"], case["entries"]
    z = _planar(case, state["coeff"]).float() + 0.0             # -0 and +0 are the same logit
    index = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :T]
    p = _softmax(z)
    value = p.gather(1, index)
    if case["kind"] == "chosen":
        value = value / value.sum(1, keepdim=True)
    shown = index
    if mask is not None:
        on = mask.bool()
        shown = torch.where(on, index, torch.arange(T, device=index.device).reshape(1, T, 1, 1))
        value = torch.where(on, value, torch.zeros_like(value))
    lists = shown.to(torch.uint8), value.to(DTYPES[case["value"]])
    if case["op"] == "route":
        return lists
    live = torch.ones_like(z[:, :1]) if mask is None else mask.float()
    M = live.sum(dtype=torch.float64)
    counts = torch.bincount(index.reshape(-1), live.expand(-1, T, -1, -1).reshape(-1).double(), minlength=L)
    share = (p * live).sum(dim=(0, 2, 3), dtype=torch.float64) / M
    top = z.amax(1, keepdim=True)
    lse = top + torch.log(torch.exp(z - top).sum(1, keepdim=True))
    loss = torch.stack([L * (counts / (M * T) * share).sum(), (lse * lse * live).sum(dtype=torch.float64) / M])
    return *lists, torch.cat([counts, M.reshape(1)]).to(torch.int64), share.float(), loss.float()


def _plain_route_grad(state):
    case, mask, counts = state["case"], state["mask"], state["counts"]
    L, T = case["L"], case["entries"]
    z = _planar(case, state["coeff"]).float()
    index, g = state["index"].long(), state["dvalue"].float()
    p = _softmax(z)
    q = p
    if case["kind"] == "chosen":                                # the softmax over the chosen alone
        q = p * torch.zeros_like(p).scatter_(1, index, 1.0)
        q = q / q.sum(1, keepdim=True)
    G = torch.zeros_like(z).scatter_(1, index, g)
    dz = q * (G - (q * G).sum(1, keepdim=True))
    M = counts[L].double()
    f = (counts[:L] / (M * T)).float().reshape(1, L, 1, 1)
    top = z.amax(1, keepdim=True)
    lse = top + torch.log(torch.exp(z - top).sum(1, keepdim=True))
    a, b = (state["dloss"].double() * torch.tensor([float(L), 2.0], device=z.device) / M).float()
    dz = dz + p * (a * (f - (f * p).sum(1, keepdim=True)) + b * lse)
    if mask is not None:
        dz = torch.where(mask.bool(), dz, torch.zeros_like(dz))
    return _stored(case, dz)


def _up_axis(x, scale, dim):
    """Cubic convolution (a = -1/2) along one axis: half-pixel centres, source indices clamped."""
    n = x.shape[dim]
    pos = (torch.arange(n * scale, device=x.device, dtype=torch.float64) + 0.5) / scale - 0.5
    base = torch.floor(pos)
    shape = [1] * x.dim()
    shape[dim] = -1

    def tap(i):
        u = (pos - (base + i)).abs()
        wt = torch.where(u <= 1, (1.5 * u - 2.5) * u * u + 1, ((-0.5 * u + 2.5) * u - 4) * u + 2)
        return wt.to(x.dtype).reshape(shape) * x.index_select(dim, (base + i).clamp(0, n - 1).long())

    return tap(-1) + tap(0) + tap(1) + tap(2)


def _plain_list_grad(state):
    case = state["case"]
    n, H, W = _shape(case)
    L, k, s, T = case["L"], case["k"], case["scale"], case["entries"]
    r = (k - 1) // 2
    dout = state["dout"].float()
    if state["mask"] is not None:
        dout = dout * state["mask"]
    pad = F.pad(_up_axis(_up_axis(state["lr"].float(), s, 2), s, 3), (r, r, r, r), mode="replicate")
    # the gradient of every pixel's filter: its neighbourhood weighted with what the loss sends back, all channels
    E = torch.stack([(pad[:, :, i // k:i // k + H, i % k:i % k + W] * dout).sum(1) for i in range(k * k)], 1)
    pieces = -(-H * W // 4096)                                  # pixels in pieces, for products and sums of no great length

    def split(x):                                               # [n][planes][H][W] -> [n * pieces][planes][4096]
        x = F.pad(x.reshape(n, -1, H * W), (0, pieces * 4096 - H * W))
        return x.reshape(n, -1, pieces, 4096).transpose(1, 2).reshape(n * pieces, -1, 4096)

    E, index = split(E), split(state["index"].long())
    D = state["dict"].reshape(1, L, k * k).expand(n * pieces, -1, -1).contiguous()
    dvalue = torch.bmm(D, E).gather(1, index)
    dvalue = dvalue.reshape(n, pieces, T, 4096).transpose(1, 2).reshape(n, T, -1)[:, :, :H * W].reshape(n, T, H, W)
    phi = torch.zeros((n * pieces, L, 4096), device=E.device).scatter_add_(1, index, split(state["value"].float()))
    ddict = torch.bmm(phi.double(), E.double().transpose(1, 2).contiguous()).sum(0)     # a long sum: in 64 bits
    return dvalue.to(state["value"].dtype), ddict.float().reshape(L, k, k)


# ---- the call -------------------------------------------------------------------------------------------------------
def _own(state):
    import paper_2303_08999_amd as sr

    case, mask = state["case"], state["mask"]
    L, T, s = case["L"], case["entries"], case["scale"]
    if case["op"] == "list_grad":
        if "workspace" not in state:
            need = sr.sr_dict_assemble_list_grad_workspace_bytes(L, case["k"])
            state["workspace"] = torch.empty(need, device="cuda", dtype=torch.uint8)
        return sr.sr_dict_assemble_list_grad(state["lr"], state["index"], state["value"], state["dict"], L, case["k"], s,
                                             case["c"], T, mask, state["dout"], state["dvalue"], state["ddict"],
                                             workspace=state["workspace"])
    kind = {"softmax": sr.SR_ROUTE_SOFTMAX, "chosen": sr.SR_ROUTE_CHOSEN}[case["kind"]]
    layout = {"planar": sr.SR_COEFF_PLANAR, "pixel_major": sr.SR_COEFF_PIXEL_MAJOR,
              "pre_shuffle": sr.SR_COEFF_PRE_SHUFFLE}[case["layout"]]
    if case["op"] == "route":
        return sr.sr_list_route(state["coeff"], L, s, T, kind, layout, mask, state["index"], state["value"])
    if case["op"] == "balance":
        if "workspace" not in state:
            state["workspace"] = torch.empty(sr.sr_list_route_workspace_bytes(L), device="cuda", dtype=torch.uint8)
        return sr.sr_list_route_balance(state["coeff"], L, s, T, kind, layout, mask, state["index"], state["value"],
                                        state["counts"], state["share"], state["loss"], workspace=state["workspace"])
    return sr.sr_list_route_grad(state["coeff"], state["index"], state["dvalue"], L, s, T, kind, layout, mask,
                                 state["counts"], state["dloss"], state["dcoeff"])


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    return _plain_list_grad(state) if op == "list_grad" else _plain_route_grad(state) if op == "route_grad" else _plain_route(state)


def work(case):
    """Inputs read once, outputs written once; the comparisons and exponentials of every logit, the filters' products."""
    n, H, W = _shape(case)
    px, L, T = n * H * W, case["L"], case["entries"]
    bv = BYTES[case["value"]]
    masked = px if case["mask"] else 0
    if case["op"] == "list_grad":
        c, kk, io = case["c"], case["k"] ** 2, BYTES[case["image"]]
        return {"bytes": masked + px * (T * (1 + 2 * bv) + c * io) + n * c * case["h"] * case["w"] * io + 8 * L * kk,
                "flops": px * c * (4 + 4.0 / case["scale"]) * 2 + px * 2 * kk * (c + 2 * T)}
    bz = BYTES[case["coeff"]]
    lists = px * T * (1 + bv)
    if case["op"] == "route_grad":
        return {"bytes": masked + px * 2 * L * bz + lists + 8 * (L + 1) + 8, "flops": px * L * 8}
    extra = 8 * (L + 1) + 4 * L + 8 if case["op"] == "balance" else 0
    return {"bytes": masked + px * L * bz + lists + extra, "flops": px * L * (6 if case["op"] == "balance" else 4)}


# ---- the same in 64 bits --------------------------------------------------------------------------------------------
def _rows(case, most):
    n, H, W = _shape(case)
    step = max(1, most // W)
    return [(b, y, min(y + step, H)) for b in range(n) for y in range(0, H, step)]


def exact(case, seed):
    d = _inputs(case, seed)
    n, H, W = _shape(case)
    L, T = case["L"], case["entries"]
    if case["op"] == "list_grad":
        return _exact_list_grad(case, d)
    z_all = _planar(case, d["coeff"])
    if case["op"] == "route_grad":
        M = float(d["counts"][L])
        f = d["counts"][:L].double().reshape(L, 1, 1) / (M * T)
        w0, w1 = (float(v) for v in d["dloss"].double().cpu())
        dz = torch.empty((n, L, H, W), device="cuda", dtype=torch.float64)
        for b, y0, y1 in _rows(case, 1 << 20):
            z = z_all[b, :, y0:y1].double().requires_grad_()
            lse = torch.logsumexp(z, 0, keepdim=True)
            index = d["index"][b, :, y0:y1].long()
            chosen = z.gather(0, index)
            value = torch.exp(chosen - (lse if case["kind"] == "softmax" else torch.logsumexp(chosen, 0, keepdim=True)))
            on = torch.ones_like(lse) if d["mask"] is None else d["mask"][b, :, y0:y1].double()
            balance = L * (f * torch.exp(z - lse) * on).sum() / M
            total = (value * d["dvalue"][b, :, y0:y1].double() * on).sum() + w0 * balance + w1 * (lse * lse * on).sum() / M
            dz[b, :, y0:y1] = torch.autograd.grad(total, z)[0]
        if case["layout"] == "pixel_major":
            return dz.permute(0, 2, 3, 1).contiguous()
        return F.pixel_unshuffle(dz, case["scale"]) if case["layout"] == "pre_shuffle" else dz
    value = torch.zeros((n, T, H, W), device="cuda", dtype=torch.float64)
    share = torch.zeros(L, device="cuda", dtype=torch.float64)
    counts, squares, M = torch.zeros_like(share), 0.0, 0.0
    for b, y0, y1 in _rows(case, 1 << 20):
        z = z_all[b, :, y0:y1].double()
        on = torch.ones_like(z[0]) if d["mask"] is None else d["mask"][b, 0, y0:y1].double()
        top, at = torch.topk(z, T, dim=0)
        lse = torch.logsumexp(z, 0)
        value[b, :, y0:y1] = torch.exp(top - (lse if case["kind"] == "softmax" else torch.logsumexp(top, 0))) * on
        if case["op"] == "balance":
            # a tie at the border goes to the lowest atoms: all above it, then as many of its equals as there is room for
            least = top[-1:]
            above, equal = z > least, z == least
            taken = above | (equal & (torch.cumsum(equal, 0) <= T - above.sum(0, keepdim=True)))
            counts += (taken * on).sum(dim=(1, 2))
            share += (torch.exp(z - lse) * on).sum(dim=(1, 2))
            squares += float((lse * lse * on).sum())
            M += float(on.sum())
        del z, at
    if case["op"] == "route":
        return None, value
    share = share / M
    loss = torch.stack([L * (counts / (M * T) * share).sum(), torch.tensor(squares / M, device="cuda", dtype=torch.float64)])
    return None, value, None, share, loss


def _exact_list_grad(case, d):
    n, H, W = _shape(case)
    L, k, s, c, T = (case[x] for x in ("L", "k", "scale", "c", "entries"))
    r = (k - 1) // 2
    up = F.pad(_up_axis(_up_axis(d["lr"].double(), s, 2), s, 3), (r, r, r, r), mode="replicate")
    atoms = d["dict"].reshape(L, k * k).double().requires_grad_()
    dvalue = torch.empty((n, T, H, W), device="cuda", dtype=torch.float64)
    ddict = torch.zeros((L, k * k), device="cuda", dtype=torch.float64)
    for b, y0, y1 in _rows(case, 1 << 17):
        value = d["value"][b, :, y0:y1].double().requires_grad_()
        index = d["index"][b, :, y0:y1].long()
        phi = torch.zeros((L, y1 - y0, W), device="cuda", dtype=torch.float64).scatter_add(0, index, value)
        filters = torch.matmul(atoms.t(), phi.reshape(L, -1)).reshape(k * k, y1 - y0, W)
        window = torch.stack([up[b, :, y0 + i // k:y1 + i // k, i % k:i % k + W] for i in range(k * k)])
        image = (filters[:, None] * window).sum(0)              # Eq. 2 with the listed terms
        dout = d["dout"][b, :, y0:y1].double()
        if d["mask"] is not None:
            dout = dout * d["mask"][b, :, y0:y1]
        gv, gd = torch.autograd.grad((image * dout).sum(), (value, atoms))
        dvalue[b, :, y0:y1] = gv
        ddict += gd
    return dvalue, ddict.reshape(L, k, k)

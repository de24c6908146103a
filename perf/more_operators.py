"""Layers over pixels or tokens, their gradients, and the clipping of all gradients: what is timed, and the same in plain torch.

What stands before the coefficients and behind their gradients.  Three operators, two of them in both directions:
`linear` (a product with bias, activation and residual: the coefficient network's head, its 1 x 1 convolutions) and
`linear_grad`; `gated` (both projections of a gated block, the activation and the product) and `gated_grad`; `clip` (the norm
over every gradient of a model, and the gradients scaled down to a largest norm).

A case is a dict of plain values; `prepare` makes what the caller holds before the call, `run` is the call (or, where `own` is
false, the same in elementary torch operations), `exact` the outputs in 64 bits, the gradients by differentiating the forward
formula.  Rows are pixels of Table I's frames, of 4K and 1080p frames, of images of odd sizes, or tokens.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}


def _layer(op, rows, c, o, dtype, act, bias=True, residual=False):
    """rows of c features to o outputs (for the gated block o is what comes out of it: its weight has 2 o rows)."""
    return {"op": op, "rows": rows, "c": c, "o": o, "dtype": dtype, "act": act, "bias": bias, "residual": residual}


def _clip(tensors, elements, dtype, over):
    """over: the gradients' norm is beyond the largest one allowed."""
    return {"op": "clip", "tensors": tensors, "elements": elements, "dtype": dtype, "over": over}


def listed():
    def named(name, case):
        return dict(case, name=name)

    return [
        # one token of a serving loop through the last product of a block: the weights have to come past once
        named("linear_token_bf16", _layer("linear", 1, 2048, 2048, "bf16", "none", residual=True)),
        # the head that makes 72 logits for every pixel of the 4K frame from 64 features
        named("linear_head_4k_f16", _layer("linear", 3840 * 2160, 64, 72, "f16", "none")),
        # two photos of odd size at x2, patches of 27 values to 121 features, an fp32 network
        named("linear_photo_f32", _layer("linear", 2 * 342 * 514, 27, 121, "f32", "gelu")),
        # a wide layer over many tokens with all that an epilogue has
        named("linear_wide_bf16", _layer("linear", 16384, 4096, 4096, "bf16", "gelu", residual=True)),
        # training of the head on a 1080p frame
        named("linear_grad_head_1080p_bf16", _layer("linear_grad", 1920 * 1080, 64, 72, "bf16", "none")),
        # training of a layer with an activation
        named("linear_grad_tokens_f16", _layer("linear_grad", 8192, 2048, 4096, "f16", "gelu")),
        # one token of a serving loop through a gated block
        named("gated_token_f16", _layer("gated", 1, 1024, 2816, "f16", "silu", bias=False)),
        # a prompt, or a batch of them
        named("gated_prompt_bf16", _layer("gated", 8192, 2048, 5632, "bf16", "silu", bias=False)),
        # the smallest training crop, 64 x 64, of an fp32 network
        named("gated_grad_crop_f32", _layer("gated_grad", 64 * 64, 64, 128, "f32", "silu")),
        # a padded batch whose sizes are no multiples of a tile
        named("gated_grad_odd_bf16", _layer("gated_grad", 8191, 1024, 2730, "bf16", "gelu")),
        # a small coefficient network with its dictionary
        named("clip_net_f32", _clip(24, 120011, "f32", True)),
        # hundreds of tensors, half of them bfloat16
        named("clip_many_mixed", _clip(290, 360000007, "mixed", True)),
    ]


# the largest listed cases: what a drawn one may cost
MOST_FLOPS = 2 * 16384 * 4096 * 4096
MOST_BYTES = 3840 * 2160 * (64 + 72) * 2


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["linear", "linear_grad", "gated", "gated_grad", "clip"])
    if op == "clip":
        tensors = log(1, 400)
        return _clip(tensors, max(tensors, log(1000, 300000000)), rng.choice(["f32", "f16", "bf16", "mixed"]), rng.random() < 0.7)
    while True:
        rows, c, o = log(1, 4000000), log(8, 4096), log(8, 4096)
        if rng.random() < 0.6:                                  # most widths are multiples of 8, as networks have them
            c, o = (c + 7) // 8 * 8, (o + 7) // 8 * 8
        acts = ["none", "relu", "gelu", "silu"]
        if op.endswith("grad"):                                 # a step at 0 has no gradient there to compare
            acts.remove("relu")
        case = _layer(op, rows, c, o, rng.choice(["f32", "f16", "bf16"]), rng.choice(acts), rng.random() < 0.7,
                      op == "linear" and rng.random() < 0.4)
        w = work(case)
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES:
            return case


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _sizes(case):
    """Elements of every tensor: matrices of several sizes, each with a vector behind it, and single values among them."""
    share = [1.0, 1.0 / 256, 2.0, 1.0 / 128, 0.5, 0.25, 1.0 / 512]
    weight = [share[i % 7] for i in range(case["tensors"])]
    left, total = case["elements"] - case["tensors"], sum(weight)
    sizes = [1 + int(left * v / total) for v in weight]
    sizes[0] += case["elements"] - sum(sizes)
    return sizes


def _kinds(case):
    return ["bf16", "f32"][:case["tensors"]] if case["dtype"] == "mixed" else [case["dtype"]]


def _views(case, flat):
    """The tensors, one behind the other in a buffer for each type, as a bucket of gradients has them."""
    at, views = [0] * len(flat), []
    for i, size in enumerate(_sizes(case)):
        j = i % len(flat)
        views.append(flat[j][at[j]:at[j] + size])
        at[j] += size
    return views


def _inputs(case, seed):
    """What a call reads: the same tensors for `run` and for `exact`."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(shape, scale, t):
        x = torch.empty(shape, device="cuda", dtype=t)
        flat = x.view(-1)
        for at in range(0, flat.numel(), 1 << 28):
            part = flat[at:at + (1 << 28)]
            part.copy_(torch.randn(part.shape, generator=g, device="cuda") * scale)
        return x

    if case["op"] == "clip":
        sizes, kinds = _sizes(case), _kinds(case)
        flat = [normal((sum(sizes[j::len(kinds)]),), 1.0, DTYPES[kind]) for j, kind in enumerate(kinds)]
        grads = _views(case, flat)
        for i, t in enumerate(grads):                           # every layer's gradients have a magnitude of their own
            t.mul_(2.0 ** -(6 + i % 5))
        expected = math.sqrt(sum(size * 4.0 ** -(6 + i % 5) for i, size in enumerate(sizes)))
        return {"flat": flat, "grads": grads, "most": expected / 3 if case["over"] else expected * 3}
    t = DTYPES[case["dtype"]]
    rows, c, o = case["rows"], case["c"], case["o"]
    wide = 2 * o if case["op"].startswith("gated") else o
    d = {"x": normal((rows, c), 1.0, t), "weight": normal((wide, c), 1.0 / math.sqrt(c), t)}
    d["bias"] = normal((wide,), 0.1, t) if case["bias"] else None
    d["residual"] = normal((rows, o), 1.0, t) if case["residual"] else None
    if case["op"].endswith("grad"):
        d["dy"] = normal((rows, o), 1.0 / 64, t)                # what a scaled loss sends back
    return d


def prepare(case, seed):
    state = _inputs(case, seed)
    state["case"] = case
    if case["op"] == "clip":
        state["flat_out"] = [torch.empty_like(t) for t in state["flat"]]
        state["out"] = _views(case, state["flat_out"])
        state["norm"] = torch.empty(2, device="cuda")
    elif case["op"].endswith("grad"):
        state["dx"], state["dweight"] = torch.empty_like(state["x"]), torch.empty_like(state["weight"])
        state["dbias"] = torch.empty_like(state["bias"]) if case["bias"] else None
    else:
        state["y"] = torch.empty((case["rows"], case["o"]), device="cuda", dtype=DTYPES[case["dtype"]])
    return state


# ---- the plain form -------------------------------------------------------------------------------------------------
def _act(name, z):
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _slope(name, z):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def _affine(state):
    z = torch.matmul(state["x"].float(), state["weight"].float().t())
    return z if state["bias"] is None else z + state["bias"].float()


def _plain_grads(state, dz):
    x, w = state["x"].float(), state["weight"].float()
    dx = torch.matmul(dz, w).to(state["x"].dtype)
    dw = torch.matmul(dz.t(), x).to(state["weight"].dtype)
    if state["bias"] is None:
        return dx, dw
    return dx, dw, dz.sum(0, dtype=torch.float64).to(state["bias"].dtype)


def _plain(state):
    case = state["case"]
    op, act = case["op"], case["act"] if "act" in case else None
    if op == "clip":
        squares = [(t.float() * t.float()).sum(dtype=torch.float64) for t in state["grads"]]
        norm = torch.sqrt(torch.stack(squares).sum())
        factor = torch.where(norm > state["most"], state["most"] / norm, torch.ones_like(norm)).float()
        return [(t.float() * factor).to(t.dtype) for t in state["flat"]], torch.stack([norm.float(), factor])
    if op == "linear":
        y = _act(act, _affine(state))
        if state["residual"] is not None:
            y = y + state["residual"].float()
        return y.to(state["x"].dtype)
    if op == "linear_grad":
        dz = state["dy"].float()
        if act != "none":
            dz = dz * _slope(act, _affine(state))
        return _plain_grads(state, dz)
    z = _affine(state)
    gate, up = z[:, :case["o"]], z[:, case["o"]:]
    if op == "gated":
        return (_act(act, gate) * up).to(state["x"].dtype)
    dy = state["dy"].float()
    return _plain_grads(state, torch.cat([dy * up * _slope(act, gate), dy * _act(act, gate)], 1))


# ---- the call -------------------------------------------------------------------------------------------------------
def _scratch(state, need):
    if "workspace" not in state:
        state["workspace"] = torch.empty(max(16, need), device="cuda", dtype=torch.uint8)
    return state["workspace"]


def _own(state):
    import paper_2303_08999_amd as sr

    case = state["case"]
    op = case["op"]
    if op == "clip":
        if "list" not in state:                                 # a program keeps its tensors' descriptions
            state["list"], state["out_list"] = sr.sr_tensor_list(state["grads"]), sr.sr_tensor_list(state["out"])
        scratch = _scratch(state, sr.sr_grad_clip_workspace_bytes(case["tensors"]))
        sr.sr_grad_clip(state["list"], state["out_list"], state["most"], state["norm"], workspace=scratch)
        return state["flat_out"], state["norm"]
    act = {"none": sr.SR_ACT_NONE, "relu": sr.SR_ACT_RELU, "gelu": sr.SR_ACT_GELU, "silu": sr.SR_ACT_SILU}[case["act"]]
    x, weight, bias = state["x"], state["weight"], state["bias"]
    if op == "linear":
        scratch = _scratch(state, sr.sr_layer_linear_workspace_bytes(case["rows"], case["c"], case["o"], x.dtype))
        return sr.sr_layer_linear(x, weight, bias, act, state["residual"], state["y"], workspace=scratch)
    if op == "gated":
        scratch = _scratch(state, sr.sr_layer_gated_workspace_bytes(case["rows"], case["c"], case["o"], x.dtype))
        return sr.sr_layer_gated(x, weight, bias, act, state["y"], workspace=scratch)
    if op == "linear_grad":
        scratch = _scratch(state, sr.sr_layer_linear_grad_workspace_bytes(case["rows"], case["c"], case["o"], x.dtype, act))
        out = sr.sr_layer_linear_grad(x, weight, bias, act, state["dy"], state["dx"], state["dweight"], state["dbias"],
                                      workspace=scratch)
    else:
        scratch = _scratch(state, sr.sr_layer_gated_grad_workspace_bytes(case["rows"], case["c"], case["o"], x.dtype))
        out = sr.sr_layer_gated_grad(x, weight, bias, act, state["dy"], state["dx"], state["dweight"], state["dbias"],
                                     workspace=scratch)
    return out if case["bias"] else out[:2]


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    """Inputs read once, outputs written once; the products, the one that a gradient makes anew among them."""
    if case["op"] == "clip":
        kinds = _kinds(case)
        moved = sum(n * BYTES[kinds[i % len(kinds)]] for i, n in enumerate(_sizes(case)))
        return {"bytes": 2 * moved + 8, "flops": 3 * case["elements"]}
    rows, c, o = case["rows"], case["c"], case["o"]
    wide = 2 * o if case["op"].startswith("gated") else o
    vectors = wide if case["bias"] else 0
    product = 2 * rows * c * wide
    if case["op"].endswith("grad"):
        again = 1 if case["act"] != "none" or wide != o else 0
        return {"bytes": BYTES[case["dtype"]] * (2 * rows * c + 2 * wide * c + 2 * vectors + rows * o),
                "flops": (2 + again) * product}
    extra = rows * o if case["residual"] else 0
    return {"bytes": BYTES[case["dtype"]] * (rows * c + wide * c + vectors + rows * o + extra), "flops": product}


# ---- the same in 64 bits --------------------------------------------------------------------------------------------
def _forward64(case, x, weight, bias):
    """The layer by torch's own functions in double precision."""
    fn = {"none": lambda v: v, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}[case["act"]]
    z = torch.nn.functional.linear(x, weight, bias)
    if case["op"].startswith("linear"):
        return fn(z)
    gate, up = z.chunk(2, 1)
    return fn(gate) * up


def exact(case, seed):
    d = _inputs(case, seed)
    if case["op"] == "clip":
        norm = math.sqrt(math.fsum(float((t.double() ** 2).sum()) for t in d["flat"]))
        factor = d["most"] / norm if norm > d["most"] else 1.0
        return [t.double() * factor for t in d["flat"]], torch.tensor([norm, factor], device="cuda", dtype=torch.float64)
    rows, o = case["rows"], case["o"]
    weight = d["weight"].double()
    bias = None if d["bias"] is None else d["bias"].double()
    step = max(1, (1 << 26) // max(case["c"], weight.shape[0]))
    if not case["op"].endswith("grad"):
        y = torch.empty((rows, o), device="cuda", dtype=torch.float64)
        for at in range(0, rows, step):
            y[at:at + step] = _forward64(case, d["x"][at:at + step].double(), weight, bias)
            if d["residual"] is not None:
                y[at:at + step] += d["residual"][at:at + step].double()
        return y
    weight.requires_grad_()
    leaves = [weight] if bias is None else [weight, bias.requires_grad_()]
    dx = torch.empty(d["x"].shape, device="cuda", dtype=torch.float64)
    sums = [torch.zeros_like(v) for v in leaves]
    for at in range(0, rows, step):
        x = d["x"][at:at + step].double().requires_grad_()
        total = (_forward64(case, x, weight, bias) * d["dy"][at:at + step].double()).sum()
        got = torch.autograd.grad(total, [x] + leaves)
        dx[at:at + step] = got[0]
        for s, v in zip(sums, got[1:]):
            s += v
    return (dx, *[s.detach() for s in sums])

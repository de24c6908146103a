"""The router, its losses and the gradients (include/sr_route.h) in 64 bits on the host: test infrastructure only.

Written from the formulas of the header, planar [n][L][H][W] float64 in, float64 out; the gradients are the formulas, and
`losses` is what a test differentiates by differences to check them.
"""
import torch

SOFTMAX, CHOSEN, VALUES = 0, 1, 2


def order(z, entries):
    """The atoms of every pixel by decreasing logit, equal ones (and -0 and +0) by increasing atom: [n][entries][H][W]."""
    return torch.sort(z + 0.0, dim=1, descending=True, stable=True).indices[:, :entries]


def softmax(z, over=None):
    """Softmax over the atoms (those where `over` is true); a masked atom has 0, and so has a pixel of none but masked ones."""
    if over is not None:
        z = torch.where(over, z, torch.full_like(z, -float("inf")))
    m = z.amax(1, keepdim=True)
    e = torch.where(torch.isneginf(z), torch.zeros_like(z), torch.exp(z - torch.where(torch.isneginf(m), torch.zeros_like(m), m)))
    s = e.sum(1, keepdim=True)
    return e / torch.where(s == 0, torch.ones_like(s), s)


def lse(z):
    """m + ln s; 0 for a pixel of none but masked atoms."""
    out = torch.logsumexp(z, 1, keepdim=True)
    return torch.where(torch.isneginf(out), torch.zeros_like(out), out)


def listed(z, index):
    return torch.zeros(z.shape, dtype=torch.bool).scatter_(1, index, True)


def live(z, mask):
    on = ~torch.isneginf(z).all(1, keepdim=True)
    return on if mask is None else on & (mask != 0)


def route(z, entries, kind, mask=None):
    index = order(z, entries)
    if kind == VALUES:
        value = z.gather(1, index)
    else:
        value = softmax(z, None if kind == SOFTMAX else listed(z, index)).gather(1, index)
    if mask is not None:
        on = mask != 0
        index = torch.where(on, index, torch.arange(entries).reshape(1, -1, 1, 1))
        value = torch.where(on, value, torch.zeros_like(value))
    return index, value


def balance(z, entries, mask=None):
    """counts (L + 1), share (L), loss (2)."""
    L = z.shape[1]
    on = live(z, mask)
    p, M = softmax(z), int(on.sum())
    hit = listed(z, order(z, entries)) & on & ~torch.isneginf(z)
    counts = hit.sum(dim=(0, 2, 3))
    over = max(M, 1)
    share = torch.where(on, p, torch.zeros_like(p)).sum(dim=(0, 2, 3)) / over
    l = lse(z)
    loss = torch.stack([L * (counts.double() / (over * entries) * share).sum(), torch.where(on, l * l, torch.zeros_like(l)).sum() / over])
    return torch.cat([counts, torch.tensor([M])]), share, loss


def losses(z, index, kind, dvalue, counts, dloss, mask=None):
    """The number whose gradient route_grad gives: <values, dvalue> + <losses, dloss>, choice and counts held fixed."""
    L, entries = z.shape[1], index.shape[1]
    on = live(z, mask)
    total = torch.zeros((), dtype=torch.float64)
    if dvalue is not None:
        v = z.gather(1, index) if kind == VALUES else softmax(z, None if kind == SOFTMAX else listed(z, index)).gather(1, index)
        keep = on if kind != VALUES else (torch.ones_like(on) if mask is None else mask != 0)
        total = total + torch.where(keep, v * dvalue, torch.zeros_like(v)).sum()
    if counts is not None:
        M = float(counts[L])
        f = counts[:L].double().reshape(1, L, 1, 1) / (M * entries)
        p, l = softmax(z), lse(z)
        total = total + float(dloss[0]) * L / M * torch.where(on, f * p, torch.zeros_like(p)).sum()
        total = total + float(dloss[1]) / M * torch.where(on, l * l, torch.zeros_like(l)).sum()
    return total


def route_grad(z, index, kind, dvalue=None, counts=None, dloss=None, mask=None):
    """(gradient, sum of the magnitudes of its terms: what a relative error of an fp32 evaluation refers to)."""
    L, entries = z.shape[1], index.shape[1]
    G = torch.zeros_like(z)
    if dvalue is not None:
        G.scatter_add_(1, index, dvalue)
    if kind == VALUES:
        dz, size = G, G.abs()
        on = torch.ones_like(z[:, :1], dtype=torch.bool) if mask is None else mask != 0
    else:
        p = softmax(z)
        q = p if kind == SOFTMAX else softmax(z, listed(z, index))
        dz = q * (G - (q * G).sum(1, keepdim=True))
        size = q * (G.abs() + (q * G.abs()).sum(1, keepdim=True))
        on = live(z, mask) & ~torch.isneginf(z)
        if counts is not None:
            M = max(float(counts[L]), 1.0)
            f = counts[:L].double().reshape(1, L, 1, 1) / (M * entries)
            w0, w1, l = float(dloss[0]) * L / M, 2 * float(dloss[1]) / M, lse(z)
            fp = (f * p).sum(1, keepdim=True)
            dz = dz + p * (w0 * (f - fp) + w1 * l)
            size = size + p * (abs(w0) * (f + fp) + abs(w1) * l.abs())
    zero = torch.zeros_like(dz)
    return torch.where(on, dz, zero), torch.where(on, size, zero)


def list_grad(up, index, value, dictionary, dout, mask=None):
    """Gradient of the list form from the up-sampled image: (dvalue, ddict, entries that name each atom)."""
    n, c, H, W = up.shape
    L, k = dictionary.shape[0], dictionary.shape[-1]
    r = (k - 1) // 2
    if mask is not None:
        on = mask != 0
        dout = torch.where(on, dout, torch.zeros_like(dout))
        value = torch.where(on, value, torch.zeros_like(value))
    pad = torch.nn.functional.pad(up, (r, r, r, r), mode="replicate")
    E = torch.stack([(pad[:, :, i // k:i // k + H, i % k:i % k + W] * dout).sum(1) for i in range(k * k)], 1)
    D = dictionary.reshape(L, k * k)
    response = torch.einsum("lj,njyx->nlyx", D, E)
    phi = torch.zeros((n, L, H, W), dtype=torch.float64).scatter_add_(1, index, value)
    ddict = torch.einsum("nlyx,njyx->lj", phi, E)
    named = torch.bincount(index.reshape(-1), minlength=L)
    return response.gather(1, index), ddict.reshape(dictionary.shape), named

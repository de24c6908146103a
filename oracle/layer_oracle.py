"""Layers over rows of features, their gradients and the clipping of gradients in 64 bits (test infrastructure only).

Written from the formulas, without differentiation by a library: tests/test_oracle_layer.py holds them to autograd and to
differences.  All arguments are double tensors on any device: x [P][C], weight [O][C] (gated: [2F][C]), bias or None."""
import math

import torch

NONE, RELU, GELU, SILU, SIGMOID = range(5)


def act(kind, z):
    if kind == RELU:
        return z.clamp(min=0)
    if kind == GELU:
        return z * torch.special.ndtr(z)
    if kind == SILU:
        return z * torch.special.expit(z)
    if kind == SIGMOID:
        return torch.special.expit(z)
    return z


def slope(kind, z):
    if kind == RELU:
        return (z > 0).to(z.dtype)
    if kind == GELU:
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if kind == SILU:
        s = torch.special.expit(z)
        return s + z * s * torch.special.expit(-z)
    if kind == SIGMOID:
        return torch.special.expit(z) * torch.special.expit(-z)
    return torch.ones_like(z)


def affine(x, weight, bias):
    z = x @ weight.t()
    return z if bias is None else z + bias


def linear(x, weight, bias, kind, residual=None):
    y = act(kind, affine(x, weight, bias))
    return y if residual is None else y + residual


def gated(x, weight, bias, kind):
    g, u = affine(x, weight, bias).chunk(2, 1)
    return act(kind, g) * u


def linear_dz(x, weight, bias, kind, dy):
    return dy * slope(kind, affine(x, weight, bias))


def gated_dz(x, weight, bias, kind, dy):
    g, u = affine(x, weight, bias).chunk(2, 1)
    return torch.cat([dy * u * slope(kind, g), dy * act(kind, g)], 1)


def behind_dz(x, weight, dz):
    """dx, dweight, dbias"""
    return dz @ weight, dz.t() @ x, dz.sum(0)


def clip(grads, most):
    """The gradients scaled down to the norm `most`, the norm and the factor."""
    norm = math.sqrt(math.fsum(float((g * g).sum()) for g in grads))
    factor = most / norm if most < norm < math.inf else 1.0
    return [g * factor for g in grads], norm, factor

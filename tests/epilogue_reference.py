"""Activations, their slopes, and the norms and rotation of heads in 64 bits, straight from their definitions: what the kernels'
tests compare with."""
import math

import torch

NAMES = ("none", "relu", "gelu", "gelu_tanh", "silu")
CUBE = 0.044715


def act(name, z):
    if name == "relu":
        return torch.where(z <= 0, torch.zeros_like(z), z)
    if name == "gelu":  # (erfc keeps the tail's relative accuracy)
        return z * 0.5 * torch.erfc(-z * math.sqrt(0.5))
    if name == "gelu_tanh":
        return z / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (z + CUBE * z ** 3)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def slope(name, z):
    if name == "relu":
        return torch.where(z <= 0, torch.zeros_like(z), torch.ones_like(z))
    if name == "gelu":
        return 0.5 * torch.erfc(-z * math.sqrt(0.5)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "none":
        return torch.ones_like(z)
    c = 2 * math.sqrt(2 / math.pi)
    u, du = (z, torch.ones_like(z)) if name == "silu" else (c * (z + CUBE * z ** 3), c * (1 + 3 * CUBE * z * z))
    return 1 / (1 + torch.exp(-u)) + z * du / ((1 + torch.exp(-u)) * (1 + torch.exp(u)))


def pairs(rotary, interleaved):
    i = torch.arange(rotary // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)


def turn(x, angle, interleaved):
    """x[t, h, :2 n] turned by angle[t, n]."""
    a, b = (p.to(x.device) for p in pairs(2 * angle.shape[1], interleaved))
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    y = x.clone()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def qk(x, positions, freqs, weight, eps, norm, interleaved):
    """The forward pass of one side, x[t, h, d] in 64 bits; freqs None: no rotation, weight None: ones."""
    if norm:
        x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt()
        if weight is not None:
            x = x * weight.double()
    return x if freqs is None else turn(x, positions.double()[:, None] * freqs, interleaved)


def qk_back(x, dy, positions, freqs, weight, eps, norm, interleaved):
    """(dx, dweight) from the formulas."""
    dn = dy if freqs is None else turn(dy, -positions.double()[:, None] * freqs, interleaved)
    if not norm:
        return dn, None
    r = 1 / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    xh = x * r
    t = dn if weight is None else dn * weight.double()
    return r * (t - xh * (t * xh).mean(-1, keepdim=True)), (dn * xh).sum((0, 1))

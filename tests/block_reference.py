"""The trained block's operators in 64 bits, by plain torch from their definitions, with
bounds on what float32 arithmetic and the roundings of the operands' type may add.

u is half a step of the type (2^-8 bf16, 2^-24 float32), f = 2^-24.  As in
tail_reference, a sum of n float32 terms whose roundings are independent is off by
less than 4 sqrt(n) f times the sum of the terms' sizes.
"""
from __future__ import annotations

import math

import torch

from tests.tail_reference import F, U, check  # noqa: F401

TINY = 1e-37


def pairs_of(dim, pairs, neighbours):
    """Columns of the pairs' first and second values."""
    i = torch.arange(pairs)
    return (2 * i, 2 * i + 1) if neighbours else (i, pairs + i)


def _turn(x, ex, angle, neighbours):
    """x's pairs turned by angle [b, l, P], and the bound of x (ex) carried through."""
    p = angle.shape[-1]
    i, j = (c.to(x.device) for c in pairs_of(x.shape[-1], p, neighbours))
    c, s = torch.cos(angle)[:, :, None], torch.sin(angle)[:, :, None]
    # the reduced angle's rounding (pi f), four units of the functions' last place, the
    # float64 angle's own
    et = 12 * F + (angle.abs() * 2.0 ** -51)[:, :, None]
    a, b, ea, eb = x[..., i], x[..., j], ex[..., i], ex[..., j]
    y, ey = x.clone(), ex.clone()
    y[..., i], y[..., j] = a * c - b * s, b * c + a * s
    both = 3 * F * (a.abs() * c.abs() + b.abs() * s.abs()) + (a.abs() + b.abs()) * et
    ey[..., i] = ea * c.abs() + eb * s.abs() + both
    ey[..., j] = eb * c.abs() + ea * s.abs() + 3 * F * (b.abs() * c.abs() + a.abs() * s.abs()) + (a.abs() + b.abs()) * et
    return y, ey


def _angle(positions, freq, sections):
    axis = torch.tensor([a for a, m in enumerate(sections) for _ in range(m)], dtype=torch.int64, device=positions.device)
    return positions.double()[axis].permute(1, 2, 0) * freq


def _counting(x, lens):
    if lens is None:
        return torch.ones(x.shape[:2], dtype=torch.bool, device=x.device)[:, :, None, None]
    return (torch.arange(x.shape[1], device=x.device) < lens[:, None])[:, :, None, None]


def rotary_forward(x, gamma, positions, freq, sections, neighbours=False, eps=1e-6, lens=None):
    """(value, bound) of one of q_out and k_out; x [batch, length, heads, dim]."""
    u, d = U[x.dtype], x.shape[-1]
    counts = _counting(x, lens)
    h = torch.where(counts, x.double(), 0.0)
    eh = torch.zeros_like(h)
    if gamma is not None:
        r = 1.0 / torch.sqrt((h * h).mean(-1, keepdim=True) + eps)
        h = h * r * gamma.double()
        eh = (2 * math.sqrt(d) + 8) * F * h.abs()
    y, ey = _turn(h, eh, _angle(positions, freq, sections), neighbours) if sections else (h, eh)
    y, ey = torch.where(counts, y, 0.0), torch.where(counts, ey, 0.0)
    return y, u * y.abs() * (1 + 2 ** -7) + 2 * ey + TINY


def rotary_backward(dy, x, gamma, positions, freq, sections, neighbours=False, eps=1e-6, lens=None):
    """[(value, bound)] of dx and, with a norm, of dgamma."""
    t = dy.dtype
    u, d = U[t], dy.shape[-1]
    counts = _counting(dy, lens)
    g = torch.where(counts, dy.double(), 0.0)
    eg = torch.zeros_like(g)
    if sections:
        g, eg = _turn(g, eg, -_angle(positions, freq, sections), neighbours)
    if gamma is None:
        return [(g, u * g.abs() * (1 + 2 ** -7) + 2 * eg + TINY)]
    x = torch.where(counts, x.double(), 0.0)
    gamma = gamma.double()
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    h = x * r
    k = (2 * math.sqrt(d) + 8) * F
    eh = k * h.abs()
    e = g * gamma
    ee = eg * gamma.abs() + F * e.abs()
    c = (e * h).mean(-1, keepdim=True)
    ec = (ee * h.abs() + e.abs() * eh).mean(-1, keepdim=True) + (4 * math.sqrt(d) + 8) * F * (e * h).abs().mean(-1, keepdim=True)
    dx = torch.where(counts, r * (e - h * c), 0.0)
    edx = k * dx.abs() + r * (ee + eh * c.abs() + h.abs() * ec + 3 * F * (e.abs() + (h * c).abs()))
    n = g.shape[0] * g.shape[1] * g.shape[2]
    dg = (g * h).sum((0, 1, 2))
    edg = (eg * h.abs() + g.abs() * eh + F * (g * h).abs()).sum((0, 1, 2)) + 4 * math.sqrt(n) * F * (g * h).abs().sum((0, 1, 2))
    return [(dx, u * dx.abs() * (1 + 2 ** -7) + 2 * torch.where(counts, edx, 0.0) + TINY), (dg, 2 * edg + F * dg.abs() + TINY)]


def gradient_norm(grads):
    return math.sqrt(sum(float(g.double().square().sum()) for g in grads))


def gradient_clip(grads, max_norm):
    """(value, bound) of the norm and of every clipped gradient: the factor is a float64,
    a product passes through float32 to the tensor's type."""
    n = gradient_norm(grads)
    max_norm = float(torch.tensor(max_norm, dtype=torch.float32))  # as the descriptor holds it
    f = max_norm / n if n > max_norm else 1.0
    # the largest subnormal step of float32 (2^-149) and of bf16 (2^-133) where the product is below them
    out = [(g.double() * f, (U[g.dtype] * (1 + 2 ** -7) + 1e-11) * (g.double() * f).abs() + (2.0 ** -133 if g.dtype == torch.bfloat16 else 2.0 ** -149))
           for g in grads]
    return (n, n * (F * 1.001 + 1e-12) + TINY), out

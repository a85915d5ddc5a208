"""Layer norm, the classifier's cross entropy and its distillation in 64 bits,
by plain torch from their definitions, with bounds on what float32 arithmetic
and the roundings of the operands' type may add to them.

u is half a step of the type (2^-8 bf16, 2^-24 float32), f = 2^-24.  A sum of n
float32 terms whose roundings are independent is off by less than
4 sqrt(n) f times the sum of the terms' sizes (each of the n roundings is at
most f times a partial sum, of standard deviation f / sqrt 3 of it; 4 sqrt n is
seven of those).
"""
from __future__ import annotations

import math

import torch

F = 2.0 ** -24
U = {torch.bfloat16: 2.0 ** -8, torch.float32: F}


def norm_forward(x, gamma, beta, eps):
    """(value, bound) of y, mean and rstd."""
    u, n = U[x.dtype], x.shape[1]
    x = x.double()
    g, b = gamma.double(), beta.double()
    mean = x.mean(1, keepdim=True)
    c = x - mean
    rstd = 1.0 / torch.sqrt((c * c).mean(1, keepdim=True) + eps)
    h = c * rstd
    y = h * g + b
    # the mean's error, and its effect on the centred values: second order in the variance
    em = (4 * math.sqrt(n) + 2) * F * x.abs().mean(1, keepdim=True)
    ec = em + F * (x.abs() + mean.abs())
    # about a mean off by d the variance is larger by d d exactly; each deviation's
    # rounding and the sum's add to that; rstd moves by half of it
    ev = (em * em + 2 * F * (c.abs() * (x.abs() + mean.abs())).mean(1, keepdim=True)) * rstd * rstd
    er = rstd * (ev / 2 + (2 * math.sqrt(n) + 6) * F)
    ey = g.abs() * (ec * rstd + c.abs() * er) + 3 * F * ((h * g).abs() + b.abs())
    return (y, u * y.abs() + ey + 1e-37), (mean[:, 0], em[:, 0] + 1e-37), (rstd[:, 0], er[:, 0])


def norm_backward(dy, x, gamma, mean, rstd):
    """(value, bound) of dx, dgamma and dbeta; the statistics are inputs."""
    u, n, rows = U[x.dtype], x.shape[1], x.shape[0]
    dy, x, g = dy.double(), x.double(), gamma.double()
    m, r = mean.double()[:, None], rstd.double()[:, None]
    h = (x - m) * r
    a = dy * g
    s0, s1 = a.mean(1, keepdim=True), (a * h).mean(1, keepdim=True)
    dx = r * (a - s0 - h * s1)
    eh = 3 * F * (x.abs() + m.abs()) * r.abs()
    k = (4 * math.sqrt(n) + 8) * F
    e1 = k * (a * h).abs().mean(1, keepdim=True) + (a.abs() * eh).mean(1, keepdim=True)
    e0 = k * a.abs().mean(1, keepdim=True)
    edx = r.abs() * (4 * F * (a.abs() + s0.abs() + (h * s1).abs()) + e0 + h.abs() * e1 + eh * s1.abs())
    kr = (4 * math.sqrt(rows) + 8) * F
    edg = kr * (dy * h).abs().sum(0) + (dy.abs() * eh).sum(0)
    return ((dx, u * dx.abs() + edx + 1e-37), ((dy * h).sum(0), edg + 1e-37),
            (dy.sum(0), kr * dy.abs().sum(0) + 1e-37))


def head(x, w, bias, ids, teacher=None, temp=1.0, dloss=None):
    """The classifier's loss and gradients: a dict of name -> (value, bound).

    ids [rows] (cross entropy) or [rows, top] with teacher.  Rows that do not
    count take no part in loss and gradients, whatever they hold; their stats and
    picked are of what they hold."""
    t = x.dtype
    u = U[t]
    n, d = x.shape
    v = w.shape[0]
    if teacher is None:
        counts = ids >= 0
        q = torch.zeros(n, v, dtype=torch.float64, device=x.device)
        q[counts.nonzero()[:, 0], ids[counts]] = 1.0
        entropy = torch.zeros(n, dtype=torch.float64, device=x.device)
    else:
        te = teacher.double().masked_fill(ids < 0, -math.inf)
        counts = (te > -math.inf).any(1)
        logq = torch.log_softmax(te[counts] / temp, 1)
        qk = torch.exp(logq)
        q = torch.zeros(n, v, dtype=torch.float64, device=x.device)
        part = torch.zeros(int(counts.sum()), v, dtype=torch.float64, device=x.device)
        part.scatter_add_(1, ids[counts].clamp(min=0), qk)
        q[counts] = part
        entropy = torch.zeros(n, dtype=torch.float64, device=x.device)
        entropy[counts] = torch.where(qk > 0, qk * logq, 0.0).sum(1)
    wd = w.double()
    z = x.double() @ wd.t()
    ez = 4 * math.sqrt(d) * F * (x.double().abs() @ wd.abs().t())
    if bias is not None:
        z = z + bias.double()
        ez = ez + F * (z.abs() + bias.double().abs())
    ez = torch.nan_to_num(ez, nan=0.0, posinf=0.0)
    zt = z / temp
    ezt = ez / temp + 2 * F * torch.nan_to_num(zt.abs(), posinf=0.0)
    lse = torch.logsumexp(zt, 1)
    # log sum exp moves by less than the largest of its logits' errors
    p = torch.exp(zt - lse[:, None])
    el = (p * ezt).sum(1) + (4 * math.sqrt(v) + 16) * F + 3 * F * lse.abs()
    # the largest logit, and the logarithm of the sum about it
    high = z.max(1)[0]
    eh = torch.nan_to_num(ez, nan=0.0).max(1)[0] + F * torch.nan_to_num(high.abs(), posinf=0.0)
    out = {"stats": (torch.stack([high, lse - high / temp], 1), torch.stack([eh, el + eh / temp + 1e-37], 1))}
    qz = torch.where(q > 0, q * zt, 0.0)
    loss = torch.where(counts, temp * temp * (entropy - qz.sum(1) + lse), 0.0)
    et = 32 * F * (q.sum(1) + entropy.abs() + qz.abs().sum(1) + lse.abs())
    out["loss"] = (loss, temp * temp * (el + (q * ezt).sum(1) + et) * counts + 1e-37)
    if teacher is not None:
        safe = ids.clamp(min=0)
        out["picked"] = (torch.where(ids >= 0, z.gather(1, safe), 0.0), ez.gather(1, safe) + 1e-37)
    if dloss is None:
        return out
    coef = torch.where(counts, dloss.double() * temp, 0.0)[:, None]
    dz = torch.where(counts[:, None], coef * (p - q), 0.0)
    xd = torch.where(counts[:, None], x.double(), 0.0)
    # p's relative error: its logit's and the log-sum-exp's, and exp2's argument and value
    ep = p * (ezt + el[:, None] + 8 * F * (zt - lse[:, None]).abs().clamp(max=1e4) + 8 * F)
    edz = torch.where(counts[:, None], coef.abs() * (ep + 40 * F * q), 0.0)
    # dz between the products: rounded once, up to 32 rows its rest too
    held = 0.0 if t != torch.bfloat16 else u if n > 32 else u * u
    edz_h = edz + held * dz.abs()
    k = 4 * F
    dx = dz @ wd
    # A rounding is at most half a step, so of variance u^2 / 3 at most, and each is
    # independent of the others: the variance of a value, and the limit on the error's
    # length in standard deviations.  A single value's two roundings may both be
    # whole half steps, 2 / sqrt(2 / 3) = 2.45 deviations; over a thousand entries of
    # dz the length is at most one deviation but for some 3%.
    few = 2.5 if n * v < 1000 else 1.25
    sdx = (u * u / 3) * (dx * dx) + (held * held / 3) * ((dz * dz) @ (wd * wd))
    out["dx"] = (dx, u * dx.abs() + (edz_h + k * math.sqrt(v) * dz.abs()) @ wd.abs() + 1e-37, few, sdx)
    dw = dz.t() @ xd
    sdw = (u * u / 3) * (dw * dw) + (held * held / 3) * ((dz * dz).t() @ (xd * xd))
    out["dw"] = (dw, u * dw.abs() + (edz_h + k * math.sqrt(n) * dz.abs()).t() @ xd.abs() + 1e-37, few, sdw)
    out["db"] = (dz.sum(0), edz.sum(0) + (k * math.sqrt(n) + 4 * F) * torch.where(counts[:, None], coef.abs() * (p + q), 0.0).sum(0) + 1e-37)
    return out


def check(name, got, want, l2=None):
    """Every value within its bound; with a variance for 16-bit types the whole error's
    length within that many deviations; l2: within this share of the value's length."""
    value, bound = want[:2]
    got_type, got = got.dtype, got.double()
    bad = (got - value).abs() > bound
    bad |= torch.isnan(got) != torch.isnan(value)
    assert not bool(bad.any()), (
        f"{name}: {int(bad.sum())} of {bad.numel()} values off, the first at {bad.nonzero()[0].tolist()}: "
        f"{float(got[bad][0])!r} against {float(value[bad][0])!r}, bound {float(bound[bad][0]):.3g}")
    off = float((got - value).norm())
    if len(want) > 2 and got_type == torch.bfloat16:
        most = want[2] * float(want[3].sum().sqrt())
        assert off <= most, f"{name}: off by {off:.3g} as a whole, at most {most:.3g}"
    if l2 is not None and float(value.norm()) > 0:
        rel = off / float(value.norm())
        assert rel <= l2, f"{name}: off by {rel:.3g} of its length, at most {l2:.3g}"

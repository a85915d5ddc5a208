"""The trained block's operators in 64 bits, by plain torch from their definitions, with
bounds on what float32 arithmetic and the roundings of the operands' type may add.

u is half a step of the type (2^-8 bf16, 2^-24 float32), f = 2^-24.  As in
tail_reference, a sum of n float32 terms whose roundings are independent is off by
less than 4 sqrt(n) f times the sum of the terms' sizes.
"""
from __future__ import annotations

import math

import torch

from tests import tail_reference
from tests.tail_reference import F, U

TINY = 1e-37
# Float32's least normal number.  The hardware's exp2 gives 0 for anything smaller, and
# the matrix cores take such operands for 0: a probability (or ds) of 2^-127 is lost as a
# whole, an absolute error that no relative bound covers (scores 87 / scale below the
# largest reach it).
FLUSH = 2.0 ** -126


def check(name, got, want):
    """As tail_reference.check; a fifth entry bounds what float32 adds to each value, so
    the whole error's length is that of the 16-bit roundings and that bound's at most."""
    tail_reference.check(name, got, want[:2])
    if len(want) > 2 and got.dtype == torch.bfloat16:
        off = float((got.double() - want[0]).norm())
        most = want[2] * float(want[3].sum().sqrt()) + float(want[4].norm())
        assert off <= most, f"{name}: off by {off:.3g} as a whole, at most {most:.3g}"


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
    r = torch.where(counts, 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps), 0.0)  # padding is in no sum
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


# ----------------------------------------------------------- cross attention

class Attention:
    """One problem in 64 bits: keys that take no part and padding replaced by zeros, scores z,
    their bound ez, and which (query, key) take part."""

    def __init__(self, q, k, v, scale=None, q_lens=None, kv_lens=None, mask=None):
        b, lq, h, d = q.shape
        lk, n = k.shape[1], h // k.shape[2]
        dev = q.device
        self.u, self.held = U[q.dtype], (U[q.dtype] if q.dtype == torch.bfloat16 else 0.0)
        self.n, self.d, self.lk, self.lq = n, d, lk, lq
        self.scale = float(torch.tensor(scale if scale else 1.0 / math.sqrt(d), dtype=torch.float32))
        qok = torch.ones(b, lq, dtype=torch.bool, device=dev) if q_lens is None else torch.arange(lq, device=dev) < q_lens[:, None]
        kok = torch.ones(b, lk, dtype=torch.bool, device=dev) if kv_lens is None else torch.arange(lk, device=dev) < kv_lens[:, None]
        if mask is not None:
            kok = kok & mask.bool()
        self.qok, self.kok = qok, kok
        self.q = torch.where(qok[:, :, None, None], q.double(), 0.0).transpose(1, 2)                       # [b, h, lq, d]
        self.k = torch.where(kok[:, :, None, None], k.double(), 0.0).transpose(1, 2).repeat_interleave(n, 1)
        self.v = torch.where(kok[:, :, None, None], v.double(), 0.0).transpose(1, 2).repeat_interleave(n, 1)
        self.on = qok[:, None, :, None] & kok[:, None, None, :]
        kt = self.k.transpose(-1, -2).contiguous()
        self.z = self.q @ kt
        self.ez = 4 * math.sqrt(d) * F * (self.q.abs() @ kt.abs())

    def forward(self):
        """(value, bound, ...) of o and stats."""
        s = self.scale
        z = torch.where(self.on, self.z, -math.inf)
        m = z.amax(-1, keepdim=True) if self.lk else torch.full_like(z.sum(-1, keepdim=True), -math.inf)
        empty = m == -math.inf
        x = torch.where(self.on, (z - torch.where(empty, 0.0, m)) * s, -math.inf)
        total = torch.exp(x).sum(-1, keepdim=True)
        l = torch.log(total)
        p = torch.where(self.on, torch.exp(x) / torch.where(empty, 1.0, total), 0.0)
        far = torch.where(self.on, x.abs(), 0.0).clamp(max=1e4)
        # a probability's numerator; below float32's normal numbers it is 0
        ep = p * (s * self.ez + 8 * F * far + 8 * F) + FLUSH * self.on
        es = ep.sum(-1, keepdim=True) + (4 * math.sqrt(max(self.lk, 1)) + 8) * F * (~empty)
        o = p @ self.v
        va = self.v.abs()
        e32 = (ep + 4 * math.sqrt(max(self.lk, 1)) * F * p + p * es) @ va
        eo = e32 + self.held * (p @ va)
        var = (self.u ** 2 / 3) * o * o + (self.held ** 2 / 3) * ((p * p) @ (va * va))
        few = 2.5 if o.numel() < 1000 else 1.25
        em = torch.where(self.on, self.ez, 0.0).amax(-1, keepdim=True) + F * torch.where(empty, 0.0, m.abs()) if self.lk else torch.zeros_like(m)
        el = es + s * em + 4 * F * torch.where(empty, 0.0, l.abs()) + 8 * F
        stats = torch.stack([m, l], -1)[..., 0, :]
        # the same infinities leave a difference that is no number
        bound = torch.where(torch.isinf(stats), 0.0, torch.stack([em, el], -1)[..., 0, :] + TINY)
        back = lambda t: t.transpose(1, 2)
        return (back(o), back(self.u * o.abs() * (1 + 2 ** -7) + eo * (1 + 2 ** -7) + TINY), few, back(var), back(e32)), (back(stats), back(bound))

    def backward(self, o, stats, dout):
        """(value, bound, ...) of dq, dk and dv from the o and stats that the library has."""
        s, held, u = self.scale, self.held, self.u
        # calls of few rows multiply by what rounding p and ds left, too, as it is rounded
        if self.q.shape[0] * self.q.shape[1] * self.lq <= 512:
            held = held * held
        ok = self.qok[:, :, None, None]
        g = torch.where(ok, dout.double(), 0.0).transpose(1, 2)
        od = torch.where(ok, o.double(), 0.0).transpose(1, 2)
        m, l = (stats.double().transpose(1, 2)[..., i:i + 1] for i in range(2))
        on = self.on & (m > -math.inf)
        x = torch.where(on, (self.z - torch.where(m > -math.inf, m, 0.0)) * s - torch.where(m > -math.inf, l, 0.0), -math.inf)
        p = torch.exp(x)
        far = torch.where(on, x.abs() + l.abs(), 0.0).clamp(max=1e4)
        ep = p * (s * self.ez + 8 * F * far + 8 * F) + FLUSH * on
        g = torch.where(m > -math.inf, g, 0.0)
        vt = self.v.transpose(-1, -2).contiguous()
        dp = g @ vt
        edp = 4 * math.sqrt(self.d) * F * (g.abs() @ vt.abs())
        # delta is the sum of p dp; of more than 128 keys it may be that of dout and o as o
        # was rounded, which is off by a known difference
        delta = (p * dp).sum(-1, keepdim=True)
        many = (self.on.sum(-1, keepdim=True) > 128).double()
        sums = (p * dp.abs()).sum(-1, keepdim=True) + (g * od).abs().sum(-1, keepdim=True)
        ede = 4 * math.sqrt(max(self.d, self.lk)) * F * sums + (p * edp + ep * dp.abs()).sum(-1, keepdim=True)
        ede = ede + many * ((g * od).sum(-1, keepdim=True) - delta).abs()
        ds = p * (dp - delta)
        eds = ep * (dp - delta).abs() + p * (edp + ede + 2 * F * (dp.abs() + delta.abs())) + FLUSH * on
        kq, kk = 4 * math.sqrt(max(self.lk, 1)) * F, 4 * math.sqrt(max(self.lq * self.n, 1)) * F
        dq = s * (ds @ self.k)
        edq = s * ((eds + kq * ds.abs()) @ self.k.abs()) + 2 * F * dq.abs()
        hdq = s * held * (ds.abs() @ self.k.abs())
        vdq = (u ** 2 / 3) * dq * dq + (held ** 2 / 3) * s * s * ((ds * ds) @ (self.k * self.k))
        t = lambda a: a.transpose(-1, -2).contiguous()
        group = lambda a: a.reshape(a.shape[0], -1, self.n, *a.shape[2:]).sum(2)
        dk, dv = s * group(t(ds) @ self.q), group(t(p) @ g)
        edk = s * group(t(eds + kk * ds.abs()) @ self.q.abs()) + 2 * F * dk.abs()
        hdk = s * held * group(t(ds.abs()) @ self.q.abs())
        edv = group(t(ep + kk * p) @ g.abs())
        hdv = held * group(t(p) @ g.abs())
        vdk = (u ** 2 / 3) * dk * dk + (held ** 2 / 3) * s * s * group(t(ds * ds) @ (self.q * self.q))
        vdv = (u ** 2 / 3) * dv * dv + (held ** 2 / 3) * group(t(p * p) @ (g * g))
        out = []
        for a, e, h, var in ((dq, edq, hdq, vdq), (dk, edk, hdk, vdk), (dv, edv, hdv, vdv)):
            few = 2.5 if a.numel() < 1000 else 1.25
            bound = u * a.abs() * (1 + 2 ** -7) + (e + h) * (1 + 2 ** -7) + TINY
            out.append((a.transpose(1, 2), bound.transpose(1, 2), few, var.transpose(1, 2), e.transpose(1, 2)))
        return out


def check_stats(got, want):
    """Infinities as they are, other values within their bounds."""
    value, bound = want
    same = got.double() == value
    off = (got.double() - value).abs()
    bad = ~same & ~(off <= bound)
    assert not bool(bad.any()), f"stats: {int(bad.sum())} values off, the first at {bad.nonzero()[0].tolist()}: {got[bad][0]} against {value[bad][0]}"

"""Rotary positions with the heads' norm on the GPU against their definition in 64
bits, forward and backward; every output and workspace lies between guards."""
import math

import pytest
import torch

import paper_2210_08650_amd as H
from tests import block_reference as R
from tests.hip_harness import Guarded

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
CODE = {BF: H.HAPI_BF16, F32: H.HAPI_F32}


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


class Case:
    def __init__(self, seed, dtype, batch, length, heads, kv_heads, dim, sections, neighbours=False, norm=True, lens=None, far=100,
                 pad=0, transposed=False, eps=1e-6):
        g = _gen(seed)
        self.dtype, self.batch, self.length, self.dim, self.norm, self.eps = dtype, batch, length, dim, norm, eps
        self.heads, self.sections, self.neighbours = (heads, kv_heads), tuple(sections), neighbours
        self.pad, self.transposed = pad, transposed
        self.x, self.dy, self.gamma = [], [], []
        for h in self.heads:
            self.x.append(self.tensor(h, torch.randn(batch, length, h, dim, generator=g, device="cuda")) if h else None)
            self.dy.append(self.tensor(h, torch.randn(batch, length, h, dim, generator=g, device="cuda")) if h else None)
            self.gamma.append(torch.randn(dim, generator=g, device="cuda") * 0.2 + 1.0 if h and norm else None)
        p = sum(sections)
        self.positions = torch.randint(-far, far + 1, (len(sections), batch, length), generator=g, device="cuda") if sections else None
        self.freq = torch.tensor([100.0 ** (-j / m) for m in sections for j in range(m)], dtype=torch.float64, device="cuda") if p else None
        self.lens = None if lens is None else torch.tensor(lens, device="cuda")

    def tensor(self, heads, values=None, guard=False):
        """[batch, length, heads, dim], in memory with `pad` values between the heads, or the
        heads outside the tokens."""
        b, l, d = self.batch, self.length, self.dim + self.pad
        shape = (b, heads, l, d) if self.transposed else (b, l, heads, d)
        if guard:
            buf = Guarded(math.prod(shape) * torch.empty(0, dtype=self.dtype).element_size())
            t = buf.view(self.dtype, shape)
            t.fill_(5.0)
        else:
            t = torch.full(shape, 7.0, dtype=self.dtype, device="cuda")
        v = t[..., :self.dim]
        if self.transposed:
            v = v.transpose(1, 2)
        if values is not None:
            v.copy_(values)
        return (v, t, buf) if guard else v

    def desc(self):
        def st(i):
            return self.x[i].stride()[:3] if self.heads[i] else ()
        d = H.Rotary(CODE[self.dtype], self.batch, self.length, *self.heads, self.dim, self.sections, self.neighbours, self.norm, self.eps,
                     st(0), st(1), st(0), st(1), stream=torch.cuda.current_stream())
        self.ws = Guarded(H.hapi_rotary_workspace_bytes(d))
        if self.ws.nbytes:
            d.set(workspace=self.ws.body, workspace_bytes=self.ws.nbytes)
        return d

    def outputs(self):
        return [self.tensor(h, guard=True) if h else (None, None, None) for h in self.heads]

    def checked(self, outs):
        torch.cuda.synchronize()
        self.ws.check()
        for v, t, buf in outs:
            if buf:
                buf.check()
                if self.pad:
                    assert bool((t[..., self.dim:] == 5.0).all()), "wrote between heads"
        return [v for v, _, _ in outs]

    def forward(self):
        d, outs = self.desc(), self.outputs()
        H.hapi_rotary_forward(d, *self.x, *self.gamma, self.positions, self.freq, self.lens, outs[0][0], outs[1][0])
        return self.checked(outs)

    def backward(self):
        d, outs = self.desc(), self.outputs()
        bufs = [Guarded(4 * self.dim) if self.norm and h else None for h in self.heads]
        dg = [b.view(F32, (self.dim,)) if b else None for b in bufs]
        xs = self.x if self.norm else [None, None]
        H.hapi_rotary_backward(d, *self.dy, *xs, *self.gamma, self.positions, self.freq, self.lens, outs[0][0], outs[1][0], *dg)
        out = self.checked(outs)
        for b in bufs:
            if b:
                b.check()
        return out, dg

    def check(self):
        y = self.forward()
        dx, dg = self.backward()
        for i, name in enumerate("qk"):
            if not self.heads[i]:
                continue
            more = (self.positions, self.freq, self.sections, self.neighbours, self.eps, self.lens)
            R.check(name + "_out", y[i], R.rotary_forward(self.x[i], self.gamma[i], *more))
            want = R.rotary_backward(self.dy[i], self.x[i], self.gamma[i], *more)
            R.check("d" + name, dx[i], want[0])
            if self.norm:
                R.check(f"d{name}_gamma", dg[i], want[1])


SHAPES = [
    # batch, length, heads, kv_heads, dim, sections
    (1, 1, 1, 0, 1, ()), (1, 1, 1, 1, 2, (1,)), (2, 3, 0, 2, 3, (1,)), (1, 197, 12, 12, 64, (16, 16)), (3, 5, 2, 1, 64, (32,)),
    (2, 7, 15, 5, 80, (10, 10, 10)), (2, 33, 3, 1, 72, (12, 12, 12)), (1, 9, 4, 4, 128, (64,)), (4, 3, 32, 8, 128, (16, 24, 24)),
    (1, 50, 5, 0, 96, (24, 8)), (2, 11, 2, 2, 33, (8, 8)), (1, 6, 2, 2, 255, (100,)), (2, 4, 3, 1, 256, (32, 32, 32, 32)),
    (1, 5, 1, 1, 254, (127,)), (3, 17, 7, 3, 40, (1, 2, 3, 4)), (2, 600, 8, 2, 16, (4, 4)), (1, 13, 6, 6, 100, (25, 25)), (5, 1, 24, 2, 64, ()),
]


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("shape", SHAPES)
def test_rotary(shape, dtype, neighbours):
    Case(sum(shape[:5]), dtype, *shape, neighbours=neighbours).check()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("batch,length,heads,kv_heads,dim,sections,neighbours,pad", [
    (8, 3001, 4, 2, 64, (16, 16), False, 0), (3, 5003, 3, 1, 128, (24, 16, 24), True, 8), (2, 4099, 15, 5, 80, (40,), False, 0),
    (7, 1009, 12, 4, 72, (8, 8), False, 0), (2, 3001, 8, 8, 96, (12, 12), True, 16)])
def test_many_tokens(batch, length, heads, kv_heads, dim, sections, neighbours, pad, dtype):
    """Enough vectors for 16 bytes a lane; some sequences shorter."""
    lens = [(length * (i + 1)) // batch - 3 * i for i in range(batch)]
    Case(41, dtype, batch, length, heads, kv_heads, dim, sections, neighbours=neighbours, pad=pad, lens=lens).check()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("shape", SHAPES[3:12])
def test_without_norm(shape, dtype):
    Case(1, dtype, *shape, norm=False).check()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("dim,pad,transposed", [(64, 8, False), (64, 3, False), (64, 0, True), (80, 1, True), (33, 2, False)])
def test_strides(dim, pad, transposed, dtype):
    Case(2, dtype, 2, 19, 4, 2, dim, (dim // 4, dim // 4), pad=pad, transposed=transposed).check()


def test_many_heads_and_tokens():
    """More vectors than the lanes of the chip: several heads to a lane, several tokens to a block."""
    Case(3, BF, 16, 197, 24, 12, 64, (16, 16)).check()
    Case(3, F32, 5, 1000, 40, 8, 128, (64,)).check()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_far_positions(dtype):
    Case(4, dtype, 2, 40, 2, 2, 64, (32,), far=1 << 30).check()


def test_padding_is_not_read():
    lens = [0, 3, 7, 9, -2]
    for norm in (True, False):
        c = Case(5, BF, 5, 7, 3, 2, 64, (16, 16), norm=norm, lens=lens)
        for x in c.x + c.dy:
            for b, n in enumerate(lens):
                x[b, max(n, 0):] = math.nan
        c.check()
    # a vector of zeros has no direction with eps = 0; padding is zeros all the same
    c = Case(5, F32, 5, 7, 3, 2, 64, (16, 16), lens=lens, eps=0.0)
    c.check()


def test_nan_stays_in_its_vector():
    c = Case(6, F32, 2, 9, 3, 1, 64, (16, 16))
    c.x[0][1, 4, 2, 5] = math.nan
    y = c.forward()[0]
    bad = torch.isnan(y)
    assert bool(bad[1, 4, 2].all()) and int(bad.sum()) == 64


def test_in_place():
    for dtype in (BF, F32):
        c = Case(7, dtype, 3, 21, 5, 2, 80, (20, 20))
        y = c.forward()
        dx, dg = c.backward()
        d = c.desc()
        x = [v.clone() for v in c.x]
        H.hapi_rotary_forward(d, *x, *c.gamma, c.positions, c.freq, None, *x)
        assert all(torch.equal(a, b) for a, b in zip(x, y))
        dy = [v.clone() for v in c.dy]
        g = [torch.empty_like(v) for v in dg]
        H.hapi_rotary_backward(d, *dy, *c.x, *c.gamma, c.positions, c.freq, None, *dy, *g)
        assert all(torch.equal(a, b) for a, b in zip(dy + g, dx + dg))


def test_unaligned_start():
    c = Case(8, BF, 2, 5, 3, 3, 64, (32,))
    y = c.forward()
    flat = [torch.empty(v.numel() + 1, dtype=BF, device="cuda") for v in c.x]
    moved = [f[1:].view(v.shape) for f, v in zip(flat, c.x)]
    for m, v in zip(moved, c.x):
        m.copy_(v)
    c.x = moved
    assert all(torch.equal(a, b) for a, b in zip(c.forward(), y))


def test_broadcast_input():
    """One entry's tokens for the whole batch (a stride of 0): read, but no place for gradients."""
    c = Case(9, F32, 3, 5, 2, 1, 64, (32,))
    d = H.Rotary(H.HAPI_F32, 3, 5, 2, 0, 64, (32,), q_stride=(0, 128, 64), stream=torch.cuda.current_stream())
    q = c.x[0][:1].expand(3, 5, 2, 64)
    out = torch.empty(3, 5, 2, 64, device="cuda")
    H.hapi_rotary_forward(d, q, None, c.gamma[0], None, c.positions, c.freq, None, out, None)
    R.check("q_out", out, R.rotary_forward(q, c.gamma[0], c.positions, c.freq, (32,)))


def test_no_tokens():
    c = Case(10, F32, 0, 5, 2, 1, 64, (32,))
    c.forward()
    dx, dg = c.backward()
    assert all(bool((g == 0).all()) for g in dg)


def test_offsets_past_32_bits():
    """2.2e9 elements from the first token to the last."""
    flat = torch.zeros((1 << 31) + (1 << 28), dtype=BF, device="cuda")
    x = flat.as_strided((3, 2, 2, 64), (1 << 30, 64, 1 << 27, 1))
    x.copy_(torch.randn(3, 2, 2, 64, generator=_gen(11), device="cuda"))
    gamma = torch.ones(64, device="cuda")
    pos = torch.arange(6, device="cuda").view(1, 3, 2)
    freq = torch.tensor([100.0 ** (-j / 32) for j in range(32)], dtype=torch.float64, device="cuda")
    d = H.Rotary(H.HAPI_BF16, 3, 2, 2, 0, 64, (32,), q_stride=x.stride()[:3], q_out_stride=x.stride()[:3], stream=torch.cuda.current_stream())
    want = R.rotary_forward(x, gamma, pos, freq, (32,))
    H.hapi_rotary_forward(d, x, None, gamma, None, pos, freq, None, x, None)
    R.check("q_out", x, want)


def test_gradient_against_differences():
    """Central differences of the library's own float32 forward pass: truncation is
    h^2 / 6 of the third derivative (some 10 of the slope's size for h = 1e-2: 2e-4),
    each y is off by 3e-6 at most, so the quotient by 3e-6 |dy|_1 / h."""
    c = Case(12, F32, 1, 4, 2, 1, 40, (6, 6))
    dx, dg = c.backward()
    dx = [v.clone() for v in dx]
    x0, g, h = [v.clone() for v in c.x], _gen(13), 1e-2
    noise = 3e-6 * sum(float(v.abs().sum()) for v in c.dy) / h

    def f(step, v):
        for i in range(2):
            c.x[i].copy_(x0[i] + step * v[i])
        return sum(float((y.double() * dy.double()).sum()) for y, dy in zip(c.forward(), c.dy))
    v = [torch.randn(x.shape, generator=g, device="cuda") for x in x0]
    slope = (f(h, v) - f(-h, v)) / (2 * h)
    want = sum(float((a.double() * b.double()).sum()) for a, b in zip(dx, v))
    size = sum(float((a.double() * b.double()).abs().sum()) for a, b in zip(dx, v))
    assert abs(slope - want) <= noise + 1e-3 * size


def test_captured_and_replayed():
    c = Case(14, BF, 4, 50, 6, 2, 64, (16, 16))
    outs = [torch.empty_like(x) for x in c.x]
    dxs = [torch.empty_like(x) for x in c.x]
    dgs = [torch.empty(64, device="cuda") for _ in c.x]
    d = c.desc()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        d.set(stream=torch.cuda.current_stream())
        H.hapi_rotary_forward(d, *c.x, *c.gamma, c.positions, c.freq, None, *outs)
        H.hapi_rotary_backward(d, *c.dy, *c.x, *c.gamma, c.positions, c.freq, None, *dxs, *dgs)
    ws = c.ws
    for k in range(3):
        for x in c.x + c.dy:
            x.copy_(torch.randn(x.shape, generator=_gen(20 + k), device="cuda"))
        c.positions += 1
        y = c.forward()
        dx, dg = c.backward()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs + dxs + dgs, y + dx + dg))
    ws.check()

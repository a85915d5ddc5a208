"""Cross attention on the GPU against its definition in 64 bits, forward and backward;
every output and workspace lies between guards."""
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
    def __init__(self, seed, dtype, batch, q_len, kv_len, heads, kv_heads, dim, q_lens=None, kv_lens=None, mask=None, pad=0,
                 transposed=False, scale=0.0, spread=1.0):
        g = _gen(seed)
        self.dtype, self.batch, self.q_len, self.kv_len, self.heads, self.kv_heads, self.dim = dtype, batch, q_len, kv_len, heads, kv_heads, dim
        self.pad, self.transposed, self.scale = pad, transposed, scale
        r = lambda l, h, k=1.0: self.tensor(l, h, torch.randn(batch, l, h, dim, generator=g, device="cuda") * k)
        self.q, self.k, self.v, self.dout = r(q_len, heads, spread), r(kv_len, kv_heads, spread), r(kv_len, kv_heads), r(q_len, heads)
        as_lens = lambda x: None if x is None else torch.tensor(x, device="cuda")
        self.q_lens, self.kv_lens = as_lens(q_lens), as_lens(kv_lens)
        self.mask = None if mask is None else torch.rand(batch, kv_len, generator=g, device="cuda") < mask

    def tensor(self, length, heads, values=None, guard=False):
        """[batch, length, heads, dim], in memory with `pad` values between the heads, or the
        heads outside the tokens."""
        b, d = self.batch, self.dim + self.pad
        shape = (b, heads, length, d) if self.transposed else (b, length, heads, d)
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

    def desc(self, backward):
        plain = self.pad == 0 and not self.transposed
        st = lambda x: () if plain else x.stride()[:3]
        d = H.Attention(CODE[self.dtype], self.batch, self.q_len, self.kv_len, self.heads, self.kv_heads, self.dim, self.scale,
                        st(self.q), st(self.k), st(self.v), st(self.dout), stream=torch.cuda.current_stream())
        self.ws = Guarded(H.hapi_cross_attention_workspace_bytes(d, backward))
        self.ws.body.fill_(0xff)  # NaN in either type, whatever is read before it is written
        if self.ws.nbytes:
            d.set(workspace=self.ws.body, workspace_bytes=self.ws.nbytes)
        return d

    def checked(self, outs):
        torch.cuda.synchronize()
        self.ws.check()
        for v, t, buf in outs:
            buf.check()
            if self.pad:
                assert bool((t[..., self.dim:] == 5.0).all()), "wrote between heads"
        return [v for v, _, _ in outs]

    def forward(self):
        d, o = self.desc(False), self.tensor(self.q_len, self.heads, guard=True)
        sb = Guarded(8 * self.batch * self.q_len * self.heads)
        st = sb.view(F32, (self.batch, self.q_len, self.heads, 2))
        st.fill_(3.0)
        H.hapi_cross_attention_forward(d, self.q, self.k, self.v, self.q_lens, self.kv_lens, self.mask, o[0], st)
        out = self.checked([o])[0]
        sb.check()
        return out, st

    def backward(self, o, st):
        d = self.desc(True)
        outs = [self.tensor(l, h, guard=True) for l, h in ((self.q_len, self.heads), (self.kv_len, self.kv_heads), (self.kv_len, self.kv_heads))]
        H.hapi_cross_attention_backward(d, self.q, self.k, self.v, self.q_lens, self.kv_lens, self.mask, o, st, self.dout, *[x[0] for x in outs])
        return self.checked(outs)

    def reference(self):
        return R.Attention(self.q, self.k, self.v, self.scale, self.q_lens, self.kv_lens, self.mask)

    def check(self):
        ref = self.reference()
        o, st = self.forward()
        want = ref.forward()
        R.check("o", o, want[0])
        R.check_stats(st, want[1])
        for name, got, w in zip(("dq", "dk", "dv"), self.backward(o, st), ref.backward(o, st, self.dout)):
            R.check(name, got, w)


SHAPES = [
    # batch, q_len, kv_len, heads, kv_heads, dim
    (1, 1, 1, 1, 1, 1), (1, 1, 1, 1, 1, 64), (2, 1, 5, 3, 1, 8), (1, 2, 33, 2, 2, 32), (2, 31, 31, 1, 1, 64), (1, 32, 32, 2, 1, 64),
    (1, 33, 63, 3, 3, 64), (2, 64, 64, 4, 2, 64), (1, 65, 65, 1, 1, 128), (2, 127, 127, 2, 2, 128), (1, 128, 128, 3, 1, 64),
    (1, 129, 129, 2, 1, 96), (3, 64, 197, 12, 12, 64), (2, 7, 1000, 16, 4, 128), (1, 1, 3000, 8, 1, 128), (2, 1, 4097, 5, 5, 64),
    (1, 300, 17, 2, 2, 64), (1, 1500, 40, 4, 1, 64), (1, 2001, 3, 1, 1, 128), (2, 77, 250, 12, 4, 80), (2, 19, 90, 6, 2, 72),
    (1, 50, 70, 5, 1, 33), (1, 40, 100, 3, 3, 100), (2, 21, 45, 7, 7, 3), (1, 90, 120, 10, 2, 127), (1, 60, 300, 24, 2, 40),
    (1, 11, 30, 64, 1, 16), (1, 3, 300, 100, 1, 128), (40, 3, 5, 2, 1, 64), (1, 513, 257, 3, 3, 32),
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("shape", SHAPES)
def test_attention(shape, dtype):
    Case(sum(shape), dtype, *shape).check()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("shape", [SHAPES[i] for i in (3, 7, 12, 13, 17, 19, 21)])
def test_lengths_and_mask(shape, dtype):
    """Ragged batches; NaN in every place that takes no part; rows that the mask leaves nothing."""
    b, lq, lk = shape[:3]
    b = max(b, 5)
    q_lens = [lq, 0, lq // 2, 1, lq + 7][:b] + [lq] * (b - 5)
    kv_lens = [lk // 3, lk, 0, -4, 1 << 40][:b] + [lk] * (b - 5)
    for mask in (None, 0.6):
        c = Case(sum(shape), dtype, b, *shape[1:], q_lens=q_lens, kv_lens=kv_lens, mask=mask)
        if mask:
            c.mask[-1] = False
        off = ~((torch.arange(lk, device="cuda") < c.kv_lens[:, None]) & (torch.ones(b, lk, dtype=torch.bool, device="cuda") if c.mask is None else c.mask))
        c.k[off] = math.nan
        c.v[off] = math.inf
        pad = ~(torch.arange(lq, device="cuda") < c.q_lens[:, None])
        c.q[pad] = math.nan
        c.dout[pad] = math.nan
        c.check()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("dim,pad,transposed", [(64, 8, False), (64, 3, False), (64, 0, True), (80, 1, True), (33, 2, False), (128, 0, True)])
def test_strides(dim, pad, transposed, dtype):
    Case(2, dtype, 2, 45, 77, 4, 2, dim, pad=pad, transposed=transposed).check()
    Case(3, dtype, 2, 1, 700, 4, 2, dim, pad=pad, transposed=transposed, mask=0.5).check()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_long_rows_and_keys(dtype):
    """Many tiles in a row: offsets, buffers that take turns, several splits."""
    Case(4, dtype, 1, 700, 5000, 2, 1, 64).check()
    Case(5, dtype, 1, 4000, 150, 2, 2, 128).check()
    Case(6, dtype, 2, 3, 9000, 4, 1, 96, kv_lens=[9000, 4321]).check()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_scores_of_all_sizes(dtype):
    """Scores near 1e4, where a row is one key's, and a scale of the caller's own."""
    Case(7, dtype, 2, 40, 90, 2, 2, 64, spread=35.0).check()
    Case(8, dtype, 2, 40, 90, 2, 2, 64, scale=0.01).check()
    Case(9, dtype, 1, 5, 300, 2, 1, 128, scale=3.0).check()


def test_rising_and_falling_scores():
    """Keys in order of their score: the running maximum moves at every tile, or never again."""
    for dtype in (BF, F32):
        for sign in (1.0, -1.0):
            c = Case(10, dtype, 1, 70, 600, 1, 1, 64)
            c.q.fill_(0.25)
            c.k.copy_((sign * torch.arange(600, device="cuda") / 20.0)[None, :, None, None].expand(1, 600, 1, 64).contiguous() / 4)
            c.check()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_one_key_has_no_gradient_of_scores(dtype):
    """Of one key p is 1 whatever its score: dq and dk are 0, not roundings."""
    for c in (Case(23, dtype, 3, 40, 1, 4, 2, 64), Case(24, dtype, 2, 5, 900, 4, 1, 128, kv_lens=[1, 1]),
              Case(25, dtype, 1, 70, 700, 2, 2, 80, mask=0.0)):
        if c.mask is not None:
            c.mask[:, 600] = True
        o, st = c.forward()
        dq, dk, _ = c.backward(o, st)
        assert not bool(dq.any()) and not bool(dk.any())
        c.check()


@pytest.mark.parametrize("b,lq,lk,h,kv,d", [
    (1, 5, 1200, 2, 2, 64), (1, 50, 1200, 2, 1, 32), (200, 3, 600, 1, 1, 40), (100, 20, 700, 6, 2, 64), (2, 64, 130, 4, 4, 64),
    (3, 13, 260, 10, 2, 24), (2, 1, 33, 64, 1, 64), (2, 31, 1, 2, 1, 64), (2, 65, 300, 2, 2, 64), (40, 10, 300, 2, 1, 32),
    (40, 30, 300, 2, 1, 32), (200, 40, 70, 1, 1, 17)])
def test_few_rows(b, lq, lk, h, kv, d):
    """Heads of up to 64 rows, one group's or many's: keys split over workgroups or not."""
    c = Case(31, BF, b, lq, lk, h, kv, d)
    c.check()
    lens = torch.arange(b, device="cuda") * 97
    Case(32, BF, b, lq, lk, h, kv, d, q_lens=(lens % (lq + 1)).tolist(), kv_lens=(lens % (lk + 1)).tolist()).check()
    Case(33, BF, b, lq, lk, h, kv, d, mask=0.7).check()
    c = Case(34, BF, b, lq, lk, h, kv, d, mask=0.0)  # few kept keys, in some blocks only
    c.mask[:, lk // 3::97] = True
    c.check()


@pytest.mark.parametrize("b,lq,lk,h,kv,d", [
    (2, 150, 300, 4, 2, 128), (3, 100, 190, 4, 4, 96), (2, 300, 77, 2, 1, 64), (4, 90, 130, 2, 2, 32), (1, 40, 700, 16, 4, 120),
    (9, 7, 90, 10, 2, 72), (3, 20, 1000, 12, 12, 128), (20, 33, 100, 1, 1, 128), (2, 257, 31, 3, 1, 96)])
def test_more_than_512_rows(b, lq, lk, h, kv, d):
    """Calls whose gradients take P and dS as they are rounded."""
    assert b * lq * h > 512
    Case(35, BF, b, lq, lk, h, kv, d).check()
    lens = torch.arange(1, b + 1, device="cuda") * 61
    Case(36, BF, b, lq, lk, h, kv, d, q_lens=(lens % (lq + 1)).tolist(), kv_lens=(lens % (lk + 1)).tolist(), pad=8).check()
    Case(37, BF, b, lq, lk, h, kv, d, mask=0.5).check()


def test_every_length_around_a_tile():
    for lk in list(range(1, 70, 3)) + [95, 96, 97, 127, 128, 129, 191, 192, 193, 255, 256, 257]:
        Case(lk, BF, 2, 5, lk, 2, 1, 64).check()
    for lq in [1, 15, 16, 17, 31, 32, 33, 47, 48, 63, 64, 65, 96, 127, 128, 129, 200]:
        Case(lq, BF, 1, lq, 50, 3, 1, 64).check()


def test_no_keys_and_no_queries():
    c = Case(11, BF, 2, 5, 0, 2, 1, 64)
    o, st = c.forward()
    assert not bool(o.any()) and bool((st == -math.inf).all())
    assert not bool(c.backward(o, st)[0].any())
    c = Case(12, BF, 2, 0, 5, 2, 1, 64)
    o, st = c.forward()
    dq, dk, dv = c.backward(o, st)
    assert not bool(dk.any()) and not bool(dv.any())
    c = Case(13, F32, 0, 4, 5, 2, 1, 64)
    c.backward(*c.forward())


def test_nan_stays_with_its_query():
    c = Case(14, BF, 2, 40, 80, 4, 2, 64)
    c.q[1, 7, 2, 3] = math.nan
    o, _ = c.forward()
    bad = torch.isnan(o)
    assert bool(bad[1, 7, 2].all()) and int(bad.sum()) == 64


def test_unaligned_output():
    c = Case(15, BF, 1, 20, 50, 2, 1, 64)
    o, st = c.forward()
    flat = torch.empty(o.numel() + 1, dtype=BF, device="cuda")
    d = c.desc(False)
    H.hapi_cross_attention_forward(d, c.q, c.k, c.v, None, None, None, flat[1:].view(o.shape), st.clone())
    assert torch.equal(flat[1:].view(o.shape), o)


def test_packed_and_broadcast_inputs():
    """Keys and values inside one projection, and one entry's keys for the whole batch."""
    g = _gen(16)
    kv = torch.randn(3, 60, 2, 2, 64, generator=g, device="cuda").to(BF)
    q = torch.randn(3, 9, 4, 64, generator=g, device="cuda").to(BF)
    k, v = kv[:, :, 0], kv[:, :, 1]
    for kk, vv in ((k, v), (k[:1].expand(3, 60, 2, 64), v[:1].expand(3, 60, 2, 64))):
        d = H.Attention(H.HAPI_BF16, 3, 9, 60, 4, 2, 64, k_stride=kk.stride()[:3], v_stride=vv.stride()[:3], stream=torch.cuda.current_stream())
        ws = Guarded(H.hapi_cross_attention_workspace_bytes(d, True))
        d.set(workspace=ws.body, workspace_bytes=ws.nbytes)
        o, st = torch.empty_like(q), torch.empty(3, 9, 4, 2, device="cuda")
        H.hapi_cross_attention_forward(d, q, kk, vv, None, None, None, o, st)
        ref = R.Attention(q, kk, vv)
        R.check("o", o, ref.forward()[0])
        dout = torch.randn(q.shape, generator=g, device="cuda").to(BF)
        grad = torch.empty_like(kv)
        if kk.stride(0) == 0:
            with pytest.raises(H.HapiError):
                H.hapi_cross_attention_backward(d, q, kk, vv, None, None, None, o, st, dout, torch.empty_like(q), kk, vv)
            continue
        dq = torch.empty_like(q)
        H.hapi_cross_attention_backward(d, q, kk, vv, None, None, None, o, st, dout, dq, grad[:, :, 0], grad[:, :, 1])
        for name, a, w in zip(("dq", "dk", "dv"), (dq, grad[:, :, 0], grad[:, :, 1]), ref.backward(o, st, dout)):
            R.check(name, a, w)


def test_offsets_past_32_bits():
    """Batch entries and heads more than 2^31 values apart."""
    flat = torch.zeros((1 << 32) + (1 << 20), dtype=BF, device="cuda")
    kb = flat.as_strided((2, 300, 1, 64), (1 << 32, 64, 64, 1))
    kb.copy_(torch.randn(2, 300, 1, 64, generator=_gen(17), device="cuda"))
    c = Case(17, BF, 2, 4, 300, 2, 1, 64)
    ref = R.Attention(c.q, kb, c.v)
    d = H.Attention(H.HAPI_BF16, 2, 4, 300, 2, 1, 64, k_stride=kb.stride()[:3], stream=torch.cuda.current_stream())
    ws = torch.empty(H.hapi_cross_attention_workspace_bytes(d, True), dtype=torch.uint8, device="cuda")
    d.set(workspace=ws, workspace_bytes=ws.numel())
    o, st = torch.empty_like(c.q), torch.empty(2, 4, 2, 2, device="cuda")
    H.hapi_cross_attention_forward(d, c.q, kb, c.v, None, None, None, o, st)
    R.check("o", o, ref.forward()[0])
    dk = torch.zeros_like(flat).as_strided(kb.shape, kb.stride())
    dq, dv = torch.empty_like(c.q), torch.empty_like(c.v)
    H.hapi_cross_attention_backward(d, c.q, kb, c.v, None, None, None, o, st, c.dout, dq, dk, dv)
    for name, a, w in zip(("dq", "dk", "dv"), (dq, dk, dv), ref.backward(o, st, c.dout)):
        R.check(name, a, w)


def test_gradient_against_differences():
    """Central differences of the library's own float32 forward pass along a random
    direction: truncation is h^2 / 6 of the third derivative (some 10 of the slope's size
    for h = 1e-2: 2e-4), each o is off by 5e-6 at most, so the quotient by 5e-6 |dout|_1 / h."""
    c = Case(18, F32, 2, 6, 9, 4, 2, 40, kv_lens=[9, 5], q_lens=[4, 6])
    o, st = c.forward()
    grads = [g.clone() for g in c.backward(o, st)]
    x0, g, h = [x.clone() for x in (c.q, c.k, c.v)], _gen(19), 1e-2
    v = [torch.randn(x.shape, generator=g, device="cuda") for x in x0]
    counts = (torch.arange(6, device="cuda") < c.q_lens[:, None])[:, :, None, None]

    def f(step):
        for x, a, b in zip((c.q, c.k, c.v), x0, v):
            x.copy_(a + step * b)
        return float(torch.where(counts, c.forward()[0].double() * c.dout.double(), 0.0).sum())
    slope = (f(h) - f(-h)) / (2 * h)
    want = sum(float((a.double() * b.double()).sum()) for a, b in zip(grads, v))
    size = sum(float((a.double() * b.double()).abs().sum()) for a, b in zip(grads, v))
    assert abs(slope - want) <= 5e-6 * float(c.dout.abs().sum()) / h + 1e-3 * size


def test_the_same_bits_again_and_on_another_stream():
    c = Case(20, BF, 2, 300, 700, 6, 2, 128, mask=0.8)
    o, st = c.forward()
    first = [x.clone() for x in [o, st] + c.backward(o, st)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        o, st = c.forward()
        again = [o, st] + c.backward(o, st)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_captured_and_replayed():
    c = Case(21, BF, 3, 5, 2000, 8, 2, 64, kv_lens=[2000, 100, 777])
    d = c.desc(True)
    ws = c.ws
    o, st = torch.empty_like(c.q), torch.empty(3, 5, 8, 2, device="cuda")
    grads = [torch.empty_like(x) for x in (c.q, c.k, c.v)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        d.set(stream=torch.cuda.current_stream())
        H.hapi_cross_attention_forward(d, c.q, c.k, c.v, None, c.kv_lens, None, o, st)
        H.hapi_cross_attention_backward(d, c.q, c.k, c.v, None, c.kv_lens, None, o, st, c.dout, *grads)
    for k in range(3):
        for x in (c.q, c.k, c.v, c.dout):
            x.copy_(torch.randn(x.shape, generator=_gen(30 + k), device="cuda"))
        c.kv_lens.copy_(torch.tensor([5 + k, 2000, 64 * k], device="cuda"))
        want = c.forward()
        back = c.backward(*want)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip([o, st] + grads, list(want) + back))
    ws.check()


def test_two_streams_at_once():
    """Two calls in flight, each with a workspace of its own."""
    cs = [Case(22 + i, BF, 2, 200, 900, 4, 2, 64) for i in range(2)]
    want = [[x.clone() for x in c.forward()] for c in cs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cs]
    got = []
    for c, s in zip(cs, streams):
        with torch.cuda.stream(s):
            d = c.desc(False)
            o, st = torch.empty_like(c.q), torch.empty(2, 200, 4, 2, device="cuda")
            got.append((c.ws, o, st))
            for _ in range(5):
                H.hapi_cross_attention_forward(d, c.q, c.k, c.v, None, None, None, o, st)
    torch.cuda.synchronize()
    for (ws, o, st), w in zip(got, want):
        ws.check()
        assert torch.equal(o, w[0]) and torch.equal(st, w[1])

"""Rotary positions at the ends of what the header allows: values that are not rotated,
16 bytes a lane at odd addresses and strides."""
import math

import pytest
import torch

import paper_2210_08650_amd as H
from tests.test_gpu_rotary import BF, F32, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("batch,length,heads,kv_heads,dim,sections", [
    (1, 3, 2, 1, 64, (8, 8)), (2, 5, 1, 1, 33, (5,)), (1, 4, 2, 2, 6, ()), (4, 700, 8, 8, 128, (16, 16)), (1, 9, 3, 0, 255, (3, 4))])
def test_values_that_are_not_rotated_keep_their_bits(batch, length, heads, kv_heads, dim, sections, dtype, neighbours):
    """Without a norm they are copied: infinities, NaN and zeros' signs among them reach no
    other value, forward and backward."""
    c = Case(91, dtype, batch, length, heads, kv_heads, dim, sections, neighbours=neighbours, norm=False)
    p = 2 * sum(sections)
    for x in c.x + c.dy:
        if x is None:
            continue
        x[..., p] = math.inf
        x[..., dim - 1] = math.nan
        x[..., (p + dim) // 2] = -0.0
    bits = torch.int16 if dtype == BF else torch.int32
    y, (dx, _) = c.forward(), c.backward()
    for i in range(2):
        if c.heads[i]:
            for got, src in ((y[i], c.x[i]), (dx[i], c.dy[i])):
                assert torch.equal(got[..., p:].contiguous().view(bits), src[..., p:].contiguous().view(bits))
                assert bool(torch.isfinite(got[..., :p]).all())


def _moved(x):
    """The same values from one element past an aligned address."""
    y = torch.empty(x.numel() + 1, dtype=x.dtype, device="cuda")[1:].view(x.shape)
    y.copy_(x)
    return y


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("batch,length,heads,kv_heads,dim,sections,neighbours", [
    (8, 3001, 4, 2, 64, (16, 16), False), (3, 5003, 6, 2, 128, (24, 16, 24), True), (5, 2003, 15, 5, 80, (40,), False)])
def test_many_tokens_at_any_element(batch, length, heads, kv_heads, dim, sections, neighbours, dtype):
    """Calls of enough vectors for 16 bytes a lane, which are then loaded and stored at their
    elements' alignment: odd strides, and the same bits one element past an aligned address."""
    widest = 8 if dtype == BF else 4
    lanes = 4
    while lanes * 2 * widest < dim:
        lanes *= 2
    assert batch * length * (heads + kv_heads) * lanes >= 256 * 1024
    lens = [(length * (i + 1)) // batch - 3 * i for i in range(batch)]
    Case(92, dtype, batch, length, heads, kv_heads, dim, sections, neighbours=neighbours, pad=1, lens=lens).check()
    c = Case(93, dtype, batch, length, heads, kv_heads, dim, sections, neighbours=neighbours, lens=lens)
    y = c.forward()
    dx, dg = c.backward()
    x, dy, out = [_moved(v) for v in c.x], [_moved(v) for v in c.dy], [_moved(torch.zeros_like(v)) for v in c.x]
    d = c.desc()
    H.hapi_rotary_forward(d, *x, *c.gamma, c.positions, c.freq, c.lens, *out)
    assert all(torch.equal(a, b) for a, b in zip(out, y))
    g = [torch.empty_like(v) for v in dg]
    H.hapi_rotary_backward(d, *dy, *x, *c.gamma, c.positions, c.freq, c.lens, *out, *g)
    torch.cuda.synchronize()
    c.ws.check()
    assert all(torch.equal(a, b) for a, b in zip(out + g, dx + dg))

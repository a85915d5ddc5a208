"""Cross attention where scores, their sums and statistics are at the ends of their ranges."""
import math

import pytest
import torch

import paper_2210_08650_amd as H
from tests import block_reference as R
from tests.test_gpu_cross_attention import BF, CODE, F32, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("far", [30.0, 100.0, 250.0, 1000.0, 1e6, 1e30])
@pytest.mark.parametrize("b,lq,lk,h,kv,d,first", [
    (1, 3, 200, 2, 2, 64, 64), (1, 5, 700, 4, 1, 64, 512), (2, 40, 400, 2, 2, 32, 256), (1, 150, 300, 2, 1, 128, 128),
    (1, 70, 300, 3, 3, 96, 64), (300, 1, 160, 2, 1, 128, 96)])
def test_keys_far_below_the_rest_come_first(b, lq, lk, h, kv, d, first, far, dtype):
    """Whole tiles of scores of -far before ordinary ones: what the first keys are measured
    from is no measure for the others, whose scores keep their low bits."""
    c = Case(51, dtype, b, lq, lk, h, kv, d)
    c.q[..., 0] = 1.0
    c.k[..., 0] = 0.0
    c.k[:, :first, :, 0] = -far
    c.check()
    # the statistics' maximum is one of the ordinary keys', which the far ones' size does not blur
    ref = c.reference()
    m = c.forward()[1][..., 0].double().transpose(1, 2)
    z, ez = ref.z[..., first:], ref.ez[..., first:]
    off = (m - z.amax(-1)).abs()
    assert bool((off <= ez.amax(-1) + 4 * R.F * (z.abs().amax(-1) + 1)).all()), float(off.max())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("less", [0.375, 0.75, 1.5, 2.5])
def test_sums_of_many_equal_probabilities(less, dtype):
    """One key and 16383 whose scores are `less` below it, in calls whose keys are not split:
    the sum is 1 + 16383 exp(-less).  Equal terms round the same way each time, so a sum of n of
    them is off by up to n / 2 units F of itself: a lane's 16 of 32 keys 8, 512 times 32 keys
    256; exp2, its argument and the joins take less than 16 more.  o is a mean of ones: its own sums
    (16 products of a block, 512 blocks) are as far off, the quotient twice that."""
    b, lk, heads, d = 1, 16384, 300, 128
    q = torch.zeros(b, 1, heads, d, dtype=dtype, device="cuda")
    q[..., 0] = 1.0
    k = torch.zeros(b, lk, 1, d, dtype=dtype, device="cuda")
    k[:, 1:, :, 0] = -less
    v = torch.ones_like(k)
    k, v = (x.expand(b, lk, heads, d) for x in (k, v))
    desc = H.Attention(CODE[dtype], b, 1, lk, heads, heads, d, scale=1.0, k_stride=k.stride()[:3], v_stride=v.stride()[:3],
                       stream=torch.cuda.current_stream())
    assert H.hapi_cross_attention_workspace_bytes(desc) == 0  # no parts
    o, st = torch.empty_like(q), torch.empty(b, 1, heads, 2, device="cuda")
    H.hapi_cross_attention_forward(desc, q, k, v, None, None, None, o, st)
    want = math.log1p((lk - 1) * math.exp(-less))
    assert not bool(st[..., 0].any())
    assert float((st[..., 1].double() - want).abs().max()) <= 280 * R.F + 2 * R.F * want
    assert float((o.double() - 1.0).abs().max()) <= (2 * 280 * R.F if dtype == F32 else R.U[BF])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lq,lk,d", [(40, 80, 64), (3, 3000, 128), (200, 50, 32)])
def test_statistics_of_nan(lq, lk, d, dtype):
    """A query of NaN is no query without a key: its statistics are NaN, as its output, and so
    are all gradients that it reaches.  A key of NaN leaves a row the others' maximum."""
    c = Case(52, dtype, 2, lq, lk, 4, 2, d)
    c.q[1, 2, 3, 1] = math.nan
    o, st = c.forward()
    bad = torch.zeros(2, lq, 4, dtype=torch.bool, device="cuda")
    bad[1, 2, 3] = True
    assert torch.equal(torch.isnan(o).all(-1), bad) and torch.equal(torch.isnan(st).all(-1), bad) and torch.equal(torch.isnan(st).any(-1), bad)
    dq, dk, dv = c.backward(o, st)
    assert torch.equal(torch.isnan(dq).all(-1), bad) and torch.equal(torch.isnan(dq).any(-1), bad)
    for g in (dk, dv):
        nan = torch.isnan(g)
        assert bool(nan[1, :, 1].all()) and int(nan.sum()) == lk * d
    c = Case(53, dtype, 1, lq, lk, 2, 2, d)
    ref = c.reference()
    c.k[0, 0, 1] = math.nan
    o, st = c.forward()
    assert bool(torch.isnan(o[:, :, 1]).all()) and bool(torch.isnan(st[:, :, 1, 1]).all()) and not bool(torch.isnan(o[:, :, 0]).any())
    z, ez = ref.z[0, 1, :, 1:], ref.ez[0, 1, :, 1:]
    assert bool(((st[0, :, 1, 0] - z.amax(-1)).abs() <= ez.amax(-1) + 4 * R.F * (z.abs().amax(-1) + 1)).all())

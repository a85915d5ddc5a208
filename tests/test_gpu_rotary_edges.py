"""Rotary positions at the ends of what the header allows: values that are not rotated,
16 bytes a lane at odd addresses and strides."""
import math

import pytest
import torch

from tests import block_reference as R
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

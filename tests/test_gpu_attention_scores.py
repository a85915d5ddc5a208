"""Cross attention where scores, their sums and statistics are at the ends of their ranges."""
import math

import pytest
import torch

from tests import block_reference as R
from tests.test_gpu_cross_attention import BF, F32, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("far", [1e6, 1e30])
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

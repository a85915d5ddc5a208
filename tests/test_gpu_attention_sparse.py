"""Cross attention whose mask leaves few of many keys: the backward pass goes through
those alone."""
import pytest
import torch

import paper_2210_08650_amd as H
from tests import block_reference as R
from tests.test_gpu_cross_attention import BF, CODE, F32, Case

pytestmark = pytest.mark.gpu


def _keep(c, each):
    """Leaves each[b] keys of entry b, anywhere, the first and the last among them."""
    c.mask[:] = False
    g = torch.Generator()
    g.manual_seed(71)
    for b, n in enumerate(each):
        at = 1 + torch.randperm(c.kv_len - 2, generator=g)[:n]
        if n > 1:
            at[0], at[1] = 0, c.kv_len - 1
        c.mask[b, at.cuda()] = True


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lq,lk,h,kv,d", [(5, 3000, 4, 2, 128), (70, 1100, 2, 1, 64), (300, 700, 3, 3, 96), (1, 9000, 6, 2, 80), (40, 2000, 1, 1, 32),
                                          (150, 400, 2, 2, 128), (33, 1000, 2, 1, 33)])
def test_few_keys_left(lq, lk, h, kv, d, dtype):
    """One key, as many as a tile and one more, 127, 128 and 129 of them (129 are no longer
    few), none, and a length behind which more are left."""
    c = Case(72, dtype, 8, lq, lk, h, kv, d, mask=0.0, kv_lens=[lk] * 7 + [lk // 2])
    _keep(c, [1, 2, 0, 33, 65, 128, 129, 150])
    c.k[~c.mask] = float("nan")
    c.v[~c.mask] = float("inf")
    c.check()
    c.mask[0] = False
    c.mask[0, lk - 2] = True
    c.k[0, lk - 2], c.v[0, lk - 2] = 1.0, 1.0
    o, st = c.forward()
    dq, dk, _ = c.backward(o, st)
    assert not bool(dq[0].any()) and not bool(dk[0].any())  # of one key


@pytest.mark.parametrize("dtype", [BF, F32])
def test_few_keys_left_of_strided_ones(dtype):
    """Keys and values with strides of their own, and past what 32-bit offsets reach, where
    every tile is walked through."""
    c = Case(73, dtype, 2, 20, 1500, 4, 2, 64, mask=0.0, pad=8)
    _keep(c, [100, 3])
    c.check()
    c = Case(74, dtype, 2, 20, 1500, 4, 2, 64, mask=0.0, transposed=True)
    _keep(c, [100, 3])
    c.check()
    # 2300 keys 2^19 elements apart: 2.4 GB of 16 bits, 4.8 of 32
    c = Case(75, dtype, 1, 70, 2300, 2, 1, 64, mask=0.0)
    _keep(c, [90])
    o, st = c.forward()
    wide = [torch.zeros(2300 << 19, dtype=dtype, device="cuda") for _ in range(2)]
    tensors = [w.as_strided((1, 2300, 1, 64), (2300 << 19, 1 << 19, 64, 1)) for w in wide]
    for t, x in zip(tensors, (c.k, c.v)):
        t.copy_(x)
    c.k, c.v = tensors
    d = H.Attention(CODE[dtype], 1, 70, 2300, 2, 1, 64, k_stride=c.k.stride()[:3], v_stride=c.v.stride()[:3], stream=torch.cuda.current_stream())
    ws = torch.empty(max(1, H.hapi_cross_attention_workspace_bytes(d, True)), dtype=torch.uint8, device="cuda")
    d.set(workspace=ws, workspace_bytes=ws.numel())
    out = [torch.zeros(2300 << 19, dtype=dtype, device="cuda").as_strided(t.shape, t.stride()) for t in tensors]
    dq = torch.empty_like(c.q)
    H.hapi_cross_attention_backward(d, c.q, c.k, c.v, None, None, c.mask, o, st, c.dout, dq, *out)
    for name, got, w in zip(("dq", "dk", "dv"), [dq] + out, c.reference().backward(o, st, c.dout)):
        R.check(name, got, w)

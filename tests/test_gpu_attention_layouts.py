"""Cross attention of tensors at addresses, widths and strides that are no whole 16 bytes."""
import pytest
import torch

import paper_2210_08650_amd as H
from tests.test_gpu_cross_attention import BF, F32, Case

pytestmark = pytest.mark.gpu


def _moved(x):
    """The same values from one element past an aligned address, with strides as they are."""
    flat = torch.empty(x.numel() + 1, dtype=x.dtype, device="cuda")
    y = flat[1:].as_strided(x.shape, x.stride())
    y.copy_(x)
    return y


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("b,lq,lk,h,kv,d", [(1, 20, 50, 2, 1, 64), (2, 300, 77, 4, 2, 64), (2, 40, 300, 3, 3, 128), (3, 5, 900, 8, 2, 96),
                                            (200, 3, 70, 1, 1, 32)])
def test_outputs_and_o_at_any_element(b, lq, lk, h, kv, d, dtype):
    """The backward pass reads o where the forward pass was let write it, and its gradients
    may lie as loosely: the same bits as at aligned addresses."""
    c = Case(61, dtype, b, lq, lk, h, kv, d)
    o, st = c.forward()
    want = c.backward(o, st)
    d = c.desc(True)
    far = _moved(torch.zeros_like(o))
    H.hapi_cross_attention_forward(d, c.q, c.k, c.v, None, None, None, far, st.clone())
    assert far.data_ptr() % 16 == far.element_size() and torch.equal(far, o)
    got = [_moved(torch.zeros_like(x)) for x in (c.q, c.k, c.v)]
    H.hapi_cross_attention_backward(d, c.q, c.k, c.v, None, None, None, far, st, c.dout, *got)
    torch.cuda.synchronize()
    c.ws.check()
    assert all(torch.equal(a, w) for a, w in zip(got, want))

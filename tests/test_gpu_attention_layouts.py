"""Cross attention of tensors at addresses, widths and strides that are no whole 16 bytes."""
import pytest
import torch

import paper_2210_08650_amd as H
from tests.test_gpu_cross_attention import BF, CODE, F32, Case

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


@pytest.mark.parametrize("dtype", [BF, F32])
def test_strides_of_one_entry(dtype):
    """Odd and huge strides where there is one entry, one token or one head: read and written
    as without them, by the same kernels."""
    for b, lq, lk, h, kv in ((1, 40, 300, 4, 2), (3, 1, 1, 2, 1), (2, 70, 90, 1, 1), (1, 1, 700, 1, 1)):
        c = Case(62, dtype, b, lq, lk, h, kv, 64)
        o, st = c.forward()
        want = [o, st] + c.backward(o, st)

        def odd(x):
            s = [77 + (1 << 22) * i if n == 1 else w for i, (n, w) in enumerate(zip(x.shape[:3], x.stride()))]
            return x.as_strided(x.shape, (*s, 1))
        c.q, c.k, c.v, c.dout = (odd(x) for x in (c.q, c.k, c.v, c.dout))
        st_of = lambda x: x.stride()[:3]
        d = H.Attention(CODE[dtype], b, lq, lk, h, kv, 64, 0.0, st_of(c.q), st_of(c.k), st_of(c.v), st_of(c.dout), stream=torch.cuda.current_stream())
        ws = torch.empty(max(1, H.hapi_cross_attention_workspace_bytes(d, True)), dtype=torch.uint8, device="cuda")
        d.set(workspace=ws, workspace_bytes=ws.numel())
        got = [odd(torch.empty(x.shape, dtype=dtype, device="cuda")) for x in (c.q, c.q, c.k, c.v)]
        st = torch.empty_like(want[1])
        H.hapi_cross_attention_forward(d, c.q, c.k, c.v, None, None, None, got[0], st)
        H.hapi_cross_attention_backward(d, c.q, c.k, c.v, None, None, None, got[0], st, c.dout, *got[1:])
        assert all(torch.equal(a, w) for a, w in zip([got[0], st] + got[1:], want))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("dim", [2, 6, 30, 34, 50, 62, 86, 98, 126])
def test_even_widths(dim, dtype):
    """Widths of 2 modulo 4, whose rows allow two values at once, dense and with such strides;
    and whole widths with strides of 2 modulo 4."""
    Case(63, dtype, 2, 45, 77, 4, 2, dim).check()
    Case(64, dtype, 2, 150, 70, 2, 2, dim, pad=4, mask=0.7).check()
    Case(65, dtype, 3, 1, 600, 4, 1, dim, pad=2).check()
    Case(66, dtype, 1, 200, 130, 2, 1, dim + 2, pad=2, transposed=True, q_lens=[150], kv_lens=[111]).check()

"""Limits of the cross attention's arguments (no GPU needed)."""
import pytest

import paper_2210_08650_amd as H
from tests.test_block_abi import AB, F32, P, _attend, _raises


@pytest.mark.parametrize("dtype,size", [(H.HAPI_BF16, 2), (F32, 4)])
def test_backward_takes_the_address_that_the_forward_pass_wrote_to(dtype, size):
    """o needs its elements' alignment in either direction, and so do the gradients that are
    written; dout is read in whole 16 bytes where the rows are."""
    at = lambda i, a: AB[:i] + [a] + AB[i + 1:]
    d = _attend(dtype=dtype).set(workspace_bytes=0)  # the checks of addresses come before the workspace's
    for i in (6, 9, 10, 11):  # o, dq, dk, dv
        _raises(H.HAPI_E_NOMEM, H.hapi_cross_attention_backward, d, *at(i, P + size))
        _raises(H.HAPI_E_INVAL, H.hapi_cross_attention_backward, d, *at(i, P + 1))
    assert "dout must be 16-byte" in _raises(H.HAPI_E_INVAL, H.hapi_cross_attention_backward, d, *at(8, P + size))
    odd = _attend(dtype=dtype, dim=63).set(workspace_bytes=0)
    _raises(H.HAPI_E_NOMEM, H.hapi_cross_attention_backward, odd, *at(8, P + size))


@pytest.mark.parametrize("kw,strides", [
    (dict(batch=1), (7, None, None)), (dict(batch=1, q_len=1, kv_len=1), (3, 5, None)), (dict(heads=1, kv_heads=1), (None, None, 33)),
    (dict(batch=1, q_len=1, kv_len=1), (1, (1 << 21) + 1, None)), (dict(batch=1, heads=1, kv_heads=1, q_len=300, kv_len=300), (9, None, 1 << 35))])
def test_strides_of_one_entry_cost_nothing(kw, strides):
    """The stride of an extent of one says nothing about where values lie."""
    sizes = dict(dict(batch=2, q_len=3, kv_len=5, heads=4, kv_heads=2, dim=64), **kw)
    of = lambda length, heads: tuple(s if s is not None else w for s, w in zip(strides, (length * heads * 64, heads * 64, 64)))
    q, k = of(sizes["q_len"], sizes["heads"]), of(sizes["kv_len"], sizes["kv_heads"])
    for back in (False, True):
        plain = H.hapi_cross_attention_workspace_bytes(_attend(**sizes), back)
        assert H.hapi_cross_attention_workspace_bytes(_attend(q_stride=q, k_stride=k, v_stride=k, o_stride=q, **sizes), back) == plain

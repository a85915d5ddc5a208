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

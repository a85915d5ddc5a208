"""Limits of the rotary positions' arguments (no GPU needed)."""
import pytest

import paper_2210_08650_amd as H
from tests.test_block_abi import P, _raises, _rotary

Q, K, QO, KO, X = P, P + (1 << 30), P + (2 << 30), P + (3 << 30), P + (4 << 30)
OTHER = dict(q_out_stride=(768, 64, 192))  # [batch, heads, tokens, head_dim]: the heads' places differ


def _forward(d, q, k, q_out, k_out):
    return _raises(H.HAPI_E_INVAL, H.hapi_rotary_forward, d, q, k, X, X, X, X, None, q_out, k_out)


def _backward(d, dq_out, dk_out, q, k, dq, dk):
    return _raises(H.HAPI_E_INVAL, H.hapi_rotary_backward, d, dq_out, dk_out, q, k, X, X, X, X, None, dq, dk, X, X)


def test_forward_in_place_is_each_tensor_in_its_own():
    """Blocks of q and of k run at once: a result that is written where the other is read is
    either's."""
    assert "q_out must not be k" in _forward(_rotary(kv_heads=4), Q, K, K, KO)
    assert "k_out must not be q" in _forward(_rotary(kv_heads=4), Q, K, QO, Q)
    assert "q_out must not be k" in _forward(_rotary(kv_heads=4), Q, K, K, Q)
    assert "the same" in _forward(_rotary(kv_heads=4), Q, K, QO, QO)
    assert "only where" in _forward(_rotary(**OTHER), Q, K, Q, KO)
    assert "only where" in _forward(_rotary(k_out_stride=(384, 64, 192)), Q, K, QO, K)


def test_backward_in_place_is_each_tensor_in_its_own():
    d = lambda **kw: _rotary(kv_heads=4, **kw)
    assert "dq must not be dk_out" in _backward(d(), QO, KO, Q, K, KO, X)
    assert "dk must not be dq_out" in _backward(d(), QO, KO, Q, K, X, QO)
    assert "the same" in _backward(d(), QO, KO, Q, K, X, X)
    assert "dq must not be k" in _backward(d(), QO, KO, Q, K, K, X)
    assert "dk must not be q" in _backward(d(), QO, KO, Q, K, X, Q)
    assert "only where" in _backward(d(**OTHER), QO, KO, Q, K, QO, X)


def test_what_may_be_in_place_gets_past_these_checks():
    """As far as the workspace's check, which comes before them, or the stream's behind them."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("the calls would run")
    for fn, args in ((H.hapi_rotary_forward, (Q, K, X, X, X, X, None, Q, K)), (H.hapi_rotary_backward, (QO, KO, Q, K, X, X, X, X, None, QO, KO, X, X)),
                     (H.hapi_rotary_forward, (Q, Q, X, X, X, X, None, QO, KO))):
        _raises(H.HAPI_E_DEVICE, fn, _rotary(), *args)
    # extents of one have no strides
    _raises(H.HAPI_E_DEVICE, H.hapi_rotary_forward, _rotary(batch=1, q_out_stride=(5, 256, 64)), Q, K, X, X, X, X, None, Q, KO)

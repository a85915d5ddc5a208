"""Host-side checks of the trained tail's entry points (no GPU needed): every
refusal happens before any device access, and the workspace sizes."""
import ctypes

import pytest
import torch

import paper_2210_08650_amd as H

BF, F32 = H.HAPI_BF16, H.HAPI_F32
P = 1 << 40  # an aligned address that is never used: the calls below fail first


def _raises(code, fn, *a):
    with pytest.raises(H.HapiError) as e:
        fn(*a)
    assert e.value.code == code, str(e.value)
    return str(e.value)


def _norm(rows=4, dim=64, dtype=BF, **kw):
    d = H.Norm(dtype, rows, dim, **kw)
    return d.set(workspace=P, workspace_bytes=1 << 40)


def _head(rows=4, dim=64, classes=10, dtype=BF, **kw):
    d = H.Head(dtype, rows, dim, classes, **kw)
    return d.set(workspace=P, workspace_bytes=1 << 40)


def test_structs_match_the_header():
    assert ctypes.sizeof(H.hapi_norm_desc) == 4 * 2 + 8 * 3 + 4 * 2 + 8 * 3
    assert ctypes.sizeof(H.hapi_head_desc) == 4 * 2 + 8 * 4 + 4 * 2 + 8 * 3


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=7), H.HAPI_E_INVAL), (dict(rows=-1), H.HAPI_E_INVAL), (dict(dim=0), H.HAPI_E_INVAL),
    (dict(dim=16385), H.HAPI_E_UNSUPPORTED), (dict(x_stride=63), H.HAPI_E_INVAL), (dict(y_stride=-1), H.HAPI_E_INVAL),
    (dict(eps=-1e-6), H.HAPI_E_INVAL), (dict(eps=float("nan")), H.HAPI_E_INVAL), (dict(eps=float("inf")), H.HAPI_E_INVAL),
    (dict(rows=1 << 50, x_stride=1 << 20), H.HAPI_E_UNSUPPORTED)])
def test_norm_descriptor_refusals(kw, code):
    d = _norm(**kw)
    _raises(code, H.hapi_layernorm_workspace_bytes, d)
    _raises(code, H.hapi_layernorm_forward, d, P, P, P, P, P, P)
    _raises(code, H.hapi_layernorm_backward, d, P, P, P, P, P, P, P, P)


def test_norm_reserved_field():
    d = _norm()
    d.c.reserved = 1
    _raises(H.HAPI_E_INVAL, H.hapi_layernorm_workspace_bytes, d)


def test_norm_pointer_refusals():
    for i in range(6):
        a = [P] * 6
        a[i] = None
        _raises(H.HAPI_E_INVAL, H.hapi_layernorm_forward, _norm(), *a)
        a[i] = P + 1
        assert "aligned" in _raises(H.HAPI_E_INVAL, H.hapi_layernorm_forward, _norm(), *a)
    for i in range(8):
        a = [P] * 8
        a[i] = None
        _raises(H.HAPI_E_INVAL, H.hapi_layernorm_backward, _norm(), *a)
        a[i] = P + 1
        _raises(H.HAPI_E_INVAL, H.hapi_layernorm_backward, _norm(), *a)
    d = _norm()
    need = H.hapi_layernorm_workspace_bytes(d)
    _raises(H.HAPI_E_NOMEM, H.hapi_layernorm_backward, d.set(workspace_bytes=need - 1), *[P] * 8)
    _raises(H.HAPI_E_INVAL, H.hapi_layernorm_backward, _norm().set(workspace=P + 16), *[P] * 8)
    _raises(H.HAPI_E_NOMEM, H.hapi_layernorm_backward, H.Norm(BF, 4, 64), *[P] * 8)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), H.HAPI_E_INVAL), (dict(rows=-1), H.HAPI_E_INVAL), (dict(dim=0), H.HAPI_E_INVAL),
    (dict(classes=0), H.HAPI_E_INVAL), (dict(top=-1), H.HAPI_E_INVAL), (dict(top=1025), H.HAPI_E_UNSUPPORTED),
    (dict(top=1, temperature=0.0), H.HAPI_E_INVAL), (dict(top=1, temperature=float("nan")), H.HAPI_E_INVAL),
    (dict(top=1, temperature=float("inf")), H.HAPI_E_INVAL), (dict(top=1, temperature=1e-39), H.HAPI_E_INVAL),
    (dict(temperature=2.0), H.HAPI_E_INVAL), (dict(x_stride=63), H.HAPI_E_INVAL), (dict(w_stride=-8), H.HAPI_E_INVAL),
    (dict(rows=(1 << 20) + 1), H.HAPI_E_UNSUPPORTED), (dict(classes=(1 << 24) + 1), H.HAPI_E_UNSUPPORTED),
    (dict(x_stride=(1 << 20) + 8), H.HAPI_E_UNSUPPORTED), (dict(dim=(1 << 20) + 8), H.HAPI_E_UNSUPPORTED)])
def test_head_descriptor_refusals(kw, code):
    d = _head(**kw)
    _raises(code, H.hapi_head_workspace_bytes, d, True)
    _raises(code, H.hapi_xent_forward, d, P, P, P, P, P, P)
    _raises(code, H.hapi_xent_backward, d, P, P, P, P, P, P, P, P, P, P)
    _raises(code, H.hapi_distill_forward, d, P, P, P, P, P, P, P, P)
    _raises(code, H.hapi_distill_backward, d, P, P, P, P, P, P, P, P, P, P, P)


def test_head_calls_match_their_descriptor():
    assert "top = 0" in _raises(H.HAPI_E_INVAL, H.hapi_xent_forward, _head(top=2), *[P] * 6)
    _raises(H.HAPI_E_INVAL, H.hapi_xent_backward, _head(top=2), *[P] * 10)
    assert "top >= 1" in _raises(H.HAPI_E_INVAL, H.hapi_distill_forward, _head(), *[P] * 8)
    _raises(H.HAPI_E_INVAL, H.hapi_distill_backward, _head(), *[P] * 11)


@pytest.mark.parametrize("call,n,top,optional", [
    ("hapi_xent_forward", 6, 0, (2,)), ("hapi_xent_backward", 10, 0, (2, 9)),
    ("hapi_distill_forward", 8, 3, (2,)), ("hapi_distill_backward", 11, 3, (2, 10))])
def test_head_pointer_refusals(call, n, top, optional):
    fn = getattr(H, call)
    for i in range(n):
        a = [P] * n
        if i not in optional:
            a[i] = None
            _raises(H.HAPI_E_INVAL, fn, _head(top=top), *a)
        a[i] = P + 1
        assert "aligned" in _raises(H.HAPI_E_INVAL, fn, _head(top=top), *a)
    for i in (0, 1):  # whole 16-byte rows are read as they lie
        a = [P] * n
        a[i] = P + 8
        _raises(H.HAPI_E_INVAL, fn, _head(top=top), *a)
    if n > 8:
        a = [P] * n
        a[2] = None
        assert "without a bias" in _raises(H.HAPI_E_INVAL, fn, _head(top=top), *a)
    d = _head(top=top)
    need = H.hapi_head_workspace_bytes(d, n > 8)
    _raises(H.HAPI_E_NOMEM, fn, d.set(workspace_bytes=need - 1), *[P] * n)
    _raises(H.HAPI_E_INVAL, fn, _head(top=top).set(workspace=P + 128), *[P] * n)


def test_tensor_arguments_must_fit_the_descriptor():
    d = _head()
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    assert "float32" in _raises(H.HAPI_E_INVAL, H.hapi_xent_forward, d, x.float(), P, P, P, P, P)
    assert "(4, 64)" in _raises(H.HAPI_E_INVAL, H.hapi_xent_forward, d, x[:3], P, P, P, P, P)
    assert "strides" in _raises(H.HAPI_E_INVAL, H.hapi_xent_forward, d,
                                torch.zeros(64, 4, dtype=torch.bfloat16).t(), P, P, P, P, P)
    assert "not on the current GPU" in _raises(H.HAPI_E_INVAL, H.hapi_xent_forward, d, x, P, P, P, P, P)
    assert "int64" in _raises(H.HAPI_E_INVAL, H.hapi_xent_forward, d, P, P, P, torch.zeros(4, dtype=torch.int32), P, P)
    _raises(H.HAPI_E_INVAL, H.hapi_layernorm_forward, _norm(), x, torch.zeros(63), P, P, P, P)


def test_workspace_sizes():
    w = H.hapi_head_workspace_bytes
    small, large = _head(rows=128, dim=768, classes=1000), _head(rows=8192, dim=2048, classes=131072)
    assert 0 < w(small, False) <= w(small, True)
    # far below the logits: 2 GB of them in 16 bits, one piece of dz^T and the
    # partial sums of dx in its place
    assert w(large, True) < 8192 * 131072 * 2 // 2
    assert w(large, False) < 8192 * 131072 * 2 // 8
    # odd widths cost padded copies of x and the weights
    odd, even = _head(rows=128, dim=777, classes=1000), _head(rows=128, dim=784, classes=1000)
    assert w(odd, False) >= w(even, False) + (1000 + 128) * 784 * 2
    assert H.hapi_layernorm_workspace_bytes(_norm(dim=768)) >= 2 * 768 * 4
    assert w(_head(rows=0), True) >= 0

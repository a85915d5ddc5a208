"""Host-side checks of the trained block's entry points (no GPU needed): every refusal
happens before any device access, and the workspace sizes."""
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


def _ready(d):
    return d.set(workspace=P, workspace_bytes=1 << 40)


# ----------------------------------------------------------------- gradients

class _At:
    """A tensor's stand-in at an address."""

    def __init__(self, address, n, dtype=torch.float32):
        self.address, self.n, self.dtype = address, n, dtype
        self.shape = (n,)

    def data_ptr(self):
        return self.address

    def numel(self):
        return self.n

    def stride(self):
        return (1,)

    def is_contiguous(self):
        return True

    def get_device(self):
        return None  # as the current device is without a GPU


@pytest.fixture
def _no_gpu(monkeypatch):
    from paper_2210_08650_amd import binding
    monkeypatch.setattr(binding, "_device", lambda: None)


def _grads(sizes=(8, 3), out=None, dtypes=None, max_norm=1.0, step=1 << 20):
    dt = dtypes or [torch.float32] * len(sizes)
    make = lambda base: [_At(base + i * step, n, t) for i, (n, t) in enumerate(zip(sizes, dt))]
    return _ready(H.Gradients(make(P), max_norm=max_norm, out=None if out is None else make(out)))


def test_structs_match_the_header():
    assert ctypes.sizeof(H.hapi_gradient_desc) == 8 + 8 * 4 + 8 + 8 * 3
    assert ctypes.sizeof(H.hapi_rotary_desc) == 4 * 13 + 4 + 8 * 2 + 8 * 12 + 8 * 3


def test_gradient_refusals(_no_gpu):
    calls = (H.hapi_gradient_norm, H.hapi_gradient_clip)
    for fn in calls:
        for m in (0.0, -1.0, float("nan"), float("inf")):
            _raises(H.HAPI_E_INVAL, fn, _grads(max_norm=m), P)
        _raises(H.HAPI_E_INVAL, fn, _grads(), None)
        _raises(H.HAPI_E_INVAL, fn, _grads(), P + 2)
        d = _grads()
        d.c.reserved = 1
        _raises(H.HAPI_E_INVAL, fn, d, P)
        d = _grads()
        d.c.count = -1
        _raises(H.HAPI_E_INVAL, fn, d, P)
        d.c.count = (1 << 20) + 1
        _raises(H.HAPI_E_UNSUPPORTED, fn, d, P)
        for i, v, code in ((0, -1, H.HAPI_E_INVAL), (1, (1 << 38) + 1, H.HAPI_E_UNSUPPORTED)):
            d = _grads()
            d._sizes[i] = v
            _raises(code, fn, d, P)
        d = _grads()
        d._dtypes[1] = 5
        _raises(H.HAPI_E_INVAL, fn, d, P)
        for a in (None, P + 2):
            d = _grads()
            d._grads[1] = a
            _raises(H.HAPI_E_INVAL, fn, d, P)
        d = _grads(dtypes=[torch.bfloat16] * 2)
        d._grads[0] = P + 1
        assert "2-byte" in _raises(H.HAPI_E_INVAL, fn, d, P)
        for field in ("grads", "sizes", "dtypes"):
            d = _grads()
            setattr(d.c, field, None)
            _raises(H.HAPI_E_INVAL, fn, d, P)
        d = _grads()
        need = H.hapi_gradient_workspace_bytes(d)
        _raises(H.HAPI_E_NOMEM, fn, d.set(workspace_bytes=need - 1), P)
        _raises(H.HAPI_E_INVAL, fn, _grads().set(workspace=P + 16), P)
    d = _grads(out=1 << 41)
    d._out[0] = None
    _raises(H.HAPI_E_INVAL, H.hapi_gradient_clip, d, P)


def test_gradients_that_overlap(_no_gpu):
    twice = lambda d: _raises(H.HAPI_E_INVAL, H.hapi_gradient_clip, d, P)
    d = _grads()
    d._grads[1] = d._grads[0]
    assert "overlap" in twice(d)
    d = _grads()
    d._grads[1] = d._grads[0] - 8  # 3 values from 8 bytes before
    assert "overlap" in twice(d)
    d = _grads(out=1 << 41)
    d._out[1] = d._grads[0]
    assert "grads[0]" in twice(d)
    d = _grads(out=1 << 41)
    d._out[0] = d._grads[0] + 16
    assert "overlaps" in twice(d)
    d = _grads((8, 8, 8), out=1 << 41)  # a wide output before the tensor that is read
    d._out[2] = d._grads[1] - 28
    assert "grads[1]" in twice(d)


def test_gradient_tensors_are_looked_over():
    t = torch.zeros(4, 6)
    _raises(H.HAPI_E_INVAL, H.Gradients, [t.double()])
    assert "consecutive" in _raises(H.HAPI_E_INVAL, H.Gradients, [t[:, :3]])
    assert "consecutive" in _raises(H.HAPI_E_INVAL, H.Gradients, [t[:1].expand(3, 6)])
    H.Gradients([t.t(), t[:, :0], t[0, 0]])
    with pytest.raises(H.HapiError):
        H.Gradients([t], out=[])
    with pytest.raises(H.HapiError):
        H.Gradients([t], out=[t.t().contiguous().t()])
    with pytest.raises(H.HapiError):
        H.Gradients([t], out=[t.bfloat16()])
    assert "current GPU" in _raises(H.HAPI_E_INVAL, H.hapi_gradient_norm, _ready(H.Gradients([t])), P)


# -------------------------------------------------------------------- rotary

def _rotary(batch=2, length=3, heads=4, kv_heads=2, dim=64, sections=(16, 16), dtype=BF, **kw):
    return _ready(H.Rotary(dtype, batch, length, heads, kv_heads, dim, sections, **kw))


FWD, BWD = [P] * 6 + [None] + [P] * 2, [P] * 8 + [None] + [P] * 4


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=3), H.HAPI_E_INVAL), (dict(dim=0), H.HAPI_E_INVAL), (dict(dim=257, sections=()), H.HAPI_E_UNSUPPORTED),
    (dict(heads=-1), H.HAPI_E_INVAL), (dict(heads=0, kv_heads=0), H.HAPI_E_INVAL), (dict(batch=-1), H.HAPI_E_INVAL),
    (dict(length=-1), H.HAPI_E_INVAL), (dict(sections=(0,)), H.HAPI_E_INVAL), (dict(sections=(16, -1)), H.HAPI_E_INVAL),
    (dict(sections=(16, 17)), H.HAPI_E_INVAL), (dict(sections=(1 << 30, 1 << 30)), H.HAPI_E_INVAL), (dict(eps=-1.0), H.HAPI_E_INVAL),
    (dict(eps=float("nan")), H.HAPI_E_INVAL), (dict(batch=1 << 16, length=1 << 14), H.HAPI_E_UNSUPPORTED),
    (dict(batch=1 << 40), H.HAPI_E_UNSUPPORTED), (dict(heads=1 << 21), H.HAPI_E_UNSUPPORTED),
    (dict(q_stride=(1, -1, 1)), H.HAPI_E_INVAL), (dict(k_out_stride=(1, 1 << 41, 1)), H.HAPI_E_UNSUPPORTED)])
def test_rotary_descriptor_refusals(kw, code):
    d = _rotary(**kw)
    _raises(code, H.hapi_rotary_workspace_bytes, d)
    _raises(code, H.hapi_rotary_forward, d, *FWD)
    _raises(code, H.hapi_rotary_backward, d, *BWD)


def test_rotary_flags():
    for field in ("neighbours", "norm", "reserved"):
        d = _rotary()
        setattr(d.c, field, 2)
        _raises(H.HAPI_E_INVAL, H.hapi_rotary_workspace_bytes, d)
    d = _rotary()
    d.c.axes = 5
    _raises(H.HAPI_E_INVAL, H.hapi_rotary_workspace_bytes, d)
    d.c.axes = 1  # and two sections
    _raises(H.HAPI_E_INVAL, H.hapi_rotary_workspace_bytes, d)
    with pytest.raises(H.HapiError):
        H.Rotary(BF, 1, 1, 1, 1, 64, (1,) * 5)


def test_rotary_pointer_refusals():
    for fn, args in ((H.hapi_rotary_forward, FWD), (H.hapi_rotary_backward, BWD)):
        for i in range(len(args)):
            for bad in (None, P + 1):
                a = list(args)
                a[i] = bad
                if args[i] is not None or bad is not None:
                    _raises(H.HAPI_E_INVAL, fn, _rotary(), *a)
    # what is not used is not given
    assert "without heads" in _raises(H.HAPI_E_INVAL, H.hapi_rotary_forward, _rotary(heads=0, norm=False), P, P, None, None, P, P, None, P, P)
    assert "not used" in _raises(H.HAPI_E_INVAL, H.hapi_rotary_forward, _rotary(norm=False), *FWD)
    d = _rotary()
    need = H.hapi_rotary_workspace_bytes(d)
    assert need > 0 and H.hapi_rotary_workspace_bytes(_rotary(norm=False)) == 0
    _raises(H.HAPI_E_NOMEM, H.hapi_rotary_backward, d.set(workspace_bytes=need - 1), *BWD)
    _raises(H.HAPI_E_INVAL, H.hapi_rotary_backward, _rotary().set(workspace=P + 16), *BWD)


@pytest.mark.parametrize("stride", [(0, 256, 64), (768, 256, 63), (700, 256, 64), (768, 64, 64), (128, 256, 64)])
def test_rotary_outputs_must_not_overlap(stride):
    assert "overlap" in _raises(H.HAPI_E_INVAL, H.hapi_rotary_forward, _rotary(q_out_stride=stride), *FWD)
    assert "overlap" in _raises(H.HAPI_E_INVAL, H.hapi_rotary_backward, _rotary(q_stride=stride), *BWD)


def test_rotary_tensors_must_fit_the_descriptor():
    d = _rotary()
    q = torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16)
    a = lambda x: [x] + FWD[1:]
    assert "bfloat16" in _raises(H.HAPI_E_INVAL, H.hapi_rotary_forward, d, *a(q.float()))
    assert "(2, 3, 4, 64)" in _raises(H.HAPI_E_INVAL, H.hapi_rotary_forward, d, *a(q[:, :2]))
    assert "strides" in _raises(H.HAPI_E_INVAL, H.hapi_rotary_forward, d, *a(torch.zeros(2, 4, 3, 64, dtype=torch.bfloat16).transpose(1, 2)))
    assert "current GPU" in _raises(H.HAPI_E_INVAL, H.hapi_rotary_forward, d, *a(q))
    pos = torch.zeros(2, 2, 6, dtype=torch.int64)[:, :, :3]
    assert "contiguous" in _raises(H.HAPI_E_INVAL, H.hapi_rotary_forward, d, P, P, P, P, pos, P, None, P, P)
    assert "float64" in _raises(H.HAPI_E_INVAL, H.hapi_rotary_forward, d, P, P, P, P, P, torch.zeros(32), None, P, P)


# ----------------------------------------------------------- cross attention

def _attend(batch=2, q_len=3, kv_len=5, heads=4, kv_heads=2, dim=64, dtype=BF, **kw):
    return _ready(H.Attention(dtype, batch, q_len, kv_len, heads, kv_heads, dim, **kw))


AF, AB = [P] * 3 + [None] * 3 + [P] * 2, [P] * 3 + [None] * 3 + [P] * 6


def test_attention_struct_matches_the_header():
    assert ctypes.sizeof(H.hapi_attention_desc) == 4 * 4 + 8 * 3 + 8 * 12 + 8 + 8 * 3


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), H.HAPI_E_INVAL), (dict(dim=0), H.HAPI_E_INVAL), (dict(dim=129), H.HAPI_E_UNSUPPORTED), (dict(heads=0), H.HAPI_E_INVAL),
    (dict(kv_heads=0), H.HAPI_E_INVAL), (dict(heads=5), H.HAPI_E_INVAL), (dict(heads=513, kv_heads=1), H.HAPI_E_UNSUPPORTED),
    (dict(batch=-1), H.HAPI_E_INVAL), (dict(q_len=-1), H.HAPI_E_INVAL), (dict(kv_len=-1), H.HAPI_E_INVAL), (dict(scale=-1.0), H.HAPI_E_INVAL),
    (dict(scale=float("nan")), H.HAPI_E_INVAL), (dict(scale=float("inf")), H.HAPI_E_INVAL), (dict(scale=3e38), H.HAPI_E_INVAL),
    (dict(batch=0, heads=1 << 30, kv_heads=1 << 30), H.HAPI_E_UNSUPPORTED), (dict(q_len=1 << 31), H.HAPI_E_UNSUPPORTED),
    (dict(kv_len=1 << 31), H.HAPI_E_UNSUPPORTED), (dict(batch=1 << 23), H.HAPI_E_UNSUPPORTED), (dict(batch=1 << 14, kv_len=1 << 20), H.HAPI_E_UNSUPPORTED),
    (dict(q_stride=(1, 2, -3)), H.HAPI_E_INVAL), (dict(v_stride=(1 << 41, 1, 1)), H.HAPI_E_UNSUPPORTED)])
def test_attention_descriptor_refusals(kw, code):
    d = _attend(**kw)
    _raises(code, H.hapi_cross_attention_workspace_bytes, d, True)
    _raises(code, H.hapi_cross_attention_forward, d, *AF)
    _raises(code, H.hapi_cross_attention_backward, d, *AB)


def test_attention_launches_of_32_bit_thread_counts():
    """128 keys of bf16 heads past 96 values are 512 threads of the backward pass."""
    for dtype, dim, most in ((BF, 97, 23), (BF, 96, 24), (F32, 128, 24)):
        kw = dict(dtype=dtype, dim=dim, q_len=1, heads=1, kv_heads=1, kv_len=1)
        _raises(H.HAPI_E_UNSUPPORTED, H.hapi_cross_attention_workspace_bytes, _attend(batch=1 << most, **kw), True)
        assert H.hapi_cross_attention_workspace_bytes(_attend(batch=(1 << most) - 1, **kw), True) >= 0


def test_attention_pointer_refusals():
    d = _attend()
    d.c.reserved = 1
    _raises(H.HAPI_E_INVAL, H.hapi_cross_attention_forward, d, *AF)
    for fn, args in ((H.hapi_cross_attention_forward, AF), (H.hapi_cross_attention_backward, AB)):
        for i, x in enumerate(args):
            for bad in (None, P + 1):
                if (x is None and bad is None) or i == 5:  # a mask is bytes, of any address
                    continue
                a = list(args)
                a[i] = bad
                _raises(H.HAPI_E_INVAL, fn, _attend(), *a)
        for i in range(3):  # whole 16-byte rows are read as they lie
            a = list(args)
            a[i] = P + 8
            assert "16-byte" in _raises(H.HAPI_E_INVAL, fn, _attend(), *a)
        need = H.hapi_cross_attention_workspace_bytes(_attend(q_len=100), True)
        assert need >= 2 * 4 * 100 * 4
        _raises(H.HAPI_E_NOMEM, fn, _attend(kv_len=2000).set(workspace_bytes=64), *args)
        _raises(H.HAPI_E_INVAL, fn, _attend().set(workspace=P + 128), *args)


@pytest.mark.parametrize("stride", [(0, 256, 64), (768, 256, 63), (700, 256, 64), (768, 64, 64)])
def test_attention_outputs_must_not_overlap(stride):
    assert "o let" in _raises(H.HAPI_E_INVAL, H.hapi_cross_attention_forward, _attend(o_stride=stride), *AF)
    assert "dq let" in _raises(H.HAPI_E_INVAL, H.hapi_cross_attention_backward, _attend(q_stride=stride), *AB)
    for name in ("k", "v"):
        d = _attend(kv_heads=4, kv_len=3, **{name + "_stride": stride})
        assert f"d{name} let" in _raises(H.HAPI_E_INVAL, H.hapi_cross_attention_backward, d, *AB)


def test_attention_tensors_must_fit_the_descriptor():
    d = _attend()
    q, k = torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 5, 2, 64, dtype=torch.bfloat16)
    call = lambda *a: _raises(H.HAPI_E_INVAL, H.hapi_cross_attention_forward, d, *(list(a) + AF[len(a):]))
    assert "bfloat16" in call(q.float())
    assert "(2, 5, 2, 64)" in call(P, q)
    assert "strides" in call(P, P, k.transpose(0, 1).contiguous().transpose(0, 1))
    assert "int64" in call(P, P, P, torch.zeros(2))
    assert "(2, 5)" in call(P, P, P, None, None, torch.zeros(2, 4, dtype=torch.bool))
    assert "bool" in call(P, P, P, None, None, torch.zeros(2, 5))
    assert "contiguous" in call(P, P, P, None, None, torch.zeros(2, 10, dtype=torch.bool)[:, ::2])
    assert "current GPU" in call(P, k)


def test_attention_workspace():
    w = H.hapi_cross_attention_workspace_bytes
    assert w(_attend(q_len=4096, kv_len=4096, heads=16), False) == 0  # rows enough: nothing is split
    few = _attend(q_len=1, kv_len=8192)
    _raises(H.HAPI_E_NOMEM, H.hapi_cross_attention_forward, few.set(workspace_bytes=w(few, False) - 1), *AF)
    # odd widths cost aligned copies
    assert w(_attend(q_len=300, kv_len=300, dim=63), False) >= 2 * 300 * (4 + 2 + 2) * 64 * 2

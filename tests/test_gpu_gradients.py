"""The gradients' norm and clipping on the GPU against 64 bits; every tensor that is
written, and the workspace, lies between guards."""
import math

import pytest
import torch

import paper_2210_08650_amd as H
from tests import block_reference as R
from tests.hip_harness import Guarded

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _make(seed, sizes, dtypes, scale=0.1):
    g = _gen(seed)
    return [(torch.randn(n, generator=g, device="cuda") * scale).to(t) for n, t in zip(sizes, dtypes)]


def _desc(grads, max_norm=1.0, out=None):
    d = H.Gradients(grads, max_norm=max_norm, out=out, stream=torch.cuda.current_stream())
    ws = Guarded(H.hapi_gradient_workspace_bytes(d))
    d.set(workspace=ws.body, workspace_bytes=ws.nbytes)
    return d, ws


def _norm(grads):
    d, ws = _desc(grads)
    n = Guarded(4)
    H.hapi_gradient_norm(d, n.view(F32, (1,)))
    torch.cuda.synchronize()
    ws.check()
    n.check()
    return float(n.view(F32, (1,)))


def _clip(grads, max_norm, in_place, shift=0):
    """The clipped copies; the originals stay.  shift: values between a guard and a tensor."""
    bufs, outs = [], []
    for g in grads:
        b = Guarded((g.numel() + shift) * g.element_size())
        o = b.body.view(g.dtype)[shift:]
        if in_place:
            o.copy_(g)
        bufs.append(b)
        outs.append(o)
    d, ws = _desc(outs if in_place else grads, max_norm, None if in_place else outs)
    n = Guarded(4)
    H.hapi_gradient_clip(d, n.view(F32, (1,)))
    torch.cuda.synchronize()
    for b in bufs + [ws, n]:
        b.check()
    return float(n.view(F32, (1,))), outs


SETS = [
    ([1], [F32]), ([1], [BF]), ([7], [BF]), ([2048 * 1000, 1000], [F32, F32]),
    ([0, 5, 0, 1], [BF, F32, F32, BF]),
    ([8191, 8192, 8193, 2047, 2049, 3, 32768 * 3 + 1], [BF, F32, BF, F32, BF, BF, F32]),
    ([5_000_011, 17, 3_000_000], [BF, F32, F32]),
    ([i % 37 for i in range(121)], [BF if i % 3 else F32 for i in range(121)]),
    ([1 + i % 301 for i in range(1300)], [BF if i % 2 else F32 for i in range(1300)]),
]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("i", range(len(SETS)))
def test_norm_and_clip(i, in_place):
    sizes, dtypes = SETS[i]
    grads = _make(i, sizes, dtypes)
    true = R.gradient_norm(grads)
    for max_norm in (true / 3, true * 3):
        (n, en), want = R.gradient_clip(grads, max_norm)
        got, outs = _clip(grads, max_norm, in_place, shift=i % 3)
        assert abs(got - n) <= en, (got, n)
        for k, (o, w) in enumerate(zip(outs, want)):
            R.check(f"tensor {k}", o, w)
            if max_norm > n:
                assert torch.equal(o, grads[k])
    assert abs(_norm(grads) - true) <= true * (R.F * 1.001 + 1e-12)


def test_no_tensors():
    assert _norm([]) == 0.0
    assert _clip([], 1.0, True)[0] == 0.0
    assert _clip([torch.empty(0, device="cuda")], 1.0, True)[0] == 0.0


def test_zeros_stay():
    n, outs = _clip([torch.zeros(1000, device="cuda")], 1.0, True)
    assert n == 0.0 and not bool(outs[0].any())


def test_not_finite_changes_nothing():
    for bad in (math.nan, math.inf, -math.inf):
        grads = _make(3, [4000, 100], [F32, BF], 10.0)
        grads[0][1234] = bad
        for in_place in (True, False):
            n, outs = _clip(grads, 1.0, in_place)
            assert not math.isfinite(n)
            for o, g in zip(outs, grads):
                assert torch.equal(o.view(torch.int16 if o.dtype == BF else torch.int32), g.view(torch.int16 if g.dtype == BF else torch.int32))


def test_large_and_small_values():
    """Squares past float32's range at either end."""
    for scale in (1e30, 3e-30):
        grads = _make(4, [70_000, 300], [F32, BF], 1.0)
        grads = [(g.double() * scale).to(g.dtype) for g in grads]
        (n, en), want = R.gradient_clip(grads, scale)
        got, outs = _clip(grads, scale, False)
        assert abs(got - n) <= en
        for o, w in zip(outs, want):
            R.check("clipped", o, w)
    # the norm itself past float32: inf, and the gradients are clipped all the same
    grads = [torch.full((100,), 3e38, device="cuda")]
    n, outs = _clip(grads, 1.0, True)
    assert n == math.inf
    R.check("clipped", outs[0], R.gradient_clip(grads, 1.0)[1][0])


def test_dense_tensors_of_any_order():
    g = torch.randn(30, 40, generator=_gen(5), device="cuda").t()
    d, ws = _desc([g], 1.0)
    n = torch.empty(1, device="cuda")
    want = R.gradient_clip([g], 1.0)[1][0]
    H.hapi_gradient_clip(d, n)
    R.check("clipped", g, want)


def test_the_same_bits_again_and_on_another_stream():
    grads = _make(6, [1_000_003, 5000], [F32, BF])
    first = _clip(grads, 0.5, False)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        second = _clip(grads, 0.5, False)
    s.synchronize()
    assert first[0] == second[0]
    assert all(torch.equal(a, b) for a, b in zip(first[1], second[1]))


def test_captured_and_replayed():
    grads = _make(7, [100_000, 333], [F32, BF])
    work = [g.clone() for g in grads]
    d, ws = _desc(work, 0.5)
    n = torch.empty(1, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        d.set(stream=torch.cuda.current_stream())
        H.hapi_gradient_clip(d, n)
    for k in (1.0, 2.0, 0.5):
        for w, g in zip(work, grads):
            w.copy_(g * k)
        want = _clip([w.clone() for w in work], 0.5, False)
        graph.replay()
        torch.cuda.synchronize()
        assert float(n) == want[0]
        assert all(torch.equal(a, b) for a, b in zip(work, want[1]))
    ws.check()


def test_large_tensor():
    """A tensor of more than 2^31 bytes and a size that is no multiple of anything."""
    g = [torch.full(((1 << 29) + 5,), 0.5, device="cuda")]
    n, outs = _clip(g, 1.0, True)
    want = math.sqrt(g[0].numel()) * 0.5
    assert abs(n - want) <= want * 2 ** -23
    assert bool((outs[0] == outs[0][0]).all()) and abs(float(outs[0][0]) * want / 0.5 - 1.0) < 2 ** -22

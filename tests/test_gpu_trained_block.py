"""The trained block's operators together, as a training step and a decoder behind
extracted features use them."""
import math

import pytest
import torch

import paper_2210_08650_amd as H
from paper_2210_08650_amd import models as PM
from tests import block_reference as R

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _ready(d, need):
    return d.set(workspace=torch.empty(max(need, 256), dtype=torch.uint8, device="cuda"), workspace_bytes=max(need, 256))


def _features(batch):
    """[batch, 197, 768] tokens of a vision transformer's first block, random weights."""
    layers = PM.vit_b16()[:3]
    g = _gen(1)
    d = H.Desc(layers, H.HAPI_BF16, stream=torch.cuda.current_stream())
    raw = torch.randn(H.hapi_raw_weight_count(d), generator=g, device="cuda") * 0.05
    packed = torch.empty(H.hapi_packed_weight_bytes(d), dtype=torch.uint8, device="cuda")
    H.hapi_pack_weights(d, raw, packed)
    need = H.hapi_workspace_bytes(d, batch, 3)
    d.set(workspace=torch.empty(need, dtype=torch.uint8, device="cuda"), workspace_bytes=need)
    images = torch.randn(batch, 3, 224, 224, generator=g, device="cuda").to(BF)
    out = torch.empty((batch,) + H.hapi_layer_shape(d, 3), dtype=BF, device="cuda")
    H.hapi_extract(d, packed, images, batch, 3, out)
    return out


def _grid(batch, tokens, side):
    """The class token at (0, 0), patch t at its row and column, both from 1."""
    t = torch.arange(tokens, device="cuda") - 1
    pos = torch.stack([torch.where(t < 0, 0, t // side + 1), torch.where(t < 0, 0, t % side + 1)])
    return pos[:, None].expand(2, batch, tokens).contiguous()


def _layernorm(x, gamma, beta):
    rows, dim = x.shape
    d = H.Norm(H.HAPI_F32, rows, dim, stream=torch.cuda.current_stream())
    _ready(d, H.hapi_layernorm_workspace_bytes(d))
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    H.hapi_layernorm_forward(d, x, gamma, beta, y, mean, rstd)

    def back(dy):
        dx, dg, db = torch.empty_like(x), torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
        H.hapi_layernorm_backward(d, dy, x, gamma, mean, rstd, dx, dg, db)
        return dx, dg, db
    return y, back


def test_training_step_behind_extracted_features():
    """Layer norm, projections, the heads' norm and rotary positions, cross attention of
    learned queries, layer norm, a classifier's cross entropy; back; clipping.  float32
    against 64 bits by autograd: each of the some 14 operators adds at most (4 sqrt(n) +
    16) 2^-24 of its result's length, 8e-6 for sums of n = 788 terms, 1.1e-4 in all; the
    norms' and the softmax's differences may stretch that tenfold."""
    b, m, heads, kv, d, classes = 4, 6, 6, 3, 64, 50
    feats = _features(b).float()
    n = feats.shape[1]
    g = _gen(2)
    r = lambda *s, k=1.0: torch.randn(s, generator=g, device="cuda") * k
    p = dict(g1=1 + r(768, k=0.1), b1=r(768, k=0.1), wk=r(kv * d, 768, k=768 ** -0.5), wv=r(kv * d, 768, k=768 ** -0.5),
             queries=r(m, heads * d), gq=1 + r(d, k=0.1), gk=1 + r(d, k=0.1), g2=1 + r(heads * d, k=0.1), b2=r(heads * d, k=0.1),
             w=r(classes, heads * d, k=0.1), bias=r(classes, k=0.1))
    targets = torch.randint(0, classes, (b * m,), generator=g, device="cuda")
    targets[3] = -100
    mask = torch.rand(b, n, generator=g, device="cuda") < 0.9
    sections = (16, 16)
    freq = torch.tensor([100.0 ** (-j / 16) for _ in range(2) for j in range(16)], dtype=torch.float64, device="cuda")
    positions = _grid(b, n, 14)
    s = torch.cuda.current_stream()

    # the library's step
    x = feats.reshape(b * n, 768)
    xn, back1 = _layernorm(x, p["g1"], p["b1"])
    k0, v = (xn @ p["wk"].t()).view(b, n, kv, d), (xn @ p["wv"].t()).view(b, n, kv, d)
    q0 = p["queries"].view(1, m, heads, d).expand(b, m, heads, d).contiguous()
    rk = H.Rotary(H.HAPI_F32, b, n, 0, kv, d, sections, stream=s)
    rq = H.Rotary(H.HAPI_F32, b, m, heads, 0, d, (), stream=s)
    _ready(rk, H.hapi_rotary_workspace_bytes(rk))
    _ready(rq, H.hapi_rotary_workspace_bytes(rq))
    k, q = torch.empty_like(k0), torch.empty_like(q0)
    H.hapi_rotary_forward(rk, None, k0, None, p["gk"], positions, freq, None, None, k)
    H.hapi_rotary_forward(rq, q0, None, p["gq"], None, None, None, None, q, None)
    at = H.Attention(H.HAPI_F32, b, m, n, heads, kv, d, stream=s)
    _ready(at, H.hapi_cross_attention_workspace_bytes(at, True))
    o, st = torch.empty_like(q), torch.empty(b, m, heads, 2, device="cuda")
    H.hapi_cross_attention_forward(at, q, k, v, None, None, mask, o, st)
    y, back2 = _layernorm(o.reshape(b * m, heads * d), p["g2"], p["b2"])
    hd = H.Head(H.HAPI_F32, b * m, heads * d, classes, stream=s)
    _ready(hd, H.hapi_head_workspace_bytes(hd, True))
    loss, stats = torch.empty(b * m, device="cuda"), torch.empty(b * m, 2, device="cuda")
    H.hapi_xent_forward(hd, y, p["w"], p["bias"], targets, loss, stats)
    dloss = torch.full((b * m,), 1.0 / (b * m - 1), device="cuda")
    dy, grads = torch.empty_like(y), {"w": torch.empty_like(p["w"]), "bias": torch.empty_like(p["bias"])}
    H.hapi_xent_backward(hd, y, p["w"], p["bias"], targets, loss, stats, dloss, dy, grads["w"], grads["bias"])
    do, grads["g2"], grads["b2"] = back2(dy)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    H.hapi_cross_attention_backward(at, q, k, v, None, None, mask, o, st, do.view(b, m, heads, d), dq, dk, dv)
    dq0, dk0 = torch.empty_like(q), torch.empty_like(k)
    grads["gq"], grads["gk"] = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    H.hapi_rotary_backward(rk, None, dk, None, k0, None, p["gk"], positions, freq, None, None, dk0, None, grads["gk"])
    H.hapi_rotary_backward(rq, dq, None, q0, None, p["gq"], None, None, None, None, dq0, None, grads["gq"], None)
    grads["queries"] = dq0.sum(0).view(m, heads * d)
    dk2, dv2 = dk0.view(b * n, kv * d), dv.view(b * n, kv * d)
    grads["wk"], grads["wv"] = dk2.t() @ xn, dv2.t() @ xn
    _, grads["g1"], grads["b1"] = back1(dk2 @ p["wk"] + dv2 @ p["wv"])
    names = sorted(p)
    want_norm = R.gradient_norm([grads[k_] for k_ in names])
    before = {k_: v_.clone() for k_, v_ in grads.items()}
    gd = H.Gradients([grads[k_] for k_ in names], max_norm=want_norm / 2, stream=s)
    _ready(gd, H.hapi_gradient_workspace_bytes(gd))
    norm = torch.empty(1, device="cuda")
    H.hapi_gradient_clip(gd, norm)
    assert abs(float(norm) - want_norm) <= want_norm * 2 ** -23
    for k_ in names:
        assert float((grads[k_] - before[k_] * 0.5).abs().max()) <= 2 ** -22 * float(before[k_].abs().max())

    # the same by autograd in 64 bits
    P = {k_: v_.double().requires_grad_() for k_, v_ in p.items()}
    ln = torch.nn.functional.layer_norm
    X = ln(x.double(), (768,), P["g1"], P["b1"], 1e-6)
    rms = lambda t, gamma: t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-6) * gamma
    K = rms((X @ P["wk"].t()).view(b, n, kv, d), P["gk"])
    angle = (positions.double()[torch.arange(32, device="cuda") // 16].permute(1, 2, 0) * freq)[:, :, None]
    c, si = torch.cos(angle), torch.sin(angle)
    K = torch.cat([K[..., :32] * c - K[..., 32:] * si, K[..., 32:] * c + K[..., :32] * si], -1)
    V = (X @ P["wv"].t()).view(b, n, kv, d)
    Q = rms(P["queries"].view(1, m, heads, d).expand(b, m, heads, d), P["gq"])
    K, V = (t.repeat_interleave(heads // kv, 2).permute(0, 2, 1, 3) for t in (K, V))
    z = (Q.permute(0, 2, 1, 3) @ K.transpose(-1, -2)) / math.sqrt(d)
    z = z.masked_fill(~mask[:, None, None, :], -math.inf)
    O = (torch.softmax(z, -1) @ V).permute(0, 2, 1, 3).reshape(b * m, heads * d)
    Y = ln(O, (heads * d,), P["g2"], P["b2"], 1e-6)
    total = torch.nn.functional.cross_entropy(Y @ P["w"].t() + P["bias"], targets, ignore_index=-100)
    total.backward()
    assert abs(float((loss.double() * dloss.double()).sum()) - float(total.detach())) <= 1e-5
    for k_ in names:
        rel = float((before[k_].double() - P[k_].grad).norm() / P[k_].grad.norm())
        assert rel <= 1e-3, (k_, rel)


def test_decoder_attends_token_by_token():
    """A decoder's requests of different encoder lengths: keys are rotated once; each
    step rotates and attends with one token, in place and with one workspace for all."""
    b, lk, steps, heads, kv, d = 5, 700, 6, 8, 2, 64
    g = _gen(3)
    kv_lens = torch.tensor([700, 1, 333, 0, 64], device="cuda")
    k = torch.randn(b, lk, kv, d, generator=g, device="cuda").to(BF)
    v = torch.randn(b, lk, kv, d, generator=g, device="cuda").to(BF)
    tokens = torch.randn(b, steps, heads, d, generator=g, device="cuda").to(BF)
    gq, gk = 1 + torch.randn(d, generator=g, device="cuda") * 0.1, 1 + torch.randn(d, generator=g, device="cuda") * 0.1
    freq = torch.tensor([10000.0 ** (-j / 32) for j in range(32)], dtype=torch.float64, device="cuda")
    pos = torch.arange(lk, device="cuda").expand(1, b, lk).contiguous()
    pad = torch.arange(lk, device="cuda") >= kv_lens[:, None]
    k[pad] = math.nan
    v[pad] = math.nan
    s = torch.cuda.current_stream()
    rk = H.Rotary(H.HAPI_BF16, b, lk, 0, kv, d, (32,), stream=s)
    H.hapi_rotary_forward(rk, None, k, None, gk, pos, freq, kv_lens, None, k)
    assert not bool(torch.isnan(k).any())
    at = H.Attention(H.HAPI_BF16, b, 1, lk, heads, kv, d, stream=s)
    _ready(at, H.hapi_cross_attention_workspace_bytes(at))
    rq = H.Rotary(H.HAPI_BF16, b, 1, heads, 0, d, (32,), stream=s)
    out, rotated = [], []
    for t in range(steps):
        q = tokens[:, t:t + 1].contiguous()
        H.hapi_rotary_forward(rq, q, None, gq, None, torch.full((1, b, 1), 5000 + t, device="cuda"), freq, None, q, None)
        o, st = torch.empty_like(q), torch.empty(b, 1, heads, 2, device="cuda")
        H.hapi_cross_attention_forward(at, q, k, v, None, kv_lens, None, o, st)
        rotated.append(q)
        out.append(o)
    want = R.rotary_forward(tokens, gq, torch.arange(5000, 5000 + steps, device="cuda").expand(1, b, steps), freq, (32,))
    R.check("q", torch.cat(rotated, 1), want)
    R.check("o", torch.cat(out, 1), R.Attention(torch.cat(rotated, 1), k, v, kv_lens=kv_lens).forward()[0])
    assert not bool(torch.cat(out, 1)[3].any())


def test_captured_graphs_that_share_a_workspace():
    """Two graphs with one workspace, replayed in turns with eager calls between them."""
    g = _gen(4)
    shapes = [(2, 3, 900, 4, 2, 64), (1, 40, 333, 6, 3, 80)]
    need = 0
    for b, lq, lk, h, kv, d in shapes:
        need = max(need, H.hapi_cross_attention_workspace_bytes(H.Attention(H.HAPI_BF16, b, lq, lk, h, kv, d), True))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    calls = []
    for b, lq, lk, h, kv, d in shapes:
        r = lambda l, n: torch.randn(b, l, n, d, generator=g, device="cuda").to(BF)
        q, k, v, do = r(lq, h), r(lk, kv), r(lk, kv), r(lq, h)
        outs = [torch.empty_like(q), torch.empty(b, lq, h, 2, device="cuda"), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)]
        desc = H.Attention(H.HAPI_BF16, b, lq, lk, h, kv, d, workspace=ws, workspace_bytes=need)

        def call(desc=desc, q=q, k=k, v=v, do=do, outs=outs):
            desc.set(stream=torch.cuda.current_stream())
            H.hapi_cross_attention_forward(desc, q, k, v, None, None, None, outs[0], outs[1])
            H.hapi_cross_attention_backward(desc, q, k, v, None, None, None, outs[0], outs[1], do, *outs[2:])
        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        calls.append((call, graph, outs, (q, k, v, do)))
    for turn in range(3):
        for call, graph, outs, inputs in calls:
            for x in inputs:
                x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
            call()
            torch.cuda.synchronize()
            want = [x.clone() for x in outs]
            for x in outs:
                x.fill_(7.0)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs, want)), turn

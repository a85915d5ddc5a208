"""The operators of a trained block behind extracted tokens, as cases that can be timed and checked.

Three operators: the heads' norm of queries and keys with rotary positions on
several axes, cross attention to an encoder's states, and the global norm of
many gradients with their clipping.  A case names one of them, its type and its
sizes; ``way`` is how far it goes: ``fwd`` the forward pass alone, ``bwd`` the
backward pass alone (rotary), ``step`` a forward and a backward pass (attention),
``norm`` the norm alone and ``clip`` the norm and the scaled gradients.

``run`` computes a case by elementary torch operations in 32 bits, or, with
``own``, by the library's entry points (``hapi_rotary_*``,
``hapi_cross_attention_*``, ``hapi_gradient_*``).  ``exact`` is the definition
in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

_EPS = 1e-6
_SIZE = {"bf16": 2, "f32": 4}
_TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def _rotary(name, way, dtype, batch, length, heads, kv_heads, dim, axes, rot=None, norm=True, neighbours=False, packed=False):
    c = dict(op="rotary", way=way, dtype=dtype, batch=batch, length=length, heads=heads, kv_heads=kv_heads, dim=dim, axes=axes,
             rot=dim if rot is None else rot, norm=norm, neighbours=neighbours, packed=packed)
    return dict(c, name=name) if name else c


def _attend(name, way, dtype, batch, q_len, kv_len, heads, kv_heads, dim, ragged=False, mask=False):
    c = dict(op="attention", way=way, dtype=dtype, batch=batch, q_len=q_len, kv_len=kv_len, heads=heads, kv_heads=kv_heads,
             dim=dim, ragged=ragged, mask=mask)
    return dict(c, name=name) if name else c


def _grads(name, way, dtype, layers, width, classes, max_norm=1.0):
    c = dict(op="gradients", way=way, dtype=dtype, layers=layers, width=width, classes=classes, max_norm=max_norm)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One image's 197 tokens, the patches on a 14 x 14 grid: a launch and little else.
        _rotary("rotary_fwd_1x197_12x64", "fwd", "bf16", 1, 197, 12, 12, 64, 2),
        # The tokens of a batch of 128 images, queries and keys inside the packed projection, and their way back.
        _rotary("rotary_fwd_128x197_12x64", "fwd", "bf16", 128, 197, 12, 12, 64, 2, packed=True),
        _rotary("rotary_bwd_128x197_12x64", "bwd", "bf16", 128, 197, 12, 12, 64, 2, packed=True),
        # A video's tokens on three axes, shared key heads, neighbouring pairs over a part of each head, 32 bits.
        _rotary("rotary_bwd_f32_3x4099_15+5x80", "bwd", "f32", 3, 4099, 15, 5, 80, 3, rot=60, neighbours=True),
        # A decoder's single token of each of 16 requests over a long encoder output, padded to different lengths.
        _attend("attention_fwd_16x1x8192_16+4x128", "fwd", "bf16", 16, 1, 8192, 16, 4, 128, ragged=True),
        # Learned queries over a batch of 128 images' extracted tokens: extraction of features, and training.
        _attend("attention_fwd_128x64x197_12x64", "fwd", "bf16", 128, 64, 197, 12, 12, 64),
        _attend("attention_step_128x64x197_12x64", "step", "bf16", 128, 64, 197, 12, 12, 64),
        # Odd lengths, a ragged batch with a key mask, 32 bits.
        _attend("attention_step_f32_3x77x1021_12+4x80", "step", "f32", 3, 77, 1021, 12, 4, 80, ragged=True, mask=True),
        # A long text over a long encoder output, training; the largest.
        _attend("attention_step_2x4096x4096_16+4x128", "step", "bf16", 2, 4096, 4096, 16, 4, 128),
        # A classifier's two tensors.
        _grads("gradients_clip_1000x2048", "clip", "f32", 0, 2048, 1000),
        # The tensors of 24 encoder blocks of width 640 and a classifier: matrices in 16 bits, vectors in 32.
        _grads("gradients_clip_24x640", "clip", "mixed", 24, 640, 1000),
        # The norm alone of a large model's gradients in 32 bits.
        _grads("gradients_norm_f32_16x2048", "norm", "f32", 16, 2048, 32000),
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Another call of the same kinds: head widths from 16 to 128, odd ones too, one token to the listed cases' most."""
    op = rng.choice(("rotary", "rotary", "attention", "attention", "attention", "gradients"))
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    if op == "gradients":
        c = _grads(None, rng.choice(("norm", "clip")), rng.choice(("bf16", "f32", "mixed")), rng.randint(0, 32),
                   _spread(rng, 16, 2000), _spread(rng, 2, 32000), rng.choice((0.1, 1.0, 10.0)))
        while sum(_sizes(c)) > 1 << 28:
            c["width"] = c["width"] * 3 // 4
        return c
    dim = rng.choice((32, 64, 64, 72, 80, 96, 128, 128, rng.randint(16, 128)))
    kv = rng.choice((1, 2, 4, 5, 8, 12))
    group = rng.choice((1, 1, 2, 3, 4, 8))
    if op == "rotary":
        axes = rng.randint(1, 3)
        rot = dim // 2 * 2 if rng.random() < 0.7 else max(2 * axes, dim // 4 * 2)
        c = _rotary(None, rng.choice(("fwd", "bwd")), dtype, _spread(rng, 1, 128), _spread(rng, 1, 4096), kv * group, kv, dim, axes, rot,
                    rng.random() < 0.7, rng.random() < 0.3, rng.random() < 0.3)
        while c["batch"] * c["length"] * (c["heads"] + c["kv_heads"]) * dim > 1 << 25:
            c["batch"], c["length"] = max(1, c["batch"] // 2), (c["length"] + 1) // 2
        return c
    q_len = 1 if rng.random() < 0.25 else _spread(rng, 2, 4096)
    c = _attend(None, rng.choice(("fwd", "step")), dtype, _spread(rng, 1, 128), q_len, _spread(rng, 1, 16384), kv * group, kv, dim,
                rng.random() < 0.4, rng.random() < 0.3)
    most = 14.0 * 2 * 16 * 4096 * 4096 * 128 / (8 if dtype == "f32" else 1)
    while (work(c)["flops"] > most or c["batch"] * c["heads"] * c["q_len"] * c["kv_len"] > 1 << 29
           or c["batch"] * c["heads"] * (c["q_len"] + c["kv_len"]) * dim > 1 << 28):
        if c["batch"] > 1:
            c["batch"] //= 2
        elif c["kv_len"] > c["q_len"]:
            c["kv_len"] //= 2
        else:
            c["q_len"] //= 2
    return c


# ------------------------------------------------------------------- inputs

def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _sections(case):
    """Pairs of each axis."""
    pairs, n = case["rot"] // 2, case["axes"]
    return [pairs // n + (a < pairs % n) for a in range(n)]


def _sizes(case):
    """The tensors of `layers` encoder blocks, and of the classifier behind them."""
    w = case["width"]
    block = [w, w, 3 * w * w, 3 * w, w * w, w, w, w, 4 * w * w, 4 * w, 4 * w * w, w]
    return block * case["layers"] + [case["classes"] * w, case["classes"]]


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    if case["op"] == "gradients":
        vectors = set((case["width"], 3 * case["width"], 4 * case["width"], case["classes"]))
        grads = []
        for n in _sizes(case):
            t = torch.float32 if case["dtype"] == "f32" or (case["dtype"] == "mixed" and n in vectors) else torch.bfloat16
            grads.append((_randn(g, n) * 0.01).to(t))
        # the clipped ones lie one after another, each type in a buffer of its own
        flat = {t: torch.empty(sum(x.numel() for x in grads if x.dtype == t), dtype=t, device="cuda") for t in {x.dtype for x in grads}}
        at, out = dict.fromkeys(flat, 0), []
        for x in grads:
            out.append(flat[x.dtype][at[x.dtype]:at[x.dtype] + x.numel()])
            at[x.dtype] += x.numel()
        return dict(grads=grads, out=out, flat=[flat[t] for t in (torch.bfloat16, torch.float32) if t in flat])
    t = _TYPE[case["dtype"]]
    b, d, h, kv = case["batch"], case["dim"], case["heads"], case["kv_heads"]
    if case["op"] == "rotary":
        n = case["length"]

        def pair():
            if case["packed"]:
                x = _randn(g, b, n, h + 2 * kv, d).to(t)
                return x[:, :, :h], x[:, :, h:h + kv]
            return _randn(g, b, n, h, d).to(t), _randn(g, b, n, kv, d).to(t)

        q, k = pair()
        s = dict(q=q, k=k, q_gamma=None, k_gamma=None)
        if case["norm"]:
            s["q_gamma"], s["k_gamma"] = _randn(g, d) * 0.1 + 1.0, _randn(g, d) * 0.1 + 1.0
        # places on a grid of `axes` sides, from a start of its own for each entry of the batch
        side = max(1, round(n ** (1.0 / case["axes"])))
        i = torch.arange(n, device="cuda")
        grid = [i // side ** a for a in range(case["axes"])]
        grid = [x % side for x in grid[:-1]] + grid[-1:]
        start = torch.randint(0, 5000, (case["axes"], b, 1), generator=g, device="cuda")
        s["positions"] = torch.stack(grid)[:, None, :] + start
        s["freq"] = torch.tensor([10000.0 ** (-j / m) for m in _sections(case) for j in range(m)], dtype=torch.float64, device="cuda")
        if case["way"] == "bwd":
            s["dq_out"], s["dk_out"] = _randn(g, b, n, h, d).to(t), _randn(g, b, n, kv, d).to(t)
        return s
    lq, lk = case["q_len"], case["kv_len"]
    s = dict(q=_randn(g, b, lq, h, d).to(t), k=_randn(g, b, lk, kv, d).to(t), v=_randn(g, b, lk, kv, d).to(t))
    s["q_lens"] = s["kv_lens"] = s["mask"] = None
    if case["ragged"]:
        # lengths of a padded batch, the longest as long as the tensors
        s["q_lens"] = (lq - (torch.rand(b, generator=g, device="cuda") * lq * 0.5).long()).clamp(min=1)
        s["kv_lens"] = (lk - (torch.rand(b, generator=g, device="cuda") * lk * 0.7).long()).clamp(min=1)
        s["q_lens"][0], s["kv_lens"][0] = lq, lk
    if case["mask"]:
        s["mask"] = torch.rand(b, lk, generator=g, device="cuda") < 0.75
    if case["way"] == "step":
        s["dout"] = _randn(g, b, lq, h, d).to(t)
    return s


def prepare(case, seed):
    """The inputs and, for the library, its descriptor, workspace and outputs."""
    s = _inputs(case, seed)
    s["case"] = case
    if not own:
        return s
    import paper_2210_08650_amd as H
    stream = torch.cuda.current_stream()
    if case["op"] == "gradients":
        s["norm"] = torch.empty(1, device="cuda")
        d = s["desc"] = H.Gradients(s["grads"], max_norm=case["max_norm"], out=s["out"] if case["way"] == "clip" else None, stream=stream)
        need = H.hapi_gradient_workspace_bytes(d)
    else:
        dt = H.HAPI_F32 if case["dtype"] == "f32" else H.HAPI_BF16
        b, dim, h, kv = case["batch"], case["dim"], case["heads"], case["kv_heads"]
        if case["op"] == "rotary":
            d = s["desc"] = H.Rotary(dt, b, case["length"], h, kv, dim, sections=_sections(case), neighbours=case["neighbours"],
                                     norm=case["norm"], eps=_EPS, q_stride=s["q"].stride()[:3], k_stride=s["k"].stride()[:3], stream=stream)
            if case["way"] == "fwd":
                s["q_out"] = torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda")
                s["k_out"] = torch.empty(s["k"].shape, dtype=s["k"].dtype, device="cuda")
                need = 0
            else:
                # the gradients lie as their tensors do
                wide = torch.empty(b, case["length"], h + 2 * kv, dim, dtype=s["q"].dtype, device="cuda") if case["packed"] else None
                s["dq"] = wide[:, :, :h] if case["packed"] else torch.empty_like(s["q"])
                s["dk"] = wide[:, :, h:h + kv] if case["packed"] else torch.empty_like(s["k"])
                s["dq_gamma"] = torch.empty(dim, device="cuda") if case["norm"] else None
                s["dk_gamma"] = torch.empty(dim, device="cuda") if case["norm"] else None
                need = H.hapi_rotary_workspace_bytes(d)
        else:
            step = case["way"] == "step"
            d = s["desc"] = H.Attention(dt, b, case["q_len"], case["kv_len"], h, kv, dim, stream=stream)
            s["o"] = torch.empty_like(s["q"])
            s["stats"] = torch.empty(b, case["q_len"], h, 2, device="cuda")
            if step:
                s["dq"], s["dk"], s["dv"] = torch.empty_like(s["q"]), torch.empty_like(s["k"]), torch.empty_like(s["v"])
            need = H.hapi_cross_attention_workspace_bytes(d, step)
    if need:
        d.set(workspace=torch.empty(need, device="cuda", dtype=torch.uint8), workspace_bytes=need)
    return s


# ------------------------------------------------------------- the operators

def _run_library(s):
    import paper_2210_08650_amd as H
    case, d = s["case"], s["desc"]
    if case["op"] == "gradients":
        if case["way"] == "norm":
            H.hapi_gradient_norm(d, s["norm"])
            return [s["norm"]]
        H.hapi_gradient_clip(d, s["norm"])
        return [s["norm"]] + s["flat"]
    if case["op"] == "rotary":
        if case["way"] == "fwd":
            H.hapi_rotary_forward(d, s["q"], s["k"], s["q_gamma"], s["k_gamma"], s["positions"], s["freq"], None, s["q_out"], s["k_out"])
            return [s["q_out"], s["k_out"]]
        H.hapi_rotary_backward(d, s["dq_out"], s["dk_out"], s["q"], s["k"], s["q_gamma"], s["k_gamma"], s["positions"], s["freq"],
                               None, s["dq"], s["dk"], s["dq_gamma"], s["dk_gamma"])
        return [s["dq"], s["dk"]] + ([s["dq_gamma"], s["dk_gamma"]] if case["norm"] else [])
    H.hapi_cross_attention_forward(d, s["q"], s["k"], s["v"], s["q_lens"], s["kv_lens"], s["mask"], s["o"], s["stats"])
    out = [s["o"], s["stats"]]
    if case["way"] == "step":
        H.hapi_cross_attention_backward(d, s["q"], s["k"], s["v"], s["q_lens"], s["kv_lens"], s["mask"], s["o"], s["stats"],
                                        s["dout"], s["dq"], s["dk"], s["dv"])
        out += [s["dq"], s["dk"], s["dv"]]
    return out


def _plain_gradients(case, s):
    total = torch.zeros(1, dtype=torch.float64, device="cuda")
    for x in s["grads"]:
        f = x.float()
        total += (f * f).sum(dtype=torch.float64)
    norm = total.sqrt()
    if case["way"] == "norm":
        return [norm.float()]
    scale = (case["max_norm"] / norm).clamp(max=1.0).float()
    for x, y in zip(s["grads"], s["out"]):
        y.copy_(x.float() * scale)
    return [norm.float()] + s["flat"]


def _split_pairs(case, x):
    """The two values of every pair, and what is not rotated."""
    r = case["rot"]
    if case["neighbours"]:
        return x[..., 0:r:2], x[..., 1:r:2], x[..., r:]
    return x[..., :r // 2], x[..., r // 2:r], x[..., r:]


def _join_pairs(case, a, b, rest):
    if case["neighbours"]:
        return torch.cat([torch.stack([a, b], -1).flatten(-2), rest], -1)
    return torch.cat([a, b, rest], -1)


def _plain_rotary(case, s):
    t = s["q"].dtype
    axis = torch.tensor([a for a, m in enumerate(_sections(case)) for _ in range(m)], device="cuda")
    # far positions: the angle in 64 bits
    angle = s["positions"].double()[axis].permute(1, 2, 0) * s["freq"]
    cos, sin = torch.cos(angle).float()[:, :, None], torch.sin(angle).float()[:, :, None]
    out, more = [], []
    for x, gamma, name in ((s["q"], s["q_gamma"], "dq_out"), (s["k"], s["k_gamma"], "dk_out")):
        x = x.float()
        r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + _EPS) if case["norm"] else None
        if case["way"] == "fwd":
            h = x * r * gamma if case["norm"] else x
            a, b, rest = _split_pairs(case, h)
            out.append(_join_pairs(case, a * cos - b * sin, b * cos + a * sin, rest).to(t))
            continue
        a, b, rest = _split_pairs(case, s[name].float())
        u = _join_pairs(case, a * cos + b * sin, b * cos - a * sin, rest)
        if case["norm"]:
            h = x * r
            more.append((u * h).sum((0, 1, 2)))
            e = u * gamma
            u = r * (e - h * (e * h).mean(-1, keepdim=True))
        out.append(u.to(t))
    return out + more


def _plain_attention(case, s):
    t = s["q"].dtype
    b, lq, lk, h, kv, d = (case[x] for x in ("batch", "q_len", "kv_len", "heads", "kv_heads", "dim"))
    n = h // kv
    scale = 1.0 / math.sqrt(d)

    def rows(x):  # [b, lq, h, d] -> [b, kv, lq * n, d]
        return x.float().reshape(b, lq, kv, n, d).permute(0, 2, 1, 3, 4).reshape(b, kv, lq * n, d)

    def back(x):
        return x.reshape(b, kv, lq, n, d).permute(0, 2, 1, 3, 4).reshape(b, lq, h, d)

    q, k, v = rows(s["q"]), s["k"].float().permute(0, 2, 1, 3).contiguous(), s["v"].float().permute(0, 2, 1, 3).contiguous()
    z = q @ k.transpose(-1, -2)
    if s["kv_lens"] is not None:
        z = z.masked_fill((torch.arange(lk, device="cuda") >= s["kv_lens"][:, None])[:, None, None, :], -math.inf)
        r = torch.arange(lq * n, device="cuda") // n
        z = z.masked_fill((r >= s["q_lens"][:, None])[:, None, :, None], -math.inf)
    if s["mask"] is not None:
        z = z.masked_fill(~s["mask"][:, None, None, :], -math.inf)
    m = z.amax(-1, keepdim=True)
    empty = m == -math.inf
    p = torch.exp((z - torch.where(empty, 0.0, m)) * scale)
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(empty, 1.0, total)
    stats = torch.cat([m, torch.log(total)], -1)
    out = [back(p @ v).to(t), stats.reshape(b, kv, lq, n, 2).permute(0, 2, 1, 3, 4).reshape(b, lq, h, 2)]
    if case["way"] == "step":
        g = rows(s["dout"])
        dv = p.transpose(-1, -2) @ g
        dp = g @ v.transpose(-1, -2)
        ds = p * (dp - (p * dp).sum(-1, keepdim=True))
        dq, dk = (ds @ k) * scale, (ds.transpose(-1, -2) @ q) * scale
        out += [back(dq).to(t), dk.permute(0, 2, 1, 3).to(t), dv.permute(0, 2, 1, 3).to(t)]
    return out


def run(state):
    if own:
        return _run_library(state)
    case = state["case"]
    return {"gradients": _plain_gradients, "rotary": _plain_rotary, "attention": _plain_attention}[case["op"]](case, state)


# ---------------------------------------------------------- counts and truth

def work(case):
    """Every input read once, every output written once.  A step of attention takes seven products, two of them forward."""
    if case["op"] == "gradients":
        n = sum(_sizes(case))
        size = 4 if case["dtype"] == "f32" else 2
        ways = 2 if case["way"] == "clip" else 1
        return {"bytes": ways * n * size + 4, "flops": (3 if case["way"] == "clip" else 2) * n}
    b, d, h, kv, size = case["batch"], case["dim"], case["heads"], case["kv_heads"], _SIZE[case["dtype"]]
    if case["op"] == "rotary":
        tokens = b * case["length"]
        n = tokens * (h + kv) * d
        fwd = case["way"] == "fwd"
        tensors = 2 if fwd or not case["norm"] else 3
        return {"bytes": tensors * n * size + 8 * tokens * case["axes"], "flops": (8 if fwd else 16) * n}
    lq, lk = case["q_len"], case["kv_len"]
    step = case["way"] == "step"
    q, k = b * lq * h * d, b * lk * kv * d
    return {"bytes": (size * (4 * q + 4 * k) if step else size * (2 * q + 2 * k)) + 8 * b * lq * h,
            "flops": (14 if step else 4) * b * h * lq * lk * d}


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "gradients":
        norm = math.sqrt(sum(float(x.double().square().sum()) for x in s["grads"]))
        value = torch.tensor([norm], dtype=torch.float64, device="cuda")
        if case["way"] == "norm":
            return [value]
        factor = min(1.0, case["max_norm"] / norm) if norm > 0 else 1.0
        return [value] + [torch.cat([x.double() * factor for x in s["grads"] if x.dtype == y.dtype]) for y in s["flat"]]
    if case["op"] == "rotary":
        sections, out, more = _sections(case), [], []
        for x, gamma, name in ((s["q"], s["q_gamma"], "dq_out"), (s["k"], s["k_gamma"], "dk_out")):
            x = x.double()
            rms = (x.square().sum(-1, keepdim=True) / case["dim"] + _EPS).sqrt()
            h = x / rms if case["norm"] else x
            fwd = case["way"] == "fwd"
            y = (h * gamma.double() if case["norm"] else h.clone()) if fwd else s[name].double()
            # one rotation of complex numbers for each pair
            pair = 0
            for a, m in enumerate(sections):
                for _ in range(m):
                    i, j = (2 * pair, 2 * pair + 1) if case["neighbours"] else (pair, pair + sum(sections))
                    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["positions"][a].double() * s["freq"][pair])
                    c = torch.complex(y[..., i], y[..., j]) * (turn if fwd else turn.conj())[..., None]
                    y[..., i], y[..., j] = c.real, c.imag
                    pair += 1
            if not fwd and case["norm"]:
                more.append((y * h).flatten(0, 2).sum(0))
                y = y * gamma.double()
                y = (y - h * ((y * h).sum(-1, keepdim=True) / case["dim"])) / rms
            out.append(y)
        return out + more
    b, lq, lk, h, kv, d = (case[x] for x in ("batch", "q_len", "kv_len", "heads", "kv_heads", "dim"))
    if 1e-12 * work(case)["flops"] + 4e-3 * b * h > 18:
        return None
    f64 = dict(dtype=torch.float64, device="cuda")
    o, stats = torch.zeros(b, lq, h, d, **f64), torch.full((b, lq, h, 2), -math.inf, **f64)
    dq, dk, dv = torch.zeros(b, lq, h, d, **f64), torch.zeros(b, lk, kv, d, **f64), torch.zeros(b, lk, kv, d, **f64)
    for e in range(b):
        nq = lq if s["q_lens"] is None else int(s["q_lens"][e])
        keep = torch.arange(lk, device="cuda")
        if s["kv_lens"] is not None:
            keep = keep[:int(s["kv_lens"][e])]
        if s["mask"] is not None:
            keep = keep[s["mask"][e][keep]]
        if nq == 0 or keep.numel() == 0:
            continue
        for i in range(h):
            c = i // (h // kv)
            q, k, v = s["q"][e, :nq, i].double(), s["k"][e, keep, c].double(), s["v"][e, keep, c].double()
            z = torch.mm(q, k.t())
            p = torch.softmax(z / math.sqrt(d), 1)
            high = z.max(1)[0]
            stats[e, :nq, i, 0] = high
            stats[e, :nq, i, 1] = torch.logsumexp((z - high[:, None]) / math.sqrt(d), 1)
            o[e, :nq, i] = torch.mm(p, v)
            if case["way"] == "step":
                g = s["dout"][e, :nq, i].double()
                dv[e, keep, c] += torch.mm(p.t(), g)
                ds = p * (torch.mm(g, v.t()) - (g * o[e, :nq, i]).sum(1, keepdim=True)) / math.sqrt(d)
                dq[e, :nq, i] = torch.mm(ds, k)
                dk[e, keep, c] += torch.mm(ds.t(), q)
    return [o, stats] + ([dq, dk, dv] if case["way"] == "step" else [])

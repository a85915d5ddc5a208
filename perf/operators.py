"""The operators that train a tail on extracted features, as cases that can be timed and checked.

Three operators: layer norm, the softmax cross entropy of a linear classifier,
and the distillation of that classifier from a teacher's top logits.  A case
names one of them, its type, its sizes and how far it goes: ``fwd`` is the
forward pass alone (evaluation), ``bwd`` the backward pass alone (layer norm),
``step`` a loss and its gradients (training).

``run`` computes a case by elementary torch operations in 32 bits, or, with
``own``, by the library's entry points (``hapi_layernorm_*``, ``hapi_xent_*``,
``hapi_distill_*``).  ``exact`` is the definition in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

_EPS = 1e-6
_SIZE = {"bf16": 2, "f32": 4}
_TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def _norm(name, dtype, rows, dim, way, stride=0):
    c = dict(op="layernorm", way=way, dtype=dtype, rows=rows, dim=dim, stride=stride)
    return dict(c, name=name) if name else c


def _head(name, op, dtype, rows, dim, classes, way, bias=True, top=1, temperature=1.0):
    c = dict(op=op, way=way, dtype=dtype, rows=rows, dim=dim, classes=classes, bias=bias)
    if op == "distill":
        c.update(top=top, temperature=temperature)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One image's 197 tokens: a launch and little else.
        _norm("layernorm_fwd_197x768", "bf16", 197, 768, "fwd"),
        # The tokens of a batch of 128 images, as the transformer normalises them.
        _norm("layernorm_fwd_25216x768", "bf16", 25216, 768, "fwd"),
        # The same tokens on the way back, with the gradients of gamma and beta.
        _norm("layernorm_bwd_25216x768", "bf16", 25216, 768, "bwd"),
        # Odd rows, an odd width and 32 bits, every row's start off alignment.
        _norm("layernorm_bwd_f32_8191x1111", "f32", 8191, 1111, "bwd"),
        # The last batch of an epoch through a small classifier: eight images.
        _head("xent_step_8x768x1000", "xent", "bf16", 8, 768, 1000, "step"),
        # One request's 128 pooled feature vectors of the benchmark model.
        _head("xent_step_128x2048x1000", "xent", "bf16", 128, 2048, 1000, "step"),
        # Evaluation over a large odd class list, no bias, a ragged batch.
        _head("xent_fwd_1000x520x50021", "xent", "bf16", 1000, 520, 50021, "fwd", bias=False),
        # A 32-bit head over many classes.
        _head("xent_step_f32_512x1024x10007", "xent", "f32", 512, 1024, 10007, "step"),
        # A training step over a large vocabulary, and the largest one: the
        # vocabulary's logits would take 2 GB in 16 bits.
        _head("xent_step_4096x768x32000", "xent", "bf16", 4096, 768, 32000, "step", bias=False),
        _head("xent_step_8192x2048x131072", "xent", "bf16", 8192, 2048, 131072, "step", bias=False),
        # Distillation: checking a student on a small batch, and a training
        # step from a teacher's 32 best classes.
        _head("distill_fwd_32x512x1000", "distill", "bf16", 32, 512, 1000, "fwd", top=10, temperature=2.0),
        _head("distill_step_4096x1024x32000", "distill", "bf16", 4096, 1024, 32000, "step", top=32, temperature=2.0),
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Another call of the same kinds: any width, odd ones too, one row to the
    listed cases' most, a thousand classes or a hundred thousand."""
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    if rng.random() < 0.35:
        dim = _spread(rng, 64, 8192)
        if rng.random() < 0.6:
            dim = max(64, dim // 64 * 64)
        rows = _spread(rng, 1, min(65536, (1 << 26) // dim))
        return _norm(None, dtype, rows, dim, rng.choice(("fwd", "bwd")), dim + 24 if rng.random() < 0.2 else 0)
    dim = _spread(rng, 64, 4096)
    if rng.random() < 0.7:
        dim = max(64, dim // 64 * 64)
    case = _head(None, rng.choice(("xent", "distill")), dtype, _spread(rng, 1, 8192), dim, _spread(rng, 100, 131072),
                 rng.choice(("fwd", "step")), rng.random() < 0.5, _spread(rng, 1, 64),
                 rng.choice((1.0, 2.0, 4.0)))
    top = 6.0 * 8192 * 2048 * 131072 / (16 if dtype == "f32" else 1)
    while work(case)["flops"] > top and case["rows"] > 1:
        case["rows"] = case["rows"] * 3 // 4
    return case


# ------------------------------------------------------------------- inputs

def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _inputs(case, seed):
    """Activations of a normalised kind, weights that give logits of a trained
    spread, one row in twenty that does not count (target -100)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    t = _TYPE[case["dtype"]]
    n, d = case["rows"], case["dim"]
    if case["op"] == "layernorm":
        wide = case["stride"] or d
        x = (_randn(g, n, wide) * 1.5 + 0.3).to(t)[:, :d]
        s = dict(x=x, gamma=_randn(g, d) * 0.1 + 1.0, beta=_randn(g, d) * 0.1)
        if case["way"] == "bwd":
            s["dy"] = _randn(g, n, d).to(t)
            x64 = x.double()
            mean = x64.mean(1)
            s["mean"] = mean.float()
            s["rstd"] = (x64.var(1, unbiased=False) + _EPS).rsqrt().float()
        return s
    v = case["classes"]
    s = dict(x=_randn(g, n, d).to(t), w=(_randn(g, v, d) * (2.0 / math.sqrt(d))).to(t),
             bias=_randn(g, v) * 0.1 if case["bias"] else None)
    lost = torch.rand(n, generator=g, device="cuda") < 0.05
    if case["op"] == "xent":
        s["targets"] = torch.randint(0, v, (n,), generator=g, device="cuda").masked_fill_(lost, -100)
    else:
        # distinct classes: a random start and a step that no multiple up to
        # the count brings back to it
        k = case["top"] = min(case["top"], v)
        start = torch.randint(0, v, (n, 1), generator=g, device="cuda")
        ids = (start + torch.arange(k, device="cuda") * max(1, v // k)) % v
        s["ids"] = ids.masked_fill_(lost[:, None], -1)
        s["teacher"] = torch.sort(_randn(g, n, k) * 3.0, dim=1, descending=True)[0]
    s["dloss"] = torch.full((n,), 1.0 / max(1, n - int(lost.sum())), device="cuda")
    return s


def prepare(case, seed):
    """The inputs and, for the library, its descriptor, workspace and outputs."""
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        import paper_2210_08650_amd as H
        dt = H.HAPI_F32 if case["dtype"] == "f32" else H.HAPI_BF16
        n, d = case["rows"], case["dim"]
        stream = torch.cuda.current_stream()
        f32 = dict(device="cuda", dtype=torch.float32)
        if case["op"] == "layernorm":
            s["desc"] = H.Norm(dt, n, d, eps=_EPS, x_stride=case["stride"], stream=stream)
            if case["way"] == "fwd":
                s["y"] = torch.empty(n, d, device="cuda", dtype=s["x"].dtype)
                s["mean"], s["rstd"] = torch.empty(n, **f32), torch.empty(n, **f32)
            else:
                s["dx"] = torch.empty(n, case["stride"] or d, device="cuda", dtype=s["x"].dtype)[:, :d]
                s["dgamma"], s["dbeta"] = torch.empty(d, **f32), torch.empty(d, **f32)
                need = H.hapi_layernorm_workspace_bytes(s["desc"])
        else:
            v = case["classes"]
            top = case["top"] if case["op"] == "distill" else 0
            s["desc"] = H.Head(dt, n, d, v, top=top, temperature=case.get("temperature", 1.0), stream=stream)
            s["loss"], s["stats"] = torch.empty(n, **f32), torch.empty(n, 2, **f32)
            if top:
                s["picked"] = torch.empty(n, top, **f32)
            if case["way"] == "step":
                s["dx"], s["dw"] = torch.empty_like(s["x"]), torch.empty_like(s["w"])
                s["dbias"] = torch.empty(v, **f32) if case["bias"] else None
            need = H.hapi_head_workspace_bytes(s["desc"], case["way"] == "step")
        if case["op"] != "layernorm" or case["way"] == "bwd":
            s["desc"].set(workspace=torch.empty(need, device="cuda", dtype=torch.uint8), workspace_bytes=need)
    return s


# ------------------------------------------------------------- the operators

def _run_library(s):
    import paper_2210_08650_amd as H
    case, d = s["case"], s["desc"]
    if case["op"] == "layernorm":
        if case["way"] == "fwd":
            H.hapi_layernorm_forward(d, s["x"], s["gamma"], s["beta"], s["y"], s["mean"], s["rstd"])
            return [s["y"], s["mean"], s["rstd"]]
        H.hapi_layernorm_backward(d, s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"], s["dx"], s["dgamma"], s["dbeta"])
        return [s["dx"], s["dgamma"], s["dbeta"]]
    step = case["way"] == "step"
    if case["op"] == "xent":
        H.hapi_xent_forward(d, s["x"], s["w"], s["bias"], s["targets"], s["loss"], s["stats"])
        if step:
            H.hapi_xent_backward(d, s["x"], s["w"], s["bias"], s["targets"], s["loss"], s["stats"], s["dloss"], s["dx"],
                                 s["dw"], s["dbias"])
        out = [s["loss"], s["stats"]]
    else:
        H.hapi_distill_forward(d, s["x"], s["w"], s["bias"], s["ids"], s["teacher"], s["loss"], s["stats"], s["picked"])
        if step:
            H.hapi_distill_backward(d, s["x"], s["w"], s["bias"], s["ids"], s["teacher"], s["stats"], s["picked"],
                                    s["dloss"], s["dx"], s["dw"], s["dbias"])
        out = [s["loss"], s["stats"], s["picked"]]
    if step:
        out += [s["dx"], s["dw"]] + ([s["dbias"]] if case["bias"] else [])
    return out


def _plain_norm(case, s):
    t = s["x"].dtype
    x = s["x"].float()
    if case["way"] == "fwd":
        mean = x.mean(1)
        c = x - mean[:, None]
        rstd = 1.0 / torch.sqrt((c * c).mean(1) + _EPS)
        return [(c * rstd[:, None] * s["gamma"] + s["beta"]).to(t), mean, rstd]
    dy = s["dy"].float()
    h = (x - s["mean"][:, None]) * s["rstd"][:, None]
    a = dy * s["gamma"]
    dx = s["rstd"][:, None] * (a - a.mean(1, keepdim=True) - h * (a * h).mean(1, keepdim=True))
    return [dx.to(t), (dy * h).sum(0), dy.sum(0)]


def _plain_head(case, s):
    t = s["x"].dtype
    x, w = s["x"].float(), s["w"].float()
    z = x @ w.t()
    if case["bias"]:
        z = z + s["bias"]
    temp = case.get("temperature", 1.0)
    zt = z / temp if temp != 1.0 else z
    top = zt.amax(1, keepdim=True)
    e = torch.exp(zt - top)
    total = e.sum(1, keepdim=True)
    logsum = torch.log(total)
    lse = (top + logsum)[:, 0]
    stats = torch.cat([z.amax(1, keepdim=True), logsum], 1)
    if case["op"] == "xent":
        counts = s["targets"] >= 0
        ids = s["targets"].clamp(min=0)[:, None]
        q = torch.ones_like(ids, dtype=torch.float32)
        loss = torch.where(counts, lse - z.gather(1, ids)[:, 0], 0.0)
        out = [loss, stats]
    else:
        counts = (s["ids"] >= 0).any(1)
        ids = s["ids"].clamp(min=0)
        u = s["teacher"] / temp
        u = u - u.amax(1, keepdim=True)
        eu = torch.exp(u)
        su = eu.sum(1, keepdim=True)
        q = eu / su
        picked = torch.where(counts[:, None], z.gather(1, ids), 0.0)
        loss = temp * temp * (q * (u - torch.log(su) - picked / temp + lse[:, None])).sum(1)
        out = [torch.where(counts, loss, 0.0), stats, picked]
    if case["way"] == "step":
        coef = torch.where(counts, s["dloss"] * temp, 0.0)[:, None]
        g = e * (coef / total)
        g.scatter_add_(1, ids, -(coef * q))
        out += [(g @ w).to(t), (g.t() @ x).to(t)] + ([g.sum(0)] if case["bias"] else [])
    return out


def run(state):
    if own:
        return _run_library(state)
    case = state["case"]
    return _plain_norm(case, state) if case["op"] == "layernorm" else _plain_head(case, state)


# ---------------------------------------------------------- counts and truth

def work(case):
    """Every input read once, every output written once.  A step takes three
    products: the logits, and the gradients of features and weights."""
    n, d, size = case["rows"], case["dim"], _SIZE[case["dtype"]]
    if case["op"] == "layernorm":
        if case["way"] == "fwd":
            return {"bytes": 2 * n * d * size + 8 * n + 8 * d, "flops": 8 * n * d}
        return {"bytes": 3 * n * d * size + 8 * n + 12 * d, "flops": 14 * n * d}
    v, step = case["classes"], case["way"] == "step"
    small = 20 * n + (4 * v * (2 if step else 1) if case["bias"] else 0)
    if case["op"] == "distill":
        small += 16 * n * min(case["top"], v)
    return {"bytes": (n + v) * d * size * (2 if step else 1) + small, "flops": (6 if step else 2) * n * d * v}


def exact(case, seed):
    s = _inputs(case, seed)
    n, d = case["rows"], case["dim"]
    x = s["x"].double()
    if case["op"] == "layernorm":
        gamma, beta = s["gamma"].double(), s["beta"].double()
        if case["way"] == "fwd":
            mean = x.sum(1) / d
            var = ((x - mean[:, None]) ** 2).sum(1) / d
            rstd = (var + _EPS) ** -0.5
            return [gamma * ((x - mean[:, None]) * rstd[:, None]) + beta, mean, rstd]
        # the statistics are inputs of the pass
        dy, r = s["dy"].double(), s["rstd"].double()[:, None]
        h = (x - s["mean"].double()[:, None]) * r
        a = gamma * dy
        proj = (a * h).sum(1, keepdim=True) / d
        return [r * (a - a.sum(1, keepdim=True) / d - h * proj), (h * dy).sum(0), dy.sum(0)]
    v, step, temp = case["classes"], case["way"] == "step", float(case.get("temperature", 1.0))
    w = s["w"].double()
    bias = s["bias"].double() if case["bias"] else torch.zeros(v, dtype=torch.float64, device="cuda")
    piece = max(1, min(n, (1 << 28) // v))  # rows at once
    loss, stats, picked, dx = [], [], [], []
    dw = torch.zeros(v, d, dtype=torch.float64, device="cuda") if step else None
    db = torch.zeros(v, dtype=torch.float64, device="cuda") if step else None
    for a in range(0, n, piece):
        xb = x[a:a + piece]
        z = torch.addmm(bias, xb, w.t())
        l = torch.logsumexp(z / temp, 1)
        high = z.max(1)[0]
        stats.append(torch.stack([high, l - high / temp], 1))
        rows = torch.arange(xb.shape[0], device="cuda")
        if case["op"] == "xent":
            t = s["targets"][a:a + piece]
            ok = t >= 0
            r = rows[ok]
            part = torch.zeros_like(l)
            part[ok] = l[ok] - z[r, t[ok]]
            want = [(r, t[ok], torch.ones(r.numel(), dtype=torch.float64, device="cuda"))]
        else:
            ids, ok = s["ids"][a:a + piece], s["ids"][a:a + piece, 0] >= 0
            logq = torch.log_softmax(s["teacher"][a:a + piece].double() / temp, 1)
            q = torch.exp(logq) * ok[:, None]
            zk = torch.zeros_like(logq)
            part = torch.zeros_like(l)
            want = []
            for k in range(ids.shape[1]):
                zk[ok, k] = z[rows[ok], ids[ok, k]]
                part += temp * temp * q[:, k] * (logq[:, k] - zk[:, k] / temp + l)
                want.append((rows[ok], ids[ok, k], q[ok, k]))
            picked.append(zk)
        loss.append(part)
        if step:
            scale = s["dloss"][a:a + piece].double() * temp * ok
            g = torch.exp(z / temp - l[:, None]) * scale[:, None]
            for r, c, q in want:
                g[r, c] -= scale[r] * q
            dx.append(g @ w)
            dw.addmm_(g.t(), xb)
            db += g.sum(0)
    out = [torch.cat(loss), torch.cat(stats)] + ([torch.cat(picked)] if picked else [])
    if step:
        out += [torch.cat(dx), dw] + ([db] if case["bias"] else [])
    return out

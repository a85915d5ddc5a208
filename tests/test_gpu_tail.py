"""The trained tail's operators on the GPU against their definitions in 64 bits:
layer norm, the classifier's cross entropy and its distillation, forward and
backward.  Bounds come from tests/tail_reference.py; every output and workspace
lies between guards."""
import math

import pytest
import torch

import paper_2210_08650_amd as H
from paper_2210_08650_amd import models as PM
from tests import tail_reference as R
from tests.hip_harness import Guarded

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
CODE = {BF: H.HAPI_BF16, F32: H.HAPI_F32}


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _guarded(shape, dtype):
    b = Guarded(math.prod(shape) * torch.empty(0, dtype=dtype).element_size())
    return b, b.view(dtype, shape)


class Outs:
    """Guarded outputs by name."""

    def __init__(self):
        self.bufs, self.t = [], {}

    def add(self, name, shape, dtype=F32):
        b, self.t[name] = _guarded(shape, dtype)
        self.bufs.append(b)
        return self.t[name]

    def check(self):
        for b in self.bufs:
            b.check()


def _strided(x, extra):
    """x's values in rows `extra` elements wider than its own."""
    if not extra:
        return x
    wide = torch.full((x.shape[0], x.shape[1] + extra), 7.0, dtype=x.dtype, device=x.device)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


# ----------------------------------------------------------------- layer norm

NORM_SHAPES = [(1, 1), (3, 1), (5, 2), (1, 768), (197, 768), (33, 7), (64, 64), (17, 127), (130, 128), (9, 129), (21, 511),
               (40, 513), (300, 1023), (12, 1111), (70, 2048), (11, 2049), (6, 4096), (5, 5000), (4, 8192), (3, 8201),
               (2, 16383), (3, 16384), (5000, 96)]


def _norm_desc(x, y, eps=1e-6, ws=None):
    d = H.Norm(CODE[x.dtype], x.shape[0], x.shape[1], eps=eps, x_stride=x.stride(0) if x.shape[0] > 1 else 0,
               y_stride=y.stride(0) if y.shape[0] > 1 else 0, stream=torch.cuda.current_stream())
    if ws is not None:
        d.set(workspace=ws.body, workspace_bytes=ws.nbytes)
    return d


def _norm_case(seed, rows, dim, dtype, xs=0, ys=0):
    g = _gen(seed)
    x = _strided((_randn(g, rows, dim) * 1.5 + 0.3).to(dtype), xs)
    dy = _strided(_randn(g, rows, dim).to(dtype), ys)
    return x, dy, _randn(g, dim) * 0.1 + 1.0, _randn(g, dim) * 0.1


def _norm_forward(x, gamma, beta, ys=0, eps=1e-6):
    rows, dim = x.shape
    o = Outs()
    y = o.add("y", (rows, dim + ys), x.dtype)
    y.fill_(5.0)
    mean, rstd = o.add("mean", (rows,)), o.add("rstd", (rows,))
    H.hapi_layernorm_forward(_norm_desc(x, y[:, :dim], eps), x, gamma, beta, y[:, :dim], mean, rstd)
    torch.cuda.synchronize()
    o.check()
    assert bool((y[:, dim:] == 5.0).all()), "wrote between rows"
    return y[:, :dim], mean, rstd


def _norm_backward(dy, x, gamma, mean, rstd, xs=0):
    rows, dim = x.shape
    o = Outs()
    dx = o.add("dx", (rows, dim + xs), x.dtype)
    dx.fill_(5.0)
    dg, db = o.add("dgamma", (dim,)), o.add("dbeta", (dim,))
    need = H.hapi_layernorm_workspace_bytes(_norm_desc(x, dy))
    ws = Guarded(need)
    H.hapi_layernorm_backward(_norm_desc(x, dy, ws=ws), dy, x, gamma, mean, rstd, dx[:, :dim], dg, db)
    torch.cuda.synchronize()
    o.check()
    ws.check()
    assert bool((dx[:, dim:] == 5.0).all()), "wrote between rows"
    return dx[:, :dim], dg, db


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,dim", NORM_SHAPES)
def test_norm(rows, dim, dtype):
    x, dy, gamma, beta = _norm_case(rows * 31 + dim, rows, dim, dtype)
    got = _norm_forward(x, gamma, beta)
    for name, a, b in zip(("y", "mean", "rstd"), got, R.norm_forward(x, gamma, beta, 1e-6)):
        R.check(name, a, b)
    mean, rstd = got[1].clone(), got[2].clone()
    for name, a, b in zip(("dx", "dgamma", "dbeta"), _norm_backward(dy, x, gamma, mean, rstd),
                          R.norm_backward(dy, x, gamma, mean, rstd)):
        R.check(name, a, b)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,dim,xs,ys", [(50, 768, 24, 8), (50, 768, 3, 0), (7, 100, 1, 5), (19, 2050, 0, 1)])
def test_norm_row_strides(rows, dim, xs, ys, dtype):
    x, dy, gamma, beta = _norm_case(5, rows, dim, dtype, xs, ys)
    y, mean, rstd = _norm_forward(x, gamma, beta, ys)
    want = R.norm_forward(x, gamma, beta, 1e-6)
    R.check("y", y, want[0])
    R.check("rstd", rstd, want[2])
    dx, dg, db = _norm_backward(dy, x, gamma, mean, rstd, xs)
    want = R.norm_backward(dy, x, gamma, mean, rstd)
    R.check("dx", dx, want[0])
    R.check("dgamma", dg, want[1])
    R.check("dbeta", db, want[2])


def test_norm_offsets_past_32_bits():
    """2.3e9 elements from the first row to the last."""
    x, dy, gamma, beta = _norm_case(6, 2200, 50, BF, 2 ** 20 - 50)
    want = R.norm_forward(x, gamma, beta, 1e-6)
    got = _norm_forward(x, gamma, beta)
    for name, t, w in zip(("y", "mean", "rstd"), got, want):
        R.check(name, t, w)
    back = _norm_backward(dy, x, gamma, got[1], got[2], 2 ** 20 - 50)
    for name, t, w in zip(("dx", "dgamma", "dbeta"), back, R.norm_backward(dy, x, gamma, got[1], got[2])):
        R.check(name, t, w)


def test_norm_unaligned_start():
    """A tensor that starts one element into its allocation."""
    for dtype in (BF, F32):
        x, dy, gamma, beta = _norm_case(6, 20, 770, dtype)
        flat = torch.empty(20 * 770 + 1, dtype=dtype, device="cuda")
        xo = flat[1:].view(20, 770)
        xo.copy_(x)
        y, mean, rstd = _norm_forward(xo, gamma, beta)
        y2, mean2, rstd2 = _norm_forward(x, gamma, beta)
        assert torch.equal(y, y2) and torch.equal(mean, mean2) and torch.equal(rstd, rstd2)


def test_norm_constant_rows_large_values_and_nan():
    gamma, beta = torch.ones(96, device="cuda"), torch.zeros(96, device="cuda")
    x = torch.zeros(4, 96, device="cuda")
    x[0] = 0.3                          # no variance: y is 0 up to eps' amplification of roundings
    x[1] = torch.arange(96.0) * 1e15    # squares near 1e34
    x[2, 5] = math.nan
    x[3] = torch.arange(96.0)
    y, mean, rstd = _norm_forward(x, gamma, beta)
    want = R.norm_forward(x, gamma, beta, 1e-6)
    for i in (0, 1, 3):
        for a, b in zip((y, mean, rstd), want):
            R.check(f"row {i}", a[i:i + 1], (b[0][i:i + 1], b[1][i:i + 1]))
    assert bool(torch.isnan(y[2]).all()) and not bool(torch.isnan(y[[0, 1, 3]]).any())


def test_norm_no_rows():
    gamma = torch.ones(48, device="cuda")
    x = torch.empty(0, 48, device="cuda")
    s = torch.empty(0, device="cuda")
    _norm_forward(x, gamma, gamma)
    _, dg, db = _norm_backward(x, x, gamma, s, s)
    assert bool((dg == 0).all()) and bool((db == 0).all())


def test_norm_gradient_against_differences():
    """Central differences of the library's own forward pass in float32: the sum
    of y dy moves by <dx, v> 2 h along v.  Truncation is h^2 / 6 of the third
    derivative (of the size of the first for |v| = 1 a value and h = 1e-2: 2e-5);
    each y is off by 1e-6 at most here, so the quotient by 1e-6 |dy|_1 / h."""
    x, dy, gamma, beta = _norm_case(8, 6, 40, F32)
    y, mean, rstd = _norm_forward(x, gamma, beta)
    dx, dg, db = _norm_backward(dy, x, gamma, mean, rstd)
    g, h = _gen(9), 1e-2
    f = lambda x_, g_, b_: float((_norm_forward(x_, g_, b_)[0].double() * dy.double()).sum())
    noise = 1e-6 * float(dy.abs().sum()) / h
    v = _randn(g, 6, 40)
    slope = (f(x + h * v, gamma, beta) - f(x - h * v, gamma, beta)) / (2 * h)
    want = float((dx.double() * v.double()).sum())
    assert abs(slope - want) <= noise + 1e-3 * float((dx * v).abs().sum())
    v = _randn(g, 40)
    slope = (f(x, gamma + h * v, beta) - f(x, gamma - h * v, beta)) / (2 * h)
    assert abs(slope - float((dg.double() * v.double()).sum())) <= noise
    slope = (f(x, gamma, beta + h * v) - f(x, gamma, beta - h * v)) / (2 * h)
    assert abs(slope - float((db.double() * v.double()).sum())) <= noise


# ------------------------------------------------------- classifier's losses

def _head_case(seed, rows, dim, classes, dtype, bias=True, top=0, spread=2.0):
    g = _gen(seed)
    c = dict(x=_randn(g, rows, dim).to(dtype), w=(_randn(g, classes, dim) * (spread / math.sqrt(dim))).to(dtype),
             bias=_randn(g, classes) * 0.5 if bias else None, teacher=None, temp=1.0,
             dloss=torch.rand(rows, generator=g, device="cuda") + 0.1)
    lost = torch.rand(rows, generator=g, device="cuda") < 0.15
    if top:
        c["ids"] = torch.randint(0, classes, (rows, top), generator=g, device="cuda")  # repeats among them
        c["ids"][torch.rand(rows, top, generator=g, device="cuda") < 0.1] = -1
        c["ids"][lost] = -5
        c["teacher"] = _randn(g, rows, top) * 3.0
        c["temp"] = 2.0
    else:
        c["ids"] = torch.randint(0, classes, (rows,), generator=g, device="cuda").masked_fill_(lost, -100)
    return c


def _head_run(c, backward=True, stream=None):
    x, w, ids, teacher = c["x"], c["w"], c["ids"], c["teacher"]
    rows, dim = x.shape
    top = ids.shape[1] if teacher is not None else 0
    xs, wsd = x.stride(0) if rows > 1 else dim, w.stride(0) if w.shape[0] > 1 else dim
    d = H.Head(CODE[x.dtype], rows, dim, w.shape[0], top=top, temperature=c["temp"], x_stride=xs, w_stride=wsd,
               stream=stream or torch.cuda.current_stream())
    o = Outs()
    loss, stats = o.add("loss", (rows,)), o.add("stats", (rows, 2))
    ws = Guarded(H.hapi_head_workspace_bytes(d, False))
    d.set(workspace=ws.body, workspace_bytes=ws.nbytes)
    if top:
        picked = o.add("picked", (rows, top))
        H.hapi_distill_forward(d, x, w, c["bias"], ids, teacher, loss, stats, picked)
    else:
        H.hapi_xent_forward(d, x, w, c["bias"], ids, loss, stats)
    torch.cuda.synchronize()
    ws.check()
    if backward:
        dxw, dww = o.add("dx", (rows, xs), x.dtype), o.add("dw", (w.shape[0], wsd), x.dtype)
        dxw.fill_(5.0)
        dww.fill_(5.0)
        db = o.add("db", (w.shape[0],)) if c["bias"] is not None else None
        ws2 = Guarded(H.hapi_head_workspace_bytes(d, True))
        d.set(workspace=ws2.body, workspace_bytes=ws2.nbytes)
        if top:
            H.hapi_distill_backward(d, x, w, c["bias"], ids, teacher, stats, picked, c["dloss"], dxw[:, :dim], dww[:, :dim], db)
        else:
            H.hapi_xent_backward(d, x, w, c["bias"], ids, loss, stats, c["dloss"], dxw[:, :dim], dww[:, :dim], db)
        torch.cuda.synchronize()
        ws2.check()
        assert bool((dxw[:, dim:] == 5.0).all()) and bool((dww[:, dim:] == 5.0).all()), "wrote between rows"
        o.t["dx"], o.t["dw"] = dxw[:, :dim], dww[:, :dim]
    o.check()
    return o.t


def _head_check(c, got):
    want = R.head(c["x"], c["w"], c["bias"], c["ids"], c["teacher"], c["temp"], c["dloss"] if "dx" in got else None)
    for name, t in got.items():
        # float32: a logit's rounding, 4e-5 at the largest spread here
        R.check(name, t, want[name], 4e-5 if name in ("dx", "dw") and t.dtype == F32 else None)
    counts = c["ids"] >= 0 if c["teacher"] is None else (c["ids"] >= 0).any(1)
    assert bool((got["loss"][~counts] == 0).all())
    if "dx" in got:
        assert bool((got["dx"][~counts] == 0).all())


HEAD_SHAPES = [(8192, 64, 100), (4096, 40, 1000), (2000, 130, 300), (20, 520, 9000), (1, 1, 1), (1, 8, 2), (2, 16, 1), (1, 64, 1000), (3, 7, 5), (8, 768, 1000), (31, 72, 127), (32, 64, 128),
               (33, 96, 129), (64, 200, 255), (65, 64, 257), (128, 512, 1000), (129, 777, 300), (200, 520, 5003),
               (257, 128, 1024), (1000, 64, 333), (300, 1030, 2000), (515, 2048, 700)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,dim,classes", HEAD_SHAPES)
def test_cross_entropy(rows, dim, classes, dtype):
    c = _head_case(rows + dim + classes, rows, dim, classes, dtype, bias=classes % 2 == 1 or rows < 100)
    _head_check(c, _head_run(c))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,dim,classes,top", [(1, 8, 3, 1), (1, 64, 1000, 7), (5, 7, 4, 9), (32, 512, 1000, 10),
                                                  (33, 100, 129, 3), (66, 96, 255, 64), (130, 777, 1003, 5),
                                                  (257, 256, 5003, 32), (40, 64, 300, 200), (3000, 64, 130, 20)])
def test_distillation(rows, dim, classes, top, dtype):
    c = _head_case(rows + dim + classes + top, rows, dim, classes, dtype, bias=rows % 2 == 1, top=top)
    _head_check(c, _head_run(c))


@pytest.mark.parametrize("top", [0, 4])
def test_several_pieces_of_the_classes(top):
    """dz^T of all classes would be 287 MB: two pieces."""
    c = _head_case(3, 2048, 64, 70001, BF, bias=True, top=top)
    _head_check(c, _head_run(c))


@pytest.mark.parametrize("rows,classes,top", [(1000, 50021, 0), (600, 33000, 3), (1300, 22100, 0)])
def test_last_round_in_smaller_tiles(rows, classes, top):
    """A few 256 x 256 tiles more than whole rounds of the CUs."""
    c = _head_case(rows, rows, 64, classes, BF, bias=True, top=top)
    _head_check(c, _head_run(c))


def test_pieces_in_float32():
    c = _head_case(4, 1100, 40, 60100, F32, bias=False)
    _head_check(c, _head_run(c))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,dim,classes,top", [(256, 40, 90, 5), (1023, 32, 60, 40), (1025, 16, 33, 3)])
def test_distillation_waves_to_a_row(rows, dim, classes, top, dtype):
    c = _head_case(rows + top, rows, dim, classes, dtype, bias=True, top=top)
    _head_check(c, _head_run(c))


@pytest.mark.parametrize("rows,dim,classes,top", [(2, 16, 2100001, 0), (3, 24, 2100001, 3), (5, 66000, 70, 0),
                                                  (40, 20000, 130, 2), (70001, 24, 11, 2)])
def test_far_ends_of_the_sizes(rows, dim, classes, top):
    """Few rows and several pieces of the classes, many features, many rows."""
    c = _head_case(rows + top, rows, dim, classes, BF, bias=True, top=top)
    _head_check(c, _head_run(c))


@pytest.mark.parametrize("which", ["x", "w"])
def test_offsets_past_32_bits(which):
    """The longest row stride: 2.3e9 elements from the first row to the last."""
    rows, classes = (2200, 100) if which == "x" else (100, 2200)
    c = _head_case(5, rows, 64, classes, BF)
    c[which] = _strided(c[which], 2 ** 20 - 64)
    _head_check(c, _head_run(c))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("dim,xs,ws", [(64, 16, 8), (64, 1, 0), (64, 0, 3), (50, 2, 6)])
def test_head_row_strides(dim, xs, ws, dtype):
    c = _head_case(21, 70, dim, 150, dtype)
    c["x"], c["w"] = _strided(c["x"], xs), _strided(c["w"], ws)
    _head_check(c, _head_run(c))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,top", [(20, 0), (150, 0), (20, 3), (150, 3)])
def test_padded_rows_may_hold_anything(rows, top, dtype):
    """Features of rows that do not count reach nothing: NaN and infinities there
    leave every other result as zeros there do."""
    c = _head_case(11, rows, 72, 200, dtype, top=top)
    lost = (c["ids"] if not top else c["ids"].amax(1)) < 0
    assert bool(lost.any())
    c["x"][lost] = 0.0
    a = _head_run(c)
    c["x"][lost] = math.nan
    c["x"][lost.nonzero()[0, 0]] = math.inf
    c["dloss"][lost] = 3.0
    b = _head_run(c)
    for name in ("loss", "dx", "dw", "db"):
        assert torch.equal(a[name], b[name]), name
    assert torch.equal(a["stats"][~lost], b["stats"][~lost])


@pytest.mark.parametrize("top", [0, 3])
def test_no_row_counts(top):
    c = _head_case(12, 40, 64, 100, BF, top=top)
    c["ids"].fill_(-1)
    got = _head_run(c)
    for name in ("loss", "dx", "dw", "db"):
        assert bool((got[name] == 0).all()), name


@pytest.mark.parametrize("top", [0, 3])
def test_no_rows(top):
    c = _head_case(12, 0, 64, 100, BF, top=top)
    got = _head_run(c)
    assert bool((got["dw"] == 0).all()) and bool((got["db"] == 0).all())


def test_rows_without_gradient_add_nothing():
    c = _head_case(13, 90, 64, 100, BF)
    c["dloss"][::2] = 0.0
    got = _head_run(c)
    _head_check(c, got)
    assert bool((got["dx"][::2] == 0).all())


@pytest.mark.parametrize("low", [-math.inf, torch.finfo(torch.float32).min])
@pytest.mark.parametrize("rows", [10, 100])
def test_classes_taken_out_by_the_bias(rows, low):
    """Classes with a bias of -inf or the lowest value have no probability and no gradient."""
    c = _head_case(14, rows, 64, 300, BF)
    out = torch.rand(300, generator=_gen(15), device="cuda") < 0.5
    out[:130] = True  # whole tiles of them
    c["bias"][out] = low
    inside = (~out).nonzero()[:, 0]
    c["ids"] = inside[torch.randint(0, len(inside), (rows,), generator=_gen(16), device="cuda")]
    got = _head_run(c)
    _head_check(c, got)
    assert bool((got["dw"][out] == 0).all()) and bool((got["db"][out] == 0).all())


@pytest.mark.parametrize("top", [0, 2])
def test_every_class_at_the_lowest_value(top):
    """All logits at the end of the range, so all equal: p = 1 / classes, and the
    loss of cross entropy log(classes)."""
    c = _head_case(17, 6, 64, 100, F32, top=top)
    c["bias"].fill_(torch.finfo(torch.float32).min)
    c["ids"].fill_(3)
    got = _head_run(c)
    coef = c["dloss"].double().sum() * c["temp"]
    want = torch.full((100,), 0.01, dtype=torch.float64, device="cuda") * coef
    want[3] = -0.99 * coef
    # a logarithm, an exponential and a sum of six
    assert float((got["db"].double() - want).abs().max()) <= 64 * R.F * float(coef)
    if not top:
        assert float((got["loss"].double() - math.log(100)).abs().max()) <= 8 * R.F * math.log(100)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_large_logits(dtype):
    """Logits of a few hundred: one class takes nearly everything."""
    c = _head_case(18, 50, 64, 120, dtype, spread=100.0)
    _head_check(c, _head_run(c))


def test_target_past_the_classes_is_nan():
    c = _head_case(19, 12, 64, 50, BF)
    c["ids"] = torch.arange(12, device="cuda") % 50
    good = _head_run(c)
    c["ids"][4] = 50
    got = _head_run(c)
    assert math.isnan(float(got["loss"][4])) and bool(torch.isnan(got["dx"][4]).all())
    keep = torch.arange(12, device="cuda") != 4
    for name in ("loss", "dx"):
        assert torch.equal(got[name][keep], good[name][keep]), name
    assert bool(torch.isnan(got["dw"]).all())


def test_distillation_entries():
    """Weights of -inf, repeated classes, entries in another order, an id past the
    classes, a teacher's NaN or +inf."""
    c = _head_case(20, 8, 64, 40, F32, top=4)
    c["ids"] = torch.tensor([[1, 2, 3, 4]] * 8, device="cuda")
    c["teacher"][1, 2] = -math.inf
    c["ids"][2] = torch.tensor([7, 7, 7, 9], device="cuda")
    c["teacher"][3] = -math.inf           # no entry: does not count
    got = _head_run(c)
    want = R.head(c["x"], c["w"], c["bias"], c["ids"], c["teacher"], c["temp"], c["dloss"])
    for name, t in got.items():
        R.check(name, t, want[name])
    assert float(got["loss"][3]) == 0 and bool((got["dx"][3] == 0).all())
    swap = dict(c, ids=c["ids"][:, [2, 0, 3, 1]].contiguous(), teacher=c["teacher"][:, [2, 0, 3, 1]].contiguous())
    again = _head_run(swap)
    for name in ("dx", "dw"):
        R.check(name, again[name], want[name])
    for what in ("id", "nan", "inf"):
        bad = dict(c, ids=c["ids"].clone(), teacher=c["teacher"].clone())
        if what == "id":
            bad["ids"][5, 1] = 40
        else:
            bad["teacher"][5, 1] = float(what)
        b = _head_run(bad)
        keep = torch.arange(8, device="cuda") != 5
        assert math.isnan(float(b["loss"][5])) and bool(torch.isnan(b["dx"][5]).all()), what
        assert torch.equal(b["loss"][keep], got["loss"][keep]) and torch.equal(b["dx"][keep], got["dx"][keep])


@pytest.mark.parametrize("rows,classes", [(20, 900), (300, 5003), (700, 33000)])
def test_a_mean_keeps_its_targets_whole(rows, classes):
    """With one dloss for all rows a target's entry of dz is -1 + p of a power of
    two, so dz's rounding to 16 bits takes at most 2^-9 of p there, not up to 2^-8
    of the whole gradient: what is left is the gradients' own rounding, 2^-8 / sqrt 3
    of their length at most, and the small entries'."""
    c = _head_case(50, rows, 96, classes, BF, bias=False, spread=1.0)
    c["dloss"].fill_(1.0 / 7782)  # a significand of 1.0527: 16 bits would put 1.0547
    got = _head_run(c)
    want = R.head(c["x"], c["w"], None, c["ids"], None, 1.0, c["dloss"])
    for name in ("dx", "dw"):
        R.check(name, got[name], want[name], 1.1 * 2.0 ** -8 / math.sqrt(3))


@pytest.mark.parametrize("top", [0, 3])
def test_head_gradient_against_differences(top):
    """Central differences of the library's own forward pass in float32, 300
    classes, h = 1e-2: sum(dloss loss) is off by about 3e-6 a row (its logits' and
    log-sum-exp's roundings), the truncation h^2 / 6 of a third derivative, which
    is at most a few |dz| |v|^3."""
    c = _head_case(22, 9, 32, 300, F32, top=top)
    got = {k: v.clone() for k, v in _head_run(c).items()}
    h, g = 1e-2, _gen(23)
    f = lambda: float((_head_run(c, backward=False)["loss"].double() * c["dloss"].double()).sum())
    noise = 4e-6 * float(c["dloss"].sum()) * c["temp"] ** 2 * 3 / h
    for key, grad in (("x", "dx"), ("w", "dw"), ("bias", "db")):
        v = _randn(g, *c[key].shape) * (0.1 if key == "w" else 1.0)
        keep = c[key]
        c[key] = keep + h * v
        up = f()
        c[key] = keep - h * v
        down = f()
        c[key] = keep
        terms = got[grad].double() * v.double()
        assert abs((up - down) / (2 * h) - float(terms.sum())) <= noise + 1e-3 * float(terms.abs().sum()), key


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,top", [(20, 0), (300, 5)])
def test_same_bits_every_time(rows, top, dtype):
    c = _head_case(24, rows, 136, 1500, dtype, top=top)
    a = {k: v.clone() for k, v in _head_run(c).items()}
    for _ in range(3):
        b = _head_run(c)
        for k in a:
            assert torch.equal(a[k], b[k]), k


def test_two_streams_at_once():
    """Calls on two streams with their own workspaces, overlapping."""
    cases = [_head_case(25 + i, 200 + 50 * i, 256, 4000, BF, top=3 * i) for i in range(2)]
    want = [{k: v.clone() for k, v in _head_run(c).items()} for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    runs = []
    for c, s in zip(cases, streams):
        x, w = c["x"], c["w"]
        top = c["ids"].shape[1] if c["teacher"] is not None else 0
        d = H.Head(H.HAPI_BF16, x.shape[0], x.shape[1], w.shape[0], top=top, temperature=c["temp"], stream=s)
        need = H.hapi_head_workspace_bytes(d, True)
        d.set(workspace=torch.empty(need, dtype=torch.uint8, device="cuda"), workspace_bytes=need)
        o = {k: torch.empty_like(v) for k, v in _head_run(c).items()}
        runs.append((d, c, o, top))
    torch.cuda.synchronize()
    for _ in range(4):
        for d, c, o, top in runs:
            if top:
                H.hapi_distill_forward(d, c["x"], c["w"], c["bias"], c["ids"], c["teacher"], o["loss"], o["stats"], o["picked"])
                H.hapi_distill_backward(d, c["x"], c["w"], c["bias"], c["ids"], c["teacher"], o["stats"], o["picked"],
                                        c["dloss"], o["dx"], o["dw"], o["db"])
            else:
                H.hapi_xent_forward(d, c["x"], c["w"], c["bias"], c["ids"], o["loss"], o["stats"])
                H.hapi_xent_backward(d, c["x"], c["w"], c["bias"], c["ids"], o["loss"], o["stats"], c["dloss"], o["dx"],
                                     o["dw"], o["db"])
    torch.cuda.synchronize()
    for (_, _, o, _), e in zip(runs, want):
        for k in e:
            assert torch.equal(o[k], e[k]), k


# ------------------------------------------------------------ them together

class Tail:
    """A trained tail over extracted features: layer norm, classifier, loss."""

    def __init__(self, rows, dim, classes, dtype, seed, top=0, stride=0, stream=None):
        g = _gen(seed)
        self.dtype, self.top = dtype, top
        self.gamma, self.beta = _randn(g, dim) * 0.1 + 1.0, _randn(g, dim) * 0.1
        self.w = (_randn(g, classes, dim) / math.sqrt(dim)).to(dtype)
        self.bias = _randn(g, classes) * 0.1
        stream = stream or torch.cuda.current_stream()
        self.norm = H.Norm(CODE[dtype], rows, dim, x_stride=stride, stream=stream)
        self.head = H.Head(CODE[dtype], rows, dim, classes, top=top, temperature=2.0 if top else 1.0, stream=stream)
        n1, n2 = H.hapi_layernorm_workspace_bytes(self.norm), H.hapi_head_workspace_bytes(self.head, True)
        ws = torch.empty(max(n1, n2), dtype=torch.uint8, device="cuda")  # one workspace: the calls are in order
        self.norm.set(workspace=ws, workspace_bytes=n1)
        self.head.set(workspace=ws, workspace_bytes=n2)
        e = lambda *s, t=F32: torch.empty(*s, dtype=t, device="cuda")
        self.y, self.dy = e(rows, dim, t=dtype), e(rows, dim, t=dtype)
        self.dx = torch.zeros(rows, stride or dim, dtype=dtype, device="cuda")[:, :dim]
        self.mean, self.rstd, self.loss, self.stats = e(rows), e(rows), e(rows), e(rows, 2)
        self.dgamma, self.dbeta, self.dbias = e(dim), e(dim), e(classes)
        self.dw = torch.empty_like(self.w)
        self.picked = e(rows, top) if top else None

    def step(self, x, ids, dloss, teacher=None):
        H.hapi_layernorm_forward(self.norm, x, self.gamma, self.beta, self.y, self.mean, self.rstd)
        if self.top:
            H.hapi_distill_forward(self.head, self.y, self.w, self.bias, ids, teacher, self.loss, self.stats, self.picked)
            H.hapi_distill_backward(self.head, self.y, self.w, self.bias, ids, teacher, self.stats, self.picked, dloss,
                                    self.dy, self.dw, self.dbias)
        else:
            H.hapi_xent_forward(self.head, self.y, self.w, self.bias, ids, self.loss, self.stats)
            H.hapi_xent_backward(self.head, self.y, self.w, self.bias, ids, self.loss, self.stats, dloss, self.dy, self.dw,
                                 self.dbias)
        H.hapi_layernorm_backward(self.norm, self.dy, x, self.gamma, self.mean, self.rstd, self.dx, self.dgamma, self.dbeta)

    def results(self):
        return [t.clone() for t in (self.loss, self.dx, self.dgamma, self.dbeta, self.dw, self.dbias)]


def test_tail_on_extracted_features():
    """A transformer's features to its second block, then one training step of a
    tail on the class tokens (rows a whole token table apart), against the same
    step by autograd in 64 bits.  The bf16 roundings between the operators (y, dz,
    dy, and the gradients' own: each 2^-8 / sqrt 3 of its tensor's length at most)
    add up to 4 such in the gradients behind all of them; 2^-8 * 4 leaves room for
    what the logits' shift by y's rounding does (2^-8 of a logit of spread 1)."""
    layers = PM.vit(image=64, patch=16, dim=128, heads=2, mlp=256, depth=2)
    d = H.Desc(layers, H.HAPI_BF16, (3, 64, 64), stream=torch.cuda.current_stream(), direct=1)
    g = _gen(30)
    raw = _randn(g, H.hapi_raw_weight_count(d)) * 0.05
    packed = torch.zeros(H.hapi_packed_weight_bytes(d), dtype=torch.uint8, device="cuda")
    H.hapi_pack_weights(d, raw, packed)
    batch, split, classes = 48, 4, 90
    images = _randn(g, batch, 3, 64, 64).to(BF)
    need = H.hapi_workspace_bytes(d, batch, split)
    d.set(workspace=torch.empty(need, dtype=torch.uint8, device="cuda"), workspace_bytes=need)
    tokens, dim = H.hapi_layer_shape(d, split)
    feats = torch.empty(batch, tokens, dim, dtype=BF, device="cuda")
    H.hapi_extract(d, packed, images, batch, split, feats)
    x = feats[:, 0]
    tail = Tail(batch, dim, classes, BF, 31, stride=tokens * dim)
    ids = torch.randint(0, classes, (batch,), generator=g, device="cuda")
    dloss = torch.full((batch,), 1.0 / batch, device="cuda")
    tail.step(x, ids, dloss)
    torch.cuda.synchronize()
    leaves = [t.double().requires_grad_() for t in (x, tail.gamma, tail.beta, tail.w, tail.bias)]
    xd, ga, be, w, b = leaves
    c = xd - xd.mean(1, keepdim=True)
    y = c / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-6) * ga + be
    z = y @ w.t() + b
    loss = torch.logsumexp(z, 1) - z.gather(1, ids[:, None])[:, 0]
    (loss * dloss.double()).sum().backward()
    loss = loss.detach()
    want = [loss, xd.grad, ga.grad, be.grad, w.grad, b.grad]
    for name, a, e in zip(("loss", "dx", "dgamma", "dbeta", "dw", "db"), tail.results(), want):
        rel = float((a.double() - e).norm() / e.norm())
        assert rel <= 4 * 2.0 ** -8, (name, rel)


@pytest.mark.parametrize("top", [0, 4])
def test_step_captured_and_replayed(top):
    """The whole step as a HIP graph, replayed with other data between the
    replays, eager work and synchronisation in between: each replay equals the
    eager step."""
    rows, dim, classes = 130, 136, 700
    tail = Tail(rows, dim, classes, BF, 40, top=top)
    g = _gen(41)
    def data():
        x = _randn(g, rows, dim).to(BF)
        ids = torch.randint(0, classes, (rows, top) if top else (rows,), generator=g, device="cuda")
        return x, ids, torch.rand(rows, generator=g, device="cuda"), _randn(g, rows, top) if top else None
    sets = [data() for _ in range(4)]
    eager = []
    for s in sets:
        tail.step(s[0], s[1], s[2], s[3])
        torch.cuda.synchronize()
        eager.append(tail.results())
    held = [t.clone() if t is not None else None for t in sets[0]]
    stream = torch.cuda.Stream()
    tail.norm.set(stream=stream)
    tail.head.set(stream=stream)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        tail.step(*held)
    for k in (1, 0, 3, 2, 2):
        for h, v in zip(held, sets[k]):
            if h is not None:
                h.copy_(v)
        for t in (tail.dx, tail.dw, tail.dbias, tail.loss):
            t.fill_(9.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(tail.results(), eager[k]):
            assert torch.equal(a, b)

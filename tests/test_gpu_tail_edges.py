"""The trained tail at the edges of what its header allows: no rows with real
addresses, entries without weight, counting rows that begin late, more tiles and rows
than one launch takes, the ends of the temperatures."""
import math

import pytest
import torch

import paper_2210_08650_amd as H
from tests import tail_reference as R
from tests.test_gpu_tail import BF, CODE, F32, _gen, _head_case, _head_check, _head_run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("top", [0, 3])
def test_no_rows_with_addresses(top, dtype):
    """Every pointer of an empty batch given, the workspace full of NaN patterns: the
    weights' gradients are zeros."""
    dim, classes = 64, 300
    w = torch.ones(classes, dim, dtype=dtype, device="cuda")
    bias = torch.ones(classes, device="cuda")
    some = torch.full((4096,), math.nan, device="cuda")
    p = some.data_ptr()
    d = H.Head(CODE[dtype], 0, dim, classes, top=top, temperature=2.0 if top else 1.0,
               stream=torch.cuda.current_stream())
    need = H.hapi_head_workspace_bytes(d, True)
    d.set(workspace=torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda"), workspace_bytes=need)
    dw, db = torch.full_like(w, 5.0), torch.full_like(bias, 5.0)
    if top:
        H.hapi_distill_backward(d, p, w, bias, p, p, p, p, p, p, dw, db)
    else:
        H.hapi_xent_backward(d, p, w, bias, p, p, p, p, p, dw, db)
    torch.cuda.synchronize()
    assert bool((dw == 0).all()) and bool((db == 0).all())
    assert bool(torch.isnan(some).all()), "wrote to a row that is not there"


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [20, 150])
@pytest.mark.parametrize("pad", [-1, 5, 200, 2 ** 40])
def test_entries_without_weight_may_name_anything(pad, rows, dtype):
    """A teacher's logit of -inf is no entry, whatever id stands beside it: the results
    are those of the id -1.  A row of nothing else does not count."""
    c = _head_case(61, rows, 72, 200, dtype, top=4)
    out = torch.rand(rows, 4, generator=_gen(62), device="cuda") < 0.3
    out[3] = True
    c["teacher"][out] = -math.inf
    c["ids"] = c["ids"].masked_fill(out, -1)
    want = {k: v.clone() for k, v in _head_run(c).items()}
    c["ids"] = c["ids"].masked_fill(out, pad)
    got = _head_run(c)
    for name in ("loss", "stats", "dx", "dw", "db"):
        assert torch.equal(got[name], want[name]), name
    assert float(got["loss"][3]) == 0 and bool((got["dx"][3] == 0).all())
    # picked holds a logit wherever the id is a class
    assert torch.equal(got["picked"][~out], want["picked"][~out])
    if not 0 <= pad < 200:
        assert bool((got["picked"][out] == 0).all())


@pytest.mark.parametrize("rows,classes,first,top", [
    (300, 5003, 64, 0), (700, 33000, 64, 0), (700, 33000, 650, 0), (5000, 700, 4700, 0), (70001, 200, 69000, 0),
    (300, 5003, 0, 2), (300, 5003, 65, 2), (5000, 700, 4700, 2), (300, 600, 290, 1024)])
def test_a_mean_keeps_its_targets_whole_wherever_it_begins(rows, classes, first, top):
    """The rows that count begin behind `first` others (a masked prompt, padding in
    front), and a teacher's one entry is the last of its row.  1 / 4080 has a
    significand of 1.0039, half a step of 16 bits from either neighbour: were dloss
    rounded, every target's entry and so the whole gradient would be off by 2^-8.
    The bound is the gradients' own rounding, 2^-8 / sqrt 3 of their length at most,
    and a tenth for the small entries' (p, of a 16-bit step of its own)."""
    c = _head_case(70, rows, 96, classes, BF, bias=False, spread=1.0)
    ids = c["ids"].clamp(min=0)
    ids[:first] = -1
    c["dloss"].fill_(1.0 / 4080)
    c["dloss"][:first] = 0.7
    c["ids"] = ids
    want = R.head(c["x"], c["w"], None, ids, None, 1.0, c["dloss"])
    if top:
        c["ids"] = torch.full((rows, top), -1, device="cuda")
        c["ids"][:, -1] = ids
        c["teacher"] = torch.zeros(rows, top, device="cuda")
    got = _head_run(c)
    for name in ("dx", "dw"):
        R.check(name, got[name], want[name], 1.1 * 2.0 ** -8 / math.sqrt(3))


def test_more_tiles_than_a_launch_takes():
    """512 x 16,385 tiles of 512 threads, 2^32 threads and more: two launches of the
    forward product.  Eight rows over and over, each as the eight alone."""
    rows, dim, classes = 131072, 16, 4194304 + 5
    d = H.Head(H.HAPI_BF16, rows, dim, classes, stream=torch.cuda.current_stream())
    need = H.hapi_head_workspace_bytes(d, False)
    if torch.cuda.mem_get_info()[0] < need + (8 << 30):
        pytest.skip(f"{need} bytes of workspace")
    g = _gen(90)
    x8, w = torch.randn(8, dim, generator=g, device="cuda").to(BF), torch.randn(classes, dim, generator=g, device="cuda").to(BF)
    bias = torch.randn(classes, generator=g, device="cuda")
    ids8 = torch.tensor([0, classes - 1, -1, 255, 4194303, 4194304, 2 ** 21, 77777], device="cuda")
    x, ids = x8.repeat(rows // 8, 1), ids8.repeat(rows // 8)
    loss, stats = torch.empty(rows, device="cuda"), torch.empty(rows, 2, device="cuda")
    d.set(workspace=torch.empty(need, dtype=torch.uint8, device="cuda"), workspace_bytes=need)
    H.hapi_xent_forward(d, x, w, bias, ids, loss, stats)
    torch.cuda.synchronize()
    want = R.head(x8, w, bias, ids8)
    R.check("loss", loss.view(-1, 8), want["loss"])
    R.check("stats", stats.view(-1, 8, 2), want["stats"])
    del d
    torch.cuda.empty_cache()  # 64 GB


def test_norm_of_more_rows_than_a_launch_takes():
    """2^30 + 37 rows, 64 to a block of 256 threads, would be 2^32 threads and more.  The same
    2^20 rows over and over, each time with the same bits."""
    rows, dim, some = 2 ** 30 + 37, 2, 2 ** 20
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("24 GB of tensors")
    g = _gen(91)
    gamma, beta = torch.rand(dim, generator=g, device="cuda") + 0.5, torch.randn(dim, generator=g, device="cuda")
    few = (torch.randn(some, dim, generator=g, device="cuda") * 1.5 + 0.3).to(BF)
    x = torch.empty(rows, dim, dtype=BF, device="cuda")
    for r in range(0, rows, some):
        x[r:r + some] = few[:rows - r]
    y, mean, rstd = torch.full_like(x, 9.0), torch.full((rows,), 9.0, device="cuda"), torch.full((rows,), 9.0, device="cuda")
    H.hapi_layernorm_forward(H.Norm(H.HAPI_BF16, rows, dim, stream=torch.cuda.current_stream()), x, gamma, beta, y, mean, rstd)
    torch.cuda.synchronize()
    for name, t, w in zip(("y", "mean", "rstd"), (y, mean, rstd), R.norm_forward(few, gamma, beta, 1e-6)):
        R.check(name, t[:some], w)
    for t in (y, mean, rstd):
        for r in range(some, rows, some):
            assert torch.equal(t[r:r + some], t[:min(some, rows - r)]), r
    del x, y, mean, rstd, t
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("power", [-60, -8, 10, 60])
def test_temperatures_at_the_ends_of_their_range(power, dtype):
    c = _head_case(95, 40, 64, 300, dtype, top=3)
    c["temp"] = 2.0 ** power
    got = _head_run(c)
    want = R.head(c["x"], c["w"], c["bias"], c["ids"], c["teacher"], c["temp"], c["dloss"])
    for name, t in got.items():
        R.check(name, t, want[name])
        assert bool(torch.isfinite(t).all()), name


def test_backward_does_not_read_the_loss():
    c = _head_case(97, 70, 64, 300, BF)
    want = {k: v.clone() for k, v in _head_run(c).items()}
    d = H.Head(H.HAPI_BF16, 70, 64, 300, stream=torch.cuda.current_stream())
    need = H.hapi_head_workspace_bytes(d, True)
    d.set(workspace=torch.empty(need, dtype=torch.uint8, device="cuda"), workspace_bytes=need)
    dx, dw, db = (torch.empty_like(t) for t in (c["x"], c["w"], c["bias"]))
    H.hapi_xent_backward(d, c["x"], c["w"], c["bias"], c["ids"], torch.full((70,), math.nan, device="cuda"), want["stats"],
                         c["dloss"], dx, dw, db)
    torch.cuda.synchronize()
    assert torch.equal(dx, want["dx"]) and torch.equal(dw, want["dw"]) and torch.equal(db, want["db"])


@pytest.mark.parametrize("rows,dim,classes,top", [(2048, 72, 8192, 0), (2047, 100, 8190, 3), (4096, 1030, 4096, 0)])
def test_float32_on_the_largest_tiles(rows, dim, classes, top):
    """A whole round of 256 x 256 tiles, or nearly."""
    c = _head_case(rows + dim, rows, dim, classes, F32, bias=True, top=top)
    _head_check(c, _head_run(c))


@pytest.mark.parametrize("rows,dim,classes,top", [(2, 16, 2100001, 0), (3, 24, 1100001, 3), (5, 66000, 70, 0),
                                                  (40, 20000, 130, 2), (70001, 24, 11, 2)])
def test_far_ends_of_the_sizes_in_float32(rows, dim, classes, top):
    c = _head_case(rows + top, rows, dim, classes, F32, bias=True, top=top)
    _head_check(c, _head_run(c))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,top", [(8, 0), (8, 3), (300, 0), (300, 3)])
def test_a_bias_without_its_gradient(rows, top, dtype):
    c = _head_case(98, rows, 64, 500, dtype, top=top)
    want = {k: v.clone() for k, v in _head_run(c).items()}
    d = H.Head(CODE[dtype], rows, 64, 500, top=top, temperature=c["temp"], stream=torch.cuda.current_stream())
    need = H.hapi_head_workspace_bytes(d, True)
    d.set(workspace=torch.empty(need, dtype=torch.uint8, device="cuda"), workspace_bytes=need)
    dx, dw = torch.empty_like(c["x"]), torch.empty_like(c["w"])
    if top:
        H.hapi_distill_backward(d, c["x"], c["w"], c["bias"], c["ids"], c["teacher"], want["stats"], want["picked"],
                                c["dloss"], dx, dw, None)
    else:
        H.hapi_xent_backward(d, c["x"], c["w"], c["bias"], c["ids"], want["loss"], want["stats"], c["dloss"], dx, dw, None)
    torch.cuda.synchronize()
    assert torch.equal(dx, want["dx"]) and torch.equal(dw, want["dw"])

"""The trained tail at the edges of what its header allows: no rows with real
addresses."""
import math

import pytest
import torch

import paper_2210_08650_amd as H
from tests.test_gpu_tail import BF, CODE, F32

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

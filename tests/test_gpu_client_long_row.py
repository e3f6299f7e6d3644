"""GPU: a row of more columns than one launch of the column sums takes."""
import pytest

import paper_1601_04033_amd as fa
from helpers import gpu

pytestmark = pytest.mark.gpu


def test_parameters_gradients_of_a_row_beyond_2_28_columns():
    """One row, so each column's sum is one term, dnormed times the normed value, whose two fp32 products torch makes
    too.  rstd comes from 2^18 squares a thread, each sum rounded: within 2^-7 of itself."""
    import torch
    gpu()
    cols = 2 ** 28 + 77
    g = torch.Generator(device="cuda").manual_seed(28)
    x, dh = (torch.empty(1, cols, device="cuda", dtype=torch.float16).normal_(generator=g) for _ in range(2))
    w = torch.ones(cols, device="cuda")
    total, h, dx = (torch.empty_like(x) for _ in range(3))
    stats = torch.empty(1, 4, device="cuda")
    fa.client_residual_norm_forward(x, None, total, h, stats, w_pre=w, b_pre=w)
    assert torch.equal(total, x)
    mean_square = sum(c.double().square().sum() for c in x.view(-1).split(1 << 26)) / cols
    assert abs(stats[0, 3].double() * mean_square.sqrt() - 1) < 2.0 ** -7
    dw, db = (torch.full((cols,), 3.0, device="cuda") for _ in range(2))
    ws = torch.empty(fa.client_residual_norm_workspace_bytes(1, cols), device="cuda", dtype=torch.uint8)
    fa.client_residual_norm_backward(x, total, stats, None, dh, dx, None, dw_pre=dw, db_pre=db, w_pre=w, b_pre=w,
                                     workspace=ws)
    assert torch.equal(db, dh.view(-1).float())
    assert torch.equal(dw, dh.view(-1).float() * (total.view(-1).float() * stats[0, 3]))

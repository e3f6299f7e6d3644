"""GPU: means and inverse roots of rows whose sums fp32 holds exactly.

Rows of small integers: sums and sums of squares are integers below 2^24, so a
mean is one division, within an ulp (2^-23 of itself), and 1 / sqrt(variance +
eps) comes from a division, a sum, a root and a division.  The first two may
be off by an ulp and half an ulp, of which the root leaves half, the last two
by half an ulp each: (1 + 1/2) / 2 + 1/2 + 1/2 ulps of 2^-23 at most, 1.75
2^-23."""
import numpy as np
import pytest

import paper_1601_04033_amd as fa
from helpers import gpu

pytestmark = pytest.mark.gpu
EPS = float(np.float32(1e-5))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("rows, cols", [(20_000, 60), (20_000, 500), (20_000, 1000), (3000, 5003), (1000, 9000)])
def test_statistics_of_exact_sums(dtype, layer, rows, cols):
    import torch
    gpu()
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    top = torch.randint(1, 17, (rows, 1), device="cuda", generator=g)
    x = torch.randint(0, 1 << 20, (rows, cols), device="cuda", generator=g) % (2 * top + 1) - top
    if layer:       # as many of each sign, so that the mean is 0 and the centred values are integers too
        x[:, 1::2] = -x[:, : cols - cols % 2 : 2]
        x[:, cols - cols % 2:] = 0
    x = x.to(getattr(torch, dtype))
    w = torch.ones(cols, device="cuda")
    total, h, stats = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, 4, device="cuda")
    fa.client_residual_norm_forward(x, None, total, h, stats, w_post=w, eps=1e-5,
                                    kind=fa.NORM_LAYER if layer else fa.NORM_RMS)
    want = 1 / (x.double().square().sum(1) / cols + EPS).sqrt()
    assert not stats[:, 0].any()
    err = (stats[:, 1].double() / want - 1).abs()
    assert err.max() <= 1.75 * 2.0 ** -23, (err.max() * 2 ** 23).item()


@pytest.mark.parametrize("cols", [60, 500, 1000, 5003, 9000])
def test_means_of_exact_sums(cols):
    import torch
    gpu()
    g = torch.Generator(device="cuda").manual_seed(cols)
    x = torch.randint(-500, 501, (3000, cols), device="cuda", generator=g).float()
    stats = torch.empty(3000, 4, device="cuda")
    total = torch.empty_like(x)
    fa.client_residual_norm_forward(x, None, total, None, stats, w_post=torch.ones(cols, device="cuda"), kind=fa.NORM_LAYER)
    want = x.double().sum(1) / cols
    assert ((stats[:, 0].double() - want).abs() <= 2.0 ** -23 * want.abs()).all()

"""GPU: activations of full gates to fp32's own accuracy, whatever the activations' type.

One row without a norm before the next block: db_post of a column is dsum times
the gate's activation, an fp32 output, and the only roundings in it are the
activation's and one product's.  The exponential is within 1 ulp of fp32 and
tanh within 2, a sum and a division within half an ulp each, so an activation
is within 2 ulps (2^-22 of itself) and the product adds 2^-24."""
import numpy as np
import pytest

import client_reference as ref
import paper_1601_04033_amd as fa
from helpers import gpu
from test_gpu_client_norm import ACT

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("act", ["sigmoid", "tanh"])
@pytest.mark.parametrize("cols", [60, 200, 500, 3000, 5003, 9000])
def test_activations_are_those_of_fp32(dtype, act, cols):
    import torch
    gpu()
    dt = getattr(torch, dtype)
    g = torch.Generator().manual_seed(cols)
    gate = torch.cat([torch.linspace(-40, 40, cols // 2), torch.randn(cols - cols // 2, generator=g) * 0.3])
    gate, x = gate.to(dt).view(1, cols).cuda(), torch.randn(1, cols, generator=g).to(dt).cuda()
    dsum = torch.randn(1, cols, generator=g).to(dt).cuda()
    ones, zeros = torch.ones(cols, device="cuda"), torch.zeros(cols, device="cuda")
    opts = dict(kind=fa.NORM_RMS, w_post=ones, b_post=zeros, gate=gate, gate_act=ACT[act])
    total, dx, dg = (torch.empty_like(x) for _ in range(3))
    stats, db = torch.empty(1, 4, device="cuda"), torch.empty(cols, device="cuda")
    fa.client_residual_norm_forward(x, None, total, None, stats, **opts)
    ws = torch.empty(fa.client_residual_norm_workspace_bytes(1, cols), device="cuda", dtype=torch.uint8)
    fa.client_residual_norm_backward(x, None, stats, dsum, None, dx, None, db_post=db, dgate=dg, workspace=ws, **opts)
    want = (dsum.double().cpu().numpy() * ref.act(gate.double().cpu().numpy(), act))[0]
    got = db.double().cpu().numpy()
    assert np.all(np.abs(got - want) <= (2.0 ** -22 + 2.0 ** -24) * np.abs(want)), np.max(np.abs(got / want - 1))

"""The losses over a vocabulary of one class at as many elements of x as make the
direct way part dx and dW: beyond 2^34, where one launch of both would come near
2^32 threads."""
import math

import pytest
import torch

import paper_1601_04033_amd as fa
from vocab_ways import way

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def test_more_elements_than_one_launch_takes():
    m, d, u = 2 ** 18 + 40, 2 ** 16, 0.5
    assert way(m, d, 1, torch.bfloat16) == "direct"
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dx = (torch.empty(m, d, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    step = 8192
    for at in range(0, m, step):
        x[at:at + step].normal_(generator=g)
    w = (torch.randn(1, d, device="cuda", generator=g) / 256).bfloat16()
    target = torch.zeros(m, device="cuda", dtype=torch.int64)
    target[::7] = -1
    loss, lse, picked = (torch.full((m,), math.nan, device="cuda") for _ in range(3))
    dw = torch.full((1, d), math.nan, device="cuda")
    ws = torch.empty(max(fa.client_vocab_workspace_bytes(m, d, 1, x.dtype, backward=k) for k in (False, True)), device="cuda",
                     dtype=torch.uint8)
    fa.client_vocab_loss_forward(x, w, target, loss, lse, picked, z_loss=u, workspace=ws)
    fa.client_vocab_loss_backward(x, w, target, lse, picked, dx, dw, z_loss=u, workspace=ws)
    # One class: lse = z, loss = u z^2, dz = 2 u z.  z is off by 8 roundings' walk of its sum of magnitudes; dz is the
    # difference of 1 + 2 u z and 1, each with a few roundings more.
    W = w[0].double()
    want, tol, mag = (torch.zeros(d, device="cuda", dtype=torch.double) for _ in range(3))
    for at in range(0, m, step):
        X = x[at:at + step].double()
        used = (target[at:at + step] == 0).double()
        z = (X @ W) * used
        ez = (8 * U * math.sqrt(d + 16) * (X.abs() @ W.abs()) + 4 * U * z.abs()) * used
        assert ((lse[at:at + step] - z).abs() <= ez).all() and ((picked[at:at + step] - z).abs() <= ez).all(), at
        assert ((loss[at:at + step] - u * z * z).abs() <= (2 * z.abs() + ez) * u * ez + 16 * U * (z * z + z.abs())).all(), at
        ed = (2 * u * ez + 16 * U * (1 + z.abs())) * used
        right = 2 * u * z[:, None] * W
        off = (dx[at:at + step] - right).abs()
        assert (off <= ed[:, None] * W.abs() * 1.01 + 2.0 ** -8 * right.abs() + 1e-37).all(), at
        want += (2 * u * z) @ X
        tol += ed @ X.abs()
        mag += (2 * u * z.abs()) @ X.abs()
        del X, right, off
    assert ((dw[0] - want).abs() <= tol + 8 * U * math.sqrt(m + 16) * mag).all()

"""GPU: the client's calls marshalled natively and in Python do the same, over
the forms of argument that the native way takes; what it does not take goes
the general way, which converts or rejects it."""
import numpy as np
import pytest

import paper_1601_04033_amd as fa
from helpers import gpu
from paper_1601_04033_amd import client

pytestmark = pytest.mark.gpu


@pytest.fixture
def both(monkeypatch):
    """Runs a function with each way of marshalling and returns the two results."""
    gpu()

    def run(f):
        native = client._native()
        a = f()
        monkeypatch.setattr(client, "_calls", fa._GeneralWay())
        b = f()
        monkeypatch.setattr(client, "_calls", native)
        return a, b
    return run


def _same(pair):
    import torch
    torch.cuda.synchronize()
    a, b = pair
    assert len(a) == len(b)
    for x, y in zip(a, b):
        assert (x is None and y is None) or torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("shape, ld", [((7, 33), 40), ((64,), 64), ((1, 5), 5)])
@pytest.mark.parametrize("with_residual", [False, True])
def test_dropout(both, dtype, shape, ld, with_residual):
    import torch
    dt = getattr(torch, dtype)
    x = torch.randn(64, ld, device="cuda").to(dt)
    x = x[0, :shape[0]] if len(shape) == 1 else x[:shape[0], :shape[1]]
    res = torch.randn_like(x) if with_residual else None

    def f():
        out = torch.zeros_like(x)
        fa.client_dropout(x, out, np.float64(0.25), np.int64(5), 7, np.int32(2), site=1, residual=res, index_base=16,
                          stream=torch.cuda.current_stream())
        return [out]
    _same(both(f))


@pytest.mark.parametrize("gate", [None, "channel", "row", "full"])
@pytest.mark.parametrize("bias", [False, True])
def test_residual_norm(both, gate, bias):
    import torch
    r, c = 9, 70
    x, res, ds, dh = (torch.randn(r, c, device="cuda").to(torch.bfloat16) for _ in range(4))
    w, v, b = (torch.randn(c, device="cuda") for _ in range(3))
    g = {None: None, "channel": torch.randn(c, device="cuda"), "row": torch.randn(r, 1, device="cuda"),
         "full": torch.randn(r, c, device="cuda").to(torch.bfloat16)}[gate]
    o = dict(kind=fa.NORM_LAYER, w_post=w, w_pre=v, b_post=b if bias else None, gate=g, gate_act=fa.GATE_TANH,
             residual_scale=0.5, eps=1e-5, dropout=(0.2, 9, 1, 2, 3), index_base=8)

    def f():
        total, h, st = torch.empty_like(x), torch.empty_like(x), torch.empty(r, 4, device="cuda")
        fa.client_residual_norm_forward(x, res, total, h, st, **o)
        dx, dr = torch.empty_like(x), torch.empty_like(x)
        dw, dv, db = (torch.empty_like(w) for _ in range(3))
        dg = None if g is None else torch.empty_like(g)
        ws = torch.empty(fa.client_residual_norm_workspace_bytes(r, c), device="cuda", dtype=torch.uint8)
        fa.client_residual_norm_backward(x, total, st, ds, dh, dx, dr, dw_post=dw, db_post=db if bias else None,
                                         dgate=dg, dw_pre=dv, workspace=ws, **o)
        return [total, h, st, dx, dr, dw, dv, db if bias else None, dg]
    _same(both(f))


def test_fp8(both):
    import torch
    x, w = torch.randn(20, 300, device="cuda").to(torch.float16), torch.randn(50, 300, device="cuda")

    def f():
        a, b = fa.client_fp8_operand(20, 300, fa.FP8_E5M2), fa.client_fp8_operand(50, 300)
        bt = fa.client_fp8_operand(300, 50)
        for t in (a, b, bt):
            t.scales.zero_()
        fa.client_fp8_quantize(x, a)
        fa.client_fp8_quantize(w, b, bt, block_rows=128)
        ws = torch.empty(fa.client_fp8_workspace_bytes(20, 50, 300), device="cuda", dtype=torch.uint8)
        c, y, z = torch.ones(20, 50, device="cuda"), torch.empty(20, 50, device="cuda"), torch.empty(20, 50, device="cuda", dtype=torch.float16)
        fa.client_fp8_matmul(a, b, c, accumulate=True, workspace=ws)
        fa.client_fp8_matmul(a, b, y, accumulate=0, workspace=ws)     # not a truth value: the general way
        fa.client_fp8_linear(x, b, z, workspace=ws)
        return [a.data, b.data, bt.data, b.scales, bt.scales, c, y, z]
    _same(both(f))


def test_refusals_are_the_same(both):
    import torch
    x, w = torch.zeros(4, 8, device="cuda"), torch.zeros(8, device="cuda")
    st = torch.zeros(4, 4, device="cuda")
    op = fa.client_fp8_operand(4, 8)
    bad = [(lambda: fa.client_dropout(x, x[:2], 0.5, 1, 0, 0), ValueError),
           (lambda: fa.client_dropout(x, x.half(), 0.5, 1, 0, 0), TypeError),
           (lambda: fa.client_dropout(x.t(), x.t(), 0.5, 1, 0, 0), TypeError),
           (lambda: fa.client_dropout(x.double(), x.double(), 0.5, 1, 0, 0), TypeError),
           (lambda: fa.client_dropout(x, x, 1.5, 1, 0, 0), fa.FasgdError),
           (lambda: fa.client_dropout(x, x, 0.5, 1, -1, 0), fa.FasgdError),
           (lambda: fa.client_residual_norm_forward(x, x, x, x, st, w_post=w[:7], w_pre=w), ValueError),
           (lambda: fa.client_residual_norm_forward(x, x, x, x, st, w_post=w.half(), w_pre=w), TypeError),
           (lambda: fa.client_residual_norm_forward(x, x, x, x, st[:2], w_post=w, w_pre=w), ValueError),
           (lambda: fa.client_residual_norm_forward(x, x, x, None, st, w_post=w, w_pre=w), fa.FasgdError),
           (lambda: fa.client_residual_norm_forward(x, x, x, x, st, w_post=w, w_pre=w, gate=x[:, :3].contiguous()), ValueError),
           (lambda: fa.client_residual_norm_forward(x, x, x, x, st, w_post=w, w_pre=w, eps=-1.0), fa.FasgdError),
           (lambda: fa.client_fp8_quantize(x, None, None), fa.FasgdError),
           (lambda: fa.client_fp8_quantize(x.cpu(), op), TypeError),
           (lambda: fa.client_fp8_matmul(op, op, x), ValueError),
           (lambda: fa.client_fp8_linear(x, op, x.half()), TypeError)]
    for call, error in bad:
        def f():
            with pytest.raises(error) as e:
                call()
            return str(e.value)
        a, b = both(f)
        assert a == b
    torch.cuda.synchronize()

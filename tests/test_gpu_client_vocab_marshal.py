"""GPU: the losses over a vocabulary marshalled natively and in Python do the
same, and refuse the same."""
import numpy as np
import pytest
import torch

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


M, D, V, K = 20, 40, 90, 5


def _inputs(dtype):
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(M, D + 8, device="cuda", generator=g).to(dtype)[:, :D]
    w = torch.randn(V, D, device="cuda", generator=g).to(dtype)
    t = torch.randint(-3, V, (M,), device="cuda", generator=g)
    i = torch.randint(0, V, (M, K), device="cuda", generator=g)
    teacher = torch.randn(M, K, device="cuda", generator=g).to(dtype)
    return x, w, t, i, teacher, torch.rand(M, device="cuda", generator=g)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_the_same_results(both, dtype):
    x, w, t, i, teacher, dloss = _inputs(dtype)
    n = fa.client_vocab_workspace_bytes(M, D, V, dtype)
    top = teacher.float().logsumexp(1)

    def f():
        ws = torch.empty(n, device="cuda", dtype=torch.uint8)
        loss, lse, p = (torch.empty(M, device="cuda") for _ in range(3))
        dx, dw = torch.empty(M, D, device="cuda", dtype=dtype), torch.ones(V, D, device="cuda")
        dw2 = torch.empty(V, D, device="cuda", dtype=dtype)
        fa.client_vocab_loss_forward(x, w, t, loss, lse, p, smoothing=np.float64(0.1), z_loss=1e-3, logit_scale=0.5,
                                     workspace=ws)
        opts = dict(smoothing=0.1, z_loss=1e-3, logit_scale=0.5, workspace=ws, stream=torch.cuda.current_stream())
        fa.client_vocab_loss_backward(x, w, t, lse, p, dx, dw, dloss=dloss, grad_scale=2, accumulate=True, **opts)
        fa.client_vocab_loss_backward(x, w, t, lse, p, None, dw2, **opts)
        loss2, lse2, p2 = torch.empty(M, device="cuda"), torch.empty(M, device="cuda"), torch.empty(M, K, device="cuda")
        dx2, dw3 = torch.empty_like(dx), torch.ones_like(dw)
        fa.client_vocab_distill_forward(x, w, i, teacher, loss2, lse2, p2, teacher_scale=0.5, teacher_lse=top,
                                        workspace=ws)
        fa.client_vocab_distill_backward(x, w, i, teacher, lse2, p2, dx2, dw3, accumulate=1, teacher_scale=0.5,
                                         teacher_lse=top, workspace=ws)      # not a truth value: the general way
        return [loss, lse, p, dx, dw, dw2, loss2, lse2, p2, dx2, dw3]
    a, b = both(f)
    torch.cuda.synchronize()
    for s, u in zip(a, b):
        assert torch.equal(s, u)


def test_refusals_are_the_same(both):
    x, w, t, i, teacher, dloss = _inputs(torch.bfloat16)
    loss, lse, p = (torch.empty(M, device="cuda") for _ in range(3))
    pk = torch.empty(M, K, device="cuda")
    dx, dw = torch.empty(M, D, device="cuda", dtype=x.dtype), torch.empty(V, D, device="cuda")
    ws = torch.empty(fa.client_vocab_workspace_bytes(M, D, V, x.dtype), device="cuda", dtype=torch.uint8)
    forward = lambda **k: fa.client_vocab_loss_forward(**{**dict(x=x, w=w, targets=t, loss=loss, lse=lse, picked=p,
                                                                 workspace=ws), **k})
    backward = lambda **k: fa.client_vocab_loss_backward(**{**dict(x=x, w=w, targets=t, lse=lse, picked=p, dx=dx, dw=dw,
                                                                   workspace=ws), **k})
    distill = lambda **k: fa.client_vocab_distill_forward(**{**dict(x=x, w=w, index=i, teacher=teacher, loss=loss,
                                                                    lse=lse, picked=pk, workspace=ws), **k})
    undo = lambda **k: fa.client_vocab_distill_backward(**{**dict(x=x, w=w, index=i, teacher=teacher, lse=lse, picked=pk,
                                                                  dx=dx, dw=dw, workspace=ws), **k})
    bad = [(lambda: forward(x=x.cpu()), TypeError), (lambda: forward(w=w.float()), TypeError),
           (lambda: forward(w=w[:, :30]), ValueError), (lambda: forward(x=x[0]), ValueError),
           (lambda: forward(targets=t.int()), TypeError), (lambda: forward(targets=t[None]), ValueError),
           (lambda: forward(targets=t[:-1]), ValueError), (lambda: forward(loss=loss[:3]), ValueError),
           (lambda: forward(lse=lse.half()), TypeError), (lambda: forward(x=x.t()), TypeError),
           (lambda: forward(smoothing=1.5), fa.FasgdError), (lambda: forward(logit_scale=0.0), fa.FasgdError),
           (lambda: forward(workspace=None), fa.FasgdError), (lambda: forward(workspace=ws[:100]), fa.FasgdError),
           (lambda: forward(z_loss=float("nan")), fa.FasgdError),
           (lambda: backward(dx=dx.float()), TypeError), (lambda: backward(dx=dx[:, :8]), ValueError),
           (lambda: backward(dw=dw.half()), TypeError), (lambda: backward(dw=dw[:8]), ValueError),
           (lambda: backward(dloss=dloss[:2]), ValueError), (lambda: backward(grad_scale=float("inf")), fa.FasgdError),
           (lambda: distill(index=t), ValueError), (lambda: distill(teacher=teacher.float()), TypeError),
           (lambda: distill(teacher=teacher[:, :2]), TypeError), (lambda: distill(teacher=teacher[:, :2].contiguous()), ValueError),
           (lambda: distill(index=i[:, :0], teacher=teacher[:, :0], picked=pk[:, :0]), fa.FasgdError),
           (lambda: distill(picked=p), ValueError), (lambda: distill(teacher_lse=lse[:2]), ValueError),
           (lambda: distill(teacher_scale=-1.0), fa.FasgdError), (lambda: undo(dw=dw[0]), ValueError),
           (lambda: undo(lse=None), fa.FasgdError)]
    for at, (call, error) in enumerate(bad):
        def f():
            with pytest.raises(error) as e:
                call()
            return str(e.value)
        a, b = both(f)
        assert a == b, at
    torch.cuda.synchronize()

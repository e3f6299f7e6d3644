"""The losses over a vocabulary on the GPU against their 64-bit forms."""
import math

import pytest
import torch

import paper_1601_04033_amd as fa
from vocab_reference import Reference

pytestmark = pytest.mark.gpu
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


class Case:
    """Inputs on the GPU, from a seed; gaps: rows lie apart, NaN between them."""

    def __init__(self, dtype, m, d, V, K=0, out=0.0, gaps=0, seed=0, short=False):
        g = torch.Generator().manual_seed(seed + 7919 * m + 31 * d + V)
        self.dt = DTYPES[dtype]
        w = torch.randn(V, d, generator=g) * d ** -0.5
        target = torch.randint(0, V, (m,), generator=g)
        x = torch.randn(m, d, generator=g) + w[target] * (torch.rand(m, 1, generator=g) * 2 * math.log(V + 1))
        left = torch.rand(m, generator=g) < out
        x[left] = math.nan                      # what is left out holds anything
        self.x, self.w = self.place(x, gaps), self.place(w, gaps)
        self.dloss = (torch.rand(m, generator=g) + 0.5).cuda() / max(m, 1)
        self.teacher = None
        if K:
            index = torch.randint(0, V, (m, K), generator=g)
            index[:, 0] = target
            if short:
                index[torch.rand(m, K, generator=g) < 0.3] = -1
                index[torch.rand(m, K, generator=g) < 0.1] = V
            index[left] = -1
            self.index = index.cuda()
            self.teacher = (4 * torch.randn(m, K, generator=g)).to(self.dt).cuda()
            if short:
                self.teacher[torch.rand(m, K, generator=g).cuda() < 0.2] = -math.inf
            self.teacher_lse = torch.logsumexp(self.teacher.float(), dim=1) + 0.1
            self.teacher_lse[self.teacher_lse == -math.inf] = 0.0
        else:
            target[left] = torch.where(torch.rand(int(left.sum()), generator=g) < 0.5, -100, V)
            self.index = target.cuda()
        self.gaps = gaps

    def place(self, t, gaps):
        if not gaps:
            return t.to(self.dt).cuda()
        buf = torch.full((t.shape[0], t.shape[1] + gaps), math.nan, dtype=self.dt)
        buf[:, :t.shape[1]] = t
        return buf.cuda()[:, :t.shape[1]]


def workspace(c, backward):
    n = fa.client_vocab_workspace_bytes(*c.x.shape, c.w.shape[0], c.dt, backward=backward)
    return torch.full((n,), 0xFF, device="cuda", dtype=torch.uint8)     # NaN in every type


def forward(c, whole=False, **kw):
    m = c.x.shape[0]
    loss, lse = (torch.full((m,), math.nan, device="cuda") for _ in range(2))
    picked = torch.full(tuple(c.index.shape), math.nan, device="cuda")
    ws = workspace(c, False)
    if c.teacher is None:
        fa.client_vocab_loss_forward(c.x, c.w, c.index, loss, lse, picked, workspace=ws, **kw)
    else:
        fa.client_vocab_distill_forward(c.x, c.w, c.index, c.teacher, loss, lse, picked, workspace=ws,
                                        teacher_lse=c.teacher_lse if whole else None, **kw)
    return loss, lse, picked


def backward(c, lse, picked, whole=False, dx=True, dw=torch.float32, **kw):
    dx = torch.full_like(c.x, math.nan) if dx else None
    dw = None if dw is None else torch.full(c.w.shape, math.nan, device="cuda", dtype=dw)
    ws = workspace(c, True)
    if c.teacher is None:
        fa.client_vocab_loss_backward(c.x, c.w, c.index, lse, picked, dx, dw, dloss=c.dloss, workspace=ws, **kw)
    else:
        fa.client_vocab_distill_backward(c.x, c.w, c.index, c.teacher, lse, picked, dx, dw, dloss=c.dloss,
                                         workspace=ws, teacher_lse=c.teacher_lse if whole else None, **kw)
    return dx, dw


def reference(c, whole=False, dw=torch.float32, **kw):
    on = dict(dloss=c.dloss, dw_dtype=dw, **kw)
    if c.teacher is not None:
        on.update(teacher=c.teacher, teacher_lse=c.teacher_lse if whole else None)
    return Reference(c.x, c.w, c.index, **on)


def check(c, whole=False, dw=torch.float32, **kw):
    grad = kw.pop("grad_scale", 1.0)
    ref = reference(c, whole, dw, grad_scale=grad, **kw)
    loss, lse, picked = forward(c, whole, **kw)
    for name, got in (("loss", loss), ("lse", lse), ("picked", picked)):
        ref.check(name, got)
    dx, dw = backward(c, lse, picked, whole, dw=dw, grad_scale=grad, **kw)
    ref.check("dx", dx)
    ref.check("dw", dw)
    return loss, lse, picked, dx, dw


SIZES = [(1, 1, 1), (1, 8, 2), (3, 5, 7), (1, 128, 300), (2, 127, 129), (17, 64, 1000), (128, 1000, 10), (130, 129, 257),
         (255, 200, 511), (300, 384, 1025), (64, 1544, 2003), (16, 4096, 3000), (15, 4000, 4099), (33, 2048, 2100),
         # beyond what goes without laid out operands
         (1025, 1, 1), (1030, 5, 7), (1100, 130, 33), (1, 8200, 3), (5, 8193, 70), (130, 8320, 257), (1300, 127, 1000),
         (1100, 8, 600), (1100, 40, 600), (1111, 72, 333), (1500, 136, 1500)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m, d, V", SIZES)
def test_loss(dtype, m, d, V):
    check(Case(dtype, m, d, V))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m, d, V, K", [(1, 4, 3, 1), (5, 33, 70, 2), (70, 128, 300, 64), (129, 257, 1030, 65), (33, 64, 5, 130),
                                        (16, 4096, 3001, 64), (1030, 40, 90, 7), (1100, 128, 300, 66), (20, 8200, 130, 20)])
@pytest.mark.parametrize("whole", [False, True])
def test_distill(dtype, m, d, V, K, whole):
    """Classes stand in a row more than once; K beyond a wave; more entries than classes."""
    check(Case(dtype, m, d, V, K), whole)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["loss", "distill"])
def test_rows_left_out_and_gaps(dtype, kind):
    """NaN in the rows that are left out, between rows and in unused entries reaches nothing."""
    for m, d, V, gaps in ((200, 72, 333, 5), (14, 129, 520, 3), (1200, 136, 520, 8), (1100, 256, 300, 8), (40, 8200, 99, 1)):
        c = Case(dtype, m, d, V, 9 if kind == "distill" else 0, out=0.4, gaps=gaps, short=kind == "distill")
        loss, lse, picked, dx, dw = check(c, whole=True)
        left = ~reference(c, True).used
        assert left.any()
        for t in (loss, lse, picked, dx):
            assert (t[left] == 0).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["loss", "distill"])
def test_every_row_left_out(dtype, kind):
    for m in (7, 70, 1030):
        c = Case(dtype, m, 96, 130, 4 if kind == "distill" else 0, out=1.1)
        loss, lse, picked = forward(c)
        dx, dw = backward(c, lse, picked)
        for t in (loss, lse, picked, dx, dw):
            assert (t == 0).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m", [90, 1100])
def test_options_of_the_loss(dtype, m):
    c = Case(dtype, m, 160, 700, out=0.2)
    check(c, smoothing=0.1, z_loss=1e-3, logit_scale=0.5, grad_scale=3.0)
    check(c, smoothing=1.0)
    check(c, z_loss=0.1, dw=c.dt)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m", [90, 1100])
def test_options_of_the_distillation(dtype, m):
    c = Case(dtype, m, 160, 700, 20, out=0.2, short=True)
    check(c, False, logit_scale=0.5, teacher_scale=0.25, grad_scale=4.0, dw=c.dt)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m", [12, 60, 1100])
def test_one_gradient_alone_and_accumulation(dtype, m):
    c = Case(dtype, m, 100, 300)
    loss, lse, picked, dx, dw = check(c)
    only_x, none = backward(c, lse, picked, dw=None)
    none2, only_w = backward(c, lse, picked, dx=False)
    assert torch.equal(only_x, dx) and torch.equal(only_w, dw) and none is None and none2 is None
    twice = dw.clone()
    fa.client_vocab_loss_backward(c.x, c.w, c.index, lse, picked, None, twice, dloss=c.dloss, accumulate=True,
                                  workspace=workspace(c, True))
    assert torch.equal(twice, dw + dw)


@pytest.mark.parametrize("dtype", DTYPES)
def test_tiles_that_fill_the_chip(dtype):
    """Blocks of 256 x 256, with ragged edges; the sums repeat bit for bit."""
    c = Case(dtype, 3333, 320, 4001, out=0.1)
    a, b = check(c, smoothing=0.05), check(c, smoothing=0.05)
    for s, t in zip(a, b):
        assert torch.equal(s, t)
    check(Case(dtype, 2600, 4100, 300))


@pytest.mark.parametrize("dtype, V", [("bf16", 540_001), ("fp16", 540_001), ("fp32", 250_003)])
def test_several_pieces_of_the_vocabulary(dtype, V):
    check(Case(dtype, 40, 64, V, out=0.1))
    check(Case(dtype, 20, 64, V, 50))


def test_no_rows():
    x = torch.empty(0, 16, device="cuda")
    w = torch.randn(20, 16, device="cuda")
    e = torch.empty(0, device="cuda")
    i = torch.empty(0, device="cuda", dtype=torch.int64)
    fa.client_vocab_loss_forward(x, w, i, e, e, e)
    dw = torch.full((20, 16), math.nan, device="cuda")
    fa.client_vocab_loss_backward(x, w, i, e, e, x.clone(), dw)
    assert (dw == 0).all()
    dw.fill_(2.0)
    fa.client_vocab_loss_backward(x, w, i, e, e, None, dw, accumulate=True)
    assert (dw == 2).all()


@pytest.mark.parametrize("kind", ["loss", "distill"])
def test_gradient_is_the_loss_s_slope(kind):
    """dx and dw against differences of the loss along random directions, in fp32: the loss is computed to about
    2^-20 of its size, the difference's curvature is of the step's square."""
    c = Case("fp32", 24, 32, 50, 6 if kind == "distill" else 0)
    kw = dict(smoothing=0.1, z_loss=1e-2) if kind == "loss" else {}
    _, lse, picked = forward(c, **kw)
    dx, dw = backward(c, lse, picked, **kw)
    g = torch.Generator(device="cuda").manual_seed(5)
    for name, at, grad in (("x", c.x, dx), ("w", c.w, dw)):
        way = torch.randn(at.shape, device="cuda", generator=g)
        way /= way.norm()
        h = 0.05
        value = []
        for sign in (1, -1):
            setattr(c, name, at + sign * h * way)
            value.append((forward(c, **kw)[0].double() * c.dloss.double()).sum())
        setattr(c, name, at)
        slope, want = (value[0] - value[1]) / (2 * h), (grad.double() * way.double()).sum()
        # third derivatives along a unit direction are below the cube of the other factor's norm per row
        other = (c.w if name == "x" else c.x).double()
        third = other.norm(dim=1).max() ** 3 if name == "x" else (other.norm(dim=1) ** 3 * c.dloss.double()).sum()
        bound = third * c.dloss.double().sum() * h * h / 6 if name == "x" else third * h * h / 6
        assert abs(slope - want) <= bound + 2.0 ** -18 * abs(value[0]) / h, (float(slope), float(want), float(bound))


@pytest.mark.parametrize("m", [100, 1100])
def test_on_another_stream_and_captured(m):
    c = Case("bf16", m, 256, 900, out=0.2)
    want = check(c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        loss, lse, picked = forward(c)
        got = (loss, lse, picked, *backward(c, lse, picked))
    side.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    out = [torch.empty_like(t) for t in want]
    wf, wb = workspace(c, False), workspace(c, True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fa.client_vocab_loss_forward(c.x, c.w, c.index, out[0], out[1], out[2], workspace=wf)
        fa.client_vocab_loss_backward(c.x, c.w, c.index, out[1], out[2], out[3], out[4], dloss=c.dloss, workspace=wb)
    for k in range(3):
        if k == 1:      # other data in the same buffers
            c.x.copy_(c.x.flip(0) * 0.5)
            c.index.copy_(c.index.flip(0))      # what is left out holds NaN: it goes along
            want = check(c)
        for t in (*out, wf, wb):
            t.fill_(255 if t.dtype == torch.uint8 else math.nan)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, out):
            assert torch.equal(a, b)

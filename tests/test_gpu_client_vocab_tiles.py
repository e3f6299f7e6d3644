"""The losses over a vocabulary where operands are laid out and go through tiles,
in every type: each case says that it goes that way."""
import math

import pytest
import torch

import paper_1601_04033_amd as fa
from test_gpu_client_vocab import DTYPES, Case, backward, check, forward, reference, workspace
from vocab_ways import way

pytestmark = pytest.mark.gpu


def tiled(dtype, m, d, V, K=0, **kw):
    assert way(m, d, V, DTYPES[dtype]) == "tiles"
    return Case(dtype, m, d, V, K, **kw)


# in order: ordinary; odd; widths beyond a piece of the contraction; few rows against many classes; more rows than
# dW's third term is taken for; one column; many rows of few classes; four classes, one class
SIZES = [(1500, 256, 5000), (1100, 385, 4099), (500, 1001, 8209), (130, 2000, 30_011), (66, 70, 262_147), (4200, 33, 4099),
         (16_800, 1, 1000), (70_001, 9, 300), (524_301, 4, 4), (524_289, 3, 1)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m, d, V", SIZES)
def test_loss(dtype, m, d, V):
    check(tiled(dtype, m, d, V), smoothing=0.1, z_loss=1e-3)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m, d, V, K", [(1500, 256, 5000, 1), (1100, 385, 4099, 7), (500, 1001, 8209, 66), (66, 70, 262_147, 130),
                                        (4200, 33, 4099, 64), (16_800, 1, 1000, 2), (524_301, 4, 4, 2)])
@pytest.mark.parametrize("whole", [False, True])
def test_distill(dtype, m, d, V, K, whole):
    check(tiled(dtype, m, d, V, K), whole)


@pytest.mark.parametrize("dtype", DTYPES)
def test_many_entries(dtype):
    """Classes many times in a row; more entries than classes."""
    check(tiled(dtype, 1100, 385, 4099, 1024, out=0.1, short=True))
    check(tiled(dtype, 70_001, 9, 300, 400))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("K", [0, 9])
@pytest.mark.parametrize("m, d, V, gaps", [(1500, 257, 5000, 5), (1500, 256, 5000, 8), (1100, 392, 4099, 3)])
def test_rows_left_out_and_gaps(dtype, K, m, d, V, gaps):
    """NaN in the rows that are left out, between rows and in unused entries reaches nothing, and what lies between the
    rows of the gradients stays."""
    c = tiled(dtype, m, d, V, K, out=0.4, gaps=gaps, short=K > 0)
    loss, lse, picked, dx, dw = check(c, whole=True)
    left = ~reference(c, True).used
    assert left.any()
    for t in (loss, lse, picked, dx):
        assert (t[left] == 0).all()
    wide = [torch.full((n + 1, d + 3), 7.0, device="cuda", dtype=t) for n, t in ((m, c.dt), (V, torch.float32))]
    into = [t[:-1, 1:d + 1] for t in wide]      # at no alignment but the type's
    kw = dict(dloss=c.dloss, workspace=workspace(c, True))
    if K:
        fa.client_vocab_distill_backward(c.x, c.w, c.index, c.teacher, lse, picked, *into, teacher_lse=c.teacher_lse, **kw)
    else:
        fa.client_vocab_loss_backward(c.x, c.w, c.index, lse, picked, *into, **kw)
    assert torch.equal(into[0], dx) and torch.equal(into[1], dw)
    for t in wide:
        t[:-1, 1:d + 1] = 7.0
        assert (t == 7).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_operands_at_no_alignment(dtype):
    """x and w begin one element into what they lie in."""
    c = tiled(dtype, 1500, 256, 5000)
    want = check(c)
    for name in ("x", "w"):
        t = getattr(c, name)
        buf = torch.full((t.numel() + 1,), math.nan, device="cuda", dtype=c.dt)
        buf[1:] = t.flatten()
        setattr(c, name, buf[1:].view(t.shape))
    loss, lse, picked = forward(c)
    for a, b in zip(want, (loss, lse, picked, *backward(c, lse, picked))):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("K", [0, 4])
def test_every_row_left_out(dtype, K):
    c = tiled(dtype, 1500, 256, 5000, K, out=1.1)
    loss, lse, picked = forward(c)
    dx, dw = backward(c, lse, picked)
    for t in (loss, lse, picked, dx, dw):
        assert (t == 0).all()
    before = torch.randn(c.w.shape, device="cuda")
    dw = before.clone()
    if not K:
        fa.client_vocab_loss_backward(c.x, c.w, c.index, lse, picked, None, dw, accumulate=True, workspace=workspace(c, True))
        assert torch.equal(dw, before)


@pytest.mark.parametrize("dtype", DTYPES)
def test_one_row_takes_part(dtype):
    for K in (0, 5):
        c = tiled(dtype, 1500, 256, 5000, K)
        c.index[:1234] = -1
        c.index[1235:] = -1
        c.x[:1234] = math.nan
        check(c)


@pytest.mark.parametrize("dtype", DTYPES)
def test_options(dtype):
    c = tiled(dtype, 1500, 160, 7000, out=0.2)
    check(c, smoothing=0.1, z_loss=1e-3, logit_scale=0.5, grad_scale=3.0)
    check(c, smoothing=1.0)
    check(c, z_loss=0.1, dw=c.dt)
    c = tiled(dtype, 1500, 160, 7000, 20, out=0.2, short=True)
    check(c, False, logit_scale=0.5, teacher_scale=0.25, grad_scale=4.0, dw=c.dt)
    check(c, True, dw=c.dt)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("K", [0, 3])
@pytest.mark.parametrize("dw_like_x", [False, True])
def test_one_gradient_alone_and_accumulation(dtype, K, dw_like_x):
    c = tiled(dtype, 1500, 257, 5000, K, out=0.1)
    kind = c.dt if dw_like_x else torch.float32
    loss, lse, picked, dx, dw = check(c, dw=kind)
    only_x, _ = backward(c, lse, picked, dw=None)
    _, only_w = backward(c, lse, picked, dx=False, dw=kind)
    assert torch.equal(only_x, dx) and torch.equal(only_w, dw)
    # added in fp32, with one rounding to dw's type: that of the sum, and that of the gradient alone in `dw`
    before = torch.randn(c.w.shape, device="cuda").to(kind)
    more = before.clone()
    kw = dict(dloss=c.dloss, accumulate=True, workspace=workspace(c, True))
    if K:
        fa.client_vocab_distill_backward(c.x, c.w, c.index, c.teacher, lse, picked, None, more, **kw)
    else:
        fa.client_vocab_loss_backward(c.x, c.w, c.index, lse, picked, None, more, **kw)
    half = torch.finfo(kind).eps / 2
    off = (more.double() - before.double() - dw.double()).abs()
    smallest = 2.0 ** -25 if kind == torch.float16 else 0.0
    assert (off <= 1.01 * half * (more.double().abs() + dw.double().abs()) + 2.0 ** -23 * before.double().abs() + 2 * smallest).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("K", [0, 5])
def test_logits_far_apart(dtype, K):
    """Probabilities that are 0 and 1."""
    c = tiled(dtype, 1500, 256, 5000, K, seed=4)
    check(c, logit_scale=100.0 if dtype != "fp16" else 10.0)
    check(c, logit_scale=1e-6)


@pytest.mark.parametrize("dtype, m, V", [("bf16", 40, 540_001), ("fp16", 40, 540_001), ("fp32", 70, 250_003)])
def test_several_pieces_of_the_vocabulary(dtype, m, V):
    check(tiled(dtype, m, 64, V, out=0.1))
    check(tiled(dtype, m, 64, V, 50, out=0.1))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("K", [0, 6])
def test_on_another_stream_and_captured(dtype, K):
    c = tiled(dtype, 1500, 256, 5000, K, out=0.2)
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
        if K:
            fa.client_vocab_distill_forward(c.x, c.w, c.index, c.teacher, *out[:3], workspace=wf)
            fa.client_vocab_distill_backward(c.x, c.w, c.index, c.teacher, *out[1:], dloss=c.dloss, workspace=wb)
        else:
            fa.client_vocab_loss_forward(c.x, c.w, c.index, *out[:3], workspace=wf)
            fa.client_vocab_loss_backward(c.x, c.w, c.index, *out[1:], dloss=c.dloss, workspace=wb)
    for k in range(3):
        if k == 1:      # other data in the same buffers, another number of rows that take part
            c.x.copy_(c.x.flip(0) * 0.5)
            c.index.copy_(c.index.flip(0))      # what is left out holds NaN: it goes along
            c.index[100:300] = -1
            want = check(c)
        for t in (*out, wf, wb):
            t.fill_(255 if t.dtype == torch.uint8 else math.nan)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, out):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype, m", [("fp32", 1100), ("bf16", 1100), ("fp16", 1100), ("bf16", 4100), ("fp16", 4100)])
def test_bits_of_a_weight_gradient(dtype, m):
    """dw in fp32 holds dz to what include/fasgd_client.h says.  With w of zeros and a given lse of 0, p is 1 and dz is
    dloss but at the targets; rows of x that are units make dw that dz, as it was held."""
    d, V = m, 4099
    assert way(m, d, V, DTYPES[dtype]) == "tiles"
    g = torch.Generator().manual_seed(m)
    dt = DTYPES[dtype]
    x, w = torch.eye(m, device="cuda", dtype=dt), torch.zeros(V, d, device="cuda", dtype=dt)
    target = torch.full((m,), V - 1, device="cuda")
    dloss = (0.5 + torch.rand(m, generator=g)).cuda()
    zero, dw = torch.zeros(m, device="cuda"), torch.full((V, d), math.nan, device="cuda")
    ws = torch.empty(fa.client_vocab_workspace_bytes(m, d, V, dt), device="cuda", dtype=torch.uint8)
    fa.client_vocab_loss_backward(x, w, target, zero, zero, None, dw, dloss=dloss, workspace=ws)
    assert (dw[-1] == 0).all()                  # p - 1
    want = dloss.expand(V - 1, m)
    if dtype == "fp32" or (dtype == "bf16" and m < 4096):       # three bf16 terms: all of its 24 bits
        assert torch.equal(dw[:-1], want)
    else:                                       # two terms, each rounding off half a step of what was left
        half = torch.finfo(dt).eps / 2
        assert ((dw[:-1] - want).abs() <= half * half * want).all()


@pytest.mark.parametrize("m", [4096, 8200])
def test_all_bits_of_a_weight_gradient_of_many_rows(m):
    """bf16: as above, dz has its 24 bits in dw however many rows there are."""
    d, V, part = m, 1030, 64
    assert way(m, d, V, torch.bfloat16) == "tiles"
    x, w = torch.eye(m, device="cuda", dtype=torch.bfloat16), torch.zeros(V, d, device="cuda", dtype=torch.bfloat16)
    dloss = (0.5 + torch.rand(m, generator=torch.Generator().manual_seed(m))).cuda()
    zero, dw = torch.zeros(m, device="cuda"), torch.full((V, d), math.nan, device="cuda")
    ws = torch.empty(fa.client_vocab_workspace_bytes(m, d, V, w.dtype), device="cuda", dtype=torch.uint8)
    target = torch.arange(m, device="cuda") % part
    fa.client_vocab_loss_backward(x, w, target, zero, zero, None, dw, dloss=dloss, workspace=ws)
    want = dloss.repeat(V, 1)
    want[target, torch.arange(m, device="cuda")] = 0.0      # p - 1
    assert torch.equal(dw, want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("K", [0, 1])
@pytest.mark.parametrize("m, V, form", [(48, 100, "direct"), (1100, 4099, "tiles")])
def test_probabilities_of_a_given_log_sum_exp(dtype, K, m, V, form):
    """With w of zeros p is exp(-lse), whose exponent in powers of two is not a number of 24 bits.  The power is off by a
    step, 2 u, its factor and their product by u each and what the factor takes up by as much (u = 2^-24); fp16 holds
    dz in 22 bits."""
    d, dt, u = m, DTYPES[dtype], 2.0 ** -24
    assert way(m, d, V, dt) == form
    lse = (11.2 + 10.0 * torch.rand(m, generator=torch.Generator().manual_seed(2))).cuda()
    x, w = torch.eye(m, device="cuda", dtype=dt), torch.zeros(V, d, device="cuda", dtype=dt)
    target, zero = torch.full((m,), V - 1, device="cuda"), torch.zeros(m, device="cuda")
    dw = torch.full((V, d), math.nan, device="cuda")
    kw = dict(grad_scale=2.0 ** 10, workspace=torch.empty(fa.client_vocab_workspace_bytes(m, d, V, dt), device="cuda", dtype=torch.uint8))
    if K:
        fa.client_vocab_distill_backward(x, w, target[:, None], torch.zeros(m, 1, device="cuda", dtype=dt), lse, zero[:, None],
                                         None, dw, **kw)
    else:
        fa.client_vocab_loss_backward(x, w, target, lse, zero, None, dw, **kw)
    want = 2.0 ** 10 * torch.exp(-lse.double())
    held = (2.0 ** -22 if form == "tiles" else 0.0) * want + 2.0 ** -28 if dtype == "fp16" else u * want
    assert ((dw[:-1] - want).abs() <= 5 * u * want + held).all()

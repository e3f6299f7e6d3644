"""The vocabulary's losses as a client uses them: behind the residual norm, into
the gradient that is pushed, eagerly and replayed; from a teacher's largest
logits; two calls at once; and sizes and entries at their ends."""
import math

import pytest
import torch

import paper_1601_04033_amd as fa
from test_gpu_client_vocab import DTYPES, Case, backward, check, forward
from vocab_reference import Reference

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


class Client:
    """normed = w_pre norm(h), logits = normed head^T, all fp32: the step between a fetch and a push."""

    def __init__(self, m, d, V, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.m, self.d, self.V = m, d, V
        self.theta = torch.randn(d + V * d, device="cuda", generator=g) * d ** -0.5
        self.theta[:d] = 1.0
        self.h = torch.randn(m, d, device="cuda", generator=g)
        self.targets = torch.randint(0, V, (m,), device="cuda", generator=g)
        self.targets[::5] = -1
        self.grad = torch.full_like(self.theta, math.nan)
        new = lambda *s: torch.full(s, math.nan, device="cuda")
        self.sum, self.normed, self.dnormed, self.dh = (new(m, d) for _ in range(4))
        self.stats, self.loss, self.lse, self.picked = new(m, 4), new(m), new(m), new(m)
        self.ws = torch.empty(max(fa.client_vocab_workspace_bytes(m, d, V, torch.float32),
                                  fa.client_vocab_workspace_bytes(m, d, V, torch.float32, backward=False),
                                  fa.client_residual_norm_workspace_bytes(m, d)), device="cuda", dtype=torch.uint8)

    def parts(self, flat):
        return flat[:self.d], flat[self.d:].view(self.V, self.d)

    def step(self, stream=None):
        w_pre, head = self.parts(self.theta)
        dw_pre, dhead = self.parts(self.grad)
        fa.client_residual_norm_forward(self.h, None, self.sum, self.normed, self.stats, w_pre=w_pre)
        on = dict(smoothing=0.1, z_loss=1e-3, workspace=self.ws)
        fa.client_vocab_loss_forward(self.normed, head, self.targets, self.loss, self.lse, self.picked, **on)
        fa.client_vocab_loss_backward(self.normed, head, self.targets, self.lse, self.picked, self.dnormed, dhead,
                                      grad_scale=1.0 / self.m, **on)
        fa.client_residual_norm_backward(self.h, self.sum, self.stats, None, self.dnormed, self.dh, None, dw_pre=dw_pre,
                                         w_pre=w_pre, workspace=self.ws)

    def expected(self):
        """The loss and the gradient in 64 bits, by torch's own differentiation, and what the gradient is a sum of, in
        magnitudes."""
        theta = self.theta.double().requires_grad_()
        w_pre, head = self.parts(theta)
        unit = (self.normed / self.theta[:self.d]).double()     # the norm's own output for weights of one
        normed = unit * w_pre
        z = normed @ head.t()
        logp = torch.log_softmax(z, dim=1)
        used = (self.targets >= 0) & (self.targets < self.V)
        t = torch.where(used, self.targets, 0)
        lse = torch.logsumexp(z, dim=1)
        rows = -0.9 * logp.gather(1, t[:, None])[:, 0] - 0.1 * logp.mean(dim=1) + 1e-3 * lse * lse
        loss = torch.where(used, rows, 0.0)
        (loss.sum() / self.m).backward()
        with torch.no_grad():
            mag = normed.abs() @ head.abs().t()
            dz = logp.exp() * (1.0 + 2e-3 * lse[:, None].abs()) + 0.1 / self.V
            dz = (dz.scatter_add(1, t[:, None], torch.full_like(dz[:, :1], 0.9)) * used[:, None]) / self.m
            behind = torch.cat([((dz @ head.abs()) * unit.abs()).sum(dim=0), (dz.t() @ normed.abs()).flatten()])
        return loss.detach(), theta.grad, behind, float(mag.max())


# laid out operands; direct
@pytest.mark.parametrize("m, d, V", [(1100, 200, 1031), (96, 200, 1031), (1, 200, 1031)])
def test_a_client_s_step(m, d, V):
    c = Client(m, d, V, 11 + m)
    if m == 1:
        c.targets[0] = 7
    c.step()
    loss, grad, behind, mag = c.expected()
    # A logit is off by at most 8 u sqrt(d + 16) of its magnitudes and 4 u of them for its terms; the log-sum-exp by
    # that and 8 u of itself and 2 u sqrt(V) for its sum; a probability by both, relative to it.  The products' sums
    # add 8 u sqrt(V + 16) or 8 u sqrt(m + 16) of their magnitudes, their terms 4 u and the norm's backward as much.
    lse = float(c.lse.abs().max())
    off = 2 * (8 * math.sqrt(d + 16) + 4) * U * mag + (16 * lse + 2 * math.sqrt(V) + 16) * U
    assert (c.loss - loss).abs().max() <= off * (2 + 2e-3 * lse) + 8 * U * loss.abs().max()
    assert ((c.grad - grad).abs() <= (off + (8 * math.sqrt(max(m, V) + 16) + 16) * 2 * U) * behind).all()

    # replayed, with pushes and fetches between: as eagerly
    theta, n, b, v, last_T = fa.allocate_state(c.theta.numel(), "cuda")
    theta.copy_(c.theta)
    state = fa.fasgd_init_state(theta, n, b, v, last_T, lam=1, alpha=0.01)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        c.step()
    torch.cuda.current_stream().wait_stream(stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.step()
    for _ in range(3):
        c.grad.fill_(math.nan)
        graph.replay()
        replayed, losses = c.grad.clone(), c.loss.clone()
        c.grad.fill_(math.nan)
        c.step()
        assert torch.equal(c.grad, replayed) and torch.equal(c.loss, losses)
        fa.fasgd_apply_updates(state, [c.grad], clients=[0], grad_ts=[state.T])
        assert not torch.equal(theta, c.theta) and torch.isfinite(theta).all()
        c.theta.copy_(theta)


def test_a_student_takes_after_its_teacher():
    """The teacher's largest logits by its own weights, the student's gradient at the teacher's weights: with all
    classes among the entries the divergence and its gradient vanish there."""
    m, d, V = 40, 64, 90
    g = torch.Generator(device="cuda").manual_seed(3)
    x, w = torch.randn(m, d, device="cuda", generator=g), torch.randn(V, d, device="cuda", generator=g) * d ** -0.5
    z = (x.double() @ w.double().t()).float()
    teacher, index = z.topk(V, dim=1)
    loss, lse, picked = torch.empty(m, device="cuda"), torch.empty(m, device="cuda"), torch.empty(m, V, device="cuda")
    ws = torch.empty(fa.client_vocab_workspace_bytes(m, d, V, x.dtype), device="cuda", dtype=torch.uint8)
    fa.client_vocab_distill_forward(x, w, index, teacher, loss, lse, picked, workspace=ws)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    fa.client_vocab_distill_backward(x, w, index, teacher, lse, picked, dx, dw, workspace=ws)
    off = float((8 * math.sqrt(d + 16) + 24) * U * (x.abs() @ w.abs().t()).max()) + 64 * U      # of a logit, and lse
    assert loss.abs().max() <= 4 * off
    assert dx.abs().max() <= 4 * off * w.abs().max() * 2 and dw.abs().max() <= 4 * off * x.abs().max() * m
    # a gradient step from other weights brings the student nearer
    other = w + 0.1 * torch.randn(V, d, device="cuda", generator=g)
    fa.client_vocab_distill_forward(x, other, index, teacher, loss, lse, picked, workspace=ws)
    fa.client_vocab_distill_backward(x, other, index, teacher, lse, picked, None, dw, grad_scale=1.0 / m, workspace=ws)
    before = loss.mean().item()
    fa.client_vocab_distill_forward(x, other - 0.01 * dw, index, teacher, loss, lse, picked, workspace=ws)
    slope = 0.01 * (dw.double() ** 2).sum().item()
    assert abs(before - loss.mean().item() - slope) <= 0.5 * slope


def test_two_calls_at_once():
    a, b = Case("bf16", 1500, 256, 5000, seed=1), Case("bf16", 700, 256, 3001, K=7, seed=2)
    want = [(*f, *backward(c, f[1], f[2])) for c, f in ((a, forward(a)), (b, forward(b)))]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = []
        for c, s in zip((a, b), streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                f = forward(c)
                got.append((*f, *backward(c, f[1], f[2])))
        torch.cuda.synchronize()
        for w, h in zip(want, got):
            assert all(torch.equal(p, q) for p, q in zip(w, h))


# a class many times in a row, more entries than classes, more than a block holds
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m, d, V, K", [(16, 64, 50, 1024), (1, 8, 5, 1024), (3, 130, 4099, 700), (1100, 72, 333, 1024),
                                        (200, 520, 70, 129)])
def test_many_entries(dtype, m, d, V, K):
    check(Case(dtype, m, d, V, K=K, out=0.1 if m > 1 else 0.0, short=m > 1))
    check(Case(dtype, m, d, V, K=K, seed=1), whole=True)


# rows too wide for a block's registers; a few rows more than 16 against many classes; many rows of few classes
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m, d, V", [(17, 5000, 300), (5, 8232, 70), (20, 16500, 33), (1, 20011, 5), (20, 1000, 5000),
                                     (40, 1001, 5003), (64, 960, 6007), (6575, 35, 25), (3001, 130, 40), (70001, 24, 9)])
def test_shapes(dtype, m, d, V):
    check(Case(dtype, m, d, V, out=0.2 if m > 5 else 0.0, gaps=d % 2))
    check(Case(dtype, m, d, V, K=3, out=0.2 if m > 5 else 0.0), dw=DTYPES[dtype])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m, d, V", [(3001, 130, 40), (40, 1001, 5003)])
def test_accumulation(dtype, m, d, V):
    """dw is added to what is there: a sum and its rounding to fp32 apart from the gradient alone."""
    c = Case(dtype, m, d, V)
    _, lse, picked = forward(c)
    _, alone = backward(c, lse, picked)
    dw = torch.randn(V, d, device="cuda")
    before = dw.clone()
    ws = torch.empty(fa.client_vocab_workspace_bytes(m, d, V, c.dt), device="cuda", dtype=torch.uint8)
    fa.client_vocab_loss_backward(c.x, c.w, c.index, lse, picked, None, dw, dloss=c.dloss, accumulate=True, workspace=ws)
    # a multiplication added in one rounding, or rounded first
    assert ((dw.double() - (before.double() + alone.double())).abs() <= U * (dw.double().abs() + 2 * alone.double().abs())).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("m", [3, 1100])
@pytest.mark.parametrize("K", [0, 5])
def test_logits_far_apart(dtype, m, K):
    """Probabilities that are 0 and 1 in fp32."""
    c = Case(dtype, m, 64, 700, K=K, seed=4)
    check(c, logit_scale=100.0)
    check(c, logit_scale=1e-6)


@pytest.mark.parametrize("m", [3, 1100])
def test_offsets_beyond_32_bits(m):
    V, d = 2 ** 31 // 4096 + 301, 4096
    g = torch.Generator(device="cuda").manual_seed(m)
    stride = 2 ** 31 // (m - 1) // 8 * 8 + 8       # the last row of x and dx begins beyond 2^31 elements
    x, dx = (torch.empty(stride * (m - 1) + d, device="cuda", dtype=torch.bfloat16).as_strided((m, d), (stride, 1))
             for _ in range(2))
    x.copy_(torch.randn(m, d, device="cuda", generator=g) * 0.5)
    w = torch.empty(V, d, device="cuda", dtype=torch.bfloat16)
    step = 2 ** 16
    for at in range(0, V, step):
        w[at:at + step] = torch.randn(min(step, V - at), d, device="cuda", generator=g) * d ** -0.5
    targets = V - 1 - torch.arange(m, device="cuda") % 300
    new = lambda: torch.empty(m, device="cuda")
    loss, lse, picked = new(), new(), new()
    ws = torch.empty(max(fa.client_vocab_workspace_bytes(m, d, V, x.dtype, backward=k) for k in (False, True)), device="cuda",
                     dtype=torch.uint8)
    fa.client_vocab_loss_forward(x, w, targets, loss, lse, picked, workspace=ws)
    dw = torch.empty(V, d, device="cuda")
    fa.client_vocab_loss_backward(x, w, targets, lse, picked, dx, dw, workspace=ws)
    X = x.double()
    parts, at_target = [], torch.empty(m, device="cuda", dtype=torch.double)
    for at in range(0, V, step):
        z = X @ w[at:at + step].double().t()
        parts.append(torch.logsumexp(z, dim=1))
        here = (targets >= at) & (targets < at + step)
        at_target[here] = z[here, targets[here] - at]
    want = torch.logsumexp(torch.stack(parts), dim=0)
    # sums of 4,096 products of magnitude below 8, and of 2^19 powers: 2^-13 holds both
    assert (lse - want).abs().max() <= 2.0 ** -13 * want.abs().max()
    assert (picked - at_target).abs().max() <= 2.0 ** -13 * 8
    assert (loss - (want - at_target)).abs().max() <= 2.0 ** -12 * want.abs().max()
    total, most = torch.zeros_like(X), torch.zeros_like(X)
    for at in range(0, V, step):
        W = w[at:at + step].double()
        dz = torch.exp(X @ W.t() - want[:, None])
        here = ((targets >= at) & (targets < at + step)).nonzero()[:, 0]
        dz[here, targets[here] - at] -= 1.0
        total += dz @ W
        most += dz.abs() @ W.abs()
        # dz in two bf16 terms, off by 2^-12 of itself for its logit
        assert ((dw[at:at + step] - dz.t() @ X).abs() <= 2.0 ** -10 * (dz.abs().t() @ X.abs()) + 1e-30).all(), at
    assert ((dx - total).abs() <= 2.0 ** -7.5 * total.abs() + 2.0 ** -8 * most).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_as_many_rows_as_there_may_be(dtype):
    check(Case(dtype, 2 ** 20, 8, 4, out=0.1))

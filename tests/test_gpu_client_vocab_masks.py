"""The losses over a vocabulary where some logits or rows are not finite: classes
masked by the lowest value of a type or by -infinity (through a column of W that
a constant activation meets), and a row that has gone astray among others."""
import math

import pytest
import torch

from test_gpu_client_vocab import DTYPES, Case, backward, forward
from vocab_reference import Reference
from vocab_ways import way

pytestmark = pytest.mark.gpu

# one block sees all classes (few of them; many rows); many blocks; tiles, whose last rows fill none
FORMS = [(5, 24, 12, "direct"), (3001, 130, 40, "direct"), (17, 64, 1000, "direct"), (2100, 72, 8200, "tiles")]
CASES = [(*form, dtype, value) for form in FORMS for dtype in DTYPES for value in ("lowest", "-inf")]


class Masked:
    """A case over the classes that are not masked, and the same among masked ones.  The masked ones weigh nothing, so
    every result is the first one's; dw of the masked classes is 0."""

    def __init__(self, dtype, m, d, V, K, value, seed=5):
        g = torch.Generator().manual_seed(seed)
        left = torch.zeros(V, dtype=torch.bool)
        left[torch.randperm(V, generator=g)[: V - max(2, V // 3)]] = True
        self.left = left.cuda()
        at = self.left.nonzero()[:, 0]
        self.small = Case(dtype, m, d, len(at), K, seed=seed)
        dt = self.small.dt
        self.small.x[:, -1], self.small.w[:, -1] = 1.0, 0.0
        self.full = Case(dtype, m, d, len(at), K, seed=seed)
        self.full.x = self.small.x
        self.full.w = torch.randn(V, d, generator=g).to(dt).cuda() * d ** -0.5
        self.full.w[at] = self.small.w
        self.full.w[~self.left, -1] = torch.finfo(dt).min if value == "lowest" else -math.inf
        self.full.index = at[self.small.index]

    def reference(self, **kw):
        c = self.small
        return Reference(c.x, c.w, c.index, teacher=c.teacher, dloss=c.dloss, **kw)


@pytest.mark.parametrize("K", [0, 3])
@pytest.mark.parametrize("m, d, V, form, dtype, value", CASES)
def test_losses_beside_masked_classes(m, d, V, form, dtype, K, value):
    assert way(m, d, V, DTYPES[dtype]) == form
    c = Masked(dtype, m, d, V, K, value)
    ref = c.reference()
    for name, got in zip(("loss", "lse", "picked"), forward(c.full)):
        ref.check(name, got)


@pytest.mark.parametrize("K", [0, 3])
@pytest.mark.parametrize("m, d, V, form, dtype, value", CASES)
def test_gradients_beside_masked_classes(m, d, V, form, dtype, K, value):
    assert way(m, d, V, DTYPES[dtype]) == form
    c = Masked(dtype, m, d, V, K, value)
    ref = c.reference()
    _, lse, picked = forward(c.full)
    dx, dw = backward(c.full, lse, picked)
    if value == "-inf":     # 0 times -infinity in the column of the masks
        dx, ref.dx, ref.tol_dx = dx[:, :-1], ref.dx[:, :-1], ref.tol_dx[:, :-1]
    ref.check("dx", dx)
    ref.check("dw", dw[c.left])
    assert (dw[~c.left] == 0).all()


@pytest.mark.parametrize("m, d, V, form", FORMS)
def test_infinite_weights_beside_any_activation(m, d, V, form):
    """fp32: an infinite weight and an activation of few or many bits, of either sign, have an infinite product.  A class
    of logits of infinity makes its row's log-sum-exp no number or infinity, one of -infinity is as if it were not there."""
    c = Masked("fp32", m, d, V, 0, "-inf")
    g = torch.Generator(device="cuda").manual_seed(1)
    x = c.full.x[:, -1]
    x.copy_(torch.rand(m, device="cuda", generator=g) + 0.5)
    x[::3] = 2.0 ** -40
    x[1::3] *= -1.0
    ref = c.reference()     # w is 0 there for the classes that are not masked
    loss, lse, picked = forward(c.full)
    for name, got in (("loss", loss), ("lse", lse), ("picked", picked)):
        got = got.clone()
        if name != "picked":
            assert not torch.isfinite(got[1::3]).any()
            got[1::3] = getattr(ref, name)[1::3].float()
        ref.check(name, got)


@pytest.mark.parametrize("K", [0, 5])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bad", ["x is NaN", "x is infinite", "dloss is NaN", "dloss is -NaN", "dloss is infinite"])
@pytest.mark.parametrize("m, d, V, form", [(200, 72, 333, "direct"), (2100, 72, 8200, "tiles")])
def test_a_row_that_is_not_finite_is_its_own_affair(m, d, V, form, bad, dtype, K):
    """The other rows' results are as if it had been left out; dw takes every row."""
    assert way(m, d, V, DTYPES[dtype]) == form
    c = Case(dtype, m, d, V, K)
    at = 77
    without = c.index.clone()
    without[at] = -100
    ref = Reference(c.x, c.w, without, teacher=c.teacher, dloss=c.dloss)
    if bad.startswith("x"):
        c.x[at, 3] = math.nan if bad.endswith("NaN") else math.inf
    elif bad.endswith("-NaN"):
        c.dloss.view(torch.int32)[at] = -1
    else:
        c.dloss[at] = math.nan if bad.endswith("NaN") else math.inf
    loss, lse, picked = forward(c)
    dx, dw = backward(c, lse, picked)
    assert not torch.isfinite(dx[at]).all()
    for name, got in (("loss", loss), ("lse", lse), ("picked", picked), ("dx", dx)):
        got = got.clone()
        got[at] = 0.0
        ref.check(name, got)


@pytest.mark.parametrize("dtype", DTYPES)
def test_coefficients_whose_sum_is_beyond_fp32(dtype):
    """One row's coefficients are finite, their sum is not: dw is right."""
    m, d, V = 2100, 72, 8200
    assert way(m, d, V, DTYPES[dtype]) == "tiles"
    c = Case(dtype, m, d, V)
    c.x *= 2.0 ** -6
    c.dloss[77] = 3e38
    _, lse, picked = forward(c)
    _, dw = backward(c, lse, picked)
    ref = Reference(c.x, c.w, c.index, dloss=c.dloss)
    ref.check("dw", dw)


@pytest.mark.parametrize("K", [0, 5])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m, d, V, form", [(200, 72, 333, "direct"), (2100, 72, 8200, "tiles")])
def test_rows_that_weigh_little_beside_others(m, d, V, form, dtype, K):
    """dx of a row is as good with a small dloss as with a large one: it is in proportion, and so is how far it may be
    off, but for the smallest numbers of its type."""
    assert way(m, d, V, DTYPES[dtype]) == form
    c = Case(dtype, m, d, V, K)
    c.w += 0.25         # so that the softmax's part of dx is not small beside the targets'
    g = torch.Generator().manual_seed(9)
    c.dloss = (10.0 ** (-7.0 * torch.rand(m, generator=g))).cuda()
    ref = Reference(c.x, c.w, c.index, teacher=c.teacher)
    _, lse, picked = forward(c)
    dx, dw = backward(c, lse, picked, grad_scale=2.0 ** 14)
    Reference(c.x, c.w, c.index, teacher=c.teacher, dloss=c.dloss, grad_scale=2.0 ** 14).check("dw", dw)
    assert torch.equal(backward(c, lse, picked, dx=False, grad_scale=2.0 ** 14)[1], dw)
    assert torch.equal(backward(c, lse, picked, dw=None, grad_scale=2.0 ** 14)[0], dx)
    least = 2.0 ** -25 if dtype == "fp16" else 0.0
    by = (c.dloss.double() * 2.0 ** 14)[:, None]
    ref.dx, ref.tol_dx = ref.dx * by, (ref.tol_dx - least) * by + least
    ref.check("dx", dx)

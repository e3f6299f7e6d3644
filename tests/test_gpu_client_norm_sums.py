"""GPU: the residual norm's gradients where fp32 holds every step exactly, so
that they are compared exactly: a row left out, taken twice or scaled shows in
the sums over rows, however many rows there are.

The backward pass takes the statistics from its caller: integer means and
1/sqrt of 1/2, 1 or 2.  With small integers everywhere, dropout at 1/2 (a
factor of 2) and gates and weights of powers of two, each term is a multiple
of 1/8 below 2^10, and sums of up to 6,000 of them are exact in fp32 in any
order.  The means over a row, in the gradients through a norm, are exact where
the columns are a power of two."""
import numpy as np
import pytest

import client_reference as ref
import paper_1601_04033_amd as fa
from helpers import gpu

pytestmark = pytest.mark.gpu

# rows that share a block (up to 512 columns), blocks of many rows with as many columns as 64 and 1,024 threads hold,
# rows of the loop; numbers of rows with and without an uneven last turn
SHAPES = [(1, 1), (1, 4), (3, 7), (6000, 24), (5003, 64), (4099, 100), (3001, 200), (2050, 512), (1111, 513), (1500, 1024),
          (1029, 2050), (700, 4096), (600, 5003), (530, 8192), (300, 12_000), (520, 17_001), (257, 16_384)]


class Exact:
    def __init__(self, rows, cols, dtype, layer, bias, gate, pre, drop):
        import torch
        self.shape, self.dt, self.layer, self.pre = (rows, cols), getattr(torch, dtype), layer, pre
        rng = np.random.default_rng(rows * 7 + cols + layer)
        ints = lambda *s: rng.integers(-3, 4, size=s).astype(np.float64)
        power = lambda n: np.exp2(rng.integers(-1, 2, size=n).astype(np.float64))
        self.x, self.s, self.dsum, self.dh = (ints(rows, cols) for _ in range(4))
        for a in (self.x, self.s, self.dsum, self.dh):
            a[:, 0] = np.where(a[:, 0] == 0, 1, a[:, 0])       # no row is without terms
        self.mean = rng.integers(-1, 2, size=(2, rows, 1)).astype(np.float64) * layer
        self.x[:, :1] += 3 * (self.x[:, :1] == self.mean[0])
        self.s[:, :1] += 3 * (self.s[:, :1] == self.mean[1])
        self.rstd = np.exp2(rng.integers(-1, 2, size=(2, rows, 1)).astype(np.float64))
        self.w_post, self.w_pre = power(cols), power(cols)
        self.bias = bias
        self.b_post, self.b_pre = (ints(cols), ints(cols)) if bias else (None, None)
        self.gate_form = gate
        self.gate = {None: None, "channel": power(cols), "row": power((rows, 1)), "full": power((rows, cols))}[gate]
        self.drop = (0.5, 11 + cols, 3, 1, 2) if drop else None
        self.m = ref.drop_factor(rows, cols, self.drop) if drop else np.ones((rows, cols))

    def want(self):
        """The gradients in fp64, by the formulas, from the given statistics."""
        xh1, xh2 = ((a - m) * r for a, m, r in zip((self.x, self.s), self.mean, self.rstd))

        def back(g, xh, rstd):
            out = g - xh * (g * xh).mean(1, keepdims=True)
            return rstd * (out - g.mean(1, keepdims=True) if self.layer else out)

        ds = self.dsum
        if self.pre:
            ds = ds + back(self.dh * self.w_pre, xh2, self.rstd[1])
        du = ds * self.m
        a = 1.0 if self.gate is None else self.gate
        z = xh1 * self.w_post + (self.b_post if self.bias else 0.0)
        terms = {"dw_post": du * a * xh1, "db_post": du * a, "dgate": du * z, "dw_pre": self.dh * xh2, "db_pre": self.dh}
        out = {k: v.sum(0) for k, v in terms.items()}
        if self.gate_form == "row":
            out["dgate"] = terms["dgate"].sum(1, keepdims=True)
        elif self.gate_form == "full":
            out["dgate"] = terms["dgate"]
        out["dresidual"], out["dbranch"] = 0.5 * ds, back(du * a * self.w_post, xh1, self.rstd[0])
        return out, terms

    def got(self):
        import torch
        rows, cols = self.shape
        dev = lambda a, dt=torch.float32: None if a is None else torch.from_numpy(a).to(dt).cuda()
        x, s, dsum, dh = (dev(a, self.dt) for a in (self.x, self.s, self.dsum, self.dh))
        st = np.concatenate([self.mean[0], self.rstd[0], self.mean[1], self.rstd[1]], axis=1)
        gate = dev(self.gate, self.dt if self.gate_form == "full" else torch.float32)
        opts = dict(kind=fa.NORM_LAYER if self.layer else fa.NORM_RMS, w_post=dev(self.w_post), b_post=dev(self.b_post),
                    gate=gate, residual_scale=0.5, dropout=self.drop)
        if self.pre:
            opts.update(w_pre=dev(self.w_pre), b_pre=dev(self.b_pre))
        out = {k: torch.full_like(x, 9.0) for k in ("dbranch", "dresidual")}
        args = {"dw_post": torch.full((cols,), 9.0, device="cuda")}
        if gate is not None:
            args["dgate"] = torch.full_like(gate, 9.0)
        if self.bias:
            args["db_post"] = torch.full((cols,), 9.0, device="cuda")
        for k in (("dw_pre", "db_pre") if self.bias else ("dw_pre",)) if self.pre else ():
            args[k] = torch.full((cols,), 9.0, device="cuda")
        ws = torch.empty(fa.client_residual_norm_workspace_bytes(rows, cols), device="cuda", dtype=torch.uint8).fill_(255)
        fa.client_residual_norm_backward(x, s if self.pre else None, dev(st), dsum, dh if self.pre else None,
                                         out["dbranch"], out["dresidual"], workspace=ws, **args, **opts)
        return {**out, **args}

    def check(self, names):
        import torch
        want, terms = self.want()
        got = self.got()
        for k in names:
            if k not in got:
                continue
            w = torch.from_numpy(want[k])
            w = w.to(self.dt) if w.shape == self.shape and k in ("dbranch", "dresidual", "dgate") and (
                k != "dgate" or self.gate_form == "full") else w.float()
            assert torch.equal(got[k].cpu(), w), (k, (got[k].cpu() != w).sum().item())
            if k.startswith(("dw", "db_")) or (k == "dgate" and self.gate_form == "channel"):
                # what the comparison finds out: any row left out, and zeros
                rows_seen = terms[k].any(axis=1) if self.drop is None else np.array([True])
                assert rows_seen.all() and want[k].any()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("layer, bias, gate, drop", [(False, False, "channel", False), (True, True, "full", True),
                                                     (True, False, "row", True), (False, True, None, False)])
@pytest.mark.parametrize("rows, cols", SHAPES)
def test_gradients_without_a_norm_before_the_next_block(dtype, layer, bias, gate, drop, rows, cols):
    gpu()
    names = ["dw_post", "db_post", "dgate", "dresidual"] + (["dbranch"] if cols & (cols - 1) == 0 else [])
    Exact(rows, cols, dtype, layer, bias, gate, False, drop).check(names)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("layer, bias", [(False, False), (True, True)])
@pytest.mark.parametrize("rows, cols", SHAPES)
def test_gradients_with_both_norms(dtype, layer, bias, rows, cols):
    gpu()
    names = ["dw_pre", "db_pre"] + (["dresidual"] if cols & (cols - 1) == 0 else [])
    Exact(rows, cols, dtype, layer, bias, "channel", True, True).check(names)

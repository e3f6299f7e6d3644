"""The losses over a vocabulary in 64 bits, straight from their formulas, and how
far fp32 kernels with 16-bit terms may be from them."""
import math

import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}     # half a step, relative


class Reference:
    """Everything a call returns, and its tolerance (tol_*), for targets (teacher None) or a teacher's entries."""

    def __init__(self, x, w, index, *, teacher=None, teacher_scale=1.0, teacher_lse=None, logit_scale=1.0,
                 smoothing=0.0, z_loss=0.0, dloss=None, grad_scale=1.0, dw_dtype=torch.float32):
        dtype, s = x.dtype, logit_scale
        m, d = x.shape
        V = w.shape[0]
        W = w.double()
        entries = index.reshape(m, -1)
        there = (entries >= 0) & (entries < V)
        if teacher is not None:
            there &= teacher.double() != -math.inf
        used = there.any(dim=1)
        X = torch.where(used[:, None], x.double(), 0.0)
        i = torch.where(there, entries, 0)
        z = s * (X @ W.t())
        lse = torch.logsumexp(z, dim=1)
        zi = torch.where(there, z.gather(1, i), 0.0)
        if teacher is None:
            q = there.double() * (1.0 - smoothing)
            loss = lse - (1.0 - smoothing) * zi[:, 0] - smoothing * z.mean(dim=1) + z_loss * lse * lse
            f, b = 1.0 + 2.0 * z_loss * lse, smoothing / V
            most = 1.0
        else:
            t = torch.where(there, teacher.double() * teacher_scale, -math.inf)
            if teacher_lse is None:
                q = torch.softmax(torch.where(used[:, None], t, 0.0), dim=1) * there
            else:
                q = torch.exp(t - teacher_lse.double()[:, None])
            loss = (torch.special.xlogy(q, q) - q * (zi - lse[:, None])).sum(dim=1)
            f, b = q.sum(dim=1), 0.0
            most = f
        g = torch.where(used, (torch.ones_like(lse) if dloss is None else dloss.double()) * grad_scale, 0.0)
        p = torch.exp(z - lse[:, None])
        dz = f[:, None] * p - b if torch.is_tensor(f) else f * p - b
        dz = dz.scatter_add(1, i, -q) * g[:, None]
        self.used = used
        self.loss, self.lse = torch.where(used, loss, 0.0), torch.where(used, lse, 0.0)
        self.picked = zi.reshape(index.shape)
        self.dx, self.dw = s * dz @ W, s * dz.t() @ X

        # A sum of d products: roundings of its fp32 partial sums, at most the sum of magnitudes each, as a random
        # walk, 8 deviations of it.  fp32 operands: three bf16 terms each, products below 2^-24 left out.
        mag = s * (X.abs() @ W.abs().t())
        u = 2.0 ** -24
        ez = mag * (8 * u * math.sqrt(d + 16) + (4 * u if dtype == torch.float32 else 0.0)) + 4 * u * z.abs()
        top = ez.max(dim=1).values
        # log-sum-exp: its logits', its own roundings, sums of V powers each 2 roundings off
        el = top + 8 * u * (lse.abs() + 1.0) + 8 * u * math.sqrt(V) / 4 + 4 * u * z.abs().max(dim=1).values
        self.tol_lse = el
        self.tol_picked = torch.where(there, ez.gather(1, i) + 4 * u * zi.abs(), 0.0).reshape(index.shape)
        eq = 16 * u * (1.0 + (0 if teacher is None else teacher.double().nan_to_num(0, 0, 0).abs().max().item() * teacher_scale))
        ei = ez.gather(1, i).max(dim=1).values
        weights = q.sum(dim=1) + (smoothing if teacher is None else 0.0)
        self.tol_loss = weights * (el + ei) + el * 2 * abs(z_loss) * lse.abs() + smoothing * (mag.mean(dim=1) * 8 * u * 16) \
            + (eq + 8 * u) * (q * (torch.where(q > 0, q, 1.0).log().abs() + zi.abs() + lse.abs()[:, None])).sum(dim=1) \
            + 8 * u * (loss.abs() + lse.abs() + abs(z_loss) * lse * lse)
        # a gradient's element: p's relative error, and the terms it is held in
        ep = (ez + el[:, None] + 4 * u * (z.abs() + lse.abs()[:, None]) + 8 * u)
        err = (g.abs() * (f if torch.is_tensor(f) else f))[:, None] * p * ep
        err = err + (g.abs()[:, None] * q * eq).sum(dim=1, keepdim=True) * torch.zeros_like(p).scatter_add(1, i, there.double()).clamp(max=1.0)
        err = err + 4 * u * (g.abs() * (b + (q.sum(dim=1))))[:, None] * (p + b)
        floor = 0.0
        if dtype == torch.float16:      # below fp16's normal range, after the largest coefficient is taken to 2^14
            top_g = (g.abs() * (most + (f.abs() if torch.is_tensor(f) else f) + b)).max() if m else 0.0
            floor = 2.0 ** -39 * top_g
        one = HALF[dtype] if dtype != torch.float32 else 2.0 ** -23
        two = one * one if dtype != torch.float32 else 2.0 ** -23
        along = 8 * u
        ax, aw = X.abs(), W.abs()
        hold = two if dw_dtype == torch.float32 else one
        self.tol_dx = s * ((err + one * dz.abs() + floor) @ aw + along * math.sqrt(V + 16) * (dz.abs() @ aw)) \
            + HALF[dtype] * 1.01 * self.dx.abs() + 1e-37
        self.tol_dw = s * ((err + hold * dz.abs() + floor).t() @ ax + along * math.sqrt(m + 16) * (dz.abs().t() @ ax)) \
            + HALF[dw_dtype] * 1.01 * self.dw.abs() + 1e-37
        if dtype == torch.float16:      # outputs below the normal range
            self.tol_dx = self.tol_dx + 2.0 ** -25
        if dw_dtype == torch.float16:
            self.tol_dw = self.tol_dw + 2.0 ** -25

    def check(self, name, got):
        want, tol = getattr(self, name), getattr(self, "tol_" + name)
        got = got.double().reshape(want.shape).to(want.device)
        off = (got - want).abs()
        bad = ~(off <= tol)
        assert not bad.any(), (name, int(bad.sum()), bad.numel(), float((off / tol.clamp(min=1e-300)).nan_to_num(1e9).max()),
                               float(off.nan_to_num(1e9).max()))

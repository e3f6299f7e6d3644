"""64-bit forms of the client's operators, for the tests: written from the
definitions in include/fasgd_client.h with numpy, apart from the kernels."""
import numpy as np


def philox4x32_10(c0, c1, c2, c3, seed):
    """Philox4x32-10 (Salmon et al., SC'11) of arrays of counter words, four uint64 arrays of 32-bit words."""
    m32 = np.uint64(0xFFFFFFFF)
    x = [np.asarray(c, dtype=np.uint64) + np.zeros_like(np.asarray(c0, dtype=np.uint64)) for c in (c0, c1, c2, c3)]
    k0, k1 = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    for _ in range(10):
        p0, p2 = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(p2 >> np.uint64(32)) ^ x[1] ^ np.uint64(k0), p2 & m32, (p0 >> np.uint64(32)) ^ x[3] ^ np.uint64(k1),
             p0 & m32]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return x


def threshold(p):
    return int(np.floor(p * 65536.0 + 0.5))


def keep_mask(rows, cols, p, seed, T, client, site, index_base=0):
    J = np.arange(rows * cols, dtype=np.uint64) + np.uint64(index_base)
    chunk, lane = J >> np.uint64(3), (J & np.uint64(7)).astype(np.int64)
    ctr1 = (chunk >> np.uint64(32)) | np.uint64(0x40000000 | site << 16)
    w = np.stack(philox4x32_10(chunk & np.uint64(0xFFFFFFFF), ctr1, np.uint64(T), np.uint64(client), seed))
    word = w[lane // 2, np.arange(J.size)]
    half = np.where(lane % 2 == 0, word & np.uint64(0xFFFF), word >> np.uint64(16))
    return (half >= threshold(p)).reshape(rows, cols)


def drop_factor(rows, cols, dropout, index_base=0):
    p, seed, T, client, site = dropout
    keep = keep_mask(rows, cols, p, seed, T, client, site, index_base)
    thr = threshold(p)
    return keep * (65536.0 / (65536 - thr) if thr < 65536 else 0.0)


def act(g, name):
    return {"identity": lambda: g, "sigmoid": lambda: 1 / (1 + np.exp(-g)), "tanh": lambda: np.tanh(g)}[name]()


def act_slope(g, name):
    a = act(g, name)
    return {"identity": lambda: np.ones_like(g), "sigmoid": lambda: a * (1 - a), "tanh": lambda: 1 - a * a}[name]()


def normed(x, layer, eps):
    """(x - mean) rstd and rstd"""
    d = x - x.mean(1, keepdims=True) if layer else x
    rstd = 1 / np.sqrt((d * d).mean(1, keepdims=True) + eps)
    return d * rstd, rstd


def _affine(xh, w, b):
    return xh * w + (0 if b is None else b)


def residual_norm_sum(branch, residual, layer, w_post, b_post, gate, gate_act, rho, eps, m):
    z = branch if w_post is None else _affine(normed(branch, layer, eps)[0], w_post, b_post)
    a = 1.0 if gate is None else act(gate, gate_act)
    u = np.where(m == 0, 0.0, a * z) * m
    return u if residual is None else rho * residual + u


def residual_norm_normed(total, layer, w_pre, b_pre, eps):
    return _affine(normed(total, layer, eps)[0], w_pre, b_pre)


def _back(g, xh, rstd, layer):
    out = g - xh * (g * xh).mean(1, keepdims=True)
    return rstd * (out - g.mean(1, keepdims=True) if layer else out)


def residual_norm_backward(branch, total, dsum, dnormed, layer, w_post, b_post, w_pre, b_pre, gate, gate_act, rho,
                           eps, m):
    """Gradients, and for each sum over rows or columns the same sum of magnitudes ("abs_" names)."""
    out = {}
    ds = np.zeros_like(branch) if dsum is None else dsum
    if w_pre is not None:
        xh2, r2 = normed(total, layer, eps)
        ds = ds + _back(dnormed * w_pre, xh2, r2, layer)
        out["dw_pre"], out["abs_dw_pre"] = (dnormed * xh2).sum(0), np.abs(dnormed * xh2).sum(0)
        out["db_pre"], out["abs_db_pre"] = dnormed.sum(0), np.abs(dnormed).sum(0)
    out["dresidual"] = rho * ds
    du = ds * m
    a = 1.0 if gate is None else act(gate, gate_act)
    xh1, r1 = (branch, None) if w_post is None else normed(branch, layer, eps)
    z = branch if w_post is None else _affine(xh1, w_post, b_post)
    if gate is not None:
        dg = np.where(m == 0, 0.0, du * z) * act_slope(gate, gate_act)
        if gate.ndim == 1:
            out["dgate"], out["abs_dgate"] = dg.sum(0), np.abs(dg).sum(0)
        elif gate.shape[1] == 1 and branch.shape[1] != 1:
            out["dgate"], out["abs_dgate"] = dg.sum(1, keepdims=True), np.abs(dg).sum(1, keepdims=True)
        else:
            out["dgate"] = dg
    dz = du * a
    if w_post is None:
        out["dbranch"] = dz + np.zeros_like(branch)
    else:
        out["dw_post"], out["abs_dw_post"] = (dz * xh1).sum(0), np.abs(dz * xh1).sum(0)
        out["db_post"], out["abs_db_post"] = dz.sum(0) + np.zeros(branch.shape[1]), np.abs(dz).sum(0)
        out["dbranch"] = _back(dz * w_post, xh1, r1, layer)
    return out


# ---- 8-bit blocks

FMAX = {"e4m3": 448.0, "e5m2": 57344.0}


def round_8bit(y, fmt):
    """Nearest value of the format, ties to even (|y| <= its largest)."""
    bits, low = (3, -6) if fmt == "e4m3" else (2, -14)
    _, ex = np.frexp(y)
    step = np.exp2((np.maximum(ex - 1, low) - bits).astype(np.float64))
    return np.round(y / step) * step


def block_exponent(amax, fmt):
    """The smallest e >= -126 with amax <= fmax 2^e (0 for amax = 0)."""
    m, k = np.frexp(amax)
    e = k - (9 if fmt == "e4m3" else 16) + (m > 0.875)
    return np.where(amax == 0, 0, np.maximum(e, -126))


def held(x, fmt, block_rows=1):
    """(values, exponents per row and block) of x held in 8 bits in blocks of 128 along its last axis."""
    r, c = x.shape
    rp, cp = -(-r // block_rows) * block_rows, -(-c // 128) * 128
    y = np.zeros((rp, cp))
    y[:r, :c] = x
    t = y.reshape(rp // block_rows, block_rows, cp // 128, 128)
    finite = np.where(np.isfinite(t), np.abs(t), 0.0)
    e = block_exponent(finite.max(axis=(1, 3), keepdims=True), fmt)
    s = np.exp2(e.astype(np.float64))
    q = np.where(np.isfinite(t), round_8bit(np.where(np.isfinite(t), t, 0.0) / s, fmt), np.nan) * s
    e_rows = np.broadcast_to(e, (rp // block_rows, block_rows, cp // 128, 1)).reshape(rp, cp // 128)
    return q.reshape(rp, cp)[:r, :c], e_rows[:r]

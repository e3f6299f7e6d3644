"""Performance cases of the client side: the operators with which a client of
the parameter server turns a fetched theta into a gradient.

  dropout   client_dropout: Philox4x32-10 keyed by (seed, T, client, site,
            index), mask never stored; forward, or forward and backward
  norm      client_residual_norm_forward / _backward: the norm after a block,
            its gate, dropout, the scaled residual sum and the norm before
            the next block, in one call each way
  linear    client_fp8_linear: activations times 8-bit weights held in blocks
            of 128 (serving and evaluation)
  train     client_fp8_quantize, client_fp8_matmul: a linear layer's forward
            product and both its gradients, weights quantized from fp32

Definitions shared by the plain forms, the 64-bit ones and the kernels:

Dropout.  thr = floor(65536 p + 1/2).  Element i (row-major index) takes the
16-bit half (i mod 2) of word (i mod 8) / 2 of Philox4x32-10 at counter
(c low 32 bits, 0x40000000 | site << 16 | c high 16 bits, T, client), c = i / 8,
key seed; it is kept iff that half is >= thr, and then scaled by
65536 / (65536 - thr).

Residual norm.  s = rho residual + drop(act(gate) N_post(branch)), stored in the
activations' type; h = N_pre(s) of s as stored.  Backward from the gradients
of s and h.

8-bit blocks.  A block of 128 along the contraction (128 x 128 for weights)
with largest magnitude amax is held as q 2^e: e the smallest integer with
amax <= fmax 2^e and e >= -126 (fmax 448 for e4m3, 57344 for e5m2; e = 0 for a
block of zeros), q = x 2^-e rounded to nearest even in that format.  Products are of the values so held.

Sizes: the 784-1000-1000-10 MLP of this repository's workloads at a minibatch
of 128, and generic block widths.
"""
import math

import torch

own = False     # False: the plain forms; True: the framework's kernels

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
FMAX_EXP = {"e4m3": 9, "e5m2": 16}      # fmax = 0.875 * 2^this
EPS = 1e-5
BLOCK = 128
MOST_ELEMENTS = 16384 * 4096
MOST_FLOPS = 3 * 2 * 8192 * 4096 * 16384


def listed():
    return [
        # the MLP's hidden activations of one minibatch: the smallest call, bound by latency
        {"name": "dropout_mlp", "kind": "dropout", "dtype": "fp32", "rows": 128, "cols": 1000, "ld": 1000, "p": 0.5,
         "residual": False, "backward": False},
        # a ragged batch of hidden rows inside a wider buffer, both directions
        {"name": "dropout_ragged", "kind": "dropout", "dtype": "fp16", "rows": 4099, "cols": 1001, "ld": 1024,
         "p": 0.2, "residual": False, "backward": True},
        # residual dropout of a training step's 16,384 tokens, both directions
        {"name": "dropout_block", "kind": "dropout", "dtype": "bf16", "rows": 16384, "cols": 4096, "ld": 4096,
         "p": 0.1, "residual": True, "backward": True},
        # one token passes from a block to the next (serving)
        {"name": "norm_token", "kind": "norm", "dtype": "bf16", "rows": 1, "cols": 4096, "norm": "rms",
         "gate": "channel", "act": "none", "p": 0.0, "rho": 1.0, "bias": False, "backward": False},
        # a layer norm with biases around the MLP's hidden layer, one gate per sample, a training step
        {"name": "norm_mlp", "kind": "norm", "dtype": "fp32", "rows": 128, "cols": 1000, "norm": "layer",
         "gate": "row", "act": "sigmoid", "p": 0.0, "rho": 0.5, "bias": True, "backward": True},
        # a ragged batch with a gate computed for every element, a training step
        {"name": "norm_ragged", "kind": "norm", "dtype": "fp16", "rows": 2053, "cols": 5003, "norm": "layer",
         "gate": "full", "act": "sigmoid", "p": 0.1, "rho": 0.7, "bias": True, "backward": True},
        # the training step of 16,384 tokens between two blocks, learned gate per channel, residual dropout
        {"name": "norm_block", "kind": "norm", "dtype": "bf16", "rows": 16384, "cols": 4096, "norm": "rms",
         "gate": "channel", "act": "tanh", "p": 0.1, "rho": 1.0, "bias": False, "backward": True},
        # one token through a layer whose weights stay in 8 bits (serving): bound by reading the weights
        {"name": "linear_token", "kind": "linear", "dtype": "bf16", "m": 1, "k": 4096, "n": 16384},
        # a few requests decoded together, ragged widths
        {"name": "linear_few", "kind": "linear", "dtype": "bf16", "m": 27, "k": 8200, "n": 4100},
        # a ragged batch evaluated
        {"name": "linear_ragged", "kind": "linear", "dtype": "fp16", "m": 4099, "k": 5003, "n": 2002},
        # the MLP's first layer, one minibatch: forward, input gradient, weight gradient
        {"name": "train_mlp", "kind": "train", "dtype": "fp32", "m": 128, "k": 784, "n": 1000, "grad": "e4m3"},
        # a block's wide layer at 8,192 tokens: forward, input gradient, weight gradient; 5-bit exponents for gradients
        {"name": "train_block", "kind": "train", "dtype": "bf16", "m": 8192, "k": 4096, "n": 16384, "grad": "e5m2"},
    ]


def _log_int(rng, lo, hi):
    x = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return x + 1 if x == 3072 else x


def draw(rng):
    kind = rng.choice(["dropout", "norm", "norm", "linear", "linear", "train", "train"])
    c = {"kind": kind, "dtype": rng.choice(["fp32", "bf16", "bf16", "fp16"])}
    if kind in ("dropout", "norm"):
        c["cols"] = _log_int(rng, 64, 8192)
        if rng.random() < 0.5:
            c["cols"] = (c["cols"] + 63) // 64 * 64
        c["rows"] = _log_int(rng, 1, MOST_ELEMENTS * 2 // SIZE[c["dtype"]] // c["cols"])
        c["p"] = rng.choice([0.0, 0.1, 0.25, 0.5]) if kind == "norm" else rng.choice([0.05, 0.1, 0.2, 0.5])
        c["backward"] = rng.random() < 0.7
        if kind == "dropout":
            c["ld"] = c["cols"] + rng.choice([0, 0, 8, 24])
            c["residual"] = rng.random() < 0.5
        else:
            c["norm"] = rng.choice(["rms", "layer"])
            c["gate"] = rng.choice(["none", "channel", "row", "full"])
            c["act"] = rng.choice(["none", "sigmoid", "tanh"])
            c["rho"] = rng.choice([1.0, 0.5, 0.22])
            c["bias"] = c["norm"] == "layer" and rng.random() < 0.7
        return c
    c["k"] = _log_int(rng, 256, 16384)
    c["n"] = _log_int(rng, 256, 16384)
    if rng.random() < 0.5:
        c["k"], c["n"] = (c["k"] + 127) // 128 * 128, (c["n"] + 127) // 128 * 128
    if kind == "linear":
        most = 64 if rng.random() < 0.5 else min(8192, MOST_FLOPS // (2 * c["k"] * c["n"]))
        c["m"] = _log_int(rng, 1, most)
    else:
        c["m"] = _log_int(rng, 32, min(8192, MOST_FLOPS // (6 * c["k"] * c["n"])))
        c["grad"] = rng.choice(["e4m3", "e5m2"])
    return c


# ---------------------------------------------------------------- inputs

def _key(seed):
    """seed, T, client, site of a pass's dropout."""
    return (seed * 0x9E3779B97F4A7C15 + 0x1234567) & (2 ** 64 - 1), 4096 + seed % 100_000, seed % 64, seed % 5


class _Gen:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed * 1_000_003 + 29)

    def normal(self, *shape, scale=1.0):
        return torch.empty(*shape, device="cuda").normal_(0.0, scale, generator=self.g)

    def activations(self, rows, cols, scale=1.0):
        """N(0, scale^2) whose rows and columns differ in scale, a few columns far out."""
        x = self.normal(rows, cols, scale=scale)
        x *= torch.exp(self.normal(rows, 1, scale=0.5))
        c = torch.exp(self.normal(cols, scale=0.5))
        c[:: max(cols // 7, 1)] *= 8.0
        return x * c


def _inputs(case, seed):
    """The case's data, from the seed alone."""
    g = _Gen(seed)
    dt = DTYPES[case["dtype"]]
    if case["kind"] == "dropout":
        r, c, ld = case["rows"], case["cols"], case["ld"]
        x = {}
        for name in ("x", "residual", "dy"):
            if (name == "residual" and not case["residual"]) or (name == "dy" and not case["backward"]):
                continue
            buf = torch.zeros(r, ld, device="cuda", dtype=dt)
            buf[:, :c] = g.activations(r, c)
            x[name] = buf[:, :c]
        return x
    if case["kind"] == "norm":
        r, c = case["rows"], case["cols"]
        x = {"branch": g.activations(r, c).to(dt), "residual": g.activations(r, c, 2.0).to(dt),
             "w_post": 1.0 + g.normal(c, scale=0.1), "w_pre": 1.0 + g.normal(c, scale=0.1)}
        x["gate"] = {"none": lambda: None, "channel": lambda: g.normal(c, scale=0.5),
                     "row": lambda: g.normal(r, 1, scale=0.5), "full": lambda: g.normal(r, c).to(dt)}[case["gate"]]()
        x["b_post"] = g.normal(c, scale=0.1) if case["bias"] else None
        x["b_pre"] = g.normal(c, scale=0.1) if case["bias"] else None
        if case["backward"]:
            x["dsum"] = g.activations(r, c, 1e-2).to(dt)
            x["dnormed"] = g.activations(r, c, 1e-2).to(dt)
        return x
    m, k, n = case["m"], case["k"], case["n"]
    x = {"x": g.activations(m, k).to(dt), "w": g.normal(n, k, scale=0.05)}
    if case["kind"] == "train":
        x["dy"] = g.activations(m, n, 1e-3).to(dt)
    return x


def prepare(case, seed):
    s = {"case": case, "key": _key(seed), **_inputs(case, seed)}
    if not own:
        if case["kind"] == "linear":
            s["w"] = _held(s["w"], "e4m3", weights=True)
        return s
    import paper_1601_04033_amd as fa
    dt = DTYPES[case["dtype"]]
    if case["kind"] == "dropout":
        s["y"] = torch.empty_like(s["x"])
        if case["backward"]:
            s["dx"] = torch.empty_like(s["x"])
    elif case["kind"] == "norm":
        r, c = case["rows"], case["cols"]
        s["sum"], s["normed"] = torch.empty_like(s["branch"]), torch.empty_like(s["branch"])
        s["stats"] = torch.empty(r, 4, device="cuda")
        if case["backward"]:
            s["dbranch"], s["dresidual"] = torch.empty_like(s["branch"]), torch.empty_like(s["branch"])
            for name in ("w_post", "b_post", "w_pre", "b_pre", "gate"):
                s["d" + name] = None if s[name] is None else torch.empty_like(s[name])
            s["ws"] = torch.empty(fa.client_residual_norm_workspace_bytes(r, c), device="cuda", dtype=torch.uint8)
    else:
        m, k, n = case["m"], case["k"], case["n"]
        s["y"] = torch.empty(m, n, device="cuda", dtype=dt)
        s["wq"] = fa.client_fp8_operand(n, k)
        if case["kind"] == "linear":
            fa.client_fp8_quantize(s.pop("w"), s["wq"], block_rows=BLOCK)
            s["ws"] = torch.empty(fa.client_fp8_workspace_bytes(m, n, k), device="cuda", dtype=torch.uint8)
        else:
            fmt = {"e4m3": fa.FP8_E4M3, "e5m2": fa.FP8_E5M2}[case["grad"]]
            s["wtq"] = fa.client_fp8_operand(k, n)
            s["xq"], s["xtq"] = fa.client_fp8_operand(m, k), fa.client_fp8_operand(k, m)
            s["dyq"], s["dytq"] = fa.client_fp8_operand(m, n, fmt), fa.client_fp8_operand(n, m, fmt)
            s["dx"] = torch.empty(m, k, device="cuda", dtype=dt)
            s["dw"] = torch.empty(n, k, device="cuda")
            s["ws"] = torch.empty(max(fa.client_fp8_workspace_bytes(m, n, k), fa.client_fp8_workspace_bytes(m, k, n),
                                      fa.client_fp8_workspace_bytes(n, k, m)), device="cuda", dtype=torch.uint8)
    return s


def run(s):
    return (_run_own if own else _run_plain)(s)


# ---------------------------------------------------------------- the framework's calls

def _run_own(s):
    import paper_1601_04033_amd as fa
    case = s["case"]
    seed, T, client, site = s["key"]
    if case["kind"] == "dropout":
        fa.client_dropout(s["x"], s["y"], case["p"], seed, T, client, site=site, residual=s.get("residual"))
        if not case["backward"]:
            return [s["y"]]
        fa.client_dropout(s["dy"], s["dx"], case["p"], seed, T, client, site=site)
        return [s["y"], s["dx"]]
    if case["kind"] == "norm":
        opts = dict(kind={"rms": fa.NORM_RMS, "layer": fa.NORM_LAYER}[case["norm"]], w_post=s["w_post"],
                    b_post=s["b_post"], gate=s["gate"],
                    gate_act={"none": fa.GATE_IDENTITY, "sigmoid": fa.GATE_SIGMOID, "tanh": fa.GATE_TANH}[case["act"]],
                    w_pre=s["w_pre"], b_pre=s["b_pre"], residual_scale=case["rho"], eps=EPS,
                    dropout=(case["p"], seed, T, client, site))
        fa.client_residual_norm_forward(s["branch"], s["residual"], s["sum"], s["normed"], s["stats"], **opts)
        out = {"sum": s["sum"], "normed": s["normed"]}
        if case["backward"]:
            fa.client_residual_norm_backward(
                s["branch"], s["sum"], s["stats"], s["dsum"], s["dnormed"], s["dbranch"], s["dresidual"],
                dw_post=s["dw_post"], db_post=s["db_post"], dgate=s["dgate"], dw_pre=s["dw_pre"], db_pre=s["db_pre"],
                workspace=s["ws"], **opts)
            for name in ("dbranch", "dresidual", "dw_post", "db_post", "dgate", "dw_pre", "db_pre"):
                if s[name] is not None:
                    out[name] = s[name]
        return out
    if case["kind"] == "linear":
        fa.client_fp8_linear(s["x"], s["wq"], s["y"], workspace=s["ws"])
        return {"y": s["y"]}
    fa.client_fp8_quantize(s["w"], s["wq"], s["wtq"], block_rows=BLOCK)
    fa.client_fp8_quantize(s["x"], s["xq"], s["xtq"])
    fa.client_fp8_matmul(s["xq"], s["wq"], s["y"], workspace=s["ws"])
    fa.client_fp8_quantize(s["dy"], s["dyq"], s["dytq"])
    fa.client_fp8_matmul(s["dyq"], s["wtq"], s["dx"], workspace=s["ws"])
    fa.client_fp8_matmul(s["dytq"], s["xtq"], s["dw"], workspace=s["ws"])
    return {"y": s["y"], "dx": s["dx"], "dw": s["dw"]}


# ---------------------------------------------------------------- plain forms (32 bits)

def _philox(c0, c1, c2, c3, key):
    """Philox4x32-10 on int64 tensors holding 32-bit words (a product's 64 bits are exact modulo 2^64)."""
    mask = 0xFFFFFFFF
    k0, k1 = key & mask, key >> 32
    x = [c0, c1, c2, c3]
    for _ in range(10):
        p0, p1 = x[0] * 0xD2511F53, x[2] * 0xCD9E8D57
        x = [((p1 >> 32) & mask) ^ x[1] ^ k0, p1 & mask, ((p0 >> 32) & mask) ^ x[3] ^ k1, p0 & mask]
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    return x


def _threshold(p):
    return int(math.floor(p * 65536 + 0.5))


def _keep(rows, cols, p, key):
    """The kept elements, a truth value each."""
    seed, T, client, site = key
    n = rows * cols
    c = torch.arange((n + 7) // 8, device="cuda", dtype=torch.int64)
    w = _philox(c & 0xFFFFFFFF, (c >> 32) | (0x40000000 | site << 16), torch.full_like(c, T),
                torch.full_like(c, client), seed)
    halves = torch.stack([h for x in w for h in (x & 0xFFFF, x >> 16)], dim=1)
    return (halves.reshape(-1)[:n] >= _threshold(p)).reshape(rows, cols)


def _scale(p):
    return 65536.0 / (65536 - _threshold(p))


def _pow2(e):
    """2^e in fp32 for int32 e in [-126, 127], exactly."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _held(x, fmt, weights=False):
    """x (fp32) as the values its 8-bit blocks of 128 along the last axis stand for."""
    r, c = x.shape
    rp, cp = (r + BLOCK - 1) // BLOCK * BLOCK if weights else r, (c + BLOCK - 1) // BLOCK * BLOCK
    y = torch.zeros(rp, cp, device=x.device)
    y[:r, :c] = x
    y = y.view(rp // BLOCK, BLOCK, cp // BLOCK, BLOCK) if weights else y.view(rp, 1, cp // BLOCK, BLOCK)
    amax = y.abs().amax(dim=(1, 3), keepdim=True)
    mant, ex = torch.frexp(amax)
    e = ex - FMAX_EXP[fmt] + (mant > 0.875)
    e = torch.where(amax > 0, e.clamp(min=-126), torch.zeros_like(e))
    q = (y * _pow2(-e)).to(torch.float8_e4m3fn if fmt == "e4m3" else torch.float8_e5m2).float()
    return (q * _pow2(e)).view(rp, cp)[:r, :c].contiguous()


def _norm(x, kind, w, b):
    mean = x.mean(dim=1, keepdim=True) if kind == "layer" else torch.zeros_like(x[:, :1])
    rstd = torch.rsqrt((x - mean).square().mean(dim=1, keepdim=True) + EPS)
    xh = (x - mean) * rstd
    y = xh * w
    return (y if b is None else y + b), xh, rstd


def _norm_backward(dy, xh, rstd, kind, w):
    q = dy * w
    t = q - xh * (q * xh).mean(dim=1, keepdim=True)
    if kind == "layer":
        t = t - q.mean(dim=1, keepdim=True)
    return t * rstd


def _run_plain(s):
    case = s["case"]
    dt = DTYPES[case["dtype"]]
    if case["kind"] == "dropout":
        keep = _keep(case["rows"], case["cols"], case["p"], s["key"])
        y = torch.where(keep, s["x"].float() * _scale(case["p"]), 0.0)
        if case["residual"]:
            y = y + s["residual"].float()
        out = [y.to(dt)]
        if case["backward"]:
            out.append(torch.where(keep, s["dy"].float() * _scale(case["p"]), 0.0).to(dt))
        return out
    if case["kind"] == "norm":
        kind = case["norm"]
        z, xh_post, rstd_post = _norm(s["branch"].float(), kind, s["w_post"], s["b_post"])
        act = {"none": lambda t: t, "sigmoid": torch.sigmoid, "tanh": torch.tanh}[case["act"]]
        gate = 1.0
        if case["gate"] != "none":
            gate = act(s["gate"].float())
        drop = 1.0
        if case["p"] > 0:
            keep = _keep(case["rows"], case["cols"], case["p"], s["key"])
            drop = torch.where(keep, _scale(case["p"]), 0.0)
        total = (case["rho"] * s["residual"].float() + gate * z * drop).to(dt)
        normed, xh_pre, rstd_pre = _norm(total.float(), kind, s["w_pre"], s["b_pre"])
        out = {"sum": total, "normed": normed.to(dt)}
        if case["backward"]:
            dh = s["dnormed"].float()
            ds = s["dsum"].float() + _norm_backward(dh, xh_pre, rstd_pre, kind, s["w_pre"])
            du = ds * drop
            dz = du * gate
            out["dbranch"] = _norm_backward(dz, xh_post, rstd_post, kind, s["w_post"]).to(dt)
            out["dresidual"] = (case["rho"] * ds).to(dt)
            out["dw_post"] = (dz * xh_post).sum(dim=0)
            if case["bias"]:
                out["db_post"] = dz.sum(dim=0)
            if case["gate"] != "none":
                slope = {"none": lambda a: 1.0, "sigmoid": lambda a: a * (1.0 - a), "tanh": lambda a: 1.0 - a * a}
                dg = du * z * slope[case["act"]](gate)
                out["dgate"] = {"channel": lambda: dg.sum(dim=0), "row": lambda: dg.sum(dim=1, keepdim=True),
                                "full": lambda: dg.to(dt)}[case["gate"]]()
            out["dw_pre"] = (dh * xh_pre).sum(dim=0)
            if case["bias"]:
                out["db_pre"] = dh.sum(dim=0)
        return out
    if case["kind"] == "linear":
        return {"y": (_held(s["x"].float(), "e4m3") @ s["w"].t()).to(dt)}
    x, dy = s["x"].float(), s["dy"].float()
    w = _held(s["w"], "e4m3", weights=True)
    y = _held(x, "e4m3") @ w.t()
    dx = _held(dy, case["grad"]) @ w
    dw = _held(dy.t(), case["grad"]) @ _held(x.t(), "e4m3").t()
    return {"y": y.to(dt), "dx": dx.to(dt), "dw": dw}


# ---------------------------------------------------------------- what one pass cannot do without

def work(case):
    if case["kind"] == "dropout":
        n = case["rows"] * case["cols"]
        tensors = 2 + case["residual"] + 2 * case["backward"]
        return {"bytes": n * SIZE[case["dtype"]] * tensors, "flops": 2 * n * (1 + case["backward"])}
    if case["kind"] == "norm":
        n = case["rows"] * case["cols"]
        full = case["gate"] == "full"
        tensors = 4 + full + (4 + full) * case["backward"]
        vectors = (2 + 2 * case["bias"] + (case["gate"] == "channel")) * (1 + case["backward"]) * case["cols"]
        vectors += (case["gate"] == "row") * (1 + case["backward"]) * case["rows"]
        return {"bytes": n * SIZE[case["dtype"]] * tensors + 4 * vectors, "flops": n * (14 + 26 * case["backward"])}
    m, k, n = case["m"], case["k"], case["n"]
    size = SIZE[case["dtype"]]
    if case["kind"] == "linear":
        return {"bytes": m * k * size + n * k + n * k // BLOCK // BLOCK + m * n * size, "flops": 2 * m * n * k}
    return {"bytes": 2 * (m * k + m * n) * size + 8 * n * k, "flops": 6 * m * n * k}


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_keep(rows, cols, p, key):
    seed, T, client, site = key
    kept = torch.empty(rows * cols, dtype=torch.bool, device="cuda")
    at, step = 0, 1 << 25
    while at < rows * cols:     # one element at a time, each with its own draw
        i = torch.arange(at, min(at + step, rows * cols), device="cuda")
        chunk, lane = i // 8, i % 8
        a, b = chunk % 2 ** 32, chunk // 2 ** 32 + 0x40000000 + site * 65536
        c, d = torch.full_like(i, T), torch.full_like(i, client)
        k0, k1 = seed % 2 ** 32, seed // 2 ** 32
        for _ in range(10):
            lo0, hi0 = _times(a, 0xD2511F53)
            lo2, hi2 = _times(c, 0xCD9E8D57)
            a, b, c, d = hi2 ^ b ^ k0, lo2, hi0 ^ d ^ k1, lo0
            k0, k1 = (k0 + 0x9E3779B9) % 2 ** 32, (k1 + 0xBB67AE85) % 2 ** 32
        word = torch.where(lane < 2, a, torch.where(lane < 4, b, torch.where(lane < 6, c, d)))
        kept[at:at + i.numel()] = torch.where(lane % 2 == 0, word % 65536, word // 65536) >= _threshold(p)
        at += step
    return kept.view(rows, cols)


def _times(x, m):
    """Low and high 32 bits of x m from 16-bit pieces."""
    xl, xh, ml, mh = x % 65536, x // 65536, m % 65536, m // 65536
    mid = xh * ml + (xl * ml) // 65536
    mid2 = xl * mh + mid % 65536
    return (mid2 % 65536) * 65536 + (xl * ml) % 65536, xh * mh + mid // 65536 + mid2 // 65536


def _double_pow2(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_held(x, fmt, rows_per_block):
    """x (fp64) rounded block by block on the 8-bit grid, from the grid's spacing."""
    r, c = x.shape
    bits, low = (3, -6) if fmt == "e4m3" else (2, -14)
    y = torch.zeros(-(-r // rows_per_block) * rows_per_block, -(-c // BLOCK) * BLOCK, dtype=torch.float64, device="cuda")
    y[:r, :c] = x
    t = y.reshape(y.shape[0] // rows_per_block, rows_per_block, -1, BLOCK)
    amax = t.abs().amax(dim=3, keepdim=True).amax(dim=1, keepdim=True)
    fmax = 0.875 * 2.0 ** FMAX_EXP[fmt]
    e = torch.frexp(amax)[1] - FMAX_EXP[fmt] - 1
    for _ in range(3):
        e = torch.where(amax > fmax * _double_pow2(e), e + 1, e)
    e = torch.where(amax > 0, e.clamp(min=-126), torch.zeros_like(e))
    t = t / _double_pow2(e)
    step = _double_pow2((torch.frexp(t)[1] - 1).clamp(min=low) - bits)
    t = torch.round(t / step) * step
    return (t * _double_pow2(e)).reshape(y.shape)[:r, :c].contiguous()


def exact(case, seed):
    x = _inputs(case, seed)
    x = {k: (v.double() if torch.is_tensor(v) else v) for k, v in x.items()}
    key = _key(seed)
    p = case.get("p", 0.0)
    if case["kind"] == "dropout":
        m = _exact_keep(case["rows"], case["cols"], p, key)
        up = 65536 / (65536 - _threshold(p))
        y = torch.where(m, x["x"] * up, 0.0)
        if case["residual"]:
            y += x["residual"]
        return [y] + ([torch.where(m, x["dy"] * up, 0.0)] if case["backward"] else [])
    if case["kind"] == "norm":
        return _exact_norm(case, x, key)
    if case["kind"] == "linear":
        return {"y": _exact_held(x["x"], "e4m3", 1) @ _exact_held(x["w"], "e4m3", BLOCK).t()}
    w = _exact_held(x["w"], "e4m3", BLOCK)
    return {"y": _exact_held(x["x"], "e4m3", 1) @ w.t(), "dx": _exact_held(x["dy"], case["grad"], 1) @ w,
            "dw": _exact_held(x["dy"].t().contiguous(), case["grad"], 1)
            @ _exact_held(x["x"].t().contiguous(), "e4m3", 1).t()}


def _exact_norm(case, x, key):
    layer = case["norm"] == "layer"
    d = case["cols"]

    def stats(t):
        mean = t.sum(1, keepdim=True) / d if layer else 0.0
        var = ((t - mean) ** 2).sum(1, keepdim=True) / d
        return (t - mean) / (var + EPS).sqrt(), 1.0 / (var + EPS).sqrt()

    def back(g, xh, rstd):
        out = g - xh * ((g * xh).sum(1, keepdim=True) / d)
        return rstd * (out - g.sum(1, keepdim=True) / d if layer else out)

    xh1, r1 = stats(x["branch"])
    z = xh1 * x["w_post"] + (x["b_post"] if case["bias"] else 0.0)
    a, slope = 1.0, 0.0
    if case["gate"] != "none":
        g = x["gate"]
        if case["act"] == "none":
            a, slope = g, torch.ones_like(g)
        elif case["act"] == "sigmoid":
            a = 1.0 / (1.0 + torch.exp(-g))
            slope = a * (1.0 - a)
        else:
            a = torch.tanh(g)
            slope = 1.0 - a ** 2
    m = 1.0
    if case["p"] > 0:
        m = _exact_keep(case["rows"], case["cols"], case["p"], key) * (65536 / (65536 - _threshold(case["p"])))
    s = case["rho"] * x["residual"] + m * a * z
    stored = s.to(DTYPES[case["dtype"]]).double()
    xh2, r2 = stats(stored)
    out = {"sum": s, "normed": xh2 * x["w_pre"] + (x["b_pre"] if case["bias"] else 0.0)}
    if not case["backward"]:
        return out
    ds = x["dsum"] + back(x["dnormed"] * x["w_pre"], xh2, r2)
    dz = ds * m * a
    out["dbranch"] = back(dz * x["w_post"], xh1, r1)
    out["dresidual"] = case["rho"] * ds
    out["dw_post"] = (dz * xh1).sum(0)
    if case["bias"]:
        out["db_post"] = dz.sum(0)
    if case["gate"] != "none":
        dg = ds * m * z * slope
        out["dgate"] = dg if case["gate"] == "full" else (dg.sum(0) if case["gate"] == "channel" else dg.sum(1, keepdim=True))
    out["dw_pre"] = (x["dnormed"] * xh2).sum(0)
    if case["bias"]:
        out["db_pre"] = x["dnormed"].sum(0)
    return out

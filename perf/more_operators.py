"""Performance cases of the client's losses over a large vocabulary: where the
gradient that a client pushes begins.

  loss      client_vocab_loss_forward / _backward: softmax cross entropy of
            logits z = s x W^T, the logits never kept
  distill   client_vocab_distill_forward / _backward: divergence from a
            teacher's top logits to the same softmax

Definitions shared by the plain forms, the 64-bit ones and the kernels, for
activations x [m][d] and class weights W [V][d]:

  z_rj = s x_r . W_j,   lse_r = log sum_j exp z_rj,   p_rj = exp(z_rj - lse_r)

Loss.  With smoothing e, z loss u and the row's target t:
  loss_r = lse_r - (1 - e) z_rt - e/V sum_j z_rj + u lse_r^2
  dz_rj  = g_r ((1 + 2 u lse_r) p_rj - e/V - (1 - e) [j = t])
A target outside [0, V) leaves the row out: loss, lse, picked logit and
gradients are 0, whatever x holds there.

Distillation.  The teacher gives K entries (i_k, t_k) a row; one with i_k
outside [0, V) is left out.  q_k is the softmax of s_t t_k over the entries,
or exp(s_t t_k - L_r) where the teacher's own log-sum-exp L is given:
  loss_r = sum_k q_k (log q_k - z_{r, i_k} + lse_r)
  dz_rj  = g_r (p_rj sum_k q_k - sum_{k: i_k = j} q_k)
A row without entries is left out.

g_r = grad_scale dloss_r.  dx = s dz W has the activations' type, dW = s dz^T x
is fp32 (a slice of the flat gradient) or of the activations' type.  The
logits at the targets or entries (picked, before any other use) are returned
beside loss and lse.

Sizes: the 1,000-wide, 10-class MLP of this repository's workloads at a
minibatch of 128, and generic widths and vocabularies.
"""
import math

import torch

own = False     # False: the plain forms; True: the framework's kernels

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
MOST = 8192 * 4096 * 131072     # m d V of the largest case
PAD = 8                         # elements between rows where a case asks for gaps


def listed():
    return [
        # the MLP's head at one minibatch, a training step: the smallest call, bound by latency
        {"name": "loss_mlp", "kind": "loss", "dtype": "fp32", "m": 128, "d": 1000, "V": 10, "out": 0.0, "smooth": 0.0,
         "zloss": 0.0, "backward": True, "dw": "fp32", "gaps": False},
        # one token scored (serving): bound by reading the weights
        {"name": "loss_token", "kind": "loss", "dtype": "bf16", "m": 1, "d": 4096, "V": 131072, "out": 0.0,
         "smooth": 0.0, "zloss": 0.0, "backward": False, "dw": "fp32", "gaps": False},
        # a padded batch evaluated, odd widths inside wider buffers
        {"name": "loss_eval", "kind": "loss", "dtype": "fp16", "m": 2053, "d": 1001, "V": 50003, "out": 0.3,
         "smooth": 0.0, "zloss": 0.0, "backward": False, "dw": "fp32", "gaps": True},
        # a training step that keeps 32 bits throughout
        {"name": "loss_fp32", "kind": "loss", "dtype": "fp32", "m": 1024, "d": 1024, "V": 16384, "out": 0.0,
         "smooth": 0.1, "zloss": 0.0, "backward": True, "dw": "fp32", "gaps": False},
        # a training step on a batch whose prompts and padding carry no loss, 16-bit weight gradient
        {"name": "loss_ragged", "kind": "loss", "dtype": "fp16", "m": 1777, "d": 1544, "V": 32003, "out": 0.25,
         "smooth": 0.1, "zloss": 1e-4, "backward": True, "dw": "same", "gaps": True},
        # the training step of 8,192 tokens
        {"name": "loss_block", "kind": "loss", "dtype": "bf16", "m": 8192, "d": 4096, "V": 131072, "out": 0.0,
         "smooth": 0.0, "zloss": 1e-4, "backward": True, "dw": "fp32", "gaps": False},
        # a small classifier learns from another one's best 16 of 1,000 classes
        {"name": "distill_mlp", "kind": "distill", "dtype": "fp32", "m": 128, "d": 1000, "V": 1000, "K": 16,
         "out": 0.0, "short": False, "whole": False, "temp": 2.0, "backward": True, "dw": "fp32", "gaps": False},
        # one short sequence, a training step: bound by the weights and their gradient
        {"name": "distill_few", "kind": "distill", "dtype": "bf16", "m": 16, "d": 4096, "V": 131072, "K": 64,
         "out": 0.0, "short": False, "whole": True, "temp": 1.0, "backward": True, "dw": "fp32", "gaps": False},
        # a student evaluated against its teacher
        {"name": "distill_eval", "kind": "distill", "dtype": "bf16", "m": 512, "d": 2048, "V": 65536, "K": 32,
         "out": 0.1, "short": False, "whole": True, "temp": 1.0, "backward": False, "dw": "fp32", "gaps": False},
        # teachers that kept a different number of classes for each row, a temperature
        {"name": "distill_ragged", "kind": "distill", "dtype": "fp16", "m": 1531, "d": 2056, "V": 50021, "K": 50,
         "out": 0.2, "short": True, "whole": False, "temp": 2.0, "backward": True, "dw": "fp32", "gaps": True},
        # the training step of 4,096 tokens
        {"name": "distill_block", "kind": "distill", "dtype": "bf16", "m": 4096, "d": 4096, "V": 131072, "K": 64,
         "out": 0.0, "short": False, "whole": True, "temp": 1.0, "backward": True, "dw": "fp32", "gaps": False},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    c = {"kind": rng.choice(["loss", "distill"]), "dtype": rng.choice(["fp32", "bf16", "bf16", "fp16"])}
    c["d"], c["V"] = _log_int(rng, 64, 8192), _log_int(rng, 10, 131072)
    if rng.random() < 0.5:
        c["d"], c["V"] = (c["d"] + 63) // 64 * 64, (c["V"] + 63) // 64 * 64
    most = MOST // (16 if c["dtype"] == "fp32" else 1)
    c["m"] = _log_int(rng, 1, max(1, min(8192, most // (c["d"] * c["V"]))))
    c["out"] = rng.choice([0.0, 0.0, 0.3])
    c["backward"] = rng.random() < 0.7
    c["dw"] = rng.choice(["fp32", "fp32", "same"])
    c["gaps"] = rng.random() < 0.3
    if c["kind"] == "loss":
        c["smooth"], c["zloss"] = rng.choice([0.0, 0.0, 0.1]), rng.choice([0.0, 1e-4])
    else:
        c["K"] = _log_int(rng, 1, min(100, c["V"]))
        c["short"], c["whole"] = rng.random() < 0.3, rng.random() < 0.5
        c["temp"] = rng.choice([1.0, 2.0])
    return c


# ---------------------------------------------------------------- inputs

def _rows_in(case):
    """Rows that take part."""
    return case["m"] - int(case["m"] * case["out"])


def _matrix(case, x):
    """x in the case's type, its rows apart where the case asks for it."""
    dt = DTYPES[case["dtype"]]
    if not case["gaps"]:
        return x.to(dt)
    buf = torch.zeros(x.shape[0], x.shape[1] + PAD, device="cuda", dtype=dt)
    buf[:, :x.shape[1]] = x
    return buf[:, :x.shape[1]]


def _inputs(case, seed):
    """The case's data, from the seed alone."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1_000_003 + 57)
    m, d, V = case["m"], case["d"], case["V"]

    def normal(*shape, scale=1.0):
        return torch.empty(*shape, device="cuda").normal_(0.0, scale, generator=g)

    def uniform(*shape):
        return torch.rand(*shape, device="cuda", generator=g)

    left_out = torch.zeros(m, device="cuda", dtype=torch.bool)
    left_out[torch.randperm(m, device="cuda", generator=g)[: m - _rows_in(case)]] = True
    w = normal(V, d, scale=d ** -0.5)
    target = (uniform(m) * V).long().clamp(max=V - 1)
    # normed activations whose channels differ in scale, turned towards their class as far as training got
    x = normal(m, d) * torch.exp(normal(d, scale=0.3))
    x += w[target] * (uniform(m, 1) * 1.5 * math.log(V))
    s = {"x": _matrix(case, x), "w": _matrix(case, w), "dloss": (0.5 + uniform(m)) / max(1, _rows_in(case))}
    if case["kind"] == "loss":
        s["target"] = torch.where(left_out, -100, target)
        return s
    K = case["K"]
    # K classes of each row, its own first, and falling logits with a long tail
    stride = 1 + (uniform(m, 1) * max(1, V // K - 1)).long()
    k = torch.arange(K, device="cuda")
    index = (target[:, None] + k * stride) % V
    t = 8.0 - 1.5 * torch.log(k + 1.0) - uniform(m, K) / (k + 1.0)
    if case["short"]:
        index = torch.where(k < 1 + (uniform(m, 1) * K).long(), index, -1)
    s["index"] = torch.where(left_out[:, None], -1, index).contiguous()
    s["teacher"] = t.to(DTYPES[case["dtype"]])
    s["teacher_lse"] = None
    if case["whole"]:
        s["teacher_lse"] = torch.log(torch.exp(t / case["temp"]).sum(dim=1) * (1.0 + 0.2 * uniform(m)))
    return s


def prepare(case, seed):
    s = {"case": case, **_inputs(case, seed)}
    if own:
        import paper_1601_04033_amd as fa
        m, d, V = case["m"], case["d"], case["V"]
        dt = DTYPES[case["dtype"]]
        s["loss"], s["lse"] = torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
        s["picked"] = torch.empty(m, *([case["K"]] if case["kind"] == "distill" else []), device="cuda")
        if case["backward"]:
            s["dx"] = torch.empty(m, d, device="cuda", dtype=dt)
            s["dw"] = torch.empty(V, d, device="cuda", dtype=torch.float32 if case["dw"] == "fp32" else dt)
        s["ws"] = torch.empty(fa.client_vocab_workspace_bytes(m, d, V, dt, backward=case["backward"]), device="cuda",
                              dtype=torch.uint8)
    return s


def _temperature(case):
    """Scale of both sides' logits and of the gradient (the temperature's square, so that it does not fade)."""
    t = case.get("temp", 1.0)
    return 1.0 / t, t * t


def run(s):
    return (_run_own if own else _run_plain)(s)


# ---------------------------------------------------------------- the framework's calls

def _run_own(s):
    import paper_1601_04033_amd as fa
    case = s["case"]
    scale, grad_scale = _temperature(case)
    out = {"loss": s["loss"], "lse": s["lse"], "picked": s["picked"]}
    if case["kind"] == "loss":
        opts = dict(smoothing=case["smooth"], z_loss=case["zloss"], workspace=s["ws"])
        fa.client_vocab_loss_forward(s["x"], s["w"], s["target"], s["loss"], s["lse"], s["picked"], **opts)
        if case["backward"]:
            fa.client_vocab_loss_backward(s["x"], s["w"], s["target"], s["lse"], s["picked"], s["dx"], s["dw"],
                                          dloss=s["dloss"], **opts)
    else:
        opts = dict(logit_scale=scale, teacher_scale=scale, teacher_lse=s["teacher_lse"], workspace=s["ws"])
        fa.client_vocab_distill_forward(s["x"], s["w"], s["index"], s["teacher"], s["loss"], s["lse"], s["picked"],
                                        **opts)
        if case["backward"]:
            fa.client_vocab_distill_backward(s["x"], s["w"], s["index"], s["teacher"], s["lse"], s["picked"], s["dx"],
                                             s["dw"], dloss=s["dloss"], grad_scale=grad_scale, **opts)
    if case["backward"]:
        out["dx"], out["dw"] = s["dx"], s["dw"]
    return out


# ---------------------------------------------------------------- plain forms (32 bits)

def _run_plain(s):
    case = s["case"]
    V = case["V"]
    scale, grad_scale = _temperature(case)
    loss_kind = case["kind"] == "loss"
    entries = s["target"][:, None] if loss_kind else s["index"]
    taken = (entries >= 0) & (entries < V)
    index = torch.where(taken, entries, 0)
    used = taken.any(dim=1)
    x = torch.where(used[:, None], s["x"].float(), 0.0)
    w = s["w"].float()
    z = x @ w.t()
    if scale != 1.0:
        z *= scale
    top = z.amax(dim=1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(dim=1, keepdim=True)
    lse = torch.log(total) + top
    picked = torch.where(taken, z.gather(1, index), 0.0)
    if loss_kind:
        smooth, zloss = case["smooth"], case["zloss"]
        q = torch.where(taken, 1.0 - smooth, 0.0)
        loss = lse - (1.0 - smooth) * picked + zloss * lse * lse
        if smooth:
            loss = loss - smooth * z.mean(dim=1, keepdim=True)
        factor, flat = 1.0 + 2.0 * zloss * lse, smooth / V
    else:
        t = torch.where(taken, s["teacher"].float() * scale, -math.inf)
        if case["whole"]:
            q = torch.exp(t - s["teacher_lse"][:, None])
        else:
            q = torch.exp(t - torch.where(used[:, None], t.amax(dim=1, keepdim=True), 0.0))
            q = q / torch.where(used, q.sum(dim=1), 1.0)[:, None]
        logq = torch.log(torch.where(q > 0, q, 1.0))
        loss = (q * (logq - (picked - lse))).sum(dim=1, keepdim=True)
        factor, flat = q.sum(dim=1, keepdim=True), 0.0
    out = {"loss": torch.where(used, loss[:, 0], 0.0), "lse": torch.where(used, lse[:, 0], 0.0),
           "picked": picked[:, 0] if loss_kind else picked}
    if case["backward"]:
        g = torch.where(used, s["dloss"] * grad_scale, 0.0)[:, None]
        dz = e.mul_(factor / total)
        if flat:
            dz -= flat
        dz.scatter_add_(1, index, -q)
        dz *= g * scale
        out["dx"] = (dz @ w).to(DTYPES[case["dtype"]])
        dw = dz.t() @ x
        out["dw"] = dw if case["dw"] == "fp32" else dw.to(DTYPES[case["dtype"]])
    return out


# ---------------------------------------------------------------- what one pass cannot do without

def work(case):
    m, d, V = case["m"], case["d"], case["V"]
    rows, size = _rows_in(case), SIZE[case["dtype"]]
    K = case.get("K", 1)
    entry = 8 + (size if case["kind"] == "distill" else 0)      # index, teacher's logit
    nbytes = rows * d * size + V * d * size + m * (K * (entry + 4) + 8)
    if case["backward"]:
        nbytes += m * d * size + V * d * (4 if case["dw"] == "fp32" else size) + 4 * m
    return {"bytes": nbytes, "flops": 2 * rows * d * V * (3 if case["backward"] else 1)}


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = _inputs(case, seed)
    m, d, V = case["m"], case["d"], case["V"]
    t = case.get("temp", 1.0)
    w = s["w"].double()
    if case["kind"] == "loss":
        entries, weight = s["target"].view(m, 1), None
    else:
        entries, weight = s["index"], s["teacher"].double() / t
    new = dict(device="cuda", dtype=torch.float64)
    out = {"loss": torch.zeros(m, **new), "lse": torch.zeros(m, **new), "picked": torch.zeros(entries.shape, **new)}
    dx, dw = torch.zeros(m, d, **new), torch.zeros(V, d, **new)
    step = max(1, (1 << 28) // V)
    for at in range(0, m, step):        # a slab of rows at a time, the rows that take part alone
        rows = torch.arange(at, min(at + step, m), device="cuda")
        rows = rows[((entries[rows] >= 0) & (entries[rows] < V)).sum(dim=1) > 0]
        if rows.numel() == 0:
            continue
        x = s["x"][rows].double()
        z = torch.matmul(x, w.t()).div_(t)
        lse = torch.logsumexp(z, dim=1)
        i = entries[rows]
        there = (i >= 0) & (i < V)
        i = i * there
        zi = torch.gather(z, 1, i)
        zi[~there] = 0.0
        if case["kind"] == "loss":
            a, e = case["zloss"], case["smooth"]
            loss = lse * (1.0 + a * lse) - (1.0 - e) * zi[:, 0] - e * z.sum(dim=1) / V
            q = torch.full_like(zi, 1.0 - e)
            much, floor = 1.0 + 2.0 * a * lse, e / V
        else:
            q = torch.exp(weight[rows] - (s["teacher_lse"][rows, None].double() if case["whole"] else 0.0)) * there
            if not case["whole"]:
                q = q / q.sum(dim=1, keepdim=True)
            loss = torch.special.xlogy(q, q).sum(dim=1) - (q * (zi - lse[:, None]) * there).sum(dim=1)
            much, floor = q.sum(dim=1), 0.0
        out["loss"][rows], out["lse"][rows], out["picked"][rows] = loss, lse, zi
        if case["backward"]:
            dz = torch.exp(z.sub_(lse[:, None]))
            dz.mul_(much[:, None]).sub_(floor)
            dz.scatter_add_(1, i, -(q * there))
            dz.mul_(s["dloss"][rows, None].double() * t)        # the square of t from the gradient's scale, 1/t from z's
            dx[rows] = dz @ w
            dw += dz.t().contiguous() @ x
    if case["kind"] == "loss":
        out["picked"] = out["picked"][:, 0]
    if case["backward"]:
        out["dx"], out["dw"] = dx, dw
    return out

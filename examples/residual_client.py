"""Clients that train a residual network through the parameter server.

Each client keeps a copy of theta, fetched when it last pushed.  It turns it
into a gradient with the client's operators, the linear layers in 8-bit blocks
and the residual norm (dropout drawn from the counter) between them, and
pushes the gradient to the FASGD server.  Evaluation keeps the weights in
8 bits and takes each layer in one call.

    python examples/residual_client.py [--updates N] [--clients L]
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_1601_04033_amd as fa  # noqa: E402

INPUTS, WIDTH, BLOCKS, CLASSES, BATCH = 784, 1000, 3, 10, 128
DROP, SEED = 0.1, 1601


def layout():
    """(name, shape) of the parameters, in theta's order."""
    out = [("in", (WIDTH, INPUTS)), ("pre0", (WIDTH,))]
    for i in range(1, BLOCKS + 1):
        out += [(f"w{i}", (WIDTH, WIDTH)), (f"post{i}", (WIDTH,)), (f"gate{i}", (WIDTH,)), (f"pre{i}", (WIDTH,))]
    return out + [("head", (CLASSES, WIDTH))]


def views(flat):
    """The parameters as views of a flat fp32 vector."""
    out, at = {}, 0
    for name, shape in layout():
        n = shape[0] * (shape[1] if len(shape) == 2 else 1)
        out[name] = flat[at:at + n].view(shape)
        at += n
    return out


def parameters():
    return sum(s[0] * (s[1] if len(s) == 2 else 1) for _, s in layout())


def initial_theta(generator):
    theta = torch.empty(parameters(), device="cuda")
    for name, p in views(theta).items():
        if p.dim() == 2:
            p.normal_(0.0, p.shape[1] ** -0.5 * (0.1 if name == "head" else 1.0), generator=generator)
        else:
            p.fill_(0.5 if name.startswith("gate") else 1.0)
    return theta


class Layer:
    """One linear layer's operands and buffers for a fixed minibatch."""

    def __init__(self, n, k):
        bf16 = dict(device="cuda", dtype=torch.bfloat16)
        self.w, self.wt = fa.client_fp8_operand(n, k), fa.client_fp8_operand(k, n)
        self.x, self.xt = fa.client_fp8_operand(BATCH, k), fa.client_fp8_operand(k, BATCH)
        self.dy = fa.client_fp8_operand(BATCH, n, fa.FP8_E5M2)
        self.dyt = fa.client_fp8_operand(n, BATCH, fa.FP8_E5M2)
        self.y, self.dx = torch.empty(BATCH, n, **bf16), torch.empty(BATCH, k, **bf16)
        need = max(fa.client_fp8_workspace_bytes(*s) for s in ((BATCH, n, k), (BATCH, k, n), (n, k, BATCH)))
        self.ws = torch.empty(need, device="cuda", dtype=torch.uint8)

    def forward(self, x, weights):
        fa.client_fp8_quantize(weights, self.w, self.wt, block_rows=128)
        fa.client_fp8_quantize(x, self.x, self.xt)
        fa.client_fp8_matmul(self.x, self.w, self.y, workspace=self.ws)
        return self.y

    def backward(self, dy, dweights):
        fa.client_fp8_quantize(dy, self.dy, self.dyt)
        fa.client_fp8_matmul(self.dyt, self.xt, dweights, workspace=self.ws)
        fa.client_fp8_matmul(self.dy, self.wt, self.dx, workspace=self.ws)
        return self.dx


class Client:
    def __init__(self, number, theta):
        self.number, self.theta, self.T = number, theta.clone(), 0
        self.grad = torch.empty_like(theta)
        self.layers = {"in": Layer(WIDTH, INPUTS), "head": Layer(CLASSES, WIDTH),
                       **{f"w{i}": Layer(WIDTH, WIDTH) for i in range(1, BLOCKS + 1)}}
        self.ws = torch.empty(fa.client_residual_norm_workspace_bytes(BATCH, WIDTH), device="cuda", dtype=torch.uint8)
        self.stats = torch.empty(BLOCKS + 1, BATCH, 4, device="cuda")
        new = lambda: torch.empty(BATCH, WIDTH, device="cuda", dtype=torch.bfloat16)
        self.sums, self.normed = [new() for _ in range(BLOCKS + 1)], [new() for _ in range(BLOCKS + 1)]
        self.dbranch, self.dsum = new(), new()

    def fetch(self, state, theta):
        self.theta.copy_(theta)
        self.T = state.T

    def norm_options(self, p, i):
        if i == 0:
            return dict(w_pre=p["pre0"])
        return dict(w_post=p[f"post{i}"], gate=p[f"gate{i}"], gate_act=fa.GATE_TANH, w_pre=p[f"pre{i}"],
                    dropout=(DROP, SEED, self.T, self.number, i))

    def gradient(self, x, labels):
        """The loss of a minibatch (a device scalar); its gradient goes to self.grad."""
        p, g, L = views(self.theta), views(self.grad), self.layers
        for i in range(BLOCKS + 1):
            if i == 0:
                branch = L["in"].forward(x, p["in"])
            else:
                branch = L[f"w{i}"].forward(torch.relu(self.normed[i - 1]), p[f"w{i}"])
            fa.client_residual_norm_forward(branch, self.sums[i - 1] if i else None, self.sums[i], self.normed[i],
                                            self.stats[i], **self.norm_options(p, i))
        logits = L["head"].forward(self.normed[BLOCKS], p["head"]).float()
        logp = torch.log_softmax(logits, dim=1)
        hot = torch.nn.functional.one_hot(labels, CLASSES)
        dnormed = L["head"].backward(((logp.exp() - hot) / BATCH).to(torch.bfloat16), g["head"])
        dsum = None
        for i in range(BLOCKS, -1, -1):
            name = f"w{i}" if i else "in"
            grads = dict(dw_pre=g[f"pre{i}"])
            if i:
                grads.update(dw_post=g[f"post{i}"], dgate=g[f"gate{i}"])
            fa.client_residual_norm_backward(L[name].y, self.sums[i], self.stats[i], dsum, dnormed, self.dbranch,
                                             self.dsum if i else None, workspace=self.ws, **grads,
                                             **self.norm_options(p, i))
            dx = L[name].backward(self.dbranch, g[name])
            if i:
                dnormed, dsum = dx * (self.normed[i - 1] > 0), self.dsum
        return -(logp * hot).sum() / BATCH


def accuracy(theta, x, labels):
    """Share of right answers, by the serving form: weights quantized once, one call per layer."""
    p = views(theta)
    held = {}
    for name, w in p.items():
        if w.dim() == 2:
            held[name] = fa.client_fp8_operand(*w.shape)
            fa.client_fp8_quantize(w, held[name], block_rows=128)

    def linear(name, a):
        w = held[name]
        y = torch.empty(a.shape[0], w.rows, device="cuda", dtype=a.dtype)
        ws = torch.empty(fa.client_fp8_workspace_bytes(a.shape[0], w.rows, w.k), device="cuda", dtype=torch.uint8)
        fa.client_fp8_linear(a, w, y, workspace=ws)
        return y

    total = normed = None
    for i in range(BLOCKS + 1):
        branch = linear("in", x) if i == 0 else linear(f"w{i}", torch.relu(normed))
        new = torch.empty_like(branch)
        opts = dict(w_pre=p["pre0"]) if i == 0 else dict(w_post=p[f"post{i}"], gate=p[f"gate{i}"],
                                                         gate_act=fa.GATE_TANH, w_pre=p[f"pre{i}"])
        fa.client_residual_norm_forward(branch, total, new, branch, torch.empty(len(x), 4, device="cuda"), **opts)
        total, normed = new, branch
    return (linear("head", normed).argmax(dim=1) == labels).float().mean()


def run(updates=200, clients=4, alpha=1.0, report=None):
    """Trains on a synthetic task (which of 10 prototypes an input is, with noise); returns the losses, the accuracy
    on fresh inputs and theta."""
    g = torch.Generator(device="cuda")
    g.manual_seed(SEED)
    prototypes = 0.15 * torch.randn(CLASSES, INPUTS, device="cuda", generator=g)

    def batch(n):
        labels = torch.randint(0, CLASSES, (n,), device="cuda", generator=g)
        return (prototypes[labels] + torch.randn(n, INPUTS, device="cuda", generator=g)).to(torch.bfloat16), labels

    theta, n, b, v, last_T = fa.allocate_state(parameters(), "cuda")
    theta.copy_(initial_theta(g))
    state = fa.fasgd_init_state(theta, n, b, v, last_T, lam=clients, alpha=alpha)
    team = [Client(c, theta) for c in range(clients)]
    losses = []
    for t in range(updates):
        client = team[t % clients]
        losses.append(client.gradient(*batch(BATCH)))
        fa.fasgd_apply_updates(state, [client.grad], clients=[client.number], grad_ts=[client.T])
        client.fetch(state, theta)
        if report and (t + 1) % report == 0:
            print(f"{t + 1} updates: loss {torch.stack(losses[-report:]).mean().item():.4f}", flush=True)
    return torch.stack(losses).cpu(), accuracy(theta, *batch(2000)).item(), theta


if __name__ == "__main__":
    a = argparse.ArgumentParser()
    a.add_argument("--updates", type=int, default=400)
    a.add_argument("--clients", type=int, default=4)
    args = a.parse_args()
    _, share, _ = run(args.updates, args.clients, report=50)
    print(f"accuracy on fresh inputs {share:.3f} (chance 0.1)")

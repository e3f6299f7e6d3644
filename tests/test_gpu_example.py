"""GPU: the example that trains a residual network through the server with the client's operators."""
import importlib.util
import os

import pytest

from helpers import gpu

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("residual_client", os.path.join(ROOT, "examples", "residual_client.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_training_lowers_the_loss_and_repeats():
    """Ten classes, so a loss of ln 10 = 2.3 and an accuracy of 0.1 at chance: after 200 updates the loss is below half
    of its start and the accuracy above 0.3, and a second run gives the same theta bit for bit."""
    import torch
    gpu()
    ex = _example()
    losses, share, theta = ex.run(200, 4)
    assert torch.isfinite(losses).all() and torch.isfinite(theta).all()
    assert losses[-20:].mean() < 0.5 * losses[:4].mean() and share > 0.3
    again, share2, theta2 = ex.run(200, 4)
    assert torch.equal(losses, again) and torch.equal(theta, theta2) and share == share2


def test_gradient_of_a_client_matches_autograd():
    """The client's gradient against torch's of the same network in fp32, without dropout: 8-bit operands round each
    value within 2^-4 (e4m3) or 2^-3 (e5m2) of itself, and activations are bf16.  Errors of that size in some 800 to
    1,000 terms average out, so each gradient points within 20 degrees of the exact one (cosine 0.94)."""
    import torch
    gpu()
    ex = _example()
    ex.DROP = 0.0
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    theta = ex.initial_theta(g)
    x = torch.randn(ex.BATCH, ex.INPUTS, device="cuda", generator=g).to(torch.bfloat16)
    labels = torch.randint(0, ex.CLASSES, (ex.BATCH,), device="cuda", generator=g)
    client = ex.Client(0, theta)
    client.gradient(x, labels)

    flat = theta.clone().requires_grad_()
    p = ex.views(flat)
    rms = lambda t, w: t * torch.rsqrt(t.square().mean(1, keepdim=True) + 1e-5) * w
    total = x.float() @ p["in"].t()
    h = rms(total, p["pre0"])
    for i in range(1, ex.BLOCKS + 1):
        total = total + torch.tanh(p[f"gate{i}"]) * rms(torch.relu(h) @ p[f"w{i}"].t(), p[f"post{i}"])
        h = rms(total, p[f"pre{i}"])
    torch.nn.functional.cross_entropy(h @ p["head"].t(), labels).backward()
    for (name, a), b in zip(ex.views(client.grad).items(), ex.views(flat.grad).values()):
        cos = torch.nn.functional.cosine_similarity(a.flatten().double(), b.flatten().double(), dim=0).item()
        assert cos > 0.94, (name, cos)

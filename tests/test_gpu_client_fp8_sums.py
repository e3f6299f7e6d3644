"""GPU: the sums of 8-bit products, full (fp32) and, where the caller asks for them, short.

Full sums.  (a) Operands whose groups of 8 products hold +200,704 and -200,704
beside products of at most 9: every partial sum is an integer below 2^24, so in
fp32 the result is exact in any order, and an arithmetic that drops what lies
far below a group's largest product is found out.  (b) Random operands, within
the bound of fp32 sums for every output type: (k / 32 + 32) 2^-24 times the sum
of magnitudes and the last rounding.

Short sums.  Integers whose products are within 2^13 of each other are exact,
and random operands are within 7 2^-13 of each group's largest product beyond
that."""
import numpy as np
import pytest

import client_reference as ref
import paper_1601_04033_amd as fa
from helpers import gpu
from test_gpu_client_fp8 import FMT, ROUND, _bound, _held, _integers, _random
from test_gpu_client_marshal import _same, both  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu

SIXTEEN = ["bfloat16", "float16"]
# one token and few rows, quantized on the way or before; few rows in the larger kernel's tiles of 64; tiles of 128,
# 192 and 256; split contractions
SIZES = [(1, 100, 4096), (3, 9000, 300), (16, 100, 1000), (12, 700, 8200), (27, 4100, 1200), (40, 700, 8000),
         (700, 40, 8000), (300, 513, 640), (128, 128, 4100), (2975, 2897, 300), (4096, 4096, 256)]


def _cancelling(rows, k, seed, opposite):
    """Integers, [rows, k]: in each group of 8, +-448 in two places (of opposite signs, or of one) and small values."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randint(-3, 4, (rows, -(-k // 8) * 8), device="cuda", generator=g).float()
    groups = x.shape[1] // 8
    place = torch.Generator(device="cuda").manual_seed(k)       # the same places in both operands
    first = torch.randint(0, 8, (groups,), device="cuda", generator=place) + 8 * torch.arange(groups, device="cuda")
    second = first - first % 8 + (first + 1 + torch.randint(0, 7, (groups,), device="cuda", generator=place)) % 8
    sign = (torch.randint(0, 2, (rows, groups), device="cuda", generator=g) * 2 - 1).float()
    x[:, first] = 448.0 * sign
    x[:, second] = (-448.0 if opposite else 448.0) * sign
    if k % 8:
        x[:, -8:] = torch.randint(-3, 4, (rows, 8), device="cuda", generator=g).float()
    return x[:, :k].contiguous()


def _exact(x, w):
    """Integer products below 2^53 in fp64."""
    return x.double() @ w.double().t()


@pytest.mark.parametrize("dtype", SIXTEEN + ["float32"])
@pytest.mark.parametrize("m, n, k", SIZES)
def test_what_large_products_leave_is_kept(dtype, m, n, k):
    import torch
    gpu()
    x, w = _cancelling(m, k, m, True), _cancelling(n, k, n + 1, False)
    want = _exact(x, w)
    assert want.abs().max() < 65504
    want = want.float().to(getattr(torch, dtype))
    a, b = fa.client_fp8_operand(m, k), fa.client_fp8_operand(n, k)
    fa.client_fp8_quantize(x, a)
    fa.client_fp8_quantize(w, b, block_rows=128)
    ws = torch.empty(fa.client_fp8_workspace_bytes(m, n, k), device="cuda", dtype=torch.uint8).fill_(255)
    out = torch.full_like(want, 7.0)
    fa.client_fp8_matmul(a, b, out, workspace=ws)
    assert torch.equal(out, want)
    out.fill_(7.0)
    fa.client_fp8_linear(x.to(want.dtype), b, out, workspace=ws)
    assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", SIXTEEN)
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("fmt_a, fmt_b", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("m, n, k", [(5, 300, 2000), (64, 130, 1000), (300, 700, 4000), (257, 255, 129)])
def test_full_sums_of_random_operands(dtype, accumulate, fmt_a, fmt_b, m, n, k):
    import torch
    gpu()
    a, b = fa.client_fp8_operand(m, k, FMT[fmt_a]), fa.client_fp8_operand(n, k, FMT[fmt_b])
    fa.client_fp8_quantize(_random(m, k, "float32", m, spread=0.5), a)
    fa.client_fp8_quantize(_random(n, k, "float32", n + 1, spread=0.5), b, block_rows=128)
    out = _random(m, n, dtype, 5)
    before = out.double().cpu().numpy() if accumulate else 0.0
    ws = torch.empty(fa.client_fp8_workspace_bytes(m, n, k), device="cuda", dtype=torch.uint8).fill_(255)
    fa.client_fp8_matmul(a, b, out, accumulate=accumulate, workspace=ws)
    va, vb = _held(a)[0], _held(b)[0]
    want, size = va @ vb.T + before, np.abs(va) @ np.abs(vb).T + np.abs(before)
    bound = ROUND[dtype] * np.abs(want) + (k / 32 + 32) * 2.0 ** -24 * size + 2.0 ** -25 * (dtype == "float16")
    over = np.abs(want) > 65504 if dtype == "float16" else np.zeros_like(want, dtype=bool)
    assert np.all((np.abs(out.double().cpu().numpy() - want) <= bound) | over)


@pytest.mark.parametrize("dtype", SIXTEEN)
@pytest.mark.parametrize("fmt_a, fmt_b", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("m, n, k", [(1, 700, 300), (16, 64, 1000), (31, 100, 260), (64, 65, 128), (100, 257, 2000),
                                     (128, 128, 4100), (300, 513, 640), (2975, 2897, 1537), (4097, 2001, 2049),
                                     (4096, 4096, 256)])
def test_short_sums_of_integers_are_exact(dtype, fmt_a, fmt_b, m, n, k):
    import torch
    gpu()
    a, b, want = _integers(m, n, k, dtype, fmt_a, fmt_b)
    out = torch.full_like(want, 7.0)
    ws = torch.empty(fa.client_fp8_workspace_bytes(m, n, k), device="cuda", dtype=torch.uint8).fill_(255)
    fa.client_fp8_matmul(a, b, out, workspace=ws, short_sums=True)
    assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", SIXTEEN)
@pytest.mark.parametrize("m, n, k, pad", [(1, 1000, 784, 0), (16, 130, 2056, 3), (27, 500, 1200, 0), (64, 300, 515, 3),
                                          (150, 700, 784, 0)])
def test_short_sums_are_within_their_bound(dtype, m, n, k, pad):
    import torch
    gpu()
    x, w = _random(m, k, dtype, m, pad, pad), _random(n, k, "float32", n, spread=0.5)
    b = fa.client_fp8_operand(n, k)
    fa.client_fp8_quantize(w, b, block_rows=128)
    ws = torch.empty(fa.client_fp8_workspace_bytes(m, n, k), device="cuda", dtype=torch.uint8).fill_(255)
    va, vb = ref.held(x.double().cpu().numpy(), "e4m3")[0], _held(b)[0]
    want, size = va @ vb.T, np.abs(va) @ np.abs(vb).T
    bound = _bound(va, vb, want, size, dtype, k)
    over = np.abs(want) > 65504 if dtype == "float16" else np.zeros_like(want, dtype=bool)
    out = torch.empty(m, n + pad, device="cuda", dtype=getattr(torch, dtype))[:, :n]
    fa.client_fp8_linear(x, b, out, workspace=ws, short_sums=True)
    assert np.all((np.abs(out.double().cpu().numpy() - want) <= bound) | over)
    a = fa.client_fp8_operand(m, k)
    fa.client_fp8_quantize(x, a)
    out.fill_(1.0)
    fa.client_fp8_matmul(a, b, out, accumulate=True, workspace=ws, short_sums=True)
    got = out.double().cpu().numpy()
    assert np.all((np.abs(got - want - 1) <= bound + ROUND[dtype] + 2.0 ** -24) | over)


def test_short_sums_are_refused_for_fp32_and_marshalled_alike(both):  # noqa: F811
    import torch
    x, w = torch.randn(20, 300, device="cuda").half(), torch.randn(50, 300, device="cuda")
    a, b = fa.client_fp8_operand(20, 300), fa.client_fp8_operand(50, 300)
    fa.client_fp8_quantize(x, a)
    fa.client_fp8_quantize(w, b, block_rows=128)
    ws = torch.empty(fa.client_fp8_workspace_bytes(20, 50, 300), device="cuda", dtype=torch.uint8)

    def f():
        y, z = (torch.empty(20, 50, device="cuda", dtype=torch.float16) for _ in range(2))
        fa.client_fp8_matmul(a, b, y, workspace=ws, short_sums=True)
        fa.client_fp8_linear(x, b, z, workspace=ws, short_sums=True)
        out = torch.zeros(20, 50, device="cuda")
        for call in (lambda: fa.client_fp8_matmul(a, b, out, workspace=ws, short_sums=True),
                     lambda: fa.client_fp8_linear(x.float(), b, out, workspace=ws, short_sums=True)):
            with pytest.raises(fa.FasgdError, match="short sums"):
                call()
        assert not out.any()
        return [y, z]
    _same(both(f))


@pytest.mark.parametrize("dtype", SIXTEEN[:1] + ["float32"])
@pytest.mark.parametrize("m, n, k", [(1, 40, 128), (3, 100, 3000), (27, 4100, 300), (300, 513, 640)])
def test_values_below_the_normal_range(dtype, m, n, k):
    """Powers of two from 2^-133 on in blocks of the smallest scale, beside values near 2^-117: held, and counted."""
    import torch
    gpu()
    g = torch.Generator(device="cuda").manual_seed(m + n + k)
    a, b = fa.client_fp8_operand(m, k), fa.client_fp8_operand(n, k)
    x = torch.zeros(m, k, device="cuda")
    x[:, 5] = 1.0
    fa.client_fp8_quantize(x, a)
    a.scales[:, :m] = 127 + 96
    q = torch.exp2(torch.randint(-7, 9, (n, k), device="cuda", generator=g).float())
    b.data.zero_()
    b.data[:, :k] = q.to(torch.float8_e4m3fn).view(torch.uint8)
    b.scales.fill_(1)
    want = (_held(a)[0] @ _held(b)[0].T)
    out = torch.full((m, n), 7.0, device="cuda", dtype=getattr(torch, dtype))
    ws = torch.empty(fa.client_fp8_workspace_bytes(m, n, k), device="cuda", dtype=torch.uint8).fill_(255)
    fa.client_fp8_matmul(a, b, out, workspace=ws)
    assert np.array_equal(out.double().cpu().numpy(), want)

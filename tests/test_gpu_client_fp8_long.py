"""GPU: products of up to 16 rows over long contractions, which are split: integers, so that any order of the fp32 sums
is exact."""
import pytest

import paper_1601_04033_amd as fa
from helpers import gpu
from test_gpu_client_fp8 import _integers
from test_gpu_client_fp8_sums import _cancelling, _exact

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype, short", [("float32", False), ("bfloat16", False), ("float16", False), ("bfloat16", True),
                                          ("float16", True)])
@pytest.mark.parametrize("fmt_a, fmt_b", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("m, n, k", [(10, 1000, 8192), (1000, 10, 20_001), (16, 16, 1 << 17), (1, 256, 16_384),
                                     (3, 2001, 15_001), (17, 3, 70_000)])
def test_split_products(dtype, short, fmt_a, fmt_b, m, n, k):
    import torch
    gpu()
    a, b, want = _integers(m, n, k, "float32", fmt_a, fmt_b)
    assert fa.client_fp8_workspace_bytes(m, n, k) >= m * k + 2 * 4 * m * n
    ws = torch.empty(fa.client_fp8_workspace_bytes(m, n, k), device="cuda", dtype=torch.uint8).fill_(255)
    buf = torch.full((m, n + 3), 3.0, device="cuda", dtype=getattr(torch, dtype))
    out = buf[:, :n]
    for add in (False, True):
        before = out.float().clone()
        fa.client_fp8_matmul(a, b, out, accumulate=add, workspace=ws, short_sums=short)
        assert torch.equal(out, (want + before if add else want).to(out.dtype))
    assert (buf[:, n:] == 3).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("m, n, k", [(1, 256, 16_384), (1, 90, 16_301), (2, 300, 8101), (7, 40, 2301), (16, 200, 16_384),
                                     (5, 64, 20_000)])
def test_split_linear_layers(dtype, m, n, k):
    """Activations quantized on the way, each part's own columns, and before."""
    import torch
    gpu()
    x, w = _cancelling(m, k, m, True), _cancelling(n, k, n + 1, False)
    want = _exact(x, w).float().to(getattr(torch, dtype))
    b = fa.client_fp8_operand(n, k)
    fa.client_fp8_quantize(w, b, block_rows=128)
    buf = torch.full((m, k + 5), float("nan"), device="cuda", dtype=want.dtype)
    buf[:, :k] = x
    ws = torch.empty(fa.client_fp8_workspace_bytes(m, n, k), device="cuda", dtype=torch.uint8).fill_(255)
    out = torch.full_like(want, 7.0)
    fa.client_fp8_linear(buf[:, :k], b, out, workspace=ws)
    assert torch.equal(out, want)
    again = torch.full_like(want, 7.0)
    fa.client_fp8_linear(buf[:, :k], b, again, workspace=ws)
    assert torch.equal(again, out)

"""GPU: client_dropout against the 64-bit form.  A kept element is one fp32
product rounded once to the type, so without a residual the result is exact;
with one the sum may be fused, which moves it by at most an fp32 ulp of its
terms before the last rounding."""
import numpy as np
import pytest

import client_reference as ref
import paper_1601_04033_amd as fa
from helpers import gpu

pytestmark = pytest.mark.gpu

ROUND = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}   # half an ulp and more


def _matrix(rows, cols, ld, dtype, seed, offset=0):
    """A [rows, cols] view with row stride ld, `offset` elements into its storage."""
    import torch
    g = torch.Generator().manual_seed(seed)
    buf = torch.full((offset + rows * ld + 8,), 7.0, dtype=dtype)
    v = buf[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    v.copy_(torch.randn(rows, cols, generator=g))
    dev = buf.cuda()
    return dev, dev[offset:offset + rows * ld].view(rows, ld)[:, :cols]


def _expected(x, mask, p, dtype):
    import torch
    scale = np.float32(65536.0 / (65536 - ref.threshold(p))) if ref.threshold(p) < 65536 else np.float32(0)
    y = x.float().cpu().numpy() * scale
    return torch.from_numpy(np.where(mask, y, np.float32(0))).to(dtype)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("rows, cols, ld, offset", [
    (1, 1, 1, 0), (1, 7, 7, 0), (1, 8, 8, 1), (3, 5, 5, 0), (17, 1, 3, 2), (33, 1001, 1024, 0), (33, 1001, 1003, 3),
    (64, 1000, 1000, 0), (5, 4096, 4104, 0), (130, 129, 129, 0), (2, 20_000, 20_000, 0),
])
def test_dropout_is_exact(dtype, rows, cols, ld, offset):
    import torch
    gpu()
    dt = getattr(torch, dtype)
    p, seed, T, client, site, base = 0.3, 0x1234_5678_9ABC_DEF0, 77, 5, 3, 8 * 13
    _, x = _matrix(rows, cols, ld, dt, rows + cols, offset)
    obuf, out = _matrix(rows, cols, ld, dt, 1, offset)
    before = obuf.clone()
    fa.client_dropout(x, out, p, seed, T, client, site=site, index_base=base)
    torch.cuda.synchronize()
    mask = ref.keep_mask(rows, cols, p, seed, T, client, site, base)
    assert torch.equal(out.cpu(), _expected(x, mask, p, dt))
    # nothing outside the matrix is written
    out.fill_(7.0)
    before.copy_(torch.where(before == before, 7.0, before))
    assert torch.equal(obuf, before)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_dropout_with_residual_in_place(dtype):
    import torch
    gpu()
    dt = getattr(torch, dtype)
    rows, cols = 37, 203
    _, x = _matrix(rows, cols, cols, dt, 3)
    _, res = _matrix(rows, cols, 208, dt, 4)
    p, key = 0.5, (42, 9, 0, 0)
    mask = ref.keep_mask(rows, cols, p, *key)
    xs = np.where(mask, x.double().cpu().numpy() * 2.0, 0.0)
    want = xs + res.double().cpu().numpy()
    out = torch.empty_like(x)
    fa.client_dropout(x, out, p, *key[:3], site=key[3], residual=res)
    bound = ROUND[dtype] * np.abs(want) + 2.0 ** -24 * (np.abs(xs) + res.double().abs().cpu().numpy())
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= bound)
    fa.client_dropout(x, x, p, *key[:3], site=key[3], residual=res)     # in place
    assert torch.equal(x, out)
    y = res.clone()
    fa.client_dropout(out, y, p, *key[:3], site=key[3], residual=res)
    fa.client_dropout(out, res, p, *key[:3], site=key[3], residual=res)  # into the residual
    assert torch.equal(res.contiguous(), y.contiguous())


def test_dropped_values_do_not_matter():
    """NaN and infinities that are dropped leave 0; kept ones pass through."""
    import torch
    gpu()
    rows, cols, p, key = 9, 257, 0.4, (7, 1, 2, 0)
    mask = torch.from_numpy(ref.keep_mask(rows, cols, p, *key))
    for bad in (float("nan"), float("inf"), float("-inf")):
        x = torch.ones(rows, cols)
        x[~mask] = bad
        d = x.cuda()
        fa.client_dropout(d, d, p, *key[:3])
        assert torch.equal((d.cpu() != 0), mask)
        x = torch.where(mask, bad, 1.0).cuda()
        fa.client_dropout(x, x, p, *key[:3])
        assert torch.equal(torch.isfinite(x.cpu()), ~mask)


@pytest.mark.parametrize("p", [0.0, 1e-6, 0.5, 1.0 - 1e-6, 1.0])
def test_probability_limits(p):
    import torch
    gpu()
    x = torch.full((100, 100), 3.0, device="cuda")
    out = torch.empty_like(x)
    fa.client_dropout(x, out, p, 5, 0, 0)
    if ref.threshold(p) == 0:
        assert torch.equal(out, x)
    elif ref.threshold(p) == 65536:
        assert not out.any()
    else:
        # binomial: six standard deviations
        kept = (out != 0).double().mean().item()
        assert abs(kept - (1 - p)) < 6 * (p * (1 - p) / x.numel()) ** 0.5 + 2.0 ** -16


def test_masks_follow_their_key_and_index():
    """Every part of the key changes the mask; a part of a matrix at its index draws what the whole draws."""
    import torch
    gpu()
    x = torch.ones(64, 512, device="cuda")

    def mask(seed=1, T=2, client=3, site=4, base=0, a=x):
        out = torch.empty_like(a)
        fa.client_dropout(a, out, 0.5, seed, T, client, site=site, index_base=base)
        return out != 0

    m = mask()
    assert torch.equal(m, mask())
    for other in (dict(seed=2), dict(seed=1 + (1 << 32)), dict(T=3), dict(client=4), dict(site=5), dict(base=8)):
        assert 0.4 < (m != mask(**other)).double().mean().item() < 0.6
    assert torch.equal(m[20:], mask(base=20 * 512, a=x[20:]))


def test_large_index_and_size():
    """Indexes beyond 32 bits: the last elements of the index range, and a matrix of more than 2^32 elements."""
    import torch
    gpu()
    base = 2 ** 51 - 1024
    x = torch.ones(4, 256, device="cuda")
    out = torch.empty_like(x)
    fa.client_dropout(x, out, 0.5, 11, 2 ** 32 - 1, 2 ** 31 - 1, site=16383, index_base=base)
    want = ref.keep_mask(4, 256, 0.5, 11, 2 ** 32 - 1, 2 ** 31 - 1, 16383, base)
    assert np.array_equal((out != 0).cpu().numpy(), want)
    rows, cols = 66_101, 65_001        # 4.2966e9 elements (more than 2^32) of 2 bytes
    x = torch.ones(rows, cols, device="cuda", dtype=torch.float16)
    fa.client_dropout(x, x, 0.5, 11, 1, 2)
    # the last row again, as a matrix of its own that starts at a multiple of 8
    i0 = (rows - 1) * cols
    head = i0 % 8
    tail = torch.ones(1, cols + head, device="cuda", dtype=torch.float16)
    fa.client_dropout(tail, tail, 0.5, 11, 1, 2, index_base=i0 - head)
    assert torch.equal(x[-1], tail[0, head:])


def test_other_stream():
    import torch
    gpu()
    x = torch.randn(512, 512, device="cuda")
    a, b = torch.empty_like(x), torch.empty_like(x)
    fa.client_dropout(x, a, 0.5, 1, 2, 3)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    fa.client_dropout(x, b, 0.5, 1, 2, 3, stream=s)
    s.synchronize()
    assert torch.equal(a, b)


def test_more_elements_than_a_launch():
    """A matrix of more elements (2^35 and three rows) than the threads of one launch cover, 64 GB."""
    import torch
    gpu()
    rows, cols = 2 ** 20 + 3, 2 ** 15
    x = torch.ones(rows, cols, device="cuda", dtype=torch.bfloat16)
    fa.client_dropout(x, x, 0.5, 77, 5, 3, site=1)
    for first in (0, 2 ** 18, 2 ** 19 - 1, 2 ** 19, 2 ** 20 - 1, rows - 1):
        part = torch.ones(1, cols, device="cuda", dtype=torch.bfloat16)
        fa.client_dropout(part, part, 0.5, 77, 5, 3, site=1, index_base=first * cols)
        assert torch.equal(x[first], part[0]), first
    want = ref.keep_mask(1, cols, 0.5, 77, 5, 3, 1, (rows - 1) * cols)
    assert np.array_equal(x[rows - 1].cpu().float().numpy() != 0, want[0])

"""Limits of the client's calls, checked on the host: what is beyond them is
rejected before anything is enqueued (so these calls never touch a device)."""
import ctypes
import os

import numpy as np
import pytest

import paper_1601_04033_amd as fa
from paper_1601_04033_amd import client

ARG = 2
BUF = np.zeros(64, np.float32)
P = (BUF.ctypes.data + 15) & ~15       # stands in for device memory: no call below reaches a launch


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fa.LIB_PATH):
        from paper_1601_04033_amd import _build
        _build.build()
    return client.bind(fa.load_library())


@pytest.mark.parametrize("m, n, k", [(2 ** 27 + 1, 1, 1), (2 ** 28, 16, 128), (2 ** 30, 1, 100)])
def test_linear_takes_as_many_rows_as_an_operand(lib, m, n, k):
    """From 2^28 rows on, a narrow layer's product would be a launch of 2^32 threads, behind a quantization that is
    already enqueued."""
    w = client.client_fp8_operand_struct(P, P, n, k, -(-k // 128) * 128, -(-n // 4) * 4, 0)
    assert lib.client_fp8_linear(P, k, m, ctypes.byref(w), P, n, 1, P, 2 ** 62, None) == ARG
    assert b"m = " in lib.fasgd_last_error()


def test_short_sums_are_of_16_bit_outputs(lib):
    """The flag in an output's type: taken with the 16-bit types, rejected with fp32 and with what is no type."""
    a = client.client_fp8_operand_struct(P, P, 4, 100, 128, 4, 0)
    ref = ctypes.byref(a)
    for dtype, text in ((0x100, b"short sums"), (0x103, b"dtype"), (0x201, b"dtype"), (-1, b"dtype")):
        assert lib.client_fp8_matmul(ref, ref, P, 4, dtype, 0, P, 1 << 20, None) == ARG
        assert text in lib.fasgd_last_error()
        assert lib.client_fp8_linear(P, 100, 4, ref, P, 4, dtype, P, 1 << 20, None) == ARG
        assert text in lib.fasgd_last_error()
    for dtype in (0x101, 0x102):        # as far as the next check
        assert lib.client_fp8_matmul(ref, ref, P, 3, dtype, 0, P, 1 << 20, None) == ARG
        assert b"row stride" in lib.fasgd_last_error()


@pytest.mark.parametrize("m, n, k", [(10, 1000, 65_536), (1000, 10, 65_536), (16, 16, 2 ** 20), (1, 256, 16_384)])
def test_long_contractions_of_few_outputs_are_split(lib, m, n, k):
    """Where 16 rows a block leave most of the 256 CUs idle, the workspace has room for parts of the contraction."""
    x = m * k + k // 128 * m
    assert fa.client_fp8_workspace_bytes(m, n, k) - x >= 4 * 4 * m * n
    assert fa.client_fp8_workspace_bytes(16, 9000, k) - 16 * k - k // 128 * 16 < 4 * 4 * 16 * 9000

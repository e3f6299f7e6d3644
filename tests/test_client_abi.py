"""The client's C ABI without a GPU: every function include/fasgd_client.h
declares is exported and bound, and the host-side checks reject bad arguments
before any launch (so these calls never touch a device)."""
import ctypes
import os
import re

import numpy as np
import pytest

import paper_1601_04033_amd as fa
from paper_1601_04033_amd import client

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "fasgd_client.h")
NULL, ARG, CLIENT, ALIGN, CAPACITY = 1, 2, 4, 5, 6


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fa.LIB_PATH):
        from paper_1601_04033_amd import _build
        _build.build()
    return client.bind(fa.load_library())


def test_header_binding_and_library_agree(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    declared = set(re.findall(r"^\s*(?:const\s+)?[a-z_0-9]+\s*\*?\s*(client_[a-z_0-9]+)\s*\(", text, flags=re.M))
    assert declared == set(fa.CLIENT_ABI_FUNCTIONS)
    for name in declared:
        assert hasattr(lib, name), name


BUF = np.zeros(4096, np.float32)
P = (BUF.ctypes.data + 15) & ~15       # stands in for device memory: no call below reaches a launch


def _dropout(lib, x=P, ldx=8, r=None, ldr=0, y=P, ldy=8, rows=4, cols=8, dtype=0, p=0.5, seed=1, T=0, c=0, site=0, base=0):
    return lib.client_dropout(x, ldx, r, ldr, y, ldy, rows, cols, dtype, p, seed, T, c, site, base, None)


@pytest.mark.parametrize("args, status, text", [
    (dict(x=None), NULL, b"x is NULL"), (dict(y=None), NULL, b"y is NULL"),
    (dict(x=P + 2), ALIGN, b"x"), (dict(r=P + 1, ldr=8, dtype=1), ALIGN, b"residual"),
    (dict(ldx=7), ARG, b"row stride 7"), (dict(ldy=-8), ARG, b"row stride"), (dict(ldx=2 ** 62), ARG, b"row stride"),
    (dict(dtype=3), ARG, b"dtype"), (dict(dtype=-1), ARG, b"dtype"),
    (dict(rows=-1), ARG, b"rows"), (dict(cols=-1), ARG, b"cols"), (dict(rows=2 ** 30, cols=2 ** 30), ARG, b"2^40"),
    (dict(rows=2 ** 62, cols=0), ARG, b"2^40"),
    (dict(p=-0.1), ARG, b"p must"), (dict(p=1.1), ARG, b"p must"), (dict(p=float("nan")), ARG, b"p must"),
    (dict(T=-1), ARG, b"T ="), (dict(T=2 ** 32), ARG, b"T ="), (dict(c=-1), CLIENT, b"client"),
    (dict(site=-1), ARG, b"site"), (dict(site=16384), ARG, b"site"),
    (dict(base=4), ARG, b"index_base"), (dict(base=-8), ARG, b"index_base"), (dict(base=2 ** 51 - 24), ARG, b"index_base"),
])
def test_dropout_rejects(lib, args, status, text):
    assert _dropout(lib, **args) == status
    assert text in lib.fasgd_last_error()


def test_empty_calls_enqueue_nothing(lib):
    assert _dropout(lib, x=None, y=None, rows=0) == 0
    assert _dropout(lib, x=None, y=None, cols=0) == 0
    assert lib.fasgd_last_error() == b""
    op = _op(rows=0)
    assert lib.client_residual_norm_forward(ctypes.byref(op), None, 0, None, 0, None, 0, None, 0, None, None) == 0


def _op(**kw):
    op = fa.client.client_residual_norm()
    op.rows, op.cols, op.dtype, op.kind = 4, 8, 0, 0
    op.w_post = op.w_pre = P
    op.residual_scale, op.eps = 1.0, 1e-5
    for k, v in kw.items():
        setattr(op, k, v)
    return op


def _forward(lib, op, branch=P, lb=8, res=P, lr=8, total=P, ls=8, normed=P, ln=8, stats=P):
    return lib.client_residual_norm_forward(ctypes.byref(op), branch, lb, res, lr, total, ls, normed, ln, stats, None)


def _backward(lib, op, branch=P, total=P, stats=P, dsum=P, dh=P, db=P, dr=P, dwp=P, dbp=None, dg=None, dwn=P, dbn=None,
              ws=P, n=1 << 20, ld=8):
    return lib.client_residual_norm_backward(ctypes.byref(op), branch, ld, total, ld, stats, dsum, ld, dh, ld, db, ld,
                                             dr, ld, dwp, dbp, dg, ld, dwn, dbn, ws, n, None)


@pytest.mark.parametrize("fields, status, text", [
    (dict(rows=-1), ARG, b"rows"), (dict(cols=0), ARG, b"cols"), (dict(cols=2 ** 31, rows=1), ARG, b"cols"),
    (dict(dtype=9), ARG, b"dtype"), (dict(kind=2), ARG, b"kind"), (dict(gate_form=4), ARG, b"gate_form"),
    (dict(gate_act=3), ARG, b"gate_act"), (dict(gate_form=1), NULL, b"gate is NULL"),
    (dict(gate_form=3), NULL, b"gate is NULL"), (dict(gate_form=3, gate=P, ld_gate=7), ARG, b"gate: row stride"),
    (dict(gate_form=2, gate=P + 2), ALIGN, b"gate"), (dict(eps=0.0), ARG, b"eps"), (dict(eps=float("nan")), ARG, b"eps"),
    (dict(residual_scale=float("inf")), ARG, b"residual_scale"), (dict(w_post=P + 1), ALIGN, b"w_post"),
    (dict(w_post=None, b_post=P), NULL, b"bias"), (dict(w_pre=None, b_pre=P), NULL, b"bias"),
    (dict(p=2.0), ARG, b"p must"), (dict(site=20000), ARG, b"site"), (dict(client=-3), CLIENT, b"client"),
])
def test_residual_norm_rejects(lib, fields, status, text):
    for call in (_forward, _backward):
        assert call(lib, _op(**fields)) == status
        assert text in lib.fasgd_last_error()


def test_residual_norm_forward_rejects(lib):
    for kw, status, text in [(dict(branch=None), NULL, b"branch"), (dict(total=None), NULL, b"sum"),
                             (dict(normed=None), NULL, b"normed"), (dict(stats=None), NULL, b"stats"),
                             (dict(branch=P + 2), ALIGN, b"branch"), (dict(lr=4), ARG, b"residual: row stride"),
                             (dict(stats=P + 2), ALIGN, b"stats")]:
        assert _forward(lib, _op(), **kw) == status
        assert text in lib.fasgd_last_error()
    assert lib.client_residual_norm_forward(None, P, 8, P, 8, P, 8, P, 8, P, None) == NULL


def test_residual_norm_backward_rejects(lib):
    for kw, status, text in [(dict(branch=None), NULL, b"branch"), (dict(total=None), NULL, b"sum"),
                             (dict(dh=None), NULL, b"dnormed"), (dict(db=None), NULL, b"dbranch"),
                             (dict(stats=None), NULL, b"stats"), (dict(ws=None), NULL, b"workspace"),
                             (dict(ws=P + 8), ALIGN, b"workspace"), (dict(n=16), CAPACITY, b"workspace"),
                             (dict(dbp=P), ARG, b"absent"), (dict(dwp=P + 2), ALIGN, b"dw_post"),
                             (dict(ld=4), ARG, b"row stride")]:
        assert _backward(lib, _op(), **kw) == status, kw
        assert text in lib.fasgd_last_error()
    assert _backward(lib, _op(w_pre=None), dwn=None) == ARG       # dnormed without its norm
    assert _backward(lib, _op(gate_form=2, gate=P), dg=None) == NULL
    assert _backward(lib, _op(gate_form=3, gate=P, ld_gate=8), dg=None) == NULL


def test_workspace_bytes(lib):
    f = fa.client_residual_norm_workspace_bytes
    assert f(0, 100) == 0 and f(-1, 5) == 0
    assert f(1, 100) >= 400 and f(10 ** 6, 100) < 10 ** 6


def test_binding_rejects_host_tensors_and_shapes():
    import torch
    x = torch.zeros(4, 8)
    with pytest.raises(TypeError):
        fa.client_dropout(x, x, 0.5, 1, 0, 0)
    with pytest.raises(TypeError):
        fa.client_residual_norm_forward(x, x, x, x, x)


def _operand(rows=4, k=100, **kw):
    o = fa.client.client_fp8_operand_struct(P, P, rows, k, -(-k // 128) * 128, -(-rows // 4) * 4, 0)
    for name, v in kw.items():
        setattr(o, name, v)
    return o


OPERAND_FAULTS = [(dict(data=None), NULL, b"data"), (dict(scales=None), NULL, b"scales"), (dict(data=P + 8), ALIGN, b"16-byte"),
                  (dict(scales=P + 2), ALIGN, b"scales"), (dict(ld=100), ARG, b"ld ="), (dict(ld=129), ARG, b"ld ="),
                  (dict(ld=2 ** 24), ARG, b"ld ="), (dict(lds=3), ARG, b"lds ="), (dict(lds=6), ARG, b"lds ="),
                  (dict(format=2), ARG, b"format"), (dict(rows=-1), ARG, b"rows"), (dict(k=-1), ARG, b"k ="),
                  (dict(k=2 ** 23 + 1), ARG, b"k =")]


@pytest.mark.parametrize("fault, status, text", OPERAND_FAULTS)
def test_operands_are_checked(lib, fault, status, text):
    good, bad, ref = _operand(), _operand(**fault), ctypes.byref
    calls = [lambda: lib.client_fp8_matmul(ref(bad), ref(good), P, 8, 0, 0, P, 1 << 20, None),
             lambda: lib.client_fp8_matmul(ref(good), ref(bad), P, 8, 0, 0, P, 1 << 20, None),
             lambda: lib.client_fp8_quantize(P, 100, 4, 100, 0, 1, ref(bad), None, None),
             lambda: lib.client_fp8_linear(P, 100, 4, ref(bad), P, 8, 0, P, 1 << 20, None)]
    for call in calls:
        assert call() == status
        assert text in lib.fasgd_last_error()


def test_fp8_calls_reject(lib):
    a, b, ref = _operand(), _operand(6), ctypes.byref

    def matmul(a=a, b=b, c=P, ldc=8, dtype=0, ws=P, n=1 << 20):
        return lib.client_fp8_matmul(ref(a) if a else None, ref(b) if b else None, c, ldc, dtype, 0, ws, n, None)
    assert matmul(a=None) == NULL and matmul(b=None) == NULL and matmul(c=None) == NULL
    assert matmul(c=P + 2) == ALIGN and matmul(ldc=5) == ARG and matmul(dtype=5) == ARG
    assert matmul(b=_operand(6, 101)) == ARG and b"differ in k" in lib.fasgd_last_error()

    def quantize(x=P, ldx=100, rows=4, cols=100, dtype=0, block=1, r=a, t=None):
        return lib.client_fp8_quantize(x, ldx, rows, cols, dtype, block, ref(r) if r else None, ref(t) if t else None, None)
    assert quantize(r=None) == NULL and quantize(x=None) == NULL and quantize(x=P + 1) == ALIGN
    assert quantize(block=64) == ARG and quantize(dtype=-1) == ARG and quantize(ldx=99) == ARG
    assert quantize(rows=5) == ARG and b"by_rows is" in lib.fasgd_last_error()
    assert quantize(t=_operand(100, 5)) == ARG and b"by_cols is" in lib.fasgd_last_error()
    assert quantize(t=_operand(100, 4, format=1)) == ARG and b"format" in lib.fasgd_last_error()

    def linear(x=P, m=4, w=b, y=P, ldy=6, dtype=1, ws=P, n=1 << 20, ldx=100):
        return lib.client_fp8_linear(x, ldx, m, ref(w) if w else None, y, ldy, dtype, ws, n, None)
    assert linear(x=None) == NULL and linear(w=None) == NULL and linear(y=None) == NULL
    assert linear(m=-1) == ARG and linear(ldy=5) == ARG and linear(ldx=99) == ARG
    assert linear(ws=None) == NULL and linear(ws=P + 4) == ALIGN and linear(n=8) == CAPACITY
    # nothing to do
    assert linear(m=0, x=None, y=None, ws=None, n=0) == 0
    assert quantize(rows=0, x=None, r=_operand(0, 100, data=None, scales=None)) == 0
    assert matmul(a=_operand(0), c=None, ws=None, n=0) == 0


def test_fp8_workspace_bytes(lib):
    f = fa.client_fp8_workspace_bytes
    assert f(0, 5, 5) == f(5, 0, 5) == f(5, 5, 0) == f(-1, 5, 5) == f(2 ** 40, 2 ** 40, 2 ** 20) == 0
    assert f(1, 1000, 784) >= 784 and f(8192, 4096, 4096) >= 8192 * 4096

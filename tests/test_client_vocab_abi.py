"""The vocabulary's losses without a GPU: host-side checks reject bad arguments
before any launch (so these calls never touch a device), empty calls enqueue
nothing, and the workspace's size follows the sizes it is asked for."""
import ctypes

import numpy as np
import pytest
import torch

import paper_1601_04033_amd as fa
from paper_1601_04033_amd import client
from test_client_abi import lib  # noqa: F401  (the bound library)

NULL, ARG, ALIGN, CAPACITY = 1, 2, 5, 6
BUF = np.zeros(4096, np.float32)
P = (BUF.ctypes.data + 15) & ~15       # stands in for device memory: no call below reaches a launch
Q = P + 4096                           # gradients


def _call(lib, name, head=(), **kw):
    """One of the four calls with arguments that pass, but for those given."""
    op = client.client_vocab_head()
    op.rows, op.cols, op.vocab, op.dtype, op.logit_scale = 4, 8, 10, 0, 1.0
    op.x, op.ld_x, op.w, op.ld_w = P, 8, P, 8
    for k, v in dict(head).items():
        setattr(op, k, v)
    a = dict(op=ctypes.byref(op), index=P, smoothing=0.0, z_loss=0.0, teacher=P, entries=2, teacher_scale=1.0,
             teacher_lse=None, loss=P, lse=P, picked=P, dloss=None, grad_scale=1.0, dx=Q, ld_dx=8, dw=Q, ld_dw=8,
             dw_dtype=0, accumulate=0, workspace=P, bytes=1 << 40)
    assert not set(kw) - set(a)
    a.update(kw)
    out = ["dloss", "grad_scale", "dx", "ld_dx", "dw", "ld_dw", "dw_dtype", "accumulate"]
    order = {"loss": ["smoothing", "z_loss"], "distill": ["teacher", "entries", "teacher_scale", "teacher_lse"]}[name.split("_")[0]]
    results = ["loss", "lse", "picked"] if name.endswith("forward") else ["lse", "picked"] + out
    args = [a[k] for k in ["op", "index"] + order + results + ["workspace", "bytes"]]
    return getattr(lib, "client_vocab_" + name)(*args, None)


CALLS = ["loss_forward", "loss_backward", "distill_forward", "distill_backward"]
BACKWARD = ["loss_backward", "distill_backward"]


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("head, status, text", [
    (dict(rows=-1), ARG, b"rows"), (dict(rows=2 ** 20 + 1), ARG, b"rows"), (dict(cols=0), ARG, b"cols"),
    (dict(cols=2 ** 16 + 1), ARG, b"cols"), (dict(vocab=0), ARG, b"vocab"), (dict(vocab=2 ** 30 + 1), ARG, b"vocab"),
    (dict(vocab=2 ** 30, cols=2 ** 11), ARG, b"2^40"), (dict(dtype=3), ARG, b"dtype"), (dict(dtype=-1), ARG, b"dtype"),
    (dict(logit_scale=0.0), ARG, b"logit_scale"), (dict(logit_scale=-1.0), ARG, b"logit_scale"),
    (dict(logit_scale=float("nan")), ARG, b"logit_scale"), (dict(logit_scale=float("inf")), ARG, b"logit_scale"),
    (dict(x=None), NULL, b"x is NULL"), (dict(w=None), NULL, b"w is NULL"), (dict(x=P + 2), ALIGN, b"x"),
    (dict(w=P + 1), ALIGN, b"w"), (dict(ld_x=7), ARG, b"row stride 7"), (dict(ld_w=-8), ARG, b"row stride"),
    (dict(ld_w=2 ** 62), ARG, b"row stride"),
])
def test_heads_are_checked(lib, name, head, status, text):  # noqa: F811
    assert _call(lib, name, head, dw_dtype=0) == status
    assert text in lib.fasgd_last_error()


@pytest.mark.parametrize("names, args, status, text", [
    (CALLS, dict(index=None), NULL, b"is NULL"), (CALLS, dict(index=P + 4), ALIGN, b"8-byte"),
    (CALLS, dict(lse=None), NULL, b"lse"), (CALLS, dict(lse=P + 2), ALIGN, b"lse"),
    (CALLS, dict(picked=None), NULL, b"picked"), (CALLS, dict(picked=P + 1), ALIGN, b"picked"),
    (CALLS, dict(workspace=None), NULL, b"workspace"), (CALLS, dict(workspace=P + 8), ALIGN, b"workspace"),
    (CALLS, dict(bytes=15), CAPACITY, b"workspace"),
    (CALLS[::2], dict(loss=None), NULL, b"loss"), (CALLS[::2], dict(loss=P + 2), ALIGN, b"loss"),
    (CALLS[:2], dict(smoothing=-0.1), ARG, b"smoothing"), (CALLS[:2], dict(smoothing=1.1), ARG, b"smoothing"),
    (CALLS[:2], dict(smoothing=float("nan")), ARG, b"smoothing"), (CALLS[:2], dict(z_loss=float("inf")), ARG, b"z_loss"),
    (CALLS[2:], dict(entries=0), ARG, b"entries"), (CALLS[2:], dict(entries=1025), ARG, b"entries"),
    (CALLS[2:], dict(entries=-1), ARG, b"entries"),
    (CALLS[2:], dict(teacher=None), NULL, b"teacher is NULL"), (CALLS[2:], dict(teacher=P + 2), ALIGN, b"teacher"),
    (CALLS[2:], dict(teacher_lse=P + 1), ALIGN, b"teacher_lse"), (CALLS[2:], dict(teacher_scale=0.0), ARG, b"teacher_scale"),
    (CALLS[2:], dict(teacher_scale=float("nan")), ARG, b"teacher_scale"),
    (BACKWARD, dict(grad_scale=float("nan")), ARG, b"grad_scale"), (BACKWARD, dict(dloss=P + 2), ALIGN, b"dloss"),
    (BACKWARD, dict(dw_dtype=1), ARG, b"dw_dtype"), (BACKWARD, dict(dw_dtype=3), ARG, b"dw_dtype"),
    (BACKWARD, dict(dx=Q + 2), ALIGN, b"dx"), (BACKWARD, dict(ld_dx=7), ARG, b"row stride 7"),
    (BACKWARD, dict(dw=Q + 1), ALIGN, b"dw"), (BACKWARD, dict(ld_dw=7), ARG, b"row stride 7"),
    (BACKWARD, dict(dx=P), ARG, b"dx may not be x"), (BACKWARD, dict(dw=P), ARG, b"dw may not be w"),
])
def test_arguments_are_checked(lib, names, args, status, text):  # noqa: F811
    for name in names:
        assert _call(lib, name, **args) == status, name
        assert text in lib.fasgd_last_error()


def test_no_description(lib):  # noqa: F811
    for name in CALLS:
        assert _call(lib, name, op=None) == NULL


def test_calls_without_work_enqueue_nothing(lib):  # noqa: F811
    nothing = dict(index=None, lse=None, picked=None, workspace=None, bytes=0)
    for name in CALLS[::2]:
        assert _call(lib, name, dict(rows=0, x=None, w=None), loss=None, **nothing) == 0
    for name in BACKWARD:
        assert _call(lib, name, dict(rows=0, x=None, w=None), dx=None, dw=None, **nothing) == 0
        assert _call(lib, name, dx=None, dw=None, workspace=None, bytes=0) == 0
    assert lib.fasgd_last_error() == b""


def test_workspace_bytes(lib):  # noqa: F811
    size = lib.client_vocab_workspace_bytes
    for bad in ((0, 8, 8, 0), (2 ** 20 + 1, 8, 8, 0), (1, 0, 8, 0), (1, 2 ** 16 + 1, 8, 0), (1, 8, 0, 0),
                (1, 8, 2 ** 30 + 1, 0), (1, 8, 8, 3), (1, 8, 8, -1)):
        assert size(*bad, 0) == 0 and size(*bad, 1) == 0
    # A long vocabulary goes through in pieces: no logit is kept beyond them.
    rows, cols, vocab = 8192, 4096, 131072
    assert 0 < size(rows, cols, vocab, 1, 0) < 2 * rows * vocab // 4
    assert size(rows, cols, vocab, 1, 1) < 3 * 2 ** 30
    # The vocabulary beyond the pieces costs a forward call its statistics, a backward one nothing.
    assert size(rows, cols, 8 * vocab, 1, 1) <= size(rows, cols, 2 * vocab, 1, 1) + 8 * vocab * 8
    assert size(rows, cols, 4 * vocab, 1, 0) < 4 * size(rows, cols, vocab, 1, 0) + 2 ** 20
    assert size(2 ** 20, 2 ** 16, 2 ** 24, 0, 1) > 2 ** 32


def test_binding_rejects_host_tensors_and_shapes():
    x, w = torch.zeros(4, 8), torch.zeros(10, 8)
    v, t, k = torch.zeros(4), torch.zeros(4, dtype=torch.int64), torch.zeros(4, 2, dtype=torch.int64)
    with pytest.raises(TypeError):
        fa.client_vocab_loss_forward(x, w, t, v, v, v)
    with pytest.raises(TypeError):
        fa.client_vocab_loss_backward(x, w, t, v, v, x, w)
    with pytest.raises(TypeError):
        fa.client_vocab_distill_forward(x, w, k, torch.zeros(4, 2), v, v, torch.zeros(4, 2))
    with pytest.raises(TypeError):
        fa.client_vocab_distill_backward(x, w, k, torch.zeros(4, 2), v, torch.zeros(4, 2), x, w)

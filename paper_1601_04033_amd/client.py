"""Binding of the client's operators (include/fasgd_client.h): dropout, the
residual norm between blocks and 8-bit matrix products, with which a client of
the parameter server turns a fetched theta into its gradient.

Argument marshalling only, as in the package's __init__ (which re-exports
these names): every step runs in the HIP kernels of libfasgd.so, there is no
fallback, and no call allocates.  Plain arguments are marshalled natively
(csrc/marshal.cpp), others below, with the same library call.  Activations are CUDA (HIP) tensors of one
dtype (float32, bfloat16 or float16) of one or two dimensions whose last
stride is 1 (rows may lie apart); parameters and their gradients are
contiguous float32 tensors.
"""
from __future__ import annotations

import ctypes

# every function include/fasgd_client.h declares
CLIENT_ABI_FUNCTIONS = ("client_dropout", "client_residual_norm_workspace_bytes", "client_residual_norm_forward",
                        "client_residual_norm_backward", "client_fp8_workspace_bytes", "client_fp8_quantize",
                        "client_fp8_matmul", "client_fp8_linear")

FP8_E4M3 = 0
FP8_E5M2 = 1
_FP8_SHORT_SUMS = 0x100

NORM_RMS = 0
NORM_LAYER = 1
GATE_IDENTITY = 0
GATE_SIGMOID = 1
GATE_TANH = 2
_GATE_NONE, _GATE_CHANNEL, _GATE_ROW, _GATE_FULL = 0, 1, 2, 3



class client_residual_norm(ctypes.Structure):
    """Mirror of the C struct client_residual_norm."""
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("kind", ctypes.c_int32), ("w_post", ctypes.c_void_p), ("b_post", ctypes.c_void_p),
                ("w_pre", ctypes.c_void_p), ("b_pre", ctypes.c_void_p), ("gate", ctypes.c_void_p),
                ("ld_gate", ctypes.c_int64), ("gate_form", ctypes.c_int32), ("gate_act", ctypes.c_int32),
                ("residual_scale", ctypes.c_float), ("eps", ctypes.c_float), ("p", ctypes.c_double),
                ("seed", ctypes.c_uint64), ("T", ctypes.c_int64), ("client", ctypes.c_int32),
                ("site", ctypes.c_int32), ("index_base", ctypes.c_int64)]


class client_fp8_operand_struct(ctypes.Structure):
    """Mirror of the C struct client_fp8_operand."""
    _fields_ = [("data", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("k", ctypes.c_int64), ("ld", ctypes.c_int64), ("lds", ctypes.c_int64), ("format", ctypes.c_int32)]


_DTYPES = None
_lib = None


def _library():
    global _lib
    if _lib is None:
        from . import load_library
        _lib = bind(load_library())
    return _lib


def bind(lib):
    """Sets the argument types of the client's functions of a loaded library."""
    P = ctypes.c_void_p
    i32, i64, u64, d = ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_double
    lib.client_dropout.argtypes = [P, i64, P, i64, P, i64, i64, i64, i32, d, u64, i64, i32, i32, i64, P]
    N = ctypes.POINTER(client_residual_norm)
    sz = ctypes.c_size_t
    lib.client_residual_norm_forward.argtypes = [N, P, i64, P, i64, P, i64, P, i64, P, P]
    lib.client_residual_norm_backward.argtypes = [N, P, i64, P, i64, P, P, i64, P, i64, P, i64, P, i64,
                                                  P, P, P, i64, P, P, P, sz, P]
    lib.client_residual_norm_workspace_bytes.argtypes = [i64, i64]
    O = ctypes.POINTER(client_fp8_operand_struct)
    lib.client_fp8_workspace_bytes.argtypes = [i64, i64, i64]
    lib.client_fp8_quantize.argtypes = [P, i64, i64, i64, i32, i32, O, O, P]
    lib.client_fp8_matmul.argtypes = [O, O, P, i64, i32, i32, P, sz, P]
    lib.client_fp8_linear.argtypes = [P, i64, i64, O, P, i64, i32, P, sz, P]
    for name in CLIENT_ABI_FUNCTIONS:
        getattr(lib, name).restype = sz if name.endswith("_bytes") else ctypes.c_int
    return lib


_calls = None     # module _marshal with the client's entry points bound, or what stands in for it


def _native():
    global _calls
    if _calls is None:
        from . import _native as package_native
        m = package_native()
        if hasattr(m, "CLIENT_ENTRY_POINTS") and isinstance(m.CLIENT_ENTRY_POINTS, tuple):
            lib = _library()
            m.bind_client([ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in m.CLIENT_ENTRY_POINTS])
        _calls = m
    return _calls


def _check(rc: int):
    if rc != 0:
        from . import FasgdError
        raise FasgdError(rc, _library().fasgd_last_error().decode())


def _stream(stream):
    from . import _stream as of
    return of(stream)


def _dtype(t, name):
    """client_dtype of a tensor."""
    global _DTYPES
    if _DTYPES is None:
        import torch
        _DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32, bfloat16 or float16, not {t.dtype}")
    return code


def _matrix(t, name, like=None):
    """(pointer, row stride) of a 1-D or 2-D tensor whose last stride is 1 and whose dtype and shape are like's."""
    import torch
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda":
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if like is not None and t is not like:
        if t.dtype != like.dtype:
            raise TypeError(f"{name} is {t.dtype}, expected {like.dtype}")
        if t.shape != like.shape:
            raise ValueError(f"{name} is {tuple(t.shape)}, expected {tuple(like.shape)}")
    dim = t.dim()
    if dim == 2:
        ld, last = t.stride()
        rows, cols = t.shape
        if last != 1 and cols > 1:
            raise TypeError(f"{name} must have a last stride of 1")
        return t.data_ptr(), (ld if rows > 1 else cols)
    if dim == 1:
        if t.stride(0) != 1 and t.numel() > 1:
            raise TypeError(f"{name} must have a last stride of 1")
        return t.data_ptr(), t.numel()
    raise ValueError(f"{name} must have one or two dimensions")


def _shape(t):
    return tuple(t.shape) if t.dim() == 2 else (1, t.numel())


def client_dropout(x, out, p: float, seed: int, T: int, client: int, site: int = 0, residual=None,
                   index_base: int = 0, stream=None) -> None:
    """out = [residual +] dropout(x) with the mask drawn from (seed, T, client,
    site, index); the backward pass is the same call on the gradient, without
    residual.  out may be x or residual."""
    rc = (_calls or _native()).client_dropout(x, out, p, seed, T, client, site, residual, index_base, stream)
    if rc is not None:
        return _check(rc) if rc else None
    px, ldx = _matrix(x, "x")
    py, ldy = _matrix(out, "out", x)
    pr, ldr = (None, 0) if residual is None else _matrix(residual, "residual", x)
    rows, cols = _shape(x)
    _check(_library().client_dropout(px, ldx, pr, ldr, py, ldy, rows, cols, _dtype(x, "x"), p,
                                     int(seed) & (2 ** 64 - 1), int(T), int(client), int(site), int(index_base),
                                     _stream(stream)))


def _vector(t, name, n):
    """Pointer of a contiguous float32 tensor of n elements, or None."""
    import torch
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda":
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if t.dtype != torch.float32 or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous float32 tensor")
    if t.numel() != n:
        raise ValueError(f"{name} has {t.numel()} elements, expected {n}")
    return t.data_ptr()


def _gate(gate, like, rows, cols):
    """(form, pointer, row stride) of a gate: float32 [cols] (per channel), float32 [rows, 1] (per row), or a matrix
    of the activations' shape and dtype."""
    import torch
    if gate is None:
        return _GATE_NONE, None, 0
    if gate.shape == like.shape and gate.dtype == like.dtype and (gate.dim() == 2 or gate.dtype != torch.float32):
        p, ld = _matrix(gate, "gate", like)
        return _GATE_FULL, p, ld
    if gate.dim() == 1:
        return _GATE_CHANNEL, _vector(gate, "gate", cols), 0
    if tuple(gate.shape) == (rows, 1):
        return _GATE_ROW, _vector(gate, "gate", rows), 0
    raise ValueError(f"gate is {tuple(gate.shape)} {gate.dtype}: expected float32 [cols] or [rows, 1], or the "
                     f"activations' {tuple(like.shape)} {like.dtype}")


def _norm_op(branch, kind, w_post, b_post, gate, gate_act, w_pre, b_pre, residual_scale, eps, dropout, index_base):
    rows, cols = _shape(branch)
    op = client_residual_norm()
    op.rows, op.cols, op.dtype, op.kind = rows, cols, _dtype(branch, "branch"), int(kind)
    op.w_post, op.b_post = _vector(w_post, "w_post", cols), _vector(b_post, "b_post", cols)
    op.w_pre, op.b_pre = _vector(w_pre, "w_pre", cols), _vector(b_pre, "b_pre", cols)
    op.gate_form, op.gate, op.ld_gate = _gate(gate, branch, rows, cols)
    op.gate_act, op.residual_scale, op.eps, op.index_base = int(gate_act), residual_scale, eps, int(index_base)
    if dropout is not None:
        op.p, seed, op.T, op.client, op.site = dropout
        op.seed = int(seed) & (2 ** 64 - 1)
    return op


def _optional(t, name, like):
    return (None, 0) if t is None else _matrix(t, name, like)


def _stats(stats, rows):
    if stats.numel() != 4 * rows:
        raise ValueError(f"stats has {stats.numel()} elements, expected 4 per row = {4 * rows}")
    return _vector(stats, "stats", 4 * rows)


def client_residual_norm_workspace_bytes(rows: int, cols: int) -> int:
    return int(_library().client_residual_norm_workspace_bytes(int(rows), int(cols)))


def client_residual_norm_forward(branch, residual, sum_out, normed, stats, *, kind: int = NORM_RMS, w_post=None,
                                 b_post=None, gate=None, gate_act: int = GATE_IDENTITY, w_pre=None, b_pre=None,
                                 residual_scale: float = 1.0, eps: float = 1e-5, dropout=None, index_base: int = 0,
                                 stream=None) -> None:
    """sum_out = residual_scale residual + drop(act(gate) N_post(branch)) and normed = N_pre(sum_out).

    w_post / w_pre: float32 [cols], None for no norm there (normed is then None too); biases float32 [cols] or None.
    gate: None, float32 [cols] (per channel), float32 [rows, 1] (per row) or a matrix like branch.  residual may be
    None.  dropout: None or (p, seed, T, client, site) as client_dropout takes them.  stats: float32 [rows, 4], kept
    for the backward pass."""
    rc = (_calls or _native()).client_residual_norm_forward(
        branch, residual, sum_out, normed, stats, kind, w_post, b_post, gate, gate_act, w_pre, b_pre, residual_scale,
        eps, dropout, index_base, stream)
    if rc is not None:
        return _check(rc) if rc else None
    op = _norm_op(branch, kind, w_post, b_post, gate, gate_act, w_pre, b_pre, residual_scale, eps, dropout, index_base)
    pb, lb = _matrix(branch, "branch")
    pr, lr = _optional(residual, "residual", branch)
    ps, ls = _matrix(sum_out, "sum_out", branch)
    pn, ln = _optional(normed, "normed", branch)
    _check(_library().client_residual_norm_forward(ctypes.byref(op), pb, lb, pr, lr, ps, ls, pn, ln,
                                                   _stats(stats, op.rows), _stream(stream)))


def client_residual_norm_backward(branch, sum_in, stats, dsum, dnormed, dbranch, dresidual, *, dw_post=None,
                                  db_post=None, dgate=None, dw_pre=None, db_pre=None, workspace=None,
                                  kind: int = NORM_RMS, w_post=None, b_post=None, gate=None,
                                  gate_act: int = GATE_IDENTITY, w_pre=None, b_pre=None, residual_scale: float = 1.0,
                                  eps: float = 1e-5, dropout=None, index_base: int = 0, stream=None) -> None:
    """The gradients of client_residual_norm_forward (same keyword arguments) from those of its sum (dsum, or None)
    and of normed (dnormed, or None without w_pre), into dbranch, dresidual (or None; may be dsum), and where given
    dw_post, db_post, dw_pre, db_pre (float32 [cols]) and dgate (like gate).  workspace: uint8,
    client_residual_norm_workspace_bytes(rows, cols) bytes."""
    rc = (_calls or _native()).client_residual_norm_backward(
        branch, sum_in, stats, dsum, dnormed, dbranch, dresidual, dw_post, db_post, dgate, dw_pre, db_pre, workspace,
        kind, w_post, b_post, gate, gate_act, w_pre, b_pre, residual_scale, eps, dropout, index_base, stream)
    if rc is not None:
        return _check(rc) if rc else None
    import torch
    op = _norm_op(branch, kind, w_post, b_post, gate, gate_act, w_pre, b_pre, residual_scale, eps, dropout, index_base)
    cols = op.cols
    pb, lb = _matrix(branch, "branch")
    ps, ls = _optional(sum_in, "sum_in", branch)
    pd, ld = _optional(dsum, "dsum", branch)
    ph, lh = _optional(dnormed, "dnormed", branch)
    pdb, ldb = _matrix(dbranch, "dbranch", branch)
    pdr, ldr = _optional(dresidual, "dresidual", branch)
    pg, lg = None, 0
    if dgate is not None:
        if gate is None or dgate.shape != gate.shape:
            raise ValueError("dgate must have the gate's shape")
        form, pg, lg = _gate(dgate, branch, op.rows, cols)
        if form != op.gate_form:
            raise TypeError("dgate must have the gate's dtype")
    from . import _dev_ptr
    pw = _dev_ptr(workspace, torch.uint8, "workspace", True)
    _check(_library().client_residual_norm_backward(
        ctypes.byref(op), pb, lb, ps, ls, _stats(stats, op.rows), pd, ld, ph, lh, pdb, ldb, pdr, ldr,
        _vector(dw_post, "dw_post", cols), _vector(db_post, "db_post", cols), pg, lg,
        _vector(dw_pre, "dw_pre", cols), _vector(db_pre, "db_pre", cols), pw,
        0 if workspace is None else workspace.numel(), _stream(stream)))


class Fp8Operand:
    """A matrix [rows, k] held in 8 bits in blocks of 128 along k (the C struct client_fp8_operand) and its tensors:
    data uint8 [rows, k rounded up to 128], scales uint8 [ceil(k / 128), rows rounded up to 4]."""

    def __init__(self, data, scales, rows: int, k: int, fmt: int):
        import torch
        ld, lds = -(-k // 128) * 128, -(-rows // 4) * 4
        for t, name, shape in ((data, "data", (rows, ld)), (scales, "scales", (ld // 128, lds))):
            if not isinstance(t, torch.Tensor) or t.device.type != "cuda":
                raise TypeError(f"{name} must be a CUDA (HIP) tensor")
            if t.dtype != torch.uint8 or not t.is_contiguous():
                raise TypeError(f"{name} must be a contiguous uint8 tensor")
            if tuple(t.shape) != shape:
                raise ValueError(f"{name} is {tuple(t.shape)}, expected {shape}")
        self.data, self.scales, self.rows, self.k, self.format = data, scales, rows, k, fmt
        self.c = client_fp8_operand_struct(data.data_ptr(), scales.data_ptr(), rows, k, ld, lds, fmt)

    def values(self):
        """The fp32 values held, [rows, k] (for inspection; torch operations)."""
        import torch
        q = self.data.view(torch.float8_e4m3fn if self.format == FP8_E4M3 else torch.float8_e5m2).float()
        s = (self.scales[:, :self.rows].int() << 23).view(torch.float32)     # 2^(byte - 127), bytes 1 .. 253
        return (q.view(self.rows, -1, 128) * s.t().unsqueeze(2)).view(self.rows, -1)[:, :self.k]


def client_fp8_operand(rows: int, k: int, fmt: int = FP8_E4M3, device="cuda") -> Fp8Operand:
    """An operand of new, unset tensors."""
    import torch
    f = dict(device=device, dtype=torch.uint8)
    return Fp8Operand(torch.empty(rows, -(-k // 128) * 128, **f), torch.empty(-(-k // 128), -(-rows // 4) * 4, **f),
                      int(rows), int(k), int(fmt))


def client_fp8_workspace_bytes(m: int, n: int, k: int) -> int:
    """Bytes of workspace of client_fp8_matmul and client_fp8_linear for an [m, n] product over k."""
    return int(_library().client_fp8_workspace_bytes(int(m), int(n), int(k)))


def client_fp8_quantize(x, by_rows=None, by_cols=None, block_rows: int = 1, stream=None) -> None:
    """Quantizes x [rows, cols] into the operand by_rows ([rows, k = cols]) and / or by_cols (the transpose,
    [cols, k = rows]); block_rows = 128 takes one scale per 128 x 128 block (weights)."""
    rc = (_calls or _native()).client_fp8_quantize(
        x, None if by_rows is None else by_rows.c, None if by_cols is None else by_cols.c, block_rows, stream)
    if rc is not None:
        return _check(rc) if rc else None
    px, ldx = _matrix(x, "x")
    rows, cols = _shape(x)
    _check(_library().client_fp8_quantize(px, ldx, rows, cols, _dtype(x, "x"), int(block_rows),
                                          None if by_rows is None else ctypes.byref(by_rows.c),
                                          None if by_cols is None else ctypes.byref(by_cols.c), _stream(stream)))


def _workspace(workspace):
    import torch
    from . import _dev_ptr
    if workspace is None:
        return None, 0
    return _dev_ptr(workspace, torch.uint8, "workspace"), workspace.numel()


def _output_type(out, short_sums):
    return _dtype(out, "out") | (_FP8_SHORT_SUMS if short_sums else 0)


def client_fp8_matmul(a: Fp8Operand, b: Fp8Operand, out, accumulate: bool = False, workspace=None, stream=None,
                      short_sums: bool = False) -> None:
    """out [a.rows, b.rows] = a b^T over their common k (accumulate: added to out).  workspace: uint8,
    client_fp8_workspace_bytes(a.rows, b.rows, k) bytes.  Sums are fp32; short_sums (out bfloat16 or float16) takes the
    8-bit matrix instruction at twice the rate, which cuts each 8 products off below 2^-13 of the largest of them."""
    rc = (_calls or _native()).client_fp8_matmul(a.c, b.c, out, accumulate, workspace, stream, short_sums)
    if rc is not None:
        return _check(rc) if rc else None
    pc, ldc = _matrix(out, "out")
    if _shape(out) != (a.rows, b.rows):
        raise ValueError(f"out is {tuple(out.shape)}, expected {(a.rows, b.rows)}")
    pw, nw = _workspace(workspace)
    _check(_library().client_fp8_matmul(ctypes.byref(a.c), ctypes.byref(b.c), pc, ldc, _output_type(out, short_sums),
                                        1 if accumulate else 0, pw, nw, _stream(stream)))


def client_fp8_linear(x, w: Fp8Operand, out, workspace=None, stream=None, short_sums: bool = False) -> None:
    """out [m, w.rows] = x w^T for x [m, w.k] of out's dtype, quantized in e4m3 on the way.  workspace: uint8,
    client_fp8_workspace_bytes(m, w.rows, w.k) bytes.  short_sums as in client_fp8_matmul."""
    rc = (_calls or _native()).client_fp8_linear(x, w.c, out, workspace, stream, short_sums)
    if rc is not None:
        return _check(rc) if rc else None
    px, ldx = _matrix(x, "x")
    py, ldy = _matrix(out, "out")
    if out.dtype != x.dtype:
        raise TypeError(f"out is {out.dtype}, expected {x.dtype}")
    m, k = _shape(x)
    if k != w.k or _shape(out) != (m, w.rows):
        raise ValueError(f"x {tuple(x.shape)} and out {tuple(out.shape)} do not fit weights [{w.rows}, {w.k}]")
    pw, nw = _workspace(workspace)
    _check(_library().client_fp8_linear(px, ldx, m, ctypes.byref(w.c), py, ldy, _output_type(out, short_sums), pw, nw,
                                        _stream(stream)))

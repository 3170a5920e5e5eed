"""Python binding of the layer body with operands in 8-bit floating point (declared in include/sx_f8.h).

As in the package's other calls, the functions only marshal arguments: shapes, types and the device are checked here
(ValueError), everything else by the library (SxError).  Codes are torch.float8_e4m3fn (or uint8) tensors [..][k], scales
uint8 (or torch.float8_e8m0fnu) tensors [..][f8_scale_ld(k)].

Every call takes the rows of a plan (`plan`, with `rows`, `n_rows` and `max_rows` as in gemm_rows), or without a plan all
rows of its arrays, the first n_rows of them where n_rows (an int32 tensor of one entry) is given.  One layer, on one
stream:

    add_rmsnorm_f8(x, a8, a_scale, gamma, eps)
    gemm_f8(a8, a_scale, w_qkv, s_qkv, [q, k, v])
    ... attention -> o
    add_rmsnorm_f8(o, o8, o_scale)                                     # rounded only
    gemm_f8(o8, o_scale, w_out, s_out, x, residual=x)
    add_rmsnorm_f8(x, a8, a_scale, gamma2, eps)
    gemm_f8(a8, a_scale, w_gate_up, s_gate_up, gu)
    silu_mul_f8(gu, f8, f_scale)
    gemm_f8(f8, f_scale, w_down, s_down, x, residual=x)

and where the feed-forward module is a mixture of experts:

    moe_route(logits, ids, weights, offsets, order, workspace)
    gemm_experts_f8(a8, a_scale, w_gate_up, s_gate_up, offsets, order, gu, gather=top_k)
    silu_mul_f8(gu, f8, f_scale, n_rows=offsets[-1:])
    gemm_experts_f8(f8, f_scale, w_down, s_down, offsets, order, y, scatter=True)
    moe_combine(y, weights, x, residual=x)
"""
from __future__ import annotations

import ctypes

import torch

from . import BF16, F32, Plan, _check, lib
from .decode import _device, _int, _need, _on, _opt, _ptr

_BF16, _F32, _I32 = torch.bfloat16, torch.float32, torch.int32
_CODES = (torch.float8_e4m3fn, torch.uint8)
_SCALES = (torch.uint8, torch.float8_e8m0fnu)
_INTS = [ctypes.c_int32 * c for c in range(5)]
_POINTERS = [ctypes.c_void_p * c for c in range(5)]


def _ld(k: int) -> int:
    return (k + 511) // 512 * 4


# (A call's host time is mostly these checks: each tensor's common case is one expression, told apart only where it fails.)

def _matrix(t, dtypes, rows: int, width: int, at: int, what: str):
    """Device pointer of a contiguous [rows][width] tensor (leading dimensions flattened) of one of these types."""
    if t.shape == (rows, width) and t.dtype in dtypes and t.get_device() == at and t.is_contiguous():
        return t.data_ptr()
    if t.dim() < 2 or t.shape[-1] != width or t.numel() != rows * width:
        raise ValueError(f"{what} must be [{rows}][{width}], not {list(t.shape)}")
    _need(t.dtype in dtypes, f"{what} must be {' or '.join(map(str, dtypes))}, not {t.dtype}")
    return _ptr(t, t.dtype, at, what)


def _wide(t, rows: int, at: int, what: str):
    """(pointer, width) of contiguous bfloat16 rows, the trailing dimensions flattened."""
    shape = t.shape
    if len(shape) == 2 and shape[0] == rows and t.dtype is _BF16 and t.get_device() == at and t.is_contiguous():
        return t.data_ptr(), shape[1]
    _need(len(shape) >= 2 and shape[0] == rows, f"{what} must have {rows} rows, not {list(shape)}")
    return _ptr(t, _BF16, at, what), shape[1:].numel()


def _like(t, rows: int, width: int, at: int, what: str):
    """Pointer of bfloat16 rows of this width, or None."""
    if t is None:
        return None
    if t.shape == (rows, width) and t.dtype is _BF16 and t.get_device() == at and t.is_contiguous():
        return t.data_ptr()
    p, w = _wide(t, rows, at, what)
    _need(w == width, f"{what} must be [{rows}][{width}], not {list(t.shape)}")
    return p


def _entries(t, n: int, at: int, what: str):
    """Pointer of an int32 array of at least n entries."""
    if not isinstance(t, torch.Tensor) or t.numel() < n:
        raise ValueError(f"{what} must be an int32 tensor of {n} entries")
    if t.dtype is _I32 and t.get_device() == at and t.is_contiguous():
        return t.data_ptr()
    return _ptr(t, _I32, at, what)


def _index(t, n: int, at: int, what: str):
    """The same; row lists of a plan come as pointers too."""
    return t if t is None or isinstance(t, int) else _entries(t, n, at, what)


def _row_args(plan, rows, n_rows, max_rows, have: int, at: int):
    """(plan handle, rows, n_rows, max_rows) of a call whose arrays have `have` rows."""
    if plan is None:
        if rows is not None:
            raise ValueError("a row list needs a plan")
        n = have if max_rows is None else max_rows
        if not -0x80000000 <= n <= have or n > 0x7fffffff:   # (a negative one is the library's to refuse)
            raise ValueError(f"max_rows {n} exceeds the arrays' {have} rows or 32 bits")
        return None, None, None if n_rows is None else _entries(n_rows, 1, at, "n_rows"), n
    info = plan.info()
    total = info["total_tokens"]
    _need(have == total, f"the arrays have {have} rows, the plan {total} tokens")
    _need(max_rows is not None, "a plan's rows need max_rows")
    return (plan.handle, _index(rows, total, at, "rows"), _index(n_rows, info["n_requests"], at, "n_rows"),
            _int(max_rows, "max_rows"))


def f8_scale_ld(k: int) -> int:
    """Bytes of a scale row of rows of k elements."""
    n = ctypes.c_int32()
    _check(lib().sx_f8_scale_ld(_int(k, "k"), ctypes.byref(n)))
    return n.value


def f8_pack_weight(w, codes, scales, stream=None):
    """w [n][k] (or stacked [experts][n][k], n a multiple of 128) rounded to 8 bits: codes like w, scales [n / 128][ld]."""
    _need(w.dim() >= 2, "w must be [n][k]")
    at, k = _device(w), w.shape[-1]
    n = w.numel() // k if k else 0
    _need(w.shape[-2] % 128 == 0 or w.dim() == 2, "a stacked weight's parts must be multiples of 128")
    _check(lib().sx_f8_pack_weight(_ptr(w, _BF16, at, "w"), n, _int(k, "k"), _matrix(codes, _CODES, n, k, at, "codes"),
                                   _matrix(scales, _SCALES, n // 128, _ld(k), at, "scales"), _on(stream, at)))


def add_rmsnorm_f8(x, y8, y_scale, gamma=None, eps: float = 1e-6, delta=None, x_out=None, y16=None, plan: Plan = None,
                   rows=None, n_rows=None, max_rows=None, x_by_token=False, y_by_token=False, stream=None):
    """s = x + delta (kept in x_out, which may be x), y = RMSNorm(s) * gamma (gamma None: y = s) into y8 and y_scale (None:
    not) and, in bfloat16, into y16."""
    at, have = _device(x), x.shape[0]
    xp, h = _wide(x, have, at, "x")
    if y8 is None or y_scale is None:
        _need(y8 is y_scale, "y8 and y_scale come together")
        yp = sp = None
    else:
        yp, sp = _matrix(y8, _CODES, have, h, at, "y8"), _matrix(y_scale, _SCALES, have, _ld(h), at, "y_scale")
    if gamma is not None and gamma.numel() != h:
        raise ValueError(f"gamma must have {h} elements")
    p, rp, np_, m = _row_args(plan, rows, n_rows, max_rows, have, at)
    _check(lib().sx_add_rmsnorm_f8(
        p, rp, np_, m, xp, 1 if x_by_token else 0, _like(delta, have, h, at, "delta"), _opt(gamma, _BF16, at, "gamma"), eps, h,
        _like(x_out, have, h, at, "x_out"), _like(y16, have, h, at, "y16"), yp, sp, 1 if y_by_token else 0, _on(stream, at)))


def silu_mul_f8(gate_up, y8, y_scale, plan: Plan = None, n_rows=None, max_rows=None, stream=None):
    """y = silu(gate) * up of rows [gate | up] of gate_up [..][2f], in 8 bits."""
    at, have = _device(gate_up), gate_up.shape[0]
    gp, w = _wide(gate_up, have, at, "gate_up")
    f = y8.shape[-1]
    yp, sp = _matrix(y8, _CODES, have, f, at, "y8"), _matrix(y_scale, _SCALES, have, _ld(f), at, "y_scale")
    if w != 2 * f:
        raise ValueError(f"gate_up must be [{have}][{2 * f}], not {list(gate_up.shape)}")
    p, _, np_, m = _row_args(plan, None, n_rows, max_rows, have, at)
    _check(lib().sx_silu_mul_f8(p, np_, m, gp, f, yp, sp, _on(stream, at)))


def gemm_f8(x8, x_scale, w8, w_scale, y, residual=None, plan: Plan = None, rows=None, n_rows=None, max_rows=None,
            x_by_token=False, y_by_token=False, stream=None):
    """y[row] = x[row] @ w.T (+ residual[row], which may be y); y: a bfloat16 tensor [..][n], or a list of up to four for a
    weight of stacked parts."""
    ys = list(y) if isinstance(y, (list, tuple)) else [y]
    _need(1 <= len(ys) <= 4, "y must be one to four tensors")
    at, have = _device(x8), x8.shape[0]
    k = x8.shape[-1]
    xp, xsp = _matrix(x8, _CODES, have, k, at, "x8"), _matrix(x_scale, _SCALES, have, _ld(k), at, "x_scale")
    outs = [_wide(t, have, at, "y") for t in ys]
    n = _int(sum([w for _, w in outs]), "the parts' width")
    wp = _matrix(w8, _CODES, n, k, at, "w8")
    wsp = _matrix(w_scale, _SCALES, n // 128, _ld(k), at, "w_scale")
    p, rp, np_, m = _row_args(plan, rows, n_rows, max_rows, have, at)
    c = len(ys)
    _check(lib().sx_gemm_f8(
        p, rp, np_, m, xp, xsp, 1 if x_by_token else 0, wp, wsp, k, c, _INTS[c](*[w for _, w in outs]),
        _like(residual, have, n, at, "residual"), _POINTERS[c](*[q for q, _ in outs]), 1 if y_by_token else 0, _on(stream, at)))


def moe_route_workspace(n_experts: int, top_k: int, max_rows: int, n_requests: int = 1) -> int:
    """Bytes of workspace that moe_route needs."""
    n = ctypes.c_int64()
    _check(lib().sx_moe_route_workspace(_int(n_experts, "n_experts"), _int(top_k, "top_k"), _int(n_requests, "n_requests"),
                                        _int(max_rows, "max_rows"), ctypes.byref(n)))
    return n.value


def moe_route(logits, ids, weights, offsets, order, workspace, renormalise=True, plan: Plan = None, n_rows=None,
              max_rows=None, stream=None):
    """ids, weights [..][top_k] of the rows' top experts by logits [..][experts] (float32 or bfloat16), and their places
    grouped by expert: offsets [experts + 1], order [rows * top_k]."""
    at, have = _device(logits), logits.shape[0]
    if logits.dim() != 2 or ids.dim() != 2:
        raise ValueError("logits must be [rows][experts] and ids [rows][top_k]")
    dtype, e, top = logits.dtype, logits.shape[1], ids.shape[1]
    if dtype is not _F32 and dtype is not _BF16:
        raise ValueError(f"logits must be float32 or bfloat16, not {dtype}")
    if offsets.numel() != e + 1 or order.numel() != have * top:
        raise ValueError("offsets needs experts + 1 and order rows * top_k entries")
    p, _, np_, m = _row_args(plan, None, n_rows, max_rows, have, at)
    _check(lib().sx_moe_route(
        p, np_, m, _ptr(logits, dtype, at, "logits"), F32 if dtype is _F32 else BF16, e, top,
        1 if renormalise else 0, _matrix(ids, (_I32,), have, top, at, "ids"), _matrix(weights, (_F32,), have, top, at, "weights"),
        _ptr(offsets, _I32, at, "offsets"), _ptr(order, _I32, at, "order"), _ptr(workspace, torch.uint8, at, "workspace"),
        workspace.numel(), _on(stream, at)))


def gemm_experts_f8(x8, x_scale, w8, w_scale, offsets, order, y, gather: int = 0, scatter=False, stream=None):
    """y [places][n]: place p of expert e (offsets[e] <= p < offsets[e + 1]) times w8[e] ([experts][n][k]).  The row of x is p,
    or order[p] // gather; the row of y is p, or with scatter order[p].  order may be None without gather and scatter."""
    at, places, x_rows = _device(x8), y.shape[0], x8.shape[0]
    k = x8.shape[-1]
    xp, xsp = _matrix(x8, _CODES, x_rows, k, at, "x8"), _matrix(x_scale, _SCALES, x_rows, _ld(k), at, "x_scale")
    yp, n = _wide(y, places, at, "y")
    _need(w8.dim() == 3, "w8 must be [experts][n][k]")
    e = w8.shape[0]
    _need(offsets.numel() == e + 1, "offsets needs experts + 1 entries")
    _check(lib().sx_gemm_experts_f8(
        _ptr(offsets, _I32, at, "offsets"), None if order is None else _entries(order, places, at, "order"), e,
        _int(places, "places"), xp, xsp, _int(x_rows, "rows of x"), _int(gather, "gather"), _matrix(w8, _CODES, e * n, k, at, "w8"),
        _matrix(w_scale, _SCALES, e * (n // 128), _ld(k), at, "w_scale"), k, n, yp, 1 if scatter else 0, _on(stream, at)))


def moe_combine(y, weights, out, residual=None, plan: Plan = None, rows=None, n_rows=None, max_rows=None,
                out_by_token=False, stream=None):
    """out[row] = residual[row] (which may be out) + sum_j weights[slot][j] * y[slot * top_k + j]."""
    at, have = _device(y), out.shape[0]
    op, h = _wide(out, have, at, "out")
    _need(weights.dim() == 2, "weights must be [rows][top_k]")
    top = weights.shape[1]
    yp, w = _wide(y, have * top, at, "y")
    if w != h:
        raise ValueError(f"y must be [{have * top}][{h}], not {list(y.shape)}")
    p, rp, np_, m = _row_args(plan, rows, n_rows, max_rows, have, at)
    _check(lib().sx_moe_combine(
        p, rp, np_, m, yp, _matrix(weights, (_F32,), have, top, at, "weights"), top, h, _like(residual, have, h, at, "residual"), op,
        1 if out_by_token else 0, _on(stream, at)))

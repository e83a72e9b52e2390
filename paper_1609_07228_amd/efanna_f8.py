"""Thin Python binding of the C ABI declared in include/efanna_f8.h: matrices in 8-bit floating point with a scale for
each block of 128.

Argument marshalling only, as in `efanna`: every step runs in the HIP kernels of libefanna_hip.so on the current stream
of the GPU that holds the tensors, and there is no CPU fallback.  Calls record nothing for autograd: results have no gradients,
whatever the arguments ask for; a layer is an autograd function around them (examples/f8_projection.py has one).
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple

import torch

from . import efanna as _efanna

# every symbol include/efanna_f8.h declares
SYMBOLS = ["efanna_f8_quantise", "efanna_f8_weights", "efanna_f8_rows", "efanna_f8_product_workspace_bytes",
           "efanna_f8_product", "efanna_f8_gradient_workspace_bytes", "efanna_f8_gradient"]

MAX_D = 65536                 # EFANNA_F8_MAX_D

_FORMAT = {torch.float8_e4m3fn: 0, torch.float8_e5m2: 1}
_known = None


def lib():
    """The library of `efanna`, which knows the arguments of these entry points too."""
    global _known
    L = _efanna.lib()
    if _known is not L:
        vp, i64, i32, sz = C.c_void_p, C.c_int64, C.c_int32, C.c_size_t
        L.efanna_f8_quantise.restype = C.c_int
        L.efanna_f8_quantise.argtypes = [vp, i32, i64, i32, i64, i32, vp, vp, vp]
        L.efanna_f8_weights.restype = C.c_int
        L.efanna_f8_weights.argtypes = [vp, i32, i32, i32, i64, i32, vp, vp, vp, vp, vp]
        L.efanna_f8_rows.restype = C.c_int
        L.efanna_f8_rows.argtypes = [vp, vp, i32, i64, i32, vp, i64, C.c_float, i32, vp, vp]
        L.efanna_f8_product_workspace_bytes.restype = sz
        L.efanna_f8_product_workspace_bytes.argtypes = [i64, i64, i32, i32]
        L.efanna_f8_product.restype = C.c_int
        L.efanna_f8_product.argtypes = [vp, vp, i32, i64, vp, vp, i32, i64, i32, i32, vp, i64, vp, sz, vp]
        L.efanna_f8_gradient_workspace_bytes.restype = sz
        L.efanna_f8_gradient_workspace_bytes.argtypes = [i64, i32, i32, i32]
        L.efanna_f8_gradient.restype = C.c_int
        L.efanna_f8_gradient.argtypes = [vp, i32, i64, i32, i64, vp, vp, i32, i32, i32, vp, i64, vp, sz, vp]
        _known = L
    return L


class F8Table(NamedTuple):
    """A matrix in 8-bit floating point (the format is described in efanna_f8.h): codes [n, 128 * ceil(d / 128)]
    float8_e4m3fn or float8_e5m2, scales [n, ceil(d / 128) rounded up to 4] uint8, both on the device; d coordinates."""
    codes: torch.Tensor
    scales: torch.Tensor
    d: int


def _format(dtype: torch.dtype) -> int:
    if dtype not in _FORMAT:
        raise ValueError(f"expected float8_e4m3fn or float8_e5m2, got {dtype}")
    return _FORMAT[dtype]


def _too_long(d: int):
    # (a 32-bit argument of the library, which would take 2^32 + 5 for 5)
    raise ValueError(f"{d} coordinates, columns or rows of weights: at most {MAX_D} are taken")


def _table(t: F8Table):
    """Checks a table's tensors against one another; returns (its row count, its format)."""
    codes, scales, d = t
    if d > MAX_D:
        _too_long(d)
    n, nb = codes.shape[0], (d + 127) // 128
    form = _format(codes.dtype)
    if scales.dtype is not torch.uint8:
        raise ValueError("expected scales in uint8")
    if codes.shape != (n, 128 * nb) or scales.shape != (n, (nb + 3) // 4 * 4):
        raise ValueError("codes and scales do not make a table of d coordinates")
    if not (codes.is_cuda and codes.is_contiguous() and scales.is_contiguous()):
        raise ValueError("expected contiguous device tensors")
    if codes.get_device() != scales.get_device():
        raise ValueError("a table's tensors are on different devices")
    return n, form


def _matrix(x: torch.Tensor):
    """Checks a matrix with dense rows on a device; returns (its element type's number, elements from row to row)."""
    code = _efanna._mx_dtype(x.dtype)
    if not x.is_cuda or x.dim() != 2 or (x.numel() > 0 and x.shape[1] > 1 and x.stride(1) != 1):
        raise ValueError("expected a device matrix with dense rows")
    if x.shape[1] > MAX_D:
        _too_long(x.shape[1])
    return code, x.stride(0) if x.shape[0] > 1 else x.shape[1]


def _empty(n: int, d: int, form: torch.dtype, device) -> F8Table:
    nb = (d + 127) // 128
    # (sizes as arguments of their own: a microsecond less than as a tuple)
    return F8Table(torch.empty(n, 128 * nb, dtype=form, device=device),
                   torch.empty(n, (nb + 3) // 4 * 4, dtype=torch.uint8, device=device), d)


def efanna_f8_quantise(X: torch.Tensor, form: torch.dtype = torch.float8_e4m3fn) -> F8Table:
    """Rows of X [n, d] (float32, float16 or bfloat16; rows may be further apart than d) as a table, a scale for each
    128 coordinates of a row: an activation kept for the backward pass, or a factor of a product."""
    number, (code, ldx) = _format(form), _matrix(X)
    n, d = X.shape
    t = _empty(n, d, form, X.device)
    lib()
    _efanna._call("efanna_f8_quantise", X, X.data_ptr(), code, n, d, ldx, number, t.codes.data_ptr(), t.scales.data_ptr())
    return t


def efanna_f8_weights(W: torch.Tensor, form: torch.dtype = torch.float8_e4m3fn):
    """(table of W [n, d], table of its transpose [d, n]), a scale for each tile of 128 x 128, so that both hold the
    same values: a layer's weights for the products of its forward and of its backward pass."""
    number, (code, ldw) = _format(form), _matrix(W)
    n, d = W.shape
    if n > MAX_D:
        _too_long(n)
    t, turned = _empty(n, d, form, W.device), _empty(d, n, form, W.device)
    lib()
    _efanna._call("efanna_f8_weights", W, W.data_ptr(), code, n, d, ldw, number, t.codes.data_ptr(), t.scales.data_ptr(),
                  turned.codes.data_ptr(), turned.scales.data_ptr())
    return t, turned


def efanna_f8_rows(table: F8Table, ids: torch.Tensor | None = None, factor: float = 1.0,
                   dtype: torch.dtype = torch.float32) -> torch.Tensor:
    """factor * rows `ids` (int32, any shape; all rows if None) of a table, [*ids.shape, d]; zeros for ids that
    are below 0 (empty slots of a graph) or not below the row count."""
    code, (n, form) = _efanna._mx_dtype(dtype), _table(table)
    if ids is not None:
        ids = _efanna._dev(ids, torch.int32)
        if ids.device != table.codes.device:
            raise ValueError("ids and table are on different devices")
    m = n if ids is None else ids.numel()
    shape = (n,) if ids is None else ids.shape
    out = torch.empty(*shape, table.d, dtype=dtype, device=table.codes.device)
    lib()
    _efanna._call("efanna_f8_rows", table.codes, table.codes.data_ptr(), table.scales.data_ptr(), form, n, table.d,
                  None if ids is None else ids.data_ptr(), m, float(factor), code, out.data_ptr())
    return out


def _room(need: int, on: torch.Tensor, given: torch.Tensor | None):
    """(address, bytes, tensor) of the workspace: `given`, or else a new one where one is needed."""
    if given is None and need == 0:
        return None, 0, None
    ws = _efanna._workspace(need, on, given)
    return ws.data_ptr(), ws.numel() * ws.element_size(), ws


def efanna_f8_product(a: F8Table, b: F8Table, dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None,
                      workspace: torch.Tensor | None = None) -> torch.Tensor:
    """a_i . b_j for all rows of two tables, [rows of a, rows of b]; the tables may differ in their format.  `out` may
    have rows that are further apart than they are long.  Results of float32 are sums as float32 makes them, those of 16 bits
    go by the faster 8-bit matrix instructions (efanna_f8.h says what these lose)."""
    code, (m, a_form), (n, b_form) = _efanna._mx_dtype(dtype), _table(a), _table(b)
    if a.d != b.d or a.codes.device != b.codes.device:
        raise ValueError("the tables differ in their dimension or device")
    out = _efanna._mx_out(out, (m, n), dtype, a.codes.device)
    ldo = out.stride(0) if m > 1 else max(n, 1)
    at, size, _keep = _room(lib().efanna_f8_product_workspace_bytes(m, n, a.d, code), a.codes, workspace)
    _efanna._call("efanna_f8_product", a.codes, a.codes.data_ptr(), a.scales.data_ptr(), a_form, m, b.codes.data_ptr(),
                  b.scales.data_ptr(), b_form, n, a.d, code, out.data_ptr(), ldo, at, size)
    return out


def efanna_f8_gradient(dY: torch.Tensor, x: F8Table, dtype: torch.dtype = torch.float32, out: torch.Tensor | None = None,
                       workspace: torch.Tensor | None = None) -> torch.Tensor:
    """dY^T X, [columns of dY, x.d]: the gradient of a layer's weights from that of its output, dY [m, n] (float32, float16
    or bfloat16; rows may be further apart than n), and its input as the table x of m rows holds it."""
    code, (kind, ldy), (m, form) = _efanna._mx_dtype(dtype), _matrix(dY), _table(x)
    if dY.shape[0] != m or dY.device != x.codes.device:
        raise ValueError("dY and the table differ in their row count or device")
    n = dY.shape[1]
    out = _efanna._mx_out(out, (n, x.d), dtype, dY.device)
    ldo = out.stride(0) if n > 1 else x.d
    at, size, _keep = _room(lib().efanna_f8_gradient_workspace_bytes(m, n, x.d, kind), dY, workspace)
    _efanna._call("efanna_f8_gradient", dY, dY.data_ptr(), kind, m, n, ldy, x.codes.data_ptr(), x.scales.data_ptr(), form, x.d,
                  code, out.data_ptr(), ldo, at, size)
    return out

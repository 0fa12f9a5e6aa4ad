"""8-bit floats: matrices of e4m3 codes with an e8m0 scale for every 128 entries of a row, and the operators
on them (see include/qgtc.h).  As in binding.py the functions carry the names of the C entry points and only marshal:
device memory is torch's, work goes to the current stream of the tensors' device."""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple

import torch

from . import binding as B

BLOCK = 128
_TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_ACTS = {"silu": 0, "gelu": 1}


def _run(fn, device: int, *args):
    """The call on the current stream of `device`, which is made the current one for it."""
    if device == torch._C._cuda_getDevice():
        status = fn(*args, B._stream())
    else:
        with torch.cuda.device(device):
            status = fn(*args, B._stream())
    if status != 0:
        raise B.QgtcError(status, fn.__name__)


def _matrix(t: torch.Tensor, what: str, device: int | None = None, shape=None, dtype=None) -> int:
    """Checks a row-major device matrix; its leading dimension."""
    if t.dim() != 2 or t.dtype not in _TYPES:
        raise TypeError(f"{what}: a matrix of float32, float16 or bfloat16 is wanted, not {t.dim()}-D {t.dtype}")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{what}: {dtype} is wanted, not {t.dtype}")
    if not t.is_cuda or (device is not None and t.get_device() != device):
        raise ValueError(f"{what}: not on the device of the other operands")
    rows, cols = t.shape
    if shape is not None and (rows, cols) != shape:
        raise ValueError(f"{what}: {shape[0]} x {shape[1]} is wanted, not {rows} x {cols}")
    if cols > 1 and t.stride(1) != 1:
        raise ValueError(f"{what}: rows have to be contiguous")
    return t.stride(0) if rows > 1 else max(cols, 1)


class Fp8:
    """A matrix in 8-bit floats: codes [rows, at least cols rounded up to 128] (float8_e4m3fn or uint8) and scales
    [rows, blocks rounded up to 4] (float8_e8m0fnu or uint8).  Codes from cols to the end of the last block are 0."""

    __slots__ = ("codes", "scales", "c", "device")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, cols: int | None = None):
        rows, width = codes.shape
        if codes.element_size() != 1 or scales.element_size() != 1 or scales.dim() != 2:
            raise TypeError("codes and scales are matrices of one byte per entry")
        if scales.shape[0] != rows or not codes.is_cuda or codes.get_device() != scales.get_device():
            raise ValueError("codes and scales: a row of each for a row of the matrix, on one device")
        if cols is None:
            cols = width
        blocks = -(-cols // BLOCK)
        if cols < 0 or width < blocks * BLOCK or scales.shape[1] < -(-blocks // 4) * 4:
            raise ValueError("codes have room for whole blocks of 128, scales for a multiple of four")
        if (width > 1 and codes.stride(1) != 1) or (scales.shape[1] > 1 and scales.stride(1) != 1):
            raise ValueError("rows have to be contiguous")
        self.codes, self.scales, self.device = codes, scales, codes.get_device()
        self.c = B._Fp8C(codes.data_ptr(), scales.data_ptr(), rows, cols, codes.stride(0) if rows > 1 and width else width,
                         scales.stride(0) if rows > 1 and scales.shape[1] else scales.shape[1])

    @property
    def rows(self): return self.c.rows
    @property
    def cols(self): return self.c.cols
    @property
    def blocks(self): return -(-self.c.cols // BLOCK)


def alloc_fp8(rows: int, cols: int, device) -> Fp8:
    """Room for a matrix; nothing of it is written yet."""
    blocks = -(-cols // BLOCK)
    return Fp8(torch.empty((rows, blocks * BLOCK), dtype=torch.float8_e4m3fn, device=device),
               torch.empty((rows, -(-blocks // 4) * 4), dtype=torch.float8_e8m0fnu, device=device), cols)


def _result(out: Fp8 | None, rows: int, cols: int, device: int) -> Fp8:
    if out is None:
        return alloc_fp8(rows, cols, torch.device("cuda", device))
    if (out.rows, out.cols) != (rows, cols) or out.device != device:
        raise ValueError(f"out: {rows} x {cols} on the operands' device is wanted, not {out.rows} x {out.cols}")
    return out


def qgtc_fp8_quantize(src: torch.Tensor, columns: bool = False, out: Fp8 | None = None) -> Fp8:
    """src in 8-bit floats, its blocks along the rows; columns: transposed, its blocks along src's columns."""
    ld = _matrix(src, "src")
    rows, cols = src.shape
    out = _result(out, *((cols, rows) if columns else (rows, cols)), src.get_device())
    _run(B.lib().qgtc_fp8_quantize, out.device, src.data_ptr(), _TYPES[src.dtype], rows, cols, ld, int(columns), C.byref(out.c))
    return out


class Norm(NamedTuple):
    """What a norm leaves; None where it was not asked for."""
    sum: torch.Tensor          # x + residual (x itself without one)
    fp8: Fp8 | None
    y: torch.Tensor | None
    rstd: torch.Tensor | None


def qgtc_rms_norm(x: torch.Tensor, weight: torch.Tensor, eps: float = 1e-6, residual: torch.Tensor | None = None,
                  fp8: bool = True, y: bool = False, rstd: bool = False, sum_out: torch.Tensor | None = None,
                  out: Fp8 | None = None) -> Norm:
    """Root-mean-square norm of x + residual times weight, in 8-bit floats (fp8) and/or in x's type (y); rstd: what
    qgtc_rms_norm_backward wants.  sum_out: where x + residual goes, x or residual themselves among others."""
    ld = _matrix(x, "x")
    rows, cols = x.shape
    device, shape = x.get_device(), (rows, cols)
    if weight.dtype not in _TYPES or weight.shape != (cols,) or not weight.is_contiguous() or weight.get_device() != device:
        raise ValueError("weight: one entry per column, contiguous, on x's device")
    n = B._NormC(_TYPES[x.dtype], _TYPES[weight.dtype], rows, cols, eps, 0, x.data_ptr(), ld, weight=weight.data_ptr())
    total = x
    if residual is not None:
        n.ld_residual = _matrix(residual, "residual", device, shape, x.dtype)
        n.residual = residual.data_ptr()
        total = sum_out if sum_out is not None else torch.empty(shape, dtype=x.dtype, device=x.device)
        n.ld_sum = _matrix(total, "sum_out", device, shape, x.dtype)
        n.sum = total.data_ptr()
    elif sum_out is not None:
        raise ValueError("sum_out: there is no residual")
    made = root = None
    if fp8 or out is not None:
        out = _result(out, rows, cols, device)
        n.out = C.pointer(out.c)
    if y:
        made = torch.empty(shape, dtype=x.dtype, device=x.device)
        n.y, n.ld_y = made.data_ptr(), max(cols, 1)
    if rstd:
        root = torch.empty(rows, dtype=torch.float32, device=x.device)
        n.rstd = root.data_ptr()
    _run(B.lib().qgtc_rms_norm, device, C.byref(n))
    return Norm(total, out, made, root)


def qgtc_rms_norm_backward(dy: torch.Tensor, sum: torch.Tensor, weight: torch.Tensor, rstd: torch.Tensor,
                           dsum: torch.Tensor | None = None, dweight: bool = True, out: torch.Tensor | None = None):
    """(gradient of x and of the residual, gradient of the weight in fp32 or None) from that of y; sum and rstd as
    qgtc_rms_norm left them, dsum the gradient that reaches the sum past the norm.  out may be dy or dsum themselves."""
    ld_sum = _matrix(sum, "sum")
    rows, cols = sum.shape
    device, shape, dtype = sum.get_device(), (rows, cols), sum.dtype
    ld_dy = _matrix(dy, "dy", device, shape, dtype)
    if weight.dtype not in _TYPES or weight.shape != (cols,) or not weight.is_contiguous() or weight.get_device() != device:
        raise ValueError("weight: one entry per column, contiguous, on the sum's device")
    if rstd.dtype != torch.float32 or rstd.shape != (rows,) or not rstd.is_contiguous() or rstd.get_device() != device:
        raise ValueError("rstd: one float32 entry per row, contiguous, on the sum's device")
    dx = out if out is not None else torch.empty(shape, dtype=dtype, device=sum.device)
    n = B._NormGradC(_TYPES[dtype], _TYPES[weight.dtype], rows, cols, dy.data_ptr(), ld_dy, sum.data_ptr(), ld_sum,
                     weight.data_ptr(), rstd.data_ptr(), dx=dx.data_ptr(), ld_dx=_matrix(dx, "out", device, shape, dtype))
    if dsum is not None:
        n.dsum, n.ld_dsum = dsum.data_ptr(), _matrix(dsum, "dsum", device, shape, dtype)
    dw = ws = None
    nbytes = 0
    if dweight:
        dw = torch.empty(cols, dtype=torch.float32, device=sum.device)
        n.dweight = dw.data_ptr()
        nbytes = B.lib().qgtc_rms_norm_backward_workspace_bytes(rows, cols)
        ws = torch.empty(nbytes, dtype=torch.uint8, device=sum.device)
    _run(B.lib().qgtc_rms_norm_backward, device, C.byref(n), ws.data_ptr() if nbytes else None, nbytes)
    return dx, dw


def _same_device(x: Fp8, *others: Fp8) -> int:
    for o in others:
        if o.device != x.device:
            raise ValueError("operands on different devices")
    return x.device


def qgtc_fp8_product(x: Fp8, w: Fp8, dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None) -> torch.Tensor:
    """x.w' (a row of w per output column), sums in fp32."""
    device = _same_device(x, w)
    shape = (x.c.rows, w.c.rows)
    if out is None:
        if dtype not in _TYPES:
            raise TypeError(f"float32, float16 or bfloat16 is wanted, not {dtype}")
        out = torch.empty(shape, dtype=dtype, device=x.codes.device)
    ld = _matrix(out, "out", device, shape)
    nbytes = B.lib().qgtc_fp8_product_workspace_bytes(shape[0], shape[1], x.c.cols)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=x.codes.device) if nbytes else None
    _run(B.lib().qgtc_fp8_product, device, C.byref(x.c), C.byref(w.c), _TYPES[out.dtype], out.data_ptr(), ld,
         ws.data_ptr() if nbytes else None, nbytes)
    return out


def qgtc_fp8_gated(x: Fp8, gate: Fp8, up: Fp8, act: str = "silu", out: Fp8 | None = None, fp8: bool = True,
                   h: torch.Tensor | None = None) -> Fp8 | None:
    """act(x.gate') * (x.up') in 8-bit floats; h: a matrix that takes it in its own type (then fp8=False leaves it at that)."""
    device = _same_device(x, gate, up)
    rows, cols = x.c.rows, gate.c.rows
    kind = ptr = ws = None
    ld = nbytes = 0
    if h is not None:
        ld = _matrix(h, "h", device, (rows, cols))
        kind, ptr = _TYPES[h.dtype], h.data_ptr()
    if fp8 or out is not None:
        out = _result(out, rows, cols, device)
        nbytes = B.lib().qgtc_fp8_gated_workspace_bytes(rows, cols, x.c.cols)
        ws = torch.empty(nbytes, dtype=torch.uint8, device=x.codes.device) if nbytes else None
    _run(B.lib().qgtc_fp8_gated, device, C.byref(x.c), C.byref(gate.c), C.byref(up.c), _ACTS[act],
         C.byref(out.c) if out is not None else None, kind or 0, ptr, ld, ws.data_ptr() if nbytes else None, nbytes)
    return out


def qgtc_fp8_gated_backward(x: Fp8, gate: Fp8, up: Fp8, dh: torch.Tensor, act: str = "silu",
                            out: torch.Tensor | None = None) -> torch.Tensor:
    """The gradients of x.gate' and of x.up' from that of qgtc_fp8_gated's result: one matrix, the first beside the second."""
    device = _same_device(x, gate, up)
    rows, cols = x.c.rows, gate.c.rows
    ld_dh = _matrix(dh, "dh", device, (rows, cols))
    if out is None:
        out = torch.empty((rows, 2 * cols), dtype=dh.dtype, device=dh.device)
    ld = _matrix(out, "out", device, (rows, 2 * cols), dh.dtype)
    to = out.data_ptr()
    _run(B.lib().qgtc_fp8_gated_backward, device, C.byref(x.c), C.byref(gate.c), C.byref(up.c), _ACTS[act], _TYPES[dh.dtype],
         dh.data_ptr(), ld_dh, to, ld, to + cols * dh.element_size(), ld)
    return out

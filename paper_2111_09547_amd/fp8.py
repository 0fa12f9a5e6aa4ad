"""8-bit floats: matrices of e4m3 codes with an e8m0 scale for every 128 entries of a row, and the operators
on them (see include/qgtc.h).  As in binding.py the functions carry the names of the C entry points and only marshal:
device memory is torch's, work goes to the current stream of the tensors' device.  Nothing is recorded for autograd, gradients are
calls of their own: a tensor that requires one is refused where torch would record (detach() it, or call under torch.no_grad())."""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple

import torch

from . import binding as B

BLOCK = 128
_MOST = 1 << 29                                          # rows and columns (sizes go to the library in 32 bits)
_TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_ACTS = {"silu": 0, "gelu": 1}


_BYTE = {torch.float8_e4m3fn, torch.float8_e8m0fnu, torch.uint8}
_E4M3, _E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
_empty, _strided = torch.empty, torch.empty_strided     # (1.6 and 1.2 us of host time)
_device_now, _stream_of = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
_byref = C.byref


class _Calls:
    """The library's functions, looked up once."""

    def __getattr__(self, name):
        fn = getattr(B.lib(), name)
        setattr(self, name, fn)
        return fn


_L = _Calls()


def _run(fn, device: int, *args):
    """The call on the current stream of `device`, which is made the current one for it."""
    if device == _device_now():
        status = fn(*args, _stream_of(device))
    else:
        with torch.cuda.device(device):
            status = fn(*args, _stream_of(device))
    if status:
        raise B.QgtcError(status, fn.__name__)


def _bytes(fn, device: int, *args) -> int:
    """A workspace's size, which goes by the device it is asked on."""
    if device == _device_now():
        return fn(*args)
    with torch.cuda.device(device):
        return fn(*args)


def _lost(what: str):
    raise ValueError(f"{what}: requires a gradient, which this call does not record (detach it, or call under torch.no_grad())")


def _matrix(t: torch.Tensor, what: str, device: int | None = None, shape=None, dtype=None) -> int:
    """Checks a row-major device matrix; its leading dimension."""
    size, step = t.shape, t.stride()
    if len(size) != 2 or t.dtype not in _TYPES:
        raise TypeError(f"{what}: a matrix of float32, float16 or bfloat16 is wanted, not {len(size)}-D {t.dtype}")
    if dtype is not None and t.dtype is not dtype:
        raise TypeError(f"{what}: {dtype} is wanted, not {t.dtype}")
    if t.requires_grad and torch.is_grad_enabled():
        _lost(what)
    if not t.is_cuda or (device is not None and t.get_device() != device):
        raise ValueError(f"{what}: not on the device of the other operands")
    if shape is None:
        if max(size) > _MOST:
            raise ValueError(f"{what}: at most 2^29 rows and columns, not {size[0]} x {size[1]}")
    elif size != shape:
        raise ValueError(f"{what}: {shape[0]} x {shape[1]} is wanted, not {size[0]} x {size[1]}")
    if size[0] > 1:
        if step[1] != 1 and size[1] > 1:
            raise ValueError(f"{what}: rows have to be contiguous")
        return step[0]
    if step[1] != 1 and size[1] > 1:
        raise ValueError(f"{what}: rows have to be contiguous")
    return size[1] or 1


class Fp8:
    """A matrix in 8-bit floats: codes [rows, at least cols rounded up to 128] (float8_e4m3fn or uint8) and scales
    [rows, blocks rounded up to 4] (float8_e8m0fnu or uint8).  Codes from cols to the end of the last block are 0."""

    __slots__ = ("codes", "scales", "c", "device", "rows", "cols", "blocks")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, cols: int | None = None):
        size, wide = codes.shape, scales.shape
        if len(size) != 2 or len(wide) != 2 or codes.dtype not in _BYTE or scales.dtype not in _BYTE:
            raise TypeError("codes and scales are matrices of one byte per entry")
        rows, width = size
        device = codes.get_device()
        if wide[0] != rows or device < 0 or scales.get_device() != device:
            raise ValueError("codes and scales: a row of each for a row of the matrix, on one device")
        if cols is None:
            cols = width
        if rows > _MOST or cols > _MOST:
            raise ValueError(f"at most 2^29 rows and columns, not {rows} x {cols}")
        blocks = (cols + 127) >> 7
        if cols < 0 or width < blocks * BLOCK or wide[1] < (blocks + 3 & ~3):
            raise ValueError("codes have room for whole blocks of 128, scales for a multiple of four")
        step, apart = codes.stride(), scales.stride()
        if (step[1] != 1 and width > 1) or (apart[1] != 1 and wide[1] > 1):
            raise ValueError("rows have to be contiguous")
        self.codes, self.scales, self.device, self.rows, self.cols, self.blocks = codes, scales, device, rows, cols, blocks
        # (one row has no row to lie apart from: its tensor may have any width)
        self.c = B._Fp8C(codes.data_ptr(), scales.data_ptr(), rows, cols, step[0] if rows > 1 and width else blocks * BLOCK,
                         apart[0] if rows > 1 and wide[1] else blocks + 3 & ~3)


def alloc_fp8(rows: int, cols: int, device) -> Fp8:
    """Room for a matrix; nothing of it is written yet."""
    if rows > _MOST or cols > _MOST:
        raise ValueError(f"at most 2^29 rows and columns, not {rows} x {cols}")
    return _room(rows, cols, device)


def _room(rows: int, cols: int, device) -> Fp8:
    m = Fp8.__new__(Fp8)
    m.rows, m.cols = rows, cols
    m.blocks = blocks = (cols + 127) >> 7
    width, words = blocks * BLOCK, blocks + 3 & ~3
    m.codes = codes = _strided((rows, width), (width, 1), dtype=_E4M3, device=device)
    m.scales = scales = _strided((rows, words), (words, 1), dtype=_E8M0, device=device)
    m.device = codes.get_device()
    if m.device < 0:
        raise ValueError("8-bit floats are on a GPU")
    m.c = B._Fp8C(codes.data_ptr(), scales.data_ptr(), rows, cols, width, words)
    return m


def _result(out: Fp8 | None, rows: int, cols: int, like: torch.Tensor) -> Fp8:
    if out is None:
        return _room(rows, cols, like.device)
    if out.rows != rows or out.cols != cols or out.device != like.get_device():
        raise ValueError(f"out: {rows} x {cols} on the operands' device is wanted, not {out.rows} x {out.cols}")
    return out


def qgtc_fp8_quantize(src: torch.Tensor, columns: bool = False, out: Fp8 | None = None) -> Fp8:
    """src in 8-bit floats, its blocks along the rows; columns: transposed, its blocks along src's columns."""
    ld = _matrix(src, "src")
    rows, cols = src.shape
    out = _result(out, cols, rows, src) if columns else _result(out, rows, cols, src)
    _run(_L.qgtc_fp8_quantize, out.device, src.data_ptr(), _TYPES[src.dtype], rows, cols, ld, 1 if columns else 0, _byref(out.c))
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
    device, shape, dtype = x.get_device(), x.shape, x.dtype
    if weight.dtype not in _TYPES or weight.shape != (cols,) or not weight.is_contiguous() or weight.get_device() != device:
        raise ValueError("weight: one entry per column, contiguous, on x's device")
    if weight.requires_grad and torch.is_grad_enabled():
        _lost("weight")
    total, made, root = x, None, None
    p_res = p_sum = p_y = p_root = p_out = None
    ld_res = ld_sum = 0
    if residual is not None:
        ld_res = _matrix(residual, "residual", device, shape, dtype)
        p_res = residual.data_ptr()
        if sum_out is None:
            total, ld_sum = _strided(shape, (cols, 1), dtype=dtype, device=x.device), cols or 1
        else:
            total, ld_sum = sum_out, _matrix(sum_out, "sum_out", device, shape, dtype)
        p_sum = total.data_ptr()
    elif sum_out is not None:
        raise ValueError("sum_out: there is no residual")
    if fp8 or out is not None:
        out = _result(out, rows, cols, x)
        p_out = C.addressof(out.c)
    if y:
        made = _strided(shape, (cols, 1), dtype=dtype, device=x.device)
        p_y = made.data_ptr()
    if rstd:
        if not cols:
            raise ValueError("rstd: x has no columns to take a mean of")
        root = _empty(rows, dtype=torch.float32, device=x.device)
        p_root = root.data_ptr()
    n = B._NormC(_TYPES[dtype], _TYPES[weight.dtype], rows, cols, eps, 0, x.data_ptr(), ld, p_res, ld_res, weight.data_ptr(),
                 p_sum, ld_sum, p_y, cols or 1, p_root, p_out)
    _run(_L.qgtc_rms_norm, device, _byref(n))
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
    if (weight.requires_grad or rstd.requires_grad) and torch.is_grad_enabled():
        _lost("weight and rstd")
    if rstd.dtype != torch.float32 or rstd.shape != (rows,) or not rstd.is_contiguous() or rstd.get_device() != device:
        raise ValueError("rstd: one float32 entry per row, contiguous, on the sum's device")
    dx = out if out is not None else _strided(shape, (cols, 1), dtype=dtype, device=sum.device)
    n = B._NormGradC(_TYPES[dtype], _TYPES[weight.dtype], rows, cols, dy.data_ptr(), ld_dy, sum.data_ptr(), ld_sum,
                     weight.data_ptr(), rstd.data_ptr(), dx=dx.data_ptr(), ld_dx=_matrix(dx, "out", device, shape, dtype))
    if dsum is not None:
        n.dsum, n.ld_dsum = dsum.data_ptr(), _matrix(dsum, "dsum", device, shape, dtype)
    dw = ws = None
    nbytes = 0
    if dweight:
        dw = _empty(cols, dtype=torch.float32, device=sum.device)
        n.dweight = dw.data_ptr()
        nbytes = _bytes(_L.qgtc_rms_norm_backward_workspace_bytes, device, rows, cols)
        ws = _empty(nbytes, dtype=torch.uint8, device=sum.device)
    _run(_L.qgtc_rms_norm_backward, device, _byref(n), ws.data_ptr() if nbytes else None, nbytes)
    return dx, dw


def _same_device(x: Fp8, *others: Fp8) -> int:
    for o in others:
        if o.device != x.device:
            raise ValueError("operands on different devices")
    return x.device


def qgtc_fp8_product(x: Fp8, w: Fp8, dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None) -> torch.Tensor:
    """x.w' (a row of w per output column), sums in fp32."""
    device = _same_device(x, w)
    shape = (x.rows, w.rows)
    if out is None:
        if dtype not in _TYPES:
            raise TypeError(f"float32, float16 or bfloat16 is wanted, not {dtype}")
        out = _strided(shape, (shape[1], 1), dtype=dtype, device=x.codes.device)
    ld = _matrix(out, "out", device, shape)
    _run(_L.qgtc_fp8_product, device, _byref(x.c), _byref(w.c), _TYPES[out.dtype], out.data_ptr(), ld)
    return out


def qgtc_fp8_gated(x: Fp8, gate: Fp8, up: Fp8, act: str = "silu", out: Fp8 | None = None, fp8: bool = True,
                   h: torch.Tensor | None = None) -> Fp8 | None:
    """act(x.gate') * (x.up') in 8-bit floats; h: a matrix that takes it in its own type (then fp8=False leaves it at that)."""
    device = _same_device(x, gate, up)
    rows, cols = x.rows, gate.rows
    kind = ptr = ws = None
    ld = nbytes = 0
    if h is not None:
        ld = _matrix(h, "h", device, (rows, cols))
        kind, ptr = _TYPES[h.dtype], h.data_ptr()
    if fp8 or out is not None:
        out = _result(out, rows, cols, x.codes)
        nbytes = _bytes(_L.qgtc_fp8_gated_workspace_bytes, device, rows, cols, x.cols)
        ws = _empty(nbytes, dtype=torch.uint8, device=x.codes.device) if nbytes else None
    _run(_L.qgtc_fp8_gated, device, _byref(x.c), _byref(gate.c), _byref(up.c), _ACTS[act],
         _byref(out.c) if out is not None else None, kind or 0, ptr, ld, ws.data_ptr() if nbytes else None, nbytes)
    return out


def qgtc_fp8_gated_backward(x: Fp8, gate: Fp8, up: Fp8, dh: torch.Tensor, act: str = "silu",
                            out: torch.Tensor | None = None) -> torch.Tensor:
    """The gradients of x.gate' and of x.up' from that of qgtc_fp8_gated's result: one matrix, the first beside the second."""
    device = _same_device(x, gate, up)
    rows, cols = x.rows, gate.rows
    ld_dh = _matrix(dh, "dh", device, (rows, cols))
    if out is None:
        out = _empty((rows, 2 * cols), dtype=dh.dtype, device=dh.device)
    ld = _matrix(out, "out", device, (rows, 2 * cols), dh.dtype)
    to = out.data_ptr()
    _run(_L.qgtc_fp8_gated_backward, device, _byref(x.c), _byref(gate.c), _byref(up.c), _ACTS[act], _TYPES[dh.dtype],
         dh.data_ptr(), ld_dh, to, ld, to + cols * dh.element_size(), ld)
    return out

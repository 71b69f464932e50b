"""Microscaled 4-bit operands and their products on torch CUDA tensors.

The formats, the layout of codes and scales and every formula are those of ``include/mor.h``; this module allocates outputs,
fills the descriptors and runs the calls on the current stream.

    a, _ = fp4.quantize(x, "e4m3_16")                  # blocks along the rows of x
    b, bt = fp4.quantize(w, "e4m3_16", cols=True)      # both directions from one read; bt is the operand of w^T
    y = fp4.matmul(a, b)                               # x w^T
    y = fp4.linear(x, w, "e8m0_32")                    # the same with its gradient (straight through the rounding)

There is no CPU path: the library raises if it has not been built.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import binding as _b

FORMATS = {"e4m3_16": _b.MOR_FP4_E4M3_16, "e8m0_32": _b.MOR_FP4_E8M0_32}
_DTYPES = {torch.bfloat16: _b.MOR_DTYPE_BF16, torch.float32: _b.MOR_DTYPE_F32}
_status = {}            # device index -> the word that products set when a bounded wait ran out
_raw_stream = torch._C._cuda_getCurrentRawStream


def _dtype(t, what: str) -> int:
    try:
        return _DTYPES[t]
    except KeyError:
        raise TypeError(f"{what}: BF16 or FP32 is wanted, got {t}") from None


def _check(status: int, where: str) -> None:
    if status != _b.MOR_OK:
        raise _b.MorError(status, where)


def _on_gpu(x: torch.Tensor, what: str) -> int:
    """Device index of a CUDA tensor; the calls run on that device's current stream, which has to be the current device's."""
    if not x.is_cuda:
        raise ValueError(f"{what} has to be a CUDA tensor")
    index = x.device.index
    if index != torch.cuda.current_device():
        raise ValueError(f"{what} is on device {index}, the current device is {torch.cuda.current_device()}")
    return index


def _rows_contiguous(x: torch.Tensor, what: str) -> None:
    if x.shape[-1] > 1 and x.stride(-1) != 1:
        raise ValueError(f"{what}: the last dimension has to be contiguous")


class Operand:
    """A stack of matrices [batch][rows, cols] in 4 bits, blocks along cols.

    ``codes``: uint8 [..., rows, ld]; ``scales``: uint8 tiles (see ``include/mor.h``); ``tensor_scale``: one float.  The tensors
    may be a caller's own (a stored weight): ``Operand(codes, scales, rows, cols, format, tensor_scale)``.
    """
    __slots__ = ("c", "device", "_keep", "_at")

    def __init__(self, codes, scales, rows: int, cols: int, format, tensor_scale):
        f = FORMATS.get(format, format)
        batch = codes.shape[0] if codes.dim() == 3 else 1
        if codes.dim() not in (2, 3) or codes.shape[-2] != rows:
            raise ValueError(f"codes: [..., {rows}, bytes] is wanted, got {tuple(codes.shape)}")
        if codes.dtype != torch.uint8 or scales.dtype != torch.uint8 or tensor_scale.dtype != torch.float32:
            raise TypeError("codes and scales are uint8, the tensor scale is FP32")
        if not (codes.is_contiguous() and scales.is_contiguous()):
            raise ValueError("codes and scales have to be contiguous")
        if scales.numel() < _b.load().mor_fp4_scale_bytes(batch, rows, cols, f):
            raise ValueError("scales: too few bytes for this shape")
        self.device = _on_gpu(codes, "codes")
        self._keep = (codes, scales, tensor_scale)
        self._at = None
        self.c = _b.mor_fp4_matrix_t(codes.data_ptr(), scales.data_ptr(), tensor_scale.data_ptr(), batch, rows, cols, codes.shape[-1], f)

    @classmethod
    def _empty(cls, batch: int, rows: int, cols: int, f: int, device, index: int):
        """Memory for codes, scales and the tensor scale in one allocation."""
        o = cls.__new__(cls)
        ld = (cols + 31) // 32 * 16
        n = batch * rows * ld                                            # multiples of 16
        block = 16 if f == _b.MOR_FP4_E4M3_16 else 32
        s = batch * ((rows + 127) // 128) * ((cols + 4 * block - 1) // (4 * block)) * 512
        buf = torch.empty(n + s + 16, dtype=torch.uint8, device=device)
        p = buf.data_ptr()
        o.device, o._keep, o._at = index, (buf,), (n, s)
        o.c = _b.mor_fp4_matrix_t(p, p + n, p + n + s, batch, rows, cols, ld, f)
        return o

    batch = property(lambda self: self.c.batch)
    rows = property(lambda self: self.c.rows)
    cols = property(lambda self: self.c.cols)

    @property
    def format(self) -> str:
        return "e4m3_16" if self.c.format == _b.MOR_FP4_E4M3_16 else "e8m0_32"

    @property
    def codes(self) -> torch.Tensor:
        if self._at is None:
            return self._keep[0]
        return self._keep[0][:self._at[0]].view(self.c.batch, self.c.rows, self.c.ld)

    @property
    def scales(self) -> torch.Tensor:
        return self._keep[1] if self._at is None else self._keep[0][self._at[0]:self._at[0] + self._at[1]]

    @property
    def tensor_scale(self) -> torch.Tensor:
        if self._at is None:
            return self._keep[2]
        at = self._at[0] + self._at[1]
        return self._keep[0][at:at + 4].view(torch.float32)


def _status_word(device, index: int) -> torch.Tensor:
    w = _status.get(index)
    if w is None:
        w = _status[index] = torch.zeros(1, dtype=torch.int32, device=device)
    return w


def quantize(x: torch.Tensor, format: str, *, rows: bool = True, cols: bool = False, amax=None, gather=None, weight=None):
    """(operand along the rows or None, operand of the transpose or None) of x [R, C] or [batch, R, C], BF16 or FP32.

    ``amax``: FP32 CUDA tensor, the tensor's largest magnitude if it is known ("e4m3_16" only).  ``gather``: an
    ``experts.Plan``; row i of the result is then the token row of the plan's row i (zero where it has none), times ``weight`` [tokens,
    top] if given.
    """
    if x.dim() not in (2, 3) or (gather is not None and x.dim() != 2):
        raise ValueError(f"x: [rows, cols] or [batch, rows, cols] is wanted, got {tuple(x.shape)}")
    f = FORMATS[format]
    index = _on_gpu(x, "x")
    _rows_contiguous(x, "x")
    dtype = _dtype(x.dtype, "x")
    n_rows, n_cols = x.shape[-2], x.shape[-1]
    batch = x.shape[0] if x.dim() == 3 else 1
    ld = x.stride(-2) if n_rows > 1 else n_cols
    if ld < n_cols:
        raise ValueError("x: rows may not overlap")
    d = _b.mor_fp4_quantize_desc_t(x.data_ptr(), dtype, f, batch, n_rows, n_cols, ld, x.stride(0) if batch > 1 else 0)
    if amax is not None:
        if amax.dtype != torch.float32 or amax.numel() != 1 or amax.device != x.device:
            raise ValueError("amax: one FP32 value on x's device is wanted")
        d.amax = amax.data_ptr()
    out_rows = n_rows
    if gather is not None:
        if gather.row.shape[0] != n_rows or gather.row.device != x.device:
            raise ValueError(f"gather: a plan for {n_rows} tokens on x's device is wanted")
        out_rows = gather.slot.shape[0]
        d.slot_of_row, d.row_of_slot, d.out_rows, d.top = gather.slot.data_ptr(), gather.row.data_ptr(), out_rows, gather.top
    if weight is not None:
        if gather is None or weight.shape != gather.row.shape or not weight.is_contiguous() or weight.device != x.device:
            raise ValueError("weight: contiguous [tokens, top] on x's device is wanted, with gather")
        d.weight, d.weight_dtype = weight.data_ptr(), _dtype(weight.dtype, "weight")
    r = Operand._empty(batch, out_rows, n_cols, f, x.device, index) if rows else None
    c = Operand._empty(batch, n_cols, out_rows, f, x.device, index) if cols else None
    ws, n = None, 0
    if f == _b.MOR_FP4_E4M3_16 and amax is None:
        n = _b.MOR_FP4_WORKSPACE_BYTES
        ws = torch.empty(n, dtype=torch.uint8, device=x.device)
    _check((_b._lib or _b.load()).mor_fp4_quantize(C.byref(d), C.byref(r.c) if rows else None, C.byref(c.c) if cols else None,
                                                   None if ws is None else ws.data_ptr(), n, _raw_stream(index)), "mor_fp4_quantize")
    return r, c


def dequantize(op: Operand, dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """The values of an operand: [rows, cols], or [batch, rows, cols] for a stack of more than one."""
    c = op.c
    shape = (c.rows, c.cols) if c.batch == 1 else (c.batch, c.rows, c.cols)
    out = torch.empty(shape, dtype=dtype, device=op._keep[0].device)
    _check(_b.load().mor_fp4_dequantize(C.byref(c), out.data_ptr(), _dtype(dtype, "dtype"), c.cols, _raw_stream(op.device)), "mor_fp4_dequantize")
    return out


def check(device=None) -> None:
    """Raises if a product on this device gave up a wait since the last check (synchronises)."""
    index = torch.cuda.current_device() if device is None else torch.device(device).index
    w = _status.get(index)
    if w is not None:
        s = int(w.item())
        w.zero_()
        _check(s, "mor_fp4_matmul")


def _matmul(a: Operand, b: Operand, out_dtype, grouping: int, plan) -> torch.Tensor:
    m, n = a.c.rows, b.c.rows
    device = a._keep[0].device
    dtype = _dtype(out_dtype, "out_dtype")
    if a.device != b.device:
        raise ValueError("the operands are on different devices")
    per = 8 if dtype == _b.MOR_DTYPE_BF16 else 4
    ldo = (n + per - 1) // per * per                                     # rows of the result start on 16 bytes
    groups = 0 if plan is None else plan.starts.shape[0] - 1
    shape = (groups, m, ldo) if grouping == _b.MOR_GROUP_REDUCE else (m, ldo)
    out = torch.empty(shape, dtype=out_dtype, device=device)
    d = _b.mor_fp4_matmul_desc_t(a.c, b.c, out.data_ptr(), dtype, grouping, ldo, None if plan is None else plan.starts.data_ptr(), groups,
                                 _status_word(device, a.device).data_ptr())
    _check((_b._lib or _b.load()).mor_fp4_matmul(C.byref(d), _raw_stream(a.device)), "mor_fp4_matmul")
    return out if ldo == n else out[..., :n]


def matmul(a: Operand, b: Operand, out_dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """a b^T: [a.rows, b.rows] (rows start on 16 bytes, so an odd width comes as a view of a wider buffer)."""
    return _matmul(a, b, out_dtype, _b.MOR_GROUP_NONE, None)


def _aligned(plan) -> None:
    if plan.align % 128 != 0:
        raise ValueError("the plan's rows have to be aligned to 128 for grouped products: experts.sort(..., align=128)")


def matmul_rows(a: Operand, b: Operand, plan, out_dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """Rows of each expert of ``plan`` times that expert's matrix of the stack b; rows past the last expert's are not written."""
    _aligned(plan)
    if a.c.rows != plan.slot.shape[0] or b.c.batch != plan.starts.shape[0] - 1:
        raise ValueError("a needs the plan's rows and b one matrix per expert")
    return _matmul(a, b, out_dtype, _b.MOR_GROUP_ROWS, plan)


def matmul_reduce(a: Operand, b: Operand, plan, out_dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """[experts, a.rows, b.rows]: the product summed over each expert's part of the reduction axis."""
    _aligned(plan)
    if a.c.cols != plan.slot.shape[0]:
        raise ValueError("the reduction axis has to be the plan's rows")
    return _matmul(a, b, out_dtype, _b.MOR_GROUP_REDUCE, plan)


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, format):
        need_x, need_w = ctx.needs_input_grad[:2]
        a, ctx.a_t = quantize(x, format, cols=need_w)
        b, ctx.b_t = quantize(w, format, cols=need_x)
        ctx.format, ctx.dtypes = format, (x.dtype, w.dtype)
        return matmul(a, b, x.dtype)

    @staticmethod
    def backward(ctx, dy):
        g, g_t = quantize(dy if dy.stride(-1) == 1 else dy.contiguous(), ctx.format, rows=ctx.needs_input_grad[0], cols=ctx.needs_input_grad[1])
        dx = matmul(g, ctx.b_t, ctx.dtypes[0]) if g is not None else None
        dw = matmul(g_t, ctx.a_t, ctx.dtypes[1]) if g_t is not None else None
        return dx, dw, None


def linear(x: torch.Tensor, w: torch.Tensor, format: str) -> torch.Tensor:
    """x [..., n_in] times w [n_out, n_in] transposed, every operand of the product and of its two gradients in 4 bits along that
    product's reduction axis.  The rounding is passed straight through in the backward pass."""
    if x.shape[-1] != w.shape[-1] or w.dim() != 2:
        raise ValueError(f"x [..., n_in] and w [n_out, n_in] are wanted, got {tuple(x.shape)} and {tuple(w.shape)}")
    y = _Linear.apply(x if x.dim() == 2 else x.reshape(-1, x.shape[-1]), w, format)
    return y if x.dim() == 2 else y.reshape(*x.shape[:-1], w.shape[0])

"""Microscaled 4-bit operands and their products on torch CUDA tensors.

The formats ("e4m3_16", "e8m0_32"), the layout of codes and scales and every formula are those of ``include/mor.h``.  The calls
check their arguments, allocate their outputs and run on the current stream of the current device:

    a, _ = fp4.quantize(x, "e4m3_16")                  # blocks along the rows of x
    b, bt = fp4.quantize(w, "e4m3_16", cols=True)      # both directions from one read; bt is the operand of w^T
    y = fp4.matmul(a, b)                               # x w^T
    y = fp4.linear(x, w, "e8m0_32")                    # the same with its gradient (straight through the rounding)

``Operand(codes, scales, rows, cols, format, tensor_scale)``
    a stack of matrices [batch][rows, cols], blocks along cols, over a caller's tensors (a stored weight): codes uint8 [..., rows,
    bytes], scales uint8 in tiles, one FP32 tensor scale.
``quantize(x, format, *, rows=True, cols=False, amax=None, gather=None, weight=None)``
    (operand along the rows or None, operand of the transpose or None) of x [R, C] or [batch, R, C], BF16 or FP32.  amax: FP32, the
    tensor's largest magnitude if it is known ("e4m3_16" only).  gather: an ``experts.Plan``; row i of the result is then the token row
    of the plan's row i (zero where it has none), times weight [tokens, top] if given.
``dequantize(op, dtype=torch.bfloat16)``
    the values: [rows, cols], or [batch, rows, cols] for a stack of more than one.
``matmul(a, b, out_dtype=torch.bfloat16)``
    a b^T.  Rows of a result start on multiples of 16 bytes, so one of another width has a row stride above its width.
``matmul_rows(a, b, plan, out_dtype=...)``
    the rows of each expert of the plan times that expert's matrix of the stack b; empty rows of the plan are not written.
``matmul_reduce(a, b, plan, out_dtype=...)``
    [experts, a.rows, b.rows]: the product summed over each expert's part of the reduction axis.
``linear(x, w, format)``
    x [..., n_in] times w [n_out, n_in] transposed; every operand of the product and of its two gradients is quantised along that
    product's reduction axis, and the rounding is passed straight through in the backward pass.  x, w and the gradient may have any strides
    (rows that overlap or are not contiguous are copied first; the other calls refuse them).

Gradients: linear has its own, of x and w, once (its backward pass cannot be differentiated again).  An ``Operand`` carries none: nothing that is
made of it through dequantize and matmul is differentiable in what was quantised.

There is no CPU path: importing this module raises if the operators have not been built.
"""
from __future__ import annotations

import os

import torch

from . import binding as _b

if not os.path.exists(os.path.join(os.path.dirname(os.path.abspath(__file__)), "_ops.so")):
    raise RuntimeError("_ops.so is missing: build it with `python -m paper_2512_22804_b200.build` (the 4-bit operators have no CPU path)")
from ._ops import Operand, dequantize, linear, matmul, matmul_reduce, matmul_rows, quantize  # noqa: E402
from ._ops import status_word as _status_word  # noqa: E402

__all__ = ["Operand", "quantize", "dequantize", "matmul", "matmul_rows", "matmul_reduce", "linear", "check"]


def check(device=None) -> None:
    """Raises if a product on this device gave up a bounded wait since the last check; its result is then undefined.  Waits for all of the
    device's streams."""
    device = torch.device("cuda" if device is None else device)
    with torch.cuda.device(device):
        word = _status_word(torch.empty(0, device="cuda"))
        torch.cuda.synchronize()
        status = int(word.item())
        if status != _b.MOR_OK:
            word.zero_()
            torch.cuda.synchronize()
            raise _b.MorError(status, "mor_fp4_matmul")

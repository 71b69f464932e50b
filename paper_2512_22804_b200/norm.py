"""Root-mean-square norm with the residual's addition, on torch CUDA tensors.

    y, h = norm.rms_norm(x, weight, residual)                      # h = x + residual, y = h / sqrt(mean(h^2) + eps) * weight
    codes, scales, h = norm.rms_norm_quantize(x, weight, residual) # y in 8 bits
    y = norm.dequantize(codes, scales)

``rms_norm(x, weight, residual=None, *, eps=1e-6)``
    y, or (y, h) with a residual, over the last dimension of x [..., columns].  x, weight and residual are BF16 or FP32; h has the
    residual's type and is rounded to it once, and y, of x's type, is the norm of that h: what the next layer adds to is what was normed.
``rms_norm_quantize(x, weight, residual=None, *, eps=1e-6, block=128, scale="e8m0")``
    (codes, scales) or (codes, scales, h).  codes: float8_e4m3fn of y * s, made from y in 32 bits; s = 448 over the largest finite magnitude of `block`
    columns (128, or None: the whole row), as FP32 ("fp32"), or cut to a power of two ("e8m0": uint8, its biased exponent).  These are the codes and
    scales that ``binding.analyze_quantize`` makes with (1, 128) and (1, 0) blocks and those scale modes; a consumer divides by s.
``dequantize(codes, scales, dtype=torch.bfloat16)``
    code / s, rounded once.

Results have rows that start on multiples of 16 bytes, so one of another width has a row stride above its width.  Inputs may have any strides (rows that
overlap or are not contiguous are copied first).  A row of zeros is zero; with eps = 0 it is NaN.

Gradients: rms_norm has its own, of x, weight and residual, once (its backward pass cannot be differentiated again).  The others have none: what they make
of tensors that require one raises when it is differentiated.  Forward-mode derivatives are refused.

The formulas are those of ``include/mor.h``.
"""
from __future__ import annotations

from . import fp4  # noqa: F401  (raises if the operators have not been built)
from ._ops import codes_values as dequantize
from ._ops import rms_norm
from ._ops import rms_norm_quantize as _quantize

__all__ = ["rms_norm", "rms_norm_quantize", "dequantize"]


def rms_norm_quantize(x, weight, residual=None, *, eps=1e-6, block=128, scale="e8m0"):
    return _quantize(x, weight, residual, eps=eps, scale=scale, block=0 if block is None else block)

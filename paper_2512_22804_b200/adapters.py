"""Low-rank adapters of many requests beside a shared projection, on torch CUDA tensors.

    y = adapters.add(base, x, a, b, ids, scale)          # base + scale[g] (x a[g]^T) b[g]^T, g = ids[token]
    y = adapters.linear(x, w, a, b, ids, scale)          # the same with the projection: w a stored 4-bit operand [n_out, n_in]

``add(base, x, a, b, ids=None, scale=1.0)``
    x BF16 [..., n_in], base BF16 or FP32 [..., n_out]; a BF16 [adapters, rank, n_in] and b BF16 [adapters, n_out, rank] (or one adapter's matrices, without
    the first dimension), rank up to 512; ids int32 [...], one for every token: an id outside 0..adapters-1 means no adapter, and the token's base comes
    back as it is.  Without ids every token has the one adapter.  scale: a number, or FP32 [adapters].  The result has base's type, is rounded
    once, and is a tensor of its own.  Infinities pass through as such but for those of b (in the gradients a, dy and x), which may become NaN.
``linear(x, w, a, b, ids=None, scale=1.0, *, w_t=None)``
    x [..., n_in] quantised to w's format and multiplied with it, the adapters added to the BF16 result.  The projection is frozen.  For a gradient of x
    the operand of w's transpose is wanted too: ``w, w_t = fp4.quantize(weight, format, cols=True)``; dy is then quantised along n_out and the rounding passed
    straight through.

Few tokens without gradients (up to 224, fewer with ranks above 32 or wide results) are one launch; more are sorted by adapter first.  x, base and the gradient
may have any strides (rows that overlap or are not contiguous are copied first); rows of results start on multiples of 16 bytes.

Gradients: of x, a and b (and base), once (the backward pass cannot be differentiated again).  ids and scale have none.  Forward-mode derivatives are refused.  The gradient of an FP32 result is
rounded to BF16 for the adapters' products.

The formulas are those of ``include/mor.h``.
"""
from __future__ import annotations

from . import fp4  # noqa: F401  (raises if the operators have not been built)
from ._ops import adapter_add as add
from ._ops import adapter_linear as linear

__all__ = ["add", "linear"]

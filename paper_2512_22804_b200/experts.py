"""Tokens sorted by expert and back, on torch CUDA tensors, and a 4-bit expert layer built on it.

    plan = experts.sort(ids, n_experts, align=128)     # ids int32 [tokens, top]; an id outside 0..n_experts-1 has no row
    xs = experts.gather(x, plan)                       # rows of each expert together
    y = experts.combine(ys, plan, weight)              # back, weights applied
    y = experts.linear(x, w, ids, weight, "e4m3_16")   # all of it with 4-bit products, differentiable

``sort(ids, n_experts, align=1)``
    a ``Plan``: starts [experts + 1], row [tokens, top] (-1: none), slot [rows] (-1: an empty row); expert by expert, slots in order,
    each expert's first row a multiple of align.
``gather(x, plan, weight=None)``
    [plan rows, hidden]: each row the token row of its slot, times weight [tokens, top] if given; zero where it has no slot.
``combine(ys, plan, weight=None, out_dtype=None)``
    [tokens, hidden]: the sum over each token's slots of weight (1 if not given) times the slot's row of ys, in ys's type or, from FP32, in
    BF16.
``combine_grad(dy, ys, plan, weight, *, rows=True)``
    (dys or None, dweight): the gradients of combine(ys, plan, weight) for dy; ys in dy's type or FP32.
``linear(x, w, ids, weight, format=None)``
    y[t] = sum over j of weight[t, j] * Q(x[t]) Q(w[ids[t, j]])^T for x [tokens, n_in].  w is a tensor [experts, n_out, n_in]
    (differentiable in x, w and weight; the rounding is passed straight through) or, for serving, a stored stack (``fp4.Operand`` with one
    matrix per expert; format is then its own).  x, w and the gradient may have any strides (rows that overlap or are not contiguous are copied
    first); ids and weight are contiguous.

Gradients: linear has its own, of x, w and weight, once (its backward pass cannot be differentiated again).  gather, combine, combine_grad and linear
with a stored stack have none: what they make of tensors that require a gradient raises when it is differentiated.  Forward-mode derivatives are refused.  In a
torch.autograd.Function of a caller's own, the gradient of gather(x, plan) is combine(dxs, plan) and that of combine is combine_grad.

The formulas are those of ``include/mor.h``.
"""
from __future__ import annotations

from . import fp4  # noqa: F401  (raises if the operators have not been built)
from ._ops import Plan, combine, combine_grad, gather, sort
from ._ops import expert_linear as linear

__all__ = ["Plan", "sort", "gather", "combine", "combine_grad", "linear"]

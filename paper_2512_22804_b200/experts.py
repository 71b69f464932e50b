"""Tokens sorted by expert and back, on torch CUDA tensors, and a 4-bit expert layer built on it.

    plan = experts.sort(ids, n_experts, align=128)     # ids [tokens, top]; an id outside 0..n_experts-1 has no row
    xs = experts.gather(x, plan)                       # rows of each expert together
    y = experts.combine(ys, plan, weight)              # back, weights applied
    y = experts.linear(x, w, ids, weight, "e4m3_16")   # all of it with 4-bit products, differentiable

The formulas are those of ``include/mor.h``.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import binding as _b
from . import fp4
from .fp4 import _check, _dtype, _on_gpu, _raw_stream, _rows_contiguous


class Plan:
    """Where every slot's row is: ``starts`` [experts + 1], ``row`` [tokens, top] (-1: none), ``slot`` [rows] (-1: empty row)."""
    __slots__ = ("starts", "row", "slot", "top", "align")

    def __init__(self, starts, row, slot, top: int, align: int):
        self.starts, self.row, self.slot, self.top, self.align = starts, row, slot, top, align


def sort(ids: torch.Tensor, n_experts: int, align: int = 1) -> Plan:
    """Rows for the slots of ids [tokens, top] (int32), expert by expert, each expert's first row a multiple of ``align``."""
    if ids.dim() != 2 or ids.dtype != torch.int32 or not ids.is_contiguous():
        raise ValueError("ids: contiguous int32 [tokens, top] is wanted")
    index = _on_gpu(ids, "ids")
    n, L = ids.numel(), _b._lib or _b.load()
    capacity = L.mor_expert_rows(n, n_experts, align)
    if capacity < 0:
        raise _b.MorError(_b.MOR_ERR_INVALID_ARG, "mor_expert_sort")
    starts = torch.empty(n_experts + 1, dtype=torch.int32, device=ids.device)
    row = torch.empty_like(ids)
    slot = torch.empty(capacity, dtype=torch.int32, device=ids.device)
    need = L.mor_expert_workspace_bytes(n, n_experts)
    ws = torch.empty(need, dtype=torch.uint8, device=ids.device)
    _check(L.mor_expert_sort(ids.data_ptr(), n, n_experts, align, starts.data_ptr(), row.data_ptr(), slot.data_ptr(), ws.data_ptr(), need,
                             _raw_stream(index)), "mor_expert_sort")
    return Plan(starts, row, slot, ids.shape[1], align)


def _desc(plan: Plan, m: torch.Tensor, weight) -> _b.mor_expert_desc_t:
    if m.dim() != 2:
        raise ValueError(f"a matrix is wanted, got {tuple(m.shape)}")
    _rows_contiguous(m, "matrix")
    d = _b.mor_expert_desc_t(plan.row.shape[0], plan.slot.shape[0], m.shape[1], plan.top, _dtype(m.dtype, "matrix"), plan.row.data_ptr(),
                             plan.slot.data_ptr())
    if weight is not None:
        if weight.shape != plan.row.shape or not weight.is_contiguous() or weight.device != m.device:
            raise ValueError(f"weight: contiguous {tuple(plan.row.shape)} on the matrix's device is wanted")
        d.weight, d.weight_dtype = weight.data_ptr(), _dtype(weight.dtype, "weight")
    return d


def _ld(m: torch.Tensor) -> int:
    return m.stride(0) if m.shape[0] > 1 else m.shape[1]


def gather(x: torch.Tensor, plan: Plan, weight=None) -> torch.Tensor:
    """[plan rows, hidden]: each row the token row of its slot, times weight [tokens, top] if given; zero where it has no slot."""
    index = _on_gpu(x, "x")
    d = _desc(plan, x, weight)
    if x.shape[0] != plan.row.shape[0]:
        raise ValueError(f"x: {plan.row.shape[0]} rows are wanted, got {x.shape[0]}")
    out = torch.empty((plan.slot.shape[0], x.shape[1]), dtype=x.dtype, device=x.device)
    _check((_b._lib or _b.load()).mor_expert_gather(C.byref(d), x.data_ptr(), _ld(x), out.data_ptr(), x.shape[1], _raw_stream(index)), "mor_expert_gather")
    return out


def combine(ys: torch.Tensor, plan: Plan, weight=None) -> torch.Tensor:
    """[tokens, hidden]: the sum over each token's slots of weight (1 if not given) times the slot's row of ys."""
    index = _on_gpu(ys, "ys")
    d = _desc(plan, ys, weight)
    if ys.shape[0] != plan.slot.shape[0]:
        raise ValueError(f"ys: {plan.slot.shape[0]} rows are wanted, got {ys.shape[0]}")
    out = torch.empty((plan.row.shape[0], ys.shape[1]), dtype=ys.dtype, device=ys.device)
    _check((_b._lib or _b.load()).mor_expert_combine(C.byref(d), ys.data_ptr(), _ld(ys), out.data_ptr(), ys.shape[1], _raw_stream(index)), "mor_expert_combine")
    return out


def combine_grad(dy: torch.Tensor, ys: torch.Tensor, plan: Plan, weight: torch.Tensor, *, rows: bool = True):
    """(dys or None, dweight): the gradients of combine(ys, plan, weight) for dy."""
    index = _on_gpu(dy, "dy")
    d = _desc(plan, dy, weight)
    if dy.shape[0] != plan.row.shape[0] or ys.shape != (plan.slot.shape[0], dy.shape[1]) or ys.dtype != dy.dtype or ys.device != dy.device:
        raise ValueError("dy: [tokens, hidden] and ys: [plan rows, hidden] of one type and device are wanted")
    _rows_contiguous(ys, "ys")
    dys = torch.empty((plan.slot.shape[0], dy.shape[1]), dtype=dy.dtype, device=dy.device) if rows else None
    dweight = torch.empty_like(weight)
    _check((_b._lib or _b.load()).mor_expert_combine_grad(C.byref(d), dy.data_ptr(), _ld(dy), ys.data_ptr(), _ld(ys), dys.data_ptr() if rows else None,
                                                          dy.shape[1], dweight.data_ptr(), _raw_stream(index)), "mor_expert_combine_grad")
    return dys, dweight


def _forward(x, stack, plan, weight, cols):
    """(y, the experts' rows, operand of x's gathered rows along the rows axis)."""
    a, a_t = fp4.quantize(x, stack.format, cols=cols, gather=plan)
    ys = fp4.matmul_rows(a, stack, plan, x.dtype)
    return combine(ys, plan, weight), ys, a_t


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, ids, weight, format):
        need_x, need_w = ctx.needs_input_grad[:2]
        plan = sort(ids, w.shape[0], 128)
        b, ctx.b_t = fp4.quantize(w, format, cols=need_x)
        y, ys, ctx.a_t = _forward(x, b, plan, weight, need_w)
        ctx.plan, ctx.format, ctx.dtypes = plan, format, (x.dtype, w.dtype)
        ctx.save_for_backward(weight, ys if ctx.needs_input_grad[3] else None)
        return y

    @staticmethod
    def backward(ctx, dy):
        need_x, need_w, _, need_weight, _ = ctx.needs_input_grad
        weight, ys = ctx.saved_tensors
        plan = ctx.plan
        dy = dy if dy.stride(-1) == 1 else dy.contiguous()
        dx = dw = dweight = None
        if need_weight:
            _, dweight = combine_grad(dy, ys, plan, weight, rows=False)
        if need_x or need_w:
            g, g_t = fp4.quantize(dy, ctx.format, rows=need_x, cols=need_w, gather=plan, weight=weight)
            if need_x:
                dx = combine(fp4.matmul_rows(g, ctx.b_t, plan, ctx.dtypes[0]), plan)
            if need_w:
                dw = fp4.matmul_reduce(g_t, ctx.a_t, plan, ctx.dtypes[1])
        return dx, dw, None, dweight, None


def linear(x: torch.Tensor, w, ids: torch.Tensor, weight: torch.Tensor, format: str = None) -> torch.Tensor:
    """y[t] = sum over j of weight[t, j] * Q(x[t]) Q(w[ids[t, j]])^T for x [tokens, n_in] and w [experts, n_out, n_in].

    ``w`` is a tensor (differentiable in x, w and weight; the rounding is passed straight through) or, for serving, a stored stack
    (``fp4.Operand`` with one matrix per expert; ``format`` is then its own)."""
    if isinstance(w, fp4.Operand):
        return _forward(x, w, sort(ids, w.batch, 128), weight, False)[0]
    if w.dim() != 3 or x.dim() != 2 or x.shape[1] != w.shape[2]:
        raise ValueError(f"x [tokens, n_in] and w [experts, n_out, n_in] are wanted, got {tuple(x.shape)} and {tuple(w.shape)}")
    return _Linear.apply(x, w, ids, weight, format)

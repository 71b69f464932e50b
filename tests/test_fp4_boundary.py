"""Refusals of the 4-bit and routing entry points, without a GPU: every bad argument is reported before anything is launched."""
import ctypes as C

import pytest

from paper_2512_22804_b200 import binding as mb
from paper_2512_22804_b200 import build as mbuild


@pytest.fixture(scope="module")
def lib():
    mbuild.build()
    return mb.load()


def matrix(batch=1, rows=256, cols=128, ld=None, fmt=0, codes=0x10000, scales=0x20000, t=0x30000):
    return mb.mor_fp4_matrix_t(codes, scales, t, batch, rows, cols, (cols + 31) // 32 * 16 if ld is None else ld, fmt)


def quant(**kw):
    d = mb.mor_fp4_quantize_desc_t(0x40000, 0, 0, 1, 256, 128, 128, 0)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def test_scale_bytes(lib):
    f = lib.mor_fp4_scale_bytes
    assert f(1, 1, 1, 0) == 512 and f(1, 128, 64, 0) == 512 and f(1, 129, 65, 0) == 2048
    assert f(1, 128, 128, 1) == 512 and f(3, 128, 129, 1) == 3 * 1024 and f(1, 0, 64, 0) == 0
    assert f(-1, 1, 1, 0) == 0 and f(1, 1, 1, 2) == 0 and f(1, 1 << 40, 1, 0) == 0


INVALID, ALIGN, WORKSPACE = mb.MOR_ERR_INVALID_ARG, mb.MOR_ERR_ALIGNMENT, mb.MOR_ERR_WORKSPACE


@pytest.mark.parametrize("d,rows,cols,want", [
    (quant(), None, None, INVALID),
    (quant(dtype=2), matrix(), None, INVALID),
    (quant(format=2), matrix(fmt=2), None, INVALID),
    (quant(rows=-1), matrix(rows=-1), None, INVALID),
    (quant(ld=127), matrix(), None, INVALID),
    (quant(x=None), matrix(), None, INVALID),
    (quant(x=0x40001), matrix(), None, ALIGN),
    (quant(dtype=1, x=0x40002), matrix(), None, ALIGN),
    (quant(), matrix(fmt=1), None, INVALID),                     # formats differ
    (quant(), matrix(rows=255), None, INVALID),
    (quant(), None, matrix(), INVALID),                          # the transpose is [128, 256]
    (quant(), matrix(ld=48), None, INVALID),                     # shorter than a row
    (quant(), matrix(ld=72), None, ALIGN),
    (quant(), matrix(codes=0x10008), None, ALIGN),
    (quant(), matrix(scales=0x20004), None, ALIGN),
    (quant(), matrix(codes=None), None, INVALID),
    (quant(), matrix(t=None), None, INVALID),
    (quant(weight=0x5000), matrix(), None, INVALID),             # weights without slots
    (quant(slot_of_row=0x5000, out_rows=256), matrix(), None, INVALID),                          # row_of_slot missing
    (quant(slot_of_row=0x5000, row_of_slot=0x6000, out_rows=256, top=0), matrix(), None, INVALID),
    (quant(slot_of_row=0x5000, row_of_slot=0x6000, out_rows=256, top=2, weight=0x7000, weight_dtype=5), matrix(), None, INVALID),
    (quant(batch=2, slot_of_row=0x5000, row_of_slot=0x6000, out_rows=256, top=1), matrix(batch=2), None, INVALID),
    (quant(), matrix(), None, WORKSPACE),                        # valid, but the maximum has to be taken and there is no scratch
])
def test_quantize_refuses(lib, d, rows, cols, want):
    assert lib.mor_fp4_quantize(C.byref(d), None if rows is None else C.byref(rows), None if cols is None else C.byref(cols), None, 0, None) == want
    assert lib.mor_fp4_quantize(None, None, None, None, 0, None) == INVALID


def test_quantize_checks_its_workspace(lib):
    d, r = quant(), matrix()
    assert lib.mor_fp4_quantize(C.byref(d), C.byref(r), None, 0x10000, mb.MOR_FP4_WORKSPACE_BYTES - 1, None) == WORKSPACE
    assert lib.mor_fp4_quantize(C.byref(d), C.byref(r), None, 0x10008, mb.MOR_FP4_WORKSPACE_BYTES, None) == ALIGN


@pytest.mark.parametrize("m,out,dtype,ld,want", [
    (matrix(), 0x1000, 2, 128, INVALID), (matrix(), 0x1000, 0, 127, INVALID), (matrix(), None, 0, 128, INVALID), (matrix(), 0x1001, 0, 128, ALIGN),
    (matrix(fmt=7), 0x1000, 0, 128, INVALID)])
def test_dequantize_refuses(lib, m, out, dtype, ld, want):
    assert lib.mor_fp4_dequantize(C.byref(m), out, dtype, ld, None) == want
    assert lib.mor_fp4_dequantize(None, 0x1000, 0, 128, None) == INVALID


def product(a=None, b=None, **kw):
    d = mb.mor_fp4_matmul_desc_t(a or matrix(), b or matrix(rows=64), 0x50000, 0, 0, 64, None, 0, None, None)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("d,want", [
    (product(out_dtype=3), INVALID),
    (product(grouping=3), INVALID),
    (product(b=matrix(rows=64, fmt=1)), INVALID),
    (product(b=matrix(rows=64, cols=160)), INVALID),
    (product(a=matrix(batch=2)), INVALID),
    (product(b=matrix(batch=2, rows=64)), INVALID),
    (product(ldo=63), INVALID),
    (product(ldo=68), ALIGN),
    (product(out=0x50008), ALIGN),
    (product(out=None), INVALID),
    (product(grouping=1, groups=2), INVALID),                                                   # no starts
    (product(grouping=1, groups=2, starts=0x6000), INVALID),                                    # one matrix, two groups
    (product(grouping=1, groups=0, starts=0x6000), INVALID),
    (product(grouping=2, groups=mb.MOR_MAX_GROUPS + 1, starts=0x6000), INVALID),
    (product(grouping=2, groups=2, starts=0x6002), ALIGN),
    (product(grouping=2, groups=1, starts=0x6000, slot_of_row=0x7000), INVALID), (product(slot_of_row=0x7000), INVALID),
    (product(a=matrix(codes=0x10004)), ALIGN),
])
def test_matmul_refuses(lib, d, want):
    assert lib.mor_fp4_matmul(C.byref(d), None) == want
    assert lib.mor_fp4_matmul(None, None) == INVALID


def test_expert_rows_and_workspace(lib):
    assert lib.mor_expert_rows(8, 64, 1) == 8 and lib.mor_expert_rows(8, 64, 128) == 1024 and lib.mor_expert_rows(0, 3, 128) == 0
    assert lib.mor_expert_rows(1000, 4, 128) == (1000 + 4 * 127) // 128 * 128
    assert lib.mor_expert_rows(1, 0, 1) == -1 and lib.mor_expert_rows(-1, 4, 1) == -1 and lib.mor_expert_rows(4, mb.MOR_MAX_GROUPS + 1, 1) == -1
    assert lib.mor_expert_workspace_bytes(1 << 20, 64) >= 148 * 64 * 4 and lib.mor_expert_workspace_bytes(8, 64) > 0


@pytest.mark.parametrize("args,want", [
    ((0x1000, 8, 0, 1, 0x2000, 0x3000, 0x4000), INVALID), ((0x1000, 8, 4, 0, 0x2000, 0x3000, 0x4000), INVALID),
    ((None, 8, 4, 1, 0x2000, 0x3000, 0x4000), INVALID), ((0x1000, 8, 4, 1, None, 0x3000, 0x4000), INVALID),
    ((0x1002, 8, 4, 1, 0x2000, 0x3000, 0x4000), ALIGN), ((0x1000, 1 << 20, 4, 1, 0x2000, 0x3000, 0x4000), WORKSPACE),
    ((0x1000, 1 << 31, 4, 1, 0x2000, 0x3000, 0x4000), INVALID)])
def test_sort_refuses(lib, args, want):
    assert lib.mor_expert_sort(*args, None, 0, None) == want


def moves(**kw):
    d = mb.mor_expert_desc_t(4, 8, 64, 2, 0, 0x1000, 0x2000)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("d,x,ldx,out,ldo,want", [
    (moves(dtype=4), 0x3000, 64, 0x4000, 64, INVALID), (moves(top=0), 0x3000, 64, 0x4000, 64, INVALID), (moves(tokens=-1), 0x3000, 64, 0x4000, 64, INVALID),
    (moves(row_of_slot=None), 0x3000, 64, 0x4000, 64, INVALID), (moves(slot_of_row=None), 0x3000, 64, 0x4000, 64, INVALID),
    (moves(weight=0x5000, weight_dtype=9), 0x3000, 64, 0x4000, 64, INVALID), (moves(weight=0x5001), 0x3000, 64, 0x4000, 64, ALIGN),
    (moves(), 0x3000, 63, 0x4000, 64, INVALID), (moves(), None, 64, 0x4000, 64, INVALID), (moves(), 0x3001, 64, 0x4000, 64, ALIGN),
    (moves(ys_dtype=3), 0x3000, 64, 0x4000, 64, INVALID), (moves(dtype=1, ys_dtype=0), 0x3000, 64, 0x4000, 64, INVALID),
    (moves(), 0x3000, 64, 0x4000, 1, INVALID), (moves(), 0x3000, 64, None, 64, INVALID)])
def test_movers_refuse(lib, d, x, ldx, out, ldo, want):
    assert lib.mor_expert_gather(C.byref(d), x, ldx, out, ldo, None) == want
    assert lib.mor_expert_combine(C.byref(d), x, ldx, out, ldo, None) == want
    assert lib.mor_expert_combine_grad(C.byref(d), x, ldx, out, ldo, out, ldo, 0x6000, None) == want
    assert lib.mor_expert_gather(None, x, ldx, out, ldo, None) == INVALID


def test_gradient_of_nothing_is_refused(lib):
    assert lib.mor_expert_combine_grad(C.byref(moves()), 0x3000, 64, 0x4000, 64, None, 64, None, None) == INVALID


def test_python_refusals(lib):
    import torch

    from paper_2512_22804_b200 import experts, fp4

    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        fp4.quantize(x, "e8m0_32")
    with pytest.raises(KeyError):
        fp4.quantize(x, "e2m1")
    with pytest.raises(ValueError, match="batch"):
        fp4.quantize(x[0], "e8m0_32")
    with pytest.raises(TypeError):
        fp4.quantize(x.half(), 7.5)
    with pytest.raises(ValueError, match="codes"):
        fp4.Operand(x.to(torch.uint8), x.to(torch.uint8), 5, 8, "e8m0_32", torch.ones(1))
    with pytest.raises(TypeError, match="uint8"):
        fp4.Operand(x, x, 4, 8, "e8m0_32", torch.ones(1))
    with pytest.raises(ValueError, match="int32"):
        experts.sort(torch.zeros(4, 2, dtype=torch.int64), 4)
    with pytest.raises(ValueError, match="n_in"):
        fp4.linear(x, torch.zeros(4, 9), "e8m0_32")
    with pytest.raises(ValueError, match="n_in"):
        experts.linear(x, torch.zeros(2, 4, 9), None, None, "e8m0_32")


@pytest.mark.parametrize("format", [2, -1, 1 << 40, 1 << 80, -(1 << 80)])
def test_numbers_that_name_no_format_are_refused(lib, format):
    import torch

    from paper_2512_22804_b200 import fp4

    byte = torch.zeros(4, 16, dtype=torch.uint8)
    with pytest.raises(ValueError, match="format"):
        fp4.Operand(byte, byte, 4, 8, format, torch.ones(1))
    with pytest.raises(ValueError, match="format"):
        fp4.quantize(torch.zeros(4, 8), format)
    with pytest.raises(ValueError, match="CUDA"):
        fp4.quantize(torch.zeros(4, 8), 1)

"""Refusals of the norm's, the adapters' and the optimizer's entry points, without a GPU: every bad argument is reported before anything is launched."""
import ctypes as C

import pytest

from paper_2512_22804_b200 import binding as mb
from paper_2512_22804_b200 import build as mbuild

INVALID, ALIGN, WORKSPACE, OK = mb.MOR_ERR_INVALID_ARG, mb.MOR_ERR_ALIGNMENT, mb.MOR_ERR_WORKSPACE, mb.MOR_OK


@pytest.fixture(scope="module")
def lib():
    mbuild.build()
    return mb.load()


def struct(kind, base, kw):
    d = kind(*base)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def norm(**kw):
    return struct(mb.mor_norm_desc_t, (4, 256, 0x10000, None, 0x20000, 256, 256, 1e-6, 0, 0, 0), kw)


def outs(**kw):
    return struct(mb.mor_norm_outputs_t, (None, 0x30000, None, None, None, 0, 256, 0, 128), kw)


@pytest.mark.parametrize("d,o,want", [
    (norm(rows=-1), outs(), INVALID), (norm(cols=-1), outs(), INVALID), (norm(cols=1 << 31, ldx=1 << 31), outs(ldy=1 << 31), INVALID),
    (norm(dtype=2), outs(), INVALID), (norm(weight_dtype=-1), outs(), INVALID), (norm(eps=-1.0), outs(), INVALID), (norm(eps=float("nan")), outs(), INVALID),
    (norm(eps=float("inf")), outs(), INVALID), (norm(x=None), outs(), INVALID), (norm(weight=None), outs(), INVALID), (norm(ldx=255), outs(), INVALID),
    (norm(x=0x10001), outs(), ALIGN), (norm(dtype=1, x=0x10002), outs(), ALIGN), (norm(weight=0x20001), outs(), ALIGN),
    (norm(), outs(y=None), INVALID),                                            # nothing to make
    (norm(), outs(h=0x50000, ldh=256), INVALID),                                # a sum without a residual
    (norm(residual=0x40000, residual_dtype=7), outs(), INVALID), (norm(residual=0x40000, ldr=100), outs(), INVALID),
    (norm(residual=0x40000, residual_dtype=1), outs(h=0x50002, ldh=256), ALIGN),
    (norm(), outs(ldy=255), INVALID), (norm(), outs(y=0x30001), ALIGN), (norm(), outs(block=64), INVALID),
    (norm(), outs(codes=0x60000, ldc=256), INVALID),                            # codes without scales
    (norm(), outs(codes=0x60000, ldc=256, scale_e8m0=0x70000, scale_f32=0x80000), INVALID),
    (norm(), outs(codes=0x60000, ldc=255, scale_e8m0=0x70000), INVALID), (norm(), outs(codes=0x60000, ldc=256, scale_f32=0x80002), ALIGN),
    (norm(rows=0, x=None), outs(y=None), OK), (norm(cols=0, ldx=0), outs(ldy=0), OK)])
def test_norm_refuses(lib, d, o, want):
    assert lib.mor_rms_norm(C.byref(d), C.byref(o), None) == want
    assert lib.mor_rms_norm(None, C.byref(o), None) == INVALID and lib.mor_rms_norm(C.byref(norm()), None, None) == INVALID


def norm_grad(lib, d, has=0, dy=0x30000, lddy=256, dx=0x40000, lddx=256, dr=None, lddr=0, dw=None, ws=None, n=0):
    return lib.mor_rms_norm_grad(C.byref(d), has, dy, lddy, dx, lddx, dr, lddr, dw, ws, n, None)


def test_norm_grad_refuses(lib):
    need = lib.mor_rms_norm_grad_workspace_bytes(4, 256)
    assert need > 0 and lib.mor_rms_norm_grad_workspace_bytes(-1, 4) == 0 and lib.mor_rms_norm_grad_workspace_bytes(4, -1) == 0
    assert norm_grad(lib, norm(), dx=None) == INVALID
    assert norm_grad(lib, norm(), dy=None) == INVALID and norm_grad(lib, norm(), dy=0x30001) == ALIGN and norm_grad(lib, norm(), lddy=255) == INVALID
    assert norm_grad(lib, norm(), lddx=255) == INVALID and norm_grad(lib, norm(), dx=0x40001) == ALIGN
    assert norm_grad(lib, norm(residual_dtype=3), has=1) == INVALID
    assert norm_grad(lib, norm(residual_dtype=1), has=1, dr=0x50002, lddr=256) == ALIGN
    assert norm_grad(lib, norm(residual_dtype=1, x=0x10002), has=1) == ALIGN
    assert norm_grad(lib, norm(), dw=0x60000) == WORKSPACE and norm_grad(lib, norm(), dw=0x60000, ws=0x70000, n=need - 1) == WORKSPACE
    assert norm_grad(lib, norm(), dw=0x60000, ws=0x70008, n=need) == ALIGN and norm_grad(lib, norm(), dw=0x60001, ws=0x70000, n=need) == ALIGN


@pytest.mark.parametrize("kw,want", [
    (dict(rows=-1), INVALID), (dict(cols=-1), INVALID), (dict(dtype=2), INVALID), (dict(block=64), INVALID), (dict(ldc=127), INVALID), (dict(ldo=127), INVALID),
    (dict(codes=None), INVALID), (dict(out=None), INVALID), (dict(e8m0=None), INVALID), (dict(f32=0x40000), INVALID), (dict(e8m0=None, f32=0x40002), ALIGN),
    (dict(out=0x30001), ALIGN), (dict(rows=0), OK), (dict(cols=0), OK)])
def test_dequantize_refuses(lib, kw, want):
    a = dict(codes=0x10000, rows=4, cols=128, ldc=128, block=128, e8m0=0x20000, f32=None, out=0x30000, dtype=0, ldo=128)
    a.update(kw)
    assert lib.mor_codes_dequantize(a["codes"], a["rows"], a["cols"], a["ldc"], a["block"], a["e8m0"], a["f32"], a["out"], a["dtype"], a["ldo"], None) == want


def adapter(**kw):
    return struct(mb.mor_adapter_desc_t, (1000, 256, 512, 4, 16, 0x10000, 0x20000, 0x30000, 0x40000, 1.0), kw)


BAD = [(dict(tokens=-1), INVALID), (dict(tokens=1 << 30), INVALID), (dict(n_in=0), INVALID), (dict(n_out=0), INVALID), (dict(n_in=(1 << 21) + 1), INVALID), (dict(n_out=(1 << 21) + 1), INVALID),
       (dict(adapters=0), INVALID), (dict(adapters=mb.MOR_MAX_GROUPS), INVALID), (dict(rank=0), INVALID), (dict(rank=513), INVALID), (dict(a=None), INVALID), (dict(b=None), INVALID),
       (dict(a=0x10001), ALIGN), (dict(b=0x20001), ALIGN), (dict(ids=0x30002), ALIGN), (dict(scale=0x40001), ALIGN)]


def add(lib, d, x=0x50000, ldx=None, base=0x60000, ldb=None, out=0x70000, ldo=None, dtype=0, train=0, ws=0x100000, n=1 << 40):
    ldx, ldb, ldo = (max(0, w if v is None else v) for v, w in ((ldx, d.n_in), (ldb, d.n_out), (ldo, d.n_out)))
    return lib.mor_adapter_add(C.byref(d), x, ldx, base, ldb, out, ldo, dtype, train, ws, n, None)


def grad(lib, d, x=0x50000, ldx=None, dy=0x60000, lddy=None, dx=0x70000, lddx=None, da=0x80000, db=0x90000, saved=0x100000, ns=1 << 40, ws=0x200000, n=1 << 40, base=None, ldb=0):
    ldx, lddy, lddx = (max(0, w if v is None else v) for v, w in ((ldx, d.n_in), (lddy, d.n_out), (lddx, d.n_in)))
    return lib.mor_adapter_grad(C.byref(d), x, ldx, dy, lddy, base, ldb, dx, lddx, da, db, saved, ns, ws, n, None)


@pytest.mark.parametrize("kw,want", BAD)
def test_adapters_refuse_their_description(lib, kw, want):
    d = adapter(**kw)
    assert add(lib, d) == want and grad(lib, d) == want
    assert lib.mor_adapter_workspace_bytes(C.byref(d), 1) == 0 and lib.mor_adapter_grad_workspace_bytes(C.byref(d)) == 0


def test_adapters_refuse(lib):
    d = adapter()
    assert lib.mor_adapter_add(None, 0, 0, 0, 0, 0, 0, 0, 0, None, 0, None) == INVALID
    assert add(lib, d, dtype=2) == INVALID and add(lib, d, x=None) == INVALID and add(lib, d, base=None) == INVALID and add(lib, d, out=None) == INVALID
    assert add(lib, d, ldx=255) == INVALID and add(lib, d, ldb=511) == INVALID and add(lib, d, ldo=511) == INVALID
    assert add(lib, d, x=0x50001) == ALIGN and add(lib, d, base=0x60002, dtype=1) == ALIGN and add(lib, d, out=0x70001) == ALIGN
    need = lib.mor_adapter_workspace_bytes(C.byref(d), 0)
    assert need > 0 and add(lib, d, ws=None) == WORKSPACE and add(lib, d, n=need - 1) == WORKSPACE and add(lib, d, ws=0x100010) == ALIGN
    train = lib.mor_adapter_workspace_bytes(C.byref(d), 1)
    assert train >= need and add(lib, d, train=1, n=train - 1) == WORKSPACE
    few = adapter(tokens=8)
    assert lib.mor_adapter_workspace_bytes(C.byref(few), 0) == 0 and lib.mor_adapter_workspace_bytes(C.byref(few), 1) > 0
    assert lib.mor_adapter_workspace_bytes(C.byref(adapter(tokens=8, rank=65)), 0) > 0
    assert add(lib, adapter(tokens=0), x=None, base=None, out=None) == OK


def test_adapter_gradients_refuse(lib):
    d = adapter()
    need = lib.mor_adapter_grad_workspace_bytes(C.byref(d))
    train = lib.mor_adapter_workspace_bytes(C.byref(d), 1)
    assert grad(lib, d, x=None) == INVALID and grad(lib, d, dy=None) == INVALID and grad(lib, d, ldx=255) == INVALID and grad(lib, d, lddy=511) == INVALID and grad(lib, d, lddx=255) == INVALID
    assert grad(lib, d, dy=0x60001) == ALIGN and grad(lib, d, da=0x80001) == ALIGN and grad(lib, d, db=0x90001) == ALIGN and grad(lib, d, dx=0x70001) == ALIGN
    assert grad(lib, d, base=0xA0000, ldb=255) == INVALID and grad(lib, d, base=0xA0001, ldb=256) == ALIGN
    assert grad(lib, d, saved=None) == WORKSPACE and grad(lib, d, ns=train - 1) == WORKSPACE and grad(lib, d, ws=None) == WORKSPACE and grad(lib, d, n=need - 1) == WORKSPACE
    assert grad(lib, d, saved=0x100080) == ALIGN and grad(lib, d, ws=0x200080) == ALIGN


def step(**kw):
    return struct(mb.mor_adamw_desc_t, (1e-3, 0.9, 0.999, 1e-8, 0.01, 1, None, None, None, None, 0, 0, 0, 1), kw)


def tensor(**kw):
    return struct(mb.mor_adamw_tensor_t, (0x10000, 0x20000, 0x30000, 0x40000, 0x50000, 1000), kw)


@pytest.mark.parametrize("d,t,want", [
    (step(param_dtype=2), tensor(), INVALID), (step(grad_dtype=2), tensor(), INVALID), (step(lr=-1.0), tensor(), INVALID), (step(lr=float("nan")), tensor(), INVALID),
    (step(beta1=1.0), tensor(), INVALID), (step(beta2=-0.1), tensor(), INVALID), (step(beta2=float("nan")), tensor(), INVALID), (step(eps=-1.0), tensor(), INVALID),
    (step(eps=float("inf")), tensor(), INVALID), (step(weight_decay=-1.0), tensor(), INVALID), (step(step=0), tensor(), INVALID), (step(device_step=2), tensor(), ALIGN),
    (step(device_lr=2), tensor(), ALIGN), (step(grad_scale=2), tensor(), ALIGN), (step(found_inf=2), tensor(), ALIGN),
    (step(), tensor(numel=-1), INVALID), (step(), tensor(numel=1 << 40), INVALID), (step(), tensor(param=None), INVALID), (step(), tensor(grad=None), INVALID),
    (step(), tensor(exp_avg=None), INVALID), (step(), tensor(exp_avg_sq=None), INVALID), (step(), tensor(scales=None), INVALID), (step(), tensor(scales=0x50001), ALIGN),
    (step(), tensor(param=0x10001), ALIGN), (step(grad_dtype=1), tensor(grad=0x20002), ALIGN), (step(eight_bits=0), tensor(exp_avg=0x30001), ALIGN),
    (step(), tensor(numel=0, param=None, grad=None), OK)])
def test_adamw_refuses(lib, d, t, want):
    assert lib.mor_adamw(C.byref(d), C.byref(t), 1, None) == want
    assert lib.mor_adamw(None, C.byref(t), 1, None) == INVALID and lib.mor_adamw(C.byref(step()), None, 1, None) == INVALID and lib.mor_adamw(C.byref(step()), None, -1, None) == INVALID
    assert lib.mor_adamw(C.byref(step()), None, 0, None) == OK


def test_moments_refuse(lib):
    f = lib.mor_adamw_moments
    assert f(1, 1, 2, -1, 4, 4, 0, None) == INVALID and f(1, 1, 2, 8, 4, 4, 2, None) == INVALID and f(1, 1, None, 8, 4, 4, 0, None) == INVALID
    assert f(None, 1, 2, 8, 4, 4, 0, None) == INVALID and f(1, None, 2, 8, 4, 4, 0, None) == INVALID and f(1, 1, 2, 8, None, None, 0, None) == INVALID
    assert f(1, 1, 3, 8, 4, 4, 0, None) == ALIGN and f(1, 1, 2, 8, 5, 4, 0, None) == ALIGN and f(1, 1, 2, 8, 4, 6, 1, None) == ALIGN and f(None, None, None, 0, None, None, 0, None) == OK


def test_adamw_refuses_numbers(lib):
    for last, want in ((1 << 31, INVALID), ((1 << 32) - 1, INVALID), ((1 << 31) - 1, OK)):
        numbers = (C.c_uint32 * 2)(0, last)
        t = (mb.mor_adamw_tensor_t * 2)(tensor(numel=0), tensor(numel=0))
        assert lib.mor_adamw(C.byref(step(numbers=C.addressof(numbers))), t, 2, None) == want

"""The 4-bit layers as autograd and serving code meets them: gradients with any strides, results that are changed in place, saved tensors,
second derivatives, streams, modes and errors."""
import os
import subprocess
import sys

import numpy as np
import pytest

from tests import plain_fp4 as plain

pytestmark = pytest.mark.gpu
FORMATS = ["e4m3_16", "e8m0_32"]
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def fp4():
    from paper_2512_22804_b200 import fp4

    return fp4


@pytest.fixture(scope="module")
def experts():
    from paper_2512_22804_b200 import experts

    return experts


def drawn(shape, seed, dtype="bf16", scale=1.0):
    import torch

    t = torch.from_numpy((np.random.default_rng(seed).standard_normal(shape) * scale).astype(np.float32)).cuda()
    return t.to(torch.bfloat16) if dtype == "bf16" else t


def layer(which, fmt, tokens, n_out, seed=0, n_in=96):
    """(inputs that take a gradient, call) of a linear layer or an expert layer."""
    import torch

    from paper_2512_22804_b200 import experts, fp4

    x = drawn((tokens, n_in), seed).requires_grad_()
    if which == "linear":
        w = drawn((n_out, n_in), seed + 1, scale=0.1).requires_grad_()
        return (x, w), lambda: fp4.linear(x, w, fmt)
    w = drawn((3, n_out, n_in), seed + 1, scale=0.1).requires_grad_()
    weight = torch.rand(tokens, 2, generator=torch.Generator().manual_seed(seed)).cuda().requires_grad_()
    ids = torch.from_numpy(np.random.default_rng(seed).integers(-1, 3, (tokens, 2)).astype(np.int32)).cuda()
    return (x, w, weight), lambda: experts.linear(x, w, ids, weight, fmt)


# ------------------------------------------------------------------------------------- gradients with any strides

@pytest.mark.parametrize("which", ["linear", "experts"])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("tokens,n_out", [(1, 40), (50, 40), (300, 137), (50, 1), (1, 1)])
def test_broadcast_gradients(fp4, which, fmt, tokens, n_out):
    """Sums over the tokens (and over everything) hand back gradients with row strides of zero: the same as dense ones."""
    import torch

    inputs, call = layer(which, fmt, tokens, n_out)
    v = drawn((n_out,), 7)
    got = torch.autograd.grad((call().sum(0) * v).sum(), inputs)
    want = torch.autograd.grad(call(), inputs, v.expand(tokens, n_out).contiguous())
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    got = torch.autograd.grad(call().sum(), inputs)
    want = torch.autograd.grad(call(), inputs, torch.ones(tokens, n_out, device="cuda", dtype=torch.bfloat16))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    got = torch.autograd.grad(call(), inputs, drawn((n_out, tokens), 8).t())
    want = torch.autograd.grad(call(), inputs, drawn((n_out, tokens), 8).t().contiguous())
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    if n_out == 1:
        got = torch.autograd.grad(call().squeeze(-1).sum(), inputs)
        want = torch.autograd.grad(call(), inputs, torch.ones(tokens, 1, device="cuda", dtype=torch.bfloat16))
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("fmt", FORMATS)
def test_broadcast_gradients_of_three_dimensions(fp4, fmt):
    import torch

    x, w, v = drawn((4, 30, 96), 1).requires_grad_(), drawn((40, 96), 2).requires_grad_(), drawn((40,), 3)
    got = torch.autograd.grad((fp4.linear(x, w, fmt).sum((0, 1)) * v).sum(), (x, w))
    want = torch.autograd.grad(fp4.linear(x, w, fmt), (x, w), v.expand(4, 30, 40).contiguous())
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("which", ["linear", "experts"])
@pytest.mark.parametrize("fmt", FORMATS)
def test_inputs_with_any_strides(fp4, which, fmt):
    import torch

    inputs, _ = layer(which, fmt, 50, 40)
    x, w = (t.detach() for t in inputs[:2])
    ids, weight = torch.arange(100, device="cuda", dtype=torch.int32).view(50, 2) % 3, torch.rand(50, 2, device="cuda")

    def call(x, w):
        from paper_2512_22804_b200 import experts

        return fp4.linear(x, w, fmt) if which == "linear" else experts.linear(x, w, ids, weight, fmt)

    row, column = x[:1].expand(50, -1), x.t().contiguous().t()
    for v in (row, column, x[:, :1].expand(-1, 96)):
        for u in (w, w.transpose(-1, -2).contiguous().transpose(-1, -2), w[..., :1, :].expand_as(w)):
            tv, tu = (t.detach().requires_grad_() for t in (v, u))
            dv, du = (t.contiguous().requires_grad_() for t in (v, u))
            y, want = call(tv, tu), call(dv, du)
            assert torch.equal(y, want)
            for a, b in zip(torch.autograd.grad(y.sum(), (tv, tu)), torch.autograd.grad(want.sum(), (dv, du))):
                assert torch.equal(a, b)


# ------------------------------------------------------------------------------------- results that are changed in place

@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("tokens", [5, 200])
@pytest.mark.parametrize("n_out", [136, 137])
def test_results_change_in_place(fp4, fmt, tokens, n_out):
    import torch

    (x, w), call = layer("linear", fmt, tokens, n_out)
    bias, dy = drawn((n_out,), 5).requires_grad_(), drawn((tokens, n_out), 6)
    y = call()
    y.add_(bias)
    torch.relu_(y)
    want = torch.relu(call() + bias)
    assert torch.equal(y, want)
    for a, b in zip(torch.autograd.grad(y, (x, w, bias), dy), torch.autograd.grad(want, (x, w, bias), dy)):
        assert torch.equal(a, b)
    x3 = x.detach().reshape(1, tokens, -1)
    y3 = fp4.linear(x3.requires_grad_(), w, fmt)
    y3 += bias
    assert torch.equal(torch.relu(y3[0]), want)


# ------------------------------------------------------------------------------------- what is kept for the backward pass

@pytest.mark.parametrize("which", ["linear", "experts"])
def test_hooks_on_saved_tensors_see_what_is_kept(fp4, which):
    """All that a backward pass needs goes through the hooks: a layer whose saved tensors are taken to the host keeps nothing on the GPU."""
    import torch

    tokens, n_out, n_in = 2048, 1024, 1024
    inputs, call = layer(which, "e8m0_32", tokens, n_out, n_in=n_in)
    dy = drawn((tokens, n_out), 9)
    want = torch.autograd.grad(call(), inputs, dy)
    def held():                                        # bytes asked for; what the allocator rounds them up to depends on what it has free
        return torch.cuda.memory_stats()["requested_bytes.all.current"]

    before = held()
    with torch.autograd.graph.save_on_cpu():
        y = call()
    assert held() - before <= y.numel() * 2
    got = torch.autograd.grad(y, inputs, dy)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("which", ["linear", "experts"])
def test_a_second_backward_pass_needs_retain_graph(fp4, which):
    import torch

    inputs, call = layer(which, "e8m0_32", 50, 40)
    y, dy = call(), drawn((50, 40), 9)
    first = torch.autograd.grad(y, inputs, dy, retain_graph=True)
    second = torch.autograd.grad(y, inputs, dy)
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    with pytest.raises(RuntimeError, match="second time"):
        torch.autograd.grad(y, inputs, dy)


# ------------------------------------------------------------------------------------- what has no derivative

@pytest.mark.parametrize("which", ["linear", "experts"])
def test_a_second_derivative_is_refused(fp4, which):
    import torch

    inputs, call = layer(which, "e8m0_32", 50, 40)
    dy = drawn((50, 40), 9)
    plain_grads = torch.autograd.grad(call(), inputs, dy)
    grads = torch.autograd.grad(call(), inputs, dy, create_graph=True)
    assert all(torch.equal(a, b) for a, b in zip(grads, plain_grads))
    for g in grads:
        loss = (g.float() ** 2).sum() + sum((t.float() ** 2).sum() for t in inputs)      # another path keeps the graph alive
        with pytest.raises(RuntimeError, match="twice"):
            torch.autograd.grad(loss, inputs, retain_graph=True)


def test_what_has_no_gradient_says_so(fp4, experts):
    import torch

    x, ys = drawn((20, 64), 1).requires_grad_(), drawn((40, 64), 2).requires_grad_()
    weight = torch.rand(20, 2, device="cuda", requires_grad=True)
    ids = torch.arange(40, device="cuda", dtype=torch.int32).view(20, 2) % 4
    plan = experts.sort(ids, 4)
    stored = fp4.quantize(drawn((4, 24, 64), 3), "e8m0_32")[0]
    plan_rows = experts.gather(x, plan)
    for out in (plan_rows, experts.gather(x.detach(), plan, weight), experts.combine(ys, plan), experts.combine(ys.detach(), plan, weight),
                *experts.combine_grad(x, ys, plan, weight.detach()), experts.linear(x, stored, ids, weight.detach())):
        with pytest.raises(RuntimeError, match="gradient"):
            out.float().sum().backward()
    with torch.no_grad():
        assert not experts.gather(x, plan).requires_grad and torch.equal(experts.gather(x, plan), plan_rows)
    assert not experts.gather(x.detach(), plan).requires_grad


# ------------------------------------------------------------------------------------- streams, modes, errors

def test_check_waits_for_every_stream(fp4):
    """A product on another stream whose bounded wait runs out after some 50 ms (a host-set hook leaves out one tile's copy)."""
    import ctypes

    import torch

    from paper_2512_22804_b200 import binding as mb

    hook = mb.load().mor_test_skip_tile_load
    hook.argtypes, hook.restype = [ctypes.c_uint32, ctypes.c_longlong], None
    a, b = (fp4.quantize(drawn((n, 512), n), "e8m0_32")[0] for n in (300, 264))
    fp4.matmul(a, b)
    fp4.check()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    hook(0, 100_000_000)
    try:
        with torch.cuda.stream(side):
            fp4.matmul(a, b)
    finally:
        hook(0xFFFFFFFF, 0)
    try:
        with pytest.raises(mb.MorError) as e:
            fp4.check()
        assert e.value.status == mb.MOR_ERR_TIMEOUT
    finally:
        torch.cuda.synchronize()
    fp4.check()


def in_fresh_process(code):
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


def test_check_after_a_first_product_in_inference_mode():
    in_fresh_process("""
import torch
from paper_2512_22804_b200 import fp4
x = torch.randn(20, 64, device="cuda").to(torch.bfloat16)
with torch.inference_mode():
    a = fp4.quantize(x, "e8m0_32")[0]
    y = fp4.matmul(a, a)
fp4.check()
with torch.inference_mode():
    fp4.check()
fp4.check("cuda:0")
fp4.check(0)
""")


def test_running_out_of_memory_is_torchs_error(fp4):
    """2 TB of result: refused by the allocator, as for torch's own product."""
    import torch

    a = fp4.quantize(torch.zeros(1 << 20, 32, device="cuda", dtype=torch.bfloat16), "e8m0_32")[0]
    with pytest.raises(torch.OutOfMemoryError):
        fp4.matmul(a, a)


@pytest.mark.parametrize("shape", [(0, 64), (64, 0), (3, 0, 64)])
def test_tensor_scale_of_nothing(fp4, shape):
    import torch

    for fmt, t in (("e8m0_32", np.float32(1)), ("e4m3_16", np.float32(2.0 ** -88) * (np.float32(1) / np.float32(2688)))):
        poison = [torch.full((512,), 255, device="cuda", dtype=torch.uint8) for _ in range(8)]
        del poison
        r, c = fp4.quantize(torch.zeros(shape, device="cuda", dtype=torch.bfloat16), fmt, cols=True)
        assert r.tensor_scale.item() == t and c.tensor_scale.item() == t
    r, _ = fp4.quantize(torch.zeros(shape, device="cuda", dtype=torch.bfloat16), "e4m3_16", amax=torch.tensor([2688.0], device="cuda"))
    assert r.tensor_scale.item() == np.float32(2688) * (np.float32(1) / np.float32(2688))


# ------------------------------------------------------------------------------------- operands far from one

@pytest.mark.parametrize("m", [5, 300])
@pytest.mark.parametrize("ea,eb", [(-60, -60), (-70, -30), (-51, -52), (-85, 60), (100, -80), (60, 40)])
def test_products_of_operands_far_from_one(fp4, m, ea, eb):
    """|x| about 2^ea and 2^eb: the product of the tensor scales alone need not be a normal number, the results are."""
    import torch

    xa, xb = (plain.bf16((np.random.default_rng(s).standard_normal((r, 300)) * 2.0 ** e).astype(np.float32)) for s, r, e in ((1, m, ea), (2, 140, eb)))
    a, b = (fp4.quantize(torch.from_numpy(v).cuda().to(torch.bfloat16), "e4m3_16")[0] for v in (xa, xb))
    va, vb = (plain.values(*plain.quantize(v, "e4m3_16"), "e4m3_16") for v in (xa, xb))
    y = fp4.matmul(a, b, torch.float32).cpu().numpy().astype(np.float64)
    assert (np.abs(y - va @ vb.T) <= np.abs(va) @ np.abs(vb).T * 2.0 ** -16 + 2.0 ** -149).all()


def test_zero_rows_beside_large_operands(fp4):
    """Both tensor scales together pass the largest number; rows of zeros still give zero."""
    import torch

    x = torch.zeros(200, 64, device="cuda", dtype=torch.bfloat16)
    x[0] = 2.0 ** 90
    a = fp4.quantize(x, "e4m3_16")[0]
    for part in (x[:4], x):
        y = fp4.matmul(fp4.quantize(part, "e4m3_16")[0], a, torch.float32)
        assert torch.isinf(y[0, 0]) and not y[1:].any() and not y[0, 1:].any()


# ------------------------------------------------------------------------------------- 32-bit rows, and one rounding

@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("start", [0, 1, 4])
def test_quantised_gather_of_32_bit_rows(fp4, experts, fmt, weighted, start):
    import torch

    for tokens, hidden in ((40, 96), (300, 333), (1100, 1544)):
        rng = np.random.default_rng(tokens)
        ids = rng.integers(-1, 6, (tokens, 3)).astype(np.int32)
        plan = experts.sort(torch.from_numpy(ids).cuda(), 6, 128)
        _, row, slot = plain.sort(ids, 6, 128)
        x, w = rng.standard_normal((tokens, hidden)).astype(np.float32), rng.random((tokens, 3)).astype(np.float32)
        rows = np.zeros((len(slot), hidden), np.float32)
        at = slot >= 0
        rows[at] = x[slot[at] // 3] * (w.reshape(-1)[slot[at]][:, None] if weighted else np.float32(1))
        wide = torch.full((tokens, hidden + start), 1e30, device="cuda")
        wide[:, start:] = torch.from_numpy(x).cuda()
        r, c = fp4.quantize(wide[:, start:], fmt, cols=True, gather=plan, weight=torch.from_numpy(w).cuda() if weighted else None)
        for op, v in ((r, rows), (c, np.ascontiguousarray(rows.T))):
            codes, byte, t = plain.quantize(v, fmt)
            assert np.array_equal(op.codes.cpu().numpy().reshape(v.shape[0], -1), plain.packed(codes))
            assert np.array_equal(op.scales.cpu().numpy().reshape(-1), plain.tiled(byte))
            assert op.tensor_scale.item() == t


def between(got, want, room, dtype):
    """got lies between the rounded ends of want -+ room."""
    low, high = ((want + s * room).astype(np.float32) for s in (-1, 1))
    if dtype == "bf16":
        low, high = plain.bf16(low), plain.bf16(high)
    got = got.detach().float().cpu().numpy()
    return bool((low <= got).all() and (got <= high).all())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("m,n,k", [(5, 33, 100), (200, 136, 300)])
def test_linear_of_32_bit_tensors(fp4, fmt, m, n, k):
    import torch

    rng = np.random.default_rng(m)
    x, w, g = (rng.standard_normal(s).astype(np.float32) for s in ((m, k), (n, k), (m, n)))
    tx, tw = (torch.from_numpy(v).cuda().requires_grad_() for v in (x, w))
    y = fp4.linear(tx, tw, fmt)
    dx, dw = torch.autograd.grad(y, (tx, tw), torch.from_numpy(g).cuda())

    def v(z):
        return plain.values(*plain.quantize(z, fmt), fmt)

    for got, a, b in ((y, v(x), v(w)), (dx, v(g), v(w.T)), (dw, v(g.T), v(x.T))):
        assert got.dtype == torch.float32 and between(got, a @ b.T, np.abs(a) @ np.abs(b).T * 2.0 ** -16, "fp32")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("tokens,top,n,k,m", [(1, 2, 8, 64, 40), (50, 3, 6, 300, 136), (400, 4, 4, 257, 264)])
def test_expert_layer_rounds_once(fp4, experts, fmt, dtype, tokens, top, n, k, m):
    """Against the formula on quantised values in 64 bits.  A product's row is a 32-bit sum (2^-16 of the sum of magnitudes), `top` of them
    are added with weights in 32 bits (top * 2^-24 more), a dot product over m columns adds m * 2^-24; each result is rounded once."""
    import torch

    rng = np.random.default_rng(tokens)
    ids = rng.integers(-1, n, (tokens, top)).astype(np.int32)
    starts, row, slot = plain.sort(ids, n, 128)
    rnd = plain.bf16 if dtype == "bf16" else (lambda z: z)
    x, w, g = (rnd(rng.standard_normal(s).astype(np.float32)) for s in ((tokens, k), (n, m, k), (tokens, m)))
    wt = rng.random((tokens, top)).astype(np.float32)
    d = torch.bfloat16 if dtype == "bf16" else torch.float32
    tx, tw, twt, tg = (torch.from_numpy(v).cuda() for v in (x, w, wt, g))
    tx, tw, twt = tx.to(d).requires_grad_(), tw.to(d).requires_grad_(), twt.requires_grad_()
    y = experts.linear(tx, tw, torch.from_numpy(ids).cuda(), twt, fmt)
    dx, dw, dwt = torch.autograd.grad(y, (tx, tw, twt), tg.to(d))
    assert y.dtype == dx.dtype == dw.dtype == d and dwt.dtype == torch.float32
    fp4.check()

    def v(z, amax=None):
        return plain.values(*plain.quantize(z, fmt, amax), fmt)

    at = slot >= 0
    rows, grows = np.zeros((len(slot), k), np.float32), np.zeros((len(slot), m), np.float32)
    rows[at] = x[slot[at] // top]
    grows[at] = g[slot[at] // top] * wt.reshape(-1)[slot[at]][:, None]
    amax = np.abs(w).max()
    qw = v(w.reshape(n * m, k)).reshape(n, m, k)
    qwt = np.stack([v(np.ascontiguousarray(w[e].T), amax) for e in range(n)])
    qx, qg, qxt, qgt = v(rows), v(grows), v(np.ascontiguousarray(rows.T)), v(np.ascontiguousarray(grows.T))
    ys, sy, dxs, sx = (np.zeros((len(slot), c)) for c in (m, m, k, k))
    for e in range(n):
        p = slice(starts[e], starts[e + 1])
        ys[p], sy[p] = qx[p] @ qw[e].T, np.abs(qx[p]) @ np.abs(qw[e]).T
        dxs[p], sx[p] = qg[p] @ qwt[e].T, np.abs(qg[p]) @ np.abs(qwt[e]).T
        assert between(dw[e], qgt[:, p] @ qxt[:, p].T, 2.0 ** -16 * np.abs(qgt[:, p]) @ np.abs(qxt[:, p]).T, dtype)

    def taken(z):
        return np.where((row >= 0)[..., None], z[np.maximum(row, 0)], 0.0)

    some = 2.0 ** -16 + top * 2.0 ** -24
    assert between(y, (taken(ys) * wt[..., None]).sum(1), some * (taken(sy) * wt[..., None]).sum(1), dtype)
    assert between(dwt, (taken(ys) * g[:, None, :]).sum(-1), (2.0 ** -16 + m * 2.0 ** -24) * (taken(sy) * np.abs(g)[:, None, :]).sum(-1), "fp32")
    assert between(dx, taken(dxs).sum(1), some * taken(sx).sum(1), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("fmt", FORMATS)
def test_more_tiles_than_are_walked(fp4, fmt, dtype):
    """Rows alone, 1122 tiles: beyond the number up to which resident CTAs walk them whatever the format."""
    x = drawn((4100, 4228), 3, dtype)
    codes, byte, t = plain.quantize(x.float().cpu().numpy(), fmt)
    r, _ = fp4.quantize(x, fmt)
    assert np.array_equal(r.codes.cpu().numpy().reshape(4100, -1), plain.packed(codes))
    assert np.array_equal(r.scales.cpu().numpy().reshape(-1), plain.tiled(byte)) and r.tensor_scale.item() == t

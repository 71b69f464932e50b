"""4-bit quantisation and products against a plain statement of them.

Quantisation is compared bit for bit: its definition fixes every rounding.  Products are compared with 64-bit sums over the
operands' values.  Tolerance, derived from the number formats: a product of two codes and two block scales is exact
in binary32; an instruction sums 64 of them after aligning them to its largest, keeping at least 23 bits, so it loses at
most 64 * 2^-23 of that product, and adds the running sum with the same loss; over all instructions that stays below
2^-16 * sum |a b|.  A BF16 result lies between the rounded ends of that interval.
"""
import numpy as np
import pytest

from tests import plain_fp4 as plain

pytestmark = pytest.mark.gpu
FORMATS = ["e4m3_16", "e8m0_32"]


@pytest.fixture(scope="module")
def fp4():
    from paper_2512_22804_b200 import fp4

    return fp4


def tensor(x, dtype="bf16"):
    import torch

    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda()
    return t.to(torch.bfloat16) if dtype == "bf16" else t


def draw(rows, cols, seed, kind="normal"):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols))
    if kind == "wide":                                   # many binades, exact zeros, whole blocks of zeros
        x = np.sign(x) * 2.0 ** rng.uniform(-40, 10, x.shape) * (rng.random(x.shape) > 0.1)
        x[:, : min(32, cols)] = 0
    if kind == "ties":                                   # values that meet rounding boundaries often
        x = rng.integers(-24, 25, x.shape) * 0.25
    if kind == "tiny":                                   # around the smallest scales
        x = x * 2.0 ** -120
    if kind == "huge":
        x = np.clip(x, -3, 3) * 2.0 ** 125
    return plain.bf16(x.astype(np.float32))


def check_operand(op, x, fmt, amax=None):
    codes, byte, t = plain.quantize(x, fmt, amax)
    got = op.codes.cpu().numpy().reshape(x.shape[0], -1)
    assert np.array_equal(got, plain.packed(codes))
    assert np.array_equal(op.scales.cpu().numpy().reshape(-1), plain.tiled(byte))
    assert op.tensor_scale.cpu().numpy()[0] == t
    return codes, byte, t


SHAPES = [(1, 1), (1, 16), (1, 4096), (2, 33), (3, 100), (128, 128), (129, 64), (127, 257), (300, 96), (40, 1000), (1000, 40), (5, 14336), (2500, 2056), (2305, 2184), (130, 38000)]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_codes_and_scales_both_directions(fp4, fmt, dtype, rows, cols):
    x = draw(rows, cols, rows * 7 + cols)
    if dtype == "fp32":
        x = (x * np.float32(1.0001)).astype(np.float32)
    r, c = fp4.quantize(tensor(x, dtype), fmt, cols=True)
    check_operand(r, x, fmt)
    check_operand(c, np.ascontiguousarray(x.T), fmt)
    only_r, none = fp4.quantize(tensor(x, dtype), fmt)
    assert none is None and bool((only_r.codes == r.codes).all()) and bool((only_r.scales == r.scales).all())
    none, only_c = fp4.quantize(tensor(x, dtype), fmt, rows=False, cols=True)
    assert none is None and bool((only_c.codes == c.codes).all()) and bool((only_c.scales == c.scales).all())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("kind", ["wide", "ties", "tiny", "huge"])
def test_hard_values(fp4, fmt, kind):
    x = draw(200, 320, 5, kind)
    r, c = fp4.quantize(tensor(x), fmt, cols=True)
    check_operand(r, x, fmt)
    check_operand(c, np.ascontiguousarray(x.T), fmt)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows,cols", [(64, 64), (300, 400)])     # the tensor maximum in one launch, and in two
def test_nan_and_infinities_stay_in_their_blocks(fp4, fmt, rows, cols):
    x = draw(rows, cols, 9)
    x[3, 5], x[10, 40], x[60, 63] = np.nan, np.inf, -np.inf
    r, c = fp4.quantize(tensor(x), fmt, cols=True)
    check_operand(r, x, fmt)
    check_operand(c, np.ascontiguousarray(x.T), fmt)
    v = fp4.dequantize(r).float().cpu().numpy()
    n = plain.BLOCK[fmt]
    want = np.zeros((rows, cols), bool)
    for i, j in ((3, 5), (10, 40), (60, 63)):
        want[i, j // n * n: j // n * n + n] = True
    assert np.array_equal(np.isnan(v), want)
    y = fp4.matmul(r, r).float().cpu().numpy()                       # a NaN scale reaches every product it enters
    bad = np.isin(np.arange(rows), (3, 10, 60))
    assert np.array_equal(np.isnan(y), bad[:, None] | bad[None, :])


@pytest.mark.parametrize("fmt", FORMATS)
def test_all_zero_and_given_maximum(fp4, fmt):
    import torch

    z = np.zeros((130, 70), np.float32)
    r, _ = fp4.quantize(tensor(z), fmt)
    check_operand(r, z, fmt)
    assert not fp4.dequantize(r).any()
    x = draw(130, 300, 3)
    amax = np.float32(1.5)                                           # smaller than the data: saturates
    r, c = fp4.quantize(tensor(x), fmt, cols=True, amax=torch.tensor([amax], device="cuda"))
    check_operand(r, x, fmt, amax)
    check_operand(c, np.ascontiguousarray(x.T), fmt, amax)


@pytest.mark.parametrize("fmt", FORMATS)
def test_strides_alignment_and_stacks(fp4, fmt):
    import torch

    x = draw(3 * 70, 200, 11).reshape(3, 70, 200)
    wide = torch.zeros(3, 80, 211, dtype=torch.bfloat16, device="cuda")      # odd pitch, odd start
    wide[:, 4:74, 3:203] = tensor(x.reshape(-1, 200)).reshape(3, 70, 200)
    odd = wide[:, 4:74, 3:203]
    flat = x.reshape(-1, 200)
    amax = np.abs(flat).max()
    for t in (odd, odd.contiguous()):
        r, c = fp4.quantize(t, fmt, cols=True)
        assert (r.batch, r.rows, r.cols, c.rows, c.cols) == (3, 70, 200, 200, 70)
        for b in range(3):
            codes, byte, _ = plain.quantize(x[b], fmt, amax)
            assert np.array_equal(r.codes[b].cpu().numpy(), plain.packed(codes))
            assert np.array_equal(r.scales.reshape(3, -1)[b].cpu().numpy(), plain.tiled(byte))
            codes, byte, _ = plain.quantize(x[b].T, fmt, amax)
            assert np.array_equal(c.codes[b].cpu().numpy(), plain.packed(codes))
            assert np.array_equal(c.scales.reshape(3, -1)[b].cpu().numpy(), plain.tiled(byte))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_that_start_anywhere(fp4, fmt, dtype):
    """Every offset from 16 bytes and odd pitches, from one tile to a tensor whose maximum is taken by a kernel of its own."""
    import torch

    for rows, cols in ((3, 20), (130, 150), (200, 301)):
        x = draw(rows, cols, rows, "wide")
        for start in range(9):
            wide = torch.full((rows, cols + start + start % 3), 2.0 ** 60, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
            wide[:, start : start + cols] = tensor(x, dtype)
            r, c = fp4.quantize(wide[:, start : start + cols], fmt, cols=True)
            check_operand(r, x, fmt)
            check_operand(c, x.T, fmt)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 4096), (130, 100), (257, 1000)])
def test_values_of_codes(fp4, fmt, rows, cols):
    import torch

    x = draw(rows, cols, 21)
    r, _ = fp4.quantize(tensor(x), fmt)
    want = plain.values(*plain.quantize(x, fmt), fmt)
    assert np.array_equal(fp4.dequantize(r, torch.float32).cpu().numpy(), want.astype(np.float32))
    assert np.array_equal(fp4.dequantize(r).float().cpu().numpy(), plain.bf16(want.astype(np.float32)))
    step = np.abs(want).max() / 3 + 1e-30                            # no value is further off than half the widest gap of its block
    assert np.abs(want - x).max() <= step


def check_product(y, a, b, out):
    y = y.float().cpu().numpy().astype(np.float64)
    want, room = a @ b.T, np.abs(a) @ np.abs(b).T * 2.0 ** -16
    assert y.shape == want.shape
    low, high = want - room, want + room
    if out == "bf16":
        low, high = plain.bf16(low.astype(np.float32)), plain.bf16(high.astype(np.float32))
    assert (low <= y).all() and (y <= high).all(), np.abs((y - want) / (room + 1e-300)).max()


def operands(fp4, m, n, k, fmt, seed=0):
    xa, xb = draw(m, k, 100 + seed), draw(n, k, 200 + seed) * np.float32(0.02)
    xb = plain.bf16(xb)
    a, _ = fp4.quantize(tensor(xa), fmt)
    b, _ = fp4.quantize(tensor(xb), fmt)
    return a, b, plain.values(*plain.quantize(xa, fmt), fmt), plain.values(*plain.quantize(xb, fmt), fmt)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("out", ["bf16", "fp32"])
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 128, 64), (1, 1000, 4096), (2, 136, 31), (16, 130, 257), (17, 64, 512), (33, 300, 100), (64, 128, 2048),
                                   (65, 520, 1000), (128, 257, 48), (100, 4096, 300)])
def test_product_of_few_rows(fp4, fmt, out, m, n, k):
    import torch

    a, b, va, vb = operands(fp4, m, n, k, fmt)
    check_product(fp4.matmul(a, b, torch.bfloat16 if out == "bf16" else torch.float32), va, vb, out)
    fp4.check()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("out", ["bf16", "fp32"])
@pytest.mark.parametrize("m,n,k", [(129, 1, 16), (256, 256, 256), (256, 256, 64), (200, 1000, 300), (513, 250, 1000), (1000, 264, 31), (300, 700, 4096),
                                   (2304, 2560, 512)])
def test_product_of_many_rows(fp4, fmt, out, m, n, k):
    import torch

    a, b, va, vb = operands(fp4, m, n, k, fmt)
    check_product(fp4.matmul(a, b, torch.bfloat16 if out == "bf16" else torch.float32), va, vb, out)
    fp4.check()


def grouped(counts, hidden, fmt, fp4, seed):
    """Rows of experts with these counts, aligned to 128, and their plan."""
    import torch

    from paper_2512_22804_b200 import experts

    ids = np.repeat(np.arange(len(counts)), counts).astype(np.int32)
    np.random.default_rng(seed).shuffle(ids)
    x = draw(len(ids), hidden, seed)
    plan = experts.sort(torch.from_numpy(ids.reshape(-1, 1)).cuda(), len(counts), 128)
    starts, row, slot = plain.sort(ids, len(counts), 128)
    rows = np.zeros((len(slot), hidden), np.float32)
    rows[slot >= 0] = x[slot[slot >= 0]]
    return plan, starts, rows, x


COUNTS = [[1], [128], [0, 5, 0], [130, 0, 1, 256, 300], [7] * 40, [500, 129, 700]]


@pytest.mark.parametrize("out", ["bf16", "fp32"])
@pytest.mark.parametrize("fmt", FORMATS)
def test_result_rows_that_start_half_a_sector_off(fp4, fmt, out):
    """Rows of 16 bytes modulo 32: the same values as in rows that start on 32 bytes."""
    import torch

    d = torch.bfloat16 if out == "bf16" else torch.float32
    n = 520 if out == "bf16" else 516
    a = fp4.quantize(tensor(draw(300, 200, 1)), fmt, amax=torch.full((1,), 5.0, device="cuda"))[0]
    w = tensor(draw(n + 24, 200, 2))
    amax = torch.full((1,), 5.0, device="cuda")
    got = fp4.matmul(a, fp4.quantize(w[:n], fmt, amax=amax)[0], d)
    want = fp4.matmul(a, fp4.quantize(w[: n // 16 * 16 + 16], fmt, amax=amax)[0], d)
    assert got.stride(0) * got.element_size() % 32 == 16 and want.stride(0) * want.element_size() % 32 == 0
    assert torch.equal(got, want[:, :n])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("counts", COUNTS, ids=str)
@pytest.mark.parametrize("n,k", [(1, 64), (136, 300), (520, 257)])
def test_products_by_groups_of_rows(fp4, fmt, counts, n, k):
    plan, starts, rows, x = grouped(counts, k, fmt, fp4, 3)
    w = plain.bf16(draw(len(counts) * n, k, 4) * np.float32(0.1))
    a, _ = fp4.quantize(tensor(x), fmt, gather=plan)
    b, _ = fp4.quantize(tensor(w).reshape(len(counts), n, k), fmt)
    va, vb = plain.values(*plain.quantize(rows, fmt), fmt), plain.values(*plain.quantize(w, fmt), fmt)
    y = fp4.matmul_rows(a, b, plan)
    for e, count in enumerate(counts):                               # an expert's rows; those that alignment adds are not written
        at = slice(starts[e], starts[e] + count)
        check_product(y[at], va[at], vb[e * n:(e + 1) * n], "bf16")
    fp4.check()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("counts", COUNTS, ids=str)
@pytest.mark.parametrize("m,n", [(1, 8), (136, 300), (300, 520)])
def test_products_by_groups_of_the_reduction(fp4, fmt, counts, m, n):
    import torch

    plan, starts, xr, x = grouped(counts, n, fmt, fp4, 5)
    _, _, gr, g = grouped(counts, m, fmt, fp4, 5)
    _, bt = fp4.quantize(tensor(x), fmt, rows=False, cols=True, gather=plan)
    _, at = fp4.quantize(tensor(g), fmt, rows=False, cols=True, gather=plan)
    va, vb = plain.values(*plain.quantize(gr.T, fmt), fmt), plain.values(*plain.quantize(xr.T, fmt), fmt)
    y = fp4.matmul_reduce(at, bt, plan, torch.float32)
    assert y.shape == (len(counts), m, n)
    for e in range(len(counts)):
        part = slice(starts[e], starts[e + 1])
        check_product(y[e], va[:, part], vb[:, part], "fp32")
    fp4.check()


def test_products_on_another_stream_and_twice_the_same(fp4):
    import torch

    a, b, va, vb = operands(fp4, 300, 520, 1024, "e4m3_16")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        y = fp4.matmul(a, b)
        z = fp4.matmul(a, b)
    s.synchronize()
    check_product(y, va, vb, "bf16")
    assert torch.equal(y, z)


def test_empty_operands(fp4):
    import torch

    x = torch.zeros(0, 64, device="cuda", dtype=torch.bfloat16)
    w = torch.ones(40, 64, device="cuda", dtype=torch.bfloat16)
    a, at = fp4.quantize(x, "e8m0_32", cols=True)
    b, _ = fp4.quantize(w, "e8m0_32")
    assert fp4.matmul(a, b).shape == (0, 40)
    for rows in (3, 300):                                            # a sum over nothing is zero
        e, _ = fp4.quantize(torch.zeros(rows, 0, device="cuda", dtype=torch.bfloat16), "e8m0_32")
        f, _ = fp4.quantize(torch.zeros(20, 0, device="cuda", dtype=torch.bfloat16), "e8m0_32")
        assert torch.equal(fp4.matmul(e, f), torch.zeros(rows, 20, device="cuda", dtype=torch.bfloat16))
    assert fp4.dequantize(at).shape == (64, 0)


def test_a_captured_step_follows_its_inputs(fp4):
    """Quantisation, product and layer inside a CUDA graph: replayed with other values in the same tensors."""
    import torch

    x, w = tensor(draw(40, 512, 1)), tensor(draw(264, 512, 2))
    b = fp4.quantize(w, "e4m3_16")[0]

    def step():
        return fp4.matmul(fp4.quantize(x, "e4m3_16")[0], b), fp4.linear(x, w, "e8m0_32")

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in (5, 6):
        x.copy_(tensor(draw(40, 512, seed)))
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(out, step()):
            assert torch.equal(got, want)


def test_gradients_of_no_tokens(fp4):
    import torch

    x = torch.zeros(0, 96, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    w = torch.ones(40, 96, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    for fmt in FORMATS:
        y = fp4.linear(x, w, fmt)
        dx, dw = torch.autograd.grad(y, (x, w), torch.zeros(0, 40, device="cuda", dtype=torch.bfloat16))
        assert y.shape == (0, 40) and dx.shape == (0, 96) and not dw.any() and dw.shape == w.shape


@pytest.mark.parametrize("fmt", FORMATS)
def test_linear_and_its_gradient(fp4, fmt):
    """y, dx and dw against the three products of values quantised along their reduction axes."""
    import torch

    m, n, k = 200, 136, 300
    x, w, g = draw(m, k, 1), plain.bf16(draw(n, k, 2) * np.float32(0.05)), draw(m, n, 3)
    tx, tw = tensor(x).requires_grad_(), tensor(w).requires_grad_()
    y = fp4.linear(tx, tw, fmt)
    dx, dw = torch.autograd.grad(y, (tx, tw), tensor(g))

    def v(z):
        return plain.values(*plain.quantize(z, fmt), fmt)

    check_product(y.detach(), v(x), v(w), "bf16")
    check_product(dx, v(g), v(w.T), "bf16")
    check_product(dw, v(g.T), v(x.T), "bf16")
    y3 = fp4.linear(tensor(x).reshape(2, 100, k), tensor(w), fmt)
    assert y3.shape == (2, 100, n) and torch.equal(y3.reshape(m, n), y)
    only = fp4.linear(tx, tw.detach(), fmt)                          # a frozen weight
    assert torch.equal(torch.autograd.grad(only, tx, tensor(g))[0], dx)


def test_gradient_against_differences(fp4):
    """Inputs that 4 bits hold exactly, moved by steps that they hold exactly too: the product is linear in them and every
    sum is a small whole number, so the difference quotient equals the gradient."""
    import torch

    rng = np.random.default_rng(8)
    x, w, g = (rng.choice([-4., -2., -1., 1., 2., 4.], s) for s in ((4, 32), (32, 32), (4, 32)))
    for z in (x, w, g):
        z[:, 0] = 4                                                  # keeps every block's scale (along rows and columns) at one
        z[0, :] = 4
    tx, tw, tg = (tensor(z, "fp32") for z in (x, w, g))
    tx.requires_grad_()
    tw.requires_grad_()
    dx, dw = torch.autograd.grad(fp4.linear(tx, tw, "e8m0_32"), (tx, tw), tg)

    def loss(x, w):
        return float((fp4.linear(tensor(x, "fp32"), tensor(w, "fp32"), "e8m0_32").double() * tg.double()).sum())

    for grad, z in ((dx, x), (dw, w)):
        for i, j in ((1, 1), (2, 17), (3, 31)):
            up, down = z.copy(), z.copy()
            up[i, j], down[i, j] = 2, 1
            d = loss(up, w) - loss(down, w) if z is x else loss(x, up) - loss(x, down)
            assert d == float(grad[i, j])


@pytest.mark.parametrize("kind", ["few rows", "many rows", "groups of rows", "groups of the reduction"])
def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_clean(fp4, kind):
    """A host-set test hook leaves out one tile's copy and shortens the wait limit to a millisecond: the call returns, the
    status word says so, and the same call without the hook is right."""
    import ctypes

    import torch

    from paper_2512_22804_b200 import binding as mb

    hook = mb.load().mor_test_skip_tile_load
    hook.argtypes, hook.restype = [ctypes.c_uint32, ctypes.c_longlong], None
    if kind in ("few rows", "many rows"):
        a, b, va, vb = operands(fp4, 20 if kind == "few rows" else 600, 600, 1500, "e4m3_16")

        def call():
            return fp4.matmul(a, b, torch.float32)
    else:
        counts = [130, 0, 300]
        plan, starts, rows, x = grouped(counts, 300, "e4m3_16", fp4, 3)
        if kind == "groups of rows":
            w = plain.bf16(draw(3 * 136, 300, 4))
            a, b = fp4.quantize(tensor(x), "e4m3_16", gather=plan)[0], fp4.quantize(tensor(w).reshape(3, 136, 300), "e4m3_16")[0]
            va, vb = plain.values(*plain.quantize(rows, "e4m3_16"), "e4m3_16")[:130], plain.values(*plain.quantize(w, "e4m3_16"), "e4m3_16")[:136]

            def call():
                return fp4.matmul_rows(a, b, plan, torch.float32)[:130]
        else:
            a = b = fp4.quantize(tensor(x), "e4m3_16", rows=False, cols=True, gather=plan)[1]
            va = vb = plain.values(*plain.quantize(rows.T, "e4m3_16"), "e4m3_16")[:, :256]

            def call():
                return fp4.matmul_reduce(a, b, plan, torch.float32)[0]
    torch.cuda.synchronize()
    hook(0, 2_000_000)
    try:
        call()
        torch.cuda.synchronize()
    finally:
        hook(0xFFFFFFFF, 0)
    with pytest.raises(mb.MorError) as e:
        fp4.check()
    assert e.value.status == mb.MOR_ERR_TIMEOUT
    check_product(call(), va, vb, "fp32")
    fp4.check()

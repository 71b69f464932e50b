"""Sorting by expert, the row movers and the 4-bit expert layer against plain statements of them.

Sorting and plain copies are compared exactly.  A weighted sum of `top` rows is taken in binary32 in slot order: |error| <= top *
2^-24 * sum |w y|; a dot product over `hidden` values is summed in binary32 in some order: |error| <= hidden * 2^-24 * sum |dy y|.
Each is then rounded once to the result's type, so the result lies between the rounded ends of that interval.
"""
import numpy as np
import pytest

from tests import plain_fp4 as plain

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def experts():
    from paper_2512_22804_b200 import experts

    return experts


def cuda(x, dtype=None):
    import torch

    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t if dtype is None else t.to(dtype)


def draw_ids(tokens, top, n, seed, masked=0.1):
    rng = np.random.default_rng(seed)
    p = rng.random(n) ** 3 + 1e-3
    ids = rng.choice(n, (tokens, top), p=p / p.sum()).astype(np.int32)
    ids[rng.random((tokens, top)) < masked] = -1
    return ids


CASES = [(1, 1, 1), (1, 8, 128), (3, 2, 5), (100, 4, 64), (4096, 1, 7), (1025, 4, 1024), (2048, 2, 33), (5000, 3, 16), (40000, 4, 64), (30000, 8, 1024)]


@pytest.mark.parametrize("align", [1, 128])
@pytest.mark.parametrize("tokens,top,n", CASES)
def test_sort(experts, tokens, top, n, align):
    ids = draw_ids(tokens, top, n, tokens + n)
    plan = experts.sort(cuda(ids), n, align)
    starts, row, slot = plain.sort(ids, n, align)
    assert np.array_equal(plan.starts.cpu().numpy(), starts)
    assert np.array_equal(plan.row.cpu().numpy(), row)
    assert np.array_equal(plan.slot.cpu().numpy(), slot)


@pytest.mark.parametrize("fill", [-1, 5, -2**31, 2**31 - 1, 0, 4])
def test_sort_of_ids_that_name_no_expert_and_of_one_expert(experts, fill):
    for tokens in (7, 3000):
        ids = np.full((tokens, 2), fill, np.int32)
        plan = experts.sort(cuda(ids), 5, 128)
        starts, row, slot = plain.sort(ids, 5, 128)
        for got, want in ((plan.starts, starts), (plan.row, row), (plan.slot, slot)):
            assert np.array_equal(got.cpu().numpy(), want)


def test_sort_of_nothing(experts):
    import torch

    plan = experts.sort(torch.zeros(0, 4, dtype=torch.int32, device="cuda"), 6, 128)
    assert plan.starts.tolist() == [0] * 7 and plan.slot.numel() == 0
    x = torch.zeros(0, 64, device="cuda", dtype=torch.bfloat16)
    assert experts.gather(x, plan).shape == (0, 64) and experts.combine(x, plan).shape == (0, 64)


def matrices(experts, tokens, top, n, hidden, align, dtype, seed):
    import torch

    rng = np.random.default_rng(seed)
    ids = draw_ids(tokens, top, n, seed)
    plan = experts.sort(cuda(ids), n, align)
    _, row, slot = plain.sort(ids, n, align)
    d = torch.bfloat16 if dtype == "bf16" else torch.float32

    def matrix(r):
        x = rng.standard_normal((r, hidden)).astype(np.float32)
        x = plain.bf16(x) if dtype == "bf16" else x
        return x, cuda(x, d)

    return plan, row, slot, matrix


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("weights", [None, "bf16", "fp32"])
@pytest.mark.parametrize("tokens,top,n,hidden,align", [(1, 8, 16, 4096, 1), (37, 2, 5, 1, 1), (100, 3, 9, 33, 128), (300, 5, 64, 520, 1), (64, 9, 4, 24, 128),
                                                       (130, 1, 3, 2056, 128)])
def test_gather_combine_and_gradient(experts, tokens, top, n, hidden, align, weights, dtype):
    import torch

    plan, row, slot, matrix = matrices(experts, tokens, top, n, hidden, align, dtype, tokens + top)
    w = np.random.default_rng(1).random((tokens, top)).astype(np.float32)
    w = plain.bf16(w) if weights == "bf16" else w
    tw = None if weights is None else cuda(w, torch.bfloat16 if weights == "bf16" else torch.float32)
    one = w if weights is not None else np.ones_like(w)
    x, tx = matrix(tokens)
    ys, tys = matrix(len(slot))
    dy, tdy = matrix(tokens)
    def rnd(v, to=dtype):
        return plain.bf16(v.astype(np.float32)) if to == "bf16" else v.astype(np.float32)

    def within(got, want, room, to):
        got = got.float().cpu().numpy()
        return (rnd(want - room, to) <= got).all() and (got <= rnd(want + room, to)).all()

    def spread(v):
        out = np.zeros((len(slot), hidden), np.float32)
        at = slot >= 0
        out[at] = rnd(v[slot[at] // top] * one.reshape(-1)[slot[at]][:, None])
        return out

    assert np.array_equal(experts.gather(tx, plan, tw).float().cpu().numpy(), spread(x))
    taken = np.where((row >= 0)[..., None], ys.astype(np.float64)[np.maximum(row, 0)], 0.0)
    want = (taken * one[..., None]).sum(1)
    assert within(experts.combine(tys, plan, tw), want, top * 2.0 ** -24 * (np.abs(taken) * one[..., None]).sum(1), dtype)
    if weights is None:
        return
    dys, dw = experts.combine_grad(tdy, tys, plan, tw)
    assert np.array_equal(dys.float().cpu().numpy(), spread(dy))
    terms = taken * dy.astype(np.float64)[:, None, :]
    want = terms.sum(-1)
    assert within(dw, want, hidden * 2.0 ** -24 * np.abs(terms).sum(-1), weights)
    none, again = experts.combine_grad(tdy, tys, plan, tw, rows=False)
    assert none is None and torch.equal(again, dw)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hidden", [30, 31, 264, 1001])
def test_rows_that_start_anywhere(experts, hidden, dtype):
    """Every offset from 16 bytes, odd pitches and widths: copies and weighted sums as from aligned rows, bit for bit."""
    import torch

    plan, row, slot, matrix = matrices(experts, 50, 5, 7, hidden, 1, dtype, hidden)
    (_, x), (ys64, ys), (dy64, dy) = matrix(50), matrix(len(slot)), matrix(50)
    w = torch.rand(50, 5, generator=torch.Generator().manual_seed(2)).cuda()

    def moved(t, start, pitch):
        wide = torch.full((t.shape[0], pitch), float("nan"), dtype=t.dtype, device="cuda")
        wide[:, start : start + hidden] = t
        return wide[:, start : start + hidden]

    def even(t):                                       # whole pieces: the width and the pitch are multiples of 32 bytes
        return torch.nn.functional.pad(t, (0, -hidden % 16))

    spread, back = experts.gather(even(x), plan, w)[:, :hidden], experts.combine(even(ys), plan, w)[:, :hidden]
    gys = experts.combine_grad(even(dy), even(ys), plan, w)[0][:, :hidden]
    taken = np.where((row >= 0)[..., None], ys64.astype(np.float64)[np.maximum(row, 0)], 0.0)
    terms = taken * dy64.astype(np.float64)[:, None, :]
    room = hidden * 2.0 ** -24 * np.abs(terms).sum(-1)
    for start in range(9):
        pitch = hidden + start + start % 4
        assert torch.equal(experts.gather(moved(x, start, pitch), plan, w), spread)
        assert torch.equal(experts.combine(moved(ys, start, pitch), plan, w), back)
        got, dw = experts.combine_grad(moved(dy, start, pitch + 1), moved(ys, start, pitch), plan, w)
        assert torch.equal(got, gys)
        dw = dw.cpu().numpy()
        assert ((terms.sum(-1) - room).astype(np.float32) <= dw).all() and (dw <= (terms.sum(-1) + room).astype(np.float32)).all()


@pytest.mark.parametrize("tokens,top,n,hidden", [(37, 2, 5, 1), (100, 3, 9, 33), (300, 5, 64, 520)])
def test_rows_of_32_bits_beside_tokens_of_16(experts, tokens, top, n, hidden):
    import torch

    plan, row, slot, matrix = matrices(experts, tokens, top, n, hidden, 128, "bf16", tokens)
    dy, tdy = matrix(tokens)
    rng = np.random.default_rng(4)
    ys = rng.standard_normal((len(slot), hidden)).astype(np.float32)
    w = rng.random((tokens, top)).astype(np.float32)
    tys, tw = cuda(ys), cuda(w)
    taken = np.where((row >= 0)[..., None], ys.astype(np.float64)[np.maximum(row, 0)], 0.0)
    want, room = (taken * w[..., None]).sum(1), top * 2.0 ** -24 * (np.abs(taken) * w[..., None]).sum(1)
    y = experts.combine(tys, plan, tw, torch.bfloat16).float().cpu().numpy()
    assert (plain.bf16((want - room).astype(np.float32)) <= y).all() and (y <= plain.bf16((want + room).astype(np.float32))).all()
    dys, dw = experts.combine_grad(tdy, tys, plan, tw)
    terms = taken * dy.astype(np.float64)[:, None, :]
    assert (np.abs(dw.double().cpu().numpy() - terms.sum(-1)) <= hidden * 2.0 ** -24 * np.abs(terms).sum(-1)).all()
    assert dys.dtype == torch.bfloat16 and torch.equal(dys, experts.gather(tdy, plan, tw))


@pytest.mark.parametrize("hidden", [36, 43, 267, 1030])
def test_rows_of_32_bits_beside_tokens_of_16_that_start_anywhere(experts, hidden):
    import torch

    plan, row, slot, matrix = matrices(experts, 40, 3, 6, hidden, 1, "bf16", hidden)
    dy, tdy = matrix(40)
    rng = np.random.default_rng(5)
    ys = rng.standard_normal((len(slot), hidden)).astype(np.float32)
    w = rng.random((40, 3)).astype(np.float32)
    tw = cuda(w)
    taken = np.where((row >= 0)[..., None], ys.astype(np.float64)[np.maximum(row, 0)], 0.0)
    want, room = (taken * w[..., None]).sum(1), 3 * 2.0 ** -24 * (np.abs(taken) * w[..., None]).sum(1)
    terms = taken * dy.astype(np.float64)[:, None, :]
    for start in range(9):
        wide = torch.full((40, hidden + start + 1), float("nan"), dtype=torch.bfloat16, device="cuda")
        wide[:, start : start + hidden] = tdy
        rows = torch.full((len(slot), hidden + start % 5), float("nan"), device="cuda")
        rows[:, start % 5 :] = cuda(ys)
        y = experts.combine(rows[:, start % 5 :], plan, tw, torch.bfloat16).float().cpu().numpy()
        assert (plain.bf16((want - room).astype(np.float32)) <= y).all() and (y <= plain.bf16((want + room).astype(np.float32))).all()
        dys, dw = experts.combine_grad(wide[:, start : start + hidden], rows[:, start % 5 :], plan, tw)
        assert (np.abs(dw.double().cpu().numpy() - terms.sum(-1)) <= hidden * 2.0 ** -24 * np.abs(terms).sum(-1)).all()
        assert torch.equal(dys, experts.gather(tdy, plan, tw))


@pytest.mark.parametrize("hidden", [8, 40, 264])
def test_rows_of_32_bits_beside_tokens_of_16_from_every_start(experts, hidden):
    """Widths of whole pieces: FP32 rows that start 4, 8, .. 32 bytes past a multiple of 32, with pitches that keep or shift the start."""
    import torch

    plan, row, slot, matrix = matrices(experts, 40, 3, 6, hidden, 1, "bf16", hidden)
    dy, tdy = matrix(40)
    rng = np.random.default_rng(6)
    ys = rng.standard_normal((len(slot), hidden)).astype(np.float32)
    w = rng.random((40, 3)).astype(np.float32)
    tw = cuda(w)
    taken = np.where((row >= 0)[..., None], ys.astype(np.float64)[np.maximum(row, 0)], 0.0)
    want, room = (taken * w[..., None]).sum(1), 3 * 2.0 ** -24 * (np.abs(taken) * w[..., None]).sum(1)
    terms = taken * dy.astype(np.float64)[:, None, :]
    for start in range(9):
        for more in (8, 12, 9):                        # the pitch: a multiple of 32 bytes, of 16, of 4
            rows = torch.full((len(slot), hidden + more), float("nan"), device="cuda")
            rows[:, start : start + hidden] = cuda(ys)
            rows = rows[:, start : start + hidden]
            y = experts.combine(rows, plan, tw, torch.bfloat16).float().cpu().numpy()
            assert (plain.bf16((want - room).astype(np.float32)) <= y).all() and (y <= plain.bf16((want + room).astype(np.float32))).all()
            dys, dw = experts.combine_grad(tdy, rows, plan, tw)
            assert (np.abs(dw.double().cpu().numpy() - terms.sum(-1)) <= hidden * 2.0 ** -24 * np.abs(terms).sum(-1)).all()
            assert torch.equal(dys, experts.gather(tdy, plan, tw))


def test_nan_of_an_empty_row_goes_nowhere_and_strides(experts):
    import torch

    plan, row, slot, matrix = matrices(experts, 50, 2, 4, 96, 128, "bf16", 3)
    ys, tys = matrix(len(slot))
    tys[torch.from_numpy(slot < 0).cuda()] = float("nan")
    y = experts.combine(tys, plan)
    assert torch.isfinite(y).all()
    masked = (row < 0).all(1)
    assert not y[torch.from_numpy(masked).cuda()].any()
    wide = torch.zeros(len(slot), 131, dtype=torch.bfloat16, device="cuda")   # odd pitch and start: one element at a time
    wide[:, 1:97] = tys
    assert torch.equal(experts.combine(wide[:, 1:97], plan), y)
    x, tx = matrix(50)
    wide = torch.zeros(50, 104, dtype=torch.bfloat16, device="cuda")          # 16-byte pitch
    wide[:, 8:] = tx
    assert torch.equal(experts.gather(wide[:, 8:], plan), experts.gather(tx, plan))


@pytest.mark.parametrize("fmt", ["e4m3_16", "e8m0_32"])
@pytest.mark.parametrize("weighted", [False, True])
def test_quantised_gather_equals_gather_then_quantise(experts, fmt, weighted):
    """The rows that quantisation gathers on the way, against the plain quantiser on the gathered 32-bit rows."""
    import torch

    from paper_2512_22804_b200 import fp4

    for tokens, hidden in ((40, 96), (300, 333), (1100, 1544)):
        plan, row, slot, matrix = matrices(experts, tokens, 3, 6, hidden, 128, "bf16", tokens)
        x, tx = matrix(tokens)
        w = np.random.default_rng(2).random((tokens, 3)).astype(np.float32)
        rows = np.zeros((len(slot), hidden), np.float32)
        at = slot >= 0
        rows[at] = x[slot[at] // 3] * (w.reshape(-1)[slot[at]][:, None] if weighted else np.float32(1))
        r, c = fp4.quantize(tx, fmt, cols=True, gather=plan, weight=cuda(w) if weighted else None)
        for op, v in ((r, rows), (c, np.ascontiguousarray(rows.T))):
            codes, byte, t = plain.quantize(v, fmt)
            assert np.array_equal(op.codes.cpu().numpy().reshape(v.shape[0], -1), plain.packed(codes))
            assert np.array_equal(op.scales.cpu().numpy().reshape(-1), plain.tiled(byte))
            assert op.tensor_scale.item() == t


@pytest.mark.parametrize("fmt", ["e4m3_16", "e8m0_32"])
@pytest.mark.parametrize("tokens", [0, 1, 300])
def test_expert_layer_where_no_token_has_an_expert(experts, fmt, tokens):
    import torch

    x = torch.ones(tokens, 64, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    w = torch.ones(4, 40, 64, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    weight = torch.ones(tokens, 2, device="cuda", requires_grad=True)
    ids = torch.full((tokens, 2), -1, device="cuda", dtype=torch.int32)
    y = experts.linear(x, w, ids, weight, fmt)
    grads = torch.autograd.grad(y, (x, w, weight), torch.ones_like(y))
    assert y.shape == (tokens, 40) and not y.any()
    for g, t in zip(grads, (x, w, weight)):
        assert g.shape == t.shape and not g.any()


@pytest.mark.parametrize("fmt", ["e4m3_16", "e8m0_32"])
@pytest.mark.parametrize("tokens,top,n,k,m", [(1, 2, 8, 64, 40), (50, 3, 6, 300, 136), (400, 2, 4, 257, 264)])
def test_expert_layer_and_its_gradient(experts, fmt, tokens, top, n, k, m):
    """Against the formula on quantised values, in 64 bits.  The rows of the gradient's product are rounded to BF16 (at
    most 2^-8) before they are added, every result once: 2^-7 of the sum of magnitudes covers both (the sums' own 2^-16 beside what
    the products of both roundings leave)."""
    import torch

    from paper_2512_22804_b200 import fp4

    rng = np.random.default_rng(tokens)
    ids = draw_ids(tokens, top, n, tokens + 1)
    _, row, slot = plain.sort(ids, n, 128)
    starts = plain.sort(ids, n, 128)[0]
    x, w = plain.bf16(rng.standard_normal((tokens, k)).astype(np.float32)), plain.bf16(rng.standard_normal((n, m, k)).astype(np.float32) * np.float32(0.1))
    g = plain.bf16(rng.standard_normal((tokens, m)).astype(np.float32))
    wt = plain.bf16(rng.random((tokens, top)).astype(np.float32))
    tx, tw, twt = (cuda(v, torch.bfloat16).requires_grad_() for v in (x, w, wt))
    y = experts.linear(tx, tw, cuda(ids), twt, fmt)
    dx, dw, dwt = torch.autograd.grad(y, (tx, tw, twt), cuda(g, torch.bfloat16))
    fp4.check()

    def v(z):
        return plain.values(*plain.quantize(z, fmt), fmt)

    def near(got, want, size):
        assert (np.abs(got.detach().double().cpu().numpy() - want) <= 2.0 ** -7 * size + 1e-30).all()

    at = slot >= 0
    rows, grows = np.zeros((len(slot), k), np.float32), np.zeros((len(slot), m), np.float32)
    rows[at] = x[slot[at] // top]
    grows[at] = g[slot[at] // top] * wt.reshape(-1)[slot[at]][:, None]
    qw = v(w.reshape(n * m, k)).reshape(n, m, k)
    # blocks of the transposes run inside one expert's matrix; the tensor maximum is that of the whole stack
    amax = np.abs(w).max()
    qwt = np.stack([plain.values(*plain.quantize(np.ascontiguousarray(w[e].T), fmt, amax), fmt) for e in range(n)])
    qx, qg, qxt, qgt = v(rows), v(grows), v(np.ascontiguousarray(rows.T)), v(np.ascontiguousarray(grows.T))
    ys, sy = np.zeros((len(slot), m)), np.zeros((len(slot), m))
    dxs, sx = np.zeros((len(slot), k)), np.zeros((len(slot), k))
    for e in range(n):
        p = slice(starts[e], starts[e + 1])
        ys[p], sy[p] = qx[p] @ qw[e].T, np.abs(qx[p]) @ np.abs(qw[e]).T
        dxs[p], sx[p] = qg[p] @ qwt[e].T, np.abs(qg[p]) @ np.abs(qwt[e]).T
        near(dw[e], qgt[:, p] @ qxt[:, p].T, np.abs(qgt[:, p]) @ np.abs(qxt[:, p]).T)

    def taken(z):
        return np.where((row >= 0)[..., None], z[np.maximum(row, 0)], 0.0)

    near(y, (taken(ys) * wt[..., None]).sum(1), (taken(sy) * wt[..., None]).sum(1))
    near(dx, taken(dxs).sum(1), taken(sx).sum(1))
    near(dwt, (taken(ys) * g[:, None, :]).sum(-1), (taken(sy) * np.abs(g)[:, None, :]).sum(-1))
    stored, _ = fp4.quantize(tw.detach(), fmt)                       # serving: the weight quantised once
    assert torch.equal(experts.linear(tx.detach(), stored, cuda(ids), twt.detach()), y)

"""Low-rank adapters against the formulas in 64 bits.

u = 2^-24.  The tensor instructions add products of BF16 (exact in 32 bits) without a promise to round to nearest, so an inner product of n terms is taken to be off by
n 2 u of the sum of its terms' magnitudes.  h enters the second product as two BF16, which leaves 2^-17 of it.  So with H = sum |x a| the
result is off by s sum_r |b| ((n_in + 8) 2 u H + 2^-17 |h|) + (rank + 2) 4 u s sum_r |h b| before its rounding, and so are the gradients with their sums.
"""
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def adapters():
    from paper_2512_22804_b200 import adapters

    return adapters


def half_step(v, dtype):
    import torch

    return v.abs() * torch.finfo(dtype).eps / 2 + 2.0 ** -134


def draw(tokens, n_in, n_out, rank, n, seed=0, base="bf16"):
    import torch

    g = torch.Generator(device="cuda").manual_seed(seed + tokens * 7 + n_in * 3 + n_out + rank)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    bf16 = torch.bfloat16
    x = r(tokens, n_in).to(bf16)
    a, b = (r(n, rank, n_in) * n_in ** -0.5).to(bf16), (r(n, n_out, rank) * 0.3).to(bf16)
    ids = torch.randint(-1, n + 1, (tokens,), generator=g, device="cuda").to(torch.int32)          # some name no adapter
    if tokens > 4:
        ids[1], ids[2] = 2 ** 31 - 1, -2 ** 31
    return x, r(tokens, n_out).to(bf16 if base == "bf16" else torch.float32), a, b, ids, torch.rand(n, generator=g, device="cuda") + 0.5


def formula(base, x, a, b, ids, scale):
    """(values, bound before rounding) of the result."""
    import torch

    y, off = base.double().clone(), torch.zeros(base.shape, dtype=torch.float64, device="cuda")
    n_in, rank = x.shape[1], a.shape[1]
    for g in range(a.shape[0]):
        at = torch.arange(x.shape[0], device="cuda") if ids is None else (ids == g).nonzero().reshape(-1)
        xs, ag, bg, s = x[at].double(), a[g].double(), b[g].double(), float(scale[g])
        h, size = xs @ ag.t(), xs.abs() @ ag.abs().t()
        y[at] += s * h @ bg.t()
        off[at] = s * ((n_in + 8) * 2 * U * size + 2.0 ** -17 * h.abs()) @ bg.abs().t() + (rank + 2) * 4 * U * s * h.abs() @ bg.abs().t()
    return y, off + U * base.double().abs()


SHAPES = [(1, 64, 64, 8, 1), (1, 4096, 1000, 16, 3), (2, 31, 33, 3, 2), (5, 8, 8, 1, 4), (16, 128, 256, 16, 1), (17, 257, 100, 24, 2), (33, 512, 4096, 32, 5), (100, 1000, 72, 17, 40),
          (255, 64, 520, 64, 3), (256, 320, 96, 33, 7), (257, 320, 96, 33, 7), (300, 100, 1001, 16, 2), (1000, 1024, 513, 48, 9), (2100, 264, 328, 65, 4), (700, 72, 200, 130, 3),
          (40, 96, 64, 100, 2), (2500, 40, 48, 8, 33), (64, 2056, 130, 64, 64), (2100, 264, 328, 64, 4), (2048, 100, 1001, 16, 3), (4100, 512, 520, 33, 5), (3000, 1000, 72, 32, 1),
          (2049, 8, 8, 4, 2), (129, 24, 16, 12, 1000)]


@pytest.mark.parametrize("base", ["bf16", "fp32"])
@pytest.mark.parametrize("tokens,n_in,n_out,rank,n", SHAPES)
def test_add(adapters, tokens, n_in, n_out, rank, n, base):
    x, y0, a, b, ids, scale = draw(tokens, n_in, n_out, rank, n, base=base)
    y = adapters.add(y0, x, a, b, ids, scale)
    want, off = formula(y0, x, a, b, ids, scale)
    assert y.dtype == y0.dtype and y.shape == y0.shape
    assert ((y.double() - want).abs() <= 1.01 * half_step(want, y.dtype) + off).all()
    none = (ids < 0) | (ids >= n)
    assert (y[none] == y0[none]).all()
    again = adapters.add(y0, x, a, b, ids, scale)
    assert (y == again).all()


@pytest.mark.parametrize("tokens,rank", [(20, 16), (20, 100), (300, 2), (1000, 24), (1000, 64), (1000, 70), (1000, 512), (3000, 40), (3000, 64)])
def test_an_fp32_base_is_rounded_once(adapters, tokens, rank):
    """Beside a base of 2^20 times the adapters' part all that counts is the last addition, half a step (u) of the result, and what 2^-17 of the part adds."""
    import torch

    x, y0, a, b, ids, scale = draw(tokens, 72, 104, rank, 2, base="fp32")
    y0, b = y0.abs() + 1, b * 2.0 ** -20
    y = adapters.add(y0, x, a, b, ids, scale)
    want, off = formula(y0, x, a, b, ids, scale)
    part = off - U * y0.double().abs()                                            # the bound without the base's share
    assert ((y.double() - want).abs() <= 1.001 * U * want.abs() + part).all()
    assert part.max() < U and (y != y0).any()


@pytest.mark.parametrize("tokens", [1, 15, 16, 100, 256, 300, 1000])
def test_one_adapter_without_ids(adapters, tokens):
    import torch

    x, y0, a, b, _, _ = draw(tokens, 200, 264, 16, 1)
    y = adapters.add(y0, x, a[0], b[0], scale=0.75)
    want, off = formula(y0, x, a, b, None, [0.75])
    assert ((y.double() - want).abs() <= 1.01 * half_step(want, y.dtype) + off).all()
    same = adapters.add(y0, x, a, b, torch.zeros(tokens, dtype=torch.int32, device="cuda"), torch.full((1,), 0.75, device="cuda"))
    assert (y == same).all()


@pytest.mark.parametrize("tokens", [20, 600])
def test_tokens_of_nobody_and_all_of_one(adapters, tokens):
    import torch

    x, y0, a, b, _, scale = draw(tokens, 128, 136, 16, 5)
    none = adapters.add(y0, x, a, b, torch.full((tokens,), -1, dtype=torch.int32, device="cuda"), scale)
    assert (none == y0).all()
    ids = torch.full((tokens,), 4, dtype=torch.int32, device="cuda")
    y = adapters.add(y0, x, a, b, ids, scale)
    want, off = formula(y0, x, a, b, ids, scale)
    assert ((y.double() - want).abs() <= 1.01 * half_step(want, y.dtype) + off).all()


def run_grads(adapters, base, x, a, b, ids, scale, dy):
    import torch

    leaves = [t.detach().requires_grad_() for t in (base, x, a, b)]
    y = adapters.add(leaves[0], leaves[1], leaves[2], leaves[3], ids, scale)
    return torch.autograd.grad(y, leaves, dy)


def check_grads(got, x, a, b, ids, scale, dy):
    import torch

    n_out, tokens, rank = b.shape[1], x.shape[0], a.shape[1]
    dx, off_x = torch.zeros(x.shape, dtype=torch.float64, device="cuda"), torch.zeros(x.shape, dtype=torch.float64, device="cuda")
    for g in range(a.shape[0]):
        at = torch.arange(tokens, device="cuda") if ids is None else (ids == g).nonzero().reshape(-1)
        xs, ag, bg, gs, s = x[at].double(), a[g].double(), b[g].double(), dy[at].double(), float(scale[g])
        u, h = s * gs @ bg, s * xs @ ag.t()
        off_u = (n_out + 8) * 2 * U * s * (gs.abs() @ bg.abs()) + 2.0 ** -17 * u.abs()
        off_h = (x.shape[1] + 8) * 2 * U * s * (xs.abs() @ ag.abs().t()) + 2.0 ** -17 * h.abs()
        dx[at], off_x[at] = u @ ag, off_u @ ag.abs() + (rank + 2) * 4 * U * u.abs() @ ag.abs()
        for name, value, want, off in (("a", got[2][g], u.t() @ xs, off_u.t() @ xs.abs() + (at.numel() + 8) * 4 * U * u.abs().t() @ xs.abs()),
                                       ("b", got[3][g], gs.t() @ h, gs.abs().t() @ off_h + (at.numel() + 8) * 4 * U * gs.abs().t() @ h.abs())):
            assert ((value.double() - want).abs() <= 1.01 * half_step(want, value.dtype) + off).all(), name
    assert ((got[1].double() - dx).abs() <= 1.01 * half_step(dx, got[1].dtype) + off_x).all()


@pytest.mark.parametrize("tokens,n_in,n_out,rank,n", [s for s in SHAPES if s[4] < 100])
def test_gradients(adapters, tokens, n_in, n_out, rank, n):
    import torch

    x, y0, a, b, ids, scale = draw(tokens, n_in, n_out, rank, n, seed=3)
    dy = torch.randn(y0.shape, device="cuda").to(torch.bfloat16)
    got = run_grads(adapters, y0, x, a, b, ids, scale, dy)
    assert (got[0] == dy).all() and all(p.shape == q.shape and p.dtype == q.dtype for p, q in zip(got, (y0, x, a, b)))
    check_grads(got, x, a, b, ids, scale, dy)
    again = run_grads(adapters, y0, x, a, b, ids, scale, dy)
    assert all((p == q).all() for p, q in zip(got, again))


def test_gradients_of_an_adapter_that_every_token_shares(adapters):
    import torch

    for tokens in (3, 5000):
        x, y0, a, b, _, _ = draw(tokens, 264, 200, 16, 1, seed=4)
        dy = torch.randn(y0.shape, device="cuda").to(torch.bfloat16)
        leaves = [t.detach().requires_grad_() for t in (x, a[0], b[0])]
        got = torch.autograd.grad(adapters.add(y0, *leaves, scale=1.5), leaves, dy)
        check_grads((None, got[0], got[1][None], got[2][None]), x, a, b, None, [1.5], dy)


def test_gradients_against_differences(adapters):
    """The loss sum(y dy) is linear in each of x, a and b, so its difference over a whole direction is its slope: kernels' gradients (rounded to BF16: 2^-9 of each
    element, 2^-9 of the sum of magnitudes at most) against the formula's values."""
    import torch

    x, y0, a, b, ids, scale = draw(300, 96, 80, 16, 3, seed=6)
    dy = torch.randn(y0.shape, device="cuda").to(torch.bfloat16)
    got = run_grads(adapters, y0, x, a, b, ids, scale, dy)
    loss = lambda x, a, b: float((formula(y0, x, a, b, ids, scale)[0] * dy.double()).sum())  # noqa: E731
    for i, grad in enumerate(got[1:]):
        at = [t.double() for t in (x, a, b)]
        way = torch.randn(at[i].shape, device="cuda", dtype=torch.float64)
        ends = [loss(*[t + sign * way if k == i else t for k, t in enumerate(at)]) for sign in (1, -1)]
        assert abs(float((grad.double() * way).sum()) - (ends[0] - ends[1]) / 2) <= 2.0 ** -8 * float((grad.double() * way).abs().sum())


def test_only_what_is_asked_for(adapters):
    import torch

    x, y0, a, b, ids, scale = draw(400, 128, 120, 16, 3)
    dy = torch.randn(y0.shape, device="cuda").to(torch.bfloat16)
    full = run_grads(adapters, y0, x, a, b, ids, scale, dy)
    for need in ((1,), (2,), (3,), (0,), (1, 3), (2, 3)):
        leaves = [t.detach().requires_grad_(i in need) for i, t in enumerate((y0, x, a, b))]
        y = adapters.add(*leaves, ids, scale)
        for i, g in zip(need, torch.autograd.grad(y, [leaves[i] for i in need], dy)):
            assert (g == full[i]).all()


def test_any_strides(adapters):
    import torch

    x, y0, a, b, ids, scale = draw(300, 128, 136, 16, 3)
    wide = torch.randn(301, 300, device="cuda").to(torch.bfloat16)
    for tokens in (40, 300):
        i = ids[:tokens]
        for xs, ys in ((wide[:tokens, 1:129], wide[1:tokens + 1, 3:139]), (wide.t()[:128, :tokens].t(), wide[:1, :136].expand(tokens, 136)), (wide[:tokens, 8:136], wide[:tokens, 16:152])):
            y = adapters.add(ys, xs, a.transpose(1, 2).contiguous().transpose(1, 2), b, i, scale)
            assert (y == adapters.add(ys.contiguous(), xs.contiguous(), a, b, i, scale)).all()
    dy = torch.randn(1, 136, device="cuda").to(torch.bfloat16).expand(300, 136)
    got = run_grads(adapters, y0, x, a, b, ids, scale, dy)
    assert all((p == q).all() for p, q in zip(got, run_grads(adapters, y0, x, a, b, ids, scale, dy.contiguous())))


def test_more_dimensions_and_none(adapters):
    import torch

    x, y0, a, b, ids, scale = draw(24, 64, 50, 8, 3)
    y = adapters.add(y0.view(2, 12, 50), x.view(2, 12, 64), a, b, ids.view(2, 12), scale)
    assert y.shape == (2, 12, 50) and (y.reshape(24, 50) == adapters.add(y0, x, a, b, ids, scale)).all()
    one = adapters.add(y0[0], x[0], a, b, ids[0], scale)
    assert one.shape == (50,) and (one == adapters.add(y0[:1], x[:1], a, b, ids[:1], scale)[0]).all()
    got = run_grads(adapters, y0[:0], x[:0], a, b, ids[:0], scale, y0[:0])
    assert got[1].shape == (0, 64) and (got[2] == 0).all() and (got[3] == 0).all()
    assert adapters.add(y0[:0], x[:0], a, b, ids[:0], scale).shape == (0, 50)
    x.requires_grad_()
    y = adapters.add(y0, x, a, b, ids, scale)
    y += 1                                                       # a result is nobody's view
    y.sum().backward()


def test_no_tokens_through_a_layer(adapters):
    """The gradient of a sum has strides of zero, that of nothing too."""
    import torch

    from paper_2512_22804_b200 import fp4

    x, y0, a, b, ids, scale = draw(5, 64, 72, 8, 2)
    w, w_t = fp4.quantize(torch.randn(72, 64, device="cuda").to(torch.bfloat16), "e8m0_32", cols=True)
    for layer in (lambda x, a, b: adapters.linear(x, w, a, b, ids[:0], scale, w_t=w_t), lambda x, a, b: adapters.add(y0[:0], x, a, b, ids[:0], scale)):
        leaves = [t.detach().requires_grad_() for t in (x[:0], a, b)]
        y = layer(*leaves)
        assert y.shape == (0, 72)
        g = torch.autograd.grad(y.sum(), leaves)
        assert g[0].shape == (0, 64) and (g[1] == 0).all() and (g[2] == 0).all()
    leaves = [x[:0].detach().requires_grad_(), b[0, :, :1].expand(72, 64).contiguous().requires_grad_()]
    g = torch.autograd.grad(fp4.linear(*leaves, "e8m0_32").sum(), leaves)
    assert g[0].shape == (0, 64) and (g[1] == 0).all()
    fp4.check()


def test_what_is_not_finite_stays_in_its_row(adapters):
    import torch

    for tokens in (30, 400):
        x, y0, a, b, ids, scale = draw(tokens, 64, 72, 16, 2)
        ids = (torch.arange(tokens, device="cuda") % 2).to(torch.int32)
        clean = adapters.add(y0, x, a, b, ids, scale)
        bad = x.clone()
        bad[3, 5], bad[8, 1] = float("nan"), float("inf")
        y = adapters.add(y0, bad, a, b, ids, scale)
        rest = torch.ones(tokens, dtype=torch.bool, device="cuda")
        rest[[3, 8]] = False
        assert (y[rest] == clean[rest]).all() and not y[3].isfinite().any() and not y[8].isfinite().any()


def test_infinities_of_ranks_that_do_not_fill_an_instruction(adapters):
    """Where all factors are positive an infinite x gives an infinite result, whatever the ranks are filled up with."""
    import torch

    bf16 = dict(device="cuda", dtype=torch.bfloat16)
    for tokens, rank in ((5, 3), (300, 3), (2500, 3), (300, 70), (2500, 40)):
        x, a, b = torch.ones(tokens, 40, **bf16), torch.ones(1, rank, 40, **bf16), torch.ones(1, 48, rank, **bf16)
        x[3, 7] = float("inf")
        y = adapters.add(torch.zeros(tokens, 48, **bf16), x, a, b)
        assert (y[3] == float("inf")).all() and (y[4] == 40 * rank).all()


def test_infinite_adapters_and_rows_that_only_fill_a_tile_up(adapters):
    """Where all factors are positive, the gradients of an adapter with an infinite element are infinite where it counts and not NaN, however many rows its last tile has
    left; another adapter's are what they are without it."""
    import torch

    bf16 = dict(device="cuda", dtype=torch.bfloat16)
    for tokens, rank in ((5, 3), (300, 16), (2500, 16), (2500, 40), (300, 70)):
        for n in (1, 2):
            ids = (torch.arange(tokens, device="cuda") % n).to(torch.int32) if n > 1 else None
            x, base, dy = torch.ones(tokens, 40, **bf16), torch.zeros(tokens, 48, **bf16), torch.ones(tokens, 48, **bf16)
            a, b = torch.ones(n, rank, 40, **bf16), torch.ones(n, 48, rank, **bf16)
            a[0, 1, 7], b[0, 3, 2] = float("inf"), float("inf")
            leaves = [t.requires_grad_() for t in (x, a, b)]
            _, da, db = torch.autograd.grad(adapters.add(base, *leaves, ids), leaves, dy)
            assert not da.isnan().any() and not db.isnan().any()
            want_da, want_db = torch.zeros_like(da, dtype=torch.bool), torch.zeros_like(db, dtype=torch.bool)
            want_da[0, 2], want_db[0, :, 1] = True, True
            assert (da.isinf() == want_da).all() and (db.isinf() == want_db).all()


@pytest.mark.parametrize("tokens,rank", [(20, 3), (300, 16), (2500, 16), (300, 70), (2500, 40)])
def test_infinities_touch_what_they_are_part_of(adapters, tokens, rank):
    """An infinite element of x, a, b or dy: a result is not finite exactly where the formula's is not (an infinity of its second product may have become NaN), and all others
    are bit for bit what they are without it."""
    import torch

    x, y0, a, b, _, scale = draw(tokens, 72, 56, rank, 2, seed=9)
    ids = (torch.arange(tokens, device="cuda") % 3 - 1).to(torch.int32)
    dy = torch.randn(y0.shape, device="cuda").to(torch.bfloat16)
    on = [(ids == g).nonzero().reshape(-1) for g in range(2)]

    def run(x, a, b, dy):
        return [adapters.add(y0, x, a, b, ids, scale), *run_grads(adapters, y0, x, a, b, ids, scale, dy)[1:]]

    def plain(x, a, b, dy):
        x, a, b, dy = (t.double() for t in (x, a, b, dy))
        y, dx, da, db = y0.double(), torch.zeros_like(x), torch.zeros_like(a), torch.zeros_like(b)
        for g, at in enumerate(on):
            h, u = (x[at].unsqueeze(1) * a[g]).sum(2), (dy[at].unsqueeze(2) * b[g]).sum(1)          # no library's zeros beside infinities
            y[at] += (h.unsqueeze(1) * b[g]).sum(2)
            dx[at] = (u.unsqueeze(2) * a[g]).sum(1)
            da[g] = (u.unsqueeze(2) * x[at].unsqueeze(1)).sum(0)
            db[g] = (dy[at].unsqueeze(2) * h.unsqueeze(1)).sum(0)
        return y, dx, da, db

    clean = run(x, a, b, dy)
    assert all(t.isfinite().all() for t in clean)
    for which, place in ((0, (4, 7)), (1, (1, 2, 7)), (2, (1, 5, 1)), (3, (4, 5))):
        for value in (float("inf"), -float("inf")):
            args = [t.clone() for t in (x, a, b, dy)]
            args[which][place] = value
            got, want = run(*args), plain(*args)
            for p, q, c in zip(got, want, clean):
                assert (p.isfinite() == q.isfinite()).all() and (p[q.isfinite()] == c[q.isfinite()]).all()
            assert any(not q.isfinite().all() for q in want)


def test_a_wait_that_runs_out_is_reported(adapters):
    """The library's test hook keeps one CTA from announcing its first products and shortens the limit to about a millisecond: the call returns, the status word says
    so, and the same call without the hook is right."""
    import ctypes

    import torch

    from paper_2512_22804_b200 import binding as mb
    from paper_2512_22804_b200 import fp4

    hook = mb.load().mor_test_skip_tile_load
    hook.argtypes, hook.restype = [ctypes.c_uint32, ctypes.c_longlong], None
    x, y0, a, b, ids, scale = draw(3000, 640, 712, 16, 2, seed=8)
    dy = torch.randn(y0.shape, device="cuda").to(torch.bfloat16)
    want = run_grads(adapters, y0, x, a, b, ids, scale, dy)
    y = adapters.add(y0, x, a, b, ids, scale)
    torch.cuda.synchronize()
    fp4.check()
    for kind in ("forward", "backward"):
        leaves = [t.detach().requires_grad_() for t in (x, a, b)]
        out = adapters.add(y0, *leaves, ids, scale)
        torch.cuda.synchronize()
        hook(0, 2_000_000)
        try:
            adapters.add(y0, x, a, b, ids, scale) if kind == "forward" else torch.autograd.grad(out, leaves, dy)
            torch.cuda.synchronize()
        finally:
            hook(0xFFFFFFFF, 0)
        with pytest.raises(mb.MorError) as error:
            fp4.check()
        assert error.value.status == mb.MOR_ERR_TIMEOUT
        assert (adapters.add(y0, x, a, b, ids, scale) == y).all()
        assert all((p == q).all() for p, q in zip(want, run_grads(adapters, y0, x, a, b, ids, scale, dy)))
        fp4.check()


def test_captured_and_on_another_stream(adapters):
    import torch

    for tokens in (48, 500):
        x, y0, a, b, ids, scale = draw(tokens, 256, 264, 16, 4)
        want = adapters.add(y0, x, a, b, ids, scale)
        dy = torch.randn(y0.shape, device="cuda").to(torch.bfloat16)
        grads = run_grads(adapters, y0, x, a, b, ids, scale, dy)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            again, more = adapters.add(y0, x, a, b, ids, scale), run_grads(adapters, y0, x, a, b, ids, scale, dy)
        side.synchronize()
        assert (again == want).all() and all((p == q).all() for p, q in zip(grads, more))
        xs, ids_s = torch.zeros_like(x), torch.zeros_like(ids)
        one, two = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(one):
            y1 = adapters.add(y0, xs, a, b, ids_s, scale)
            g1 = run_grads(adapters, y0, xs, a, b, ids_s, scale, dy)
        with torch.cuda.graph(two, pool=one.pool()):
            y2 = adapters.add(y0, xs, a, b, ids_s, scale)
        xs.copy_(x)
        ids_s.copy_(ids)
        for _ in range(2):
            one.replay()
            two.replay()
        torch.cuda.synchronize()
        assert (y1 == want).all() and (y2 == want).all() and all((p == q).all() for p, q in zip(grads, g1))


def test_two_streams_at_once(adapters):
    """Calls on two streams, forward and backward and the 4-bit product beside them, give bit for bit what they give one after the other."""
    import torch

    from paper_2512_22804_b200 import fp4

    calls = []
    for seed in (11, 12):
        x, y0, a, b, ids, scale = draw(3000, 640, 712, 24, 3, seed=seed)
        dy = torch.randn(y0.shape, device="cuda").to(torch.bfloat16)
        w = fp4.quantize(torch.randn(704, 640, device="cuda").to(torch.bfloat16), "e8m0_32")[0]
        calls.append((x, y0, a, b, ids, scale, dy, w))

    def run(x, y0, a, b, ids, scale, dy, w):
        return [adapters.add(y0, x, a, b, ids, scale), *run_grads(adapters, y0, x, a, b, ids, scale, dy),
                adapters.linear(x, w, a, b[:, :704].contiguous(), ids, scale)]

    want = [run(*c) for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for _ in range(5):
        for c, s in zip(calls, streams):
            with torch.cuda.stream(s):
                got.append(run(*c))
    torch.cuda.synchronize()
    for n, results in enumerate(got):
        assert all((p == q).all() for p, q in zip(want[n % 2], results))
    fp4.check()


@pytest.mark.parametrize("fmt", ["e8m0_32", "e4m3_16"])
@pytest.mark.parametrize("tokens", [3, 300])
def test_linear(adapters, fmt, tokens):
    """The projection's product as the 4-bit operators make it, then the adapters on its BF16 result; the gradient of x the same way round."""
    import torch

    from paper_2512_22804_b200 import fp4

    x, _, a, b, ids, scale = draw(tokens, 256, 320, 16, 3)
    weight = (torch.randn(320, 256, device="cuda") * 0.05).to(torch.bfloat16)
    w, w_t = fp4.quantize(weight, fmt, cols=True)
    y0 = fp4.matmul(fp4.quantize(x, fmt)[0], w)
    assert (adapters.linear(x, w, a, b, ids, scale) == adapters.add(y0, x, a, b, ids, scale)).all()
    leaves = [t.detach().requires_grad_() for t in (x, a, b)]
    y = adapters.linear(*leaves[:1], w, *leaves[1:], ids, scale, w_t=w_t)
    want, off = formula(y0, x, a, b, ids, scale)
    assert ((y.double() - want).abs() <= 1.01 * half_step(want, y.dtype) + off).all()
    dy = torch.randn(y.shape, device="cuda").to(torch.bfloat16)
    got = torch.autograd.grad(y, leaves, dy)
    through = fp4.matmul(fp4.quantize(dy, fmt)[0], w_t).double()
    plain = run_grads(adapters, y0, x, a, b, ids, scale, dy)
    assert (got[1] == plain[2]).all() and (got[2] == plain[3]).all()
    # plain's dx is rounded (half a step of it); the layer's is rounded once after the sum
    assert ((got[0].double() - through - plain[1].double()).abs() <= 1.01 * half_step(through.abs() + plain[1].double().abs(), torch.bfloat16) * 2 + 1e-6 * through.abs().max()).all()
    stored = fp4.Operand(w_t.codes, w_t.scales, w_t.rows, w_t.cols, fmt, w_t.tensor_scale)
    y = adapters.linear(leaves[0].view(1, tokens, 256), w, *leaves[1:], ids.view(1, tokens), scale, w_t=stored)
    assert y.shape == (1, tokens, 320)
    assert all((p == q).all() for p, q in zip(got, torch.autograd.grad(y, leaves, dy.view(1, tokens, 320))))
    fp4.check()


def test_autograd(adapters):
    import torch

    x, y0, a, b, ids, scale = draw(20, 64, 72, 8, 2)
    x.requires_grad_()
    (g,) = torch.autograd.grad(adapters.add(y0, x, a, b, ids, scale).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="differentiated twice"):
        g.sum().backward()
    y = adapters.add(y0, x, a, b, ids, scale)
    y.sum().backward()
    with pytest.raises(RuntimeError):
        y.sum().backward()
    seen = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: seen.append(t.numel()) or t, lambda t: t):
        adapters.add(y0, x, a, b, ids, scale)
    assert len(seen) >= 5


def test_forward_mode_is_refused(adapters):
    import torch
    import torch.autograd.forward_ad as forward

    from paper_2512_22804_b200 import fp4

    x, y0, a, b, ids, scale = draw(20, 64, 72, 8, 2)
    w, w_t = fp4.quantize(torch.zeros(72, 64, device="cuda", dtype=torch.bfloat16), "e8m0_32", cols=True)
    with forward.dual_level():
        for i in (0, 1, 2, 3, 5):
            args = [forward.make_dual(t, torch.ones_like(t)) if k == i else t for k, t in enumerate((y0, x, a, b, ids, scale))]
            with pytest.raises(RuntimeError, match="forward-mode"):
                adapters.add(*args)
            if i > 0:
                with pytest.raises(RuntimeError, match="forward-mode"):
                    adapters.linear(args[1], w, *args[2:], w_t=w_t)


def test_refusals(adapters):
    import torch

    from paper_2512_22804_b200 import fp4

    x, y0, a, b, ids, scale = draw(20, 64, 72, 8, 2)
    add = adapters.add
    w, w_t = fp4.quantize(torch.zeros(72, 64, device="cuda", dtype=torch.bfloat16), "e8m0_32", cols=True)
    for bad in (lambda: add(y0, x[:, :63], a, b, ids), lambda: add(y0[:, :71], x, a, b, ids), lambda: add(y0[:19], x, a, b, ids), lambda: add(y0, x, a, b[:1], ids), lambda: add(y0, x, a, b[:, :, :7], ids),
                lambda: add(y0, x, a, b), lambda: add(y0, x, a, b, ids[:19]), lambda: add(y0, x, a, b, ids.long()), lambda: add(y0, x, a, b, ids, scale[:1]),
                lambda: add(y0, x, a, b, ids, scale.double()), lambda: add(y0, x, a, b, ids, float("inf")), lambda: add(y0, x, a, b, ids, scale.clone().requires_grad_()),
                lambda: add(y0.cpu(), x, a, b, ids), lambda: add(y0, x, a.cpu(), b, ids), lambda: add(y0, x, a, b, ids.cpu()), lambda: add(y0, x, a[:0], b[:0], ids),
                lambda: add(y0, x, torch.zeros(1, 513, 64, device="cuda", dtype=torch.bfloat16), torch.zeros(1, 72, 513, device="cuda", dtype=torch.bfloat16)),
                lambda: adapters.linear(x[:, :32], w, a, b, ids), lambda: adapters.linear(x.clone().requires_grad_(), w, a, b, ids), lambda: adapters.linear(x, w, a, b, ids, w_t=w)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: add(y0, x.float(), a, b, ids), lambda: add(y0, x, a.float(), b, ids), lambda: add(y0.half(), x, a, b, ids), lambda: add(y0, x, a), lambda: adapters.linear(x, y0, a, b, ids)):
        with pytest.raises(TypeError):
            bad()

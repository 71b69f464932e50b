"""The AdamW step against the formulas in 64 bits, its codes and random roundings, and the optimizer built on it.

u = 2^-24.  In 32 bits m and v are sums of two products (3 u of their terms), the root and the quotient add 4 u, the update two more operations: p is
off by 12 u of the update's size, taken with m's terms' magnitudes (the root halves v's share), and 3 u of |p|.  A code may differ from the formula's only where the random number lies within 2^-16 / 8 + 64 u t of the
point that decides (t, at most 16, is a value in distances of codes).
"""
import math

import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def optim():
    from paper_2512_22804_b200 import optim

    return optim


def T(name):
    import torch

    return {"bf16": torch.bfloat16, "fp32": torch.float32}[name]


def mix(z):
    z = z & 0xFFFFFFFF
    z = ((z ^ (z >> 16)) * 0x7FEB352D) & 0xFFFFFFFF
    z = ((z ^ (z >> 15)) * 0x846CA68B) & 0xFFFFFFFF
    return z ^ (z >> 16)


def words(n, number, step, seed):
    """(of the moments, of the parameter) for every element."""
    import torch

    i = torch.arange(n, device="cuda")
    key = mix(mix((seed + 0x9E3779B9 * step) & 0xFFFFFFFF) + number)
    z = mix(mix((i >> 32) ^ key) + i)
    return z, mix(z ^ 0x9E3779B9)


def power(a):
    """Scale of blocks with these largest magnitudes, in 64 bits."""
    import torch

    e = torch.floor(torch.log2(448 / torch.where(a > 0, a, 448.0))).clamp(max=126)
    near = torch.exp2(e + 1) * a <= 448                                    # log2 next to a whole number
    return torch.exp2(torch.where(near & (e < 126) & (a > 0), e + 1, e))


def values(codes, scales, column):
    import torch

    n = codes.numel()
    s = torch.exp2(scales[:, column].double() - 127).repeat_interleave(128)[:n]
    return codes.reshape(-1).double() / s


def new_state(n, seed):
    """Moments in codes as an optimizer has them after some steps."""
    import torch

    g = torch.Generator(device="cuda").manual_seed(seed)
    pad = -n % 128
    out, scales = [], []
    for k in range(2):
        x = torch.randn(n, generator=g, device="cuda") * torch.exp2(torch.randn(n, generator=g, device="cuda") * 3 - 12)
        x = x if k == 0 else x.abs()
        b = torch.nn.functional.pad(x, (0, pad)).view(-1, 128)
        s = power(b.abs().amax(1, keepdim=True).double())
        out.append((b.double() * s).float().to(torch.float8_e4m3fn).view(-1)[:n].contiguous())
        scales.append((torch.log2(s) + 127).to(torch.uint8).view(-1))
    return out[0], out[1], torch.stack(scales, 1).contiguous()


def formula(p, g, m, v, step, lr, b1, b2, eps, decay):
    # of m's two terms, which may cancel: b1, 1 - b1, both products and the sum are rounded, each by u of a term at most, so m is off by 3 u of their magnitudes' sum
    terms = (b1 * m).abs() + ((1 - b1) * g).abs()
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    d = lr / (1 - b1 ** step) * m / (v.sqrt() / math.sqrt(1 - b2 ** step) + eps)
    size = lr / (1 - b1 ** step) * terms / (v.sqrt() / math.sqrt(1 - b2 ** step) + eps)
    return p * (1 - lr * decay) - d, m, v, size


def check_param(got, want, size, p, z, dtype):
    """In 32 bits within the bound; in BF16 one of the two neighbours, the one that the random number says unless it is next to the deciding point."""
    import torch

    off = 16 * U * size + 4 * U * p.abs() + 4 * U * want.abs() + 1e-44
    if dtype == torch.float32:
        assert ((got.double() - want).abs() <= off).all()
        return
    d = torch.exp2(torch.floor(torch.log2(want.abs().clamp(min=2.0 ** -126))) - 7)
    t = want.abs() / d
    u = (z & 0xFFFF).double() / 65536
    chosen = torch.sign(want) * torch.floor(t + u) * d
    unsure = ((t + u) - torch.round(t + u)).abs() <= off / d + 2.0 ** -16
    assert ((got.double() == chosen) | unsure).all() and ((got.double() - want).abs() <= 1.001 * d + off).all()
    assert unsure.double().mean() < 0.05


def check_codes(codes, scales, column, x, z):
    """x: the moment (or the second's root) in 64 bits."""
    import torch

    n = x.numel()
    b = torch.nn.functional.pad(x, (0, -n % 128)).view(-1, 128)
    a = b.abs().amax(1)
    s = torch.exp2(scales[:, column].double() - 127)
    assert ((s == power(a * (1 + 16 * U))) | (s == power(a * (1 - 16 * U))))[a > 1e-30].all() and (scales[:, column][a == 0] == 127).all()
    w = (b * s.unsqueeze(1)).view(-1)[:n]
    d = torch.exp2(torch.floor(torch.log2(w.abs().clamp(min=2.0 ** -6))) - 3)
    t = w.abs() / d
    k = torch.floor(t)
    if column == 0:
        u = (z & 0xFFFF).double() / 65536
        q = torch.floor(t + u)
        margin = ((t + u) - torch.round(t + u)).abs()
    else:
        u = (z >> 16).double() / 65536
        q = torch.where(u * (2 * k + 1) < (t - k) * (t + k), k + 1, k)
        q = torch.where(t > 0, q.clamp(min=1), q)
        margin = (u * (2 * k + 1) - (t - k) * (t + k)).abs() / (2 * k + 1)
        # where t is next to a whole number k, 32 bits may see it on either side: from below (k - 1) the upper code, k, is taken unless u is next to 1, from
        # above the lower one, k again, unless u is next to 0
        whole = (t - torch.round(t)).abs() <= 64 * U * t.clamp(min=1)
        margin = torch.where(whole, torch.minimum(margin, torch.minimum(u, 1 - u)), margin)
    unsure = margin <= 2.0 ** -19 + 64 * U * t.clamp(min=1)
    got = codes.reshape(-1).double()
    assert ((got == torch.sign(w) * q * d) | unsure).all() and ((got.abs() - w.abs()).abs() <= 1.001 * d).all()
    assert unsure.double().mean() < 0.01 or n < 1000


SIZES = [1, 7, 127, 128, 129, 2048, 4095, 4096, 4097, 100_003]


@pytest.mark.parametrize("grad", ["bf16", "fp32"])
@pytest.mark.parametrize("param", ["bf16", "fp32"])
@pytest.mark.parametrize("bits", [8, 32])
def test_step(optim, bits, param, grad):
    import torch

    g = torch.Generator(device="cuda").manual_seed(11)
    r = lambda n: torch.randn(n, generator=g, device="cuda")  # noqa: E731
    params = [(r(n) * 0.1).to(T(param)) for n in SIZES]
    grads = [torch.where(torch.rand(n, generator=g, device="cuda") < 0.1, 0.0, r(n) * torch.exp2(r(n) * 3 - 10)).to(T(grad)) for n in SIZES]
    before = [p.double() for p in params]
    if bits == 8:
        m, v, scales = (list(t) for t in zip(*(new_state(n, n) for n in SIZES)))
        old = [(values(a, s, 0), values(b, s, 1).square()) for a, b, s in zip(m, v, scales)]
    else:
        m, v, scales = [r(n) * 1e-3 for n in SIZES], [(r(n) * 1e-3).square() for n in SIZES], None
        old = [(a.double(), b.double()) for a, b in zip(m, v)]
    kw = dict(lr=3e-3, eps=1e-8, weight_decay=0.1)
    optim.adamw_(params, grads, m, v, scales, step=7, beta1=0.9, beta2=0.99, seed=12345678901, **kw)
    for i, n in enumerate(SIZES):
        want, wm, wv, size = formula(before[i], grads[i].double(), *old[i], 7, kw["lr"], 0.9, 0.99, kw["eps"], kw["weight_decay"])
        z, zp = words(n, i, 7, 12345678901)
        check_param(params[i], want, size, before[i], zp, T(param))
        if bits == 32:
            assert ((m[i].double() - wm).abs() <= 3 * U * (old[i][0].abs() + grads[i].double().abs()) + 1e-44).all()
            assert ((v[i].double() - wv).abs() <= 4 * U * wv + 1e-44).all()
        else:
            check_codes(m[i], scales[i], 0, wm, z)
            check_codes(v[i], scales[i], 1, wv.sqrt(), z)
            mv, vv = optim.moments(m[i], v[i], scales[i])
            assert (mv.double() == values(m[i], scales[i], 0)).all() and (vv.double() == values(v[i], scales[i], 1).square()).all()
            assert (optim.moments(m[i], v[i], scales[i], torch.bfloat16)[0] == mv.to(torch.bfloat16)).all()


@pytest.mark.parametrize("count", [1, 16, 17, 128, 129, 600])
def test_many_tensors_are_each_their_own(optim, count):
    """A list gives what the calls one by one give, but for the random numbers, which go by the tensor's place: in 32 bits all is the same."""
    import torch

    g = torch.Generator(device="cuda").manual_seed(count)
    sizes = [int(n) for n in torch.randint(0, 9000, (count,), generator=torch.Generator().manual_seed(count))]
    make = lambda: [torch.randn(n, generator=g, device="cuda") for n in sizes]  # noqa: E731
    p, gr, m, v = make(), make(), make(), [t.square() for t in make()]
    copies = [[t.clone() for t in ts] for ts in (p, m, v)]
    optim.adamw_(p, gr, m, v, step=3)
    for i in range(count):
        optim.adamw_([copies[0][i]], [gr[i]], [copies[1][i]], [copies[2][i]], step=3)
    for a, b in zip((p, m, v), copies):
        assert all((x == y).all() for x, y in zip(a, b))
    m8, v8, s8 = (list(t) for t in zip(*(new_state(max(1, n), n) for n in sizes)))
    p8 = [torch.zeros(max(1, n), device="cuda", dtype=torch.bfloat16) for n in sizes]
    old = [(values(a, s, 0), values(b, s, 1).square()) for a, b, s in zip(m8, v8, s8)]
    optim.adamw_(p8, [torch.ones_like(t) for t in p8], m8, v8, s8, step=1, lr=1.0)
    for i, t in enumerate(p8):
        zero = torch.zeros(t.numel(), dtype=torch.float64, device="cuda")
        want, _, _, size = formula(zero, zero + 1, *old[i], 1, 1.0, 0.9, 0.999, 1e-8, 0.0)
        check_param(t, want, size, zero, words(t.numel(), i, 1, 0)[1], torch.bfloat16)


def test_numbers_of_tensors(optim):
    """A tensor's number takes the place of its place: two calls with numbers give what one call gives, in launches of up to 512 tensors, and the largest number is
    the formula's too."""
    import torch

    def make():
        g = torch.Generator(device="cuda").manual_seed(5)
        sizes = [200 + i for i in range(600)]
        m, v, s = (list(t) for t in zip(*(new_state(n, n) for n in sizes)))
        return [torch.zeros(n, device="cuda", dtype=torch.bfloat16) for n in sizes], [torch.randn(n, generator=g, device="cuda") for n in sizes], m, v, s

    one, two = make(), make()
    optim.adamw_(*one, step=3, seed=8)
    odd, even = ([t[k::2] for t in two] for k in (1, 0))
    optim.adamw_(*odd, step=3, seed=8, numbers=list(range(1, 600, 2)))
    optim.adamw_(*even, step=3, seed=8, numbers=tuple(range(0, 600, 2)))
    assert all((a.float() == b.float()).all() for i in (0, 2, 3, 4) for a, b in zip(one[i], two[i]))
    n = 3000
    p, g = torch.zeros(n, device="cuda", dtype=torch.bfloat16), torch.randn(n, device="cuda")
    optim.adamw_([p], [g], [torch.zeros(n, device="cuda")], [torch.zeros(n, device="cuda")], step=2, lr=1e-2, seed=4, numbers=[2 ** 31 - 1])
    zero = torch.zeros(n, dtype=torch.float64, device="cuda")
    want, _, _, size = formula(zero, g.double(), zero, zero, 2, 1e-2, 0.9, 0.999, 1e-8, 0.0)
    check_param(p, want, size, zero, words(n, 2 ** 31 - 1, 2, 4)[1], torch.bfloat16)
    for bad in ([1, 2], [-1], [2 ** 31]):
        with pytest.raises(ValueError):
            optim.adamw_([p], [g], [g.clone()], [g.clone()], step=1, numbers=bad)
    for bad in ([1.0], 3):
        with pytest.raises(TypeError):
            optim.adamw_([p], [g], [g.clone()], [g.clone()], step=1, numbers=bad)


def test_no_two_parameters_share_random_numbers(optim):
    """Equal parameters with equal gradients in two groups, or of two gradients' types, are rounded apart, as in one call; a parameter's random numbers do not depend on
    which others have a gradient."""
    import torch

    torch.manual_seed(0)
    d = torch.randn(4096, device="cuda").to(torch.bfloat16)
    g = torch.randn(4096, device="cuda").to(torch.bfloat16) * 1e-3

    def run(groups, types=(torch.bfloat16, torch.bfloat16), missing=()):
        p = [torch.nn.Parameter(d.clone()) for _ in range(2)]
        o = optim.AdamW([{"params": [t]} for t in p] if groups else p, seed=1)
        for i, t in enumerate(p):
            if i not in missing:
                if types[i] == torch.float32:
                    t.grad_dtype = None
                t.grad = g.to(types[i])
        o.step()
        return p, [o.state[t] for t in p]

    p, s = run(False)
    assert (p[0] != p[1]).float().mean() > 0.1 and (s[0]["exp_avg"].float() != s[1]["exp_avg"].float()).float().mean() > 0.1
    q, t = run(True)
    assert all((a == b).all() for a, b in zip(p, q)) and all((a["exp_avg"].float() == b["exp_avg"].float()).all() for a, b in zip(s, t))
    q, t = run(False, (torch.bfloat16, torch.float32))
    assert all((a == b).all() for a, b in zip(p, q)) and all((a["exp_avg"].float() == b["exp_avg"].float()).all() for a, b in zip(s, t))
    q, t = run(False, missing=(0,))
    assert (p[1] == q[1]).all() and (s[1]["exp_avg"].float() == t[1]["exp_avg"].float()).all()


def test_views_that_start_anywhere(optim):
    import torch

    for shift in (1, 3, 8):
        n = 5000
        buf = lambda dtype: torch.zeros(n + 64, device="cuda", dtype=dtype)[shift:shift + n]  # noqa: E731
        m, v, s = new_state(n, 5)
        p = torch.randn(n, device="cuda").to(torch.bfloat16)
        g = torch.randn(n, device="cuda").to(torch.bfloat16)
        state = [t.clone() for t in (p, g, m, v, s)]
        moved = [buf(t.dtype) for t in (p, g, m, v)]
        for to, t in zip(moved, (p, g, m, v)):
            to.copy_(t)
        guard = [t._base if t._base is not None else t for t in moved]
        optim.adamw_([state[0]], [state[1]], [state[2]], [state[3]], [state[4]], step=4, seed=9)
        optim.adamw_([moved[0]], [moved[1]], [moved[2]], [moved[3]], [s], step=4, seed=9)
        assert all((a.float() == b.float()).all() for a, b in zip(state, moved + [s]))
        for t in guard:
            assert (t[:shift].float() == 0).all() and (t[shift + n:].float() == 0).all()


def test_rounding_keeps_the_mean(optim):
    """Moments and BF16 parameters that a nearest rounding would never move: over 512 seeds the mean is the formula's within six deviations of a mean of roundings
    (each off by half a distance at most, so a deviation of a mean is at most d / 2 / sqrt(512))."""
    import torch

    n, seeds = 1280, 512
    m, v, s = new_state(n, 3)
    p = torch.randn(n, device="cuda").to(torch.bfloat16)
    g = torch.randn(n, device="cuda") * 1e-3
    om, ov = values(m, s, 0), values(v, s, 1).square()
    want, wm, wv, _ = formula(p.double(), g.double(), om, ov, 100, 1e-4, 0.9, 0.999, 1e-8, 0.0)
    total = [torch.zeros(n, dtype=torch.float64, device="cuda") for _ in range(3)]
    for seed in range(seeds):
        t = [x.clone() for x in (p, m, v, s)]
        optim.adamw_([t[0]], [g], [t[1]], [t[2]], [t[3]], step=100, lr=1e-4, seed=seed)
        total[0] += t[0].double()
        total[1] += values(t[1], t[3], 0)
        total[2] += values(t[2], t[3], 1).square()
    mean = [t / seeds for t in total]
    scale = [power(torch.nn.functional.pad(x, (0, -n % 128)).view(-1, 128).amax(1)).repeat_interleave(128)[:n] for x in (wm.abs(), wv.sqrt())]
    step = lambda w: torch.exp2(torch.floor(torch.log2(w.abs().clamp(min=2.0 ** -6))) - 3)  # noqa: E731
    dp = torch.exp2(torch.floor(torch.log2(want.abs())) - 7)
    dm = step(wm * scale[0]) / scale[0]
    w = wv.sqrt() * scale[1]
    dv = (2 * w + step(w)) * step(w) / scale[1].square()                    # distance of neighbouring squares
    # 16 random bits: the chance itself is good to 2^-16
    for got, x, d in ((mean[0], want, dp), (mean[1], wm, dm), (mean[2], wv, dv)):
        ok = (got - x).abs() <= 6 * d / 2 / math.sqrt(seeds) + d * 2.0 ** -15 + 1e-6 * x.abs()
        if d is dv:
            ok |= w < 2.0 ** -9                                             # below the smallest code: kept above zero
        assert ok.all()


def test_a_root_above_zero_stays_above_zero_and_zeros_stay(optim):
    import torch

    n = 256
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    m, v = (torch.zeros(n, device="cuda").to(torch.float8_e4m3fn) for _ in range(2))
    s = torch.full((2, 2), 127, dtype=torch.uint8, device="cuda")
    optim.adamw_([p], [g], [m], [v], [s], step=1)
    assert (s == 127).all() and (p == 0).all() and (m.float() == 0).all() and (v.float() == 0).all()
    g[0], g[1:128] = 1.0, 1e-9
    optim.adamw_([p], [g], [m], [v], [s], step=1)
    assert (v.float()[:128] > 0).all() and (v.float()[128:] == 0).all() and p.isfinite().all()


def test_the_smallest_roots_beside_the_largest(optim):
    """Roots from 2^62 down to 2^-62 in blocks of one largest each (without memory of the step before a root is the gradient's magnitude, exactly): a root above zero is at
    least the smallest code however far below its block's largest it lies, up to a ratio of 2^-124."""
    import torch

    k = torch.arange(-62, 63, device="cuda")
    for top in (62, 30, 0, -30):
        g = torch.zeros(256, device="cuda")
        low = k[k <= top]
        g[:low.numel()] = torch.exp2(low.float()) * torch.where(low % 2 == 0, 1.0, -1.0)
        g[128:][:low.numel()] = torch.exp2(low.float()) * 1.375
        p, (m, v) = torch.zeros(256, device="cuda"), (torch.zeros(256, device="cuda").to(torch.float8_e4m3fn) for _ in range(2))
        s = torch.full((2, 2), 127, dtype=torch.uint8, device="cuda")
        optim.adamw_([p], [g], [m], [v], [s], step=1, beta2=0.0)
        roots = v.float().view(2, 128)
        w = g.abs().view(2, 128) * torch.exp2(s[:, 1:].float() - 127)
        assert (roots[:, low.numel():] == 0).all() and (roots[:, :low.numel()] >= 2.0 ** -9).all()
        assert (roots[w < 2.0 ** -9] <= 2.0 ** -9).all() and p.isfinite().all()
        check_codes(v, s, 1, g.double().abs(), words(256, 0, 1, 0)[0])


def test_extremes(optim):
    import torch

    n = 640
    p = torch.zeros(n, device="cuda")
    g = torch.zeros(n, device="cuda")
    g[3], g[130], g[260], g[261], g[400:500] = float("nan"), float("inf"), 3e38, 1e-30, 1e-38
    m, v = (torch.zeros(n, device="cuda").to(torch.float8_e4m3fn) for _ in range(2))
    s = torch.full((5, 2), 127, dtype=torch.uint8, device="cuda")
    optim.adamw_([p], [g], [m], [v], [s], step=1, eps=1e-8)
    mv, vv = optim.moments(m, v, s)
    assert mv[3].isnan() and vv[3].isnan() and p[3].isnan()
    assert mv[130].isnan() and vv[130].isnan() and vv[260].isnan()                # its square is beyond 32 bits
    keep = torch.ones(n, dtype=torch.bool, device="cuda")
    keep[[3, 130]] = False
    assert p[keep].isfinite().all() and mv[keep].isfinite().all() and (vv[261:384] == 0).all()
    assert abs(float(mv[260]) - 3e37) < 3e36 * 1.3


def test_scalars_on_the_gpu(optim):
    import torch

    n = 3000
    make = lambda: [torch.randn(n, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")]  # noqa: E731
    g = [torch.randn(n, device="cuda")]
    a, b, c = make(), make(), make()
    state = lambda: ([torch.zeros(n, device="cuda")], [torch.zeros(n, device="cuda")])  # noqa: E731
    one = lambda v, t=torch.float32: torch.full((1,), v, dtype=t, device="cuda")  # noqa: E731
    sa, sb, sc = state(), state(), state()
    optim.adamw_(a, g, *sa, step=5, lr=1e-2)
    optim.adamw_(b, g, *sb, step=one(5, torch.int32), lr=one(1e-2))
    assert ((a[0] - b[0]).abs() <= 1e-2 * 32 * U * 4 + 4 * U * a[0].abs()).all() and (sa[0][0] == sb[0][0]).all()
    optim.adamw_(c, [g[0] * 4], *sc, step=5, lr=1e-2, grad_scale=one(0.25))
    assert (c[0] == a[0]).all() and (sc[1][0] == sa[1][0]).all()
    for bad in (1.0, float("nan"), float("inf")):
        before = c[0].clone()
        optim.adamw_(c, g, *sc, step=6, lr=1e-2, found_inf=one(bad))
        assert (c[0] == before).all() and (sc[1][0] == sa[1][0]).all()
    optim.adamw_(c, g, *sc, step=6, lr=1e-2, found_inf=one(0.0))
    assert (c[0] != before).any()
    for b1 in (0.0, 0.9):                                                        # without memory
        p = make()
        optim.adamw_(p, g, *state(), step=1, beta1=b1, beta2=0.0, lr=0.5, eps=0.0)
        assert ((p[0] - (a0 := make()[0]) + 0.5 * torch.sign(g[0])).abs() <= 1e-5).all(), a0


def test_more_than_2_to_the_32_elements(optim):
    """The last elements of a tensor whose numbers pass 32 bits: the same as a formula says for them, random numbers included."""
    import torch

    n = 2 ** 32 + 5000
    p, g = torch.zeros(n, device="cuda", dtype=torch.bfloat16), torch.zeros(n, device="cuda", dtype=torch.bfloat16)
    m, v = torch.zeros(n, device="cuda", dtype=torch.float8_e4m3fn), torch.zeros(n, device="cuda", dtype=torch.float8_e4m3fn)
    s = torch.full(((n + 127) // 128, 2), 127, dtype=torch.uint8, device="cuda")
    k = 5000 + 256
    gen = torch.Generator(device="cuda").manual_seed(2)
    g[-k:] = torch.randn(k, generator=gen, device="cuda").to(torch.bfloat16)
    g[:k] = g[-k:]
    optim.adamw_([p], [g], [m], [v], [s], step=2, lr=1e-2, seed=4)
    zero = torch.zeros(k, dtype=torch.float64, device="cuda")
    want, wm, wv, size = formula(zero, g[-k:].double(), zero, zero, 2, 1e-2, 0.9, 0.999, 1e-8, 0.0)
    i = torch.arange(n - k, n, device="cuda")
    key = mix(mix((4 + 0x9E3779B9 * 2) & 0xFFFFFFFF) + 0)
    z = mix(mix((i >> 32) ^ key) + (i & 0xFFFFFFFF))
    check_param(p[-k:], want, size, zero, mix(z ^ 0x9E3779B9), torch.bfloat16)
    first = (n - k + 127) // 128 * 128 - (n - k)                                 # the first whole block
    check_codes(m[n - k + first:], s[(n - k + first) // 128:], 0, wm[first:], z[first:])
    assert (p[-k:] != p[:k]).any() and (p[k:-k] == 0).all()


def test_optimizer_in_32_bits_is_torch_s(optim):
    """Twenty steps beside torch's AdamW in FP32: each step's update is off by 16 u of its size of about lr, and differences pass on through the decay alone."""
    import torch

    torch.manual_seed(0)
    p = [torch.nn.Parameter(torch.randn(s, device="cuda")) for s in ((33, 7), (4000,), ())]
    q = [torch.nn.Parameter(t.detach().clone()) for t in p]
    kw = dict(lr=1e-2, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1)
    ours, theirs = optim.AdamW(p, bits=32, **kw), torch.optim.AdamW(q, **kw)
    for step in range(20):
        for a, b in zip(p, q):
            a.grad = torch.randn_like(a)
            b.grad = a.grad.clone()
        if step == 5:
            p[0].grad = q[0].grad = None
        ours.step()
        theirs.step()
    for a, b in zip(p, q):
        assert ((a - b).abs() <= 20 * (1e-2 * 64 * U * 4 + 8 * U * b.abs())).all()


@pytest.mark.parametrize("bits", [8, 32])
def test_optimizer_state_is_stored_and_loaded(optim, bits):
    import io

    import torch

    def fresh():
        torch.manual_seed(1)
        p = [torch.nn.Parameter(torch.randn(300, 10, device="cuda").to(torch.bfloat16)), torch.nn.Parameter(torch.randn(50, device="cuda"))]
        return p, optim.AdamW([{"params": p[:1], "lr": 1e-2}, {"params": p[1:]}], bits=bits, seed=3)

    def run(p, o, steps):
        for k in steps:
            for t in p:
                t.grad = torch.randn(t.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(k)).to(t.dtype)
            o.step()

    p, o = fresh()
    run(p, o, range(6))
    q, o2 = fresh()
    run(q, o2, range(3))
    file = io.BytesIO()
    torch.save((o2.state_dict(), [t.detach() for t in q]), file)
    file.seek(0)
    state, data = torch.load(file, weights_only=True)
    r, o3 = fresh()
    with torch.no_grad():
        for t, d in zip(r, data):
            t.copy_(d)
    o3.load_state_dict(state)
    assert o3.state[r[0]]["exp_avg"].dtype == (torch.float8_e4m3fn if bits == 8 else torch.float32)
    run(r, o3, range(3, 6))
    assert all((a == b).all() for a, b in zip(p, r))
    run(q, o2, range(3, 6))                                                       # the stored one was no alias
    assert all((a == b).all() for a, b in zip(p, q))


def test_optimizer_captured(optim):
    import torch

    def fresh(capturable):
        torch.manual_seed(1)
        p = [torch.nn.Parameter(torch.randn(n, device="cuda").to(t)) for n, t in ((5000, torch.bfloat16), (700, torch.float32), (300, torch.bfloat16))]
        lr = torch.full((1,), 1e-2, device="cuda") if capturable else 1e-2
        return p, optim.AdamW(p, lr=lr, seed=3, capturable=capturable)

    grads = [torch.randn(n, device="cuda") for n in (5000, 700, 300)]
    p, o = fresh(False)
    for _ in range(5):
        for t, g in zip(p, grads):
            t.grad = g.to(t.dtype)
        o.step()
    q, c = fresh(True)
    for t, g in zip(q, grads):
        t.grad = g.to(t.dtype)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.step()
    for _ in range(4):
        graph.replay()
    torch.cuda.synchronize()
    assert int(c.param_groups[0]["step"]) == 5
    r, again = fresh(True)                     # the count goes through a stored state, on whatever device that was loaded
    state = c.state_dict()
    state["param_groups"][0]["step"] = state["param_groups"][0]["step"].cpu()
    again.load_state_dict(state)
    for t, g in zip(r, grads):
        t.grad = g.to(t.dtype)
    again.step()
    assert int(again.param_groups[0]["step"]) == 6 and int(c.param_groups[0]["step"]) == 5
    for a, b in zip(p, q):                     # the bias corrections are made another way: an update differs by some u, a BF16 rounding may fall the other way
        d = (a.detach().double() - b.detach().double()).abs()
        assert (d <= 5e-6 + a.detach().double().abs() * (2.0 ** -7 if a.dtype == torch.bfloat16 else 1e-5)).all() and (d > 1e-6).double().mean() < 0.01


@pytest.mark.parametrize("captured", [False, True])
def test_each_parameter_counts_its_own_steps_with_capturable(optim, captured):
    """Parameters that start later or miss steps, beside the optimizer that counts on the host: the moments are the same, and an update differs by the bias corrections,
    made in 32 bits (their arguments by 2 u, their values by 4 u more) on top of the 16 u of its size, which for these gradients is within 4 lr."""
    import torch

    lr, sizes = 1e-2, (300, 5000, 40, 77)
    with_grad = [(0, 1, 2)] * 3 + [(0, 2)] * 4 + [(0, 1, 2, 3)] * 2 + [(1, 3)] * 3 + [(0, 1, 2, 3)]

    def fresh(capturable):
        torch.manual_seed(1)
        p = [torch.nn.Parameter(torch.randn(n, device="cuda")) for n in sizes]
        return p, optim.AdamW(p, lr=lr, bits=32, capturable=capturable)

    grads = [torch.randn(n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(n)) for n in sizes]
    p, o = fresh(False)
    q, c = fresh(True)
    graphs = {}
    for k, some in enumerate(with_grad):
        for ps in (p, q):
            for i, t in enumerate(ps):
                t.grad = grads[i].clone() * (k + 1) if i in some and (ps is p or not captured) else None
        o.step()
        if not captured:
            c.step()
            continue
        for i in some:
            if not hasattr(q[i], "static"):
                q[i].static = torch.empty_like(q[i])
            q[i].static.copy_(grads[i] * (k + 1))
            q[i].grad = q[i].static
        seen = {i for before in with_grad[:k] for i in before}
        if not set(some) <= seen:
            c.step()                                       # a parameter's first step takes its memory
        else:
            if some not in graphs:
                graphs[some] = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graphs[some]):
                    c.step()
            graphs[some].replay()
    torch.cuda.synchronize()
    assert int(c.param_groups[0]["step"]) == len(with_grad)
    for a, b in zip(p, q):
        assert int(c.state[b]["step"]) == o.state[a]["step"]
        assert all((o.state[a][m] == c.state[b][m]).all() for m in ("exp_avg", "exp_avg_sq"))
        assert ((a.detach().double() - b.detach().double()).abs() <= len(with_grad) * (4 * lr * 32 * U + 8 * U * a.detach().abs())).all()


def test_captures_that_could_not_go_on_are_refused(optim):
    """Nothing is changed by a refused capture, and the optimizer goes on after it."""
    import torch

    def fresh(capturable):
        p = [torch.nn.Parameter(torch.zeros(300, device="cuda")) for _ in range(2)]
        return p, optim.AdamW([{"params": p[:1]}, {"params": p[1:]}], bits=32, lr=1e-2, capturable=capturable)

    def capture(o, message):
        with pytest.raises(RuntimeError, match=message):
            with torch.cuda.graph(torch.cuda.CUDAGraph()):
                o.step()

    one = torch.ones(300, device="cuda")
    for capturable in (True, False):
        p, o = fresh(capturable)
        p[0].grad = one
        if capturable:
            capture(o, "first step")
            assert not o.state[p[0]]
        o.step()
        p[1].grad = one
        capture(o, "first step" if capturable else "capturable=True")
        assert int(o.state[p[0]]["step"]) == 1 and (p[1] == 0).all()
        o.step()
        assert int(o.state[p[0]]["step"]) == 2 and int(o.state[p[1]]["step"]) == 1
        assert ((p[1] + 1e-2).abs() <= 1e-2 * 32 * U).all()


def test_counts_of_steps_are_stored_and_loaded(optim):
    import copy
    import io

    import torch

    def fresh():
        torch.manual_seed(1)
        p = [torch.nn.Parameter(torch.randn(n, device="cuda").to(t)) for n, t in ((5000, torch.bfloat16), (700, torch.float32), (300, torch.bfloat16), (10, torch.float32))]
        return p, optim.AdamW([{"params": p[:2]}, {"params": p[2:]}], lr=1e-2, seed=3, capturable=True)

    def run(p, o, steps):
        for k in steps:
            for i, t in enumerate(p):
                t.grad = torch.randn(t.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(k)).to(t.dtype) if i != 2 or k > 1 else None
            o.step()

    p, o = fresh()
    run(p, o, range(6))
    q, o2 = fresh()
    run(q, o2, range(3))
    assert [int(o2.state[t]["step"]) for t in q] == [3, 3, 1, 3]
    file = io.BytesIO()
    torch.save((o2.state_dict(), [t.detach() for t in q]), file)
    file.seek(0)
    state, data = torch.load(file, weights_only=True)
    r, o3 = fresh()
    with torch.no_grad():
        for t, d in zip(r, data):
            t.copy_(d)
    o3.load_state_dict(state)
    run(r, o3, range(3, 6))
    assert all((a == b).all() for a, b in zip(p, r)) and [int(o3.state[t]["step"]) for t in r] == [6, 6, 4, 6]
    assert [int(o2.state[t]["step"]) for t in q] == [3, 3, 1, 3]                 # the stored ones were no aliases
    both = copy.deepcopy((q, o2))                                                # counts that lie anywhere
    run(both[0], both[1], range(3, 6))
    assert all((a == b).all() for a, b in zip(p, both[0]))
    assert all((a == b).all() for a, b in zip(p, both[0]))
    old = o2.state_dict()                                                        # as it was stored when a group's parameters shared its count
    old = {"state": {i: dict(s, step=0) for i, s in old["state"].items()}, "param_groups": old["param_groups"]}
    r, o3 = fresh()
    o3.load_state_dict(old)
    assert [int(o3.state[t]["step"]) for t in r] == [3, 3, 3, 3]
    for group in o2.param_groups:                                                # counted on the host for a while, and a parameter waits there
        group["capturable"] = False
    run(q, o2, range(3, 5))
    for group in o2.param_groups:
        group["capturable"] = True
    q[1].grad = None
    o2.step()
    assert [int(o2.state[t]["step"]) for t in q] == [6, 5, 4, 6]
    o3.load_state_dict(o2.state_dict())
    assert [int(o3.state[t]["step"]) for t in r] == [6, 5, 4, 6]


def test_steps_of_several_tensors_on_the_gpu(optim):
    """One call with a step's number for every tensor is the calls one by one, in launches of up to 512 tensors."""
    import torch

    n = 520
    make = lambda: [[torch.full((130,), 1.0, device="cuda") for _ in range(n)], [torch.full((130,), 0.5, device="cuda") for _ in range(n)],  # noqa: E731
                    [torch.full((130,), 0.1, device="cuda") for _ in range(n)], [torch.full((130,), 0.01, device="cuda") for _ in range(n)]]
    a, b = make(), make()
    steps = torch.arange(1, n + 1, dtype=torch.int32, device="cuda") % 37 + 1
    optim.adamw_(*a, step=steps)
    for i in range(n):
        optim.adamw_(*[[t[i]] for t in b], step=steps[i])
    assert all((x == y).all() for s, t in zip(a, b) for x, y in zip(s, t))
    assert (a[0][0] != a[0][1]).any()
    for bad in (steps[:-1], steps[:2], torch.stack((steps, steps), 1)[:, 0], steps.long(), steps.cpu()):
        with pytest.raises(ValueError):
            optim.adamw_(*a, step=bad)


def test_autograd_sees_the_change(optim):
    import torch

    p = torch.randn(100, device="cuda", requires_grad=True)
    y = (p * p).sum()
    optim.adamw_([p.detach()], [torch.ones(100, device="cuda")], [torch.zeros(100, device="cuda")], [torch.zeros(100, device="cuda")], step=1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_what_requires_a_gradient_is_changed_under_no_grad_only(optim):
    import torch

    z = lambda: torch.zeros(64, device="cuda")  # noqa: E731
    for i in (0, 2, 3):
        args = [z() if k != 1 else z() + 1 for k in range(4)]
        args[i].requires_grad_()
        with pytest.raises(RuntimeError, match="no_grad"):
            optim.adamw_(*[[t] for t in args], step=1)
        assert all((t == 0).all() for k, t in enumerate(args) if k != 1) and args[i]._version == 0
        with torch.no_grad():
            optim.adamw_(*[[t] for t in args], step=1)
        assert (args[0] != 0).all() and args[0].requires_grad == (i == 0)
        between = args[i] * 1
        args = [t.detach() for t in args]
        args[i] = between                                                         # nor what was made of one
        with pytest.raises(RuntimeError, match="no_grad"):
            optim.adamw_(*[[t] for t in args], step=1)


def test_nothing_that_is_written_may_be_shared(optim):
    """Each refused call leaves all tensors alone; gradients may be shared among themselves."""
    import torch

    f = lambda n=256: torch.zeros(n, device="cuda")  # noqa: E731
    e = lambda n=256: torch.zeros(n, device="cuda").to(torch.float8_e4m3fn)  # noqa: E731
    s = lambda n=256: torch.full((n // 128, 2), 127, dtype=torch.uint8, device="cuda")  # noqa: E731
    one = torch.ones(256, device="cuda")
    x, y, z, t, u = f(), f(512), e(), e(512), s()
    cases = [([f(), f()], [one, one], [x, x], [f(), f()]), ([f(), f()], [one, one], [f(), f()], [x, x]), ([f()], [one], [x], [x]), ([x], [one], [x], [f()]), ([x], [one], [f()], [x]),
             ([f(), f()], [one, one], [x, f()], [f(), x]), ([f(), f()], [one, one], [y[:256], y[128:384]], [f(), f()]), ([y[:256]], [one], [f()], [y[255:511]]), ([x], [x], [f()], [f()]),
             ([f(), f()], [one, y[1:257]], [y[:256], f()], [f(), f()]), ([f(), f()], [one, one], [z, z], [e(), e()], [s(), s()]), ([f(), f()], [one, one], [e(), e()], [e(), e()], [u, u]),
             ([f(), f()], [one, one], [e(), t[:256]], [t[200:456], e()], [s(), s()])]
    for case in cases:
        with pytest.raises(ValueError, match="share memory"):
            optim.adamw_(*case, step=1)
    torch.cuda.synchronize()
    assert all((v.float() == 0).all() for v in (x, y, z, t)) and (u == 127).all()
    p, q = [f(), f()], [f(), f()]
    optim.adamw_(p, [one, one], [f(), f()], [f(), f()], step=1)
    optim.adamw_(q, [one, one.clone()], [f(), f()], [f(), f()], step=1)
    assert all((a == b).all() and (a != 0).all() for a, b in zip(p, q))
    buf = f(3 * 256)                                                              # neighbours share nothing
    optim.adamw_([buf[256:512]], [one], [buf[512:]], [buf[:256]], step=1)
    assert (buf[256:512] == p[0]).all() and (buf[512:] != 0).all() and (buf[:256] != 0).all()


def test_forward_mode_is_refused(optim):
    import torch
    import torch.autograd.forward_ad as forward

    z = lambda: torch.zeros(64, device="cuda")  # noqa: E731
    with forward.dual_level():
        for i in range(2):
            args = [[forward.make_dual(t, torch.ones_like(t)) if k == i else t] for k, t in enumerate((z(), z(), z(), z()))]
            with pytest.raises(RuntimeError, match="forward-mode"):
                optim.adamw_(*args, step=1)


def test_refusals(optim):
    import torch

    f = lambda n=256, t=torch.float32: torch.zeros(n, device="cuda", dtype=t)  # noqa: E731
    e = torch.float8_e4m3fn
    s = torch.full((2, 2), 127, dtype=torch.uint8, device="cuda")
    call = optim.adamw_
    p = f()
    for bad in (lambda: call([f()], [f()], [f()], [f()]), lambda: call([f()], [f()], [f()], [f()], step=0), lambda: call([f(), f()], [f()], [f()], [f()], step=1),
                lambda: call([f()], [f(255)], [f()], [f()], step=1), lambda: call([f()], [f()], [f(255)], [f()], step=1), lambda: call([f(512)[::2]], [f()], [f()], [f()], step=1),
                lambda: call([f()], [f(512)[::2]], [f()], [f()], step=1), lambda: call([f()], [f()], [f(256, e)], [f(256, e)], step=1),
                lambda: call([f()], [f()], [f(256, e)], [f(256, e)], [s[:1]], step=1), lambda: call([f()], [f()], [f(256, e)], [f(256, e)], [s.float()], step=1),
                lambda: call([f().cpu()], [f()], [f()], [f()], step=1), lambda: call([f()], [f().cpu()], [f()], [f()], step=1),
                lambda: call([p, p], [f(), f()], [f(), f()], [f(), f()], step=1), lambda: call([p[:200], p[100:]], [f(200), f(156)], [f(200), f(156)], [f(200), f(156)], step=1),
                lambda: call([f()], [f()], [f()], [f()], step=f(1)), lambda: call([f()], [f()], [f()], [f()], step=1, lr=f(2)), lambda: call([f()], [f()], [f()], [f()], step=1, grad_scale=f(2)),
                lambda: optim.moments(f(256, e), f(255, e), s), lambda: optim.moments(f(256, e), f(256, e), s[:1]), lambda: optim.AdamW([p.requires_grad_()], bits=4),
                lambda: optim.AdamW([p], betas=(0.9, 1.0)), lambda: optim.AdamW([p], lr=-1.0), lambda: optim.AdamW([p], lr=f(1))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: call([f(256, torch.half)], [f()], [f()], [f()], step=1), lambda: call([f()], [f(256, torch.half)], [f()], [f()], step=1), lambda: call([f()], [f()], [f()], [f(256, e)], step=1),
                lambda: call([f(), f(256, torch.bfloat16)], [f(), f()], [f(), f()], [f(), f()], step=1), lambda: call([f()], [f()], [f(256, torch.bfloat16)], [f()], step=1),
                lambda: call(f(), [f()], [f()], [f()], step=1), lambda: call([f()], [f()], [None], [f()], step=1), lambda: optim.moments(f(), f(), s)):
        with pytest.raises(TypeError):
            bad()
    from paper_2512_22804_b200.binding import MorError

    for kw in (dict(lr=-1.0), dict(beta1=1.0), dict(beta2=-0.5), dict(eps=float("nan")), dict(weight_decay=-0.1)):
        with pytest.raises(MorError):
            call([f()], [f()], [f()], [f()], step=1, **kw)

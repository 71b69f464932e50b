"""The norm, its gradient and its 8-bit output against the formulas in 64 bits.

h = x + residual is one addition in binary32 and one rounding: compared bit for bit.  u = 2^-24.  A row's sum of squares is taken in at most `depth` additions
from any element to the result, depth = max(32, columns / 1024) + 40 (a thread's own elements, then warps, then the CTA), so it is off by depth * u of itself, its
root by half of that; a division, a root, a multiplication by 1 / columns and two by the factors add 6 u.  So y in 32 bits is within
(depth / 2 + 6) u |y| of the formula, and its rounding adds half a step of its type.  The gradient's mean of g h is off by (depth + 6) u mean(|g h|).
Scales and codes are made from y in 32 bits: a scale is that of an amax within the same bound, a code is within half a distance of its neighbours.
"""
import math

import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def norm():
    from paper_2512_22804_b200 import norm

    return norm


def T(name):
    import torch

    return {"bf16": torch.bfloat16, "fp32": torch.float32}[name]


def half_step(v, dtype):
    import torch

    return v.abs() * torch.finfo(dtype).eps / 2 + (2.0 ** -134 if dtype == torch.bfloat16 else 2.0 ** -150)


def draw(rows, cols, x, r, w, seed=0):
    import torch

    g = torch.Generator(device="cuda").manual_seed(seed + rows * 131 + cols)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    gain = torch.where(torch.rand(cols, generator=g, device="cuda") < 0.02, 30.0, 1.0)
    return (n(rows, cols) * gain).to(T(x)), None if r is None else (3 * n(rows, cols)).to(T(r)), (1 + 0.2 * n(cols)).to(T(w))


def depth(cols):
    return max(32, cols / 1024) + 40


def formula(h, w, eps):
    h, w = h.double(), w.double()
    rs = 1 / (h.pow(2).mean(-1, keepdim=True) + eps).sqrt()
    return h * rs * w, rs


SHAPES = [(1, 1), (3, 7), (1, 4096), (5, 255), (2, 256), (9, 257), (17, 512), (33, 1000), (4, 1024), (7, 1025), (3, 2048), (301, 1500), (5, 4096), (2, 4097), (3, 8192), (2, 12001),
          (2, 16384), (2, 16385), (1, 40001), (1300, 64)]
TYPES = [("bf16", None, "bf16"), ("bf16", "bf16", "bf16"), ("bf16", "fp32", "fp32"), ("fp32", "fp32", "bf16"), ("fp32", "bf16", "fp32")]


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_norm(norm, rows, cols, types):
    x, r, w = draw(rows, cols, *types)
    got = norm.rms_norm(x, w, r, eps=1e-5)
    y, h = (got, x) if r is None else got
    if r is not None:
        assert h.dtype == r.dtype and (h == (x.float() + r.float()).to(r.dtype)).all()
    want, _ = formula(h, w, 1e-5)
    assert y.dtype == x.dtype and y.shape == x.shape
    assert ((y.double() - want).abs() <= (1 + 2 * U) * half_step(want, y.dtype) * (1 + 1e-4) + (depth(cols) / 2 + 6) * U * want.abs()).all()


def check_codes(codes, scales, y, block, kind):
    """Of one row-major matrix, y in 64 bits."""
    import torch

    rows, cols = y.shape
    rel = (depth(cols) / 2 + 6) * U
    n = cols if block is None else 128
    b = torch.nn.functional.pad(y, (0, -cols % n)).reshape(rows, -1, n)
    a = b.abs().amax(2)
    if kind == "e8m0":
        assert scales.dtype == torch.uint8
        fit = lambda a: torch.floor(torch.log2(448 / a.double())) + 127  # noqa: E731
        low, high = fit(a * (1 + rel)), fit(a * (1 - rel))
        s = scales.double()
        ok = ((s >= low) & (s <= high)) | ((a == 0) & (s == 127)) | (a == 0)
        assert ok.all()
        s = torch.exp2(s - 127)
    else:
        assert scales.dtype == torch.float32
        s = scales.double()
        assert ((s - 448 / a).abs() <= (rel * 1.01 + U) * 448 / a)[a > 0].all() and (s[a == 0] == 1).all()
    v = b * s.unsqueeze(2)
    d = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    c = torch.nn.functional.pad(codes.double(), (0, -cols % n)).reshape(rows, -1, n)
    off = (c - v).abs()
    near = d / 2 + 1.01 * rel * v.abs() + U * v.abs()                      # next to a power of two the distance above counts
    assert (off <= torch.maximum(near, torch.where(v.abs() >= d * 15.999, d, 0.0))).all()
    return s


@pytest.mark.parametrize("block,kind", [(128, "e8m0"), (128, "fp32"), (None, "e8m0"), (None, "fp32")])
@pytest.mark.parametrize("types", TYPES[:3])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantised(norm, rows, cols, types, block, kind):
    import torch

    x, r, w = draw(rows, cols, *types, seed=5)
    out = norm.rms_norm_quantize(x, w, r, eps=1e-5, block=block, scale=kind)
    h = x if r is None else out[2]
    if r is not None:
        assert (h == (x.float() + r.float()).to(r.dtype)).all()
    codes, scales = out[:2]
    assert codes.dtype == torch.float8_e4m3fn and codes.shape == x.shape and scales.shape == (rows, 1 if block is None else (cols + 127) // 128)
    y, _ = formula(h, w, 1e-5)
    s = check_codes(codes, scales, y, block, kind)
    for dtype in (torch.bfloat16, torch.float32):
        v = norm.dequantize(codes, scales, dtype)
        exact = codes.double() / s.repeat_interleave(cols if block is None else 128, 1)[:, :cols]
        assert v.dtype == dtype and (v == exact.float().to(dtype)).all()


def test_values_of_every_code_and_scales_of_any_size(norm):
    """Bit for bit the quotient in 32 bits, whatever the scale: random ones of every exponent, the ends of the range, zero, infinity."""
    import torch

    g = torch.Generator(device="cuda").manual_seed(31)
    codes = torch.arange(256, device="cuda", dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).repeat(4096, 1)
    scales = torch.exp2(torch.rand(4096, 1, generator=g, device="cuda", dtype=torch.float64) * 276 - 148).float()
    scales[:8, 0] = torch.tensor([0.0, float("inf"), 2.0 ** -149, 3.402823466e+38, 2.0 ** -100, 2.0 ** 100, 1.0, -3.0])
    want = codes.float() / scales
    for dtype in (torch.float32, torch.bfloat16):
        v, exact = norm.dequantize(codes, scales.expand(4096, 1), dtype), want.to(dtype)
        whole = torch.int32 if dtype == torch.float32 else torch.int16
        assert (exact.isnan() == v.isnan()).all() and ((v.view(whole) == exact.view(whole)) | exact.isnan()).all()


@pytest.mark.parametrize("block,kind", [(128, 1), (128, 2), (None, 1), (None, 2)])
def test_codes_are_those_of_the_analysis(norm, block, kind):
    """Rows of +-1 are normed to +-weight exactly (eps 0), a BF16 tensor that the analysis takes too: the codes and scales are the same bytes."""
    import torch

    from paper_2512_22804_b200 import binding as mb

    rows, cols = 64, 1040
    g = torch.Generator(device="cuda").manual_seed(3)
    sign = torch.where(torch.rand(rows, cols, generator=g, device="cuda") < 0.5, -1.0, 1.0).to(torch.bfloat16)
    w = torch.exp2(torch.randn(cols, generator=g, device="cuda") * 4).to(torch.bfloat16)
    w[::17] = 0
    codes, scales = norm.rms_norm_quantize(sign, w, eps=0.0, block=block, scale="e8m0" if kind == 1 else "fp32")
    y = (sign.float() * w.float()).to(torch.bfloat16)
    want = mb.analyze_quantize(y, mb.Recipe((1, 128) if block else (1, 0), (mb.MOR_FMT_E4M3, mb.MOR_FMT_BF16), mb.MOR_CRIT_TENSOR_MEAN_REL, scale_mode=kind))
    assert (codes.view(torch.uint8) & 127 == want.codes_view() & 127).all() and ((codes.float() != 0) <= (codes.view(torch.uint8) == want.codes_view())).all()
    assert (scales == (want.scale_e8m0 if kind == 1 else want.scale_f32).reshape(scales.shape)).all()


def gradients(norm, x, r, w, dy, dh, eps):
    import torch

    x, w = x.detach().requires_grad_(), w.detach().requires_grad_()
    if r is None:
        return torch.autograd.grad(norm.rms_norm(x, w, eps=eps), (x, w), dy) + (None,)
    r = r.detach().requires_grad_()
    out = norm.rms_norm(x, w, r, eps=eps)
    dx, dw, dr = torch.autograd.grad(out if dh is not None else out[0], (x, w, r), (dy, dh) if dh is not None else dy)
    return dx, dw, dr


@pytest.mark.parametrize("other", [True, False])
@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_gradient(norm, rows, cols, types, other):
    import torch

    x, r, w = draw(rows, cols, *types, seed=9)
    if r is None and other:
        pytest.skip("no sum without a residual")
    g = torch.Generator(device="cuda").manual_seed(1)
    dy = torch.randn(rows, cols, generator=g, device="cuda").to(x.dtype)
    dh = torch.randn(rows, cols, generator=g, device="cuda").to(r.dtype) if other else None
    dx, dw, dr = gradients(norm, x, r, w, dy, dh, 1e-5)
    h = x if r is None else (x.float() + r.float()).to(r.dtype)
    _, rs = formula(h, w, 1e-5)
    hd, gd = h.double(), dy.double() * w.double()
    xh = hd * rs
    mean, size = (gd * xh).mean(1, keepdim=True), (gd * xh).abs().mean(1, keepdim=True)
    want = rs * (gd - xh * mean)
    rel = (depth(cols) / 2 + 8) * U
    off = rs * (rel * (gd.abs() + 2 * xh.abs() * mean.abs()) + xh.abs() * (depth(cols) + 8) * U * size)
    if dh is not None:
        want = want + dh.double()
        off = off + U * (want.abs() + dh.double().abs())
    for got, like in ((dx, x),) + (((dr, r),) if r is not None else ()):
        assert got.dtype == like.dtype and got.shape == like.shape
        assert ((got.double() - want).abs() <= 1.01 * half_step(want, got.dtype) + off * 1.01).all()
    term = dy.double() * xh
    want = term.sum(0)
    assert dw.dtype == w.dtype
    assert ((dw.double() - want).abs() <= 1.01 * half_step(want, dw.dtype) + 1.01 * (rel + (rows + 24) * U) * term.abs().sum(0)).all()


def test_gradient_against_differences(norm):
    """The kernel's gradient, FP32, against central differences of the formula in 64 bits: with a step of 1e-5 those are good to 1e-9 of the values' size here, the
    kernel to some 1e-6."""
    import torch

    x, r, w = draw(6, 130, "fp32", "fp32", "fp32", seed=2)
    g = torch.Generator(device="cuda").manual_seed(4)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    dy, dh = n(6, 130), n(6, 130)
    dx, dw, dr = gradients(norm, x, r, w, dy, dh, 1e-5)

    def loss(x, r, w):
        h = x + r
        return float((formula(h, w, 1e-5)[0] * dy.double()).sum() + (h * dh.double()).sum())

    for i, got in enumerate((dx, dr, dw)):
        at = [t.double() for t in (x, r, w)]
        way = n(*at[i].shape).double()
        ends = []
        for sign in (1, -1):
            moved = list(at)
            moved[i] = at[i] + sign * 1e-5 * way
            ends.append(loss(*moved))
        slope = (ends[0] - ends[1]) / 2e-5
        assert abs(float((got.double() * way).sum()) - slope) <= 1e-5 * float((got.double() * way).abs().sum())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_any_strides_and_starts(norm, dtype):
    import torch

    base = torch.randn(40, 777, device="cuda").to(T(dtype))
    w = torch.randn(2 * 320, device="cuda").to(T(dtype))[::2]
    for x in (base[:, 1:321], base[3:, 5:325], base[::2, 8:328], base.t()[:40, :32].t()[:, :40].repeat(1, 8), base[:1, :320].expand(9, 320), base.t()[:320, :40].t()):
        r = x * 0.5
        wx = w[: x.shape[1]]
        y, h = norm.rms_norm(x, wx, r)
        y2, h2 = norm.rms_norm(x.contiguous(), wx.contiguous(), r.contiguous())
        assert (y == y2).all() and (h == h2).all()
        c, s, _ = norm.rms_norm_quantize(x, wx, r)
        c2, s2, _ = norm.rms_norm_quantize(x.contiguous(), wx.contiguous(), r.contiguous())
        assert (c.view(torch.uint8) == c2.view(torch.uint8)).all() and (s == s2).all()
        dy = torch.randn(x.shape[1], device="cuda").to(x.dtype).expand(x.shape)
        a = gradients(norm, x, r, wx, dy, None, 1e-6)
        b = gradients(norm, x.contiguous(), r.contiguous(), wx.contiguous(), dy.contiguous(), None, 1e-6)
        assert all((p == q).all() for p, q in zip(a, b))


def test_more_dimensions_and_none(norm):
    import torch

    x = torch.randn(3, 5, 77, device="cuda").to(torch.bfloat16)
    w = torch.randn(77, device="cuda").to(torch.bfloat16)
    y, h = norm.rms_norm(x, w, x)
    flat, _ = norm.rms_norm(x.reshape(15, 77), w, x.reshape(15, 77))
    assert y.shape == x.shape and (y.reshape(15, 77) == flat).all()
    codes, scales, _ = norm.rms_norm_quantize(x, w, x)
    assert codes.shape == x.shape and scales.shape == (3, 5, 1) and norm.dequantize(codes, scales).shape == x.shape
    assert norm.rms_norm(x[0, 0], w).shape == (77,) and (norm.rms_norm(x[0, 0], w) == norm.rms_norm(x[0], w)[0]).all()
    for shape in ((0, 77), (4, 0, 77), (5, 0)):
        e, we = torch.zeros(shape, device="cuda", dtype=torch.bfloat16), w[: shape[-1]]
        y, h = norm.rms_norm(e, we, e)
        assert y.shape == h.shape == shape
        codes, scales, h = norm.rms_norm_quantize(e, we, e)
        assert codes.shape == shape and scales.shape == shape[:-1] + ((shape[-1] + 127) // 128,) and norm.dequantize(codes, scales).shape == shape
        dx, dw, dr = gradients(norm, e, e, we, e, e, 1e-6)
        assert dx.shape == dr.shape == shape and (dw == 0).all()
    y = norm.rms_norm(x, w)
    y += 1                                                       # a result is nobody's view
    x2 = x.clone().requires_grad_()
    y = norm.rms_norm(x2, w)
    y += 1
    y.sum().backward()


def test_zeros_and_what_is_not_finite(norm):
    import torch

    x = torch.randn(8, 300, device="cuda")
    x[0] = 0
    x[1, 5], x[2, 7], x[3] = float("nan"), float("inf"), 3e38
    w = torch.ones(300, device="cuda")
    y = norm.rms_norm(x, w)
    assert (y[0] == 0).all() and y[1].isnan().all() and y[2, 7].isnan() and (y[2, :7] == 0).all() and (y[3] == 0).all() and y[4:].isfinite().all()
    assert norm.rms_norm(x, w, eps=0.0)[0].isnan().all()
    w[9], w[200] = float("nan"), float("inf")
    for kind in ("e8m0", "fp32"):
        codes, scales = norm.rms_norm_quantize(x, w, scale=kind)
        b = codes.view(torch.uint8)
        assert (b[1] == 0x7F).all() and (b[4:, 9] == 0x7F).all() and (b[4:, 200] & 0x7F == 0x7E).all()
        assert (b[0, :9] == 0).all() and (scales[0, 0] == (127 if kind == "e8m0" else 1)).all() and scales.float().isfinite().all()
        assert b[0, 200] == 0x7F                                 # zero times infinity


def test_repeated_captured_and_on_another_stream(norm):
    import torch

    x, r, w = draw(700, 1504, "bf16", "fp32", "bf16")
    dy, dh = torch.randn_like(x), torch.randn_like(r)
    first = gradients(norm, x, r, w, dy, dh, 1e-6)
    y, h = norm.rms_norm(x, w, r)
    codes, scales, _ = norm.rms_norm_quantize(x, w, r)
    for _ in range(3):
        assert all((a == b).all() for a, b in zip(first, gradients(norm, x, r, w, dy, dh, 1e-6)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = gradients(norm, x, r, w, dy, dh, 1e-6)
    side.synchronize()
    assert all((a == b).all() for a, b in zip(first, again))
    xs, rs = torch.zeros_like(x), torch.zeros_like(r)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ys, hs = norm.rms_norm(xs, w, rs)
        cs, ss, _ = norm.rms_norm_quantize(xs, w, rs)
        grads = gradients(norm, xs, rs, w, dy, dh, 1e-6)
    xs.copy_(x)
    rs.copy_(r)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert (ys == y).all() and (hs == h).all() and (cs.view(torch.uint8) == codes.view(torch.uint8)).all() and (ss == scales).all()
    assert all((a == b).all() for a, b in zip(first, grads))


def test_autograd(norm):
    import torch

    x, r, w = draw(4, 64, "fp32", "fp32", "fp32")
    for t in (x, r, w):
        t.requires_grad_()
    y, h = norm.rms_norm(x, w, r)
    (gx,) = torch.autograd.grad(h.sum(), x, retain_graph=True)           # h alone
    assert (gx == 1).all()
    (g,) = torch.autograd.grad(y.sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="differentiated twice"):
        g.sum().backward()
    y, h = norm.rms_norm(x, w, r)
    y.sum().backward()
    with pytest.raises(RuntimeError):
        y.sum().backward()                                               # its tensors are given back
    for t in norm.rms_norm_quantize(x, w, r)[2:]:
        with pytest.raises(RuntimeError, match="no gradient"):
            t.sum().backward()


def test_refusals(norm):
    import torch

    x, w = torch.zeros(4, 64, device="cuda", dtype=torch.bfloat16), torch.zeros(64, device="cuda", dtype=torch.bfloat16)
    for bad in (lambda: norm.rms_norm(x, w[:63]), lambda: norm.rms_norm(x, w, x[:3]), lambda: norm.rms_norm(x.cpu(), w), lambda: norm.rms_norm(x, w, eps=-1.0),
                lambda: norm.rms_norm(x, w, eps=float("nan")), lambda: norm.rms_norm_quantize(x, w, block=64), lambda: norm.rms_norm(x, w.cpu()), lambda: norm.rms_norm(x, w, x.cpu()),
                lambda: norm.dequantize(x.to(torch.float8_e4m3fn), torch.zeros(4, 2, device="cuda")), lambda: norm.dequantize(x.to(torch.float8_e4m3fn), torch.zeros(3, 1, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: norm.rms_norm(x.half(), w), lambda: norm.rms_norm(x, w.double()), lambda: norm.rms_norm(x, w, x.half()), lambda: norm.rms_norm(x),
                lambda: norm.rms_norm_quantize(x, w, scale=3), lambda: norm.dequantize(x, torch.zeros(4, 1, device="cuda")),
                lambda: norm.dequantize(x.to(torch.float8_e4m3fn), torch.zeros(4, 1, device="cuda", dtype=torch.bfloat16))):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(KeyError):
        norm.rms_norm_quantize(x, w, scale="e5m2")


@pytest.mark.parametrize("scale", ["e8m0", "fp32"])
def test_rows_without_columns_have_a_scale(norm, scale):
    """The largest magnitude of nothing is 0, whose scale is 1; the scales' memory held something else before."""
    import torch

    kind = torch.uint8 if scale == "e8m0" else torch.float32
    x = torch.zeros(700, 0, device="cuda", dtype=torch.bfloat16)
    for _ in range(3):
        junk = torch.full((700,), 7, device="cuda", dtype=kind)
        del junk
        codes, scales = norm.rms_norm_quantize(x, x[0], scale=scale, block=None)
        assert codes.shape == (700, 0) and scales.shape == (700, 1) and (scales == (127 if scale == "e8m0" else 1)).all()
        assert norm.dequantize(codes, scales).shape == (700, 0)
    assert norm.rms_norm_quantize(x, x[0], scale=scale)[1].shape == (700, 0)
    assert norm.rms_norm_quantize(x[:0], x[0], scale=scale, block=None)[1].shape == (0, 1)


@pytest.mark.parametrize("residual", ["bf16", "fp32"])
def test_an_unused_result_costs_nothing(norm, residual):
    """Gradients of y alone and of h alone are those with zeros for the other, and y alone fills and reads no such zeros: what the pass takes beyond its results is the
    workspace of the weight's gradient."""
    import torch

    x, r, w = draw(1000, 4096, "bf16", residual, "bf16")
    dy, dh = torch.randn(1000, 4096, device="cuda").to(T("bf16")), torch.randn(1000, 4096, device="cuda").to(T(residual))

    def grads(used, given):
        leaves = [t.detach().requires_grad_() for t in (x, w, r)]
        results = norm.rms_norm(*leaves)
        out = [results[i] for i in used]
        del results
        torch.cuda.synchronize()
        before = torch.cuda.memory_allocated()
        torch.cuda.reset_peak_memory_stats()
        g = torch.autograd.grad(out, leaves, given)
        return g, torch.cuda.max_memory_allocated() - before

    both, _ = grads((0, 1), (dy, torch.zeros_like(dh)))
    alone, most = grads((0,), (dy,))
    assert all((a == b).all() for a, b in zip(both, alone))
    made = sum(1000 * 4096 * t.element_size() for t in ((x,) if residual == "bf16" else (x, r)))
    assert most <= made + 148 * 4096 * 4 + 2 ** 20
    both, _ = grads((0, 1), (torch.zeros_like(dy), dh))
    alone, _ = grads((1,), (dh,))
    assert all((a == b).all() for a, b in zip(both, alone)) and (alone[1] == 0).all()


@pytest.mark.parametrize("residual", ["bf16", "fp32"])
def test_no_second_derivative_by_either_gradient(norm, residual):
    import torch

    x, r, w = draw(6, 64, "bf16", residual, "bf16")
    for i in range(2):
        given = [torch.ones(6, 64, device="cuda", dtype=T(t)) for t in ("bf16", residual)]
        given[i].requires_grad_()
        leaves = [t.detach().requires_grad_() for t in (x, w, r)]
        for g in torch.autograd.grad(norm.rms_norm(*leaves), leaves, given, create_graph=True):
            with pytest.raises(RuntimeError, match="differentiated twice"):
                torch.autograd.grad(g.sum(), given[i], allow_unused=True, retain_graph=True)


def test_forward_mode_is_refused(norm):
    """A dual tensor may not lose its tangent in silence, whether something else needs a gradient or not."""
    import torch
    import torch.autograd.forward_ad as forward

    from paper_2512_22804_b200 import experts

    x, r, w = draw(6, 64, "bf16", "fp32", "bf16")
    codes, scales = norm.rms_norm_quantize(x, w, scale="fp32")
    plan = experts.sort(torch.zeros(6, 1, dtype=torch.int32, device="cuda"), 1)
    with forward.dual_level():
        dual = lambda t: forward.make_dual(t, torch.ones_like(t))  # noqa: E731
        for call in (lambda: norm.rms_norm(dual(x), w), lambda: norm.rms_norm(x, dual(w)), lambda: norm.rms_norm(x, w, dual(r)), lambda: norm.rms_norm(dual(x), w.clone().requires_grad_()),
                     lambda: norm.rms_norm_quantize(dual(x), w), lambda: norm.rms_norm_quantize(x, w, dual(r)), lambda: norm.dequantize(codes, dual(scales)),
                     lambda: experts.gather(dual(x), plan), lambda: experts.combine(dual(x), plan)):
            with pytest.raises(RuntimeError, match="forward-mode"):
                call()
        assert (norm.rms_norm(x, w, r)[0] == norm.rms_norm(dual(x).detach(), w, r)[0]).all()

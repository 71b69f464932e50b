"""The norm, the adapters beside 4-bit projections and the optimizer together, as the example uses them: it runs, and its gradients and its step are those of the
operators called one by one."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("fp4_adapters_example", os.path.join(ROOT, "examples", "fp4_adapters.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("fmt", ["e4m3_16", "e8m0_32"])
def test_the_example_runs(example, fmt):
    losses, apart, size = example.run(steps=6, format=fmt)
    assert len(losses) == 6 and all(math.isfinite(v) for v in losses) and size > 0.0
    if fmt == "e8m0_32":            # no scale spans tokens, and a token's sums do not depend on the others'
        assert apart == 0.0


@pytest.mark.parametrize("tokens", [5, 700])
def test_gradients_and_step_are_those_of_the_operators(example, tokens):
    import torch

    from paper_2512_22804_b200 import adapters, fp4, norm, optim

    torch.manual_seed(3)
    fmt = "e8m0_32"
    block = example.Block(256, 512, 3, 8, fmt)
    with torch.no_grad():
        for b in (block.b_up, block.b_down):
            b.copy_(torch.randn_like(b) * 0.1)
    x = torch.randn(tokens, 256, device="cuda").to(torch.bfloat16).requires_grad_()
    h = torch.randn(tokens, 256, device="cuda").requires_grad_()
    ids = torch.randint(-1, 3, (tokens,), device="cuda", dtype=torch.int32)
    out, stream = block(x, h, ids)
    dout, dstream = torch.randn_like(out), torch.randn_like(stream)
    params = [block.gain, block.a_up, block.b_up, block.a_down, block.b_down]
    got = torch.autograd.grad((out, stream), [x, h] + params, (dout, dstream))

    def adapted(y, w, a, b):
        return adapters.add(fp4.matmul(fp4.quantize(y, fmt)[0], w), y, a, b, ids, 2.0)

    def back(y, w_t, a, b, dy):
        """Gradients of y, a and b: through the operand of the transpose, the adapters on top."""
        leaves = [t.detach().requires_grad_() for t in (y, a, b)]
        base = torch.zeros(y.shape[0], b.shape[1], device="cuda", dtype=torch.bfloat16)
        dy_y, da, db = torch.autograd.grad(adapters.add(base, *leaves, ids, 2.0), leaves, dy)
        through = fp4.matmul(fp4.quantize(dy, fmt)[0], w_t)
        return through, dy_y, da, db

    with torch.no_grad():
        y0, s0 = norm.rms_norm(x, block.gain, h)
        y1 = adapted(y0, block.up, block.a_up, block.b_up)
        y2 = torch.relu(y1) ** 2
        y3 = adapted(y2, block.down, block.a_down, block.b_down)
    assert (out == y3).all() and (stream == s0).all()
    through, on_top, da_down, db_down = back(y2, block.down_t, block.a_down, block.b_down, dout)
    assert (got[5] == da_down).all() and (got[6] == db_down).all()
    # the layer adds the adapters' part in 32 bits and rounds once: here that part is rounded too.  A rounding to BF16 is off by 2^-8 of the value at most (half
    # of eps, 2^-7), so by two such of the magnitudes' sum together
    near = lambda a, b: (a.float() - b.float()).abs() <= 2.01 * 2.0 ** -8 * (through.float().abs() + on_top.float().abs()) + 1e-30  # noqa: E731
    leaf = y2.detach().requires_grad_()
    z = adapters.linear(leaf, block.down, block.a_down.detach(), block.b_down.detach(), ids, 2.0, w_t=block.down_t)
    (dy2,) = torch.autograd.grad(z, leaf, dout)
    assert near(dy2, through.float() + on_top.float()).all()
    y1g = y1.detach().requires_grad_()
    (dy1,) = torch.autograd.grad(torch.relu(y1g) ** 2, y1g, dy2)
    leaf = [t.detach().requires_grad_() for t in (y0, block.a_up, block.b_up)]
    z = adapters.linear(leaf[0], block.up, leaf[1], leaf[2], ids, 2.0, w_t=block.up_t)
    dy0, da_up, db_up = torch.autograd.grad(z, leaf, dy1)
    assert (got[3] == da_up).all() and (got[4] == db_up).all()
    leaf = [t.detach().requires_grad_() for t in (x, block.gain, h)]
    dx, dgain, dh = torch.autograd.grad(norm.rms_norm(*leaf), leaf, (dy0, dstream))
    assert (got[0] == dx).all() and (got[1] == dh).all() and (got[2] == dgain).all()

    before = [p.detach().clone() for p in params]
    optimizer = optim.AdamW(params, lr=1e-2, bits=8, weight_decay=0.1, seed=5)
    for p, g in zip(params, got[2:]):
        p.grad = g
    optimizer.step()
    state = [optimizer._new_state(p, 8) for p in before]
    optim.adamw_(before, list(got[2:]), [s["exp_avg"] for s in state], [s["exp_avg_sq"] for s in state], [s["scales"] for s in state], step=1, lr=1e-2, weight_decay=0.1, seed=5)
    assert all((p == q).all() for p, q in zip(params, before))
    fp4.check()

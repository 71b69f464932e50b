"""4-bit operators and row movers on matrices of more than 2^31 elements: the last rows and columns are right."""
import numpy as np
import pytest

from tests import plain_fp4 as plain

pytestmark = pytest.mark.gpu


def room(gigabytes):
    import torch

    if torch.cuda.mem_get_info()[0] < gigabytes * 2 ** 30:
        pytest.skip(f"needs {gigabytes} GiB of device memory")


@pytest.mark.parametrize("fmt", ["e4m3_16", "e8m0_32"])
def test_quantise_and_back(fmt):
    import torch

    from paper_2512_22804_b200 import fp4

    room(40)
    rows, cols = 66000, 33000                                        # 2.18e9 elements
    x = torch.empty(rows, cols, device="cuda", dtype=torch.bfloat16)
    g = torch.Generator(device="cuda").manual_seed(3)
    for i in range(0, rows, 6000):
        x[i:i + 6000] = torch.randn(x[i:i + 6000].shape, generator=g, device="cuda")
    r, c = fp4.quantize(x, fmt, cols=True)
    amax = float(x.abs().max())
    assert r.tensor_scale.item() == (1.0 if fmt == "e8m0_32" else np.float32(amax) * (np.float32(1) / np.float32(2688)))
    tail = x[-300:].float().cpu().numpy()
    want = plain.values(*plain.quantize(tail, fmt, amax), fmt)
    v = fp4.dequantize(r)
    assert np.array_equal(v[-300:].float().cpu().numpy(), plain.bf16(want.astype(np.float32)))
    del v, r
    tail = np.ascontiguousarray(x[:, -300:].float().cpu().numpy().T)
    want = plain.values(*plain.quantize(tail, fmt, amax), fmt)
    v = fp4.dequantize(c)
    assert np.array_equal(v[-300:].float().cpu().numpy(), plain.bf16(want.astype(np.float32)))


def test_product():
    import torch

    from paper_2512_22804_b200 import fp4

    room(20)
    m, n, k = 66000, 33000, 96
    a, b = (torch.randn(s, k, device="cuda").to(torch.bfloat16) for s in (m, n))
    qa, qb = (fp4.quantize(t, "e8m0_32")[0] for t in (a, b))
    y = fp4.matmul(qa, qb)
    fp4.check()
    va, vb = (plain.values(*plain.quantize(t[-200:].float().cpu().numpy(), "e8m0_32"), "e8m0_32") for t in (a, b))
    want = va @ vb.T
    slack = np.abs(va) @ np.abs(vb).T * 2.0 ** -16
    got = y[-200:, -200:].float().cpu().numpy()
    assert (plain.bf16((want - slack).astype(np.float32)) <= got).all() and (got <= plain.bf16((want + slack).astype(np.float32))).all()


def test_row_movers():
    import torch

    from paper_2512_22804_b200 import experts

    room(30)
    tokens, top, hidden, n = 35000, 4, 16384, 8                      # 140000 sorted rows: 2.29e9 elements
    ids = torch.arange(tokens * top, device="cuda", dtype=torch.int32).view(tokens, top) % n
    plan = experts.sort(ids, n)
    x = torch.randn(tokens, hidden, device="cuda", dtype=torch.bfloat16)
    xs = experts.gather(x, plan)
    slot = plan.slot[-500:].long()
    assert torch.equal(xs[-500:], x[slot // top])
    assert torch.equal(experts.combine(xs, plan).float(), (4 * x.float()).to(torch.bfloat16).float())
    w = torch.ones(tokens, top, device="cuda")
    dys, dw = experts.combine_grad(x, xs, plan, w)
    assert torch.equal(dys[-500:], xs[-500:])
    assert torch.allclose(dw[-300:], (x[-300:].float() ** 2).sum(1, keepdim=True).expand(-1, 4), rtol=2e-3)

"""The plain statements that the 4-bit and routing tests compare with are themselves tested, on the CPU."""
import numpy as np
import pytest
import torch

from tests import plain_fp4 as plain


def test_scale_codes_are_those_of_the_format():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(plain.E4M3, t.astype(np.float64), equal_nan=True)


def test_nearest_even_on_every_midpoint():
    for table in (plain.GRID, plain.E4M3[:127]):
        mid = (table[:-1] + table[1:]) / 2
        i = np.arange(len(mid))
        assert np.array_equal(plain.nearest_even(mid, table), np.where(i % 2 == 0, i, i + 1))
        assert np.array_equal(plain.nearest_even(np.nextafter(mid, 0), table), i)
        assert np.array_equal(plain.nearest_even(np.nextafter(mid, np.inf), table), i + 1)
        assert np.array_equal(plain.nearest_even(table, table), np.arange(len(table)))
        assert plain.nearest_even(np.array([1e30]), table)[0] == len(table) - 1


def test_bf16_rounding_is_torchs():
    x = np.random.default_rng(0).standard_normal(10000).astype(np.float32) * np.float32(7)
    x = np.concatenate([x, np.array([0, -0.0, 1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8], np.float32)])
    assert np.array_equal(plain.bf16(x), torch.from_numpy(x).to(torch.bfloat16).float().numpy())


@pytest.mark.parametrize("fmt", ["e4m3_16", "e8m0_32"])
def test_values_are_near_what_was_quantised(fmt):
    """No value is further off than half the widest gap of its block's grid (and what saturation cuts): a code's step is at
    most 2 below 6 steps of the scale, and the scale itself is at most a/6 rounded up by 2^-4 (E4M3), or more than a/8 (E8M0)."""
    x = plain.bf16(np.random.default_rng(1).standard_normal((50, 330)).astype(np.float32))
    v = plain.values(*plain.quantize(x, fmt), fmt)
    n = plain.BLOCK[fmt]
    a = np.zeros((50, -(-330 // n) * n))
    a[:, :330] = np.abs(x)
    a = np.repeat(a.reshape(50, -1, n).max(-1), n, axis=1)[:, :330]
    room = a / 6 * (1 + 2.0 ** -4) if fmt == "e4m3_16" else a / 4
    assert (np.abs(v - x) <= room + 1e-12).all()
    assert np.sqrt(((v - x) ** 2).mean() / (x.astype(np.float64) ** 2).mean()) < 0.2


def test_packing_and_tiles():
    c = np.arange(3 * 5, dtype=np.uint8).reshape(3, 5) % 16
    p = plain.packed(c)
    assert p.shape == (3, 16) and p[0, 0] == c[0, 0] | c[0, 1] << 4 and p[2, 2] == c[2, 4] and not p[:, 3:].any()
    b = np.arange(130 * 5, dtype=np.int64).reshape(130, 5) % 251
    t = plain.tiled(b.astype(np.uint8)).reshape(2, 2, 32, 4, 4)
    for r, k in ((0, 0), (1, 4), (33, 3), (127, 2), (128, 0), (129, 4)):
        assert t[r // 128, k // 4, r % 32, r % 128 // 32, k % 4] == b[r, k]


def test_sort_by_hand():
    starts, row, slot = plain.sort([[2, 0], [-1, 2], [0, 5]], 3, 4)
    assert starts.tolist() == [0, 4, 4, 8]
    assert row.tolist() == [[4, 0], [-1, 5], [1, -1]]
    assert slot.tolist() == [1, 4, -1, -1, 0, 3, -1, -1, -1, -1, -1, -1]

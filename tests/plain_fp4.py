"""Plain statements of the 4-bit formats, the products and the routing, for the tests: NumPy on the CPU, one step of the
definition at a time.  The quantiser takes its steps in binary32 where the definition says so; products and sums are in
64 bits.  Nothing here is shared with the CUDA library."""
import numpy as np

GRID = np.array([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=np.float64)
BLOCK = {"e4m3_16": 16, "e8m0_32": 32}
F = np.float32


def e4m3_values():
    """Value of every E4M3 code (NaN at 0x7F and 0xFF) from its fields."""
    v = np.empty(256)
    for c in range(256):
        s, e, m = c >> 7, (c >> 3) & 15, c & 7
        a = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        v[c] = np.nan if c & 127 == 127 else (-a if s else a)
    return v


E4M3 = e4m3_values()


def nearest_even(v, table):
    """Index of the entry of the ascending table nearest to each v >= 0; ties to the even index; the last from its midpoint up."""
    hi = np.clip(np.searchsorted(table, v), 1, len(table) - 1)
    lo = hi - 1
    dl, dh = v - table[lo], table[hi] - v
    return np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)


def quantize(x, fmt, amax=None):
    """(codes 0..15 [rows, cols], scale bytes [rows, blocks], tensor scale) of FP32 values [rows, cols], blocks along cols."""
    x = np.asarray(x, dtype=F)
    rows, cols = x.shape
    n = BLOCK[fmt]
    blocks = -(-cols // n)
    p = np.zeros((rows, blocks * n), F)
    p[:, :cols] = x
    b = p.reshape(rows, blocks, n)
    finite = np.isfinite(b)
    bad = ~finite.all(-1)
    mag = np.where(finite, np.abs(b), F(0))
    a = np.where(bad, F(0), mag.max(-1, initial=0))
    if fmt == "e8m0_32":
        with np.errstate(divide="ignore"):
            e = np.where(a > 0, np.floor(np.log2(np.maximum(a, F(2.0 ** -149)).astype(np.float64))), -300) - 2
        e = np.clip(e, -127, 127).astype(int)
        byte = np.where(bad, 255, e + 127).astype(np.uint8)
        y = np.where(bad[..., None], 0, b.astype(np.float64)) * (2.0 ** -e.astype(np.float64))[..., None]
        t = F(1)
    else:
        top = mag.max(initial=0) if amax is None else amax
        top = max(F(top), F(2.0 ** -88))
        t = F(top) * (F(1) / F(2688))
        s = (a.astype(F) * F(448 / 65536)) / (F(top) * F(2.0 ** -16))
        code = nearest_even(np.minimum(s, F(448)).astype(np.float64), E4M3[:127]).astype(np.uint8)
        byte = np.where(bad, 127, code).astype(np.uint8)
        sv = E4M3[code].astype(F)
        with np.errstate(divide="ignore"):
            q = np.where(sv == 0, F(0), F(1) / (sv * t))
        with np.errstate(invalid="ignore", over="ignore"):
            y = np.where(bad[..., None], F(0), b) * q[..., None]
    c = nearest_even(np.abs(y).astype(np.float64), GRID).astype(np.uint8) + np.where(np.signbit(y) & ~bad[..., None], 8, 0).astype(np.uint8)
    return c.reshape(rows, -1)[:, :cols], byte, t


def values(codes, byte, t, fmt):
    """What codes, scale bytes and tensor scale stand for: binary32 products as the definition has them, in 64 bits."""
    n = BLOCK[fmt]
    g = np.concatenate([GRID, -GRID])[codes]
    s = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127)) if fmt == "e8m0_32" else E4M3[byte]
    s = np.repeat(s, n, axis=1)[:, :codes.shape[1]]
    return ((g * s).astype(F) * F(t)).astype(np.float64)


def packed(codes):
    """Two codes to a byte, rows padded with zeros to a multiple of 16 bytes."""
    rows, cols = codes.shape
    p = np.zeros((rows, -(-cols // 32) * 32), np.uint8)
    p[:, :cols] = codes
    return p[:, 0::2] | (p[:, 1::2] << 4)


def tiled(byte):
    """Scale bytes [rows, blocks] in tiles of 128 x 4, zeros where there is no block."""
    rows, blocks = byte.shape
    rt, kt = -(-rows // 128), -(-blocks // 4)
    out = np.zeros((rt, kt, 512), np.uint8)
    for r in range(rows):
        k = np.arange(blocks)
        out[r // 128, k // 4, (r % 32) * 16 + (r // 32 % 4) * 4 + k % 4] = byte[r]
    return out.reshape(-1)


def bf16(x):
    """Values rounded to BF16 (nearest even), as FP32."""
    u = np.asarray(x, dtype=F).view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16 << 16).astype(np.uint32)
    return np.where(np.isnan(x), F(np.nan), r.view(F))


def sort(ids, experts, align):
    """(starts, row of each slot, slot of each row) by walking the slots in order."""
    flat = [int(i) for i in np.asarray(ids).reshape(-1)]
    counts = [0] * experts
    for i in flat:
        if 0 <= i < experts:
            counts[i] += 1
    starts = [0]
    for c in counts:
        starts.append(starts[-1] + -(-c // align) * align)
    capacity = (len(flat) + min(len(flat), experts) * (align - 1)) // align * align
    row, slot, nxt = [-1] * len(flat), [-1] * capacity, list(starts)
    for s, i in enumerate(flat):
        if 0 <= i < experts:
            row[s] = nxt[i]
            slot[nxt[i]] = s
            nxt[i] += 1
    return np.array(starts), np.array(row, dtype=np.int64).reshape(np.shape(ids)), np.array(slot, dtype=np.int64)

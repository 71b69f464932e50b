"""What is measured of the 4-bit operators and of the routing that feeds them.

Three operators, alone and as a linear layer or an expert layer uses them:

* ``quantize``  a tensor to microscaled E2M1 codes along its rows (and columns), and the values those codes stand for
* ``linear``    y = Q(x) Q(w)^T with 4-bit operands; training adds dx = Q(dy) Q(w^T)^T and dw = Q(dy^T) Q(x^T)^T
* ``route``     tokens sorted by expert, gathered, brought back with weights applied; training adds the gradients
* ``experts``   all of it: the tokens of each expert through that expert's 4-bit weight matrix and back

Formats.  "e8m0_32": blocks of 32, scale 2^e with e = floor(log2 a) - 2 held to -127..127, a the block's largest magnitude.
"e4m3_16": blocks of 16; with A the tensor's largest magnitude (at least 2^-88), tensor scale t = A / 2688 and block scale
s = E4M3(448 a / A), value = code * s * t.  Codes are E2M1 (0, .5, 1, 1.5, 2, 3, 4, 6 and their negatives), rounded to
nearest even and saturated, two to a byte with the even element in the low half.  Block scales are stored in tiles of 128 rows x
4 blocks, 512 bytes each: byte ``(row % 32) * 16 + (row // 32 % 4) * 4 + block % 4``.
"""
import math

import torch

own = False

BLOCK = {"e8m0_32": 32, "e4m3_16": 16}
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
MIDS = (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ------------------------------------------------------------------------------------------------ cases ----

def listed():
    return [
        # one token's activation on its way into a 4-bit linear layer
        {"name": "quantize_one_row", "op": "quantize", "rows": 1, "cols": 4096, "fmt": "e8m0_32", "both": False, "dtype": "bf16"},
        # a gradient accumulated in 32 bits, of a ragged batch and an odd width, for both products of the backward pass
        {"name": "quantize_ragged_both", "op": "quantize", "rows": 1003, "cols": 4099, "fmt": "e4m3_16", "both": True, "dtype": "fp32"},
        # the widest activation of a layer (8192 tokens, FFN 14336), both directions for the training step
        {"name": "quantize_large_both", "op": "quantize", "rows": 8192, "cols": 14336, "fmt": "e4m3_16", "both": True, "dtype": "bf16"},
        # decoding: one token through the up projection, activation range known from calibration
        {"name": "linear_one_token", "op": "linear", "tokens": 1, "n_in": 4096, "n_out": 14336, "fmt": "e4m3_16", "train": False},
        # decoding for a small batch of sequences through the down projection
        {"name": "linear_48_tokens", "op": "linear", "tokens": 48, "n_in": 14336, "n_out": 4096, "fmt": "e8m0_32", "train": False},
        # prefill of a long prompt through the up projection
        {"name": "linear_prefill", "op": "linear", "tokens": 8192, "n_in": 4096, "n_out": 14336, "fmt": "e4m3_16", "train": False},
        # a training step of the output projection: three products, three tensors quantised both ways
        {"name": "linear_train", "op": "linear", "tokens": 8192, "n_in": 4096, "n_out": 4096, "fmt": "e8m0_32", "train": True},
        # the same with sizes that are multiples of nothing: packed sequences, a pruned width
        {"name": "linear_train_ragged", "op": "linear", "tokens": 1187, "n_in": 1500, "n_out": 2731, "fmt": "e4m3_16", "train": True},
        # decoding: one token spread over 8 of 128 experts and back
        {"name": "route_one_token", "op": "route", "tokens": 1, "top": 8, "experts": 128, "hidden": 4096, "train": False},
        # a training step's dispatch, combine and both gradients
        {"name": "route_train", "op": "route", "tokens": 8192, "top": 4, "experts": 64, "hidden": 4096, "train": True},
        # decoding for a small batch through an expert layer: most experts see one token or none
        {"name": "experts_32_tokens", "op": "experts", "tokens": 32, "top": 4, "experts": 32, "n_in": 2048, "n_out": 1024,
         "fmt": "e4m3_16", "train": False},
        # a training step of an expert layer
        {"name": "experts_train", "op": "experts", "tokens": 8192, "top": 4, "experts": 32, "n_in": 2048, "n_out": 1024,
         "fmt": "e8m0_32", "train": True},
    ]


def _log(rng, lo, hi):
    """A whole number, uniform in its logarithm; every second one is brought to a multiple of 8 or 128, as most real sizes are."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    m = rng.choice((1, 1, 8, 128))
    return max(lo, min(hi, (v + m - 1) // m * m))


def draw(rng):
    op = rng.choice(("quantize", "linear", "linear", "route", "experts"))
    fmt = rng.choice(("e8m0_32", "e4m3_16"))
    if op == "quantize":
        return {"op": op, "rows": _log(rng, 1, 8192), "cols": _log(rng, 32, 14336), "fmt": fmt, "both": rng.random() < 0.5,
                "dtype": rng.choice(("bf16", "bf16", "fp32"))}
    if op == "linear":
        train = rng.random() < 0.5
        return {"op": op, "tokens": _log(rng, 64 if train else 1, 8192), "n_in": _log(rng, 256, 4096), "n_out": _log(rng, 256, 4096 if train else 14336),
                "fmt": fmt, "train": train}
    if op == "route":
        experts = _log(rng, 4, 128)
        return {"op": op, "tokens": _log(rng, 1, 8192), "top": rng.randint(1, 4), "experts": experts, "hidden": _log(rng, 256, 4096),
                "train": rng.random() < 0.5}
    return {"op": op, "tokens": _log(rng, 1, 8192), "top": rng.randint(1, 4), "experts": _log(rng, 4, 32), "n_in": _log(rng, 256, 2048),
            "n_out": _log(rng, 256, 1024), "fmt": fmt, "train": rng.random() < 0.5}


# ----------------------------------------------------------------------------------------------- inputs ----

def _activation(g, rows, cols):
    """Heavy-tailed values with a few outlier channels."""
    x = torch.randn(rows, cols, generator=g, device="cuda") / (0.5 + 0.5 * torch.rand(rows, 1, generator=g, device="cuda"))
    gain = torch.where(torch.rand(cols, generator=g, device="cuda") < 0.004, 30.0, 1.0)
    return (x * gain).to(torch.bfloat16)


def _gradient(g, rows, cols):
    """Signed magnitudes over many binades, 5 % exact zeros."""
    m = torch.exp2((torch.randn(rows, cols, generator=g, device="cuda") * 3.0 - 13.0).clamp_(-30.0, 4.0))
    u = torch.rand(rows, cols, generator=g, device="cuda")
    return torch.where(u < 0.05, 0.0, torch.where(u < 0.525, -m, m))


def _weight(g, *shape):
    return (torch.randn(*shape, generator=g, device="cuda") * 0.02).to(torch.bfloat16)


def _routing(g, tokens, top, experts):
    """Expert ids and weights per token: some experts are popular, an eighth of the tokens is masked (no expert at all)."""
    score = torch.randn(tokens, experts, generator=g, device="cuda") + torch.randn(1, experts, generator=g, device="cuda")
    best, ids = torch.topk(score, top, dim=1)
    weight = torch.softmax(best, dim=1)
    if tokens > 1:
        ids = torch.where(torch.rand(tokens, 1, generator=g, device="cuda") < 0.125, -1, ids)
    return ids.to(torch.int32), weight


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    op = case["op"]
    if op == "quantize":
        x = _gradient(g, case["rows"], case["cols"]) if case["dtype"] == "fp32" else _activation(g, case["rows"], case["cols"])
        s["x"] = x.to(DTYPES[case["dtype"]])
        return s
    if op == "linear":
        s["x"] = _activation(g, case["tokens"], case["n_in"])
        w = _weight(g, case["n_out"], case["n_in"])
        if case["train"]:
            s["w"] = w
            s["dy"] = _gradient(g, case["tokens"], case["n_out"]).to(torch.bfloat16)
        else:
            s["w"] = _stored(w, case["fmt"])
            s["amax"] = s["x"].float().abs().max().reshape(1) * 0.9      # a calibrated range: the largest values saturate
        return s
    s["ids"], s["weight"] = _routing(g, case["tokens"], case["top"], case["experts"])
    if op == "route":
        rows = case["tokens"] * case["top"]
        s["x"] = _activation(g, case["tokens"], case["hidden"])
        s["ys"] = _activation(g, rows, case["hidden"])                   # what the experts gave back for the sorted rows
        if case["train"]:
            s["dy"] = _gradient(g, case["tokens"], case["hidden"]).to(torch.bfloat16)
            s["dxs"] = _gradient(g, rows, case["hidden"]).to(torch.bfloat16)
        return s
    s["weight"] = s["weight"].to(torch.bfloat16)                         # the router of a BF16 model hands over BF16
    s["x"] = _activation(g, case["tokens"], case["n_in"])
    w = _weight(g, case["experts"], case["n_out"], case["n_in"])
    if case["train"]:
        s["w"] = w
        s["dy"] = _gradient(g, case["tokens"], case["n_out"]).to(torch.bfloat16)
    else:
        s["w"] = _stored(w, case["fmt"])
    return s


# ------------------------------------------------------------------------------------------ plain forms ----

def _blocks(x, n):
    """[..., cols] as [..., blocks, n], zero-filled."""
    x = torch.nn.functional.pad(x, (0, -x.shape[-1] % n))
    return x.unflatten(-1, (-1, n))


def _e2m1_index(y):
    """Index into GRID of the nearest value; ties go to the even index, everything from 5 up saturates to 6."""
    a = y.abs()
    i = (a > MIDS[0]).to(torch.uint8)
    i += a >= MIDS[1]
    i += a > MIDS[2]
    i += a >= MIDS[3]
    i += a > MIDS[4]
    i += a >= MIDS[5]
    i += a > MIDS[6]
    return i


def _quantise(x, fmt, amax=None):
    """(index, negative, block scale, tensor scale) of 32-bit values, blocks along the last axis."""
    b = _blocks(x, BLOCK[fmt])
    a = b.abs().amax(-1, keepdim=True)
    if fmt == "e8m0_32":
        e = (torch.frexp(a).exponent - 3).clamp(-127, 127)
        e = torch.where(a == 0, -127, e)
        one = torch.ones_like(a)
        s, t = torch.ldexp(one, e), torch.ones(1, device=x.device)
        y = b * torch.ldexp(one, -e)
    else:
        amax = x.abs().max() if amax is None else amax
        amax = amax.float().clamp(min=2.0 ** -88).reshape(1)
        t = amax / 2688.0
        s = ((a * (448.0 / 65536)) / (amax * (1.0 / 65536))).clamp(max=448.0).to(torch.float8_e4m3fn).float()
        y = b * torch.where(s == 0, 0.0, 1.0 / (s * t))
    return _e2m1_index(y), torch.signbit(b), s, t


def _values(index, negative, s, t, cols):
    """What codes and scales stand for, in 32 bits."""
    v = torch.tensor(GRID, device=s.device)[index.int()]
    return ((torch.where(negative, -v, v) * s) * t).flatten(-2)[..., :cols]


def _fake(x, fmt, amax=None):
    """Quantised along the last axis and back."""
    return _values(*_quantise(x.float(), fmt, amax), x.shape[-1])


def _tiles(s):
    """Block scales [..., rows, blocks] (bytes) in tiles of 128 x 4."""
    s = torch.nn.functional.pad(s, (0, -s.shape[-1] % 4, 0, -s.shape[-2] % 128))
    s = s.unflatten(-1, (-1, 4)).unflatten(-3, (-1, 4, 32))              # [..., row tile, 4, 32, block tile, 4]
    return s.movedim(-2, -4).transpose(-2, -3).contiguous()              # [..., row tile, block tile, 32, 4, 4]


def _untiled(tiles, rows, blocks):
    s = tiles.transpose(-2, -3).movedim(-4, -2)
    return s.flatten(-2).flatten(-4, -2)[..., :rows, :blocks]


def _stored(w, fmt):
    """A weight as a serving program keeps it: packed codes [..., rows, bytes], tiled block scales, tensor scale."""
    index, negative, s, t = _quantise(w.float(), fmt)
    code = (index + 8 * negative.to(torch.uint8)).flatten(-2)
    code = torch.nn.functional.pad(code, (0, -code.shape[-1] % 32))
    codes = code[..., 0::2] + 16 * code[..., 1::2]
    if fmt == "e8m0_32":
        b = (torch.frexp(s).exponent + 126).to(torch.uint8)
    else:
        b = s.to(torch.float8_e4m3fn).view(torch.uint8)
    return {"codes": codes.contiguous(), "scales": _tiles(b.squeeze(-1)), "tensor_scale": t, "rows": w.shape[-2], "cols": w.shape[-1]}


def _decoded(w, fmt):
    """The values of _stored()'s weight in 32 bits."""
    c = torch.stack((w["codes"] & 15, w["codes"] >> 4), -1).flatten(-2)
    n = -(-w["cols"] // BLOCK[fmt])
    s = _untiled(w["scales"], w["rows"], n)
    s = torch.ldexp(torch.ones(s.shape, device=s.device), s.int() - 127) if fmt == "e8m0_32" else s.view(torch.float8_e4m3fn).float()
    c = c[..., :n * BLOCK[fmt]].unflatten(-1, (n, BLOCK[fmt]))
    return _values(c & 7, c >= 8, s.unsqueeze(-1), w["tensor_scale"], w["cols"])


def _sorted_rows(ids, experts, align):
    """(starts [experts + 1], row of each slot or -1, slot of each row or -1) of slots sorted by expert, each expert's rows
    starting at a multiple of `align`."""
    flat = ids.reshape(-1).long()
    flat = torch.where((flat >= 0) & (flat < experts), flat, experts)
    order = torch.argsort(flat, stable=True)
    counts = torch.zeros(experts + 1, dtype=torch.long, device=ids.device).scatter_add_(0, flat, torch.ones_like(flat))
    padded = (counts[:experts] + align - 1) // align * align
    zero = torch.zeros(1, dtype=torch.long, device=ids.device)
    starts, plain = torch.cat((zero, padded.cumsum(0))), torch.cat((zero, counts.cumsum(0)))
    at = torch.empty_like(flat)
    at[order] = torch.arange(flat.numel(), device=ids.device)
    row = torch.where(flat < experts, starts[flat] + at - plain[flat], -1)
    capacity = _capacity(ids.numel(), experts, align)
    slot = torch.full((capacity + 1,), -1, dtype=torch.long, device=ids.device)
    slot[torch.where(row < 0, capacity, row)] = torch.arange(flat.numel(), device=ids.device)
    return starts, row.reshape(ids.shape), slot[:capacity]


def _capacity(slots, experts, align):
    """Rows that `slots` slots can take at most: each of up to min(slots, experts) experts may leave align - 1 empty."""
    return (slots + min(slots, experts) * (align - 1)) // align * align


def _gathered(x, slot, top, weight=None):
    """Sorted rows of x in 32 bits (zero where a row has no slot)."""
    r = x.float()[(slot // top).clamp(min=0)]
    if weight is not None:
        r = r * weight.float().reshape(-1)[slot.clamp(min=0)].unsqueeze(1)
    return torch.where((slot >= 0).unsqueeze(1), r, 0.0)


def _taken(ys, row):
    """[tokens, top, n]: each slot's row of ys in 32 bits (zero where it has none)."""
    return torch.where((row >= 0).unsqueeze(-1), ys.float()[row.clamp(min=0)], 0.0)


def _tile_expert(starts, rows):
    """Expert of each tile of 128 sorted rows; tiles past the last row count to the last expert (their rows are zero)."""
    at = torch.arange(rows // 128, device=starts.device) * 128
    return (torch.searchsorted(starts, at, right=True) - 1).clamp(max=starts.numel() - 2)


def _plain(s):
    op, bf16 = s["op"], torch.bfloat16
    if op == "quantize":
        out = {"rows": _fake(s["x"], s["fmt"]).to(bf16)}
        if s["both"]:
            out["cols"] = _fake(s["x"].t(), s["fmt"]).to(bf16)
        return out
    if op == "linear":
        fmt, x = s["fmt"], s["x"]
        if not s["train"]:
            return {"y": (_fake(x, fmt, s["amax"]) @ _decoded(s["w"], fmt).t()).to(bf16)}
        w, dy = s["w"], s["dy"]
        return {"y": (_fake(x, fmt) @ _fake(w, fmt).t()).to(bf16),
                "dx": (_fake(dy, fmt) @ _fake(w.t(), fmt).t()).to(bf16),
                "dw": (_fake(dy.t(), fmt) @ _fake(x.t(), fmt).t()).to(bf16)}
    if op == "route":
        starts, row, slot = _sorted_rows(s["ids"], s["experts"], 1)
        out = {"starts": starts.int(), "row": row.int(), "xs": _gathered(s["x"], slot, s["top"]).to(bf16)}
        taken = _taken(s["ys"], row)
        out["y"] = (taken * s["weight"].unsqueeze(-1)).sum(1).to(bf16)
        if s["train"]:
            out["dys"] = _gathered(s["dy"], slot, s["top"], s["weight"]).to(bf16)
            out["dweight"] = (taken * s["dy"].float().unsqueeze(1)).sum(-1)
            out["dx"] = _taken(s["dxs"], row).sum(1).to(bf16)
        return out
    fmt, x, top, experts = s["fmt"], s["x"], s["top"], s["experts"]
    starts, row, slot = _sorted_rows(s["ids"], experts, 128)
    of = _tile_expert(starts, slot.numel())
    xs = _gathered(x, slot, top)
    w = _fake(s["w"], fmt) if s["train"] else _decoded(s["w"], fmt)
    ys = torch.bmm(_fake(xs, fmt).unflatten(0, (-1, 128)), w[of].transpose(1, 2)).flatten(0, 1)
    taken = _taken(ys, row)
    out = {"y": (taken * s["weight"].float().unsqueeze(-1)).sum(1).to(bf16)}
    if s["train"]:
        dys = _gathered(s["dy"], slot, top, s["weight"])
        out["dweight"] = (taken * s["dy"].float().unsqueeze(1)).sum(-1).to(bf16)
        dxs = torch.bmm(_fake(dys, fmt).unflatten(0, (-1, 128)), _fake(s["w"].transpose(1, 2), fmt)[of].transpose(1, 2)).flatten(0, 1)
        out["dx"] = _taken(dxs, row).sum(1).to(bf16)
        dt = _fake(dys.t(), fmt).unflatten(1, (-1, 128)).transpose(0, 1)                     # [tile, n_out, 128]
        xt = _fake(xs.t(), fmt).unflatten(1, (-1, 128)).transpose(0, 1)
        dw = torch.zeros(experts, dt.shape[1], xt.shape[1], device=x.device).index_add_(0, of, torch.bmm(dt, xt.transpose(1, 2)))
        out["dw"] = dw.to(bf16)
    return out


# --------------------------------------------------------------------------------------- the framework's ----

def _operand(fp4, w, fmt):
    return fp4.Operand(w["codes"], w["scales"], w["rows"], w["cols"], fmt, w["tensor_scale"])


def _own(s):
    from paper_2512_22804_b200 import experts, fp4
    op = s["op"]
    if op == "quantize":
        rows, cols = fp4.quantize(s["x"], s["fmt"], cols=s["both"])
        out = {"rows": fp4.dequantize(rows)}
        if s["both"]:
            out["cols"] = fp4.dequantize(cols)
        return out
    if op == "linear":
        if not s["train"]:
            a, _ = fp4.quantize(s["x"], s["fmt"], amax=s["amax"])
            return {"y": fp4.matmul(a, _operand(fp4, s["w"], s["fmt"]))}
        x, w = s["x"].detach().requires_grad_(), s["w"].detach().requires_grad_()
        y = fp4.linear(x, w, s["fmt"])
        dx, dw = torch.autograd.grad(y, (x, w), s["dy"])
        return {"y": y, "dx": dx, "dw": dw}
    if op == "route":
        plan = experts.sort(s["ids"], s["experts"])
        out = {"starts": plan.starts, "row": plan.row, "xs": experts.gather(s["x"], plan), "y": experts.combine(s["ys"], plan, s["weight"])}
        if s["train"]:
            out["dys"], out["dweight"] = experts.combine_grad(s["dy"], s["ys"], plan, s["weight"])
            out["dx"] = experts.combine(s["dxs"], plan)
        return out
    if not s["train"]:
        return {"y": experts.linear(s["x"], _operand(fp4, s["w"], s["fmt"]), s["ids"], s["weight"])}
    x, w, weight = (s[k].detach().requires_grad_() for k in ("x", "w", "weight"))
    y = experts.linear(x, w, s["ids"], weight, s["fmt"])
    dx, dw, dweight = torch.autograd.grad(y, (x, w, weight), s["dy"])
    return {"y": y, "dx": dx, "dw": dw, "dweight": dweight}


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------- work ----

def work(case):
    """Bytes that have to be read and written and operations that have to be done; of masked tokens an eighth is taken off."""
    op = case["op"]
    per = {"e8m0_32": 0.5 + 1 / 32, "e4m3_16": 0.5 + 1 / 16}.get(case.get("fmt"))
    if op == "quantize":
        n = case["rows"] * case["cols"]
        return {"bytes": n * ((2 if case["dtype"] == "bf16" else 4) + (4 if case["both"] else 2)), "flops": 0}
    if op == "linear":
        m, k, n = case["tokens"], case["n_in"], case["n_out"]
        if not case["train"]:
            return {"bytes": 2 * m * k + per * n * k + 2 * m * n, "flops": 2.0 * m * n * k}
        return {"bytes": 2 * 2 * (m * k + n * k + m * n), "flops": 6.0 * m * n * k}
    share = 0.875 if case["tokens"] > 1 else 1.0
    t, slots = case["tokens"], case["tokens"] * case["top"]
    if op == "route":
        row = 2 * case["hidden"]
        reads = t * row + slots * row * share                             # x; the experts' rows
        writes = slots * row + t * row                                    # xs; y
        if case["train"]:
            reads += t * row + slots * row * share                        # dy; dxs (the experts' rows are counted)
            writes += slots * row + t * row + 4 * slots                   # dys; dx; dweight
        return {"bytes": reads + writes + 12 * slots, "flops": 0}
    k, n, e = case["n_in"], case["n_out"], case["experts"]
    used = min(e, slots)
    if not case["train"]:
        return {"bytes": 2 * t * (k + n) + per * used * n * k + 8 * slots, "flops": 2.0 * share * slots * n * k}
    return {"bytes": 4 * t * (k + n) + 4 * e * n * k + 12 * slots, "flops": 6.0 * share * slots * n * k}


# ------------------------------------------------------------------------------- the definition in 64 bits ----

def _nearest(v, step):
    """v / step to the nearest whole number, ties to even, times step."""
    return torch.round(v / step) * step


def _power(e):
    """2^e exactly, from its bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _binade(v):
    """floor(log2 v) exactly."""
    return torch.frexp(v).exponent - 1


def _exact_fake(x, fmt, amax=None):
    """The definition of quantisation along the last axis and back, every quantity in 64 bits."""
    x = x.double()
    n, cols = BLOCK[fmt], x.shape[-1]
    b = torch.cat((x, x.new_zeros(*x.shape[:-1], -cols % n)), -1)
    b = b.reshape(*b.shape[:-1], -1, n)
    a = b.abs().amax(-1, keepdim=True)
    if fmt == "e8m0_32":
        d = _power(_binade(a.clamp(min=2.0 ** -125)) - 2)
    else:
        top = (x.abs().max() if amax is None else amax.double()).clamp(min=2.0 ** -88)
        s = (448 * a / top).clamp(max=448.0)
        d = _nearest(s, _power(_binade(s.clamp(min=2.0 ** -6)) - 3)) * (top / 2688)
    y = torch.where(d > 0, b / torch.where(d > 0, d, 1.0), 0.0).clamp(-6.0, 6.0)
    y = _nearest(y, _power(_binade(y.abs().clamp(min=1.0)) - 1)) * d
    return y.reshape(*y.shape[:-2], -1)[..., :cols]


def _exact_decoded(w, fmt):
    """The values of a stored weight: byte by byte from the layout."""
    grid = torch.tensor(GRID + tuple(-v for v in GRID), dtype=torch.float64, device="cuda")
    rows, cols, n = w["rows"], w["cols"], BLOCK[fmt]
    k = torch.arange(cols, device="cuda")
    r = torch.arange(rows, device="cuda").unsqueeze(1)
    byte = w["codes"][..., k // 2].int()
    v = grid[torch.where(k % 2 == 0, byte % 16, byte // 16)]
    block = torch.arange(-(-cols // n), device="cuda")
    tiles = -(-block.numel() // 4)
    at = (r // 128 * tiles + block // 4) * 512 + r % 32 * 16 + r // 32 % 4 * 4 + block % 4
    b = w["scales"].reshape(*w["codes"].shape[:-2], -1)[..., at].int()
    if fmt == "e8m0_32":
        s = _power(b - 127)
    else:
        e, m = b // 8, b % 8
        s = torch.where(e == 0, m * 2.0 ** -9, (8 + m) * _power(e - 10))
    return v * s.double()[..., k // n] * w["tensor_scale"].double()


def exact(case, seed):
    s = prepare(case, seed)
    op, fmt = case["op"], case.get("fmt")
    if op == "quantize":
        return {"rows": _exact_fake(s["x"], fmt), **({"cols": _exact_fake(s["x"].t(), fmt)} if case["both"] else {})}
    if op == "linear":
        if not case["train"]:
            return {"y": _exact_fake(s["x"], fmt, s["amax"]) @ _exact_decoded(s["w"], fmt).t()}
        x, w, dy = s["x"], s["w"], s["dy"]
        return {"y": _exact_fake(x, fmt) @ _exact_fake(w, fmt).t(), "dx": _exact_fake(dy, fmt) @ _exact_fake(w.t(), fmt).t(),
                "dw": _exact_fake(dy.t(), fmt) @ _exact_fake(x.t(), fmt).t()}
    # expert by expert: the slots of each, in order
    ids, weight, top, experts = s["ids"].reshape(-1).cpu(), s["weight"].double().reshape(-1), case["top"], case["experts"]
    align = 1 if op == "route" else 128
    slots = [torch.nonzero(ids == e).reshape(-1).cuda() for e in range(experts)]
    starts = [0]
    for at in slots:
        starts.append(starts[-1] + (at.numel() + align - 1) // align * align)
    rows = _capacity(ids.numel(), experts, align)
    x = s["x"].double()

    def spread(source, scale=None):
        out = torch.zeros(rows, source.shape[1], dtype=torch.float64, device="cuda")
        for e, at in enumerate(slots):
            part = source[at // top]
            out[starts[e]:starts[e] + at.numel()] = part if scale is None else part * scale[at].unsqueeze(1)
        return out

    def collect(source, scale=None):
        out = torch.zeros(case["tokens"], source.shape[1], dtype=torch.float64, device="cuda")
        for e, at in enumerate(slots):
            part = source[starts[e]:starts[e] + at.numel()]
            out.index_add_(0, at // top, part if scale is None else part * scale[at].unsqueeze(1))
        return out

    def dots(source, dy):
        out = torch.zeros(ids.numel(), dtype=torch.float64, device="cuda")
        for e, at in enumerate(slots):
            out[at] = (source[starts[e]:starts[e] + at.numel()] * dy[at // top]).sum(1)
        return out.reshape(case["tokens"], top)

    if op == "route":
        out = {"starts": None, "row": None, "xs": spread(x), "y": collect(s["ys"].double(), weight)}
        if case["train"]:
            dy = s["dy"].double()
            out.update(dys=spread(dy, weight), dweight=dots(s["ys"].double(), dy), dx=collect(s["dxs"].double()))
        return out
    xs = spread(x)
    w = _exact_fake(s["w"], fmt) if case["train"] else _exact_decoded(s["w"], fmt)

    def per_expert(source, matrices):
        out = torch.zeros(rows, matrices.shape[1], dtype=torch.float64, device="cuda")
        for e in range(experts):
            out[starts[e]:starts[e + 1]] = source[starts[e]:starts[e + 1]] @ matrices[e].t()
        return out

    ys = per_expert(_exact_fake(xs, fmt), w)
    out = {"y": collect(ys, weight)}
    if case["train"]:
        dy = s["dy"].double()
        dys = spread(dy, weight)
        dxs = per_expert(_exact_fake(dys, fmt), _exact_fake(s["w"].transpose(1, 2), fmt))
        dt, xt = _exact_fake(dys.t(), fmt), _exact_fake(xs.t(), fmt)
        dw = torch.stack([dt[:, a:b] @ xt[:, a:b].t() for a, b in zip(starts, starts[1:])])
        out.update(dx=collect(dxs), dweight=dots(ys, dy), dw=dw)
    return out

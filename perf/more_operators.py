"""What is measured of the operators beside a 4-bit projection: the norm before it, the adapters next to it, and the step that trains them.

* ``norm``      h = x + residual, y = h / sqrt(mean(h^2) + eps) * w, with its gradient, or with y as E4M3 codes and scales
* ``adapters``  out = base + scale[g] * (x a[g]^T) b[g]^T with an adapter g for every token; training adds the gradients of x, a and b
* ``adamw``     one step over many tensors, moments in 32 bits or as E4M3 codes with one scale for 128 elements

8-bit output of the norm: s = 448 / max|y| over 128 columns or a whole row, either as it is ("fp32") or cut to a power of two ("e8m0", kept
as a biased exponent); code = E4M3(y s), nearest even; value = code / s.

8-bit moments: blocks of 128 consecutive elements of a tensor share a power of two s, the largest that keeps the block's largest magnitude
times s within 448 (biased exponent at most 253; 127 for a block of zeros).  The first moment is kept as E4M3 of m s, the second as E4M3 of w =
sqrt(v) s, both between two neighbouring codes n d and (n + 1) d by a random number: with t = |m s| / d, the upper one if t + u >= n + 1; with t = w / d,
the upper one if u (2n + 1) < (t - n) (t + n), which keeps the mean of the square, and never zero for a w that is not.  BF16 parameters are rounded with a
random number too: 16 random bits are added below the kept ones, which are then cut off.  The random numbers are 16-bit fractions of mixed words: with
mix(z) = two rounds of xor-shift and multiplication (see ``_mix``), key = mix(mix(seed + 0x9E3779B9 step) + tensor number), z = mix(mix(element >> 32 ^ key)
+ element low half): the low half of z for m, the high half for v, the low half of mix(z ^ 0x9E3779B9) for the parameter.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
BLOCK = 128
EPS = 1e-6
ADAM = {"lr": 2e-3, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "weight_decay": 0.01}


# ------------------------------------------------------------------------------------------------ cases ----

def listed():
    return [
        # decoding: one token's residual stream, normed and quantised for the next projection
        {"name": "norm_one_token", "op": "norm", "rows": 1, "cols": 4096, "x": "bf16", "residual": "bf16", "out": "e8m0_128"},
        # a prompt of 8192 tokens, one FP32 scale a token as a row-scaled 8-bit product takes it
        {"name": "norm_prompt_rows", "op": "norm", "rows": 8192, "cols": 4096, "x": "bf16", "residual": "bf16", "out": "fp32_row"},
        # a training step's norm: forward and gradient, the residual's own gradient joining
        {"name": "norm_train", "op": "norm", "rows": 8192, "cols": 4096, "x": "bf16", "residual": "bf16", "out": "train"},
        # the same with a residual stream in 32 bits and sizes that are multiples of nothing
        {"name": "norm_train_ragged", "op": "norm", "rows": 1187, "cols": 1501, "x": "bf16", "residual": "fp32", "out": "train"},
        # decoding: one request through its adapter beside an up projection
        {"name": "adapters_one_token", "op": "adapters", "tokens": 1, "n_in": 4096, "n_out": 14336, "rank": 16, "adapters": 8, "train": False},
        # decoding for a batch of sequences of many tenants
        {"name": "adapters_48_tokens", "op": "adapters", "tokens": 48, "n_in": 4096, "n_out": 4096, "rank": 32, "adapters": 24, "train": False},
        # prompts of several requests packed together through an up projection
        {"name": "adapters_prompts", "op": "adapters", "tokens": 8192, "n_in": 4096, "n_out": 14336, "rank": 32, "adapters": 16, "train": False},
        # fine-tuning one adapter beside a square projection
        {"name": "adapters_train", "op": "adapters", "tokens": 8192, "n_in": 4096, "n_out": 4096, "rank": 64, "adapters": 1, "train": True},
        # fine-tuning a few at once, sizes that are multiples of nothing
        {"name": "adapters_train_ragged", "op": "adapters", "tokens": 1187, "n_in": 1500, "n_out": 2731, "rank": 24, "adapters": 5, "train": True},
        # the step of a fine-tuning run: many small tensors, BF16, 8-bit moments
        {"name": "adamw_many_small", "op": "adamw", "tensors": 128, "numel": 65536, "param": "bf16", "grad": "bf16", "moments": "8bit"},
        # the step of a layer's matrices with everything in 32 bits
        {"name": "adamw_layer", "op": "adamw", "tensors": 7, "numel": 14680064, "param": "fp32", "grad": "fp32", "moments": "32bit"},
        # the same with gradients of a BF16 backward pass and moments in 8 bits
        {"name": "adamw_layer_8bit", "op": "adamw", "tensors": 7, "numel": 14680064, "param": "fp32", "grad": "bf16", "moments": "8bit"},
    ]


def _log(rng, lo, hi):
    """A whole number, uniform in its logarithm; every second one is brought to a multiple of 8 or 128, as most real sizes are."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    m = rng.choice((1, 1, 8, 128))
    return max(lo, min(hi, (v + m - 1) // m * m))


def draw(rng):
    op = rng.choice(("norm", "adapters", "adapters", "adamw"))
    if op == "norm":
        out = rng.choice(("e8m0_128", "fp32_128", "e8m0_row", "fp32_row", "train", "train"))
        wide = rng.random() < 0.25
        return {"op": op, "rows": _log(rng, 1, 2048 if wide else 8192), "cols": _log(rng, 64, 16384 if wide else 4096),
                "x": rng.choice(("bf16", "bf16", "fp32")), "residual": rng.choice(("none", "bf16", "fp32")), "out": out}
    if op == "adapters":
        train = rng.random() < 0.5
        rank = _log(rng, 4, 64)
        return {"op": op, "tokens": _log(rng, 64 if train else 1, 8192), "n_in": _log(rng, 256, 4096), "n_out": _log(rng, 256, 4096 if train else 14336),
                "rank": rank, "adapters": rng.randint(1, min(64, 512 // rank)), "train": train}
    tensors = _log(rng, 1, 200)
    return {"op": op, "tensors": tensors, "numel": _log(rng, 256, 60_000_000 // tensors), "param": rng.choice(("bf16", "fp32")),
            "grad": rng.choice(("bf16", "fp32")), "moments": rng.choice(("8bit", "8bit", "32bit"))}


# ----------------------------------------------------------------------------------------------- inputs ----

def _activation(g, rows, cols):
    """Heavy-tailed values with a few outlier channels."""
    x = torch.randn(rows, cols, generator=g, device="cuda") / (0.5 + 0.5 * torch.rand(rows, 1, generator=g, device="cuda"))
    gain = torch.where(torch.rand(cols, generator=g, device="cuda") < 0.004, 30.0, 1.0)
    return x * gain


def _gradient(g, *shape):
    """Signed magnitudes over many binades, 5 % exact zeros."""
    m = torch.exp2((torch.randn(*shape, generator=g, device="cuda") * 3.0 - 13.0).clamp_(-30.0, 4.0))
    u = torch.rand(*shape, generator=g, device="cuda")
    return torch.where(u < 0.05, 0.0, torch.where(u < 0.525, -m, m))


def _sizes(case):
    """Sizes of the tensors: about `numel` each, the same for every seed; some are odd."""
    rng = random.Random(case["tensors"] * 1000003 + case["numel"])
    if case["tensors"] > 16:
        return [max(1, int(case["numel"] * rng.choice((0.25, 0.5, 1.0, 1.0, 1.6)) - rng.choice((0, 0, 0, 1, 37)))) for _ in range(case["tensors"])]
    return [case["numel"]] * case["tensors"]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    op = case["op"]
    if op == "norm":
        rows, cols = case["rows"], case["cols"]
        s["x_in"] = _activation(g, rows, cols).to(DTYPES[case["x"]])
        s["r_in"] = None if case["residual"] == "none" else (_activation(g, rows, cols) * 4).to(DTYPES[case["residual"]])
        s["w"] = (1 + 0.1 * torch.randn(cols, generator=g, device="cuda")).to(DTYPES[case["x"]])
        if case["out"] == "train":
            s["dy"] = _gradient(g, rows, cols).to(DTYPES[case["x"]])
            s["dh"] = None if s["r_in"] is None else _gradient(g, rows, cols).to(DTYPES[case["residual"]])
        return s
    if op == "adapters":
        t, k, n, r, e = (case[i] for i in ("tokens", "n_in", "n_out", "rank", "adapters"))
        bf16 = torch.bfloat16
        s["x"] = _activation(g, t, k).to(bf16)
        s["base"] = torch.randn(t, n, generator=g, device="cuda").to(bf16)          # what the shared projection gave
        s["a"] = (torch.randn(e, r, k, generator=g, device="cuda") * k ** -0.5).to(bf16)
        s["b"] = (torch.randn(e, n, r, generator=g, device="cuda") * 0.1).to(bf16)
        s["scale"] = torch.rand(e, generator=g, device="cuda") + 0.5
        if case["train"]:
            s["dy"] = _gradient(g, t, n).to(bf16)
        if case["train"] and e == 1:
            s["ids"] = None                                                         # every token goes through the one adapter
        elif case["train"] or t > 256:                                              # requests or samples one after the other
            at = torch.randint(0, t, (max(1, t // 100),), generator=g, device="cuda")
            cut = torch.zeros(t, dtype=torch.long, device="cuda").index_fill_(0, at, 1).cumsum(0)
            of = torch.randint(-1, e, (t + 1,), generator=g, device="cuda")         # -1: a request of the base model
            s["ids"] = of[cut].to(torch.int32)
        else:
            s["ids"] = torch.randint(0 if t == 1 else -1, e, (t,), generator=g, device="cuda").to(torch.int32)
        return s
    # parameters, gradients and moments are views of one buffer each, as a run keeps them that reduces its gradients in one call
    sizes = _sizes(case)
    room = [-(-n // BLOCK) * BLOCK for n in sizes]
    total = sum(room)
    s["sizes"] = sizes
    of = torch.repeat_interleave(torch.arange(len(room), device="cuda"), torch.tensor(room, device="cuda"))
    starts = torch.tensor([0] + room, device="cuda").cumsum(0)
    s["starts"] = starts
    inside = (torch.arange(total, device="cuda") - starts[of]) < torch.tensor(sizes, device="cuda")[of]

    def flat(values, dtype):
        return torch.where(inside, values, 0.0).to(dtype)

    p = flat(torch.randn(total, generator=g, device="cuda") * 0.02, DTYPES[case["param"]])
    grad = flat(_gradient(g, total), DTYPES[case["grad"]])
    m = flat(_gradient(g, total), torch.float32)
    v = (_gradient(g, total).square() + m.square() * 0.5) * inside
    del inside, of
    s["p"], s["g"] = p, grad
    s["step"], s["seed"] = 1000 + seed % 1000, seed
    if case["moments"] == "32bit":
        s["m"], s["v"] = m, v
    else:
        s["m"], ms = _nearest_codes(m)
        s["v"], vs = _nearest_codes(torch.sqrt(v))
        s["scales"] = torch.stack((ms, vs), 1).contiguous()                          # [blocks, 2]
    s["lists"] = [[t[:n] for t, n in zip(s[i].split(room), sizes)] for i in ("p", "g", "m", "v")]
    if case["moments"] == "8bit":
        s["lists"].append(list(s["scales"].split([n // BLOCK for n in room])))
    return s


def _nearest_codes(x):
    """A stored state: E4M3 codes, nearest, and the biased exponents of their blocks' scales."""
    s, e = _power_scale(x.view(-1, BLOCK).abs().amax(1, keepdim=True))
    return (x.view(-1, BLOCK) * s).to(torch.float8_e4m3fn).view(-1), e.view(-1)


# ------------------------------------------------------------------------------------------ plain forms ----

def _power_scale(a, most=253):
    """(scale, biased exponent) of the largest power of two that keeps a within 448."""
    f, e = torch.frexp(a)                                      # a = f 2^e with f in [0.5, 1); 448 = 0.875 2^9
    e = torch.where(f <= 0.875, 9 - e, 8 - e).clamp(max=most - 127)
    e = torch.where(a == 0, 0, e)
    return torch.ldexp(torch.ones_like(a), e), (e + 127).to(torch.uint8)


def _plain_norm(s):
    x, r, w = s["x_in"], s["r_in"], s["w"].float()
    h = x if r is None else (x.float() + r.float()).to(r.dtype)
    hf = h.float()
    rs = 1.0 / torch.sqrt(hf.square().mean(1, keepdim=True) + EPS)
    xh = hf * rs
    y = xh * w
    out = {} if r is None else {"h": h}
    if s["out"] != "train":
        n = BLOCK if s["out"].endswith("_128") else y.shape[1]
        b = torch.nn.functional.pad(y, (0, -y.shape[1] % n)).unflatten(1, (-1, n))
        a = b.abs().amax(2, keepdim=True)
        if s["out"].startswith("e8m0"):
            scale = _power_scale(a, 254)[0]
        else:
            scale = torch.where(a == 0, 1.0, (448.0 / a).clamp(max=torch.finfo(torch.float32).max))
        v = (b * scale).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).float() / scale
        out["y"] = v.flatten(1)[:, :y.shape[1]].to(torch.bfloat16)
        return out
    dy = s["dy"].float()
    gw = dy * w
    dh = rs * (gw - xh * (gw * xh).mean(1, keepdim=True))
    if r is not None:
        dh = dh + s["dh"].float()
        out["dr"] = dh.to(r.dtype)
    out.update(y=y.to(x.dtype), dx=dh.to(x.dtype), dw=(dy * xh).sum(0).to(x.dtype))
    return out


def _plain_adapters(s):
    x, a, b = s["x"].float(), s["a"].float(), s["b"].float()
    e, r, k = a.shape
    ids = torch.zeros(x.shape[0], dtype=torch.int32, device=x.device) if s["ids"] is None else s["ids"]
    on = (ids.unsqueeze(1) == torch.arange(e, device=x.device)).float() * s["scale"]            # [tokens, adapters]
    on = on.repeat_interleave(r, 1)
    a2, b2 = a.reshape(e * r, k), b.transpose(1, 2).reshape(e * r, -1)
    h = (x @ a2.t()) * on
    out = {"y": (s["base"].float() + h @ b2).to(s["base"].dtype)}
    if s["train"]:
        dy = s["dy"].float()
        u = (dy @ b2.t()) * on
        bf16 = torch.bfloat16
        out["dx"] = (u @ a2).to(bf16)
        out["da"] = (u.t() @ x).view(e, r, k).to(bf16)
        out["db"] = (h.t() @ dy).view(e, r, -1).transpose(1, 2).to(bf16)
    return out


def _mix(z):
    """32-bit words (in 64-bit integers): two rounds of xor-shift and multiplication."""
    z = z & 0xFFFFFFFF
    z = z ^ (z >> 16)
    z = (z * 0x7FEB352D) & 0xFFFFFFFF
    z = z ^ (z >> 15)
    z = (z * 0x846CA68B) & 0xFFFFFFFF
    return z ^ (z >> 16)


def _random(s):
    """Random words of every element of the flat buffer: one for the moments, one for the parameter."""
    n = s["p"].numel()
    at = torch.arange(n, device="cuda")
    starts = s["starts"]
    of = torch.searchsorted(starts, at, right=True) - 1
    at -= starts[of]
    first = _mix(torch.full((1,), s["seed"], device="cuda") + 0x9E3779B9 * s["step"])
    key = _mix(first + of)
    z = _mix(_mix((at >> 32) ^ key) + (at & 0xFFFFFFFF))
    return z, _mix(z ^ 0x9E3779B9)


def _steps(w):
    """Distance of neighbouring E4M3 values at |w|."""
    return torch.ldexp(torch.ones_like(w), torch.frexp(w).exponent.clamp(min=-5) - 4)


def _plain_adamw(s):
    c = ADAM
    step = s["step"]
    eight = s["moments"] == "8bit"
    if eight:
        e = s["scales"].int() - 127
        one = torch.ones(e.shape[0], 1, device="cuda")
        m = (s["m"].float().view(-1, BLOCK) * torch.ldexp(one, -e[:, :1])).view(-1)
        v = (s["v"].float().view(-1, BLOCK) * torch.ldexp(one, -e[:, 1:])).view(-1).square()
    else:
        m, v = s["m"], s["v"]
    g = s["g"].float()
    m = c["beta1"] * m + (1 - c["beta1"]) * g
    v = c["beta2"] * v + (1 - c["beta2"]) * g * g
    root = torch.sqrt(v)
    bias1, bias2 = 1 - c["beta1"] ** step, math.sqrt(1 - c["beta2"] ** step)
    p = s["p"].float()
    p = p * (1 - c["lr"] * c["weight_decay"]) - (c["lr"] / bias1) * (m / (root / bias2 + c["eps"]))
    del g
    if eight or s["param"] == "bf16":
        z, zp = _random(s)
    if s["param"] == "bf16":
        bits = p.view(torch.int32) + (zp & 0xFFFF).int()
        p = (bits & -65536).view(torch.float32).to(torch.bfloat16)
        del bits
    s["p"].copy_(p)
    del p
    if not eight:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return {"p": s["p"], "m": s["m"], "v": s["v"]}
    out = {"p": s["p"]}
    for name, x, u, column in (("m", m, z & 0xFFFF, 0), ("v", root, z >> 16, 1)):
        u = u.float() * (1.0 / 65536)
        b = x.view(-1, BLOCK)
        scale, e = _power_scale(b.abs().amax(1, keepdim=True))
        w = (b * scale).view(-1).abs()
        d = _steps(w)
        t = w / d
        n = torch.floor(t)
        if name == "m":
            q = torch.floor(t + u) * d
        else:
            up = u * (2 * n + 1) < (t - n) * (t + n)
            q = torch.where(w > 0, torch.where(up, n + 1, n).clamp(min=1.0), 0.0) * d
        q = torch.where(x < 0, -q, q).view(-1, BLOCK)
        s[name].copy_(q.view(-1))
        s["scales"][:, column] = e.view(-1)
        value = q / scale
        out[name] = (value if name == "m" else value.square()).view(-1).to(torch.bfloat16)
    return out


def _plain(s):
    return {"norm": _plain_norm, "adapters": _plain_adapters, "adamw": _plain_adamw}[s["op"]](s)


# --------------------------------------------------------------------------------------- the framework's ----

def _own(s):
    from paper_2512_22804_b200 import adapters, norm, optim
    op = s["op"]
    if op == "norm":
        x, r, w = s["x_in"], s["r_in"], s["w"]
        if s["out"] != "train":
            scale, block = s["out"].split("_")
            codes, scales, *h = norm.rms_norm_quantize(x, w, r, eps=EPS, block=BLOCK if block == "128" else None, scale=scale)
            return {"y": norm.dequantize(codes, scales), **({"h": h[0]} if h else {})}
        x, w = x.detach().requires_grad_(), w.detach().requires_grad_()
        if r is None:
            y = norm.rms_norm(x, w, eps=EPS)
            dx, dw = torch.autograd.grad(y, (x, w), s["dy"])
            return {"y": y, "dx": dx, "dw": dw}
        r = r.detach().requires_grad_()
        y, h = norm.rms_norm(x, w, r, eps=EPS)
        dx, dr, dw = torch.autograd.grad((y, h), (x, r, w), (s["dy"], s["dh"]))
        return {"y": y, "h": h, "dx": dx, "dr": dr, "dw": dw}
    if op == "adapters":
        if not s["train"]:
            return {"y": adapters.add(s["base"], s["x"], s["a"], s["b"], s["ids"], s["scale"])}
        x, a, b = (s[i].detach().requires_grad_() for i in ("x", "a", "b"))
        y = adapters.add(s["base"], x, a, b, s["ids"], s["scale"])
        dx, da, db = torch.autograd.grad(y, (x, a, b), s["dy"])
        return {"y": y, "dx": dx, "da": da, "db": db}
    optim.adamw_(*s["lists"], step=s["step"], seed=s["seed"], **ADAM)
    if s["moments"] == "32bit":
        return {"p": s["p"], "m": s["m"], "v": s["v"]}
    m, v = optim.moments(s["m"], s["v"], s["scales"], torch.bfloat16)
    return {"p": s["p"], "m": m, "v": v}


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------- work ----

def work(case):
    op = case["op"]
    size = {"bf16": 2, "fp32": 4, "none": 0}
    if op == "norm":
        n, x, r = case["rows"] * case["cols"], size[case["x"]], size[case["residual"]]
        if case["out"] != "train":
            return {"bytes": n * (x + 2 * r + 2) + case["cols"] * x, "flops": 0}                    # x, r; h, the values of y
        return {"bytes": n * (4 * x + 4 * r) + 2 * case["cols"] * x, "flops": 0}                    # x, r, dy, dh; y, h, dx, dr
    if op == "adapters":
        t, k, n, r, e = (case[i] for i in ("tokens", "n_in", "n_out", "rank", "adapters"))
        used = min(e, t)
        if not case["train"]:
            return {"bytes": 2 * t * k + 4 * t * n + 2 * used * r * (k + n), "flops": 2.0 * t * r * (k + n)}
        return {"bytes": 4 * t * k + 6 * t * n + 4 * used * r * (k + n), "flops": 6.0 * t * r * (k + n)}
    n = sum(_sizes(case))
    p, g = size[case["param"]], size[case["grad"]]
    if case["moments"] == "32bit":
        return {"bytes": n * (2 * p + g + 16), "flops": 0}
    return {"bytes": n * (2 * p + g + 4 + 4 + 4 / BLOCK), "flops": 0}                                # the moments' values are written too


# ------------------------------------------------------------------------------- the definition in 64 bits ----

def _two_to(e):
    """2^e exactly, from its bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _binade(v):
    """floor(log2 v) exactly (of zero: something small)."""
    return torch.frexp(v).exponent - 1


def _cut_scale(a, most):
    """floor(log2(448 / a)), at most `most`; zero for zero."""
    e = _binade(448 / torch.where(a == 0, 448.0, a))
    return e.clamp(max=most)


def _exact_norm(s):
    x = s["x_in"].double()
    h = x if s["r_in"] is None else (x + s["r_in"].double())
    out = {} if s["r_in"] is None else {"h": h}
    if s["r_in"] is not None:
        h = h.to(s["r_in"].dtype).double()                     # the residual stream as it is kept
    w, cols = s["w"].double(), x.shape[1]
    rs = (h.pow(2).sum(1, keepdim=True) / cols + EPS).pow(-0.5)
    y = h * rs * w
    if s["out"] == "train":
        dy = s["dy"].double()
        dot = (dy * w * h).sum(1, keepdim=True)
        dh = dy * w * rs - h * rs.pow(3) * dot / cols + (0 if s["r_in"] is None else s["dh"].double())
        out.update(y=y, dx=dh, dw=(dy * h * rs).sum(0))
        if s["r_in"] is not None:
            out["dr"] = dh
        return out
    n = BLOCK if s["out"].endswith("_128") else cols
    b = torch.cat((y, y.new_zeros(y.shape[0], -cols % n)), 1).reshape(y.shape[0], -1, n)
    a = b.abs().amax(2, keepdim=True)
    s_ = _two_to(_cut_scale(a, 127)) if s["out"].startswith("e8m0") else 448 / torch.where(a == 0, 448.0, a)
    z = b * s_
    d = _two_to(_binade(z.abs().clamp(min=2.0 ** -6)) - 3)
    out["y"] = (torch.round(z / d) * d / s_).reshape(y.shape[0], -1)[:, :cols]
    return out


def _exact_adapters(s):
    x, base = s["x"].double(), s["base"].double()
    y = base.clone()
    e, r, k = s["a"].shape
    dx, da, db = torch.zeros_like(x), torch.zeros(e, r, k, device="cuda", dtype=torch.float64), torch.zeros(e, base.shape[1], r, device="cuda", dtype=torch.float64)
    for g in range(e):
        at = torch.arange(x.shape[0], device="cuda") if s["ids"] is None else torch.nonzero(s["ids"] == g).reshape(-1)
        a, b, scale = s["a"][g].double(), s["b"][g].double(), s["scale"][g].double()
        h = x[at] @ a.t() * scale
        y[at] += h @ b.t()
        if s["train"]:
            dy = s["dy"][at].double()
            u = dy @ b * scale
            dx[at] = u @ a
            da[g], db[g] = u.t() @ x[at], dy.t() @ h
    return {"y": y, "dx": dx, "da": da, "db": db} if s["train"] else {"y": y}


def _exact_adamw(s):
    lr, b1, b2, eps, decay = (float(ADAM[i]) for i in ("lr", "beta1", "beta2", "eps", "weight_decay"))
    t, outs = s["step"], {"p": [], "m": [], "v": []}

    def scramble(z):
        for shift, factor in ((16, 0x7FEB352D), (15, 0x846CA68B)):
            z = ((z ^ (z >> shift)) * factor) % 2 ** 32
        return z ^ (z >> 16)

    at = 0
    first = scramble((s["seed"] + 0x9E3779B9 * t) % 2 ** 32)
    for number, size in enumerate(s["sizes"]):
        room = -(-size // BLOCK) * BLOCK
        part = slice(at, at + room)
        p, g = s["p"][part].double(), s["g"][part].double()
        m, v = s["m"][part].double(), s["v"][part].double()
        if s["moments"] == "8bit":
            e = s["scales"][at // BLOCK:(at + room) // BLOCK].long() - 127
            m = (m.view(-1, BLOCK) / _two_to(e[:, :1])).view(-1)
            v = (v.view(-1, BLOCK) / _two_to(e[:, 1:])).view(-1) ** 2
        at += room
        m = b1 * m + (1 - b1) * g
        v = b2 * v + (1 - b2) * g ** 2
        p = p - lr * decay * p - lr * (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + eps)
        i = torch.arange(room, device="cuda")
        z = scramble((scramble(scramble((first + number) % 2 ** 32) ^ (i >> 32)) + i % 2 ** 32) % 2 ** 32)
        if s["param"] == "bf16":
            d = _two_to(_binade(p.abs().clamp(min=2.0 ** -126)) - 7)
            up = (scramble(z ^ 0x9E3779B9) % 65536).double() / 65536
            p = torch.sign(p) * torch.floor(p.abs() / d + up) * d
        if s["moments"] == "8bit":
            for name, x, u in (("m", m, z % 65536), ("v", v.sqrt(), z // 65536)):
                b = x.view(-1, BLOCK)
                scale = _two_to(_cut_scale(b.abs().amax(1, keepdim=True), 126))
                w, u = b * scale, u.double().view(-1, BLOCK) / 65536
                d = _two_to(_binade(w.abs().clamp(min=2.0 ** -6)) - 3)
                lo = torch.floor(w.abs() / d) * d
                hi = lo + d
                if name == "m":
                    q = torch.where(lo + u * d + (w.abs() - lo) >= hi, hi, lo)
                else:
                    q = torch.where(u * (hi ** 2 - lo ** 2) < w ** 2 - lo ** 2, hi, lo)
                    q = torch.where((w > 0) & (q == 0), hi, q)
                x = (torch.sign(w) * q / scale).view(-1)
                if name == "m":
                    m = x
                else:
                    v = x ** 2
        for name, x in (("p", p), ("m", m), ("v", v)):
            outs[name].append(x)
    return {k: torch.cat(v) for k, v in outs.items()}


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "adapters": _exact_adapters, "adamw": _exact_adamw}[case["op"]](s)

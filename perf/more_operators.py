"""Performance cases of linear layers in 8-bit floats and of the optimizer step beside them.

A case is a dict of plain values.  Its "kind" names the operator that one pass runs:

* ``quantize``      ``quantize_fp8``: codes of 8 bits with a power-of-two scale for each block of 128, of a matrix, of
                    its transpose, or of both;
* ``linear``        ``linear_fp8``: the product of activations, quantized on the way, and weights held in 8 bits;
* ``linear_grad``   ``linear_fp8_grad``: the gradients of a training step;
* ``grouped``       ``linear_fp8_grouped``: rows sorted by expert, each expert with weights of its own;
* ``grouped_grad``  ``linear_fp8_grouped_grad``: its gradients;
* ``adamw``         ``adamw_step``: AdamW over many tensors, states in 32 bits or in 8.

``own`` chooses the side: False computes the plain form with torch, True calls the library.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}
BLOCK = 128                                           # columns (and for weights rows) that share a scale
MOST_CODE = 448.0                                     # the largest 8-bit float (1 sign, 4 exponent, 3 fraction bits)
LR, BETAS, EPS, DECAY = 3e-4, (0.9, 0.999), 1e-8, 0.1
SEED = 20                                             # of the rounding of 8-bit states

# the kept values of a 4096-wide layer's q, k, v, o, gate, up and down at 70%, and its two norms
LAYER = "5033165,5033165,5033165,5033165,13526630,13526630,13526630,4096,4096"


def listed():
    return [
        # one token's activations between two layers: latency
        {"name": "quantize_b1", "kind": "quantize", "rows": 1, "cols": 4096, "block": 1, "form": "rows", "dtype": "bf16"},
        # a training step's gradient, for dX along its columns and for dW along its tokens
        {"name": "quantize_both_2048", "kind": "quantize", "rows": 2048, "cols": 11008, "block": 1, "form": "both",
         "dtype": "bf16"},
        # one token through the 4096-wide layer's gate
        {"name": "linear_b1", "kind": "linear", "rows": 1, "n": 11008, "k": 4096, "block": 128, "dtype": "bf16"},
        # a small batch, sizes that fit no tile, a scale for each row of the weights
        {"name": "linear_b24_odd", "kind": "linear", "rows": 24, "n": 1111, "k": 1000, "block": 1, "dtype": "fp16"},
        # a prompt of 2048 tokens through the gate
        {"name": "linear_2048", "kind": "linear", "rows": 2048, "n": 11008, "k": 4096, "block": 128, "dtype": "bf16"},
        # a training step's gradients of a square projection
        {"name": "linear_grad_2048", "kind": "linear_grad", "rows": 2048, "n": 4096, "k": 4096, "dtype": "bf16"},
        # a decode step of 32 users, whose tokens went to some of 8 experts
        {"name": "grouped_b32", "kind": "grouped", "rows": 32, "experts": 8, "n": 5632, "k": 2048, "block": 128,
         "dtype": "bf16"},
        # prompts over 16 experts, some of them popular and some without a row
        {"name": "grouped_4096", "kind": "grouped", "rows": 4096, "experts": 16, "n": 5632, "k": 2048, "block": 128,
         "dtype": "bf16"},
        # the gradients of a ragged training batch, sizes that fit no tile
        {"name": "grouped_grad_1500", "kind": "grouped_grad", "rows": 1500, "experts": 8, "n": 1000, "k": 2048,
         "dtype": "bf16"},
        # norms and biases: many small tensors, 32-bit states
        {"name": "adamw_small", "kind": "adamw", "sizes": "1,4096,4096,77,1000,128,129,2048,11008,5,4096,333,512,2047,64,640",
         "bits": 32, "param": "fp32", "grad": "fp32", "copy": False},
        # the kept values of a sparse layer: fp32 masters, 16-bit copies that the products read
        {"name": "adamw_layer_32", "kind": "adamw", "sizes": LAYER, "bits": 32, "param": "fp32", "grad": "bf16",
         "copy": True},
        # the same with states of 8 bits
        {"name": "adamw_layer_8", "kind": "adamw", "sizes": LAYER, "bits": 8, "param": "fp32", "grad": "bf16",
         "copy": True},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        case = _drawn(rng)
        if _cost(case) <= most:
            return case


def _width(rng):
    n = _log_int(rng, 64, 11008)
    return n if rng.random() < 0.4 else max(64, n // 64 * 64)


def _drawn(rng):
    kind = rng.choice(["quantize", "linear", "linear", "linear_grad", "grouped", "grouped", "grouped_grad", "adamw"])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    if kind == "quantize":
        return {"kind": kind, "rows": _log_int(rng, 1, 8192), "cols": _width(rng), "block": rng.choice([1, 1, 128]),
                "form": rng.choice(["rows", "transposed", "both"]), "dtype": rng.choice(["bf16", "fp16", "fp32"])}
    if kind == "linear":
        return {"kind": kind, "rows": _log_int(rng, 1, 4096), "n": _width(rng), "k": _width(rng),
                "block": rng.choice([1, 128, 128]), "dtype": dtype}
    if kind == "linear_grad":
        return {"kind": kind, "rows": _log_int(rng, 8, 4096), "n": _width(rng), "k": _width(rng), "dtype": dtype}
    if kind in ("grouped", "grouped_grad"):
        case = {"kind": kind, "rows": _log_int(rng, 1, 4096), "experts": rng.choice([2, 4, 7, 8, 16, 32, 64]),
                "n": min(4096, _width(rng)), "k": min(4096, _width(rng)), "dtype": dtype}
        while case["experts"] * case["n"] * case["k"] > 1 << 28:
            case["experts"] //= 2
        return case if kind == "grouped_grad" else dict(case, block=rng.choice([1, 128, 128]))
    sizes = [_log_int(rng, 1, 4_000_000) for _ in range(_log_int(rng, 1, 40))]
    return {"kind": kind, "sizes": ",".join(map(str, sizes)), "bits": rng.choice([8, 32]),
            "param": rng.choice(["fp32", "fp32", "bf16"]), "grad": rng.choice(["fp32", "bf16", "fp16"]),
            "copy": rng.random() < 0.5}


# ------------------------------------------------------------------------------------------------ the format, plainly


def _up(n, to=BLOCK):
    return -(-n // to) * to


def _power(e):
    """2^e of int32 exponents in [-126, 127] as float32."""
    return ((e + 127) << 23).view(torch.float32)


def _scale_bytes(amax):
    """The byte e + 127 of the least e >= -127 with amax <= 448 2^e."""
    m, ex = torch.frexp(amax)                         # amax = m 2^ex, 448 = 0.875 2^9
    return torch.where(amax == 0, 0, (ex - 9 + (m > 0.875).int() + 127).clamp(min=0)).int()


def _pad(x, rows, cols):
    return torch.nn.functional.pad(x, (0, cols - x.shape[-1], 0, rows - x.shape[-2]))


def _encode(x, block):
    """(codes float8 [..., R, C'], bytes uint8 [..., R / block, C' / 128]) of float32 x [..., R, C]."""
    *lead, R, C = x.shape
    g = _pad(x, _up(R, block), _up(C)).view(*lead, -1, block, _up(C) // BLOCK, BLOCK)
    byte = _scale_bytes(g.abs().amax((-3, -1)))
    codes = (g * _power(127 - byte)[..., :, None, :, None]).to(torch.float8_e4m3fn)
    return codes.view(*lead, -1, _up(C))[..., :R, :], byte.to(torch.uint8)


def _decode(codes, byte, block, cols):
    """float32 values [..., R, cols] of codes [..., R, C'] under bytes [..., R / block, C' / 128]."""
    *lead, R, C = codes.shape
    s = _power(byte.int() - 127).repeat_interleave(block, -2)[..., :R, :]
    return (codes.float().view(*lead, R, -1, BLOCK) * s[..., None]).view(*lead, R, C)[..., :cols]


def _round_trip(x, block=1):
    return _decode(*_encode(x.float(), block), block, x.shape[-1])


def _mix(x):
    """A hash of int32 words: shifts and odd multipliers (2^32 over the golden ratio, over the root of 3) in turn."""
    x = (x ^ ((x >> 16) & 0xFFFF)) * -1640531535
    x = (x ^ ((x >> 15) & 0x1FFFF)) * -1815266771
    return x ^ ((x >> 16) & 0xFFFF)


def _wrap(n):
    n &= 0xFFFFFFFF
    return n - (1 << 32) if n >> 31 else n


def _random20(state):
    """20 random bits for each state element, two of them, from (seed, step, tensor, index)."""
    first = torch.full((1,), _wrap(SEED ^ (state["step"] * 1779033703)), dtype=torch.int32, device="cuda")
    key = _mix(_mix(first) + state["ordinal"])        # of each block of 128
    h = _mix(state["index"] + key.repeat_interleave(BLOCK))
    return (h >> 12) & 0xFFFFF, (_mix(h + 1) >> 12) & 0xFFFFF


def _encode_stochastic(x, rnd, keep):
    """Blocks of 128 of float32 x, each value to one of the two codes beside it, upwards where rnd / 2^20 is not below
    the distance to the upper one.  keep: what is not zero does not become zero."""
    byte = _scale_bytes(x.view(-1, BLOCK).abs().amax(-1))
    s = (x.view(-1, BLOCK) * _power(127 - byte)[:, None]).view(-1)
    a = s.abs()
    large = ((a.view(torch.int32) + rnd) & ~0xFFFFF).view(torch.float32)
    small = torch.floor(a * 512.0 + rnd.float() * 2.0 ** -20) * 2.0 ** -9
    a = torch.where(a >= 2.0 ** -6, large, small)
    if keep:
        a = torch.where(x > 0, a.clamp(min=2.0 ** -9), a)
    return torch.copysign(a, s).to(torch.float8_e4m3fn), byte.to(torch.uint8)


# ------------------------------------------------------------------------------------------------ inputs


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rand(gen, shape, dtype=torch.float32):
    return torch.randn(shape, generator=gen, device="cuda").to(dtype)


def _activations(gen, rows, cols, dtype):
    """Rows of unequal size with a few large channels, as layers make them."""
    x = _rand(gen, (rows, cols)) * torch.exp(0.5 * _rand(gen, (rows, 1)))
    return (x * torch.where(torch.rand((cols,), generator=gen, device="cuda") < 0.01, 12.0, 1.0)).to(dtype)


def _starts(case):
    """starts [experts + 1] of rows spread unevenly, about one expert in five without any (the sizes are part of the
    case: a plain form that pads has to know the largest)."""
    rng = random.Random("%d %d %d %d" % (case["rows"], case["experts"], case["n"], case["k"]))
    share = [0.0 if rng.random() < 0.2 else rng.expovariate(1.0) for _ in range(case["experts"])]
    if not sum(share):
        share[-1] = 1.0
    at, total, starts = 0.0, sum(share), [0]
    for s in share:
        at += s
        starts.append(round(case["rows"] * at / total))
    starts[-1] = case["rows"]
    return starts


def _most(case):
    s = _starts(case)
    return max(b - a for a, b in zip(s, s[1:]))


def _live(case):
    s = _starts(case)
    return sum(b > a for a, b in zip(s, s[1:]))


def _sizes(case):
    return [int(n) for n in case["sizes"].split(",")]


def prepare(case, seed):
    gen = _gen(seed)
    kind, s = case["kind"], {"case": dict(case)}
    if kind == "quantize":
        s["x"] = _activations(gen, case["rows"], case["cols"], DTYPES[case["dtype"]])
        return s
    if kind != "adamw":
        dtype, lead = DTYPES[case["dtype"]], (case["experts"],) if "experts" in case else ()
        w = _rand(gen, (*lead, case["n"], case["k"])) * 0.02
        s["x"] = _activations(gen, case["rows"], case["k"], dtype)
        grad = kind.endswith("grad")
        if grad:                                      # the transposed weights, whose rows dX is summed over
            w = w.transpose(-1, -2).contiguous()
            s["dy"] = _activations(gen, case["rows"], case["n"], dtype) * 1e-3
        block = case.get("block", BLOCK)
        s["codes"], s["scales"] = _encode(w, block)
        s["codes"] = s["codes"].contiguous()
        if lead:
            s["starts"] = torch.tensor(_starts(case), dtype=torch.int32, device="cuda")
        if own:
            import paper_2405_03594_amd as spl

            s["weight"] = spl.Fp8Matrix.of(s["codes"], s["scales"], case["n"] if grad else case["k"], block)
        return s
    return _prepare_adamw(case, gen, s)


def _prepare_adamw(case, gen, s):
    sizes = _sizes(case)
    begin, total = [], 0
    for n in sizes:
        begin.append(total)
        total += _up(n)
    spans = [(a, n) for a, n in zip(begin, sizes)]

    def flat(x):                                      # tensors side by side, each from a multiple of 128 on, zeros between
        for (a, n) in spans:
            x[a + n:a + _up(n)] = 0
        return x

    pd, gd = DTYPES[case["param"]], DTYPES[case["grad"]]
    p = flat(_rand(gen, (total,)) * 0.02)
    size = torch.exp(_rand(gen, (total // BLOCK,))).repeat_interleave(BLOCK) * 1e-3
    g, m = flat(_rand(gen, (total,)) * size), flat(_rand(gen, (total,)) * size * 0.3)
    r = flat((_rand(gen, (total,)).abs() * 0.3 + 0.8) * size)
    s.update(p=p.to(pd), g=g.to(gd), grad_scale=torch.rand((1,), generator=gen, device="cuda") * 0.5 + 0.5, step=100)
    if case["copy"]:
        s["copy"] = p.to(torch.bfloat16)
    if case["bits"] == 32:
        s.update(m=m, v=r * r)
    else:
        for name, x in (("m", m), ("r", r)):
            codes, byte = _encode(x.view(-1, BLOCK), 1)
            s[name], s[name + "_scale"] = codes.reshape(-1), byte.reshape(-1)
        blocks = torch.tensor([_up(n) // BLOCK for n in sizes], device="cuda")
        s["ordinal"] = torch.arange(len(sizes), dtype=torch.int32, device="cuda").repeat_interleave(blocks)
        first = torch.tensor(begin, device="cuda").repeat_interleave(blocks * BLOCK)
        s["index"] = (torch.arange(total, device="cuda") - first).int()
    if own:
        import paper_2405_03594_amd as spl

        def parts(x):
            return [x[a:a + n] for a, n in spans]

        def states(name):
            if case["bits"] == 32:
                return parts(s["v" if name == "r" else name])
            return [spl.Fp8Vector(s[name][a:a + _up(n)].view(torch.uint8), s[name + "_scale"][a // BLOCK:(a + _up(n)) // BLOCK], n)
                    for a, n in spans]

        s["plan"] = spl.adamw_plan(parts(s["p"]), parts(s["g"]), states("m"), states("r"), weight_decay=DECAY,
                                   copies=parts(s["copy"]) if case["copy"] else None)
    return s


# ------------------------------------------------------------------------------------------------ one pass


def run(state):
    return _RUN[state["case"]["kind"]](state)


def _values(codes, byte):
    """Codes and scales as the numbers that they stand for."""
    return codes.view(torch.float8_e4m3fn), byte.view(torch.float8_e8m0fnu)


def _run_quantize(s):
    case, x = s["case"], s["x"]
    form, block = case["form"], case["block"]
    if own:
        import paper_2405_03594_amd as spl

        if form == "both":
            q, t = spl.quantize_fp8_both(x, block=block)
            got = [q, t]
        else:
            got = [spl.quantize_fp8(x, block=block, transposed=form == "transposed")]
        return [_values(q.codes, q.block_scales()) for q in got]
    wide = x.float()
    got = []
    if form != "transposed":
        got.append(_encode(wide, block))
    if form != "rows":
        got.append(_encode(wide.t(), block))
    return [_values(*q) for q in got]


def _run_linear(s):
    case = s["case"]
    if own:
        import paper_2405_03594_amd as spl

        return spl.linear_fp8(s["x"], s["weight"])
    w = _decode(s["codes"], s["scales"], case["block"], case["k"])
    return (_round_trip(s["x"]) @ w.t()).to(s["x"].dtype)


def _run_linear_grad(s):
    case = s["case"]
    if own:
        import paper_2405_03594_amd as spl

        return spl.linear_fp8_grad(s["dy"], s["x"], s["weight"])
    wt = _decode(s["codes"], s["scales"], BLOCK, case["n"])
    dx = (_round_trip(s["dy"]) @ wt.t()).to(s["x"].dtype)
    dyt, xt = _round_trip(s["dy"].t()), _round_trip(s["x"].t())
    return dx, dyt @ xt.t()


def _spread(x, starts, most):
    """(rows [experts, most', C] float32 with zeros behind an expert's rows, the place of each row of x)."""
    E, P = starts.numel() - 1, _up(most)
    row = torch.arange(x.shape[0], dtype=torch.int32, device=x.device)
    e = torch.searchsorted(starts[1:], row, right=True)
    place = e * P + (row - starts[e])
    out = torch.zeros((E * P, x.shape[1]), device=x.device)
    out[place] = x.float()
    return out.view(E, P, -1), place


def _run_grouped(s):
    case = s["case"]
    if own:
        import paper_2405_03594_amd as spl

        return spl.linear_fp8_grouped(s["x"], s["weight"], s["starts"])
    w = _decode(s["codes"], s["scales"], case["block"], case["k"])
    x, place = _spread(_round_trip(s["x"]), s["starts"], _most(case))
    y = torch.bmm(x, w.transpose(1, 2).contiguous())
    return y.view(-1, case["n"])[place].to(s["x"].dtype)


def _run_grouped_grad(s):
    case = s["case"]
    if own:
        import paper_2405_03594_amd as spl

        return spl.linear_fp8_grouped_grad(s["dy"], s["x"], s["weight"], s["starts"])
    wt = _decode(s["codes"], s["scales"], BLOCK, case["n"])
    dy, place = _spread(_round_trip(s["dy"]), s["starts"], _most(case))
    dx = torch.bmm(dy, wt.transpose(1, 2).contiguous()).view(-1, case["k"])[place].to(s["x"].dtype)
    dyt, _ = _spread(s["dy"], s["starts"], _most(case))
    xt, _ = _spread(s["x"], s["starts"], _most(case))
    dyt, xt = (_round_trip(t.transpose(1, 2).contiguous()) for t in (dyt, xt))
    return dx, torch.bmm(dyt, xt.transpose(1, 2).contiguous())


def _run_adamw(s):
    case = s["case"]
    s["step"] += 1
    if own:
        import paper_2405_03594_amd as spl

        spl.adamw_step(s["plan"], lr=LR, betas=BETAS, eps=EPS, step=s["step"], grad_scale=s["grad_scale"], seed=SEED)
    else:
        b1, b2 = BETAS
        eight = case["bits"] == 8
        g = s["g"].float() * s["grad_scale"]
        m = _decode(s["m"].view(-1, BLOCK), s["m_scale"].view(-1, 1), 1, BLOCK).view(-1) if eight else s["m"]
        if eight:
            r = _decode(s["r"].view(-1, BLOCK), s["r_scale"].view(-1, 1), 1, BLOCK).view(-1)
            v = r * r
        else:
            v = s["v"]
        m = m * b1 + g * (1.0 - b1)
        v = v * b2 + (g * g) * (1.0 - b2)
        root = torch.sqrt(v)
        t = s["step"]
        p = s["p"].float() * (1.0 - LR * DECAY) - (LR / (1.0 - b1 ** t)) * (m / (root * (1.0 - b2 ** t) ** -0.5 + EPS))
        s["p"].copy_(p)
        if case["copy"]:
            s["copy"].copy_(p)
        if eight:
            u, w = _random20(s)
            for name, x, bits, keep in (("m", m, u, False), ("r", root, w, True)):
                codes, byte = _encode_stochastic(x, bits, keep)
                s[name].copy_(codes)
                s[name + "_scale"].copy_(byte)
        else:
            s["m"].copy_(m)
            s["v"].copy_(v)
    out = [s["p"]] + ([s["copy"]] if case["copy"] else [])
    if case["bits"] == 8:
        return out + [_values(s[name], s[name + "_scale"]) for name in ("m", "r")]
    return out + [s["m"], s["v"]]


_RUN = {"quantize": _run_quantize, "linear": _run_linear, "linear_grad": _run_linear_grad, "grouped": _run_grouped,
        "grouped_grad": _run_grouped_grad, "adamw": _run_adamw}


# ------------------------------------------------------------------------------------------------ what a pass needs


def _held(rows, cols, block):
    """Bytes of a matrix in 8 bits."""
    return rows * cols + -(-rows // block) * -(-cols // BLOCK)


def work(case):
    kind = case["kind"]
    if kind == "quantize":
        n = case["rows"] * case["cols"]
        held = {"rows": _held(case["rows"], case["cols"], case["block"]),
                "transposed": _held(case["cols"], case["rows"], case["block"])}
        held["both"] = held["rows"] + held["transposed"]
        return {"bytes": n * BYTES[case["dtype"]] + held[case["form"]], "flops": 4 * n}
    if kind == "adamw":
        n = sum(_sizes(case))
        state = 8 if case["bits"] == 32 else 2 + 2 / BLOCK
        each = 2 * BYTES[case["param"]] + BYTES[case["grad"]] + 2 * state + (2 if case["copy"] else 0)
        return {"bytes": n * each, "flops": 16 * n}
    rows, n, k, b = case["rows"], case["n"], case["k"], BYTES[case["dtype"]]
    experts = _live(case) if "experts" in case else 1
    weights = experts * _held(n, k, case.get("block", BLOCK))
    if kind.endswith("grad"):
        whole = case.get("experts", 1)                # an expert without rows has a gradient of zeros
        return {"bytes": rows * (n + 2 * k) * b + weights + 4 * whole * n * k, "flops": 4 * rows * n * k}
    return {"bytes": rows * (n + k) * b + weights, "flops": 2 * rows * n * k}


# ------------------------------------------------------------------------------------------------ in 64 bits


def _nearest64(s):
    """The 8-bit float next to each float64, ties to even."""
    k = torch.floor(torch.log2(s.abs().clamp(min=2.0 ** -40)))
    k = torch.where(s.abs() >= torch.exp2(k + 1), k + 1, torch.where(s.abs() < torch.exp2(k), k - 1, k)).clamp(min=-6)
    step = torch.exp2(k - 3)
    return torch.round(s / step) * step


def _exponent64(amax):
    e = torch.floor(torch.log2(amax.clamp(min=1e-300) / MOST_CODE)) - 1
    for _ in range(3):
        e = torch.where(amax > MOST_CODE * torch.exp2(e), e + 1, e)
    return torch.where(amax == 0, -127.0, e.clamp(min=-127.0))


def _coded64(x, block=1):
    """(codes, exponents, values) of x [R, C] in float64: what the format holds of it."""
    x = x.double()
    R, C = x.shape
    g = torch.zeros((_up(R, block), _up(C)), dtype=torch.float64, device=x.device)
    g[:R, :C] = x
    g = g.view(-1, block, _up(C) // BLOCK, BLOCK)
    e = _exponent64(g.abs().amax((1, 3)))
    s = torch.exp2(e)[:, None, :, None]
    c = _nearest64(g / s)
    return c.view(-1, _up(C))[:R], e, (c * s).view(-1, _up(C))[:R, :C]


def _held64(x, block=1):
    return _coded64(x, block)[2]


def _weights64(s, block, cols, at=None):
    c, b = (s["codes"], s["scales"]) if at is None else (s["codes"][at], s["scales"][at])
    e = torch.exp2(b.double() - 127.0).repeat_interleave(block, 0)[:c.shape[0]].repeat_interleave(BLOCK, 1)
    return (c.double() * e)[:, :cols]


def exact(case, seed):
    kind, s = case["kind"], prepare(case, seed)
    if kind == "quantize":
        sides = [s["x"]] * (case["form"] != "transposed") + [s["x"].t()] * (case["form"] != "rows")
        return [[c, torch.exp2(e)] for c, e, _ in (_coded64(x, case["block"]) for x in sides)]
    if kind == "linear":
        return _held64(s["x"]) @ _weights64(s, case["block"], case["k"]).t()
    if kind == "linear_grad":
        return (_held64(s["dy"]) @ _weights64(s, BLOCK, case["n"]).t(), _held64(s["dy"].t()) @ _held64(s["x"].t()).t())
    if kind == "adamw":
        return _exact_adamw(case, s)
    at = _starts(case)
    width = case["n"] if kind == "grouped" else case["k"]
    rows = torch.zeros((case["rows"], width), dtype=torch.float64, device="cuda")
    x = s["x"] if kind == "grouped" else s["dy"]
    dw = []
    for e, (a, b) in enumerate(zip(at, at[1:])):
        if b > a:
            cols = case["k"] if kind == "grouped" else case["n"]
            rows[a:b] = _held64(x[a:b]) @ _weights64(s, case.get("block", BLOCK), cols, e).t()
        if kind == "grouped_grad":
            zero = torch.zeros((case["n"], case["k"]), dtype=torch.float64, device="cuda")
            dw.append(_held64(s["dy"][a:b].t()) @ _held64(s["x"][a:b].t()).t() if b > a else zero)
    return rows if kind == "grouped" else (rows, torch.stack(dw))


def _hash64(x):
    """_mix on 32-bit words held in int64."""
    x = ((x ^ (x >> 16)) * 2654435761) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 2479700525) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _exact_adamw(case, s):
    b1, b2 = BETAS
    t = s["step"] + 1
    g = s["g"].double() * s["grad_scale"].double()
    if case["bits"] == 8:
        m, r = (s[n].double() * torch.exp2(s[n + "_scale"].double() - 127.0).repeat_interleave(BLOCK) for n in ("m", "r"))
        v = r * r
    else:
        m, v = s["m"].double(), s["v"].double()
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    p = s["p"].double() * (1 - LR * DECAY) - LR * (m / (1 - b1 ** t)) / (torch.sqrt(v / (1 - b2 ** t)) + EPS)
    out = [p] + ([p] if case["copy"] else [])
    if case["bits"] == 32:
        return out + [m, v]
    word = (SEED ^ (t * 1779033703)) & 0xFFFFFFFF
    key = _hash64((_hash64(torch.tensor([word], device="cuda")) + s["ordinal"].long()) & 0xFFFFFFFF)
    h = _hash64((s["index"].long() + key.repeat_interleave(BLOCK)) & 0xFFFFFFFF)
    for x, bits in ((m, h >> 12), (torch.sqrt(v), _hash64((h + 1) & 0xFFFFFFFF) >> 12)):
        e = _exponent64(x.view(-1, BLOCK).abs().amax(-1))
        c = x / torch.exp2(e).repeat_interleave(BLOCK)
        k = torch.floor(torch.log2(c.abs().clamp(min=2.0 ** -60)))
        step = torch.exp2(k.clamp(min=-6) - 3)
        a = torch.floor(c.abs() / step + bits.double() / 2 ** 20) * step
        if x is not m:
            a = torch.where(x > 0, a.clamp(min=2.0 ** -9), a)
        out.append([torch.copysign(a, c), torch.exp2(e)])
    return out

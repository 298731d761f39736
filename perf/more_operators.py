"""What a training step over the leaves of boosted trees adds with a normalised hidden row and an optimizer that keeps
states, case by case.

Layer norm forward (`ln`) and backward (`ln_grad`, with the sums of the weight's and bias's gradients over the rows), and
an AdamW step over many tensors at once (`adamw`), with states in 32 bits or in 8 bits per element, the clipping
factor applied on the way and 16-bit copies of the parameters written with them.  `run` computes them in plain torch
operations in 32 bits, or, with `own` set, through this repository's calls.
"""
import functools
import itertools
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
WIDTH = {"f32": 4, "bf16": 2, "f16": 2, "none": 0}
BLOCK = 256             # elements of a tensor that share an exponent where states have 8 bits
CODES_M, CODES_V = 897, 769   # code c > 0 is the float with bits (c + this) << 20, times the block's power of two
BETAS, EPS, DECAY, LR, SEED = (0.9, 0.999), 1e-8, 0.01, 1e-3, 0x1234567890AB


@functools.lru_cache(maxsize=1)
def _context():
    """The handle a program keeps for all its calls."""
    from paper_2207_09682_b200 import binding
    return binding.Context(binding.make_params())


# ---- cases --------------------------------------------------------------------------------------

def listed():
    return [
        # scoring one row; latency
        dict(name="norm of one row", kind="ln", rows=1, dim=256, type="bf16", weights="f32", pad=0),
        # odd sizes, the rows a column slice of a wider matrix
        dict(name="norm, slice", kind="ln", rows=4099, dim=770, type="f32", weights="f32", pad=30),
        # the hidden rows of a training batch
        dict(name="norm, batch", kind="ln", rows=65536, dim=256, type="bf16", weights="f32", pad=0),
        # wide rows
        dict(name="norm, wide", kind="ln", rows=16384, dim=8192, type="bf16", weights="bf16", pad=0),
        # gradient of a small model; latency
        dict(name="norm grad, small", kind="ln_grad", rows=64, dim=16, type="f32", weights="f32", pad=0),
        # gradient at odd sizes, half precision: rows that start anywhere
        dict(name="norm grad, odd", kind="ln_grad", rows=7777, dim=129, type="f16", weights="f32", pad=0),
        # gradient of a large training batch
        dict(name="norm grad, batch", kind="ln_grad", rows=65536, dim=1024, type="bf16", weights="f32", pad=0),
        # parameters of a small model, states in 32 bits; latency
        dict(name="adamw, small", kind="adamw", tensors=6, elements=60011, bits=32, type="f32", grads="f32", copies="none", clipped=False),
        # hundreds of parameters of ragged sizes, clipped, 16-bit copies for the products
        dict(name="adamw, large", kind="adamw", tensors=300, elements=200_000_000, bits=32, type="f32", grads="f32", copies="bf16", clipped=True),
        # the same kinds with states in 8 bits: odd sizes, half-precision gradients with a loss scale
        dict(name="adamw 8 bit, odd", kind="adamw", tensors=37, elements=1_000_003, bits=8, type="f32", grads="f16", copies="f16", clipped=True),
        # table of 25500 leaves x 256 and classifier of 65536 classes x 1024, states in 8 bits
        dict(name="adamw 8 bit, large", kind="adamw", tensors=3, elements=73_702_400, bits=8, type="f32", grads="bf16", copies="bf16", clipped=True),
        # parameters kept in 16 bits only
        dict(name="adamw 8 bit, bf16", kind="adamw", tensors=100, elements=30_000_001, bits=8, type="bf16", grads="bf16", copies="none", clipped=False),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["ln", "ln_grad", "adamw", "adamw"])
    if kind == "adamw":
        tensors, bits = _log(rng, 1, 1000), rng.choice([8, 32])
        return dict(kind=kind, tensors=tensors, elements=max(tensors, _log(rng, 1000, 70_000_000 if bits == 8 else 150_000_000)), bits=bits, type=rng.choice(["f32", "f32", "bf16", "f16"]),
                    grads=rng.choice(["f32", "bf16", "f16"]), copies=rng.choice(["none", "bf16", "f16"]), clipped=rng.random() < 0.5)
    rows, dim = _log(rng, 1, 65536), _log(rng, 8, 8192)
    if rng.random() < 0.5:
        dim = -(-dim // 8) * 8      # hidden sizes are mostly multiples of 8
    rows = min(rows, 60_000_000 // dim)
    kind_of = rng.choice(["f32", "bf16", "f16"])
    return dict(kind=kind, rows=rows, dim=dim, type=kind_of, weights=rng.choice(["f32", kind_of]), pad=rng.choice([0, 0, 0, 1, 24]))


# ---- inputs -------------------------------------------------------------------------------------

def _randn(shape, gen, dtype=torch.float32):
    return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)


def _sizes(case):
    """Ragged sizes that add up to the case's elements, the same for every seed: most of them small, a few large."""
    tensors, elements = case["tensors"], case["elements"]
    w = torch.rand(tensors, generator=torch.Generator().manual_seed(tensors), dtype=torch.float64).pow(6)
    n = (w / w.sum() * (elements - tensors)).long() + 1
    n[0] += elements - int(n.sum())
    return n.tolist()


def _views(flat, sizes, per=1):
    """Tensors of these sizes inside `flat`, each from a multiple of BLOCK elements on; `per`: elements that share an entry."""
    at = [0, *itertools.accumulate(-(-n // BLOCK) * (BLOCK // per) for n in sizes)]
    return [flat[a:a + -(-n // per)] for a, n in zip(at, sizes)]


def _pack_nearest(x, offset):
    """Codes [n] and exponents [n / BLOCK] of the values x >= 0, rounded to the nearest."""
    blocks = x.view(-1, BLOCK)
    exponent = (blocks.amax(1).view(torch.int32) >> 23).clamp(min=1)
    scaled = torch.ldexp(blocks, (127 - exponent).unsqueeze(1))
    code = ((scaled.view(torch.int32) + (1 << 19)) >> 20) - offset
    code = torch.where(scaled > 0, code.clamp(min=1), 0)
    return code.to(torch.uint8).view(-1), exponent.to(torch.uint8)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind, s = case["kind"], {"case": case}
    dtype = TYPES[case["type"]]
    if kind in ("ln", "ln_grad"):
        n, d, pad, wtype = case["rows"], case["dim"], case["pad"], TYPES[case["weights"]]
        # sums of embeddings: rows of different sizes and offsets
        size = torch.rand((n, 1), generator=gen, device="cuda").mul_(1.5).add_(0.1)
        s["x"] = _randn((n, d + pad), gen).add_(0.3 * _randn((n, 1), gen)).mul_(size).to(dtype)[:, :d]
        s["weight"] = (1.0 + 0.2 * _randn(d, gen)).to(wtype)
        if kind == "ln":
            s["bias"] = (0.1 * _randn(d, gen)).to(wtype)
        else:
            s["grad"] = (0.1 * _randn((n, d + pad), gen)).to(dtype)[:, :d]
            x = s["x"].double()
            s["mean"] = x.mean(1).float()
            s["rstd"] = (x.var(1, unbiased=False) + 1e-5).rsqrt().float()
        return s
    # parameters, gradients and states lie in one buffer each; the gaps between the tensors hold zeros
    sizes = _sizes(case)
    total = sum(-(-n // BLOCK) * BLOCK for n in sizes)
    starts = torch.tensor([0, *itertools.accumulate(-(-n // BLOCK) * BLOCK for n in sizes)][:-1], device="cuda")
    edge = torch.zeros(total + 1, dtype=torch.int8, device="cuda")
    edge[starts] += 1
    edge.index_add_(0, starts + torch.tensor(sizes, device="cuda"), torch.full((len(sizes),), -1, dtype=torch.int8, device="cuda"))
    inside = edge[:total].cumsum(0, dtype=torch.int8) > 0
    scale = 1024.0 if case["grads"] == "f16" else 1.0
    # sizes of gradients differ from block to block, and a part of the elements has had none so far
    size = torch.exp(1.5 * _randn(total // BLOCK, gen)).mul_(1e-3).repeat_interleave(BLOCK)
    size *= inside & (torch.rand(total, generator=gen, device="cuda") > 0.02)
    s["flat_grad"] = (size * _randn(total, gen) * scale).to(TYPES[case["grads"]])
    s["flat_param"] = (0.05 * _randn(total, gen) * inside).to(dtype)
    m = 0.3 * size * _randn(total, gen)
    v = size.square_().mul_(torch.rand(total, generator=gen, device="cuda").add_(0.5))
    if case["bits"] == 32:
        s["flat_m"], s["flat_v"], s["flat_exponents"] = m, v, None
    else:
        code, exponent_m = _pack_nearest(m.abs(), CODES_M)
        s["flat_m"] = torch.where((m < 0) & (code > 0), code + 128, code)
        s["flat_v"], exponent_v = _pack_nearest(v, CODES_V)
        s["flat_exponents"] = torch.stack([exponent_m, exponent_v], 1).contiguous()
        s["exponents"] = _views(s["flat_exponents"], sizes, BLOCK)
    s["flat_copy"] = None if case["copies"] == "none" else torch.zeros(total, dtype=TYPES[case["copies"]], device="cuda")
    for name in ("param", "grad", "m", "v", "copy"):
        s[name] = None if s["flat_" + name] is None else _views(s["flat_" + name], sizes)
    s["norm"] = s["flat_grad"].double().square().sum().sqrt().float().reshape(1)
    s["max_norm"] = float(s["norm"]) / scale * (0.25 if case["clipped"] else 4.0)
    s["loss_scale"], s["step"] = scale, 1000
    return s


# ---- the operators ------------------------------------------------------------------------------

def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"ln": _own_ln, "ln_grad": _own_ln_grad, "adamw": _own_adamw}[kind](state)
    return {"ln": _ln, "ln_grad": _ln_grad, "adamw": _adamw}[kind](state)


def _own_ln(s):
    r = _context().layer_norm(s["x"], s["weight"], s["bias"])
    return {"out": r.out, "mean": r.mean, "rstd": r.rstd}


def _own_ln_grad(s):
    gx, gw, gb = _context().layer_norm_backward(s["grad"], s["x"], s["mean"], s["rstd"], s["weight"])
    return {"grad_x": gx, "grad_weight": gw, "grad_bias": gb}


def _own_adamw(s):
    c, packed = _context(), s["case"]["bits"] == 8
    c.adamw(s["param"], s["grad"], s["m"], s["v"], s["step"], LR, betas=BETAS, eps=EPS, weight_decay=DECAY, exponents=s["exponents"] if packed else None,
            copies=s["copy"], norm=s["norm"], max_norm=s["max_norm"], loss_scale=s["loss_scale"], seed=SEED)
    out = {"params": s["flat_param"], "copies": s["flat_copy"]}
    if not packed:
        return {**out, "m": s["flat_m"], "v": s["flat_v"]}
    (m,), (v,) = c.adamw_values([s["flat_m"]], [s["flat_v"]], [s["flat_exponents"]], dtype=torch.bfloat16)
    return {**out, "m": m, "v": v}


def _ln(s):
    x = s["x"].float()
    mean = x.sum(1, keepdim=True) / x.shape[1]
    x = x - mean
    rstd = 1.0 / ((x * x).sum(1, keepdim=True) / x.shape[1] + 1e-5).sqrt()
    out = x * rstd * s["weight"].float() + s["bias"].float()
    return {"out": out.to(s["x"].dtype), "mean": mean.squeeze(1), "rstd": rstd.squeeze(1)}


def _ln_grad(s):
    g, rstd, d = s["grad"].float(), s["rstd"].unsqueeze(1), s["x"].shape[1]
    xh = (s["x"].float() - s["mean"].unsqueeze(1)) * rstd
    wg = g * s["weight"].float()
    gx = (wg - wg.sum(1, keepdim=True) / d - xh * ((wg * xh).sum(1, keepdim=True) / d)) * rstd
    wtype = s["weight"].dtype
    return {"grad_x": gx.to(s["x"].dtype), "grad_weight": (g * xh).sum(0).to(wtype), "grad_bias": g.sum(0).to(wtype)}


def _mix(x):
    """A hash of 32-bit numbers (held in 64 bits)."""
    x = ((x ^ (x >> 16)) * 0x9E3779B9) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0xBB67AE85) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random(blocks, step, device):
    """32 random bits for each element: a hash of the seed, the step, the block's number and the element's place in it."""
    key = torch.tensor([SEED & 0xFFFFFFFF], device=device)
    key = _mix(_mix(_mix(key) ^ (SEED >> 32)) ^ step)
    return _mix(_mix(key ^ torch.arange(blocks, device=device)).unsqueeze(1) ^ torch.arange(BLOCK, device=device))


def _value(code, exponent, offset):
    """What codes [blocks, BLOCK] stand for (the exponents are 1 to 254 here)."""
    one = torch.where(code > 0, (code + offset) << 20, 0).view(torch.float32)
    return one * ((exponent.int() << 23).view(torch.float32)).unsqueeze(1)


def _pack(x, random16, offset, keep):
    """Codes and exponents of x >= 0 [blocks, BLOCK], rounded up with the probability that keeps the mean; `keep`: what is
    above zero stays above zero."""
    exponent = x.amax(1).view(torch.int32) >> 23
    scaled = x * (((254 - exponent) << 23).view(torch.float32)).unsqueeze(1)
    r = (random16.int() << 4) + 8
    code = ((scaled.view(torch.int32) + r) >> 20) - offset
    least = 1.25 * 2.0 ** (((offset + 1) >> 3) - 127)
    small = scaled > 0.0 if keep else r.float() * (least * 2.0 ** -20) < scaled
    return torch.where(scaled < least, small.int(), code), exponent


def _adamw(s):
    case, p = s["case"], s["flat_param"].float()
    coef = (s["max_norm"] * s["loss_scale"] / s["norm"].double()).clamp(max=1.0) / s["loss_scale"]
    g = s["flat_grad"].float() * coef.float()
    b1, b2 = BETAS
    if case["bits"] == 32:
        m, v = s["flat_m"], s["flat_v"]
    else:
        g = g.view(-1, BLOCK)
        raw, exponents = s["flat_m"].int().view(-1, BLOCK), s["flat_exponents"]
        m = _value(raw & 127, exponents[:, 0], CODES_M)
        m = torch.where(raw > 127, -m, m)
        v = _value(s["flat_v"].int().view(-1, BLOCK), exponents[:, 1], CODES_V)
    m = m * b1 + g * (1 - b1)
    v = v * b2 + (g * (1 - b2)) * g
    step = (m / (1 - b1 ** s["step"]) / ((v / (1 - b2 ** s["step"])).sqrt() + EPS)).view(-1)
    p = p * (1 - LR * DECAY) - LR * step
    s["flat_param"].copy_(p)
    if s["flat_copy"] is not None:
        s["flat_copy"].copy_(p)
    out = {"params": s["flat_param"], "copies": s["flat_copy"]}
    if case["bits"] == 32:
        s["flat_m"].copy_(m)
        s["flat_v"].copy_(v)
        return {**out, "m": s["flat_m"], "v": s["flat_v"]}
    random = _random(len(m), s["step"], m.device)
    code, exponent_m = _pack(m.abs(), random >> 16, CODES_M, False)
    s["flat_m"].copy_(torch.where((m < 0) & (code > 0), code + 128, code).view(-1))
    value_m = torch.where(m < 0, -1.0, 1.0) * _value(code, exponent_m, CODES_M)
    code, exponent_v = _pack(v, random & 0xFFFF, CODES_V, True)
    s["flat_v"].copy_(code.view(-1))
    exponents.copy_(torch.stack([exponent_m, exponent_v], 1))
    return {**out, "m": value_m.view(-1).bfloat16(), "v": _value(code, exponent_v, CODES_V).view(-1).bfloat16()}


# ---- the definition in 64 bits ------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "ln":
        x = s["x"].double()
        var, mean = torch.var_mean(x, 1, unbiased=False)
        rstd = (var + 1e-5).pow(-0.5)
        return {"out": torch.addcmul(s["bias"].double(), (x - mean[:, None]) * rstd[:, None], s["weight"].double()), "mean": mean, "rstd": rstd}
    if case["kind"] == "ln_grad":
        # as the derivative of (x - mean) / sqrt(var + eps) along every input, with the given mean and rstd
        g, d = s["grad"].double(), case["dim"]
        xh = (s["x"].double() - s["mean"].double()[:, None]).mul_(s["rstd"].double()[:, None])
        wg = g * s["weight"].double()
        along = torch.einsum("nd,nd->n", wg, xh) / d
        gx = (wg - wg.mean(1, keepdim=True) - xh * along[:, None]).mul_(s["rstd"].double()[:, None])
        return {"grad_x": gx, "grad_weight": torch.einsum("nd,nd->d", g, xh), "grad_bias": torch.einsum("nd->d", g)}
    b1, b2 = BETAS
    factor = min(1.0, s["max_norm"] * s["loss_scale"] / float(s["norm"])) / s["loss_scale"]
    g = s["flat_grad"].double() * factor
    if case["bits"] == 32:
        m, v = s["flat_m"].double(), s["flat_v"].double()
    else:
        m, v = _exact_value(s["flat_m"], s["flat_exponents"][:, 0], 897, True), _exact_value(s["flat_v"], s["flat_exponents"][:, 1], 769, False)
    m = torch.lerp(g, m, b1)
    v = torch.lerp(g * g, v, b2)
    p = s["flat_param"].double()
    p = p - LR * DECAY * p - LR * (m / (1 - b1 ** s["step"])) / ((v / (1 - b2 ** s["step"])).sqrt() + EPS)
    out = {"params": p, "copies": None if s["flat_copy"] is None else p}
    if case["bits"] == 8:
        m, v = _exact_rounded(m, s["step"], 16, 897, False), _exact_rounded(v, s["step"], 0, 769, True)
    return {**out, "m": m, "v": v}


def _exact_value(raw, exponent, offset, signed):
    code = (raw.long() & 127 if signed else raw.long()) + offset
    value = torch.ldexp((8 + code % 8).double() / 8, code // 8 - 127)
    value[code == offset] = 0.0
    if signed:
        value = torch.where(raw > 127, -value, value)
    return torch.ldexp(value.view(-1, BLOCK), exponent.long()[:, None] - 127).view(-1)


def _exact_rounded(x, step, shift, offset, keep):
    """Stochastic rounding to the codes' values, from their definition: the two neighbours and the place between them."""
    def mix(k):
        k = (k ^ k >> 16) * 0x9E3779B9 % 2 ** 32
        k = (k ^ k >> 15) * 0xBB67AE85 % 2 ** 32
        return k ^ k >> 16
    key = mix(mix(mix(SEED % 2 ** 32) ^ SEED >> 32) ^ step)
    at = torch.arange(x.numel(), device=x.device)
    random = mix(mix(key ^ at // BLOCK) ^ at % BLOCK)
    random = ((random >> shift) % 2 ** 16).double().add_(0.5).mul_(2.0 ** -16)       # in (0, 1)
    size = x.abs()
    exponent = torch.frexp(size.view(-1, BLOCK).amax(1)).exponent - 1                # 2^exponent <= largest < 2^(exponent + 1)
    exponent = exponent.clamp(min=-127).repeat_interleave(BLOCK)
    size = torch.ldexp(size, -exponent)
    least = 1.25 * 2.0 ** ((offset + 1) // 8 - 127)
    gap = torch.ldexp(torch.ones_like(size), torch.frexp(size).exponent - 4)        # between neighbours: an eighth of the power of two below
    down = torch.floor(size / gap) * gap
    near = down + gap * (size - down + gap * random >= gap)
    low = least * ((size > 0) if keep else (random * least < size))
    near = torch.where(size < least, low, near)
    return torch.ldexp(near, exponent) * torch.sign(x)


# ---- what a pass cannot do without --------------------------------------------------------------

def work(case):
    if case["kind"] == "adamw":
        n, packed = case["elements"], case["bits"] == 8
        each = 2 * WIDTH[case["type"]] + WIDTH[case["grads"]] + WIDTH[case["copies"]] + (4 + 4 if packed else 16)   # 8 bits: codes read and written, values returned
        return {"bytes": n * each + (4 * n // BLOCK if packed else 0), "flops": (40 if packed else 16) * n}
    n, d, w = case["rows"], case["dim"], WIDTH[case["type"]]
    if case["kind"] == "ln":
        return {"bytes": 2 * w * n * d + 8 * n + 2 * d * WIDTH[case["weights"]], "flops": 8 * n * d}
    return {"bytes": 3 * w * n * d + 8 * n + 3 * d * WIDTH[case["weights"]], "flops": 14 * n * d}

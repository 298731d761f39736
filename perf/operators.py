"""What the training step of a softmax classifier over the leaves of boosted trees is made of, case by case.

Four operators: the embedding bag over leaf numbers (`embed`) and its gradient (`embed_grad`), the softmax
cross entropy over many classes without kept logits, forward alone (`loss`) and with its gradients (`train`),
and the clipping of gradients by their global norm (`clip`).  `run` computes them in plain torch operations in
32 bits, or, with `own` set, through this repository's calls.
"""
import functools
import itertools
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
WIDTH = {"f32": 4, "bf16": 2, "f16": 2}


@functools.lru_cache(maxsize=1)
def _context():
    """The handle a program keeps for all its calls."""
    from paper_2207_09682_b200 import binding
    return binding.Context(binding.make_params())


# ---- cases --------------------------------------------------------------------------------------

def listed():
    return [
        # scoring one row: its leaf in each of 100 trees of 255 leaves; latency
        dict(name="embed one row", kind="embed", rows=1, bag=100, entries=25500, dim=64, type="bf16", wide_index=False, pad=0),
        # plain lookup of one token per row in a table that is a column slice of a wider one, odd sizes
        dict(name="embed tokens, slice", kind="embed", rows=4099, bag=1, entries=50021, dim=770, type="f32", wide_index=True, pad=30),
        # a training batch over 100 trees of 255 leaves
        dict(name="embed batch", kind="embed", rows=65536, bag=100, entries=25500, dim=256, type="bf16", wide_index=False, pad=0),
        # gradient of a small model: 10 trees of 31 leaves; latency
        dict(name="embed grad, small", kind="embed_grad", rows=64, bag=10, entries=310, dim=16, type="f32", wide_index=False, pad=0),
        # gradient at odd sizes, 64-bit tokens, half precision
        dict(name="embed grad, odd", kind="embed_grad", rows=5003, bag=37, entries=4699, dim=100, type="f16", wide_index=True, pad=0),
        # gradient of the training batch
        dict(name="embed grad, batch", kind="embed_grad", rows=65536, bag=100, entries=25500, dim=256, type="bf16", wide_index=False, pad=0),
        # loss of a single row against 32000 classes; the weights are read once
        dict(name="loss of one row", kind="loss", rows=1, classes=32000, dim=512, type="bf16", bias=False, masked=0.0),
        # evaluation of a held-out set with a thousand classes
        dict(name="loss, evaluation", kind="loss", rows=20000, classes=1000, dim=256, type="f16", bias=True, masked=0.0),
        # a training step at odd sizes, a third of the rows without a label, half precision with a loss scale
        dict(name="train, odd", kind="train", rows=777, classes=10007, dim=129, type="f16", bias=True, masked=0.3),
        # a large training step
        dict(name="train, large", kind="train", rows=8192, classes=65536, dim=1024, type="bf16", bias=False, masked=0.1),
        # the gradients of a small model, below the bound, in place: the norm alone
        dict(name="clip, small", kind="clip", tensors=6, elements=60011, types="f32", clipped=False),
        # hundreds of gradients of mixed types and ragged sizes, above the bound
        dict(name="clip, large", kind="clip", tensors=300, elements=400_000_000, types="mixed", clipped=True),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["embed", "embed_grad", "loss", "train", "clip"])
    if kind in ("embed", "embed_grad"):
        bag = 1 if rng.random() < 0.3 else _log(rng, 2, 128)
        rows = _log(rng, 1, 65536)
        dim = _log(rng, 1, 1024)
        entries = _log(rng, 100, 200_000) if bag == 1 else bag * _log(rng, 4, 255)
        dim = max(1, min(dim, 65536 * 100 * 256 // (rows * bag), 25500 * 256 * 8 // entries))
        return dict(kind=kind, rows=rows, bag=bag, entries=entries, dim=dim, type=rng.choice(["f32", "bf16", "f16"]),
                    wide_index=rng.random() < 0.5, pad=rng.choice([0, 0, 1, 24]))
    if kind in ("loss", "train"):
        return dict(kind=kind, rows=_log(rng, 1, 8192), classes=_log(rng, 2, 65536), dim=_log(rng, 8, 1024), type=rng.choice(["bf16", "f16"]),
                    bias=rng.random() < 0.5, masked=rng.choice([0.0, 0.1, 0.5, 0.9]))
    tensors = _log(rng, 1, 1000)
    return dict(kind=kind, tensors=tensors, elements=max(tensors, _log(rng, 1000, 300_000_000)), types=rng.choice(["f32", "bf16", "mixed"]),
                clipped=rng.random() < 0.5)


# ---- inputs -------------------------------------------------------------------------------------

def _tokens(case, gen):
    """Leaf numbers: tree k holds entries [k * L, (k + 1) * L), and its rows crowd into few of its leaves; about one
    in fifty is missing (-1: a tree that a row has no leaf in).  One token per row: skewed over the whole table."""
    rows, bag, n = case["rows"], case["bag"], case["entries"]
    u = torch.rand((rows, bag), generator=gen, device="cuda", dtype=torch.float64)
    leaves = max(1, n // bag)
    tok = (u.pow(3) * leaves).long().clamp_(max=leaves - 1) + leaves * torch.arange(bag, device="cuda")
    tok[torch.rand((rows, bag), generator=gen, device="cuda") < 0.02] = -1
    tok = tok[:, 0].contiguous() if bag == 1 else tok
    return tok if case["wide_index"] else tok.int()


def _matrix(rows, cols, pad, dtype, gen, scale=1.0):
    """[rows, cols], a slice of a matrix with `pad` more columns."""
    m = torch.randn((rows, cols + pad), generator=gen, device="cuda").mul_(scale).to(dtype)
    return m[:, :cols]


def _sizes(case):
    """Ragged sizes that add up to the case's elements, the same for every seed: most of them small, a few large."""
    tensors, elements = case["tensors"], case["elements"]
    w = torch.rand(tensors, generator=torch.Generator().manual_seed(tensors), dtype=torch.float64).pow(6)
    n = (w / w.sum() * (elements - tensors)).long() + 1
    n[0] += elements - int(n.sum())
    return n.tolist()


def _views(flat, sizes):
    """Tensors of these sizes inside `flat`, each from a multiple of 64 elements on."""
    at = [0, *itertools.accumulate(-(-n // 64) * 64 for n in sizes)]
    return [flat[a:a + n] for a, n in zip(at, sizes)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind, s = case["kind"], {"case": case}
    if kind in ("embed", "embed_grad"):
        dtype = TYPES[case["type"]]
        s["tokens"] = _tokens(case, gen)
        s["scale"] = 1.0 / math.sqrt(case["bag"])
        if kind == "embed":
            s["table"] = _matrix(case["entries"], case["dim"], case["pad"], dtype, gen, 0.5)
        else:
            s["grad"] = _matrix(case["rows"], case["dim"], case["pad"], dtype, gen, 0.1)
    elif kind in ("loss", "train"):
        dtype = TYPES[case["type"]]
        n, v, d = case["rows"], case["classes"], case["dim"]
        s["hidden"] = _matrix(n, d, 0, dtype, gen)
        s["weight"] = _matrix(v, d, 0, dtype, gen, 2.0 / math.sqrt(d))
        s["bias"] = torch.randn(v, generator=gen, device="cuda") if case["bias"] else None
        labels = torch.randint(0, v, (n,), generator=gen, device="cuda", dtype=torch.int32)
        masked = torch.rand(n, generator=gen, device="cuda") < case["masked"]
        s["labels"] = labels.masked_fill_(masked, -1)
        s["hidden"][masked, 0] = math.inf      # rows without a label hold what their buffer held before
        s["loss_scale"] = torch.full((1,), 4096.0, device="cuda") if case["type"] == "f16" else None
    else:
        # the gradients of a type lie in one buffer, as they do where they are summed over ranks; the gaps hold zeros
        names = {"f32": ["f32"], "bf16": ["bf16"], "mixed": ["bf16", "f32", "f16"]}[case["types"]][:case["tensors"]]
        s["flat"], s["grads"], s["out"] = [], [], [] if case["clipped"] else None
        s["flat_out"] = [] if case["clipped"] else s["flat"]
        for i, t in enumerate(names):
            sizes = _sizes(case)[i::len(names)]
            flat = torch.zeros(sum(-(-n // 64) * 64 for n in sizes), dtype=TYPES[t], device="cuda")
            s["flat"].append(flat)
            for g in _views(flat, sizes):
                g.copy_(torch.randn(g.shape, generator=gen, device="cuda").mul_(0.01))
                s["grads"].append(g)
            if case["clipped"]:
                s["flat_out"].append(torch.zeros_like(flat))
                s["out"] += _views(s["flat_out"][-1], sizes)
        norm = 0.01 * math.sqrt(case["elements"])
        s["max_norm"] = norm * (0.25 if case["clipped"] else 4.0)
    return s


# ---- the operators ------------------------------------------------------------------------------

def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"embed": _own_embed, "embed_grad": _own_embed_grad, "loss": _own_loss, "train": _own_train, "clip": _own_clip}[kind](state)
    return {"embed": _embed, "embed_grad": _embed_grad, "loss": _loss, "train": _train, "clip": _clip}[kind](state)


def _own_embed(s):
    return _context().embed(s["table"], s["tokens"], scale=s["scale"])


def _own_embed_grad(s):
    return _context().embed_backward(s["grad"], s["tokens"], s["case"]["entries"], scale=s["scale"])


def _own_loss(s):
    r = _context().softmax_ce(s["hidden"], s["weight"], s["labels"], bias=s["bias"])
    return {"loss": r.loss, "losses": r.losses, "lse": r.lse}


def _own_train(s):
    c = _context()
    r = c.softmax_ce(s["hidden"], s["weight"], s["labels"], bias=s["bias"])
    d_hidden, d_weight, d_bias = c.softmax_ce_backward(s["hidden"], s["weight"], s["labels"], r.lse, bias=s["bias"], grad_loss=s["loss_scale"])
    out = {"loss": r.loss, "losses": r.losses, "lse": r.lse, "d_hidden": d_hidden, "d_weight": d_weight}
    return out if d_bias is None else {**out, "d_bias": d_bias}


def _own_clip(s):
    norm = _context().clip_grad_norm(s["grads"], s["max_norm"], out=s["out"])
    return {"norm": norm, "flat": s["flat_out"]}


def _two_dim(tokens):
    return tokens.long().unsqueeze(1) if tokens.dim() == 1 else tokens.long()


def _embed(s):
    tok = _two_dim(s["tokens"])
    rows = s["table"].float()[tok.clamp(min=0)]
    rows.masked_fill_((tok < 0).unsqueeze(2), 0.0)
    return (rows.sum(1) * s["scale"]).to(s["table"].dtype)


def _embed_grad(s):
    tok, n = _two_dim(s["tokens"]), s["case"]["entries"]
    g = s["grad"].float() * s["scale"]
    out = torch.zeros((n + 1, g.shape[1]), device=g.device)
    out.index_add_(0, torch.where(tok < 0, n, tok).reshape(-1), g.unsqueeze(1).expand(-1, tok.shape[1], -1).reshape(-1, g.shape[1]))
    return out[:n].to(s["grad"].dtype)


def _logits(s):
    has = s["labels"] >= 0
    label = s["labels"].clamp(min=0).long().unsqueeze(1)
    h = torch.where(has.unsqueeze(1), s["hidden"].float(), 0.0)
    w = s["weight"].float()
    z = h @ w.t()
    if s["bias"] is not None:
        z += s["bias"]
    top = z.max(1, keepdim=True).values
    lse = top + (z - top).exp().sum(1, keepdim=True).log()
    losses = torch.where(has, (lse - z.gather(1, label)).squeeze(1), 0.0)
    return has, label, h, w, z, lse, losses, losses.sum() / has.sum().clamp(min=1)


def _loss(s):
    has, _, _, _, _, lse, losses, loss = _logits(s)
    return {"loss": loss.reshape(1), "losses": losses, "lse": torch.where(has, lse.squeeze(1), 0.0)}


def _train(s):
    has, label, h, w, z, lse, losses, loss = _logits(s)
    p = z.sub_(lse).exp_()
    p.scatter_add_(1, label, torch.full_like(lse, -1.0))
    each = has / has.sum().clamp(min=1)
    p *= (each if s["loss_scale"] is None else each * s["loss_scale"]).unsqueeze(1)
    dtype = s["hidden"].dtype
    out = {"loss": loss.reshape(1), "losses": losses, "lse": torch.where(has, lse.squeeze(1), 0.0),
           "d_hidden": (p @ w).to(dtype), "d_weight": (p.t() @ h).to(dtype)}
    return out if s["bias"] is None else {**out, "d_bias": p.sum(0)}


def _clip(s):
    flat = [x.float() for x in s["flat"]]
    norm = torch.stack([x.square().sum() for x in flat]).sum().sqrt()
    coef = (s["max_norm"] / norm).clamp(max=1.0)
    return {"norm": norm.reshape(1), "flat": [(x * coef).to(y.dtype) for x, y in zip(flat, s["flat"])]}


# ---- the definition in 64 bits ------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "embed":
        tok, table = _two_dim(s["tokens"]), s["table"].double()
        out = torch.zeros((case["rows"], case["dim"]), dtype=torch.float64, device="cuda")
        for k in range(tok.shape[1]):
            here = tok[:, k] >= 0
            out[here] += table[tok[here, k]]
        return out * s["scale"]
    if kind == "embed_grad":
        tok, g = _two_dim(s["tokens"]), s["grad"].double()
        out = torch.zeros((case["entries"], case["dim"]), dtype=torch.float64, device="cuda")
        for k in range(tok.shape[1]):
            here = tok[:, k] >= 0
            out.index_put_((tok[here, k],), g[here], accumulate=True)
        return out * s["scale"]
    if kind == "clip":
        norm = math.sqrt(sum(float(x.double().square().sum()) for x in s["flat"]))
        coef = min(1.0, s["max_norm"] / norm)
        return {"norm": torch.tensor([norm], dtype=torch.float64), "flat": [x.double() * coef for x in s["flat"]]}
    w, labels = s["weight"].double(), s["labels"].long()
    n = case["rows"]
    count = max(1, int((labels >= 0).sum()))
    f64 = dict(dtype=torch.float64, device="cuda")
    losses, lses = torch.zeros(n, **f64), torch.zeros(n, **f64)
    d_hidden, d_weight, d_bias = torch.zeros((n, case["dim"]), **f64), torch.zeros_like(w), torch.zeros(case["classes"], **f64)
    each = (1.0 if s["loss_scale"] is None else float(s["loss_scale"])) / count
    for rows in (labels >= 0).nonzero().squeeze(1).split(1024):
        h = s["hidden"][rows].double()
        z = h @ w.t() + (0.0 if s["bias"] is None else s["bias"].double())
        lse = torch.logsumexp(z, 1)
        at = torch.arange(len(rows), device="cuda")
        losses[rows], lses[rows] = lse - z[at, labels[rows]], lse
        if kind == "train":
            p = torch.exp(z - lse[:, None])
            p[at, labels[rows]] -= 1.0
            p *= each
            d_hidden[rows] = p @ w
            d_weight += p.t() @ h
            d_bias += p.sum(0)
    out = {"loss": losses.sum().reshape(1) / count, "losses": losses, "lse": lses}
    if kind == "train":
        out.update({"d_hidden": d_hidden, "d_weight": d_weight})
        if s["bias"] is not None:
            out["d_bias"] = d_bias
    return out


# ---- what a pass cannot do without --------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind in ("embed", "embed_grad"):
        w, d = WIDTH[case["type"]], case["dim"]
        m = case["rows"] * case["bag"]
        index = m * (8 if case["wide_index"] else 4)
        entries = min(case["entries"], m) if kind == "embed" else case["entries"]     # rows looked up; rows of the gradient
        return {"bytes": index + w * d * (entries + case["rows"]), "flops": m * d}
    if kind in ("loss", "train"):
        n, v, d, w = case["rows"], case["classes"], case["dim"], WIDTH[case["type"]]
        live = max(1, round(n * (1 - case["masked"])))
        inputs = w * d * (live + v) + 4 * n + (4 * v if case["bias"] else 0)
        if kind == "loss":
            return {"bytes": inputs + 8 * n, "flops": 2 * live * v * d}
        return {"bytes": inputs + 8 * n + w * d * (n + v) + (4 * v if case["bias"] else 0), "flops": 6 * live * v * d}
    names = {"f32": ["f32"], "bf16": ["bf16"], "mixed": ["bf16", "f32", "f16"]}[case["types"]][:case["tensors"]]
    total = sum(WIDTH[t] * sum(_sizes(case)[i::len(names)]) for i, t in enumerate(names))
    return {"bytes": total * (2 if case["clipped"] else 1), "flops": (3 if case["clipped"] else 2) * case["elements"]}

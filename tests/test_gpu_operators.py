"""Operators on top of the trees against plain implementations in 64 bits.

Tolerances.  An output of type T is rounded once: relative error u(T) = 2^-8 (bf16), 2^-11 (f16), 2^-24 (f32) of
its exact value, plus the error of single-precision sums: a sum of n terms added in any order is off by at most
n * 2^-24 * (sum of the terms' magnitudes); the kernels add in chains and trees far shorter than n, so that bound
holds with room.  Below half precision's normal range the spacing is 2^-24: half of that is added.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}


@pytest.fixture(scope="module")
def ctx():
    from paper_2207_09682_b200 import binding
    c = binding.Context(binding.make_params())
    yield c
    c.close()


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def within(got, want, slack, what=""):
    """|got - want| <= one rounding of want to got's type + slack (all in 64 bits)."""
    bound = want.abs() * UNIT[got.dtype] * (1 + 2.0 ** -9) + TINY[got.dtype] + slack
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), "%s: off by %.3g where %.3g is allowed" % (
        what, float((off - bound).max() + bound.flatten()[(off - bound).argmax()]), float(bound.flatten()[(off - bound).argmax()]))


# ---- embedding -----------------------------------------------------------------------------------

def embed_case(rows, bag, entries, dim, dtype, pad, wide, seed, missing=0.1):
    g = gen(seed)
    table = torch.randn((entries, dim + pad), generator=g, device="cuda").to(dtype)[:, :dim]
    tok = torch.randint(0, entries, (rows, bag), generator=g, device="cuda")
    tok[torch.rand((rows, bag), generator=g, device="cuda") < missing] = -1
    return table, tok if wide else tok.int()


def embed_exact(table, tok, scale):
    rows = table.double()[tok.long().clamp(min=0)]
    rows[tok < 0] = 0.0
    return rows.sum(1) * scale, rows.abs().sum(1) * abs(scale)


EMBED = [
    # rows, bag, entries, dim, pad
    (1, 1, 1, 1, 0), (1, 100, 2550, 64, 0), (3, 7, 11, 5, 0), (5, 1, 40, 770, 30), (33, 2, 100, 129, 0), (64, 10, 310, 16, 0),
    (257, 3, 50, 256, 8), (1000, 37, 4699, 100, 0), (2, 1000, 3000, 8, 1), (17, 5, 90, 1024, 0), (1, 3, 7, 2050, 0), (4097, 1, 513, 24, 0),
]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,bag,entries,dim,pad", EMBED)
def test_embed(ctx, rows, bag, entries, dim, pad, dtype):
    table, tok = embed_case(rows, bag, entries, dim, DTYPES[dtype], pad, rows % 2 == 1, 17 * rows + bag)
    got = ctx.embed(table, tok, scale=0.37)
    want, size = embed_exact(table, tok, float(torch.tensor(0.37, dtype=torch.float32)))
    within(got, want, (bag + 1) * 2.0 ** -24 * size)
    if bag == 1:
        assert torch.equal(ctx.embed(table, tok[:, 0], scale=0.37), got)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,bag,entries,dim,pad", EMBED)
def test_embed_backward(ctx, rows, bag, entries, dim, pad, dtype):
    dtype = DTYPES[dtype]
    _, tok = embed_case(rows, bag, entries, 1, dtype, 0, rows % 2 == 0, 13 * rows + bag)
    grad = torch.randn((rows, dim + pad), generator=gen(rows), device="cuda").to(dtype)[:, :dim]
    got = ctx.embed_backward(grad, tok, entries, scale=0.37)
    check_embed_grad(got, grad, tok, entries, float(torch.tensor(0.37, dtype=torch.float32)))


def check_embed_grad(got, grad, tok, entries, scale):
    index = torch.where(tok.long() < 0, entries, tok.long()).reshape(-1)
    each = grad.double().unsqueeze(1).expand(-1, tok.shape[1], -1).reshape(-1, grad.shape[1]) * scale
    want = torch.zeros((entries + 1, grad.shape[1]), dtype=torch.float64, device="cuda").index_add_(0, index, each)[:entries]
    size = torch.zeros((entries + 1, grad.shape[1]), dtype=torch.float64, device="cuda").index_add_(0, index, each.abs())[:entries]
    count = torch.bincount(index, minlength=entries + 1)[:entries].unsqueeze(1)
    within(got, want, (count + 1) * 2.0 ** -24 * size)


@pytest.mark.parametrize("rows,bag,entries,dim", [(4096, 1, 3, 8), (5000, 8, 2, 40), (3000, 40, 200000, 12), (70000, 3, 1, 4), (20000, 20, 2049, 33),
                                                  (300000, 2, 70000, 4)])
def test_embed_backward_long_lists(ctx, rows, bag, entries, dim):
    """More pairs than one counting launch sorts, tokens that fill many tiles, one to three radix passes."""
    g = gen(rows)
    tok = (torch.rand((rows, bag), generator=g, device="cuda", dtype=torch.float64).pow(2) * entries).int()
    grad = torch.randn((rows, dim), generator=g, device="cuda")
    first = ctx.embed_backward(grad, tok, entries, scale=1.0)
    check_embed_grad(first, grad, tok, entries, 1.0)
    assert torch.equal(ctx.embed_backward(grad, tok, entries, scale=1.0), first)   # the same bits every time


@pytest.mark.parametrize("rows,bag,entries,dim,wide", [(70000, 2, 70000, 8, False), (5000, 3, 1 << 21, 4, True), ((1 << 24) + 5, 1, 500, 2, False),
                                                       (65536, 2, 65535, 4, True), (65537, 2, 65535, 4, False), (1, 7000, 1 << 22, 1, True)])
def test_embed_backward_long_lists_of_one_word_pairs_and_two_word_pairs(ctx, rows, bag, entries, dim, wide):
    """Token and row together have 32 bits, more, or just as many."""
    table, tok = embed_case(rows, bag, entries, dim, torch.float32, 0, wide, 2)
    grad = torch.randn((rows, dim), generator=gen(3), device="cuda")
    check_embed_grad(ctx.embed_backward(grad, tok, entries, scale=0.5), grad, tok, entries, 0.5)


@pytest.mark.parametrize("entries", [40, 300, 70000])
def test_embed_backward_long_lists_of_one_token(ctx, entries):
    """Every pair of a tile has the same digits."""
    tok = torch.full((9000, 5), entries - 1, dtype=torch.int32, device="cuda")
    grad = torch.randn((9000, 3), generator=gen(4), device="cuda")
    check_embed_grad(ctx.embed_backward(grad, tok, entries), grad, tok, entries, 1.0)


def test_embed_backward_keeps_the_order_of_rows(ctx):
    """Sums of whole numbers are exact in any order; a permutation of the rows must not change them."""
    g = gen(5)
    tok = torch.randint(0, 977, (6000, 3), generator=g, device="cuda")
    grad = torch.randint(-8, 9, (6000, 16), generator=g, device="cuda").float()
    perm = torch.randperm(6000, generator=g, device="cuda")
    a = ctx.embed_backward(grad, tok, 977)
    assert torch.equal(a, ctx.embed_backward(grad[perm].contiguous(), tok[perm].contiguous(), 977))
    ones = torch.ones((6000, 1), device="cuda")
    assert torch.equal(ctx.embed_backward(ones, tok, 977).flatten().long(), torch.bincount(tok.flatten(), minlength=977))


def test_embed_missing_and_bad_tokens(ctx):
    table = torch.randn((10, 12), device="cuda")
    tok = torch.tensor([[-1, -1], [3, -7], [10, 4], [2 ** 31 + 1, 9]], device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = ctx.embed(table, tok, status=status)
    assert int(status) == 1
    assert torch.equal(out[0], torch.zeros(12, device="cuda")) and torch.equal(out[1], table[3])
    assert torch.equal(out[2], table[4]) and torch.equal(out[3], table[9])
    status.zero_()
    grad = torch.randn((4, 12), device="cuda")
    d = ctx.embed_backward(grad, tok, 10, status=status)
    assert int(status) == 1
    want = torch.zeros((10, 12), device="cuda")
    want[3], want[4], want[9] = grad[1], grad[2], grad[3]
    assert torch.equal(d, want)
    status.zero_()
    ctx.embed(table, tok[:2], status=status)
    assert int(status) == 0
    # nothing but missing tokens, and no rows at all
    assert not ctx.embed_backward(grad, torch.full((4, 3), -1, device="cuda"), 10).any()
    assert not ctx.embed_backward(grad[:0], torch.zeros((0, 3), dtype=torch.int64, device="cuda"), 10).any()
    assert ctx.embed(table, torch.zeros((0, 3), dtype=torch.int64, device="cuda")).shape == (0, 12)


def test_embed_infinite_and_nan_rows_stay_where_they_are(ctx):
    table = torch.randn((6, 8), device="cuda")
    table[5] = math.nan
    out = ctx.embed(table, torch.tensor([[0, 1], [5, -1], [2, -1]], device="cuda"))
    assert torch.isfinite(out[[0, 2]]).all() and torch.isnan(out[1]).all()


def test_embed_backward_never_uses_rows_without_tokens(ctx):
    tok = torch.randint(0, 40, (3000, 3), device="cuda")
    tok[::3] = -1
    grad = torch.randn((3000, 24), device="cuda").half()
    grad[::3] = math.nan
    got = ctx.embed_backward(grad, tok, 40)
    grad[::3] = 0.0
    check_embed_grad(got, grad, tok, 40, 1.0)


def test_embed_strides(ctx):
    """Rows of tokens, of the table and of the outputs that lie apart; outputs leave the gaps alone."""
    wide_table = torch.randn((50, 40), device="cuda")
    tokens = torch.randint(0, 50, (30, 9), device="cuda", dtype=torch.int32)[:, 2:6]
    out = torch.full((30, 32), 7.0, device="cuda")
    ctx.embed(wide_table[:, 3:20], tokens, out=out[:, 5:22])
    want, size = embed_exact(wide_table[:, 3:20], tokens, 1.0)
    within(out[:, 5:22], want, 5 * 2.0 ** -24 * size)
    assert bool((out[:, :5] == 7).all()) and bool((out[:, 22:] == 7).all())
    d = torch.full((50, 20), 7.0, device="cuda")
    ctx.embed_backward(out[:, 5:22], tokens, 50, grad_table=d[:, 1:18])
    check_embed_grad(d[:, 1:18], out[:, 5:22], tokens, 50, 1.0)
    assert bool((d[:, :1] == 7).all()) and bool((d[:, 18:] == 7).all())


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,bag,entries,dim,left,right", [(600, 7, 9001, 33, 1, 2), (3000, 4, 30000, 8, 8, 0), (40, 200, 200000, 6, 2, 4), (5, 3, 1 << 20, 300, 0, 0),
                                                             (7, 900, 20011, 2, 0, 2), (1, 7000, 70001, 1, 1, 0)])
def test_embed_backward_few_pairs_beside_the_entries(ctx, rows, bag, entries, dim, left, right, dtype):
    """Nearly every row of the gradient is zero; what lies between the rows stays as it is."""
    grad = torch.randn((rows, dim), generator=gen(6), device="cuda").to(DTYPES[dtype])
    tok = torch.randint(-1, entries, (rows, bag), generator=gen(7), device="cuda")
    tok[:, 0] = entries - 1
    wide = torch.full((entries, left + dim + right), 7.0, device="cuda", dtype=DTYPES[dtype])
    got = wide[:, left:left + dim]
    ctx.embed_backward(grad, tok, entries, grad_table=got)
    assert bool((wide[:, :left] == 7).all()) and bool((wide[:, left + dim:] == 7).all())
    hit = torch.zeros(entries, dtype=torch.bool, device="cuda")
    hit[tok[tok >= 0]] = True
    assert not got[~hit].any()
    index = torch.where(tok < 0, entries, tok).reshape(-1)
    each = grad.double().unsqueeze(1).expand(-1, bag, -1).reshape(-1, dim)
    zeros = torch.zeros((entries + 1, dim), dtype=torch.float64, device="cuda")
    want, size = zeros.index_add(0, index, each)[:entries], zeros.index_add(0, index, each.abs())[:entries]
    count = torch.bincount(index, minlength=entries + 1)[:entries].unsqueeze(1)
    within(got, want, (count + 1) * 2.0 ** -24 * size + UNIT[DTYPES[dtype]] * want.abs() + TINY[DTYPES[dtype]])


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,bag,entries,dim,left,right", [(7001, 40, 900, 51, 1, 1), (20000, 40, 640, 54, 0, 0), (20011, 50, 500, 92, 3, 1), (3000, 40, 600, 417, 0, 0),
                                                             (900, 60, 240000, 515, 0, 0)])
def test_embed_rows_that_are_read_often_and_start_anywhere(ctx, rows, bag, entries, dim, left, right, dtype):
    """Enough is read of rows that do not start on 16 bytes for a copy that does; results as ever, the gaps of the outputs left alone."""
    dtype = DTYPES[dtype]
    table, tok = embed_case(rows, bag, entries, dim, dtype, right, False, rows)
    wide = torch.full((rows, left + dim + right), 7.0, device="cuda", dtype=dtype)
    out = ctx.embed(table, tok, scale=0.5, out=wide[:, left:left + dim])
    want, size = embed_exact(table, tok, 0.5)
    within(out, want, (bag + 1) * 2.0 ** -24 * size)
    assert bool((wide[:, :left] == 7).all()) and bool((wide[:, left + dim:] == 7).all())
    wide = torch.full((entries, left + dim + right), 7.0, device="cuda", dtype=dtype)
    grad = out.clone() if left + right == 0 else torch.randn((rows, dim + right), generator=gen(rows), device="cuda").to(dtype)[:, :dim]
    got = ctx.embed_backward(grad, tok, entries, scale=0.5, grad_table=wide[:, left:left + dim])
    check_embed_grad(got, grad, tok, entries, 0.5)
    assert bool((wide[:, :left] == 7).all()) and bool((wide[:, left + dim:] == 7).all())


def test_embed_gradient_by_differences(ctx):
    """d sum(w * embed(table)) / d table against central differences (the function is linear: only rounding is left)."""
    g = gen(3)
    table = torch.randn((9, 5), generator=g, device="cuda")
    tok = torch.randint(-1, 9, (12, 4), generator=g, device="cuda")
    w = torch.randn((12, 5), generator=g, device="cuda")
    grad = ctx.embed_backward(w, tok, 9, scale=0.5)
    f = lambda t: float((ctx.embed(t, tok, scale=0.5).double() * w.double()).sum())  # noqa: E731
    step = 0.25
    for v in range(9):
        for d in range(5):
            up, down = table.clone(), table.clone()
            up[v, d] += step
            down[v, d] -= step
            # f is a sum of 240 products of numbers below 10 in size, each rounded to 2^-24 a few times
            assert abs((f(up) - f(down)) / (2 * step) - float(grad[v, d])) <= 240 * 10 * 2.0 ** -22 / step


# ---- clipping ------------------------------------------------------------------------------------

CLIP = [
    # sizes, types, offset of every tensor in elements
    ([1], ["f32"], 0), ([5, 0, 17, 4096, 4097], ["f32"], 0), ([100000, 3, 70001], ["bf16"], 0), ([33, 9000, 1, 64, 12345], ["f32", "bf16", "f16"], 0),
    ([10000, 5, 3, 2, 1], ["f16"], 3), ([7, 8195, 20000], ["f32", "bf16"], 1), ([300000] * 3, ["f32"], 0), (list(range(0, 130)), ["f32", "f16"], 0),
    ([11] * 1500, ["bf16"], 0),
]


def clip_case(sizes, types, offset, seed):
    g = gen(seed)
    return [torch.randn(n + offset, generator=g, device="cuda").to(DTYPES[types[i % len(types)]])[offset:] for i, n in enumerate(sizes)]


@pytest.mark.parametrize("part", [0.0, 0.3, 2.0])
@pytest.mark.parametrize("sizes,types,offset", CLIP)
def test_clip(ctx, sizes, types, offset, part):
    grads = clip_case(sizes, types, offset, len(sizes))
    before = [t.clone() for t in grads]
    exact = math.sqrt(sum(float(t.double().square().sum()) for t in grads))
    out = [torch.full_like(t, 9.0) for t in grads]
    norm = ctx.clip_grad_norm(grads, part * exact, out=out)
    assert abs(float(norm) - exact) <= 2.0 ** -23 * exact
    assert all(torch.equal(a, b) for a, b in zip(grads, before))
    coef = min(1.0, part)
    for o, b in zip(out, before):
        within(o, b.double() * coef, 3 * 2.0 ** -24 * coef * b.double().abs())
    again = ctx.clip_grad_norm(grads, part * exact)
    assert torch.equal(again, norm)
    assert all(torch.equal(a, b) for a, b in zip(grads, out))
    if part >= 1:
        assert all(torch.equal(a, b) for a, b in zip(grads, before))


def test_clip_output_of_another_alignment(ctx):
    g = torch.randn(9999, device="cuda")
    out = torch.zeros(10002, device="cuda")[3:]
    norm = float(ctx.clip_grad_norm([g], 1.0, out=[out]))
    within(out, g.double() / norm, 4 * 2.0 ** -24 * g.double().abs() / norm)


@pytest.mark.parametrize("value", [1e-30, 1e30, 3e38])
def test_clip_norms_beyond_the_range_of_single_precision_squares(ctx, value):
    g = torch.full((4096,), value, device="cuda")
    norm = ctx.clip_grad_norm([g], 0.5 * value)
    want = 64.0 * float(torch.tensor(value, dtype=torch.float32))
    if want < 3.4e38:
        assert abs(float(norm) - want) <= 2.0 ** -23 * want
    assert abs(float(g[7]) * 128 / value - 1) <= 2.0 ** -22     # value * (0.5 * value) / (64 * value)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_clip_leaves_tensors_alone_when_the_norm_is_not_finite(ctx, bad):
    a, b = torch.randn(5000, device="cuda"), torch.randn(77, device="cuda").half()
    a[4321] = bad
    before = [a.clone(), b.clone()]
    norm = ctx.clip_grad_norm([a, b], 1e-3)
    assert not math.isfinite(float(norm))
    assert torch.equal(torch.nan_to_num(a, nan=5.0), torch.nan_to_num(before[0], nan=5.0)) and torch.equal(b, before[1])


def test_clip_nothing(ctx):
    assert float(ctx.clip_grad_norm([], 1.0)) == 0.0
    z = torch.zeros(100, device="cuda")
    assert float(ctx.clip_grad_norm([z, z[:0]], 1.0)) == 0.0 and not z.any()
    g = torch.ones(4, device="cuda")
    assert float(ctx.clip_grad_norm([g], math.inf)) == 2.0 and bool((g == 1).all())
    ctx.clip_grad_norm([g], 0.0)
    assert not g.any()


# ---- softmax cross entropy -----------------------------------------------------------------------

def softmax_case(rows, classes, dim, dtype, bias, masked, seed, pad=0, wide=False):
    g = gen(seed)
    h = torch.randn((rows, dim + pad), generator=g, device="cuda").to(dtype)[:, :dim]
    w = (torch.randn((classes, dim + pad), generator=g, device="cuda") * 2 / math.sqrt(dim)).to(dtype)[:, :dim]
    b = torch.randn(classes, generator=g, device="cuda") if bias else None
    y = torch.randint(0, classes, (rows,), generator=g, device="cuda")
    y[torch.rand(rows, generator=g, device="cuda") < masked] = -1
    return h, w, b, y if wide else y.int()


def softmax_exact(h, w, b, y, scale=1.0):
    has = y >= 0
    h = torch.where(has.unsqueeze(1), h.double(), 0.0)
    z = h @ w.double().t() + (0.0 if b is None else b.double())
    lse = torch.logsumexp(z, 1)
    at = torch.arange(len(y), device="cuda")
    losses = torch.where(has, lse - z[at, y.long().clamp(min=0)], 0.0)
    p = torch.exp(z - lse[:, None])
    p[at, y.long().clamp(min=0)] -= 1.0
    p[~has] = 0.0
    count = max(1, int(has.sum()))
    return dict(losses=losses, lse=torch.where(has, lse, 0.0), loss=losses.sum() / count, g=p, s=scale / count, h=h, z=z)


SOFTMAX = [
    # rows, classes, dim, bias, masked
    (1, 1, 1, False, 0.0), (1, 2, 8, True, 0.0), (1, 32000, 512, False, 0.0), (3, 257, 64, True, 0.0), (128, 256, 64, False, 0.0),
    (129, 255, 65, True, 0.3), (300, 1000, 72, False, 0.5), (777, 1003, 129, True, 0.3), (1000, 10, 200, True, 0.9), (513, 4099, 40, False, 0.1),
    (9000, 300, 16, True, 0.2), (257, 513, 1000, True, 0.0), (40, 70, 8, False, 1.0),
    # one and two rows with and without aligned operands; more than one column tile of d; long and short products that are cut or not
    (1, 70, 264, True, 0.0), (2, 5003, 520, True, 0.0), (2, 31, 17, False, 0.0), (2, 100, 64, True, 0.6), (3000, 40, 300, True, 0.1),
    (300, 3000, 520, False, 0.1), (2500, 2100, 24, True, 0.2), (700, 600, 1300, False, 0.0), (100, 9000, 2050, False, 0.0),
]


def check_loss(r, e, h, w):
    # a logit: its products are exact in single precision, their sum is off by at most dim * 2^-23 * sum |h w| (the tensor
    # cores round towards zero); exponentials and logarithms add 2^-20 of the sum they belong to, the label's logit one more
    size = (e["h"].abs() @ w.double().abs().t()).max(1).values
    slack = h.shape[1] * 2.0 ** -23 * size * 2 + 2.0 ** -18 + 2.0 ** -22 * e["lse"].abs()
    assert bool(((r.lse.double() - e["lse"]).abs() <= slack).all())
    assert bool(((r.losses.double() - e["losses"]).abs() <= 2 * slack).all())
    assert abs(float(r.loss) - float(e["loss"])) <= 2 * float(slack.max()) + 2.0 ** -23 * abs(float(e["loss"]))
    masked = e["lse"] == 0
    assert not r.losses[masked].any()


def check_grads(got, e, h, w, dtype):
    u = UNIT[dtype]
    g, s = e["g"], e["s"]
    # g: off by what its logit is off (below 2^-14 at these sizes), then rounded to `dtype` once
    err = g.abs() * (u + 2.0 ** -13) + 2.0 ** -14 * (g.abs() > 0) * torch.exp(e["z"] - torch.logsumexp(e["z"], 1, keepdim=True)) + TINY[dtype]
    chain = 2.0 ** -22
    dh, dw, db = got
    within(dh, s * (g @ w.double()), abs(s) * ((err + chain * g.abs()) @ w.double().abs()), "d_hidden")
    within(dw, s * (g.t() @ e["h"]), abs(s) * ((err + chain * g.abs()).t() @ e["h"].abs()), "d_weight")
    if db is not None:
        free = 2.0 ** -14 * (g.abs() + torch.exp(e["z"] - torch.logsumexp(e["z"], 1, keepdim=True)) * (g.abs() > 0))
        within(db, s * g.sum(0), abs(s) * free.sum(0), "d_bias")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows,classes,dim,bias,masked", SOFTMAX)
def test_softmax_ce(ctx, rows, classes, dim, bias, masked, dtype):
    h, w, b, y = softmax_case(rows, classes, dim, DTYPES[dtype], bias, masked, rows + classes, wide=rows % 2 == 1)
    e = softmax_exact(h, w, b, y, 64.0)
    h[y < 0] = math.nan                                    # rows without a label hold anything
    r = ctx.softmax_ce(h, w, y, bias=b)
    check_loss(r, e, h, w)
    scale = torch.full((1,), 64.0, device="cuda")
    got = ctx.softmax_ce_backward(h, w, y, r.lse, bias=b, grad_loss=scale)
    check_grads(got, e, h, w, DTYPES[dtype])
    assert not got[0][y < 0].any()
    again = ctx.softmax_ce_backward(h, w, y, r.lse, bias=b, grad_loss=scale)
    assert all(a is None or torch.equal(a, x) for a, x in zip(again, got))   # the same bits every time
    assert all(torch.equal(a, x) for a, x in zip(ctx.softmax_ce(h, w, y, bias=b), r))


def test_softmax_ce_strides(ctx):
    h, w, b, y = softmax_case(200, 300, 50, torch.bfloat16, True, 0.2, 9, pad=7)
    e = softmax_exact(h, w, b, y)
    r = ctx.softmax_ce(h, w, y, bias=b)
    check_loss(r, e, h, w)
    dh, dw = torch.full((200, 61), 7.0, device="cuda").bfloat16(), torch.full((300, 53), 7.0, device="cuda").bfloat16()
    got = ctx.softmax_ce_backward(h, w, y, r.lse, bias=b, grad_hidden=dh[:, 3:53], grad_weight=dw[:, 2:52])
    check_grads(got, e, h, w, torch.bfloat16)
    assert bool((dh[:, :3] == 7).all()) and bool((dh[:, 53:] == 7).all()) and bool((dw[:, :2] == 7).all()) and bool((dw[:, 52:] == 7).all())


def test_softmax_ce_aligned_outputs_leave_the_gaps_alone(ctx):
    """Rows of 50 elements on 128 bytes: what lies between them is neither read nor written."""
    h, w, b, y = softmax_case(300, 300, 50, torch.float16, True, 0.2, 11)
    wide_h, wide_w = torch.full((300, 64), math.nan, device="cuda").half(), torch.full((300, 64), math.nan, device="cuda").half()
    wide_h[:, :50], wide_w[:, :50] = h, w
    h, w = wide_h[:, :50], wide_w[:, :50]
    e = softmax_exact(h, w, b, y, 1024.0)
    r = ctx.softmax_ce(h, w, y, bias=b)
    dh, dw = torch.full((300, 64), 7.0, device="cuda").half(), torch.full((302, 64), 7.0, device="cuda").half()
    got = ctx.softmax_ce_backward(h, w, y, r.lse, bias=b, grad_loss=torch.full((1,), 1024.0, device="cuda"), grad_hidden=dh[:, :50], grad_weight=dw[:300, :50])
    check_grads(got, e, h, w, torch.float16)
    assert bool((dh[:, 50:] == 7).all()) and bool((dw[:, 50:] == 7).all()) and bool((dw[300:] == 7).all())


def test_softmax_ce_all_classes_at_the_lowest_value(ctx):
    """Every class masked by the type's lowest value: a uniform distribution, up to the rounding of numbers of that size."""
    h, w, b, y = softmax_case(20, 300, 64, torch.bfloat16, True, 0.0, 4)
    b[:] = torch.finfo(torch.float32).min
    r = ctx.softmax_ce(h, w, y, bias=b)
    assert bool((r.lse == torch.finfo(torch.float32).min).all()) and bool((r.losses == 0).all())
    assert all(bool(torch.isfinite(t).all()) for t in ctx.softmax_ce_backward(h, w, y, r.lse, bias=b))


def test_softmax_ce_large_logits_and_excluded_classes(ctx):
    """Logits in the thousands neither overflow nor lose the loss; a bias of -infinity or of the type's lowest value takes a class out."""
    h, w, b, y = softmax_case(150, 400, 64, torch.bfloat16, True, 0.0, 4)
    b[100:400] = -math.inf
    b[90:100] = torch.finfo(torch.float32).min
    y = y % 90
    w = (w.float() * 300).bfloat16()
    e = softmax_exact(h, w, b, y)
    r = ctx.softmax_ce(h, w, y, bias=b)
    check_loss(r, e, h, w)
    dh, dw, db = ctx.softmax_ce_backward(h, w, y, r.lse, bias=b)
    assert torch.isfinite(dh).all() and torch.isfinite(dw).all() and not dw[90:].any() and not db[90:].any()
    # the label's own class excluded: an infinite loss
    y[3] = 200
    assert float(ctx.softmax_ce(h, w, y, bias=b).losses[3]) == math.inf


def test_softmax_ce_labels_out_of_range(ctx):
    h, w, b, y = softmax_case(70, 33, 24, torch.float16, False, 0.0, 2)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ctx.softmax_ce(h, w, y, status=status)
    assert int(status) == 0
    bad = y.clone()
    bad[5] = 33
    r = ctx.softmax_ce(h, w, bad, status=status)
    assert int(status) == 1
    y[5] = -1
    assert all(torch.equal(a, x) for a, x in zip(ctx.softmax_ce(h, w, y), r))


def test_softmax_ce_without_rows_or_labels(ctx):
    h, w, b, y = softmax_case(0, 33, 24, torch.float16, True, 0.0, 2)
    r = ctx.softmax_ce(h, w, y, bias=b)
    assert float(r.loss) == 0.0 and r.lse.shape == (0,)
    dh, dw, db = ctx.softmax_ce_backward(h, w, y, r.lse, bias=b)
    assert dh.shape == (0, 24) and not dw.any() and not db.any()


def test_softmax_ce_many_pieces(ctx):
    """More classes than one piece of the probabilities holds (3 * 2^26 / rows)."""
    h, w, b, y = softmax_case(40000, 5000, 16, torch.bfloat16, True, 0.4, 6)
    e = softmax_exact(h, w, b, y)
    r = ctx.softmax_ce(h, w, y, bias=b)
    check_loss(r, e, h, w)
    check_grads(ctx.softmax_ce_backward(h, w, y, r.lse, bias=b), e, h, w, torch.bfloat16)


def test_softmax_ce_long_products(ctx):
    """Tiles of two accumulators, cut into fragments."""
    h, w, b, y = softmax_case(5000, 31000, 1024, torch.bfloat16, True, 0.1, 3)
    e = softmax_exact(h, w, b, y)
    r = ctx.softmax_ce(h, w, y, bias=b)
    check_loss(r, e, h, w)
    check_grads(ctx.softmax_ce_backward(h, w, y, r.lse, bias=b), e, h, w, torch.bfloat16)


@pytest.mark.parametrize("rows,classes,dim,dtype", [(5000, 90000, 1024, "bf16"), (20000, 31000, 40, "f16")])
def test_softmax_ce_several_pieces_and_a_narrow_last_one(ctx, rows, classes, dim, dtype):
    """Fragments of the hidden rows' gradient that three pieces and more add to, whole tiles and cut ones."""
    h, w, b, y = softmax_case(rows, classes, dim, DTYPES[dtype], True, 0.1, 4)
    e = softmax_exact(h, w, b, y, 1024.0)
    r = ctx.softmax_ce(h, w, y, bias=b)
    check_loss(r, e, h, w)
    check_grads(ctx.softmax_ce_backward(h, w, y, r.lse, bias=b, grad_loss=torch.full((1,), 1024.0, device="cuda")), e, h, w, DTYPES[dtype])


def test_softmax_ce_infinite_grad_loss_leaves_rows_without_a_label_at_zero(ctx):
    h, w, b, y = softmax_case(300, 70, 24, torch.float16, True, 0.4, 5)
    inf = torch.full((1,), math.inf, device="cuda")
    r = ctx.softmax_ce(h, w, y, bias=b)
    dh, dw, db = ctx.softmax_ce_backward(h, w, y, r.lse, bias=b, grad_loss=inf)
    assert not dh[y < 0].any() and not torch.isfinite(dh[y >= 0]).any()
    y[:] = -1
    dh, dw, db = ctx.softmax_ce_backward(h, w, y, ctx.softmax_ce(h, w, y, bias=b).lse, bias=b, grad_loss=inf)
    assert not dh.any() and not dw.any() and not db.any()


def test_softmax_ce_gradient_by_differences(ctx):
    """The loss along a direction in H, W and b: central differences of the kernel's own loss."""
    h, w, b, y = softmax_case(60, 50, 24, torch.float16, True, 0.2, 8)
    r = ctx.softmax_ce(h, w, y, bias=b)
    dh, dw, db = ctx.softmax_ce_backward(h, w, y, r.lse, bias=b)
    g = gen(1)
    for which, grad in ((0, dh), (1, dw), (2, db)):
        x = (h, w, b)[which]
        # a direction whose steps are exact in x's type: multiples of the spacing of numbers below 8
        step = torch.randint(-1, 2, x.shape, generator=g, device="cuda").to(x.dtype) * 2.0 ** -6
        x = (x.float() * 2.0 ** 7).round().mul(2.0 ** -7).to(x.dtype)
        at = [h, w, b]
        at[which] = x
        r0 = ctx.softmax_ce(at[0], at[1], y, bias=at[2])
        grad = ctx.softmax_ce_backward(at[0], at[1], y, r0.lse, bias=at[2])[which]
        at[which] = x + step
        up = float(ctx.softmax_ce(at[0], at[1], y, bias=at[2]).loss)
        at[which] = x - step
        down = float(ctx.softmax_ce(at[0], at[1], y, bias=at[2]).loss)
        want = float((grad.double() * step.double()).sum())
        # third-order term: |step| * |logit change|^2; the loss itself is exact to 2^-17; the gradient to 2^-11 of its terms
        slack = 2.0 ** -16 + 2.0 ** -10 * float((grad.double().abs() * step.double().abs()).sum())
        dz = max(2.0 ** -6 * float(w.double().abs().sum(1).max()), 2.0 ** -6 * float(h.double().abs().sum(1).max()), 2.0 ** -6)
        assert abs((up - down) / 2 - want) <= slack + dz ** 3


def test_calls_on_other_streams(ctx):
    """Calls on two streams share one work buffer: each must wait for the other's."""
    h, w, b, y = softmax_case(600, 2000, 64, torch.bfloat16, True, 0.2, 8)
    tok = torch.randint(0, 500, (20000, 4), device="cuda")
    grad = torch.randn((20000, 8), device="cuda")
    r = ctx.softmax_ce(h, w, y, bias=b)
    want = ctx.softmax_ce_backward(h, w, y, r.lse, bias=b)
    want_e = ctx.embed_backward(grad, tok, 500)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        got = ctx.softmax_ce_backward(h, w, y, r.lse, bias=b, stream=s1)
        got_e = ctx.embed_backward(grad, tok, 500, stream=s2)
        torch.cuda.synchronize()
        assert torch.equal(got_e, want_e) and all(torch.equal(a, x) for a, x in zip(got, want))


def test_calls_in_a_graph(ctx):
    h, w, b, y = softmax_case(300, 900, 64, torch.bfloat16, True, 0.2, 8)
    tok = torch.randint(0, 500, (2000, 4), device="cuda")
    table = torch.randn((500, 64), device="cuda").bfloat16()

    def step():
        out = ctx.embed(table, tok)
        d = ctx.embed_backward(out, tok, 500)
        r = ctx.softmax_ce(h, w, y, bias=b)
        return [out, d, *r, *ctx.softmax_ce_backward(h, w, y, r.lse, bias=b), ctx.clip_grad_norm([d], 0.1)]

    want = [t.clone() for t in step()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, x) for a, x in zip(got, want))


# ---- refusals --------------------------------------------------------------------------------------

def test_refusals(ctx):
    from paper_2207_09682_b200 import binding
    table = torch.randn((10, 12), device="cuda")
    tok = torch.zeros((3, 2), dtype=torch.int32, device="cuda")
    h, w = torch.zeros((4, 8), device="cuda").half(), torch.zeros((5, 8), device="cuda").half()
    y = torch.zeros(4, dtype=torch.int64, device="cuda")
    lse = torch.zeros(4, device="cuda")
    bad = [
        lambda: ctx.embed(table.double(), tok), lambda: ctx.embed(table, tok.float()), lambda: ctx.embed(table.t(), tok),
        lambda: ctx.embed(table.cpu(), tok), lambda: ctx.embed(table, tok, out=torch.empty((3, 11), device="cuda")),
        lambda: ctx.embed(table, tok, scale=math.nan), lambda: ctx.embed(table, tok[:, :0]), lambda: ctx.embed(table[:, :0], tok),
        lambda: ctx.embed_backward(table, tok, 10), lambda: ctx.embed_backward(table[:3], tok, 0),
        lambda: ctx.softmax_ce(h.float(), w.float(), y), lambda: ctx.softmax_ce(h, w.bfloat16(), y), lambda: ctx.softmax_ce(h, w[:, :7], y),
        lambda: ctx.softmax_ce(h, w, y.float()), lambda: ctx.softmax_ce(h, w, y[:3]), lambda: ctx.softmax_ce(h, w[:0], y),
        lambda: ctx.softmax_ce(h, w, y, bias=torch.zeros(5, device="cuda").half()),
        lambda: ctx.softmax_ce_backward(h, w, y, lse.double()), lambda: ctx.softmax_ce_backward(h, w, y, lse, grad_loss=torch.ones(2, device="cuda")),
        lambda: ctx.softmax_ce_backward(h, w, y, lse, grad_weight=torch.empty((5, 9), device="cuda").half()),
        lambda: ctx.clip_grad_norm([table], -1.0), lambda: ctx.clip_grad_norm([table], math.nan), lambda: ctx.clip_grad_norm([table.long()], 1.0),
        lambda: ctx.clip_grad_norm([table.t()], 1.0), lambda: ctx.clip_grad_norm([table], 1.0, out=[]),
    ]
    for call in bad:
        with pytest.raises(binding.QgbdtError) as e:
            call()
        assert e.value.code == binding.ERR_ARG
    assert torch.isfinite(ctx.embed(table, tok)).all()   # still in order

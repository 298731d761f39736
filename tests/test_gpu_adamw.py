"""The AdamW step against its formula in 64 bits, and states of 8 bits against their definition.

Tolerances.  u = 2^-24 is one rounding in single precision.  m and v are sums of two products: a factor, a product and (v:
another product) the sum are rounded, and the gradient's factor and its product, twice in v: at most 5 u (m) and 8 u (v) of
the terms' magnitudes.  The change of a parameter is a quotient of them: m, v under a root, five further operations that are
rounded to 2 u at most (root and quotient included), three factors: below 30 u of itself, plus what m's cancellation makes of
its terms.  The parameter is rounded with its product and its sum: 3 u, and once more to its type.  In denormal numbers a
rounding is 2^-150.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U, TINY = 2.0 ** -24, 2.0 ** -148
BLOCK = 256


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
    info = torch.finfo(got.dtype)
    bound = want.abs() * (info.eps / 2) * (1 + 2.0 ** -9) + info.tiny * info.eps + slack
    off = (got.double() - want).abs()
    bad = ~(off <= bound)
    assert not bool(bad.any()), "%s: off by %.3g where %.3g is allowed (%d of %d)" % (what, float(off[bad].max()), float(bound.expand_as(off)[bad].min()), int(bad.sum()), off.numel())


class Case:
    """Parameters, gradients and states of ragged sizes, as views at offsets of `shift` elements into larger buffers."""

    def __init__(self, sizes, ptype="f32", gtype="f32", ctype=None, bits=32, seed=1, shift=0, scale=1.0):
        g = gen(seed)
        self.around = []

        def tensors(dtype, make):
            out = []
            for n in sizes:
                flat = torch.full((n + shift + 9,), 5, device="cuda").to(dtype)
                self.around.append((flat, n, shift))
                out.append(flat[shift:shift + n])
                out[-1].copy_(make(n))
            return out

        randn = lambda n: torch.randn(n, generator=g, device="cuda")  # noqa: E731
        self.sizes, self.bits = sizes, bits
        self.p = tensors(DTYPES[ptype], lambda n: randn(n) * 0.1)
        self.g = tensors(DTYPES[gtype], lambda n: randn(n) * scale * torch.exp(randn(n)))
        self.copies = None if ctype is None else tensors(DTYPES[ctype], lambda n: torch.zeros(n))
        if bits == 32:
            self.m = tensors(torch.float32, lambda n: randn(n) * 0.3)
            self.v = tensors(torch.float32, lambda n: randn(n).square())
            self.e = None
        else:
            byte = lambda n: torch.randint(0, 256, (n,), generator=g, device="cuda")  # noqa: E731
            self.m, self.v = tensors(torch.uint8, byte), tensors(torch.uint8, byte)
            self.e = [torch.randint(100, 130, (-(-n // BLOCK), 2), generator=g, device="cuda").to(torch.uint8) for n in sizes]

    def all(self):
        return [t for l in (self.p, self.m, self.v, self.e, self.copies) if l is not None for t in l]

    def states(self, ctx):
        """m, v in 64 bits."""
        if self.bits == 32:
            return [t.double() for t in self.m], [t.double() for t in self.v]
        return [decode(m, e[:, 0], 897, True) for m, e in zip(self.m, self.e)], [decode(v, e[:, 1], 769, False) for v, e in zip(self.v, self.e)]

    def check_around(self):
        for flat, n, shift in self.around:
            edge = torch.cat([flat[:shift], flat[shift + n:]])
            assert bool((edge == 5).all())

    def step(self, ctx, step, lr, **more):
        ctx.adamw(self.p, self.g, self.m, self.v, step, lr, exponents=self.e, copies=self.copies, **more)


def power_of_two(k):
    """Exactly (a library's pow is not)."""
    return ((k.long() + 1023) << 52).view(torch.float64)


def decode(code, exponent, offset, signed):
    """What codes stand for, from the definition: the float with bits (c + offset) << 20, times 2^(E - 127); E = 255: NaN."""
    c = code.long()
    size = c & 127 if signed else c
    value = torch.where(size > 0, ((size + offset) << 20).int().view(torch.float32).double(), 0.0)
    if signed:
        value = torch.where(c > 127, -value, value)
    power = power_of_two(exponent.long() - 127).repeat_interleave(BLOCK)[:len(code)]
    return value * torch.where(exponent.repeat_interleave(BLOCK)[:len(code)] == 255, math.nan, power)


def formula(g, m, v, p, step, lr, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, coef=1.0):
    """(m, v, p, and the magnitude of m's and v's terms) after a step, in 64 bits."""
    b1, b2 = betas
    g = g.double() * coef
    m, m_size = b1 * m + (1 - b1) * g, b1 * m.abs() + (1 - b1) * g.abs()
    v = b2 * v + (1 - b2) * g * g
    denominator = (v / (1 - b2 ** step)).sqrt() + eps
    rate = lr / (1 - b1 ** step)
    change = rate * m / denominator
    p = p.double()
    p, slack = p - lr * weight_decay * p - change, 3 * U * (p.abs() + change.abs()) + 30 * U * change.abs() + 5 * U * rate * m_size / denominator
    return m, v, p, m_size, slack


def check_32(case, before, ctx, step, lr, coef=1.0, **more):
    ps, ms, vs = before
    for i in range(len(case.sizes)):
        m, v, p, m_size, slack = formula(case.g[i], ms[i], vs[i], ps[i], step, lr, coef=coef, **more)
        within(case.p[i], p, slack, "param %d" % i)
        if case.copies is not None:
            within(case.copies[i], p, slack + p.abs() * (torch.finfo(case.p[i].dtype).eps / 2 if case.p[i].dtype == torch.float32 else 0), "copy %d" % i)
        if case.bits == 32:
            within(case.m[i], m, 5 * U * m_size + TINY, "m %d" % i)
            within(case.v[i], v, 8 * U * v + TINY, "v %d" % i)
    case.check_around()


def before(case, ctx):
    return [[p.double().clone() for p in case.p], *[[t.clone() for t in l] for l in case.states(ctx)]]


RAGGED = [1, 0, 255, 256, 257, 3, 4096, 5000, 2, 0, 2048, 70001]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("shift", [0, 1, 8, 16])
@pytest.mark.parametrize("ptype,gtype,ctype", [("f32", "f32", None), ("f32", "bf16", "bf16"), ("f32", "f16", "f16"), ("bf16", "bf16", None), ("f16", "f32", "f32"),
                                               ("bf16", "f16", "bf16"), ("f16", "f16", None)])
def test_types_and_sizes(ctx, ptype, gtype, ctype, shift, bits):
    case = Case(RAGGED, ptype, gtype, ctype, bits, 3, shift)
    was = before(case, ctx)
    case.step(ctx, 7, 0.01, seed=5)
    check_32(case, was, ctx, 7, 0.01)
    if bits == 8:
        check_codes(case, was, 7, 5)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("options", [dict(betas=(0.0, 0.0), eps=1e-3, weight_decay=0.0), dict(betas=(0.95, 0.98), eps=0.0, weight_decay=0.3), dict(eps=1.0)])
@pytest.mark.parametrize("step,lr", [(1, 1e-3), (2, 0.0), (100000, 0.5)])
def test_options(ctx, step, lr, options, bits):
    case = Case([300, 1111], bits=bits)
    was = before(case, ctx)
    case.step(ctx, step, lr, **options)
    check_32(case, was, ctx, step, lr, **options)
    if bits == 8:
        check_codes(case, was, step, 0, betas=options.get("betas", (0.9, 0.999)))


@pytest.mark.parametrize("tensors", [31, 32, 33, 64, 399, 400, 401, 1000])
@pytest.mark.parametrize("bits", [32, 8])
def test_many_tensors(ctx, tensors, bits):
    """More than a launch takes; blocks are numbered through all of them."""
    sizes = [(37 * i) % 1500 for i in range(tensors)]
    case = Case(sizes, "f32", "bf16", "bf16", bits, tensors)
    was = before(case, ctx)
    case.step(ctx, 3, 0.02, seed=1 << 40)
    check_32(case, was, ctx, 3, 0.02)
    if bits == 8:
        check_codes(case, was, 3, 1 << 40)


# ---- clipping, device numbers, order -----------------------------------------------------------------

@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("scale", [1.0, 512.0])
@pytest.mark.parametrize("fraction", [0.25, 1.0, 3.0, 0.0, math.inf])
def test_clipping_factor(ctx, fraction, scale, bits):
    """As clip_grad_norm has it, with the norm that it reports; a norm of zero is not clipped."""
    case = Case([3000, 17, 70000], "f32", "f16", None, bits, 4, scale=0.01 * scale)
    norm = ctx.clip_grad_norm(case.g, math.inf)
    max_norm = fraction * float(norm) / scale
    coef = min(1.0, max_norm * scale / float(norm)) / scale
    was = before(case, ctx)
    case.step(ctx, 5, 0.01, norm=norm, max_norm=max_norm, loss_scale=scale)
    check_32(case, was, ctx, 5, 0.01, coef=coef)
    case = Case([300], bits=bits)
    case.g[0].zero_()
    was = before(case, ctx)
    case.step(ctx, 5, 0.01, norm=ctx.clip_grad_norm(case.g, math.inf), max_norm=max_norm)
    check_32(case, was, ctx, 5, 0.01)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("norm,max_norm,scale", [(3e38, 1e-2, 1.0), (2e38, 1e-6, 4.0), (1e38, 1.0, 2.0 ** 20), (1e30, math.inf, 1e39), (3e38, 1e-40, 1.0), (1e38, 0.0, 1.0)])
@pytest.mark.parametrize("eps", [1e-12, 1e-8])
def test_clipping_factors_below_single_precision(ctx, eps, norm, max_norm, scale, bits):
    """Factors below 2^-126 are as exact as others: gradients near the upper end of the range come out as the formula has them."""
    case = Case([3000, 17, 5001], "f32", "f32", None, bits, 8, scale=1e33)
    for t in (case.m + case.v + (case.e or [])):
        t.zero_()
    norm = torch.full((1,), norm, device="cuda")
    coef = min(1.0, max_norm * scale / float(norm)) / scale
    assert coef < 2.0 ** -126
    was = before(case, ctx)
    case.step(ctx, 5, 0.01, norm=norm, max_norm=max_norm, loss_scale=scale, eps=eps)
    check_32(case, was, ctx, 5, 0.01, coef=coef, eps=eps)
    if not math.isfinite(max_norm):      # the same without a norm
        again = Case([3000, 17, 5001], "f32", "f32", None, bits, 8, scale=1e33)
        for t in (again.m + again.v + (again.e or [])):
            t.zero_()
        again.step(ctx, 5, 0.01, loss_scale=scale, eps=eps)
        assert all(torch.equal(a, b) for a, b in zip(again.all(), case.all()))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [math.inf, math.nan, -math.inf])
def test_a_norm_that_is_not_finite_leaves_everything(ctx, bad, bits):
    case = Case([3000, 17], "f32", "f32", "bf16", bits)
    case.g[1][3] = bad
    was = [t.clone() for t in case.all()]
    case.step(ctx, 5, 0.01, norm=ctx.clip_grad_norm(case.g, math.inf), max_norm=1.0)
    assert all(torch.equal(a, b) for a, b in zip(case.all(), was))


@pytest.mark.parametrize("bits", [32, 8])
def test_step_and_rate_in_device_memory_and_in_a_graph(ctx, bits):
    eager, replayed = Case([3000, 17, 70000], "f32", "bf16", "bf16", bits), Case([3000, 17, 70000], "f32", "bf16", "bf16", bits)
    one = Case([3000, 17, 70000], "f32", "bf16", "bf16", bits)
    step, lr = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):           # the first call there is: it needs no work buffer
        step += 1
        replayed.step(ctx, step, lr, seed=9)
    for t in range(1, 6):
        rate = float(torch.tensor(0.01 / t, dtype=torch.float32))
        lr.fill_(rate)
        eager.step(ctx, torch.full((1,), t, device="cuda"), torch.full((1,), rate, device="cuda"), seed=9)
        was = before(one, ctx)
        one.step(ctx, t, rate, seed=9)
        check_32(one, was, ctx, t, rate)
        graph.replay()
    torch.cuda.synchronize()
    assert int(step) == 5 and all(torch.equal(a, b) for a, b in zip(eager.all(), replayed.all()))
    for a, b in zip(eager.p, one.p):        # factors from the host and from the device differ by a rounding
        assert float((a - b).abs().max()) <= 1e-6


@pytest.mark.parametrize("bits", [32, 8])
def test_other_streams_and_the_same_bits(ctx, bits):
    cases = [Case([5000, 300, 100000], "f32", "bf16", "f16", bits, 5) for _ in range(4)]
    torch.cuda.synchronize()
    for t in (1, 2, 3):
        for case in cases[1:]:
            case.step(ctx, t, 0.01, stream=torch.cuda.Stream())
            torch.cuda.synchronize()
        cases[0].step(ctx, t, 0.01)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for c in cases[1:] for a, b in zip(c.all(), cases[0].all()))


def test_extreme_gradients_and_moments(ctx):
    """Elements that have had no gradient stand still, whatever their neighbours hold; infinities and NaN go their way alone."""
    case = Case([1000], "f32", "f32")
    for t in (*case.m, *case.v, *case.g):
        t.zero_()
    case.g[0][5], case.g[0][6], case.g[0][7], case.g[0][8] = math.inf, math.nan, 1e18, 1e-18
    was = case.p[0].clone()
    case.step(ctx, 1, 0.01, weight_decay=0.0)
    still = torch.ones(1000, dtype=torch.bool, device="cuda")
    still[5:9] = False
    assert torch.equal(case.p[0][still], was[still]) and not torch.isfinite(case.p[0][5:7]).any()
    # g / (|g| + eps) = 1 for any size of g that is not small beside eps
    assert abs(float(was[7] - case.p[0][7]) - 0.01) <= 2.0 ** -23
    assert abs(float(was[8] - case.p[0][8])) <= 0.01 * 1e-9


@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-18, 1e-14, 1e-11, 3e-11, 1e-8])
def test_small_moments_and_small_eps(ctx, eps):
    """An exp_avg_sq from 2^-126 to 2^-100 counts as what it is, a smaller one (zero too) as 2^-126; NaN stays NaN."""
    n = 27 * 64
    case = Case([n + 3], bits=32)
    case.g[0].zero_()
    case.p[0].zero_()
    v = power_of_two(torch.arange(-126, -99, device="cuda")).repeat_interleave(64) * (1.01 + torch.rand(n, dtype=torch.float64, generator=gen(3), device="cuda"))
    case.v[0][:n] = v.float()
    case.v[0][n:] = torch.tensor([0.0, 2.0 ** -149, math.nan], device="cuda")
    case.m[0][:n] = (v.sqrt() * torch.rand(n, dtype=torch.float64, generator=gen(4), device="cuda")).float()
    case.m[0][n:] = 2.0 ** -64
    was = before(case, ctx)
    case.step(ctx, 3, 0.01, eps=eps, weight_decay=0.0)
    assert torch.isnan(case.p[0][-1])
    for t in (case.p, case.m, case.v, *was):
        t[0] = t[0][:n]
    case.g[0], case.sizes = case.g[0][:n], [n]
    least = -0.01 / (1 - 0.9 ** 3) * 0.9 * 2.0 ** -64 / (math.sqrt(2.0 ** -126 / (1 - 0.999 ** 3)) + eps)
    flat = case.around[0][0]
    assert bool(((flat[n:n + 2].double() - least).abs() <= 40 * U * abs(least)).all())
    m, v, p, m_size, slack = formula(case.g[0], was[1][0], was[2][0], was[0][0], 3, 0.01, eps=eps, weight_decay=0.0)
    assert bool((v >= 2.0 ** -126).all())
    within(case.p[0], p, slack)


# ---- states of 8 bits ----------------------------------------------------------------------------------

def mix(x):
    x = ((x ^ (x >> 16)) * 0x9E3779B9) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0xBB67AE85) & 0xFFFFFFFF
    return x ^ (x >> 16)


def check_codes(case, was, step, seed, betas=(0.9, 0.999)):
    """Codes and exponents after a step: each code is the one that its definition gives for the value in 64 bits, or, where the value
    is within 8 u of where the decision turns, its neighbour."""
    number = close = total = 0
    for i, n in enumerate(case.sizes):
        blocks = -(-n // BLOCK)
        if n == 0:
            continue
        m, v, *_ = formula(case.g[i], was[1][i], was[2][i], was[0][i], step, 0.0, betas=betas)
        key = mix(mix(mix(torch.tensor(seed & 0xFFFFFFFF)) ^ (seed >> 32)) ^ step).cuda()
        at = torch.arange(n, device="cuda")
        random = mix(mix(key ^ (number + at // BLOCK)) ^ (at % BLOCK))
        number += blocks
        for name, x, code, e, offset, r, signed in (("m", m, case.m[i], case.e[i][:, 0], 897, random >> 16, True), ("v", v, case.v[i], case.e[i][:, 1], 769, random & 0xFFFF, False)):
            top = torch.zeros(blocks * BLOCK, dtype=torch.float64, device="cuda")
            top[:n] = x.abs()
            top = top.view(-1, BLOCK).amax(1)
            power = power_of_two(e.long() - 127)
            # 2^(E - 127) <= largest < 2^(E - 126), give or take 8 u (a block without a value above zero has E = 0)
            assert bool(((top >= power * (1 - 8 * U)) & (top < 2 * power * (1 + 8 * U)) | (e == 0) & (top < 2.0 ** -126)).all()), name
            y = x.abs() / power.repeat_interleave(BLOCK)[:n]
            turn = ((r.double() + 0.5) * 2.0 ** -16)              # rounded up where the place between the neighbours is above 1 - turn
            least = 1.25 * 2.0 ** ((offset + 1) // 8 - 127)
            gap = power_of_two(torch.frexp(y.clamp(min=least)).exponent - 4)
            down = torch.floor(y / gap) * gap
            place = (y - down) / gap
            want = down + gap * (place + turn >= 1.0)
            low = (y > 0).double() if not signed else (turn * least < y).double()
            want = torch.where(y < least, low * least, want)
            got = decode(code, torch.full_like(e, 127), offset, signed).abs()
            # m's terms may cancel: its error is 5 u of them
            size = y if not signed else (betas[0] * was[1][i].abs() + (1 - betas[0]) * case.g[i].double().abs()) / power.repeat_interleave(BLOCK)[:n]
            near = ((place + turn - 1.0).abs() * gap <= 8 * U * size) | (place * gap <= 8 * U * size) | ((1 - place) * gap <= 8 * U * size) | \
                   ((y - least).abs() <= 8 * U * size) | ((turn * least - y).abs() <= 8 * U * size)
            wrong = (got != want) & ~(near & ((got - want).abs() <= 2 * gap))
            assert not bool(wrong.any()), (name, i, int(wrong.sum()), float(y[wrong][0]), float(got[wrong][0]), float(want[wrong][0]))
            close, total = close + int((near & (y > 0)).sum()), total + n
            if signed:
                sign = decode(code, torch.full_like(e, 127), offset, True)
                assert bool((sign * x >= 0).all())
            else:
                assert bool(((code > 0) == (x > 0)).all())
    # few are near a turn: 0.1 g has four significant bits for about one in forty values of g in bfloat16
    assert total < 5000 or close < 0.05 * total


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_values(ctx, dtype):
    """Every code at several exponents, exactly; views that start anywhere."""
    for shift in (0, 1, 8):
        codes = torch.arange(256, dtype=torch.uint8, device="cuda").repeat(6)
        m, v = (torch.cat([torch.zeros(shift, dtype=torch.uint8, device="cuda"), codes])[shift:] for _ in range(2))
        e = torch.tensor([[0, 255], [1, 254], [127, 127], [200, 40], [255, 0], [254, 1]], dtype=torch.uint8, device="cuda")
        (gm,), (gv,) = ctx.adamw_values([m], [v], [e], dtype=dtype)
        for got, code, column, offset, signed in ((gm, m, 0, 897, True), (gv, v, 1, 769, False)):
            want = decode(code, e[:, column], offset, signed)
            want = want.to(torch.float32)      # overflows of the largest exponent, denormals of the smallest
            if dtype == torch.bfloat16:
                want = want.to(torch.bfloat16)
            assert got.dtype == dtype and torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(), want.nan_to_num())
    one, many = ctx.adamw_values([m[:n] for n in (0, 1, 300, 256, 7)], [v[:n] for n in (0, 1, 300, 256, 7)], [e[:-(-n // BLOCK)] for n in (0, 1, 300, 256, 7)])
    assert [len(t) for t in one] == [len(t) for t in many] == [0, 1, 300, 256, 7]
    assert torch.equal(many[2].nan_to_num(), decode(v[:300], e[:2, 1], 769, False).float().nan_to_num())


@pytest.mark.parametrize("scale", [1e-30, 1e-18, 1.0, 1e17])
def test_sizes_of_states(ctx, scale):
    """Over the range of single precision; an element far below its block's largest keeps a v above zero."""
    case = Case([1024], bits=8)
    for t in (*case.m, *case.v, *case.e):
        t.zero_()
    case.g[0].copy_(torch.randn(1024, generator=gen(2), device="cuda") * scale)
    case.g[0][::2] *= 1e-6
    case.g[0][1::8] = 0.0
    for t in (1, 2, 3):
        was = before(case, ctx)
        case.step(ctx, t, 0.01, seed=2)
        if scale > 1e-18:
            check_codes(case, was, t, 2)
        change = (case.p[0].double() - was[0][0] * (1 - 0.01 * 0.01)).abs()
        assert bool((change <= 0.1).all()) and bool((change[1::8] <= 1e-12 + 2.0 ** -24).all())
    if scale >= 1e-18:
        held = (case.g[0].double() ** 2 * 0.001).float() > 0
        assert bool((case.v[0][held] > 0).all())


@pytest.mark.parametrize("small", [1e-3, 1e-6, 1e-10, 1e-18])
@pytest.mark.parametrize("n", [1024, 777])
def test_moments_far_below_their_neighbours(ctx, n, small):
    """An exp_avg_sq above zero never becomes zero, not even where its block's largest is 2^200 times it."""
    case = Case([n], bits=8)
    for t in (*case.m, *case.v, *case.e):
        t.zero_()
    case.g[0].fill_(small)
    case.g[0][::100] = 1e19
    case.g[0][1::100] = 0.0
    was = before(case, ctx)
    case.step(ctx, 1, 0.01, seed=4)
    check_codes(case, was, 1, 4)
    assert torch.equal(case.v[0] > 0, case.g[0] != 0)


def test_rounding_keeps_the_mean(ctx):
    """400 000 elements with the same history under different seeds and places: the means of m and v follow the formula to six
    standard deviations of the mean; v follows gradients that became ten times smaller."""
    n = 400_000
    case = Case([n], bits=8)
    for t in (*case.m, *case.v, *case.e):
        t.zero_()
    m = v = 0.0
    for t in range(1, 1201):
        g = (1.0 if t <= 300 else 0.1) * (1.0 + 0.5 * math.sin(t))
        case.g[0].fill_(g)
        case.step(ctx, t, 0.0, seed=3)
        g = float(case.g[0][0])
        m, v = 0.9 * m + 0.1 * g, 0.999 * v + 0.001 * g * g
        if t == 300:
            most = v
        if t % 300 == 0:
            (gm,), (gv,) = ctx.adamw_values(case.m, case.v, case.e)
            for got, want in ((gm.double(), m), (gv.double(), v)):
                deviation = float(got.std()) / math.sqrt(n)
                # 16 random bits, centred; the sums' own roundings, t of them at most
                assert abs(float(got.mean()) - want) <= 6 * deviation + t * 2 * U * abs(want), (t, float(got.mean()), want, deviation)
                assert float(got.std()) <= 0.5 * abs(want)
    assert v < 0.5 * most                   # (most of what was gathered has gone)


def test_blocks_that_are_not_finite(ctx):
    case = Case([1000], bits=8, seed=6)
    case.g[0][300], case.g[0][700] = math.inf, math.nan
    other = Case([1000], bits=8, seed=6)
    case.step(ctx, 2, 0.01)
    other.step(ctx, 2, 0.01)
    (m,), (v,) = ctx.adamw_values(case.m, case.v, case.e)
    assert torch.isnan(m[256:768]).all() and torch.isnan(v[256:768]).all()
    for k in ("p", "m", "v"):
        a, b = getattr(case, k)[0], getattr(other, k)[0]
        assert torch.equal(a[:256], b[:256]) and torch.equal(a[768:], b[768:])
    case.g[0].fill_(1.0)
    case.step(ctx, 3, 0.01)                 # and stay so
    (m,), _ = ctx.adamw_values(case.m, case.v, case.e)
    assert torch.isnan(m[256:768]).all() and torch.isfinite(m[:256]).all() and torch.isnan(case.p[0][256:768]).all()


def test_more_elements_than_31_bits(ctx):
    """Offsets beyond 2^31 elements: the last blocks of a tensor against the same blocks alone (its number within the call shifted by
    as many blocks of other tensors)."""
    n = 2 ** 31 + 1000
    p, g = (torch.zeros(n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2))
    e = torch.zeros((-(-n // BLOCK), 2), dtype=torch.uint8, device="cuda")
    g[-1500:] = torch.randn(1500, generator=gen(1), device="cuda").bfloat16()
    p[:1500] = 1.0
    ctx.adamw([p], [g], [m], [v], 1, 0.5, exponents=[e], weight_decay=0.25)
    tail = n - (n // BLOCK - 5) * BLOCK                      # the last blocks, from a block's start
    assert bool((p[:1500] == 0.875).all()) and not p[1500:-1500].any()
    want = -0.5 * torch.sign(g[-1500:].double())
    assert bool(((p[-1500:].double() - want).abs() <= 2.0 ** -8 * 0.5 + 1e-5).all())
    (gm,), (gv,) = ctx.adamw_values([m[-tail:]], [v[-tail:]], [e[-(-(-tail // BLOCK)):]])
    want = 0.1 * g[-1500:].double()
    assert bool(((gm[-1500:].double() - want).abs() <= want.abs() / 8 + 1e-5).all()) and not m[:-1500].any()
    (fm,), (fv,) = ctx.adamw_values([m], [v], [e], dtype=torch.bfloat16)
    assert torch.equal(fm[-tail:].float(), gm) and torch.equal(fv[-tail:].float(), gv)


# ---- refusals and bookkeeping --------------------------------------------------------------------------

def test_refusals(ctx):
    from paper_2207_09682_b200 import binding
    t = lambda n=300, dtype=torch.float32: torch.ones(n, dtype=dtype, device="cuda")  # noqa: E731
    p, g, m, v = t(), t(), t(), t()
    byte, e = t(300, torch.uint8), t(2 * 2, torch.uint8).view(2, 2)
    many = lambda **k: ctx.adamw([p], [g], [m], [v], k.pop("step", 1), k.pop("lr", 0.1), **k)  # noqa: E731
    matrix = torch.ones((20, 15), device="cuda")
    bad = [
        lambda: ctx.adamw([p], [g, g], [m], [v], 1, 0.1), lambda: ctx.adamw([p], [g], [], [v], 1, 0.1), lambda: ctx.adamw([p], [t(299)], [m], [v], 1, 0.1),
        lambda: ctx.adamw([p], [g], [t(301)], [v], 1, 0.1), lambda: ctx.adamw([p.double()], [g], [m], [v], 1, 0.1), lambda: ctx.adamw([p], [g.long()], [m], [v], 1, 0.1),
        lambda: ctx.adamw([p], [g], [m.half()], [v], 1, 0.1), lambda: ctx.adamw([p], [g], [byte], [byte], 1, 0.1), lambda: many(exponents=[e]),
        lambda: ctx.adamw([p], [g], [byte], [byte.clone()], 1, 0.1, exponents=[e[:1]]), lambda: ctx.adamw([p], [g], [byte], [byte.clone()], 1, 0.1, exponents=[e.int()]),
        lambda: ctx.adamw([p], [g], [byte], [byte.clone()], 1, 0.1, exponents=[e.t()]),
        lambda: ctx.adamw([matrix.t()], [g], [m], [v], 1, 0.1), lambda: ctx.adamw([p.cpu()], [g], [m], [v], 1, 0.1), lambda: ctx.adamw([torch._neg_view(p)], [g], [m], [v], 1, 0.1),
        lambda: ctx.adamw([p, p], [g, g], [m, t()], [v, t()], 1, 0.1), lambda: ctx.adamw([p[10:], p[:20]], [g[10:], g[:20]], [m[10:], m[:20]], [v[10:], v[:20]], 1, 0.1),
        lambda: many(step=0), lambda: many(step=torch.ones(1, device="cuda")), lambda: many(step=torch.ones(2, dtype=torch.int64, device="cuda")), lambda: many(lr=-1.0),
        lambda: many(lr=math.nan), lambda: many(lr=torch.ones(1, device="cuda").double()), lambda: many(betas=(1.0, 0.9)), lambda: many(betas=(0.9, -0.1)), lambda: many(eps=-1.0),
        lambda: many(weight_decay=-1.0), lambda: many(weight_decay=math.inf), lambda: many(loss_scale=0.0), lambda: many(norm=t(1), max_norm=-1.0), lambda: many(norm=t(2)),
        lambda: many(copies=[t(299)]), lambda: many(copies=[t(300).long()]), lambda: many(copies=[]),
        lambda: ctx.adamw_values([byte], [byte], [e[:1]]), lambda: ctx.adamw_values([m], [byte], [e]), lambda: ctx.adamw_values([byte], [byte], [e], dtype=torch.float16),
    ]
    for k, call in enumerate(bad):
        with pytest.raises(binding.QgbdtError) as error:
            call()
        assert error.value.code == binding.ERR_ARG, k
    with pytest.raises(TypeError):
        many(step=1.5)
    assert all(bool((x == 1).all()) for x in (p, g, m, v, byte, e))
    many()
    assert bool((p != 1).all())


def test_bookkeeping(ctx):
    """Versions, gradients that require one, parameters that do, lists of any kind, tensors on another stream."""
    p, g, m, v, c = (torch.ones(300, device="cuda") for _ in range(5))
    p.requires_grad_()
    ctx.adamw(iter([p]), (g,), [m], [v], 1, 0.1, copies=[c])
    assert p._version == m._version == v._version == c._version == 1 and g._version == 0 and p.requires_grad
    g.requires_grad_()
    with pytest.warns(UserWarning, match="grads requires a gradient"):
        ctx.adamw([p], [g], [m], [v], 2, 0.1)
    with torch.no_grad():
        ctx.adamw([p], [g], [m], [v], 3, 0.1)
    ctx.adamw([], [], [], [], 1, 0.1)
    step = torch.ones(1, dtype=torch.int64, device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.no_grad():
        ctx.adamw(iter([p]), iter([g]), iter([m]), iter([v]), step, torch.ones(1, device="cuda"), copies=iter([c]), stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(c, p.detach())


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("tensors", [15, 16, 17, 55, 56, 57, 400, 401, 801])
def test_where_the_tables_of_tensors_change(ctx, tensors, bits):
    """Up to 16, 56 and 400 tensors per launch, and more launches; the values of 8-bit states through all of them."""
    sizes = [(53 * i + 300) % 900 for i in range(tensors)]
    case = Case(sizes, "f32", "bf16", "bf16", bits, tensors)
    was = before(case, ctx)
    case.step(ctx, 3, 0.02, seed=11)
    check_32(case, was, ctx, 3, 0.02)
    if bits == 8:
        check_codes(case, was, 3, 11)
        for dtype in (torch.float32, torch.bfloat16):
            m, v = ctx.adamw_values(case.m, case.v, case.e, dtype=dtype)
            for i, n in enumerate(sizes):
                assert m[i].shape == v[i].shape == (n,) and m[i].dtype == v[i].dtype == dtype
                assert torch.equal(m[i].double(), decode(case.m[i], case.e[i][:, 0], 897, True)) and torch.equal(v[i].double(), decode(case.v[i], case.e[i][:, 1], 769, False))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("tensors", [3, 30, 500])
def test_small_eps_in_many_tensors(ctx, tensors, bits):
    """An eps that needs the maximum goes through the large tables whatever the number of tensors."""
    case = Case([(71 * i + 1) % 700 for i in range(tensors)], "f32", "f16", None, bits, tensors)
    was = before(case, ctx)
    case.step(ctx, 3, 0.02, eps=0.0, seed=12)
    check_32(case, was, ctx, 3, 0.02, eps=0.0)
    if bits == 8:
        check_codes(case, was, 3, 12)

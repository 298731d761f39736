"""Layer norm, forward and backward, against the formulas in 64 bits.

Tolerances.  u = 2^-24 is one rounding in single precision; an output of type T is rounded once more, by at most
finfo(T).eps / 2 of its value.  A sum over a row of d elements passes through at most d / 256 + 80 additions in a row (a
thread's own elements, the lanes of a warp, the warps of a block), so that it is off by at most that many u times the sum
of its terms' magnitudes.  A sum over n rows: a block or a group of threads adds the rows it has, at most n / 16 + 200 of them
one after the other, joins included.
"""
import ctypes as C
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = 2.0 ** -24


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


def make(rows, dim, dtype, wtype, pad=0, seed=1, shift=0, offset=0.3):
    """x, g [rows, dim] inside wider matrices (from column `shift` on), weight, bias."""
    g = gen(seed)
    m = [torch.randn((rows, dim + pad + shift), generator=g, device="cuda") for _ in range(2)]
    m[0] = (m[0] + offset) * (0.1 + torch.rand((rows, 1), generator=g, device="cuda"))
    x, grad = (t.to(dtype)[:, shift:shift + dim] for t in m)
    w, b = 1.0 + 0.3 * torch.randn(dim, generator=g, device="cuda"), 0.2 * torch.randn(dim, generator=g, device="cuda")
    return x, grad, w.to(wtype), b.to(wtype)


def check_forward(r, x, w, b, eps=1e-5):
    d = x.shape[1]
    chain = d / 256 + 80
    x = x.double()
    w = torch.ones(d, dtype=torch.float64, device="cuda") if w is None else w.double()
    b = torch.zeros(d, dtype=torch.float64, device="cuda") if b is None else b.double()
    mean = x.mean(1, keepdim=True)
    off = x - mean
    var = (off * off).mean(1, keepdim=True) + eps
    rstd = var.rsqrt()
    d_mean = (chain + 2) * U * x.abs().mean(1, keepdim=True)            # the sum, times 1 / d
    # var: terms off by two roundings of (x - mean), which the mean's error shifts (its square is left: the terms themselves add
    # up to zero), the sum, the factor and the fused addition; rstd is half as far off, and one rounding
    rel = ((chain + 6) * U + d_mean ** 2 / var) / 2 + 2 * U
    within(r.mean, mean.squeeze(1), d_mean.squeeze(1), "mean")
    within(r.rstd, rstd.squeeze(1), (rel * rstd).squeeze(1), "rstd")
    xh = off * rstd
    slack = w.abs() * (d_mean * rstd + xh.abs() * (rel + 3 * U)) + 2 * U * (w * xh).abs() + U * b.abs()
    within(r.out, xh * w + b, slack, "out")


def check_backward(got, g, x, mean, rstd, w):
    n, d = x.shape
    chain, rows = d / 256 + 80, n / 16 + 200
    g, x, mean, rstd = g.double(), x.double(), mean.double()[:, None], rstd.double()[:, None]
    weight = torch.ones(d, dtype=torch.float64, device="cuda") if w is None else w.double()
    xh = (x - mean) * rstd
    wg = g * weight
    c1, c2 = wg.mean(1, keepdim=True), (wg * xh).mean(1, keepdim=True)
    # xh is off by two roundings, w g by one; the sums by their chains, the factor 1 / d by one
    d1 = (chain + 3) * U * wg.abs().mean(1, keepdim=True)
    d2 = (chain + 6) * U * (wg * xh).abs().mean(1, keepdim=True)
    slack = rstd * (d1 + xh.abs() * d2 + 5 * U * (wg.abs() + c1.abs() + (xh * c2).abs()))
    within(got[0], (wg - c1 - xh * c2) * rstd, slack, "grad_x")
    if w is None:
        assert got[1] is None and got[2] is None
        return
    within(got[1], (g * xh).sum(0), (rows + 4) * U * (g * xh).abs().sum(0), "grad_weight")
    within(got[2], g.sum(0), (rows + 4) * U * g.abs().sum(0), "grad_bias")


SIZES = [
    # rows, dim, pad
    (1, 1, 0), (3, 2, 0), (2, 3, 1), (1, 8, 0), (5, 7, 0), (64, 16, 0), (33, 24, 8), (17, 31, 0), (9, 32, 0), (40, 33, 5), (1000, 64, 0), (7, 100, 0), (300, 129, 0),
    (1, 256, 0), (4099, 256, 0), (7, 257, 0), (129, 511, 1), (65, 512, 0), (31, 520, 0), (513, 770, 30), (150, 1000, 24), (600, 1023, 0), (700, 1024, 0), (1, 1025, 0),
    (20, 1032, 0), (37, 2047, 0), (300, 2048, 0), (3, 2050, 6), (10, 4095, 2), (150, 4096, 0), (5, 5000, 0), (149, 8192, 0), (9, 8191, 0), (2, 8193, 0), (6, 8200, 0),
    (160, 12288, 0), (4, 16384, 0), (3, 16385, 0), (2, 40000, 0), (1, 100003, 0), (1, 1 << 20, 0), (3, 300001, 3), (70, 12289, 0), (1200, 8200, 0),
    (300, 14336, 0), (300, 14340, 0), (1000, 16384, 0), (20, 9000, 24), (160, 16376, 0),
]


@pytest.mark.parametrize("dtype,wtype", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("f16", "f16")])
@pytest.mark.parametrize("rows,dim,pad", SIZES)
def test_both_directions(ctx, rows, dim, pad, dtype, wtype):
    x, g, w, b = make(rows, dim, DTYPES[dtype], DTYPES[wtype], pad, 3 * rows + dim)
    r = ctx.layer_norm(x, w, b)
    assert r.out.dtype == x.dtype and r.out.shape == x.shape and r.mean.shape == r.rstd.shape == (rows,)
    check_forward(r, x, w, b)
    got = ctx.layer_norm_backward(g, x, r.mean, r.rstd, w)
    assert got[0].dtype == x.dtype and got[1].dtype == got[2].dtype == w.dtype
    check_backward(got, g, x, r.mean, r.rstd, w)
    again = ctx.layer_norm_backward(g, x, r.mean, r.rstd, w)      # the same bits every time
    assert all(torch.equal(p, q) for p, q in zip(got, again))


@pytest.mark.parametrize("rows,dim", [(70000, 24), (65536, 256), (100003, 40), (30011, 515), (20000, 1024), (9000, 4096), (1 << 20, 8), (300000, 1), (1 << 18, 33)])
def test_many_rows(ctx, rows, dim):
    x, g, w, b = make(rows, dim, torch.bfloat16, torch.float32, 0, 2)
    r = ctx.layer_norm(x, w, b)
    check_forward(r, x, w, b)
    check_backward(ctx.layer_norm_backward(g, x, r.mean, r.rstd, w), g, x, r.mean, r.rstd, w)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,dim,pad,shift", [(50, 64, 7, 1), (50, 64, 12, 4), (9, 1024, 1, 3), (3, 9000, 3, 5), (50, 64, 8, 8),
                                                 (3000, 128, 1, 1), (3000, 256, 1, 7), (2000, 512, 3, 1), (1500, 1024, 1, 5), (700, 1536, 1, 2),
                                                 (700, 4096, 1, 3), (400, 8192, 5, 7)])
def test_rows_that_start_anywhere(ctx, rows, dim, pad, shift, dtype):
    """Inputs and outputs inside wider matrices; what is around the outputs stays as it was."""
    x, g, w, b = make(rows, dim, DTYPES[dtype], DTYPES[dtype], pad, 5, shift)
    r = ctx.layer_norm(x, w, b)
    check_forward(r, x, w, b)
    got = ctx.layer_norm_backward(g, x, r.mean, r.rstd, w)
    check_backward(got, g, x, r.mean, r.rstd, w)
    for left in (1, 8):
        around = torch.full((rows + 2, dim + 2 * left), 7.0, device="cuda").to(x.dtype)
        into = around[1:-1, left:-left]
        q = ctx.layer_norm(x, w, b, out=into)
        assert q.out.data_ptr() == into.data_ptr()
        check_forward(q, x, w, b)           # rows that allow other vectors are summed in another order
        into.fill_(7.0)
        assert bool((around == 7.0).all())
        check_backward(ctx.layer_norm_backward(g, x, r.mean, r.rstd, w, grad_x=into), g, x, r.mean, r.rstd, w)
        into.fill_(7.0)
        assert bool((around == 7.0).all())


@pytest.mark.parametrize("rows,dim", [(70, 64), (70, 129), (300, 1024), (200, 2048), (5, 8192), (500, 16384), (3, 20000), (3, 20001)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place(ctx, rows, dim, dtype):
    x, g, w, b = make(rows, dim, DTYPES[dtype], torch.float32, 0, 6)
    r = ctx.layer_norm(x, w, b)
    want = ctx.layer_norm_backward(g, x, r.mean, r.rstd, w)
    y = x.clone()
    q = ctx.layer_norm(y, w, b, out=y)
    assert torch.equal(y, r.out) and torch.equal(q.mean, r.mean) and torch.equal(q.rstd, r.rstd)
    for into in (0, 1):
        inputs = [g.clone(), x.clone()]
        got = ctx.layer_norm_backward(*inputs, r.mean, r.rstd, w, grad_x=inputs[into])
        assert got[0].data_ptr() == inputs[into].data_ptr() and all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("rows,dim", [(70, 64), (70, 129), (200, 2048), (3, 20000)])
def test_without_weight_or_bias(ctx, rows, dim):
    x, g, w, b = make(rows, dim, torch.float16, torch.float32, 0, 7)
    for weight, bias in ((None, None), (w, None), (None, b)):
        r = ctx.layer_norm(x, weight, bias)
        check_forward(r, x, weight, bias)
        check_backward(ctx.layer_norm_backward(g, x, r.mean, r.rstd, weight), g, x, r.mean, r.rstd, weight)


def test_no_rows_and_single_rows_of_any_stride(ctx):
    """C ABI too: sums over no rows are zeros; results that are not wanted; the stride of a single row means nothing."""
    from paper_2207_09682_b200 import binding
    for dim in (8, 33, 20000):
        x, g, w, b = make(0, dim, torch.bfloat16, torch.bfloat16)
        r = ctx.layer_norm(x, w, b)
        assert r.out.shape == (0, dim) and r.mean.shape == (0,)
        gx, gw, gb = ctx.layer_norm_backward(g, x, r.mean, r.rstd, w)
        assert gx.shape == (0, dim) and not gw.any() and not gb.any()
        x, g, w, b = make(1, dim, torch.bfloat16, torch.bfloat16)
        r = ctx.layer_norm(x, w, b)
        p = lambda t: C.c_void_p(None if t is None else t.data_ptr())  # noqa: E731
        far, stream, out = C.c_int64(1 << 50), C.c_void_p(torch.cuda.current_stream().cuda_stream), torch.zeros_like(x)
        assert ctx.lib.qgbdt_layer_norm(ctx.h, p(x), far, 1, p(w), p(b), 1, C.c_int64(1), dim, C.c_double(1e-5), p(out), far, None, None, stream) == binding.OK
        assert torch.equal(out, r.out)
        want = ctx.layer_norm_backward(g, x, r.mean, r.rstd, w)
        for gw, gb in ((None, None), (torch.ones_like(w), None), (None, torch.ones_like(w))):
            assert ctx.lib.qgbdt_layer_norm_backward(ctx.h, p(g), far, p(x), far, 1, p(r.mean), p(r.rstd), p(w), 1, C.c_int64(1), dim, p(out), far, p(gw), p(gb),
                                                     stream) == binding.OK
            assert torch.equal(out, want[0]) and (gw is None or torch.equal(gw, want[1])) and (gb is None or torch.equal(gb, want[2]))


@pytest.mark.parametrize("dim", [16, 100, 1024, 3000, 20000])
def test_rows_of_equal_values_large_offsets_and_infinities(ctx, dim):
    """Equal values leave the bias (the mean of a row's equal values may be one rounding off, which rstd = eps^-1/2 scales); a row
    with an infinity or a NaN is NaN where it is and leaves the others alone."""
    x, g, w, b = make(12, dim, torch.float32, torch.float32, 0, 9)
    x[0], x[1] = 0.0, 4.0
    x[2] = 3.7
    x[3] += 1e4
    r = ctx.layer_norm(x, w, b)
    check_forward(r, x, w, b)
    assert torch.equal(r.out[0], b) and float(r.mean[0]) == 0.0
    check_backward(ctx.layer_norm_backward(g, x, r.mean, r.rstd, w), g, x, r.mean, r.rstd, w)
    y = x.clone()
    y[5, dim // 2], y[7, 0], y[8, dim - 1] = math.inf, math.nan, -math.inf
    q = ctx.layer_norm(y, w, b)
    bad = torch.zeros(12, dtype=torch.bool, device="cuda")
    bad[[5, 7, 8]] = True
    assert torch.equal(q.out[~bad], r.out[~bad]) and torch.equal(q.rstd[~bad], r.rstd[~bad])
    assert not torch.isfinite(q.out[7]).any() and torch.isnan(q.rstd[bad]).all()
    gx = ctx.layer_norm_backward(g, y, q.mean, q.rstd, w)[0]
    assert torch.equal(gx[~bad], ctx.layer_norm_backward(g, x, r.mean, r.rstd, w)[0][~bad]) and torch.isnan(gx[bad]).all()
    # no eps: the same, with an infinite rstd for equal values
    z = ctx.layer_norm(x, w, b, eps=0.0)
    assert math.isinf(float(z.rstd[0])) and torch.isnan(z.out[0]).all()
    check_forward(binding_rows(z, 4), x[4:], w, b, 0.0)


def binding_rows(r, start):
    return type(r)(r.out[start:], r.mean[start:], r.rstd[start:])


@pytest.mark.parametrize("dim", [12, 100, 1500])
def test_gradients_by_differences(ctx, dim):
    """sum(c * out) along a direction in x, weight and bias: central differences of the kernel's own results."""
    x, c, w, b = make(6, dim, torch.float32, torch.float32, 0, 4)
    r = ctx.layer_norm(x, w, b)
    grads = ctx.layer_norm_backward(c, x, r.mean, r.rstd, w)
    step = 2.0 ** -6

    def plain(x, w, b):
        off = x - x.mean(1, keepdim=True)
        return (c.double() * (off * ((off * off).mean(1, keepdim=True) + 1e-5).rsqrt() * w + b)).sum()

    for k, grad in enumerate(grads):
        at = [t.double() for t in (x, w, b)]
        e = torch.randint(-1, 2, at[k].shape, generator=gen(k), device="cuda").double() * step
        ends, exact = [], []
        for sign in (1, -1):
            moved = list(at)
            moved[k] = (at[k] + sign * e).float().double()
            ends.append(float((c.double() * ctx.layer_norm(*(t.float() for t in moved)).out.double()).sum()))
            exact.append(float(plain(*moved)))
        leaves = [t.requires_grad_() for t in at]
        slope = float((torch.autograd.grad(plain(*leaves), leaves[k])[0] * e).sum())
        curved = abs((exact[0] - exact[1]) / 2 - slope)      # what a difference over 2 steps leaves out, by the formula in 64 bits
        # the outputs of both ends are off by their sums' chains (90 u of values of a few units); the gradient by 100 u of its terms
        slack = 2 * 100 * U * float((c.abs() * (r.out.abs() + 4 * w.abs())).sum()) + 100 * U * float((grad.abs() * e.abs()).sum()) * 4
        assert abs((ends[0] - ends[1]) / 2 - float((grad.double() * e).sum())) <= curved + slack


def test_rows_far_apart(ctx):
    """Offsets beyond 2^31 elements."""
    wide = torch.zeros((3, 2 ** 30 + 8), dtype=torch.float16, device="cuda")
    for dim in (40, 41, 9000):
        x, g, w, b = make(3, dim, torch.float16, torch.float32, 0, 8)
        far = wide[:, :dim]
        far.copy_(x)
        r, q = ctx.layer_norm(x, w, b), ctx.layer_norm(far, w, b)
        assert all(torch.equal(s, t) for s, t in zip(r, q))
        want = ctx.layer_norm_backward(g, x, r.mean, r.rstd, w)
        got = ctx.layer_norm_backward(g, far, r.mean, r.rstd, w)
        assert all(torch.equal(s, t) for s, t in zip(got, want))
        ctx.layer_norm(far, w, b, out=far)
        assert torch.equal(far, r.out) and not wide[:, dim:dim + 8].any()


def test_other_streams_and_graphs(ctx):
    """Calls on two streams share the work buffer of the sums; two graphs that are replayed after one another do."""
    cases = [make(rows, dim, torch.bfloat16, torch.float32, 0, rows) for rows, dim in ((5000, 256), (3000, 1024), (700, 4096), (50, 9000))]
    stats = [ctx.layer_norm(x, w, b) for x, _, w, b in cases]
    want = [ctx.layer_norm_backward(g, x, r.mean, r.rstd, w) for (x, g, w, _), r in zip(cases, stats)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(5):
        got = [ctx.layer_norm_backward(g, x, r.mean, r.rstd, w, stream=s) for (x, g, w, _), r, s in zip(cases, stats, streams)]
        again = [ctx.layer_norm(x, w, b, stream=s) for (x, _, w, b), s in zip(cases, streams)]
        torch.cuda.synchronize()
        for a, b in zip(got + again, want + stats):
            assert all(torch.equal(p, q) for p, q in zip(a, b))
    graphs = []
    for x, g, w, b in cases:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            r = ctx.layer_norm(x, w, b)
            out = ctx.layer_norm_backward(g, x, r.mean, r.rstd, w)
        graphs.append((graph, r, out))
    for _ in range(3):
        for graph, _, _ in graphs:
            graph.replay()
    torch.cuda.synchronize()
    for (_, r, out), s, w in zip(graphs, stats, want):
        assert all(torch.equal(p, q) for p, q in zip((*r, *out), (*s, *w)))


def test_bookkeeping(ctx):
    """Versions of written tensors, inputs that require a gradient, refusals of the module that takes tensors apart."""
    from paper_2207_09682_b200 import binding
    x, g, w, b = make(5, 16, torch.float16, torch.float32)
    r = ctx.layer_norm(x, w, b)
    out = torch.zeros_like(x)
    ctx.layer_norm(x, w, b, out=out)
    assert out._version == 1 and x._version == 0
    ctx.layer_norm_backward(g, x, r.mean, r.rstd, w, grad_x=out)
    assert out._version == 2 and g._version == 0
    # mean and rstd lie in one buffer, but are tensors of their own
    assert r.mean._version == r.rstd._version == 0 and not r.mean.requires_grad and r.mean.is_contiguous() and r.rstd.is_contiguous()
    was = r.rstd.clone()
    r.mean.add_(0.0)
    assert r.mean._version == 1 and r.rstd._version == 0 and torch.equal(r.rstd, was)
    scale = torch.ones(5, device="cuda", requires_grad=True)
    (r.mean * scale).sum().backward()
    assert torch.equal(scale.grad, r.mean)
    with torch.inference_mode():
        assert torch.equal(ctx.layer_norm(x, w, b).out, r.out)
    leaf = w.clone().requires_grad_()
    with pytest.warns(UserWarning, match="weight requires a gradient"):
        assert not ctx.layer_norm(x, leaf, b).out.requires_grad
    with pytest.warns(UserWarning, match="weight requires a gradient"):
        assert not ctx.layer_norm_backward(g, x, r.mean, r.rstd, leaf)[1].requires_grad
    bad = [
        lambda: ctx.layer_norm(x.double()), lambda: ctx.layer_norm(x.t()), lambda: ctx.layer_norm(x[0]), lambda: ctx.layer_norm(x[:, :0]), lambda: ctx.layer_norm(x.cpu()),
        lambda: ctx.layer_norm(x, w[:15]), lambda: ctx.layer_norm(x, w.bfloat16()), lambda: ctx.layer_norm(x, w, b.half()), lambda: ctx.layer_norm(x, w.double()),
        lambda: ctx.layer_norm(x, w, b, eps=-1.0), lambda: ctx.layer_norm(x, w, b, eps=math.nan), lambda: ctx.layer_norm(x, w, b, out=out[:4]),
        lambda: ctx.layer_norm(x, w, b, out=out.float()), lambda: ctx.layer_norm(x.expand(5, 16)[:1].expand(5, 16), w, b), lambda: ctx.layer_norm(x, w.view(4, 4).t()),
        lambda: ctx.layer_norm(torch._neg_view(x)), lambda: ctx.layer_norm(torch.empty((0, 2 ** 32 + 1), device="cuda")),
        lambda: ctx.layer_norm_backward(g.float(), x, r.mean, r.rstd, w), lambda: ctx.layer_norm_backward(g[:4], x, r.mean, r.rstd, w),
        lambda: ctx.layer_norm_backward(g, x, r.mean[:4], r.rstd, w), lambda: ctx.layer_norm_backward(g, x, r.mean, r.rstd.double(), w),
        lambda: ctx.layer_norm_backward(g, x, None, r.rstd, w), lambda: ctx.layer_norm_backward(g, x, r.mean, r.rstd, w, grad_x=out.float()),
        lambda: ctx.layer_norm_backward(g[:, ::2], x[:, ::2], r.mean, r.rstd, w[::2]),
    ]
    for call in bad:
        with pytest.raises(binding.QgbdtError) as e:
            call()
        assert e.value.code == binding.ERR_ARG
    assert torch.equal(ctx.layer_norm(x, w, b).out, r.out)


def test_outputs_over_inputs(ctx):
    """An output that overlaps an input without being it is refused; one whose rows lie between the input's is not."""
    from paper_2207_09682_b200 import binding
    _, _, w, b = make(1, 40, torch.float32, torch.float32)
    wide = torch.randn((60, 100), generator=gen(2), device="cuda")
    x, was = wide[:, :40], wide.clone()
    for out in (wide[:, 1:41], wide[:, 39:79], wide[1:, :40], wide.view(-1)[:60 * 50].view(60, 50)[:, :40], w.expand(1, 40), b.view(1, 40)):
        k = min(len(out), 59)
        with pytest.raises(binding.QgbdtError) as e:
            ctx.layer_norm(x[:k], w, b, out=out[:k])
        assert e.value.code == binding.ERR_ARG
    stats = torch.zeros(59, device="cuda")
    for g, y in ((x, wide[:, 60:]), (wide[:, 60:], x)):
        with pytest.raises(binding.QgbdtError):
            ctx.layer_norm_backward(g[:59], y[:59], stats, stats, w, grad_x=wide[1:, 20:60] if g is x else wide[:59, 30:70])
    with pytest.raises(binding.QgbdtError):
        ctx.layer_norm_backward(x[:1], wide[:1, 60:], stats[:1], stats[:1], w, grad_x=w.view(1, 40))
    assert torch.equal(wide, was)
    r = ctx.layer_norm(x, w, b, out=wide[:, 40:80])
    check_forward(r, was[:, :40], w, b)
    assert torch.equal(wide[:, :40], was[:, :40]) and torch.equal(wide[:, 80:], was[:, 80:])
    normed = r.out.clone()
    got = ctx.layer_norm_backward(x, r.out, r.mean, r.rstd, w, grad_x=r.out)
    check_backward(got, was[:, :40], normed, r.mean, r.rstd, w)
    assert torch.equal(wide[:, :40], was[:, :40]) and torch.equal(wide[:, 80:], was[:, 80:])


@pytest.mark.parametrize("rows,dim", [(70, 64), (70, 129), (3000, 40), (200, 2048), (3, 20000), (0, 16)])
def test_bias_without_a_weight_has_a_gradient(ctx, rows, dim):
    from paper_2207_09682_b200 import binding
    for dtype, btype in ((torch.float16, torch.float32), (torch.bfloat16, torch.bfloat16)):
        x, g, w, b = make(rows, dim, dtype, btype, 0, 7)
        r = ctx.layer_norm(x, None, b)
        gx, gw, gb = ctx.layer_norm_backward(g, x, r.mean, r.rstd, bias=b)
        assert gw is None and gb.dtype == btype
        within(gb, g.double().sum(0), (rows / 16 + 204) * U * g.double().abs().sum(0), "grad_bias")
        plain = ctx.layer_norm_backward(g, x, r.mean, r.rstd)
        assert torch.equal(gx, plain[0]) and plain[1] is None and plain[2] is None
        both = ctx.layer_norm_backward(g, x, r.mean, r.rstd, w, bias=b, stream=torch.cuda.current_stream())
        want = ctx.layer_norm_backward(g, x, r.mean, r.rstd, w)
        assert all(torch.equal(p, q) for p, q in zip(both, want))
        for bad in (b[1:], b.double(), b.cpu()):
            with pytest.raises(binding.QgbdtError):
                ctx.layer_norm_backward(g, x, r.mean, r.rstd, bias=bad)

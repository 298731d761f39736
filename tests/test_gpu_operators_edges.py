"""Operators on top of the trees at the edges of their range: small probabilities in half precision, streams and captured
graphs over the shared work buffer, extreme norms, sizes and strides, autograd's bookkeeping.  Tolerances are derived beside
each check; u(T) = 2^-9 (bf16), 2^-12 (f16) and 2^-24 (f32) is the relative error of one rounding to nearest."""
import ctypes as C
import math
import warnings

import pytest
import torch

pytestmark = pytest.mark.gpu


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


@pytest.mark.parametrize("rows,classes,dim", [(600, 300, 64), (777, 1003, 129), (3000, 5000, 520), (5000, 31000, 1024)])
def test_rare_classes_keep_their_gradients_in_half_precision(ctx, rows, classes, dim):
    """A third of the classes has probabilities near 2e-8 in every row, below the 2^-25 at which a half-precision number
    vanishes; with the loss scale their gradients are ordinary numbers of the outputs' type.  Column 0 of the hidden rows is
    zero, so that the rare classes' weights of 100 there change no logit and fill column 0 of the rows' gradient alone."""
    h = 1.0 + 0.1 * torch.randn((rows, dim), generator=gen(1), device="cuda")
    w = torch.randn((classes, dim), generator=gen(2), device="cuda") * (0.1 / math.sqrt(dim))
    common = classes * 2 // 3
    h[:, 0], w[:, 0], w[common:, 0] = 0.0, 0.0, 100.0
    h, w = h.half(), w.half()
    b = torch.zeros(classes, device="cuda")
    b[common:] = math.log(2e-8 * common)
    y = torch.randint(0, common, (rows,), generator=gen(3), device="cuda")
    r = ctx.softmax_ce(h, w, y, bias=b)
    dh, dw, db = ctx.softmax_ce_backward(h, w, y, r.lse, bias=b, grad_loss=torch.full((1,), 65536.0, device="cuda"))
    z = h.double() @ w.double().t() + b.double()
    p = torch.exp(z - torch.logsumexp(z, 1, keepdim=True))[:, common:] * (65536.0 / rows)
    # all terms of these sums are positive, so that relative errors stay: p and the output are rounded to 2^-12 each; logits
    # and lse behind p are off by dim * 2^-23 * sum |h w| <= 2^-11.5 each (1024 terms of 0.0025); the sums themselves, in chains of a
    # few hundred, by 2^-15: below 2^-9 in all
    for got, want in ((dw[common:], p.t() @ h.double()), (dh[:, 0], p @ w[common:, 0].double()), (db[common:], p.sum(0))):
        assert bool(((got.double() - want).abs() <= 2.0 ** -9 * want.abs()).all())


# ---- streams, captured graphs, the shared work buffer ----------------------------------------------

def loss_case(rows, classes, dim, seed):
    h = torch.randn((rows, dim), generator=gen(seed), device="cuda").bfloat16()
    w = (torch.randn((classes, dim), generator=gen(seed + 1), device="cuda") * 0.2).bfloat16()
    return h, w, torch.randint(0, classes, (rows,), generator=gen(seed + 2), device="cuda")


def captured_context(case):
    """A context over whose work buffer a graph has been captured; the graph (which reads `case`), its outputs, what they
    have to be."""
    from paper_2207_09682_b200 import binding
    c = binding.Context(binding.make_params())
    want = [t.clone() for t in c.softmax_ce(*case)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = c.softmax_ce(*case)
    return c, graph, got, want


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_a_call_that_grows_the_buffer_after_a_capture_waits_for_the_last_call(ctx):
    """Both calls count their blocks in the same words; the graph keeps the buffer that it was captured over."""
    cases = [loss_case(rows, classes, 64, rows) for rows, classes in ((300, 700), (8192, 30000), (8191, 60000))]
    want = [[t.clone() for t in ctx.softmax_ce(*case)] for case in cases]
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for k in range(3):
        c, graph, got, _ = captured_context(cases[0])
        torch.cuda.synchronize()
        first = [c.softmax_ce(*cases[0], stream=a) for _ in range(50)]   # in flight when the next call grows the buffer
        second = c.softmax_ce(*cases[1], stream=b)
        third = c.softmax_ce(*cases[2], stream=a)
        torch.cuda.synchronize()
        assert all(same(r, want[0]) for r in first) and same(second, want[1]) and same(third, want[2])
        graph.replay()
        torch.cuda.synchronize()
        assert same(got, want[0])
        del graph
        c.close()


def test_calls_on_several_streams_of_one_capture_are_ordered(ctx):
    """Forked branches of a graph that use the same work buffer: the later call waits for the earlier one's branch."""
    a, b = loss_case(8192, 30000, 64, 1), loss_case(8000, 20000, 64, 2)
    tok = torch.randint(0, 900, (30000, 4), generator=gen(5), device="cuda")
    grad = torch.randn((30000, 16), generator=gen(6), device="cuda")
    want_a, want_b, want_e = ctx.softmax_ce(*a), ctx.softmax_ce(*b), ctx.embed_backward(grad, tok, 900)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        got_b = ctx.softmax_ce(*b, stream=side)
        got_a = ctx.softmax_ce(*a)
        got_e = ctx.embed_backward(grad, tok, 900, stream=side)
        got_a2 = ctx.softmax_ce(*a)
        main.wait_stream(side)
    for _ in range(5):
        graph.replay()
    torch.cuda.synchronize()
    assert same(got_a, want_a) and same(got_b, want_b) and same([got_e], [want_e]) and same(got_a2, want_a)


def test_several_captures_one_after_another_and_side_by_side(ctx):
    """More captures than a context follows at a time; a call belongs to the capture of its own stream."""
    case = loss_case(700, 900, 64, 7)
    want = [t.clone() for t in ctx.softmax_ce(*case)]
    torch.cuda.synchronize()
    graphs = []
    for _ in range(6):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = ctx.softmax_ce(*case), ctx.softmax_ce(*case)
        graphs.append((graph, got))
    for graph, got in graphs:
        graph.replay()
        torch.cuda.synchronize()
        assert same(got[0], want) and same(got[1], want)
    one, two = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(s):
        one.capture_begin(capture_error_mode="relaxed")
        first = ctx.softmax_ce(*case)
    with torch.cuda.stream(t):
        two.capture_begin(capture_error_mode="relaxed")
        second = ctx.softmax_ce(*case)
    with torch.cuda.stream(s):
        third = ctx.softmax_ce(*case)
        one.capture_end()
    with torch.cuda.stream(t):
        two.capture_end()
    for graph, results in ((one, (first, third)), (two, (second,))):
        graph.replay()
        torch.cuda.synchronize()
        assert all(same(r, want) for r in results)


def test_outgrown_buffers_that_no_graph_was_captured_over_are_freed():
    """Work buffers of 0.5 to 2 GB one after the other, in a context over whose first, small buffer a graph was captured."""
    case = loss_case(300, 700, 64, 3)   # the graph reads it
    c, graph, got, want = captured_context(case)
    weight = torch.zeros((65536, 64), device="cuda").bfloat16()
    torch.cuda.synchronize()
    before = None
    for rows in (1 << 16, 1 << 17, 1 << 18):   # 8 bytes per row and 128 classes
        hidden = torch.zeros((rows, 64), device="cuda").bfloat16()
        c.softmax_ce(hidden, weight, torch.zeros(rows, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
        del hidden
        torch.cuda.empty_cache()
        free = torch.cuda.mem_get_info()[0]
        if before is None:
            before, first = free, 8 * rows * 512
    # the last buffer holds four times the first one's bytes: 3 times more are gone, not 5 (with an eighth on top of each)
    assert before - free < 4 * first * 1.125
    graph.replay()
    torch.cuda.synchronize()
    assert same(got, want)
    del graph
    c.close()


def test_tensors_of_a_call_on_another_stream_are_recorded_there(ctx, monkeypatch):
    """Whatever sequence they come in, and when the call is refused."""
    from paper_2207_09682_b200 import binding
    seen = []
    record = torch.Tensor.record_stream
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: (seen.append(t.data_ptr()), record(t, s))[1])
    grads, out = [[torch.ones(n, device="cuda") for n in (5, 70, 900)] for _ in range(2)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    for of in (list, tuple, iter, lambda x: {i: t for i, t in enumerate(x)}.values(), lambda x: (t.view(-1) for t in x)):
        seen.clear()
        ctx.clip_grad_norm(of(grads), 2.0, out=of(out), stream=stream)
        assert sorted(seen) == sorted(t.data_ptr() for t in grads + out)
    torch.cuda.synchronize()
    norm = math.sqrt(975)
    assert all(bool(((o - 2.0 / norm).abs() <= 2.0 ** -22).all()) for o in out)
    seen.clear()
    with pytest.raises(binding.QgbdtError):
        ctx.embed(grads[0].view(1, 5), torch.zeros(2, device="cuda"), stream=stream)
    assert grads[0].data_ptr() in seen


# ---- clipping --------------------------------------------------------------------------------------

@pytest.mark.parametrize("copies", [1, 40])
@pytest.mark.parametrize("dtype,value", [(torch.float32, 3e38), (torch.bfloat16, 2.0 ** 127), (torch.float32, 1e36), (torch.float32, 1e30)])
def test_clip_factors_below_single_precision(ctx, dtype, value, copies):
    """One launch and two; norms beyond single precision, which are reported as infinity and clipped by all the same."""
    grads = [torch.full((4096,), value, device="cuda").to(dtype)] * copies
    x = float(grads[0][0])
    norm, bound = math.sqrt(4096 * copies) * x, 1.5e-4
    out = [torch.zeros_like(g) for g in grads]
    got = float(ctx.clip_grad_norm(grads, bound, out=out))
    assert got == math.inf if norm > 3.4028235e38 else abs(got - norm) <= 2.0 ** -23 * norm
    want = bound * x / norm
    # the factor in double or single precision, the product, the type: one rounding each
    u = 2.0 ** -9 if dtype == torch.bfloat16 else 2.0 ** -24
    assert all(bool(((o.double() - want).abs() <= (u + 2.0 ** -23) * want).all()) for o in out)
    in_place = [grads[0].clone() for _ in range(copies)]
    ctx.clip_grad_norm(in_place, bound)
    assert same(in_place, out)


# ---- autograd's bookkeeping ------------------------------------------------------------------------

def test_tensors_that_a_call_writes_get_a_new_version(ctx):
    """As with torch's own in-place operations; a tensor that was saved for a backward pass is noticed."""
    tok = torch.zeros(3, dtype=torch.int32, device="cuda")
    h, w, y = loss_case(20, 30, 8, 1)
    lse = ctx.softmax_ce(h, w, y).lse
    calls = [
        lambda t: ctx.embed(torch.randn((8, 4), device="cuda"), tok, out=t[:3, :4]),
        lambda t: ctx.embed_backward(torch.randn((3, 4), device="cuda"), tok, 8, grad_table=t[:8, :4]),
        lambda t: ctx.clip_grad_norm([t], 0.5), lambda t: ctx.clip_grad_norm([torch.ones_like(t)], 0.5, out=[t]),
        lambda t: ctx.embed(torch.randn((8, 4), device="cuda"), tok, out=t[:3, :4], stream=torch.cuda.current_stream()),
    ]
    for call in calls:
        t = torch.ones((30, 8), device="cuda")
        before = t._version
        call(t)
        assert t._version > before
    gh, gw = torch.zeros_like(h), torch.zeros_like(w)
    ctx.softmax_ce_backward(h, w, y, lse, grad_hidden=gh, grad_weight=gw)
    assert gh._version > 0 and gw._version > 0 and h._version == 0 and w._version == 0
    t = torch.ones(30, device="cuda")
    ctx.clip_grad_norm([t], math.inf)                          # the norm alone
    ctx.clip_grad_norm([t], 0.5, out=[torch.empty_like(t)])
    assert t._version == 0
    x, saved = torch.randn((3, 4), device="cuda", requires_grad=True), torch.randn((3, 4), device="cuda")
    product = (x * saved).sum()
    ctx.embed(torch.randn((8, 4), device="cuda"), tok, out=saved)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        product.backward()
    with torch.inference_mode():
        inside = torch.ones(30, device="cuda")
    ctx.clip_grad_norm([inside], 0.5)
    assert float(inside[0]) < 1.0


def test_inputs_that_require_a_gradient_are_taken_with_a_warning(ctx, recwarn):
    tok = torch.zeros(3, dtype=torch.int32, device="cuda")
    h, w, y = loss_case(20, 30, 8, 1)
    r = ctx.softmax_ce(h, w, y)
    leaf = lambda t: t.detach().clone().requires_grad_()  # noqa: E731
    calls = [
        ("table", lambda: ctx.embed(leaf(torch.ones((8, 4), device="cuda")), tok)),
        ("grad_out", lambda: ctx.embed_backward(leaf(torch.ones((3, 4), device="cuda")), tok, 8)),
        ("hidden", lambda: ctx.softmax_ce(leaf(h), w, y)), ("weight", lambda: ctx.softmax_ce(h, leaf(w), y)),
        ("bias", lambda: ctx.softmax_ce(h, w, y, bias=leaf(torch.zeros(30, device="cuda")))),
        ("hidden", lambda: ctx.softmax_ce_backward(leaf(h), w, y, r.lse)),
        ("gradients", lambda: ctx.clip_grad_norm([leaf(torch.ones(4, device="cuda"))], 1.0)),
    ]
    for name, call in calls:
        with pytest.warns(UserWarning, match=name + " requires a gradient, but autograd does not record"):
            result = call()
        first = result if isinstance(result, torch.Tensor) else result[0]
        assert not first.requires_grad
        with torch.no_grad():
            call()
    assert not recwarn.list    # neither without gradients nor under no_grad()
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        with pytest.raises(UserWarning):
            calls[0][1]()
    assert same(ctx.softmax_ce(h, w, y), r)


# ---- sizes and strides -----------------------------------------------------------------------------

def test_columns_beyond_32_bits_are_refused(ctx):
    """Not taken modulo 2^32 (no memory is behind these tensors: they have no rows)."""
    from paper_2207_09682_b200 import binding
    table = torch.randn((8, 4), device="cuda")
    for columns in (2 ** 32 + 1, 2 ** 31, 2 ** 33 + 4):
        tok = torch.empty((0, columns), dtype=torch.int32, device="cuda")
        for call in (lambda: ctx.embed(table, tok), lambda: ctx.embed_backward(table[:0], tok, 8), lambda: ctx.embed_backward(torch.empty((0, columns), device="cuda"), tok[:, :1], 8),
                     lambda: ctx.softmax_ce(torch.empty((0, columns), device="cuda").half(), table.half(), torch.empty(0, dtype=torch.int32, device="cuda"))):
            with pytest.raises(binding.QgbdtError) as e:
                call()
            assert e.value.code == binding.ERR_ARG


def test_strides_of_single_rows_and_rows_far_apart(ctx):
    """C ABI: the stride of a single row means nothing; rows of the weight's gradient more than 2^31 bytes apart; strides that
    no copy takes are refused before anything is written."""
    from paper_2207_09682_b200 import binding
    p = lambda t: C.c_void_p(None if t is None else t.data_ptr())  # noqa: E731
    i64, stream = C.c_int64, C.c_void_p(torch.cuda.current_stream().cuda_stream)

    def loss(h, ldh, w, ldw, y):
        lse, value = torch.zeros(len(h), device="cuda"), torch.zeros(1, device="cuda")
        rc = ctx.lib.qgbdt_softmax_ce(ctx.h, p(h), i64(ldh), p(w), i64(ldw), 2, None, p(y), 0, i64(len(h)), i64(len(w)), h.shape[1], p(value), None, p(lse), None, stream)
        return rc, value, lse

    def grads(h, ldh, w, ldw, y, lse, dh, lddh, dw, lddw):
        return ctx.lib.qgbdt_softmax_ce_backward(ctx.h, p(h), i64(ldh), p(w), i64(ldw), 2, None, p(y), 0, i64(len(h)), i64(len(w)), w.shape[1], p(lse), None,
                                                 p(dh), i64(lddh), p(dw), i64(lddw), None, None, stream)

    far = 1 << 40
    for rows, classes, dim in ((5, 1, 8), (1, 5, 8), (1, 1, 13), (1, 70, 13), (300, 1, 13)):
        h = torch.randn((rows, dim), generator=gen(1), device="cuda").half()
        w = torch.randn((classes, dim), generator=gen(2), device="cuda").half()
        y = torch.zeros(rows, dtype=torch.int32, device="cuda")
        want = ctx.softmax_ce(h, w, y)
        want_dh, want_dw, _ = ctx.softmax_ce_backward(h, w, y, want.lse)
        ldh, ldw = far if rows == 1 else dim, far if classes == 1 else dim
        rc, value, lse = loss(h, ldh, w, ldw, y)
        assert rc == binding.OK and torch.equal(value, want.loss) and torch.equal(lse, want.lse)
        dh, dw = torch.ones_like(h), torch.ones_like(w)
        assert grads(h, ldh, w, ldw, y, lse, dh, ldh, dw, ldw) == binding.OK
        assert torch.equal(dh, want_dh) and torch.equal(dw, want_dw)
        none = torch.empty((0, dim), device="cuda").half()
        assert grads(none, dim, w, ldw, y, lse, none, dim, dw, ldw) == binding.OK and not dw.any()
    h, w, y = torch.ones((2, 8), device="cuda").half(), torch.ones((2, 8), device="cuda").half(), torch.zeros(2, dtype=torch.int32, device="cuda")
    assert loss(h, far, w, 8, y)[0] == binding.ERR_ARG and loss(h, 8, w, far, y)[0] == binding.ERR_ARG
    # no rows: zeros into rows 2^31 bytes apart
    wide = torch.ones((2, 2 ** 30 + 8), dtype=torch.float16, device="cuda")
    _, dw, _ = ctx.softmax_ce_backward(h[:0], w, y[:0], torch.empty(0, device="cuda"), grad_weight=wide[:, :8])
    assert not dw.any() and bool((wide[:, 8:16] == 1).all())
    # the embedding's table, output and gradients of one row
    table, tok, out = torch.randn((1, 7), device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros((1, 7), device="cuda")
    one = C.c_float(1.0)
    assert ctx.lib.qgbdt_embed(ctx.h, p(table), 0, i64(1), 7, i64(far), p(tok), 0, i64(1), 1, i64(far), one, p(out), i64(far), None, stream) == binding.OK
    assert torch.equal(out, table)
    out.zero_()
    assert ctx.lib.qgbdt_embed_backward(ctx.h, p(table), 0, i64(far), p(tok), 0, i64(1), 1, i64(far), one, p(out), i64(1), 7, i64(far), None, stream) == binding.OK
    assert torch.equal(out, table)


def test_tensors_whose_memory_does_not_hold_their_values_are_refused(ctx):
    """Sparse ones (as the gradients of embeddings may be) and those with a pending negation."""
    from paper_2207_09682_b200 import binding
    table, tok = torch.randn((8, 4), device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    negative = torch._neg_view(table)
    for bad in (table.to_sparse(), table.to_sparse_csr(), negative):
        for call in (lambda: ctx.clip_grad_norm([table, bad], 1.0), lambda: ctx.embed(bad, tok), lambda: ctx.embed_backward(bad[:3] if bad is negative else bad, tok, 8),
                     lambda: ctx.embed(table, tok, out=bad)):
            with pytest.raises(binding.QgbdtError) as e:
                call()
            assert e.value.code == binding.ERR_ARG
    want = math.sqrt(float(table.double().square().sum()))
    assert abs(float(ctx.clip_grad_norm([negative.resolve_neg()], math.inf)) - want) <= 2.0 ** -22 * want


# ---- the classifier over leaves --------------------------------------------------------------------

@pytest.mark.parametrize("dtype,scale", [(torch.bfloat16, 1.0), (torch.float16, 256.0)])
def test_a_step_rounds_the_gradients_to_16_bits_once(ctx, dtype, scale):
    """What gradients() gives is clipped and applied in single precision."""
    from paper_2207_09682_b200.leaf_model import LeafClassifier
    net = LeafClassifier(ctx, 6, 9, 70, 20, dtype=dtype, loss_scale=scale, seed=2)
    tokens = torch.randint(0, 9, (300, 6), generator=gen(5), device="cuda") + 9 * torch.arange(6, device="cuda")
    labels = torch.randint(0, 70, (300,), generator=gen(6), device="cuda")
    _, grads = net.gradients(tokens, labels)
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in grads)) / scale
    before = [p.double().clone() for p in (net.table, net.weight, net.bias)]
    net.step(tokens, labels, lr=0.5, max_norm=0.3 * norm)
    for p, q, g in zip((net.table, net.weight, net.bias), before, grads):
        moved = 0.5 * 0.3 * g.double() / scale
        # the factor, its product and the rate's: 2^-24 each, the norm 2^-24; the parameter itself 2^-24
        assert bool(((p.double() - (q - moved)).abs() <= 2.0 ** -24 * (q.abs() + moved.abs()) + 2.0 ** -21 * moved.abs()).all())

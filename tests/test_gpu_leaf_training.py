"""Training steps of the classifier over tree leaves with a layer norm and AdamW: embedding, norm, loss, their gradients,
the gradients' norm and the optimizer together, against the formulas in 64 bits; the same steps from a captured graph."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ctx():
    from paper_2207_09682_b200 import binding
    c = binding.Context(binding.make_params())
    yield c
    c.close()


def batch(rows=300, trees=6, leaves=9, classes=70, seed=5):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    tokens = torch.randint(0, leaves, (rows, trees), generator=gen, device="cuda") + leaves * torch.arange(trees, device="cuda")
    tokens[torch.rand((rows, trees), generator=gen, device="cuda") < 0.05] = -1
    return tokens, torch.randint(-1, classes, (rows,), generator=gen, device="cuda")


def classifier(ctx, dtype, scale, bits, dim=20, **more):
    from paper_2207_09682_b200.leaf_model import LeafClassifier
    net = LeafClassifier(ctx, 6, 9, 70, dim, dtype=dtype, loss_scale=scale, seed=2, layer_norm=True, optimizer="adamw", state_bits=bits, **more)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    net.norm_weight += 0.2 * torch.randn(dim, generator=gen, device="cuda")
    net.norm_bias += 0.2 * torch.randn(dim, generator=gen, device="cuda")
    return net


@pytest.mark.parametrize("dim", [20, 33])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype,scale", [(torch.bfloat16, 1.0), (torch.float16, 256.0)])
def test_step_against_the_formulas(ctx, dtype, scale, bits, dim):
    """Gradients: as a whole (2-norm) within a few roundings to `dtype` (u = eps / 2): the probabilities' differences, d_hidden, the norm's
    gradient and the sum are rounded once each on the way to the table's; the norm of the output rows is rounded in front of the classifier,
    which the formula is given as it was.  The step: a change of a parameter is m / sqrt(v) of its own gradient, lr at most in the first step."""
    net = classifier(ctx, dtype, scale, bits, dim)
    tokens, labels = batch()
    r, grads = net.gradients(tokens, labels)
    assert len(grads) == len(net.parameters()) == 5 and all(g.shape == p.shape for g, p in zip(grads, net.parameters()))
    t, w = net.table16.double().requires_grad_(), net.weight16.double().requires_grad_()
    b, nw, nb = (p.double().requires_grad_() for p in (net.bias, net.norm_weight, net.norm_bias))
    sums = torch.where((tokens >= 0).unsqueeze(2), t[tokens.clamp(min=0)], 0.0).sum(1) * net.scale
    sums = sums + (ctx.embed(net.table16, tokens, scale=net.scale).double() - sums).detach()      # forward values as rounded
    off = sums - sums.mean(1, keepdim=True)
    h = off * ((off * off).mean(1, keepdim=True) + 1e-5).rsqrt() * nw + nb
    h = h + (net.hidden(tokens).double() - h).detach()
    loss = torch.nn.functional.cross_entropy(h @ w.t() + b, labels, ignore_index=-1)
    (loss * scale).backward()
    assert abs(float(r.loss) - float(loss.detach())) <= 1e-5
    u = torch.finfo(dtype).eps / 2
    for got, want in zip(grads, (t.grad, w.grad, b.grad, nw.grad, nb.grad)):
        assert float((got.double() - want).norm()) <= 4 * u * float(want.norm())
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in grads)) / scale
    was = [p.double().clone() for p in net.parameters()]
    step = net.step(tokens, labels, lr=0.01, max_norm=0.25 * norm)
    assert abs(float(step.norm) - norm) <= 1e-5 * norm and int(net.steps) == 1
    for p, q, g in zip(net.parameters(), was, grads):
        g = g.double() * (0.25 / scale)
        # in the first step m / (1 - b1) = g and v / (1 - b2) = g^2, up to 40 roundings of 2^-24; g itself has the clipping's factor (2^-20)
        change = g / (g.abs() + 1e-8)
        slack = 0.01 * 2.0 ** -18 + 2.0 ** -23 * q.abs() + 0.01 * 2.0 ** -18 * change.abs()
        assert bool(((p.double() - (q * (1 - 0.01 * 0.01) - 0.01 * change)).abs() <= slack).all())
    assert torch.equal(net.table16, net.table.to(dtype)) and torch.equal(net.weight16, net.weight.to(dtype))
    m, v, e = net.states
    if bits == 8:
        m, v = ctx.adamw_values(m, v, e)
    for g, a, c in zip(grads, m, v):
        g = g.double() * (0.25 / scale)
        rounding = 1 / 8 if bits == 8 else 2.0 ** -20      # of 8 bits: below one step up or down
        for got, want, floor in ((a, 0.1 * g, 1.25 * 2.0 ** -15), (c, 0.001 * g * g, 1.25 * 2.0 ** -31)):
            assert bool(((got.double() - want).abs() <= rounding * (1 + 1e-5) * want.abs() + (2 * floor * float(want.abs().max()) if bits == 8 else 1e-30)).all())


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_from_a_graph(ctx, bits):
    """A whole step, captured once and replayed, gives the same bits as eager steps."""
    eager, captured = (classifier(ctx, torch.bfloat16, 1.0, bits) for _ in range(2))
    tokens, labels = batch()
    for _ in range(2):      # the work buffer grows before the capture
        eager.step(tokens, labels, 0.01, 1.0)
        captured.step(tokens, labels, 0.01, 1.0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = captured.step(tokens, labels, 0.01, 1.0)
    for _ in range(4):
        graph.replay()
        want = eager.step(tokens, labels, 0.01, 1.0)
        torch.cuda.synchronize()
        assert torch.equal(got.loss, want.loss) and torch.equal(got.norm, want.norm)
    assert int(captured.steps) == 6 and all(torch.equal(p, q) for p, q in zip(captured.parameters(), eager.parameters()))
    assert all(torch.equal(p, q) for a, b in zip(captured.states, eager.states) if a is not None for p, q in zip(a, b))
    del graph


@pytest.mark.parametrize("bits", [32, 8])
def test_overflow_leaves_parameters_and_states(ctx, bits):
    net = classifier(ctx, torch.float16, 2.0 ** 40, bits)
    was = [p.clone() for p in net.parameters()]
    step = net.step(*batch(), lr=0.1, max_norm=1.0)
    assert not math.isfinite(float(step.norm)) and int(net.steps) == 0
    assert all(torch.equal(p, q) for p, q in zip(net.parameters(), was)) and not any(bool(t.any()) for l in net.states if l is not None for t in l)


def test_layer_norm_with_gradient_descent(ctx):
    from paper_2207_09682_b200.leaf_model import LeafClassifier
    net = LeafClassifier(ctx, 6, 9, 70, 24, layer_norm=True)
    tokens, labels = batch()
    _, grads = net.gradients(tokens, labels)
    was = [p.double().clone() for p in net.parameters()]
    net.step(tokens, labels, lr=0.5)
    for p, q, g in zip(net.parameters(), was, grads):
        assert bool(((p.double() - (q - 0.5 * g.double())).abs() <= 2.0 ** -23 * (q.abs() + g.abs())).all())
    with pytest.raises(ValueError):
        LeafClassifier(ctx, 6, 9, 70, 24, optimizer="adam")


@pytest.mark.parametrize("more", [["--layer-norm", "--optimizer", "adamw", "--state-bits", "8"], ["--optimizer", "adamw"], ["--layer-norm"]])
def test_example_runs(more):
    spec = importlib.util.spec_from_file_location("leaf_classifier", os.path.join(ROOT, "examples", "leaf_classifier.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, right, most = example.main(["--rows", "5000", "--classes", "20", "--dim", "32", "--epochs", "2", *more])
    assert len(losses) == 2 and all(math.isfinite(x) for x in losses) and 0.0 <= right <= 1.0

"""The classifier over tree leaves: tokens against a walk through the trees on the CPU, a step's gradients against the
formula in 64 bits, training end to end."""
import importlib.util
import math
import os

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def trained(rows, trees):
    from paper_2207_09682_b200 import binding, synth
    wl = synth.tiny(device="cuda", rows=rows)
    ctx = binding.Context(binding.make_params(**wl.params))
    ctx.load_binned(wl.bins, wl.n_bins)
    model = ctx.train(wl.labels, torch.zeros(rows, device="cuda"), 0, trees)
    return wl, ctx, model


def test_leaf_tokens_against_a_walk():
    from paper_2207_09682_b200.leaf_model import leaf_tokens
    wl, ctx, model = trained(3000, 3)
    tokens = leaf_tokens(ctx, model).cpu().numpy()
    data = wl.bins.cpu().numpy()
    for k in range(3):
        t = model.tree(k)
        for i in range(0, 3000, 7):
            node = 0
            while node >= 0:
                left = data[i, t["feature"][node]] <= t["bin"][node]
                node = int(t["left"][node] if left else t["right"][node])
            assert tokens[i, k] == k * model.L + ~node
        assert (np.bincount(tokens[:, k] - k * model.L, minlength=t["num_leaves"]) == t["leaf_count"]).all()


@pytest.mark.parametrize("dtype,scale", [(torch.bfloat16, 1.0), (torch.float16, 256.0)])
def test_step_against_the_formula(dtype, scale):
    """Table gradient through the embedding: each of its terms is a row of d_hidden, which is rounded to `dtype` once (relative
    2^-8 or 2^-11), as is the sum; d_hidden itself is off by the rounding of the probabilities' differences (the same again)."""
    from paper_2207_09682_b200 import binding
    from paper_2207_09682_b200.leaf_model import LeafClassifier
    ctx = binding.Context(binding.make_params())
    net = LeafClassifier(ctx, 6, 9, 70, 20, dtype=dtype, loss_scale=scale, seed=2)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    tokens = torch.randint(0, 9, (300, 6), generator=gen, device="cuda") + 9 * torch.arange(6, device="cuda")
    labels = torch.randint(-1, 70, (300,), generator=gen, device="cuda")
    r, (dt, dw, db) = net.gradients(tokens, labels)
    t, w = net.table16.double().requires_grad_(), net.weight16.double().requires_grad_()
    b = net.bias.double().requires_grad_()
    h = t[tokens].sum(1) * net.scale
    h = h + (net.hidden(tokens).double() - h).detach()     # the forward value as rounded
    loss = torch.nn.functional.cross_entropy(h @ w.t() + b, labels, ignore_index=-1)
    (loss * scale).backward()
    assert abs(float(r.loss) - float(loss)) <= 1e-5
    u = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -11
    for got, want in ((dt, t.grad), (dw, w.grad), (db, b.grad)):
        assert float((got.double() - want).norm()) <= 3 * u * float(want.norm())
    before = [p.clone() for p in (net.table, net.weight, net.bias)]
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in (dt, dw, db))) / scale
    step = net.step(tokens, labels, lr=0.5, max_norm=0.25 * norm)
    assert abs(float(step.norm) - norm) <= 1e-5 * norm
    moved = math.sqrt(sum(float((p - q).double().square().sum()) for p, q in zip((net.table, net.weight, net.bias), before)))
    assert abs(moved - 0.5 * 0.25 * norm) <= 2 * u * moved


def test_overflow_leaves_the_parameters():
    from paper_2207_09682_b200 import binding
    from paper_2207_09682_b200.leaf_model import LeafClassifier
    ctx = binding.Context(binding.make_params())
    net = LeafClassifier(ctx, 2, 4, 10, 8, dtype=torch.float16, loss_scale=2.0 ** 40)
    before = [p.clone() for p in (net.table, net.weight, net.bias)]
    step = net.step(torch.tensor([[0, 5], [1, 6]], device="cuda"), torch.tensor([3, 4], device="cuda"), lr=0.1, max_norm=1.0)
    assert not math.isfinite(float(step.norm))
    assert all(torch.equal(p, q) for p, q in zip((net.table, net.weight, net.bias), before))


def test_example_learns():
    spec = importlib.util.spec_from_file_location("leaf_classifier", os.path.join(ROOT, "examples", "leaf_classifier.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, right, most = example.main(["--rows", "20000", "--classes", "50", "--dim", "32", "--epochs", "3"])
    assert losses[-1] < losses[0] < math.log(50) and right > 1.5 * most

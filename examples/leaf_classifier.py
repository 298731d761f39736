"""Boosted trees as features of a classifier with many classes.

Trains trees on a synthetic binary task, sends the rows through them, and trains a softmax classifier over
their leaves to tell one of --classes classes that depend on the same features.

    python examples/leaf_classifier.py [--rows 50000] [--classes 500] [--dim 64] [--epochs 5]
                                       [--layer-norm] [--optimizer adamw [--state-bits 8]]
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2207_09682_b200 import binding, synth  # noqa: E402
from paper_2207_09682_b200.leaf_model import LeafClassifier, leaf_tokens  # noqa: E402


def classes_of(bins: torch.Tensor, n_bins: int, classes: int, seed: int = 3) -> torch.Tensor:
    """A class per row: the nearest of `classes` points in the space of four of the features."""
    gen = torch.Generator(device=bins.device)
    gen.manual_seed(seed)
    x = bins[:, :4].float() / n_bins
    return torch.cdist(x, torch.rand((classes, 4), generator=gen, device=bins.device)).argmin(1).int()


def main(argv=None) -> tuple:
    ap = argparse.ArgumentParser(description=__doc__)
    ap.add_argument("--rows", type=int, default=50_000)
    ap.add_argument("--classes", type=int, default=500)
    ap.add_argument("--dim", type=int, default=64)
    ap.add_argument("--epochs", type=int, default=5)
    ap.add_argument("--batch", type=int, default=1024)
    ap.add_argument("--lr", type=float, default=None, help="4 for sgd, 0.01 for adamw")
    ap.add_argument("--layer-norm", action="store_true", help="normalise the sums of embeddings")
    ap.add_argument("--optimizer", choices=["sgd", "adamw"], default="sgd")
    ap.add_argument("--state-bits", type=int, choices=[8, 32], default=32, help="of AdamW's states")
    a = ap.parse_args(argv)
    lr = a.lr if a.lr is not None else 4.0 if a.optimizer == "sgd" else 0.01
    wl = synth.tiny(device="cuda", rows=a.rows)
    ctx = binding.Context(binding.make_params(**wl.params))
    ctx.load_binned(wl.bins, wl.n_bins)
    trees = wl.params["num_trees"]
    model = ctx.train(wl.labels, torch.zeros(a.rows, device="cuda"), 0, trees)
    tokens, labels = leaf_tokens(ctx, model), classes_of(wl.bins, wl.n_bins, a.classes)
    net = LeafClassifier(ctx, trees, model.L, a.classes, a.dim, layer_norm=a.layer_norm, optimizer=a.optimizer, state_bits=a.state_bits)
    losses = []
    for epoch in range(a.epochs):
        order = torch.randperm(a.rows, device="cuda")
        for at in order.split(a.batch):
            step = net.step(tokens[at], labels[at], lr, max_norm=1.0)
        losses.append(float(net.loss(tokens, labels).loss))
        print("epoch %d: loss %.4f, gradient norm of the last batch %.3f" % (epoch, losses[-1], float(step.norm)))
    right = float((net.predict(tokens) == labels).float().mean())
    most = float(torch.bincount(labels).max()) / a.rows
    print("right on %.1f %% of the rows (always naming the most frequent class: %.1f %%)" % (100 * right, 100 * most))
    return losses, right, most


if __name__ == "__main__":
    main()

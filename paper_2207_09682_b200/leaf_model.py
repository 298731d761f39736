"""Softmax classifier over the leaves of boosted trees.

The leaves that a row reaches in the trees of a trained model are learned categorical features of it: leaf l of
tree k is entry k * num_leaves + l of an embedding table, a row is the scaled sum of its leaves' embeddings, and
a linear layer with softmax cross entropy tells its class.  One table serves any number of classes, where
boosting itself would grow a tree per class.  The operators are the calls of include/qgbdt.h; this module keeps
the parameters and strings the calls of a training step together.
"""
from __future__ import annotations

import math
from typing import NamedTuple

import torch

from . import binding


def leaf_tokens(ctx: binding.Context, model: binding.HostModel, stream=None) -> torch.Tensor:
    """Tokens [N, trees] (int32, CUDA) of the rows loaded in `ctx`: entry k * num_leaves + leaf of tree k.

    The rows are sent through the trees by the row partition (the splits of a tree are replayed in the order in
    which they were made, which gives its leaves the numbers the model has); leaves the context at the root."""
    L = model.L
    if ctx.params.num_leaves < L:
        raise ValueError("the context allows %d leaves, the model has up to %d" % (ctx.params.num_leaves, L))
    tokens = torch.empty((ctx.n_rows, model.num_trees), dtype=torch.int32)
    for k in range(model.num_trees):
        tree = model.tree(k)
        ctx.reset_leaves(stream)
        leaf_of = {0: 0}   # leaf that node i splits: its left child keeps the number, the right child gets i + 1
        for i in range(tree["num_leaves"] - 1):
            leaf = leaf_of[i]
            right, _, _ = ctx.split_leaf(leaf, int(tree["feature"][i]), int(tree["bin"][i]), stream)
            for child, number in ((int(tree["left"][i]), leaf), (int(tree["right"][i]), right)):
                if child >= 0:
                    leaf_of[child] = number
        for leaf in range(tree["num_leaves"]):
            tokens[ctx.get_leaf_rows(leaf), k] = k * L + leaf
    ctx.reset_leaves(stream)
    return tokens.cuda()


class Step(NamedTuple):
    loss: torch.Tensor    # [1], mean over the labelled rows
    norm: torch.Tensor    # [1], of the gradients before clipping


class LeafClassifier:
    """Embedding table [trees * num_leaves, dim], weight [classes, dim], bias [classes]; trained by gradient descent
    with the gradients clipped to a global norm.  Parameters are kept in float32; the embedding and the products
    run on copies of type `dtype` (bfloat16 or float16, the latter with a loss scale)."""

    def __init__(self, ctx: binding.Context, n_trees: int, num_leaves: int, n_classes: int, dim: int, dtype=torch.bfloat16,
                 loss_scale: float = 1.0, seed: int = 0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.ctx, self.dtype, self.loss_scale = ctx, dtype, loss_scale
        self.scale = 1.0 / math.sqrt(n_trees)
        self.table = torch.randn((n_trees * num_leaves, dim), generator=gen, device="cuda")
        self.weight = torch.randn((n_classes, dim), generator=gen, device="cuda") / math.sqrt(dim)
        self.bias = torch.zeros(n_classes, device="cuda")
        self._copies()
        self._grad_loss = torch.full((1,), loss_scale, device="cuda")

    def _copies(self):
        self.table16, self.weight16 = self.table.to(self.dtype), self.weight.to(self.dtype)

    def hidden(self, tokens: torch.Tensor) -> torch.Tensor:
        return self.ctx.embed(self.table16, tokens, scale=self.scale)

    def loss(self, tokens: torch.Tensor, labels: torch.Tensor) -> binding.SoftmaxCE:
        """Losses of rows against their labels (negative: no label)."""
        return self.ctx.softmax_ce(self.hidden(tokens), self.weight16, labels, bias=self.bias)

    def gradients(self, tokens: torch.Tensor, labels: torch.Tensor) -> tuple:
        """(outputs of the forward call, gradients of the table, the weight and the bias, times the loss scale)."""
        c, h = self.ctx, self.hidden(tokens)
        r = c.softmax_ce(h, self.weight16, labels, bias=self.bias)
        dh, dw, db = c.softmax_ce_backward(h, self.weight16, labels, r.lse, bias=self.bias, grad_loss=self._grad_loss)
        return r, [c.embed_backward(dh, tokens, self.table.shape[0], scale=self.scale), dw, db]

    def step(self, tokens: torch.Tensor, labels: torch.Tensor, lr: float, max_norm: float = math.inf) -> Step:
        """One step of gradient descent on a batch.  A norm that is not finite (an overflow of float16) leaves the
        parameters as they are."""
        r, grads = self.gradients(tokens, labels)
        grads = [g.float() for g in grads]   # clipped as the parameters are kept: `dtype` has rounded them once, that is enough
        norm = self.ctx.clip_grad_norm(grads, max_norm * self.loss_scale)
        finite = torch.isfinite(norm)
        for p, g in zip((self.table, self.weight, self.bias), grads):
            p.sub_(torch.where(finite, g * (lr / self.loss_scale), 0.0))
        self._copies()
        return Step(r.loss, norm / self.loss_scale)

    def predict(self, tokens: torch.Tensor, rows: int = 8192) -> torch.Tensor:
        """Most probable class of every row."""
        return torch.cat([(self.hidden(t).float() @ self.weight16.float().t() + self.bias).argmax(1) for t in tokens.split(rows)])

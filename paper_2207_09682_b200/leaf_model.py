"""Softmax classifier over the leaves of boosted trees.

The leaves that a row reaches in the trees of a trained model are learned categorical features of it: leaf l of
tree k is entry k * num_leaves + l of an embedding table, a row is the scaled sum of its leaves' embeddings, and
a linear layer with softmax cross entropy tells its class; a layer norm may stand between them.  One table serves any number of classes, where
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
    """Embedding table [trees * num_leaves, dim], weight [classes, dim], bias [classes], and with `layer_norm` the norm's weight and
    bias [dim]; trained by gradient descent ("sgd") or by AdamW ("adamw", states in 32 or 8 bits, the same decay for all
    parameters) with the gradients clipped to a global norm.  Parameters are kept in float32; the embedding and the products run on copies of type `dtype` (bfloat16 or
    float16, the latter with a loss scale)."""

    def __init__(self, ctx: binding.Context, n_trees: int, num_leaves: int, n_classes: int, dim: int, dtype=torch.bfloat16,
                 loss_scale: float = 1.0, seed: int = 0, layer_norm: bool = False, optimizer: str = "sgd", state_bits: int = 32,
                 betas: tuple = (0.9, 0.999), weight_decay: float = 0.01):
        if optimizer not in ("sgd", "adamw"):
            raise ValueError("optimizer must be 'sgd' or 'adamw'")
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.ctx, self.dtype, self.loss_scale = ctx, dtype, loss_scale
        self.scale = 1.0 / math.sqrt(n_trees)
        self.table = torch.randn((n_trees * num_leaves, dim), generator=gen, device="cuda")
        self.weight = torch.randn((n_classes, dim), generator=gen, device="cuda") / math.sqrt(dim)
        self.bias = torch.zeros(n_classes, device="cuda")
        self.norm_weight = torch.ones(dim, device="cuda") if layer_norm else None
        self.norm_bias = torch.zeros(dim, device="cuda") if layer_norm else None
        self._copies()
        self._grad_loss = torch.full((1,), loss_scale, device="cuda")
        self.optimizer, self.betas, self.weight_decay, self.seed = optimizer, betas, weight_decay, seed
        if optimizer == "adamw":
            self.states = binding.adamw_states(self.parameters(), state_bits)
            self.steps = torch.zeros(1, dtype=torch.int64, device="cuda")   # those that were taken

    def parameters(self) -> list:
        """In the order of gradients()."""
        return [p for p in (self.table, self.weight, self.bias, self.norm_weight, self.norm_bias) if p is not None]

    def _copies(self):
        self.table16, self.weight16 = self.table.to(self.dtype), self.weight.to(self.dtype)

    def hidden(self, tokens: torch.Tensor) -> torch.Tensor:
        """What the classes are told from: the scaled sums of embeddings, normalised if the model has a layer norm."""
        h = self.ctx.embed(self.table16, tokens, scale=self.scale)
        return h if self.norm_weight is None else self.ctx.layer_norm(h, self.norm_weight, self.norm_bias, out=h).out

    def loss(self, tokens: torch.Tensor, labels: torch.Tensor) -> binding.SoftmaxCE:
        """Losses of rows against their labels (negative: no label)."""
        return self.ctx.softmax_ce(self.hidden(tokens), self.weight16, labels, bias=self.bias)

    def gradients(self, tokens: torch.Tensor, labels: torch.Tensor) -> tuple:
        """(outputs of the forward call, gradients of parameters(), times the loss scale)."""
        c, sums = self.ctx, self.ctx.embed(self.table16, tokens, scale=self.scale)
        h, norm, of_norm = sums, None, []
        if self.norm_weight is not None:
            norm = c.layer_norm(sums, self.norm_weight, self.norm_bias)
            h = norm.out
        r = c.softmax_ce(h, self.weight16, labels, bias=self.bias)
        dh, dw, db = c.softmax_ce_backward(h, self.weight16, labels, r.lse, bias=self.bias, grad_loss=self._grad_loss)
        if norm is not None:
            dh, *of_norm = c.layer_norm_backward(dh, sums, norm.mean, norm.rstd, self.norm_weight, grad_x=dh)
        return r, [c.embed_backward(dh, tokens, self.table.shape[0], scale=self.scale), dw, db, *of_norm]

    def step(self, tokens: torch.Tensor, labels: torch.Tensor, lr: float, max_norm: float = math.inf) -> Step:
        """One step on a batch.  A norm that is not finite (an overflow of float16) leaves the parameters as they are."""
        r, grads = self.gradients(tokens, labels)
        if self.optimizer == "adamw":
            # the factor of the clipping is applied by the step itself, in single precision
            norm = self.ctx.clip_grad_norm(grads, math.inf)
            self.steps += torch.isfinite(norm)
            m, v, exponents = self.states
            self.ctx.adamw(self.parameters(), grads, m, v, self.steps, lr, betas=self.betas, weight_decay=self.weight_decay, exponents=exponents,
                           copies=[self.table16, self.weight16] + [None] * (len(grads) - 2), norm=norm, max_norm=max_norm, loss_scale=self.loss_scale, seed=self.seed)
            return Step(r.loss, norm / self.loss_scale)
        grads = [g.float() for g in grads]   # clipped as the parameters are kept: `dtype` has rounded them once, that is enough
        norm = self.ctx.clip_grad_norm(grads, max_norm * self.loss_scale)
        finite = torch.isfinite(norm)
        for p, g in zip(self.parameters(), grads):
            p.sub_(torch.where(finite, g * (lr / self.loss_scale), 0.0))
        self._copies()
        return Step(r.loss, norm / self.loss_scale)

    def predict(self, tokens: torch.Tensor, rows: int = 8192) -> torch.Tensor:
        """Most probable class of every row."""
        return torch.cat([(self.hidden(t).float() @ self.weight16.float().t() + self.bias).argmax(1) for t in tokens.split(rows)])

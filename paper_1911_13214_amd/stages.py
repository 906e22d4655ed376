"""Stages of a language-model chain for the sequence executor: autograd
functions and modules around ``ops``.

A stage that runs again under a schedule has to compute what it computed the
first time, and what it keeps for its backward (w_abar) is what the schedule
budgets.  So the dropout here draws its mask from (seed, step) and keeps
nothing, the residual seam keeps its block's output, its sum and 16 bytes a
row, the loss keeps 4 bytes a token and no logits, and every gradient is the
same bit for bit on every call.  Inputs of any layout are taken, as in
``linear_cross_entropy(x[:, :-1], w, tokens[:, 1:])``: those that the operators
refuse are copied (and the copy is what is kept).  Second derivatives exist for the dropout
alone; the others raise where one is taken.

``language_chain`` builds a chain of them: token lookup, residual blocks and
the loss over the vocabulary, ready for ``executor.run_sequence``."""
from __future__ import annotations

import functools
import math

import torch
from torch import nn

from . import ops


def _rows(t):
    """A tensor as the operators take matrices: an input that is a slice of
    several dimensions or transposed is copied, and a gradient that autograd
    hands on so or broadcast."""
    if t is None or t.is_contiguous():
        return t
    try:
        ops._matrix(t, "t")
    except ValueError:
        return t.contiguous()
    return t


class _Refuse(torch.autograd.Function):
    """Passes first derivatives on; raises where one is differentiated."""

    @staticmethod
    def forward(ctx, *grads):
        return tuple(None if g is None else g.view_as(g) for g in grads)

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("the kernels compute first derivatives only: a derivative of one has been asked for")


def _first_order(backward):
    """A backward whose results come from kernels, without a graph.  Under
    create_graph they depend on what the forward kept as well as on the
    gradients that arrive, so they are marked whether or not those require one:
    a second derivative through them raises instead of leaving its terms out."""
    @functools.wraps(backward)
    def run(ctx, *grads):
        with torch.no_grad():
            out = backward(ctx, *grads)
        if not torch.is_grad_enabled():
            return out
        return _Refuse.apply(*(None if g is None else g.detach().requires_grad_() for g in out))
    return run


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, p, seed, step, step_tensor):
        ctx.draw = (p, seed, step)
        # saved, so that autograd notices a step that was advanced in between
        ctx.save_for_backward(step_tensor)
        return ops.dropout(_rows(x), p, seed, step, _rows(residual), step_tensor=step_tensor)

    @staticmethod
    def backward(ctx, dy):
        dx = None
        if ctx.needs_input_grad[0]:
            # linear: the gradient is a dropout itself, with a gradient of its own
            dx = _Dropout.apply(_rows(dy), None, *ctx.draw, *ctx.saved_tensors)
        return dx, dy if ctx.needs_input_grad[1] else None, None, None, None, None


def dropout(x, p, seed, step=0, residual=None, step_tensor=None):
    """ops.dropout with a gradient; nothing is kept between the two.
    ``step_tensor`` must still hold the forward's value in the backward, which
    raises otherwise."""
    return _Dropout.apply(x, residual, p, seed, step, step_tensor)


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, tokens, table, scale, padding):
        tokens = tokens.contiguous()
        ctx.save_for_backward(tokens)
        ctx.how = (table.shape[0], scale, padding)
        return ops.embedding(tokens, _rows(table), scale)

    @staticmethod
    @_first_order
    def backward(ctx, dy):
        rows, scale, padding = ctx.how
        return None, ops.embedding_backward(ctx.saved_tensors[0], _rows(dy), rows, scale, padding=padding), None, None


def embedding(tokens, table, scale=1.0, padding=None):
    """ops.embedding with the table's gradient (0 for the token ``padding``)."""
    return _Embedding.apply(tokens, table, scale, padding)


_PARAMS = ("post_weight", "post_bias", "gate", "pre_weight", "pre_bias")


class _ResidualNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, z, post, pre, residual_scale, eps, *params):
        x, z = _rows(x), _rows(z)
        params = [_rows(q) if name == "gate" or q is None else q.contiguous() for name, q in zip(_PARAMS, params)]
        ctx.how = dict(post=post, pre=pre, residual_scale=residual_scale, eps=eps)
        y, h, stats = ops.residual_norm(x, z, **ctx.how, **dict(zip(_PARAMS, params)))
        # without a block y is x itself: only h is a result
        alone = y is x
        ctx.alone = alone
        ctx.save_for_backward(y if h is not None else None, z, stats, *params)
        ctx.set_materialize_grads(False)
        return h if alone else (y, h)

    @staticmethod
    @_first_order
    def backward(ctx, *grads):
        dy, dh = (None if g is None else _rows(g) for g in ((None, grads[0]) if ctx.alone else grads))
        y, z, stats, *params = ctx.saved_tensors
        how = dict(zip(_PARAMS, params))
        if dh is None and ctx.how["pre"] != "none":
            if dy is None:
                return (None,) * (6 + len(_PARAMS))
            dh = torch.zeros_like(dy)
        g = ops.residual_norm_backward(dy, dh, y, z, stats, **ctx.how, **how)
        return (g["x"], g.get("z"), None, None, None, None, *(g.get(k) for k in _PARAMS))


def residual_norm(x, z=None, *, post="none", post_weight=None, post_bias=None, gate=None, residual_scale=1.0,
                  pre="none", pre_weight=None, pre_bias=None, eps=1e-5):
    """ops.residual_norm with gradients: (y, h), h None without ``pre``."""
    out = _ResidualNorm.apply(x, z, post, pre, residual_scale, eps, post_weight, post_bias, gate, pre_weight, pre_bias)
    return out if isinstance(out, tuple) else (x, out)


class _CrossEntropy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, h, w, targets, ignore):
        h, w = _rows(h), _rows(w)
        targets = (targets.long() if targets.dtype == torch.int32 else targets).contiguous()
        loss, lse = ops.linear_cross_entropy(h, w, targets, ignore)
        ctx.save_for_backward(h, w, targets, lse)
        ctx.ignore = ignore
        return loss

    @staticmethod
    @_first_order
    def backward(ctx, grad_loss):
        h, w, targets, lse = ctx.saved_tensors
        return (*ops.linear_cross_entropy_backward(h, w, targets, lse, grad_loss.contiguous(), ctx.ignore,
                                                   need_h=ctx.needs_input_grad[0], need_w=ctx.needs_input_grad[1]),
                None, None)


def linear_cross_entropy(h, w, targets, ignore=-100):
    """ops.linear_cross_entropy with gradients: the loss of each token.
    ``targets`` may be int32 as well."""
    return _CrossEntropy.apply(h, w, targets, ignore)


# ---- modules -----------------------------------------------------------------------

class Dropout(nn.Module):
    """Dropout that is the same whenever its stage runs again in a step: the
    mask follows from ``seed`` (one for each place in the model) and ``step``,
    which the training loop sets (``set_step``)."""

    def __init__(self, p, seed):
        super().__init__()
        self.p, self.seed, self.step = p, seed, 0

    def forward(self, x, residual=None):
        if not self.training or self.p == 0.0:
            return x if residual is None else residual + x
        return dropout(x, self.p, self.seed, self.step, residual)

    def extra_repr(self):
        return f"p={self.p}, seed={self.seed}"


def set_step(stages, step):
    """Sets the step of every Dropout in a list of stages."""
    for s in stages:
        for mod in s.modules():
            if isinstance(mod, Dropout):
                mod.step = step


class Embedding(nn.Module):
    """Rows of a table by token, times ``scale``."""

    def __init__(self, rows, width, scale=1.0, padding=None):
        super().__init__()
        self.weight = nn.Parameter(torch.randn(rows, width) / math.sqrt(width))
        self.scale, self.padding = scale, padding

    def forward(self, tokens):
        return embedding(tokens, self.weight, self.scale, self.padding)


class Seam(nn.Module):
    """What lies between a block and the next: (x, z) -> (y, h) with
    y = residual_scale * x + gate * post(z) and h = pre(y); the gate is one
    learned factor per channel."""

    def __init__(self, width, post="rms", pre="rms", gate=True, residual_scale=1.0, eps=1e-5):
        super().__init__()
        self.kinds = dict(post=post, pre=pre, residual_scale=residual_scale, eps=eps)

        def ones(on):
            return nn.Parameter(torch.ones(width)) if on else None

        def zeros(on):
            return nn.Parameter(torch.zeros(width)) if on else None

        self.post_weight, self.post_bias = ones(post != "none"), zeros(post == "layer")
        self.pre_weight, self.pre_bias = ones(pre != "none"), zeros(pre == "layer")
        self.gate = ones(gate)

    def forward(self, x, z=None):
        return residual_norm(x, z, **self.kinds, post_weight=self.post_weight, post_bias=self.post_bias,
                             gate=self.gate, pre_weight=self.pre_weight, pre_bias=self.pre_bias)


class Block(nn.Module):
    """A stage: two residual branches (Linear, GELU, Linear, dropout) with the
    seams before, between and after them."""

    def __init__(self, width, inner, p, seed, residual_scale=1.0):
        super().__init__()
        self.enter = Seam(width, post="none", gate=False)
        self.between = Seam(width, residual_scale=residual_scale)
        self.leave = Seam(width, pre="none", residual_scale=residual_scale)
        self.first, self.second = (nn.Sequential(nn.Linear(width, inner), nn.GELU(), nn.Linear(inner, width))
                                   for _ in range(2))
        self.drops = nn.ModuleList(Dropout(p, 2 * seed + k) for k in range(2))

    def forward(self, x):
        _, h = self.enter(x)
        y, h = self.between(x, self.drops[0](self.first(h)))
        return self.leave(y, self.drops[1](self.second(h)))[0]


class Loss(nn.Module):
    """The last stage: a norm, the projection onto the vocabulary and the mean
    cross entropy over the tokens that have a target.  The targets are the
    stage's own, set before a step."""

    def __init__(self, rows, width, ignore=-100):
        super().__init__()
        self.enter = Seam(width, post="none", gate=False)
        self.weight = nn.Parameter(torch.randn(rows, width) / math.sqrt(width))
        self.ignore, self.targets = ignore, None

    def forward(self, x):
        _, h = self.enter(x)
        loss = linear_cross_entropy(h, self.weight, self.targets, self.ignore)
        return loss.sum() / (self.targets != self.ignore).sum().clamp(min=1)


def language_chain(blocks, seed, rows=32000, width=1024, p=0.1, device="cuda", dtype=torch.bfloat16):
    """Stages of a chain: token lookup, ``blocks`` residual blocks whose inner
    widths are drawn from {width, 2 width, 4 width}, the loss.  Seeded
    weights."""
    from . import chaingen

    rng = chaingen.SplitMix64(seed)
    with torch.random.fork_rng(devices=[]):
        torch.manual_seed(seed)
        stages = [Embedding(rows, width, scale=math.sqrt(width))]
        stages += [Block(width, width << rng.uniform(0, 2), p, seed * 1000 + k) for k in range(blocks)]
        stages.append(Loss(rows, width))
    return [s.to(device=device, dtype=dtype) for s in stages]

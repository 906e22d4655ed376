"""Autograd around the operators, without a GPU: the kernels' calls are
replaced by the 64-bit implementations of ops_model.py."""
import pytest
import torch

import ops_model as m
from paper_1911_13214_amd import stages as lm


@pytest.fixture
def model_ops(monkeypatch):
    """ops' functions in stages, computed on the CPU without a graph, as the
    kernels' results are."""
    def residual_norm(x, z=None, **how):
        params = {k: how.get(k) for k in ("post_weight", "post_bias", "gate", "pre_weight", "pre_bias")}
        kinds = {k: how[k] for k in ("post", "pre", "residual_scale", "eps")}
        y, h = m.residual_norm(x, z, **kinds, **params)
        return (x if z is None and how["residual_scale"] == 1.0 else y), h, torch.zeros(x.shape[0], 4)

    def residual_norm_backward(dy, dh, y, z, stats, **how):
        lead = dy if dy is not None else dh
        g = {"x": lead * how["residual_scale"]}
        if z is not None:
            g["z"] = lead.clone()
        return {**g, **{k: torch.zeros_like(v) for k, v in how.items() if torch.is_tensor(v)}}

    def dropout(x, p, seed, step=0, residual=None, step_tensor=None):
        return m.dropout(x, p, seed, step + (0 if step_tensor is None else int(step_tensor)), residual)

    def xent_backward(h, w, targets, lse, grad_loss, ignore, need_h, need_w):
        p = m.cross_entropy_grad(h, w, targets, grad_loss, ignore)
        return (p @ w.double() if need_h else None), (p.t() @ h.double() if need_w else None)

    stand_in = dict(
        dropout=dropout, embedding=m.embedding,
        embedding_backward=lambda tokens, grad, rows, scale, padding: m.embedding_grad(tokens, grad, rows, scale,
                                                                                       padding)[0],
        residual_norm=residual_norm, residual_norm_backward=residual_norm_backward,
        linear_cross_entropy=m.cross_entropy, linear_cross_entropy_backward=xent_backward)
    for name, f in stand_in.items():
        monkeypatch.setattr(lm.ops, name, torch.no_grad()(f))


def leaf(*shape, seed=0):
    return m.normal(torch.Generator().manual_seed(seed + shape[0]), *shape).requires_grad_()


CALLS = {
    "dropout": lambda x, w, t: lm.dropout(x, 0.3, 7, 2),
    "embedding": lambda x, w, t: lm.embedding(t, x, 2.0),
    "residual_norm": lambda x, w, t: lm.residual_norm(x, 2 * x, post="rms", pre="layer")[1],
    "residual_norm_alone": lambda x, w, t: lm.residual_norm(x, pre="rms")[1],
    "linear_cross_entropy": lambda x, w, t: lm.linear_cross_entropy(x, w, t),
}


@pytest.mark.parametrize("name", [k for k in CALLS if k != "dropout"])
@pytest.mark.parametrize("outer", ["sum", "square"])
def test_second_derivatives_are_refused(model_ops, name, outer):
    # Their terms would be left out without a word.  Also where the gradient
    # that arrives is a constant (a sum's): the first derivative still depends
    # on what the forward kept.
    x, w, t = leaf(6, 8), leaf(9, 8), torch.arange(6)
    value = (lambda y: y.sum()) if outer == "sum" else (lambda y: y.square().sum())
    first, = torch.autograd.grad(value(CALLS[name](x, w, t)), x, create_graph=True)
    assert torch.equal(first.detach(), torch.autograd.grad(value(CALLS[name](x, w, t)), x)[0])
    with pytest.raises(RuntimeError, match="first derivatives only"):
        (first.square().sum() + x.square().sum()).backward()


def test_second_derivatives_of_dropout(model_ops):
    # y = s k x with a mask k, s = 1 / (1 - q): the gradient of sum(y^2) is
    # 2 s^2 k x and that of its square's sum 8 s^4 k x.  A few roundings in 64
    # bits each.
    x = leaf(6, 8)
    s = 65536 / (65536 - round(65536 * 0.3))
    k = m.keep_mask(48, 0.3, 7, 2).view(6, 8).double()
    first, = torch.autograd.grad(lm.dropout(x, 0.3, 7, 2).square().sum(), x, create_graph=True)
    assert torch.allclose(first, 2 * s ** 2 * k * x, rtol=2.0 ** -49, atol=0)
    second, = torch.autograd.grad(first.square().sum(), x)
    assert torch.allclose(second, 8 * s ** 4 * k * x, rtol=2.0 ** -49, atol=0)


def test_a_step_advanced_before_the_backward_is_noticed(model_ops):
    # the gradient would be drawn from another mask than the result
    x, step = leaf(6, 8), torch.tensor([3])
    y = lm.dropout(x, 0.3, 7, 2, step_tensor=step)
    g, = torch.autograd.grad(y.sum(), x, retain_graph=True)
    assert torch.equal(g, lm.ops.dropout(torch.ones(6, 8).double(), 0.3, 7, 5))
    step += 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()

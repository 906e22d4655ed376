"""The modules of a language chain on the GPU: gradients through autograd, and
the whole chain under the sequences of a schedule."""
import pytest
import torch

import ops_model as m
from paper_1911_13214_amd import executor as ex
from paper_1911_13214_amd import ops

pytestmark = pytest.mark.gpu


def gradients(stages, x, dy, seq):
    for f in stages:
        for q in f.parameters():
            q.grad = None
    g = ex.run_sequence(stages, x, dy, seq)
    return g, [q.grad.clone() for f in stages for q in f.parameters()]


def chain(L, seed=3, rows=513, width=72, batch=50, dtype=torch.float32):
    from paper_1911_13214_amd import stages as lm
    stages = lm.language_chain(L - 2, seed, rows=rows, width=width, dtype=dtype, p=0.2)
    lm.set_step(stages, 5)
    g = torch.Generator().manual_seed(seed)
    tokens = torch.randint(0, rows, (batch + 1,), generator=g).cuda()
    targets = tokens[1:].clone()
    targets[::5] = -100
    stages[-1].targets = targets
    return stages, tokens[:-1].contiguous(), torch.ones((), device="cuda")


@pytest.mark.parametrize("L", [2, 3, 4])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_every_schedule_of_a_language_chain_gives_the_same_gradients(L, dtype):
    import model
    print("language chain", L, dtype, flush=True)
    stages, x, dy = chain(L, dtype=dtype)
    ref = gradients(stages, x, dy, ex.store_all_sequence(L))
    assert ref[0] is None and all(q.isfinite().all() and q.any() for q in ref[1])
    for _, seq in model.persistent_schedules(1, L):
        out = gradients(stages, x, dy, seq)
        assert all(torch.equal(a, b) for a, b in zip(out[1], ref[1])), seq


def test_a_language_chains_loss_and_gradients_in_64_bits():
    # the chain again from torch's 64-bit functions, masks from the model.
    # Six or so layers of 32-bit sums of at most 72 * 4 terms, logits of order
    # 1: 2^-24 times a few hundred, relative to each gradient's largest value.
    from paper_1911_13214_amd import stages as lm
    stages, x, dy = chain(4)
    out = gradients(stages, x, dy, ex.store_all_sequence(4))[1]
    params = [q.detach().cpu().double().requires_grad_() for f in stages for q in f.parameters()]
    names = [(k, n) for k, f in enumerate(stages) for n, _ in f.named_parameters()]
    p = dict(zip(names, params))
    y = p[0, "weight"][x.cpu()] * stages[0].scale

    def seam(k, name, x, z=None):
        s = getattr(stages[k], name)
        get = {n: p.get((k, f"{name}.{n}")) for n in ("post_weight", "post_bias", "gate", "pre_weight", "pre_bias")}
        return m.residual_norm(x, z, **s.kinds, **get)

    def branch(k, name, h):
        h = torch.nn.functional.linear(h, p[k, f"{name}.0.weight"], p[k, f"{name}.0.bias"])
        return torch.nn.functional.linear(torch.nn.functional.gelu(h), p[k, f"{name}.2.weight"], p[k, f"{name}.2.bias"])

    def drop(d, t):
        keep = m.keep_mask(t.numel(), d.p, d.seed, d.step).reshape(t.shape)
        q = round(65536 * d.p) / 65536
        return t * keep / (1 - q)

    for k in (1, 2):
        h = seam(k, "enter", y)[1]
        y, h = seam(k, "between", y, drop(stages[k].drops[0], branch(k, "first", h)))
        y = seam(k, "leave", y, drop(stages[k].drops[1], branch(k, "second", h)))[0]
    h = seam(3, "enter", y)[1]
    loss, _ = m.cross_entropy(h, p[3, "weight"], stages[3].targets.cpu(), -100)
    mean = loss.sum() / (stages[3].targets != -100).sum().cpu()
    with torch.no_grad():
        t = x
        for f in stages:
            t = f(t)
    assert abs(float(t) - float(mean)) < 512 * m.U32 * 10
    for name, got, ref in zip(names, out, torch.autograd.grad(mean, params)):
        err = (got.cpu().double() - ref).abs().max()
        assert err <= 2048 * m.U32 * ref.abs().max(), (name, float(err), float(ref.abs().max()))
    assert lm.Dropout(0.5, 1).eval()(x) is x


def test_dropout_follows_the_step():
    from paper_1911_13214_amd import stages as lm
    d = lm.Dropout(0.5, 77).cuda()
    x = torch.ones(40, 64, device="cuda", requires_grad=True)
    r = torch.randn(40, 64, device="cuda", requires_grad=True)
    d.step = 1
    a, b = d(x, r), d(x, r)
    d.step = 2
    c = d(x, r)
    assert torch.equal(a, b) and not torch.equal(a, c)
    d.step = 1
    y = d(x, r)
    d.step = 9  # a gradient belongs to the step of its forward
    w = torch.randn(40, 64, device="cuda")
    gx, gr = torch.autograd.grad(y, (x, r), w)
    assert torch.equal(gx, ops.dropout(w, 0.5, 77, 1)) and torch.equal(gr, w)


def test_optimal_sequences_of_a_language_chain_run_within_their_budgets():
    print("executor validate language L=10", flush=True)
    res = ex.validate(L=10, seed=2, width=512, batch=2048, slots=500, n_budgets=10, repeats=3, chain="language",
                      rows=8000)
    ok = [r for r in res["rows"] if r["feasible"]]
    assert len(ok) >= 3 and ok[0]["recomputed_forwards"] > 0
    assert res["all_gradients_equal"]
    for r in ok:
        # the allocator rounds blocks to 512 bytes
        assert r["measured_bytes"] <= r["budget_bytes"] * 1.02 + (8 << 20), r


def test_gradients_that_arrive_broadcast_or_transposed():
    # what autograd hands on for a sum (no strides) or through a transpose is
    # the same gradient as a dense one, bit for bit
    from paper_1911_13214_amd import stages as lm
    g = torch.Generator().manual_seed(4)
    x, z = (m.normal(g, 24, 40, dtype=torch.float32).cuda().requires_grad_() for _ in range(2))
    table = m.normal(g, 30, 40, dtype=torch.float32).cuda().requires_grad_()
    tokens = torch.randint(0, 30, (24,), generator=g).cuda()
    w = m.normal(g, 40, dtype=torch.float32).cuda().requires_grad_()
    calls = [(lambda: lm.dropout(x, 0.3, 7, 2, z), (x, z)), (lambda: lm.embedding(tokens, table, 2.0), (table,)),
             (lambda: lm.residual_norm(x, z, post="rms", pre="layer", pre_weight=w)[0], (x, z)),
             (lambda: lm.residual_norm(x, z, post="rms", pre="layer", pre_weight=w)[1], (x, z, w)),
             (lambda: lm.residual_norm(x, pre="rms", pre_weight=w)[1], (x, w)),
             (lambda: lm.linear_cross_entropy(x, table, tokens), (x, table))]
    for k, (call, wrt) in enumerate(calls):
        y = call()
        for dy in (torch.ones(1, device="cuda").expand_as(y), torch.randn(y.shape[::-1], device="cuda").t()):
            print("gradient layout", k, dy.stride(), flush=True)
            a = torch.autograd.grad(y, wrt, dy, retain_graph=True)
            b = torch.autograd.grad(y, wrt, dy.contiguous(), retain_graph=True)
            assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_inputs_that_are_slices_or_transposed():
    # what the operators refuse (rows that are not one pitch apart, columns
    # that are not adjacent, tokens that are not dense) is copied, and gives
    # what the dense tensors give, bit for bit, gradients included
    from paper_1911_13214_amd import stages as lm
    g = torch.Generator().manual_seed(14)

    def leaf(*shape):
        return m.normal(g, *shape, dtype=torch.float32).cuda().requires_grad_()

    x, z = leaf(3, 9, 40), leaf(3, 9, 40)
    table, gate = leaf(40, 40), leaf(1, 40)
    tokens = torch.randint(0, 40, (3, 9), generator=g).cuda()
    before, after = (lambda t: t[:, :-1]), (lambda t: t[:, 1:])
    turned = lambda t: t.transpose(0, 1)
    calls = [
        # the loss of the next token
        lambda c: lm.linear_cross_entropy(c(before(x)), table, c(after(tokens))),
        lambda c: lm.linear_cross_entropy(c(before(x)), c(table.t()), c(after(tokens).int())),
        lambda c: lm.embedding(c(before(tokens)), c(table.t()), 2.0, 3),
        lambda c: lm.embedding(c(turned(tokens)), table),
        lambda c: lm.dropout(c(turned(x)), 0.3, 7, 2, c(turned(z))),
        lambda c: lm.dropout(c(x.transpose(1, 2)), 0.3, 7, 2),
        lambda c: lm.residual_norm(c(turned(x)), c(turned(z)), post="rms", pre="layer", gate=c(gate.expand(9, 40)),
                                   pre_weight=c(table[:, 1]))[1],
        lambda c: lm.residual_norm(c(x.transpose(1, 2)[:, :, ::3]), pre="rms")[1]]
    for k, call in enumerate(calls):
        print("input layout", k, flush=True)
        out = []
        for c in (lambda t: t, lambda t: t.contiguous()):
            y = call(c)
            dy = torch.linspace(-1, 1, y.numel(), device="cuda").view_as(y)
            out.append([y, *torch.autograd.grad(y, (x, z, table, gate), dy, allow_unused=True)])
        for a, b in zip(*out):
            assert (a is None and b is None) or torch.equal(a, b), k

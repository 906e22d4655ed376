"""The operators that mix tokens, as a program uses them: their autograd
functions and modules, chains under a schedule, other streams, captured graphs,
infinities and NaN in places that a row does not see."""
import math

import pytest
import torch

import mix_model
import ops_model as m
from paper_1911_13214_amd import executor as ex
from paper_1911_13214_amd import ops

pytestmark = pytest.mark.gpu
TYPES = ["f32", "bf16", "f16"]


def normal(seed, *shape, dtype="f32", std=1.0):
    return m.normal(torch.Generator().manual_seed(seed), *shape, dtype=m.DTYPES[dtype], std=std).cuda()


# ---- places that a row does not see -----------------------------------------------------

def attend(q, k, v, dout, **how):
    out, lse = ops.window_attention(q, k, v, **how)
    return out, lse, *ops.window_attention_backward(dout, q, k, v, out, lse, **how)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_padding_may_hold_anything(dtype, bad):
    print("padding", dtype, bad, flush=True)
    n, lengths = 150, torch.tensor([97, 150, 3], dtype=torch.int32, device="cuda")
    t = [normal(i, 3, n, h, 64, dtype=dtype) for i, h in enumerate((4, 2, 2, 4))]
    for how in (dict(), dict(window=20, sinks=3)):
        want = attend(*t, lengths=lengths, **how)
        dirty = [x.clone() for x in t]
        for x in dirty:
            for b, end in enumerate(lengths.tolist()):
                x[b, end:] = bad
        got = attend(*dirty, lengths=lengths, **how)
        for b, end in enumerate(lengths.tolist()):
            assert all(torch.equal(x[b], y[b]) for x, y in zip(got, want))
            assert (got[0][b, end:] == 0).all() and (got[1][b, end:] == -math.inf).all()
            assert all((x[b, end:] == 0).all() for x in got[2:])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("n,h", [(100, 2), (14, 2), (40, 4)])
def test_rows_take_nothing_from_keys_they_do_not_see(dtype, bad, n, h):
    """A bad key or value changes the rows that see it alone; bad queries and
    gradients change the keys that their row sees alone."""
    print("unseen", dtype, bad, n, h, flush=True)
    window, sinks, at = 9, 2, 6
    q, k, v, dout = (normal(i, 1, n, y, 64, dtype=dtype) for i, y in enumerate((h, 2, 2, h)))
    see = mix_model.visible(1, n, n, window, sinks)[0]
    sees = see[:, at].cuda()
    # where infinities or NaN come up, products are added one by one instead: the
    # formula's bounds hold for both orders, equality does not
    val, err = mix_model.attention(*(x.cpu() for x in (q, k, v)), window, sinks, dout=dout.cpu())
    for i in (1, 2):
        dirty = [q, k, v, dout]
        dirty[i] = dirty[i].clone()
        dirty[i][:, at] = bad
        got = attend(*dirty, window=window, sinks=sinks)
        for x, name in ((got[0], "out"), (got[2], "dq")):
            m.close(x[:, ~sees], val[name][:, ~sees.cpu()], err[name][:, ~sees.cpu()], (i, name))
        if i == 2 or bad != -math.inf:
            assert not torch.isfinite(got[0][:, sees].float()).all()
    seen = see[at].cuda()
    for i in (0, 3):
        dirty = [q, k, v, dout]
        dirty[i] = dirty[i].clone()
        dirty[i][:, at] = bad
        got = attend(*dirty, window=window, sinks=sinks)
        others = torch.arange(n) != at
        for x, name in ((got[0], "out"), (got[2], "dq")):
            m.close(x.cpu()[:, others], val[name][:, others], err[name][:, others], (i, name))
        for x, name in ((got[3], "dk"), (got[4], "dv")):  # of keys that the row does not see
            m.close(x[:, ~seen], val[name][:, ~seen.cpu()], err[name][:, ~seen.cpu()], (i, name))
            assert not torch.isfinite(x[:, seen].float()).all() or i == 0


@pytest.mark.parametrize("dtype", TYPES)
def test_scores_of_minus_infinity_mask(dtype):
    """A column of ones in the queries and of minus infinity in a key hides
    that key from every row; a row that sees only such keys is NaN, as the
    formula is."""
    q, k, v = (normal(i, 1, 40, 2, 64, dtype=dtype) for i in range(3))
    q[..., 5] = 1.0
    k[..., 5] = 0.0
    hide = [0, 7, 8, 30]
    k[:, hide, :, 5] = -math.inf
    out, lse = ops.window_attention(q, k, v)
    assert out[:, 0].isnan().all()
    k[:, hide, :, 5] = 0.0
    qd, kd, vd = (x.double().cpu().permute(0, 2, 1, 3) for x in (q, k, v))
    s = (qd @ kd.transpose(-1, -2)) / 8
    hidden = torch.ones(40, 40, dtype=torch.bool).triu(1)
    hidden[:, hide] = True
    s = s.masked_fill(hidden, -math.inf)
    ref = (torch.softmax(s, -1) @ vd).permute(0, 2, 1, 3)
    # the bounds of mix_model, at their largest
    slack = (m.UNIT[q.dtype] + m.U32 * 80 * 64) * float(v.abs().double().amax())
    m.close(out[:, 1:], ref[:, 1:], slack, dtype)


# ---- layouts -----------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
def test_strides(dtype):
    """Heads out of one projection, heads before tokens, batch inside: the bits
    of dense ones."""
    b, n, h, hk, d = 2, 70, 6, 2, 64
    fused = normal(1, b, n, h + 2 * hk, d, dtype=dtype)
    q, k, v = fused[:, :, :h], fused[:, :, h:h + hk], fused[:, :, h + hk:]
    dout = normal(2, b, n, h, d, dtype=dtype)
    for how in (dict(), dict(window=11, sinks=1)):
        want = attend(*(x.contiguous() for x in (q, k, v, dout)), **how)
        before = [x.transpose(1, 2).contiguous().transpose(1, 2) for x in (q, k, v, dout)]
        inside = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v, dout)]
        for t in ([q, k, v, dout], before, inside):
            assert all(torch.equal(x, y) for x, y in zip(attend(*t, **how), want))
    one = attend(*(x[0] for x in (q, k, v, dout)))
    all_ = attend(q, k, v, dout)
    assert all(torch.equal(x, y[0]) for x, y in zip(one, all_))
    # one key head for a batch, by a stride of 0
    shared = attend(q, k[:1].expand(b, n, hk, d), v[:1].expand(b, n, hk, d), dout)
    dense = attend(q, k[:1].repeat(b, 1, 1, 1), v[:1].repeat(b, 1, 1, 1), dout)
    assert all(torch.equal(x, y) for x, y in zip(shared, dense))


@pytest.mark.parametrize("dtype", TYPES)
def test_step_strides(dtype):
    b, h, hk, d, slots = 3, 4, 2, 64, 50
    at = torch.tensor([49, 3, 20], dtype=torch.int32, device="cuda")
    heads = normal(1, b, h + 2 * hk, d, dtype=dtype)
    q, k, v = heads[:, :h], heads[:, h:h + hk], heads[:, h + hk:]
    caches = normal(2, 2, b, slots, hk, d, dtype=dtype)
    dense = [c.clone() for c in caches]
    want = ops.window_attention_step(q.contiguous(), k.contiguous(), v.contiguous(), *dense, at, window=17, sinks=2)
    both = caches.permute(1, 3, 2, 0, 4).contiguous().permute(3, 0, 2, 1, 4)  # keys and values side by side
    out = torch.full((b, h + 1, d), 7.0, dtype=q.dtype, device="cuda")
    got = ops.window_attention_step(q, k, v, both[0], both[1], at, window=17, sinks=2, out=out[:, 1:])
    assert torch.equal(got, want) and (out[:, 0] == 7).all()
    assert torch.equal(both[0], dense[0]) and torch.equal(both[1], dense[1])


# ---- long -------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
def test_parts_of_the_keys_and_of_the_rows(dtype):
    """Few rows against many keys, and few keys' tiles against many rows: sums
    in parts, joined."""
    from test_gpu_attention import check
    check(dtype, 1, 5, 4100, 2, 1, 64, train=False)
    check(dtype, 1, 100, 3000, 1, 1, 128, train=False)
    check(dtype, 2, 33, 2500, 4, 2, 64, window=2000, sinks=5, train=False, positions=[2467, 1500])
    check(dtype, 1, 1500, 1500, 2, 1, 64, window=70, sinks=3)
    check(dtype, 1, 700, 700, 4, 1, 64)
    check(dtype, 1, 1, 1500, 40, 1, 128)


def test_more_parts_than_a_workgroup_joins():
    """One tile of rows against keys for more than 256 parts: values that are
    the keys' own numbers, so that a part left out shows, uniform scores."""
    n, keys = 40, 300000
    q, k = torch.zeros(1, n, 1, 8, device="cuda"), torch.zeros(1, keys, 1, 8, device="cuda")
    v = (torch.arange(keys, device="cuda", dtype=torch.float32) / keys)[None, :, None, None].expand(1, keys, 1, 8)
    out, lse = ops.window_attention(q, k, v.contiguous())
    seen = torch.arange(keys - n + 1, keys + 1, dtype=torch.float64)
    # sums of 300000 terms in parts of 1200, in lanes of 600: 600 + 256 roundings
    m.close(out[0, :, 0], ((seen - 1) / 2 / keys)[:, None].expand(n, 8), 900 * m.U32)
    m.close(lse[0, :, 0], torch.log(seen), 900 * m.U32)


def test_a_cache_past_32_bits():
    """A cache whose slots lie more than 2^31 elements and 2^32 bytes apart."""
    slots, hk, d = 2 ** 20 + 64, 16, 128  # 4.3 GB each
    k, v = (torch.zeros(1, slots, hk, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    g = torch.Generator().manual_seed(1)
    near = [m.normal(g, 1, 64, hk, d, dtype=torch.bfloat16) for _ in range(2)]
    q, new_k, new_v = (m.normal(g, 1, n, d, dtype=torch.bfloat16) for n in (hk, hk, hk))
    k[:, slots - 65:slots - 1], v[:, slots - 65:slots - 1] = near[0].cuda(), near[1].cuda()
    at = torch.tensor([slots - 1], device="cuda")
    out = ops.window_attention_step(q.cuda(), new_k.cuda(), new_v.cuda(), k, v, at, window=65)
    whole = [torch.cat([x, y[:, None]], 1) for x, y in zip(near, (new_k, new_v))]
    val, err = mix_model.attention(q[:, None], *whole)
    m.close(out, val["out"][:, 0], err["out"][:, 0])
    assert torch.equal(k[:, -1].cpu(), new_k) and torch.equal(v[:, -1].cpu(), new_v)
    # and as keys of a piece of a prompt: positions past the first 2^31 elements
    far, lse = ops.window_attention(q.cuda()[:, None].expand(1, 40, hk, d), k, v, window=30,
                                    positions=at - 39)
    assert lse.isfinite().all()
    m.close(far[:, -1], mix_model.attention(q[:, None], *whole, window=30)[0]["out"][:, 0], err["out"][:, 0] * 4)


def test_without_elements():
    for n, keys in ((0, 0), (0, 5), (5, 0)):
        q, k = torch.zeros(2, n, 4, 64, device="cuda"), torch.ones(2, keys, 2, 64, device="cuda")
        out, lse, dq, dk, dv = attend(q, k, k, q)
        assert (out == 0).all() and out.shape == q.shape and (lse == -math.inf).all() and (dq == 0).all()
        assert dk.shape == k.shape and (dk == 0).all() and (dv == 0).all()
    q, c = torch.zeros(0, 4, 64, device="cuda"), torch.zeros(0, 7, 4, 64, device="cuda")
    assert ops.window_attention_step(q, q, q, c, c, torch.zeros(0, dtype=torch.int32, device="cuda")).shape == q.shape


# ---- refusals -----------------------------------------------------------------------------------

def test_refusals():
    x, w = torch.zeros(2, 8, 4, 64, device="cuda"), torch.ones(64, device="cuda")
    at = torch.zeros(2, dtype=torch.int32, device="cuda")
    cache, other, one = torch.zeros(2, 16, 4, 64, device="cuda"), torch.zeros(2, 16, 4, 64, device="cuda"), x[:, 0]
    odd = torch.zeros(2, 8, 4, 66, device="cuda")[..., 1:65]
    half, double = x.half(), x.double()
    lse = torch.zeros(2, 8, 4, device="cuda")
    bad = [
        lambda: ops.head_norm_rotate(double), lambda: ops.head_norm_rotate(x, half), lambda: ops.head_norm_rotate(x[0, 0]),
        lambda: ops.head_norm_rotate(x, x[:, :4]), lambda: ops.head_norm_rotate(x, norm="batch"),
        lambda: ops.head_norm_rotate(x, rotary=66), lambda: ops.head_norm_rotate(x, rotary=3),
        lambda: ops.head_norm_rotate(x, eps=-1.0), lambda: ops.head_norm_rotate(x, base=0.0),
        lambda: ops.head_norm_rotate(x, k_weight=w), lambda: ops.head_norm_rotate(x, q_weight=w, norm="none"),
        lambda: ops.head_norm_rotate(x, q_weight=w[:32]), lambda: ops.head_norm_rotate(x, positions=at),
        lambda: ops.head_norm_rotate(x, positions=torch.zeros(8, device="cuda")),
        lambda: ops.head_norm_rotate(x, frequencies=[1.0]), lambda: ops.head_norm_rotate(x.transpose(-1, -2)),
        lambda: ops.head_norm_rotate(x, x, out=(x, None)), lambda: ops.head_norm_rotate(x, out=(x[:1].expand(2, 8, 4, 64), None)),
        lambda: ops.head_norm_rotate_backward(x, None, x, x), lambda: ops.head_norm_rotate_backward(x[:1], None, x),
        lambda: ops.window_attention(double, double, double), lambda: ops.window_attention(x, half, x),
        lambda: ops.window_attention(x, x[:1], x[:1]), lambda: ops.window_attention(x, x[:, :, :3], x[:, :, :3]),
        lambda: ops.window_attention(x, x, x[:, :4]), lambda: ops.window_attention(x, x, x, window=0),
        lambda: ops.window_attention(x, x, x, sinks=-1), lambda: ops.window_attention(x, x, x, scale=0.0),
        lambda: ops.window_attention(x, x, x, scale=math.nan), lambda: ops.window_attention(x, x, x, positions=at[:1]),
        lambda: ops.window_attention(x, x, x, lengths=at.float()), lambda: ops.window_attention(odd, odd, odd),
        lambda: ops.window_attention(*(x[..., :60],) * 3), lambda: ops.window_attention(*(torch.zeros(1, 1, 1, 136, device="cuda"),) * 3),
        lambda: ops.window_attention(x.transpose(-1, -2), x, x),
        lambda: ops.window_attention_backward(x, x, x, x, x, lse[:1]), lambda: ops.window_attention_backward(x, x, x, x, half, lse),
        lambda: ops.window_attention_backward(x[:1], x, x, x, x, lse),
        lambda: ops.window_attention_step(x, one, one, cache, other, at), lambda: ops.window_attention_step(one, one, one, cache, other, None),
        lambda: ops.window_attention_step(one, one, one, cache, other, at, ring=True),
        lambda: ops.window_attention_step(one, one, one, cache, other, at, ring=True, window=15, sinks=2),
        lambda: ops.window_attention_step(one, one[:1], one, cache, other, at),
        lambda: ops.window_attention_step(one, one, one, cache, cache, at),
        lambda: ops.window_attention_step(one, one, one, cache, other[:, :8], at),
        lambda: ops.window_attention_step(one, one, one, cache[:1].expand(2, 16, 4, 64), other, at),
        lambda: ops.window_attention_step(one, one, one, cache[:, :0], other[:, :0], at),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            print("not refused", i)


# ---- streams and graphs ----------------------------------------------------------------------------

def together(t, at, caches, stream=None):
    """All operators, one after the other, as a training step and a decoding
    step use them."""
    kw = {} if stream is None else dict(stream=stream)
    q, k = ops.head_norm_rotate(t["q"], t["k"], q_weight=t["w"], k_weight=t["w"], positions=t["at"], **kw)
    how = dict(window=20, sinks=2, lengths=t["lengths"])
    out, lse = ops.window_attention(q, k, t["v"], **how, **kw)
    dq, dk, dv = ops.window_attention_backward(t["dout"], q, k, t["v"], out, lse, **how, **kw)
    g = ops.head_norm_rotate_backward(dq, dk, t["q"], t["k"], q_weight=t["w"], k_weight=t["w"], positions=t["at"], **kw)
    far, _ = ops.window_attention(q[:, -3:].contiguous(), t["long_k"], t["long_v"], stats=False, **kw)
    step = ops.window_attention_step(q[:, 0], k[:, 0], t["v"][:, 0], *caches, at, window=20, sinks=2, ring=True, **kw)
    return [out, lse, dv, *(g[x] for x in sorted(g)), far, step, *caches]


def inputs(seed, dtype):
    b, n, h, hk, d = 2, 60, 4, 2, 64
    fused = normal(seed, b, n, h + 2 * hk, d, dtype=dtype)
    t = dict(q=fused[:, :, :h], k=fused[:, :, h:h + hk], v=fused[:, :, h + hk:], w=normal(seed + 1, d, dtype=dtype),
             dout=normal(seed + 2, b, n, h, d, dtype=dtype), at=torch.arange(n, device="cuda") + seed,
             lengths=torch.tensor([n, 40 + seed % 10], device="cuda"), long_k=normal(seed + 3, b, 2048, hk, d, dtype=dtype),
             long_v=normal(seed + 4, b, 2048, hk, d, dtype=dtype))
    return t, torch.tensor([seed % 30, 200 + seed], device="cuda"), normal(seed + 5, 2, b, 30, hk, d, dtype=dtype)


@pytest.mark.parametrize("dtype", TYPES)
def test_another_stream(dtype):
    t, at, caches = inputs(3, dtype)
    want = together(t, at, caches.clone())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = together(t, at, caches, side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("dtype", TYPES)
def test_a_captured_graph_replayed_on_new_inputs(dtype):
    sets = [inputs(s, dtype) for s in (3, 40, 77)]
    t, at, caches = ({k: v.clone() for k, v in sets[0][0].items()}, sets[0][1].clone(), sets[0][2].clone())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        together(t, at, caches)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = together(t, at, caches)
    for turn in range(2):
        for u, where, c in sets:
            want = together(u, where, c.clone())
            for k in t:
                t[k].copy_(u[k])
            at.copy_(where)
            caches.copy_(c)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(out, want)), turn


def test_two_graphs_with_a_pool_between_them():
    sets = [inputs(s, "bf16") for s in (5, 21)]
    want = [together(t, at, c.clone()) for t, at, c in sets]
    graphs, outs, pool = [], [], None
    for t, at, c in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, pool=pool):
            outs.append(together(t, at, c))
        pool = g.pool()
        graphs.append(g)
    for order in ((0, 1), (0, 1)):
        for i in order:
            graphs[i].replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(outs[i], want[i])), i


# ---- autograd, modules, chains ---------------------------------------------------------------------------

def test_gradients_of_all_together_in_64_bits():
    """Norms, rotation and attention through autograd, with inputs of other
    layouts, against 64-bit automatic differentiation: a few hundred 32-bit
    roundings, relative to each result's largest value."""
    from paper_1911_13214_amd import stages as lm
    b, n, h, hk, d = 2, 45, 4, 2, 24
    leaves = [normal(i, *s).requires_grad_() for i, s in enumerate([(b, n, d, h), (b, hk, n, d), (b, n, hk, d), (d,), (d,)])]
    lengths = torch.tensor([45, 30], device="cuda")
    w = normal(9, b, d, h, n)

    def run(q, k, v, qw, kw, rotate, attend):
        q, k = q.transpose(2, 3), k.transpose(1, 2)
        q, k = rotate(q, k, qw, kw)
        return attend(q, k, v).permute(0, 3, 2, 1)

    for norm in ("rms", "layer", "none"):
        some = norm != "none"
        got = run(*leaves[:3], *(leaves[3:] if some else (None, None)),
                  lambda q, k, qw, kw: lm.head_norm_rotate(q, k, norm=norm, q_weight=qw, k_weight=kw, rotary=16),
                  lambda q, k, v: lm.window_attention(q, k, v, window=11, sinks=2, lengths=lengths))
        args = leaves if some else leaves[:3]
        grads = torch.autograd.grad(got, args, w)
        double = [x.detach().cpu().double().requires_grad_() for x in leaves]
        see = mix_model.visible(b, n, n, 11, 2, lengths=lengths)[:, None]

        def exact(q, k, v):
            q, k, v = q.permute(0, 2, 1, 3), *(x.permute(0, 2, 1, 3).repeat_interleave(h // hk, 1) for x in (k, v))
            s = (q @ k.transpose(-1, -2) / d ** 0.5).masked_fill(~see, -1e30)
            return (torch.softmax(s, -1) * see @ v).permute(0, 2, 1, 3)

        at = torch.arange(n).expand(b, n)
        ref = run(*double[:3], *(double[3:] if some else (None, None)),
                  lambda q, k, qw, kw: [mix_model.rotation(x, y, norm, 1e-5, at, 16) for x, y in ((q, qw), (k, kw))], exact)
        want = torch.autograd.grad(ref, double if some else double[:3], w.cpu().double())
        for x, y in zip((got, *grads), (ref, *want)):
            assert (x.detach().cpu().double() - y).abs().max() <= 1024 * m.U32 * y.detach().abs().max(), norm


def test_second_derivatives_raise():
    from paper_1911_13214_amd import stages as lm
    q = normal(1, 1, 6, 2, 16).requires_grad_()
    for y in (lm.head_norm_rotate(q)[0], lm.window_attention(q, q, q)):
        g, = torch.autograd.grad(y.square().sum(), q, create_graph=True)
        with pytest.raises(RuntimeError):
            g.sum().backward()


def gradients(stages, x, dy, seq):
    for f in stages:
        for q in f.parameters():
            q.grad = None
    ex.run_sequence(stages, x, dy, seq)
    return [q.grad.clone() for f in stages for q in f.parameters()]


def chain(L, dtype, attention, seed=3, rows=300, width=64, batch=2, tokens=37, lengths=None):
    from paper_1911_13214_amd import stages as lm
    stages = lm.language_chain(L - 2, seed, rows=rows, width=width, dtype=dtype, p=0.1, attention=attention)
    lm.set_step(stages, 5)
    lm.set_lengths(stages, lengths)
    g = torch.Generator().manual_seed(seed)
    text = torch.randint(0, rows, (batch, tokens + 1), generator=g).cuda()
    targets = text[:, 1:].clone()
    if lengths is not None:
        targets[torch.arange(tokens, device="cuda") >= lengths[:, None]] = -100
    stages[-1].targets = targets
    return stages, text[:, :-1].contiguous(), torch.ones((), device="cuda")


HOW = dict(heads=4, kv_heads=2, head_width=16, window=9, sinks=2)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_every_schedule_of_a_chain_with_attention_gives_the_same_gradients(dtype):
    import model
    print("chain with attention", dtype, flush=True)
    lengths = torch.tensor([37, 21], dtype=torch.int32, device="cuda")
    stages, x, dy = chain(4, dtype, HOW, lengths=lengths)
    ref = gradients(stages, x, dy, ex.store_all_sequence(4))
    assert all(q.isfinite().all() and q.any() for q in ref)
    for _, seq in model.persistent_schedules(1, 4):
        assert all(torch.equal(a, b) for a, b in zip(gradients(stages, x, dy, seq), ref)), seq
    # without attention's stages a chain is what it was
    from paper_1911_13214_amd import stages as lm
    assert not any(isinstance(mod, lm.Attention) for f in lm.language_chain(2, 1, rows=10, width=8) for mod in f.modules())


def test_the_gradients_of_a_chain_with_attention_are_those_of_differences():
    """The loss along a direction of all parameters: central differences of a
    chain in 32 bits.  The loss is of order 6 with an error of a few 2^-24 of
    it, the step 2^-6 of weights of order 1 / sqrt(64): the difference is off by
    about 2^-20 / 2^-5 and by the third derivative times 2^-12."""
    stages, x, dy = chain(3, torch.float32, HOW)
    params = [q for f in stages for q in f.parameters()]
    grads = gradients(stages, x, dy, ex.store_all_sequence(3))
    way = [normal(100 + i, *q.shape) * q.detach().abs().mean() for i, q in enumerate(params)]

    def loss(e):
        with torch.no_grad():
            for q, d in zip(params, way):
                q += e * d
            t = x
            for f in stages:
                t = f(t)
            for q, d in zip(params, way):
                q -= e * d
        return float(t)

    want = sum(float((g.double() * d.double()).sum()) for g, d in zip(grads, way))
    size = sum(float((g.double() * d.double()).square().sum()) for g, d in zip(grads, way)) ** 0.5
    got = (loss(2.0 ** -8) - loss(-2.0 ** -8)) / 2.0 ** -7
    assert abs(got - want) <= 0.02 * max(size, abs(want)), (got, want, size)


def test_attention_token_by_token():
    """The module's step, with linear and ring caches, against its forward: both
    lie within their 32-bit error of each other."""
    from paper_1911_13214_amd import stages as lm
    torch.manual_seed(5)
    mod = lm.Attention(48, 4, 2, 16, window=9, sinks=2).cuda()
    x = normal(6, 3, 40, 48)
    with torch.no_grad():
        want = mod(x)
    for ring, slots in ((False, 40), (True, 11)):
        kc, vc = (torch.full((3, slots, 2, 16), math.nan, device="cuda") for _ in range(2))
        at = torch.zeros(3, dtype=torch.int64, device="cuda")
        for i in range(40):
            got = mod.step(x[:, i], kc, vc, at, ring=ring)
            assert (got - want[:, i]).abs().max() <= 256 * m.U32 * want.abs().max(), (ring, i)
            at += 1


def test_optimal_sequences_of_a_chain_with_attention_run_within_their_budgets():
    print("executor validate language with attention", flush=True)
    res = ex.validate(L=8, seed=2, width=512, batch=2048, slots=500, n_budgets=6, repeats=3, chain="language", rows=8000,
                      attention=dict(heads=8, kv_heads=2, window=256, sinks=4))
    ok = [r for r in res["rows"] if r["feasible"]]
    assert len(ok) >= 2 and res["all_gradients_equal"]
    for r in ok:
        # the allocator rounds blocks to 512 bytes
        assert r["measured_bytes"] <= r["budget_bytes"] * 1.02 + (8 << 20), r


def test_float16_gradients_of_large_values_and_small_probabilities():
    """Scores' gradients that leave float16's range at the scale that keeps
    small probabilities exact: values of 2000 all of one sign, times gradients
    of one sign; and long rows, whose probabilities are small."""
    from test_gpu_attention import check
    n, d = 80, 64
    g = torch.Generator().manual_seed(3)
    q, k = (m.normal(g, 1, n, 2, d, dtype=torch.float16) for _ in range(2))
    v = (m.normal(g, 1, n, 2, d, std=1.0).abs() * 1000 + 1000).half()
    dout = (m.normal(g, 1, n, 2, d).abs() + 1.0).half()
    val, err = mix_model.attention(q, k, v, dout=dout)
    got = attend(*(x.cuda() for x in (q, k, v, dout)))
    for x, name in zip((got[0], *got[2:]), ("out", "dq", "dk", "dv")):
        m.close(x, val[name], err[name], name)
    check("f16", 1, 1400, 1400, 1, 1, 64)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [8, 32, 64])
def test_the_rounding_of_the_output_stays_out_of_the_queries_gradients(dtype, d):
    """Keys that are all the same: the gradients of a row's scores sum to 0, and
    with them dq and, over the rows, what dk takes from each.  Values next to 8,
    so that do times the rounded output misses that sum by far more than the
    roundings of the single gradients."""
    n, t = 700, m.DTYPES[dtype]
    unit, scale = m.UNIT[t], d ** -0.5
    g = torch.Generator().manual_seed(d)
    q, dout = m.normal(g, 1, n, 1, d, dtype=t), m.normal(g, 1, n, 1, d, dtype=t)
    k = torch.full((1, n, 1, d), 0.5, dtype=t)
    step = 2.0 ** -4 if dtype == "bf16" else 2.0 ** -7  # between numbers from 8 on
    v = (8 + step * torch.randint(0, 2, (1, n, 1, d), generator=g)).to(t)
    out, lse = ops.window_attention(q.cuda(), k.cuda(), v.cuda())
    dq, dk, _ = ops.window_attention_backward(dout.cuda(), q.cuda(), k.cuda(), v.cuda(), out, lse)
    do, vv, o, qq = (x[0, :, 0].double().cpu() for x in (dout, v, out, q))
    see = torch.ones(n, n, dtype=torch.float64).tril()
    p = see / see.sum(1, keepdim=True)
    dp, rough = do @ vv.T, (do * o).sum(1, keepdim=True)
    missing = (p * (dp - rough)).sum(1, keepdim=True)
    # roundings of P (dP - delta) and, for what is put right, of P; sums of n
    # terms in 32 bits of the size of do v; float16's P below 2^-14 lose 2^-25
    size = m.U32 * (n + d + 32) * do.abs() @ vv.abs().T.amax(1, keepdim=True)
    least = 2.0 ** -25 * see.sum(1, keepdim=True) if dtype == "f16" else 0.0
    off = unit * (p * (dp - rough).abs()).sum(1, keepdim=True) + (unit + least) * missing.abs() + size
    if dtype == "f16":
        # dS times 2^(3 - e) and more: what is below 2^-14 loses 2^-25 of it
        off += 2.0 ** -25 * 2.0 ** -2 * do.abs().amax(1, keepdim=True) * see.sum(1, keepdim=True)
    # (a result below float16's normal numbers is off by 2^-25, half its least step)
    bound = scale * 0.5 * off * (1 + unit) + m.TINY[t]
    assert (dq[0, :, 0].double().cpu().abs() <= bound).all()
    # what the test can tell: rows that would miss 4 times their bound (in float16 a
    # share of them: o misses 2^-9 on average, sqrt(d) of that in delta, and 4 times
    # the bound of the 32-bit sums is 4 * 2^-24 * (700 + d) * 8 * sqrt(d), the same)
    assert (scale * 0.5 * missing.abs() > 4 * bound)[300:].any()
    want = scale * (p * (dp - (p * dp).sum(1, keepdim=True))).T @ qq
    err = scale * (p * (unit * (dp - rough).abs() + unit * missing.abs() + size)).T @ qq.abs() + unit * want.abs()
    if dtype == "f16":
        err += scale * 2.0 ** -27 * (see.T @ (do.abs().amax() * qq.abs()))
    assert ((dk[0, :, 0].double().cpu() - want).abs() <= err * (1 + unit) + m.TINY[t]).all()

"""The operators of a chain's stages on the GPU against plain 64-bit
implementations (ops_model.py).  Tolerances: one rounding of the result's type
plus a bound on the 32-bit arithmetic before it, stated at each test."""
import ctypes
import itertools

import pytest
import torch

import ops_model as m
import xent_plan
from paper_1911_13214_amd import ops

pytestmark = pytest.mark.gpu
TYPES = ["f32", "bf16", "f16"]


def gpu(t):
    return None if t is None else t.cuda()


# ---- dropout --------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(1,), (7,), (8,), (9,), (3, 5), (64, 33), (2, 3, 40), (5, 1000)])
def test_dropout(dtype, shape):
    print("dropout", dtype, shape, flush=True)
    g = torch.Generator().manual_seed(len(shape) + shape[-1])
    x, r = m.normal(g, *shape, dtype=m.DTYPES[dtype]), m.normal(g, *shape, dtype=m.DTYPES[dtype])
    for p, seed, step, res in [(0.1, 5, 0, None), (0.5, 2 ** 63 + 12345, 2 ** 40 + 7, r), (0.0, 1, 1, r), (1.0, 1, 1, r),
                               (0.37, -1, -2, None)]:
        out = ops.dropout(gpu(x), p, seed, step, residual=gpu(res))
        ref = m.dropout(x, p, seed % 2 ** 64, step % 2 ** 64, res)
        # the factor and the product are rounded once each, and the sum
        slack = 4 * m.U32 * ((x.double() * 2.1).abs() + ref.abs())
        m.close(out, ref, slack, (p, seed, step))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols,pitch", [(8, 16), (40, 48), (33, 40), (3, 5), (1, 4), (17, 17 + 8)])
def test_dropout_of_strided_rows_has_the_mask_of_dense_ones(dtype, cols, pitch):
    print("dropout strided", dtype, cols, pitch, flush=True)
    g = torch.Generator().manual_seed(cols)
    whole = m.normal(g, 21, pitch, dtype=m.DTYPES[dtype]).cuda()
    x, r = whole[:, :cols], m.normal(g, 21, cols, dtype=m.DTYPES[dtype]).cuda()
    dense = ops.dropout(x.contiguous(), 0.3, 9, 4, residual=r)
    assert torch.equal(ops.dropout(x, 0.3, 9, 4, residual=r), dense)
    out = torch.full((21, pitch + 3), 7.0, dtype=x.dtype, device="cuda")
    ops.dropout(x, 0.3, 9, 4, residual=r, out=out[:, 1:1 + cols])
    assert torch.equal(out[:, 1:1 + cols], dense)
    assert (out[:, 0] == 7).all() and (out[:, 1 + cols:] == 7).all()
    # in place, and from a pointer that is aligned to one element only
    y = x.contiguous()
    assert ops.dropout(y, 0.3, 9, 4, residual=r, out=y) is y and torch.equal(y, dense)
    odd = torch.empty(21 * cols + 1, dtype=x.dtype, device="cuda")[1:].view(21, cols)
    odd.copy_(x)
    assert torch.equal(ops.dropout(odd, 0.3, 9, 4, residual=r), dense)


def test_dropped_infinities_and_nans_vanish():
    x = torch.full((4, 64), float("nan"))
    keep = m.keep_mask(x.numel(), 0.5, 3, 8).view(4, 64)
    x[keep] = 1.0
    x[~keep & (torch.arange(64) % 2 == 0)] = float("inf")
    out = ops.dropout(x.cuda(), 0.5, 3, 8).cpu()
    assert torch.equal(out, torch.where(keep, 2.0, 0.0))


def test_dropout_steps_from_the_device_and_in_a_graph():
    x = torch.ones(3, 50, device="cuda")
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    out = torch.empty_like(x)
    want = [ops.dropout(x, 0.4, 21, 100 + k) for k in range(4)]
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ops.dropout(x, 0.4, 21, 100, step_tensor=step, out=out)
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        ops.dropout(x, 0.4, 21, 100, step_tensor=step, out=out)
    for k in range(4):
        step.fill_(k)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[k]), k
        assert torch.equal(ops.dropout(x, 0.4, 21, 100, step_tensor=step), want[k])
    assert not torch.equal(want[0], want[1])


def test_operators_without_elements():
    x = torch.zeros(0, 5, device="cuda")
    assert ops.dropout(x, 0.5, 1).shape == (0, 5)
    none = torch.zeros(0, dtype=torch.int64, device="cuda")
    assert ops.embedding(none, torch.ones(4, 5, device="cuda")).shape == (0, 5)
    assert torch.equal(ops.embedding_backward(none, x, 4), torch.zeros(4, 5, device="cuda"))
    w = torch.ones(5, device="cuda")
    y, h, st = ops.residual_norm(x, x, post="rms", post_weight=w, gate=w, pre="layer", pre_weight=w, pre_bias=w)
    g = ops.residual_norm_backward(x, x, y, x, st, post="rms", post_weight=w, gate=w, pre="layer", pre_weight=w,
                                   pre_bias=w)
    assert g["x"].shape == (0, 5)
    for k in ("post_weight", "gate", "pre_weight", "pre_bias"):
        assert torch.equal(g[k], torch.zeros(5, device="cuda")), k


# ---- embedding --------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [1, 7, 8, 9, 64, 515, 2056])
def test_embedding(dtype, cols):
    print("embedding", dtype, cols, flush=True)
    g = torch.Generator().manual_seed(cols)
    table = m.normal(g, 37, cols, dtype=m.DTYPES[dtype])
    for n, scale, tt in [(1, 1.0, torch.int64), (5, 3.25, torch.int32), (1030, -0.7, torch.int64)]:
        tokens = torch.randint(0, 37, (n,), generator=g)
        if n == 5:
            tokens[1], tokens[3] = -1, 37  # outside the table
        out = ops.embedding(tokens.to(tt).cuda(), table.cuda(), scale).cpu()
        ref = m.embedding(tokens, table, scale)
        lost = ref.isnan()
        assert torch.equal(out.isnan(), lost)
        # the scale is rounded to 32 bits, and the product
        m.close(torch.where(lost, 0.0, out), torch.where(lost, 0.0, ref),
                2 * m.U32 * torch.where(lost, 0.0, ref).abs(), (n, scale))
    # leading dimensions, a table and a result with other pitches
    tokens = torch.randint(0, 37, (3, 4), generator=g).cuda()
    wide = torch.zeros(37, cols + 5, dtype=table.dtype, device="cuda")
    wide[:, 2:2 + cols] = table.cuda()
    out = torch.full((3, 4, cols + 3), 7.0, dtype=table.dtype, device="cuda")
    ops.embedding(tokens, wide[:, 2:2 + cols], 2.0, out=out[..., 1:1 + cols])
    assert torch.equal(out[..., 1:1 + cols], ops.embedding(tokens, table.cuda(), 2.0))
    assert (out[..., 0] == 7).all() and (out[..., 1 + cols:] == 7).all()


def tokens_of(kind, n, rows, g):
    if kind == "uniform":
        return torch.randint(0, rows, (n,), generator=g)
    if kind == "one":
        return torch.full((n,), rows // 2)
    if kind == "last":  # the table's ends
        return torch.where(torch.rand(n, generator=g) < 0.5, 0, rows - 1)
    t = (torch.rand(n, generator=g, dtype=torch.float64) ** 4 * rows).long()  # most tokens small
    t[::7] = -3
    t[5::11] = rows + 2
    return t


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["uniform", "one", "last", "skewed"])
@pytest.mark.parametrize("n,rows,cols", [(1, 5, 8), (31, 3, 5), (32, 700, 64), (33, 1, 12), (65, 600, 7),
                                         (1000, 513, 129), (2049, 300000, 3), (5000, 4000, 70), (4097, 70000, 16)])
def test_embedding_gradient(dtype, kind, n, rows, cols):
    print("embedding gradient", dtype, kind, n, rows, cols, flush=True)
    g = torch.Generator().manual_seed(n + rows + cols)
    tokens = tokens_of(kind, n, rows, g)
    dy = m.normal(g, n, cols, dtype=m.DTYPES[dtype])
    for scale, padding in [(1.0, None), (-2.5, 0)]:
        out = ops.embedding_backward(tokens.cuda(), dy.cuda(), rows, scale, padding=padding)
        ref, mag = m.embedding_grad(tokens, dy, rows, scale, padding)
        # n terms in 32 bits, each partial sum below mag
        m.close(out, ref, (n + 4) * m.U32 * mag, (scale, padding))
        assert torch.equal(out, ops.embedding_backward(tokens.int().cuda(), dy.cuda(), rows, scale, padding=padding))


@pytest.mark.parametrize("n", [3, 700, 2048, 2049])
@pytest.mark.parametrize("rows", [2, 512, 513, 262144, 262145, 3000000])
def test_embedding_gradient_by_table_size(n, rows):
    # one, two and three digits of the sort, in one launch (up to 2048 tokens)
    # and in one each
    print("embedding gradient digits", n, rows, flush=True)
    g = torch.Generator().manual_seed(n + rows)
    tokens = tokens_of("uniform", n, rows, g)
    tokens[-1], tokens[0] = rows - 1, 0
    dy = m.normal(g, n, 9, dtype=torch.float32)
    ref, mag = m.embedding_grad(tokens, dy, rows, 1.0)
    m.close(ops.embedding_backward(tokens.cuda(), dy.cuda(), rows), ref, (n + 4) * m.U32 * mag)


@pytest.mark.parametrize("n,rows", [(32768, 300), (32769, 70000), (140001, 300), (530000, 70000), (1100003, 3000000)])
@pytest.mark.parametrize("kind", ["uniform", "one", "skewed"])
def test_embedding_gradient_of_many_tokens(n, rows, kind):
    # the largest sort whose workgroups count all keys, and some whose digits
    # are counted beforehand: one, two and three of them, one to three parts a
    # workgroup, the last one not whole
    print("embedding gradient of many tokens", n, rows, kind, flush=True)
    g = torch.Generator().manual_seed(n + rows)
    tokens = tokens_of(kind, n, rows, g)
    dy = m.normal(g, n, 3, dtype=torch.float32)
    out = ops.embedding_backward(tokens.cuda(), dy.cuda(), rows, padding=1)
    ref, mag = m.embedding_grad(tokens, dy, rows, 1.0, 1)
    m.close(out, ref, (n + 4) * m.U32 * mag)
    assert torch.equal(out, ops.embedding_backward(tokens.int().cuda(), dy.cuda(), rows, padding=1))
    # exact in whole numbers: no token is lost or added twice
    dy = torch.randint(-3, 4, (n, 3), generator=g).float()
    ref, mag = m.embedding_grad(tokens, dy, rows, 1.0, 1)
    if float(mag.max()) < 2.0 ** 24:
        assert torch.equal(ops.embedding_backward(tokens.cuda(), dy.cuda(), rows, padding=1).cpu().double(), ref)


def test_embedding_gradients_time_does_not_grow_with_the_square_of_the_tokens():
    # four times the tokens: four times the time and, for the caches' sake, at
    # most half as much again, where a cost that grows with their square gives
    # sixteen times
    ms = []
    for n in (1 << 20, 1 << 22):
        tokens = torch.randint(0, 500, (n,), device="cuda")
        dy = torch.ones(n, 1, device="cuda")
        ops.embedding_backward(tokens, dy, 500)
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        for _ in range(5):
            out = ops.embedding_backward(tokens, dy, 500)
        b.record()
        b.synchronize()
        assert int(out.sum()) == n
        ms.append(a.elapsed_time(b))
    print("embedding gradient, ms of five", ms, flush=True)
    assert ms[1] < 6 * ms[0], ms


def test_embedding_gradient_ignores_what_has_none():
    g = torch.Generator().manual_seed(4)
    tokens = torch.randint(0, 50, (300,), generator=g)
    dy = m.normal(g, 300, 24, dtype=torch.float32)
    tokens[10:20], tokens[30:40] = 60, -1
    dy[10:20], dy[30:40] = float("nan"), float("inf")
    dy[tokens == 7] = float("nan")
    ref, mag = m.embedding_grad(tokens, dy.nan_to_num(0, 0, 0), 50, 1.0, 7)
    m.close(ops.embedding_backward(tokens.cuda(), dy.cuda(), 50, padding=7), ref, 304 * m.U32 * mag)
    # strided gradients and results
    wide = torch.randn(300, 40, device="cuda")
    out = torch.full((50, 32), 7.0, device="cuda")
    ops.embedding_backward(tokens.cuda(), wide[:, 3:27], 50, padding=7, out=out[:, 5:29])
    assert torch.equal(out[:, 5:29], ops.embedding_backward(tokens.cuda(), wide[:, 3:27].contiguous(), 50, padding=7))
    assert (out[:, :5] == 7).all() and (out[:, 29:] == 7).all()


# ---- residual norm ------------------------------------------------------------------

def seam(g, rows, cols, dtype, post, pre, gate, biases, weights=True, z=True):
    t = m.DTYPES[dtype]
    s = dict(x=m.normal(g, rows, cols, dtype=t, std=2.0),
             z=m.normal(g, rows, cols, dtype=t, std=0.7, mean=0.3) if z else None)
    how = dict(post=post, pre=pre, residual_scale=0.8, eps=1e-5,
               post_weight=m.normal(g, cols, dtype=t, std=0.2, mean=1.0) if weights and post != "none" else None,
               post_bias=m.normal(g, cols, dtype=t, std=0.2) if biases and post != "none" else None,
               gate=m.normal(g, gate, cols, dtype=t, std=0.5) if gate else None,
               pre_weight=m.normal(g, cols, dtype=t, std=0.2, mean=1.0) if weights and pre != "none" else None,
               pre_bias=m.normal(g, cols, dtype=t, std=0.2) if biases and pre != "none" else None)
    return s, how


def wide(t):
    return t.double() if torch.is_tensor(t) else t


def forward_slack(s, how):
    """Bounds on the 32-bit errors of y and h: every value is a few products
    and sums of rounded terms; sums over a row are trees of at most 32 + 10
    levels, so a mean and 1 / deviation are within 64 roundings."""
    x, z = wide(s["x"]), wide(s["z"])
    size = (how["residual_scale"] * x).abs()
    if z is not None:
        out, n, r = m.norm(how["post"], z, None, None, how["eps"])
        b = n.abs() + r * z.abs().mean(1, keepdim=True) if how["post"] != "none" else n.abs()
        if how["post_weight"] is not None:
            b = b * wide(how["post_weight"]).abs()
        if how["post_bias"] is not None:
            b = b + wide(how["post_bias"]).abs()
        if how["gate"] is not None:
            gt = wide(how["gate"])
            b = b * gt.abs().repeat_interleave(x.shape[0] // gt.shape[0], 0)
        size = size + b
    y_slack = 128 * m.U32 * size
    if how["pre"] == "none":
        return y_slack, None
    y = m.residual_norm(x, z, **{k: wide(v) for k, v in how.items()})[0]
    _, n, r = m.norm(how["pre"], y, None, None, how["eps"])
    h = 128 * m.U32 * (n.abs() + r * y.abs().mean(1, keepdim=True)) + r * (y_slack + y_slack.mean(1, keepdim=True)) + \
        n.abs() * (n.abs() * r * y_slack).mean(1, keepdim=True)
    if how["pre_weight"] is not None:
        h = h * wide(how["pre_weight"]).abs()
    if how["pre_bias"] is not None:
        h = h + 2 * m.U32 * wide(how["pre_bias"]).abs()
    return y_slack, h


def check_seam(s, how, dy, dh):
    gs, gh = {k: gpu(v) for k, v in s.items()}, {k: gpu(v) if torch.is_tensor(v) else v for k, v in how.items()}
    y, h, stats = ops.residual_norm(gs["x"], gs["z"], **gh)
    leaves = {k: wide(v).requires_grad_() for k, v in {**s, **how}.items() if torch.is_tensor(v)}
    ref_y, ref_h = m.residual_norm(leaves["x"], leaves.get("z"), **{k: leaves.get(k, v) for k, v in how.items()})
    ys, hs = forward_slack(s, how)
    m.close(y, ref_y.detach(), ys, "y")
    if ref_h is not None:
        m.close(h, ref_h.detach(), hs, "h")
    else:
        assert h is None
    again = ops.residual_norm(gs["x"], gs["z"], **gh, stats=False)
    assert torch.equal(again[0], y) and again[2] is None

    g = ops.residual_norm_backward(gpu(dy), gpu(dh) if ref_h is not None else None, y, gs["z"], stats, **gh)
    outs = [o for o, d in ((ref_y, dy), (ref_h, dh)) if o is not None and d is not None]
    gouts = [wide(d) for o, d in ((ref_y, dy), (ref_h, dh)) if o is not None and d is not None]
    names = [k for k in ("x", "z", "pre_weight", "pre_bias", "post_weight", "post_bias", "gate") if k in leaves]
    ref = dict(zip(names, torch.autograd.grad(outs, [leaves[k] for k in names], gouts)))
    assert set(g) == set(names)

    # The backward takes n of the pre norm from y as it was rounded (one
    # rounding of the type), everything else from 32-bit values.  Bounds: d*
    # is the error of *, each sum of products bounded term by term.
    x, z = wide(s["x"]), wide(s["z"])
    u = m.UNIT[y.dtype]
    yy = ref_y.detach()
    e = 256 * m.U32
    t = wide(dy).abs() if dy is not None else torch.zeros_like(x)
    dt = e * t
    if ref_h is not None:
        _, n2, r2 = m.norm(how["pre"], yy, None, None, how["eps"])
        c = wide(dh).abs() * (wide(how["pre_weight"]).abs() if how["pre_weight"] is not None else 1.0)
        dn2 = r2 * (u * (yy.abs() + ys) + ys + ys.mean(1, keepdim=True)) + e * (n2.abs() + r2 * yy.abs().mean(1, True)) + \
            n2.abs() * (n2.abs() * r2 * ys).mean(1, keepdim=True)
        du = r2 * (c + c.mean(1, True) + n2.abs() * (c * n2.abs()).mean(1, True))
        dt = dt + e * du + r2 * (dn2 * (c * n2.abs()).mean(1, True) + n2.abs() * (c * dn2).mean(1, True)) + \
            du * (n2.abs() * r2 * ys).mean(1, True)
        t = t + du
        if "pre_weight" in g:
            m.close(g["pre_weight"], ref["pre_weight"],
                    (wide(dh).abs() * (dn2 + (2 * x.shape[0] + 64) * m.U32 * n2.abs())).sum(0), "pre_weight")
        if "pre_bias" in g:
            m.close(g["pre_bias"], ref["pre_bias"], (x.shape[0] + 64) * m.U32 * wide(dh).abs().sum(0), "pre_bias")
    m.close(g["x"], ref["x"], how["residual_scale"] * dt + e * ref["x"].abs(), "x")
    if z is None:
        return
    gt = wide(how["gate"]).abs().repeat_interleave(x.shape[0] // how["gate"].shape[0], 0) if how["gate"] is not None \
        else torch.ones_like(x)
    w1 = wide(how["post_weight"]).abs() if how["post_weight"] is not None else 1.0
    b1 = wide(how["post_bias"]).abs() if how["post_bias"] is not None else 0.0
    _, n1, r1 = m.norm(how["post"], z, None, None, how["eps"])
    n1, dn1 = n1.abs(), e * (n1.abs() + (r1 * z.abs().mean(1, True) if how["post"] != "none" else 0.0))
    db, ddb = gt * t, gt * (dt + e * t)
    rows_e = (2 * x.shape[0] + 64) * m.U32
    if how["post"] == "none":
        dz_slack = ddb
    else:
        c, dc = db * w1, (ddb + e * db) * w1
        dz_slack = r1 * (dc + dc.mean(1, True) + n1 * (dc * n1 + c * dn1).mean(1, True) +
                         dn1 * (c * n1).mean(1, True)) + \
            e * r1 * (c + c.mean(1, True) + n1 * (c * n1).mean(1, True))
    m.close(g["z"], ref["z"], dz_slack, "z")
    if "post_weight" in g:
        m.close(g["post_weight"], ref["post_weight"], (ddb * n1 + db * dn1 + rows_e * db * n1).sum(0), "post_weight")
    if "post_bias" in g:
        m.close(g["post_bias"], ref["post_bias"], (ddb + rows_e * db).sum(0), "post_bias")
    if "gate" in g:
        b = n1 * w1 + b1
        part = (dt * b + t * dn1 * w1 + rows_e * t * b).reshape(how["gate"].shape[0], -1, x.shape[1]).sum(1)
        m.close(g["gate"], ref["gate"], part, "gate")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 5), (2, 8), (5, 63), (4, 512), (6, 515), (33, 1024), (4, 1025),
                                       (8, 2048), (4, 2055), (2, 4099), (3, 8200), (2, 16384)])
def test_residual_norm_sizes(dtype, rows, cols):
    print("residual norm", dtype, rows, cols, flush=True)
    g = torch.Generator().manual_seed(rows * cols)
    s, how = seam(g, rows, cols, dtype, "rms", "layer", 1, True)
    check_seam(s, how, m.normal(g, rows, cols, dtype=m.DTYPES[dtype]), m.normal(g, rows, cols, dtype=m.DTYPES[dtype]))


@pytest.mark.parametrize("post,pre", list(itertools.product(["none", "rms", "layer"], repeat=2)))
@pytest.mark.parametrize("gate,biases,weights", [(0, False, True), (1, True, True), (4, True, False), (24, False, True)])
def test_residual_norm_forms(post, pre, gate, biases, weights):
    print("residual norm", post, pre, gate, biases, weights, flush=True)
    g = torch.Generator().manual_seed(7)
    s, how = seam(g, 24, 100, "f32", post, pre, gate, biases, weights)
    d = [m.normal(g, 24, 100, dtype=torch.float32) for _ in range(2)]
    check_seam(s, how, d[0], d[1])
    if pre != "none":
        check_seam(s, how, None, d[1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,gate", [(2100, 1), (2100, 3), (1400, 700), (3000, 0), (1536, 1536)])
def test_residual_norm_sums_over_many_rows(dtype, rows, gate):
    print("residual norm rows", dtype, rows, gate, flush=True)
    g = torch.Generator().manual_seed(rows)
    s, how = seam(g, rows, 72, dtype, "layer", "rms", gate, True)
    check_seam(s, how, m.normal(g, rows, 72, dtype=m.DTYPES[dtype]), m.normal(g, rows, 72, dtype=m.DTYPES[dtype]))


@pytest.mark.parametrize("dtype,rows,cols,post,pre,gate", [
    ("bf16", 1030, 4103, "rms", "layer", 0), ("f32", 600, 4104, "layer", "rms", 6), ("f16", 300, 8191, "none", "rms", 300),
    ("bf16", 70, 16383, "layer", "layer", 1), ("f32", 33, 8208, "none", "none", 3), ("f16", 530, 5120, "rms", "none", 2)])
def test_residual_norm_of_wide_rows(dtype, rows, cols, post, pre, gate):
    print("residual norm wide", dtype, rows, cols, post, pre, gate, flush=True)
    g = torch.Generator().manual_seed(rows + cols)
    s, how = seam(g, rows, cols, dtype, post, pre, gate, post != "none")
    dy, dh = (m.normal(g, rows, cols, dtype=m.DTYPES[dtype]) for _ in range(2))
    check_seam(s, how, dy, dh)
    if pre != "none":
        check_seam(s, how, None, dh)


def test_residual_norm_without_a_block():
    g = torch.Generator().manual_seed(3)
    s, how = seam(g, 9, 70, "bf16", "none", "rms", 0, False, z=False)
    how["residual_scale"] = 1.0
    x = gpu(s["x"])
    y, h, st = ops.residual_norm(x, pre="rms", pre_weight=gpu(how["pre_weight"]))
    assert y is x
    check_seam(s, how, None, m.normal(g, 9, 70, dtype=torch.bfloat16))
    how["residual_scale"] = 0.5
    check_seam(s, how, m.normal(g, 9, 70, dtype=torch.bfloat16), m.normal(g, 9, 70, dtype=torch.bfloat16))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_layer_norm_gradient_of_rows_far_from_zero(dtype):
    # y's rounding is larger than the rows' deviation: the gradient is that of
    # the norm at y as rounded.  Deviations there are 0 or a few spacings, so
    # sums over a row are exact up to 32-bit rounding of the mean (relative to
    # the mean, 2^-24 * 64 * 300, against spacings of 0.25 and more).
    g = torch.Generator().manual_seed(31)
    x = m.normal(g, 40, 65, std=0.02, mean=300.0).to(m.DTYPES[dtype])
    dh = m.normal(g, 40, 65, dtype=x.dtype)
    # a scale that makes y need rounding again
    how = dict(pre="layer", residual_scale=1.01, eps=1e-5)
    y, _, st = ops.residual_norm(x.cuda(), **how)
    leaf = y.cpu().double().requires_grad_()
    out, n, r = m.norm("layer", leaf, None, None, 1e-5)
    ref = torch.autograd.grad(out, leaf, dh.double())[0] * 1.01
    got = ops.residual_norm_backward(None, dh.cuda(), y, None, st, **how)["x"]
    n, r, c = n.detach().abs(), r.detach(), dh.double().abs()
    dn = r * 64 * m.U32 * 310 + 256 * m.U32 * n
    du = r * (c + c.mean(1, True) + n * (c * n).mean(1, True))
    m.close(got, ref, 1.01 * (256 * m.U32 * du + du * (n * dn).mean(1, True) +
                              r * (dn * (c * n).mean(1, True) + (n + dn) * (c * dn).mean(1, True))))


def test_residual_norm_of_strided_rows():
    g = torch.Generator().manual_seed(5)
    for cols in (64, 100, 2050):
        big = [m.normal(g, 12, cols + 9, dtype=torch.bfloat16).cuda()[:, 3:3 + cols] for _ in range(5)]
        x, z, gate, dy, dh = big
        gate = gate[:4]
        w = m.normal(g, cols, dtype=torch.bfloat16).cuda()
        how = dict(post="layer", post_weight=w, pre="rms", pre_weight=w)
        a = ops.residual_norm(x, z, gate=gate, **how)
        b = ops.residual_norm(x.contiguous(), z.contiguous(), gate=gate.contiguous(), **how)
        assert all(torch.equal(p, q) for p, q in zip(a, b))
        ga = ops.residual_norm_backward(dy, dh, a[0], z, a[2], gate=gate, **how)
        gb = ops.residual_norm_backward(dy.contiguous(), dh.contiguous(), a[0], z.contiguous(), a[2],
                                        gate=gate.contiguous(), **how)
        assert set(ga) == set(gb) and all(torch.equal(ga[k], gb[k]) for k in ga)


def test_residual_norm_gradient_against_differences():
    # L = sum(c y) + sum(d h): central differences along a random direction of
    # every argument at once.  Rounding of the values: 2^-24 of terms whose
    # magnitudes sum to S, over a step of 2 * 2^-6; curvature: below 2^-12 of
    # the third derivative's size, bounded with the 64-bit model's own
    # difference.
    g = torch.Generator().manual_seed(6)
    rows, cols, step = 16, 96, 2.0 ** -6
    s, how = seam(g, rows, cols, "f32", "layer", "rms", 4, True)
    tensors = {k: v for k, v in {**s, **how}.items() if torch.is_tensor(v)}
    fixed = {k: v for k, v in how.items() if not torch.is_tensor(v)}
    along = {k: m.normal(g, *v.shape, dtype=torch.float32) for k, v in tensors.items()}
    c, d = (m.normal(g, rows, cols, dtype=torch.float32) for _ in range(2))

    def value(e, f):
        t = {k: v + e * along[k] for k, v in tensors.items()}
        x, z = t.pop("x"), t.pop("z")
        y, h = f(x, z, t)
        return float((c.double() * y.cpu().double()).sum() + (d.double() * h.cpu().double()).sum()), \
            float((c.double() * y.cpu().double()).abs().sum() + (d.double() * h.cpu().double()).abs().sum())

    def kernel(x, z, t):
        return ops.residual_norm(x.cuda(), z.cuda(), **{k: v.cuda() for k, v in t.items()}, **fixed)[:2]

    def model(x, z, t):
        return m.residual_norm(x.double(), z.double(), **{k: v.double() for k, v in t.items()}, **fixed)

    y, h, st = kernel_out = ops.residual_norm(s["x"].cuda(), s["z"].cuda(), **{k: gpu(v) if torch.is_tensor(v) else v
                                                                               for k, v in how.items()})
    grads = ops.residual_norm_backward(c.cuda(), d.cuda(), y, s["z"].cuda(), st,
                                       **{k: gpu(v) if torch.is_tensor(v) else v for k, v in how.items()})
    analytic = sum(float((grads[k].cpu().double() * along[k].double()).sum()) for k in tensors)
    size = sum(float((grads[k].cpu().double() * along[k].double()).abs().sum()) for k in tensors)
    (up, mag), (down, _) = value(step, kernel), value(-step, kernel)
    numeric = (up - down) / (2 * step)
    exact = (value(step, model)[0] - value(-step, model)[0]) / (2 * step)
    tiny = (value(step / 64, model)[0] - value(-step / 64, model)[0]) / (2 * step / 64)
    curvature = abs(exact - tiny)
    assert abs(numeric - analytic) <= curvature * 1.1 + 256 * m.U32 * (mag / step + size)


def test_operators_run_on_the_stream_they_are_given():
    g = torch.Generator().manual_seed(8)
    x = m.normal(g, 512, 1024, dtype=torch.float32).cuda()
    tokens = torch.randint(0, 100, (512,), generator=g).cuda()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    a = ops.dropout(x, 0.2, 1, stream=side)
    b = ops.embedding_backward(tokens, x, 100, stream=side)
    c = ops.residual_norm(x, x, pre="rms", stream=side)[1]
    with torch.cuda.stream(side):
        d = ops.dropout(x, 0.2, 1)
    side.synchronize()
    assert torch.equal(a, ops.dropout(x, 0.2, 1)) and torch.equal(a, d)
    assert torch.equal(b, ops.embedding_backward(tokens, x, 100))
    assert torch.equal(c, ops.residual_norm(x, x, pre="rms")[1])


def test_the_binding_refuses_mismatched_tensors():
    x = torch.zeros(4, 8, device="cuda")
    t = torch.zeros(4, dtype=torch.int64, device="cuda")
    bad = [lambda: ops.dropout(x.double(), 0.1, 1), lambda: ops.dropout(x, 1.5, 1),
           lambda: ops.dropout(x, 0.1, 1, residual=x[:2]), lambda: ops.dropout(x, 0.1, 1, residual=x.half()),
           lambda: ops.dropout(x.t(), 0.1, 1), lambda: ops.dropout(x, 0.1, 1, out=x[:2]),
           lambda: ops.dropout(x, 0.1, 1, step_tensor=t), lambda: ops.embedding(t.float(), x),
           lambda: ops.embedding(t.cpu(), x), lambda: ops.embedding(t, x[0]),
           lambda: ops.embedding_backward(t, x[:2], 4), lambda: ops.embedding_backward(t, x, 4, out=x[:, :4]),
           lambda: ops.residual_norm(x, pre="batch"), lambda: ops.residual_norm(x, x[:2]),
           lambda: ops.residual_norm(x, x, gate=x[:3]), lambda: ops.residual_norm(x, gate=x),
           lambda: ops.residual_norm(x, x, post_weight=x[0]), lambda: ops.residual_norm(x, pre="rms", eps=-1.0),
           lambda: ops.residual_norm(x, pre="rms", pre_weight=x[0].half()),
           lambda: ops.residual_norm(torch.zeros(2, 16385, device="cuda"), pre="rms"),
           lambda: ops.residual_norm_backward(x, None, x, x, x, pre="rms"),
           lambda: ops.residual_norm_backward(x, x, x, x, x, pre="rms"),
           lambda: ops.residual_norm_backward(None, None, x, x, x)]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print("not refused:", k)


# ---- cross entropy ---------------------------------------------------------------------

def xent_case(n, rows, cols, dtype, seed=0, scale=1.0, ignored=0.3):
    g = torch.Generator().manual_seed(seed + n + rows + cols)
    h = m.normal(g, n, cols, dtype=m.DTYPES[dtype])
    w = m.normal(g, rows, cols, dtype=m.DTYPES[dtype], std=scale / cols ** 0.5)
    t = torch.randint(0, rows, (n,), generator=g)
    t[torch.rand(n, generator=g) < ignored] = -100
    return h, w, t, m.normal(g, n, dtype=torch.float32)


def check_xent(h, w, t, gl, ignore=-100):
    """Bounds.  A logit is a sum of `cols` products: 32-bit sums of exact
    products (three-term products of 32-bit tensors are within 2^-22 of each
    product), so it is within s = (cols + 32) 2^-24 of the sum of its terms'
    magnitudes A, plus 2^-22 A for 32-bit tensors.  lse and loss are within
    that of the largest A plus the exponentials' and logarithm's few
    roundings.  P is within its relative error (the logit's and lse's absolute
    ones, and one rounding to 16 bits, or 2^-23) of |softmax| + |target|
    times the gradient; dh and dw sum such terms in 32 bits."""
    gh, gw, gt, ggl = (x.cuda() for x in (h, w, t, gl))
    loss, lse = ops.linear_cross_entropy(gh, gw, gt, ignore)
    ref_loss, ref_lse = m.cross_entropy(h, w, t, ignore)
    n, cols = h.shape
    rows = w.shape[0]
    a = h.double().abs() @ w.double().abs().t()
    s = ((cols + 32) * m.U32 + (2.0 ** -22 if h.dtype == torch.float32 else 0.0)) * a
    top = s.max(1).values
    slack = top + 32 * m.U32 * (1 + ref_lse.abs())
    m.close(lse, ref_lse, slack, "lse")
    m.close(loss, ref_loss, slack + top + 4 * m.U32 * a.max(1).values, "loss")
    dh, dw = ops.linear_cross_entropy_backward(gh, gw, gt, lse, ggl, ignore)
    p = m.cross_entropy_grad(h, w, t, gl, ignore)
    soft = torch.softmax(h.double() @ w.double().t(), 1)
    some = (t != ignore).double().unsqueeze(1)
    size = gl.double().abs().unsqueeze(1) * some
    unit = 2.0 ** -23 if h.dtype == torch.float32 else m.UNIT[h.dtype]
    dp = size * soft * (2 * s + 2 * slack.unsqueeze(1) + 64 * m.U32) * 1.1 + p.abs() * (unit + 8 * m.U32)
    if h.dtype == torch.float16:
        # P is scaled to a largest gradient of 2^11 at least: half a
        # subnormal's spacing below
        dp = dp + size.max() * 2.0 ** -36 * some
    pa = p.abs() + dp
    aw, ah = w.double().abs(), h.double().abs()
    three = 2.0 ** -22 if h.dtype == torch.float32 else 0.0
    m.close(dh, p @ w.double(), dp @ aw + ((rows + 64) * m.U32 + three) * (pa @ aw), "dh")
    m.close(dw, p.t() @ h.double(), dp.t() @ ah + ((n + 64) * m.U32 + three) * (pa.t() @ ah), "dw")
    return loss, lse, dh, dw


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,rows,cols", [(1, 1, 1), (1, 300, 64), (2, 3, 7), (5, 129, 8), (16, 1000, 40), (17, 255, 72),
                                         (33, 257, 65), (64, 513, 128), (65, 700, 136), (127, 128, 200),
                                         (130, 1025, 63), (257, 300, 264), (300, 2000, 512), (700, 600, 96)])
def test_cross_entropy(dtype, n, rows, cols):
    print("cross entropy", dtype, n, rows, cols, flush=True)
    check_xent(*xent_case(n, rows, cols, dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,rows,cols", [(1, 24700, 64), (16, 25001, 72), (33, 24600, 136), (64, 26000, 24)])
def test_cross_entropy_of_few_tokens_and_many_rows(dtype, n, rows, cols):
    print("cross entropy", dtype, n, rows, cols, flush=True)
    check_xent(*xent_case(n, rows, cols, dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,rows,cols,ignored", [(9000, 300, 70, 0.0), (3001, 130, 300, 0.1), (2500, 1000, 129, 0.9),
                                                 (1100, 7, 8, 0.5)])
def test_cross_entropy_of_many_tokens_and_few_rows(dtype, n, rows, cols, ignored):
    print("cross entropy", dtype, n, rows, cols, ignored, flush=True)
    check_xent(*xent_case(n, rows, cols, dtype, ignored=ignored))


@pytest.mark.parametrize("dtype", TYPES)
def test_cross_entropy_of_large_logits_and_certain_tokens(dtype):
    # logits of up to about 40: some softmaxes are one target, others ties
    h, w, t, gl = xent_case(96, 500, 64, dtype, scale=10.0)
    w[7] = w[9]
    check_xent(h, w, t, gl)
    t[:] = (h.double() @ w.double().t()).argmax(1)
    check_xent(h, w, t, gl)
    check_xent(h * 0, w, t, gl)


@pytest.mark.parametrize("dtype", TYPES)
def test_cross_entropy_without_targets(dtype):
    h, w, t, gl = xent_case(70, 300, 72, dtype, ignored=1.0)
    loss, _, dh, dw = check_xent(h, w, t, gl)
    assert not loss.any() and not dh.any() and not dw.any()
    # what such tokens hold does not matter, nor does the gradient of their loss
    h, w, t, gl = xent_case(70, 300, 72, dtype, ignored=0.4)
    some = t != -100
    h2, gl2 = h.clone(), gl.clone()
    bad = torch.nonzero(~some).squeeze(1)
    h2[bad[::2]], h2[bad[1::2]], gl2[bad] = float("nan"), float("inf"), float("nan")
    ref = check_xent(h, w, t, gl)
    out = ops.linear_cross_entropy(h2.cuda(), w.cuda(), t.cuda())
    assert torch.equal(out[0], ref[0])
    g2 = ops.linear_cross_entropy_backward(h2.cuda(), w.cuda(), t.cuda(), out[1], gl2.cuda())
    assert torch.equal(g2[0], ref[2]) and torch.equal(g2[1], ref[3])
    # another value may stand for "no target", one of the rows among them
    t3 = torch.where(some, t, 5)
    ref3 = check_xent(h, w, t3, gl, ignore=5)
    assert not ref3[0][(t3 == 5).cuda()].any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,count", [(65, 1), (300, 8), (300, 64), (300, 256), (520, 257), (1100, 1025), (2100, 2048)])
def test_cross_entropy_of_few_tokens_that_count(dtype, n, count):
    # the backward works on those with a gradient alone: in one run, spread
    # out, and among targets whose loss has no gradient
    h, w, t, gl = xent_case(n, 270, 72, dtype, ignored=0.0)
    for k, some in enumerate((torch.arange(n) >= n - count, torch.arange(n) < count,
                              torch.argsort(torch.rand(n, generator=torch.Generator().manual_seed(n))) < count)):
        print("cross entropy tokens that count", dtype, n, count, k, flush=True)
        out = check_xent(h, w, torch.where(some, t, -100), gl)
        assert not out[2][~some.cuda()].any()
        again = ops.linear_cross_entropy_backward(h.cuda(), w.cuda(), t.cuda(), out[1], torch.where(some, gl, 0.0).cuda())
        assert torch.equal(again[0], out[2]) and torch.equal(again[1], out[3])


def test_cross_entropy_of_many_tokens_with_a_target_outside_the_vocabulary():
    h, w, t, gl = xent_case(150, 290, 72, "bf16")
    t[3], t[148] = 290, -7
    loss, lse = ops.linear_cross_entropy(h.cuda(), w.cuda(), t.cuda())
    assert loss.cpu().isnan().nonzero().squeeze(1).tolist() == [3, 148]
    dh, dw = ops.linear_cross_entropy_backward(h.cuda(), w.cuda(), t.cuda(), lse, gl.cuda())
    assert dh.cpu().isnan().all(1).nonzero().squeeze(1).tolist() == [3, 148] and dw.isnan().all()


def test_cross_entropy_of_targets_outside_the_vocabulary_is_nan():
    h, w, t, gl = xent_case(20, 50, 16, "f32", ignored=0.0)
    t[3], t[8] = 50, -7
    loss, lse = ops.linear_cross_entropy(h.cuda(), w.cuda(), t.cuda())
    assert loss.cpu().isnan().nonzero().squeeze(1).tolist() == [3, 8]
    dh, dw = ops.linear_cross_entropy_backward(h.cuda(), w.cuda(), t.cuda(), lse, gl.cuda())
    assert dh.cpu().isnan().all(1).nonzero().squeeze(1).tolist() == [3, 8] and dw.isnan().all()


@pytest.mark.parametrize("dtype", TYPES)
def test_cross_entropy_of_strided_and_unaligned_rows(dtype):
    for cols, off, pitch in [(64, 0, 72), (64, 1, 80), (56, 3, 61), (33, 0, 33)]:
        print("cross entropy strides", dtype, cols, off, pitch, flush=True)
        h, w, t, gl = xent_case(40, 290, cols, dtype, seed=off)
        ref = check_xent(h, w, t, gl)
        gh, gw = torch.zeros(40, pitch, dtype=h.dtype), torch.zeros(290, pitch, dtype=h.dtype)
        gh[:, off:off + cols], gw[:, off:off + cols] = h, w
        gh, gw = gh.cuda()[:, off:off + cols], gw.cuda()[:, off:off + cols]
        loss, lse = ops.linear_cross_entropy(gh, gw, t.cuda())
        dh, dw = ops.linear_cross_entropy_backward(gh, gw, t.cuda(), lse, gl.cuda())
        for a, b in zip((loss, lse, dh, dw), ref):
            assert torch.equal(a, b)
        only = ops.linear_cross_entropy_backward(gh, gw, t.cuda(), lse, gl.cuda(), need_w=False)
        assert only[1] is None and torch.equal(only[0], ref[2])
        only = ops.linear_cross_entropy_backward(gh, gw, t.cuda(), lse, gl.cuda(), need_h=False)
        assert only[0] is None and torch.equal(only[1], ref[3])


def test_cross_entropy_leading_dimensions_and_no_tokens():
    h, w, t, gl = xent_case(24, 100, 32, "bf16")
    a = ops.linear_cross_entropy(h.cuda(), w.cuda(), t.cuda())
    b = ops.linear_cross_entropy(h.view(4, 6, 32).cuda(), w.cuda(), t.view(4, 6).cuda())
    assert b[0].shape == (4, 6) and torch.equal(a[0], b[0].view(-1))
    none = torch.zeros(0, dtype=torch.int64, device="cuda")
    loss, lse = ops.linear_cross_entropy(h[:0].cuda(), w.cuda(), none)
    dh, dw = ops.linear_cross_entropy_backward(h[:0].cuda(), w.cuda(), none, lse, loss)
    assert loss.shape == (0,) and dh.shape == (0, 32) and torch.equal(dw, torch.zeros_like(w).cuda())


def test_cross_entropy_gradient_against_differences():
    # sum of c * loss along a random direction of h and w: central difference
    # of the 32-bit losses (rounding 2^-24 of the sum's terms over the step),
    # its curvature taken from the 64-bit model
    h, w, t, c = xent_case(48, 333, 40, "f32")
    g = torch.Generator().manual_seed(12)
    vh, vw = m.normal(g, *h.shape, dtype=torch.float32), m.normal(g, *w.shape, dtype=torch.float32, std=0.1)
    step = 2.0 ** -7

    def value(e, f):
        loss = f(h + e * vh, w + e * vw)
        return float((c.double() * loss.cpu().double()).sum()), float((c.double() * loss.cpu().double()).abs().sum())

    def kernel(h, w):
        return ops.linear_cross_entropy(h.cuda(), w.cuda(), t.cuda())[0]

    def model(h, w):
        return m.cross_entropy(h, w, t, -100)[0]

    lse = ops.linear_cross_entropy(h.cuda(), w.cuda(), t.cuda())[1]
    dh, dw = (x.cpu().double() for x in ops.linear_cross_entropy_backward(h.cuda(), w.cuda(), t.cuda(), lse, c.cuda()))
    analytic = float((dh * vh).sum() + (dw * vw).sum())
    size = float((dh * vh).abs().sum() + (dw * vw).abs().sum())
    (up, mag), (down, _) = value(step, kernel), value(-step, kernel)
    exact = (value(step, model)[0] - value(-step, model)[0]) / (2 * step)
    tiny = (value(step / 64, model)[0] - value(-step / 64, model)[0]) / (2 * step / 64)
    numeric = (up - down) / (2 * step)
    assert abs(numeric - analytic) <= 1.1 * abs(exact - tiny) + 256 * m.U32 * (mag / step + size)


def test_the_cross_entropy_binding_refuses_mismatched_tensors():
    h, w = torch.zeros(4, 8, device="cuda"), torch.zeros(5, 8, device="cuda")
    t = torch.zeros(4, dtype=torch.int64, device="cuda")
    x = torch.zeros(4, device="cuda")
    f, b = ops.linear_cross_entropy, ops.linear_cross_entropy_backward
    for call in (lambda: f(h, w[:, :4], t), lambda: f(h, w.half(), t), lambda: f(h, w, t.int()),
                 lambda: f(h, w, t[:3]), lambda: f(h, w, t.cpu()), lambda: f(h.t(), w, t),
                 lambda: b(h, w, t, x.half(), x), lambda: b(h, w, t, x, x[:3]), lambda: b(h, w, t, x, x.cpu())):
        with pytest.raises(ValueError):
            call()
    assert b(h, w, t, x, x, need_h=False, need_w=False) == (None, None)


@pytest.mark.parametrize("dtype,n,rows,cols", [("f32", 3, 700000, 8), ("bf16", 2, 2200000, 7), ("f16", 3, 1100000, 8)])
def test_cross_entropy_over_pieces_of_the_vocabulary(dtype, n, rows, cols):
    # few tokens and many rows: several pieces in the backward and, where
    # operands are copied, in the forward
    print("cross entropy pieces", dtype, n, rows, cols, flush=True)
    h, w, t, gl = xent_case(n, rows, cols, dtype, ignored=0.0)
    t[0], t[1] = rows - 1, 0
    check_xent(h, w, t, gl)


@pytest.mark.parametrize("dtype,n,rows,cols", [("bf16", 70, 70000, 1001), ("f32", 70, 25000, 1001),
                                               ("f32", 70, 360000, 8), ("f16", 2100, 33000, 8)])
def test_cross_entropy_of_many_tokens_over_pieces_of_the_vocabulary(dtype, n, rows, cols):
    # two pieces each: of copied rows of w (forward and backward), of P
    print("cross entropy pieces, many tokens", dtype, n, rows, cols, flush=True)
    h, w, t, gl = xent_case(n, rows, cols, dtype)
    t[0], t[1] = rows - 1, 0
    check_xent(h, w, t, gl)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 16, 17, 32, 33, 64])
def test_cross_entropy_of_few_tokens_over_many_rows(dtype, n):
    # enough rows for the waves to take rows of their own (64 or 128 a
    # workgroup, 512 workgroups), an odd number of them
    rows = 32801 if n <= 16 else 65601
    print("cross entropy few tokens", dtype, n, rows, flush=True)
    h, w, t, gl = xent_case(n, rows, 40, dtype, ignored=0.2)
    check_xent(h, w, t, gl)


def test_a_call_on_a_stream_keeps_off_blocks_that_another_one_still_uses():
    # Blocks of the sizes that the call will ask for, written and read by work
    # that waits on the current stream when they are freed: the call runs
    # beside that work and may not be given them.
    g = torch.Generator().manual_seed(9)
    x, z = (m.normal(g, 768, 1024, dtype=torch.bfloat16).cuda() for _ in range(2))
    w = m.normal(g, 1000, 1024, dtype=torch.bfloat16, std=0.03).cuda()
    t = torch.randint(0, 1000, (768,), generator=g).cuda()
    _, lse = ops.linear_cross_entropy(x, w, t)
    y, _, stats = ops.residual_norm(x, z, pre="layer")
    dl = torch.ones(768, device="cuda")
    n = ops._norm(x, z, "none", None, None, None, 1.0, "layer", None, None, 1e-5)
    need = ctypes.c_uint64()
    ops.rotor.lib().rotor_residual_norm_workspace_bytes(ctypes.byref(n), ctypes.byref(need))
    calls = [(lambda **kw: ops.dropout(x, 0.2, 1, **kw), 0),
             (lambda **kw: ops.embedding_backward(t, x, 1000, **kw),
              ops._workspace_bytes("rotor_embedding_workspace_bytes", 768, 1000, 1024)),
             (lambda **kw: ops.residual_norm_backward(x, z, y, z, stats, pre="layer", **kw), need.value),
             (lambda **kw: ops.linear_cross_entropy_backward(x, w, t, lse, dl, **kw),
              ops._workspace_bytes("rotor_xent_workspace_bytes", 1, 768, 1024, 1000, 1, 1))]
    side = torch.cuda.Stream()
    for k, (call, scratch) in enumerate(calls):
        print("streams", k, flush=True)
        want = tensors_of(call())
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        torch.cuda._sleep(50_000_000)
        busy = [torch.full((v.numel() * v.element_size(),), 3, dtype=torch.uint8, device="cuda") for v in want]
        if scratch:
            busy.append(torch.full((scratch,), 3, dtype=torch.uint8, device="cuda"))
        kept = [b.clone() for b in busy]
        del busy
        out = tensors_of(call(stream=side))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        assert all((b == 3).all() for b in kept)


def tensors_of(out):
    return list(out.values()) if isinstance(out, dict) else list(out) if isinstance(out, tuple) else [out]


# ---- more workgroups than a grid holds along one index -----------------------------

def test_dropout_of_more_elements_than_one_grid_index_holds():
    n = 2 ** 35 + 4099
    if torch.cuda.mem_get_info()[0] < 2 * n + (8 << 30):
        pytest.skip("needs 72 GiB")
    print("dropout", n, flush=True)
    x = torch.ones(n, dtype=torch.float16, device="cuda")
    assert ops.dropout(x, 0.5, 2 ** 40 + 3, 8, out=x) is x
    for first in (0, 2 ** 34 - 64, 2 ** 35 - 4096, n - n % 8 - 64):
        have = x[first:first + 4096].cpu()
        keep = [word >> (16 * half) & 0xFFFF
                for g in range(first // 8, -(-(first + have.numel()) // 8))
                for word in m.philox((g & 0xFFFFFFFF, g >> 32, 8, 0), (3, 2 ** 8)) for half in range(2)]
        keep = torch.tensor(keep[:have.numel()]) >= 2 ** 15
        assert torch.equal(have, torch.where(keep, 2.0, 0.0).half()), first
    # every element was reached: none is left at 1
    assert all(not (part == 1).any() for part in x.split(2 ** 31))


def test_residual_norm_of_more_rows_than_one_grid_index_holds():
    rows = 2 ** 26 + 5
    print("residual norm", rows, flush=True)
    x = torch.randn(rows, 2, device="cuda", dtype=torch.float16)
    _, h, _ = ops.residual_norm(x, pre="rms", stats=False)
    half = rows // 2
    for a, b in ((0, half), (half, rows)):
        assert torch.equal(h[a:b], ops.residual_norm(x[a:b], pre="rms", stats=False)[1])


def test_embedding_of_more_tokens_than_one_grid_index_holds():
    n = 2 ** 26 + 5
    print("embedding", n, flush=True)
    tokens = torch.randint(0, 50, (n,), device="cuda", dtype=torch.int32)
    table = torch.randn(50, 2, device="cuda", dtype=torch.float16)
    assert torch.equal(ops.embedding(tokens, table), table[tokens])


def test_embedding_gradient_of_more_tokens_than_one_grid_index_holds():
    n = 2 ** 29 + 77
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GiB")
    print("embedding gradient", n, flush=True)
    tokens = torch.randint(0, 500, (n,), device="cuda", dtype=torch.int32)
    tokens[:1000] = 499
    dy = torch.ones(n, 1, device="cuda")
    out = ops.embedding_backward(tokens, dy, 500)
    counts = sum(torch.bincount(part, minlength=500) for part in tokens.split(2 ** 27))
    assert torch.equal(out[:, 0].long(), counts) and int(counts.max()) < 2 ** 24


def test_cross_entropy_of_more_copies_than_one_grid_index_holds():
    # rows of an odd pitch are copied, eight columns a thread: 2^32 threads.
    # Seven kinds of rows; a logit is within 2^-24 a product of its terms'
    # magnitudes' sum, lse and loss within that and a few roundings.
    n, cols = 2 ** 19 + 9, 65535
    if torch.cuda.mem_get_info()[0] < 160 << 30:
        pytest.skip("needs 160 GiB")
    print("cross entropy copies", n, cols, flush=True)
    g = torch.Generator().manual_seed(2)
    kinds = m.normal(g, 7, cols, dtype=torch.bfloat16)
    w = m.normal(g, 3, cols, dtype=torch.bfloat16, std=2.0 ** -10)
    h = torch.empty(n, cols, dtype=torch.bfloat16, device="cuda")
    for k in range(7):
        h[k::7] = kinds[k].cuda()
    t = torch.arange(n, device="cuda") % 3
    loss, lse = ops.linear_cross_entropy(h, w.cuda(), t)
    ref_loss, ref_lse = m.cross_entropy(kinds.repeat(3, 1), w, torch.arange(21) % 3, -100)
    slack = (cols + 32) * m.U32 * float((kinds.double().abs() @ w.double().abs().t()).max()) + 2.0 ** -18
    for out, ref in ((lse, ref_lse), (loss, ref_loss)):
        m.close(out[:21], ref, 2 * slack)
        # the same row and target, the same bits
        assert torch.equal(out, out[:21].repeat(n // 21 + 1)[:n])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,rows,cols", [(3, 300, 64), (40, 700, 33), (64, 300, 64), (150, 700, 72), (150, 700, 71)])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_cross_entropy_of_tokens_without_a_target_over_a_row_that_is_not_finite(dtype, n, rows, cols, value):
    # what the others' gradients turn into does not reach a token without one
    h, w, t, gl = xent_case(n, rows, cols, dtype, ignored=0.4)
    t[0], t[1] = 5, -100
    w[rows // 2, cols // 3] = value
    gl[2] = 0.0
    loss, lse = ops.linear_cross_entropy(h.cuda(), w.cuda(), t.cuda())
    dh, _ = ops.linear_cross_entropy_backward(h.cuda(), w.cuda(), t.cuda(), lse, gl.cuda())
    none = (t == -100) | (gl == 0)
    assert not loss[(t == -100).cuda()].any()
    assert torch.equal(dh[none.cuda()], torch.zeros(int(none.sum()), cols, dtype=h.dtype, device="cuda"))
    assert dh[0].isnan().any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,rows,cols,ignored", xent_plan.CHECKED)
def test_cross_entropy_through_every_product(dtype, n, rows, cols, ignored):
    # each of the five products with large and with small tiles, over many
    # steps, odd and even numbers of them, several tiles a workgroup (which
    # sizes reach what is held in test_ops.py)
    print("cross entropy products", dtype, n, rows, cols, ignored, flush=True)
    h, w, t, gl = xent_case(n, rows, cols, dtype, ignored=0.0)
    t[torch.randperm(n, generator=torch.Generator().manual_seed(n))[:round(n * ignored)]] = -100
    check_xent(h, w, t, gl)


@pytest.mark.parametrize("n,rows,cols", [(24, 60000, 64), (24, 60000, 63), (40, 60000, 64), (300, 60000, 72)])
def test_cross_entropy_in_f16_of_tokens_with_small_gradients(n, rows, cols):
    # Losses weighted by 1 down to 2^-22, times a loss scale: a token's row of
    # dh is as exact relative to its own gradient, although P of 16 bits is
    # 2^-16 of that for most rows of w.  These have a part in common, which dh
    # loses if such terms vanish.
    print("cross entropy f16 weights", n, rows, cols, flush=True)
    h, w, t, _ = xent_case(n, rows, cols, "f16", ignored=0.0)
    w = (w.double() + m.normal(torch.Generator().manual_seed(1), cols, std=0.3)).half()
    h = (h.double() / 4).half()
    e = (torch.arange(n) * 5) % 23
    gl = 2.0 ** (12 - e.double()).float()
    loss, lse = ops.linear_cross_entropy(h.cuda(), w.cuda(), t.cuda())
    dh, dw = ops.linear_cross_entropy_backward(h.cuda(), w.cuda(), t.cuda(), lse, gl.cuda())
    # as in check_xent, but what P loses below the range of 16-bit floats: half
    # a subnormal's spacing, 2^-25, where the largest gradient is scaled to 2^15
    # and a smaller one by up to 2^8 more, to half of that at least
    p = m.cross_entropy_grad(h, w, t, gl, -100)
    soft = torch.softmax(h.double() @ w.double().t(), 1)
    a = h.double().abs() @ w.double().abs().t()
    s = (cols + 32) * m.U32 * a
    slack = s.max(1).values + 32 * m.U32 * (1 + m.cross_entropy(h, w, t, -100)[1].abs())
    lift = (e - 1).clamp(0, 8).double()
    dp = gl.double().unsqueeze(1) * soft * (2 * s + 2 * slack.unsqueeze(1) + 64 * m.U32) * 1.1 + \
        p.abs() * (m.UNIT[torch.float16] + 8 * m.U32) + (2.0 ** (12 - 40 - lift)).unsqueeze(1)
    aw, ah = w.double().abs(), h.double().abs()
    pa = p.abs() + dp
    m.close(dh, p @ w.double(), dp @ aw + (rows + 64) * m.U32 * (pa @ aw), "dh")
    # h is divided by what its gradient was multiplied by, in 16 bits
    dah = (2.0 ** (lift - 25)).unsqueeze(1).expand_as(ah)
    m.close(dw, p.t() @ h.double(), dp.t() @ ah + pa.t() @ dah + (n + 64) * m.U32 * (pa.t() @ ah), "dw")


def xent_bounds(h, w, t, gl):
    """Reference values and bounds of loss, lse, dh and dw, as in check_xent."""
    ref_loss, ref_lse = m.cross_entropy(h, w, t, -100)
    n, cols, rows = *h.shape, w.shape[0]
    a = h.double().abs() @ w.double().abs().t()
    three = 2.0 ** -22 if h.dtype == torch.float32 else 0.0
    s = ((cols + 32) * m.U32 + three) * a
    top = s.max(1).values
    slack = top + 32 * m.U32 * (1 + ref_lse.abs())
    p = m.cross_entropy_grad(h, w, t, gl, -100)
    some = (t != -100).double().unsqueeze(1)
    size = gl.double().abs().unsqueeze(1) * some
    unit = 2.0 ** -23 if h.dtype == torch.float32 else m.UNIT[h.dtype]
    soft = torch.softmax(h.double() @ w.double().t(), 1)
    dp = size * soft * (2 * s + 2 * slack.unsqueeze(1) + 64 * m.U32) * 1.1 + p.abs() * (unit + 8 * m.U32)
    if h.dtype == torch.float16:
        dp = dp + size.max() * 2.0 ** -36 * some
    pa, aw, ah = p.abs() + dp, w.double().abs(), h.double().abs()
    return (ref_loss, slack + top + 4 * m.U32 * a.max(1).values), (ref_lse, slack), \
        (p @ w.double(), dp @ aw + ((rows + 64) * m.U32 + three) * (pa @ aw)), \
        (p.t() @ h.double(), dp.t() @ ah + ((n + 64) * m.U32 + three) * (pa.t() @ ah))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,rows,cols", [(3, 400, 64), (20, 400, 63), (64, 400, 72), (150, 700, 72), (150, 700, 71),
                                         (1100, 9000, 136)])
@pytest.mark.parametrize("mask", ["inf", "lowest"])
def test_cross_entropy_of_rows_masked_by_a_bias(dtype, n, rows, cols, mask):
    # a column of ones in h, a bias in w: rows whose bias is minus infinity, or
    # the type's lowest value, are not there
    print("cross entropy masked rows", dtype, n, rows, cols, mask, flush=True)
    h, w, t, gl = xent_case(n, rows, cols, dtype, ignored=0.2)
    h[:, -1] = 1.0
    keep = torch.ones(rows, dtype=torch.bool)
    keep[torch.randperm(rows, generator=torch.Generator().manual_seed(3))[:rows // 3]] = False
    keep[0], keep[rows - 1] = True, False
    place = torch.cumsum(keep, 0) - 1
    t = torch.where((t != -100) & ~keep[t.clamp(min=0)], 0, t)
    masked = w.clone()
    masked[~keep, -1] = -float("inf") if mask == "inf" else torch.finfo(w.dtype).min
    loss, lse = ops.linear_cross_entropy(h.cuda(), masked.cuda(), t.cuda())
    dh, dw = ops.linear_cross_entropy_backward(h.cuda(), masked.cuda(), t.cuda(), lse, gl.cuda())
    want = xent_bounds(h, w[keep], torch.where(t == -100, t, place[t.clamp(min=0)]), gl)
    # the column of the bias is 0 times infinity in dh
    got = (loss, lse, dh[:, :-1], dw[keep.cuda()])
    for what, out, (ref, slack) in zip(("loss", "lse", "dh", "dw"), got, want):
        ref, slack = (ref[:, :-1], slack[:, :-1]) if what == "dh" else (ref, slack)
        m.close(out, ref, slack, what)
    assert not dw[~keep.cuda()].any()
    if mask == "lowest":
        m.close(dh[:, -1:], want[2][0][:, -1:], want[2][1][:, -1:], "dh of the bias")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_operators_in_a_captured_graph(dtype):
    # replays on new inputs, with eager calls and synchronizations between
    # them, give what eager calls give, bit for bit
    print("graph", dtype, flush=True)
    g = torch.Generator().manual_seed(77)
    t = m.DTYPES[dtype]
    x, z, dy, dh = (m.normal(g, 300, 96, dtype=t).cuda() for _ in range(4))
    w, gate = m.normal(g, 700, 96, dtype=t, std=0.1).cuda(), m.normal(g, 3, 96, dtype=t).cuda()
    tokens = torch.randint(0, 700, (300,), generator=g).cuda()
    many = torch.randint(0, 700, (40000,), generator=g).cuda()
    rows = m.normal(g, 40000, 9, dtype=t).cuda()
    few = x[:7].clone()
    gl = torch.ones(300, device="cuda")

    def step():
        how = dict(post="rms", gate=gate, pre="layer", pre_weight=w[0].contiguous())
        y, h, st = ops.residual_norm(x, z, **how)
        out = [y, h, *ops.residual_norm_backward(dy, dh, y, z, st, **how).values()]
        out += [ops.embedding(tokens, w, 2.0), ops.embedding_backward(tokens, dy, 700),
                ops.embedding_backward(many, rows, 700)]
        for a, n in ((h, 300), (few, 7)):
            loss, lse = ops.linear_cross_entropy(a, w, tokens[:n])
            out += [loss, *ops.linear_cross_entropy_backward(a, w, tokens[:n], lse, gl[:n])]
        return out

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(4):
        for a in (x, z, dy, dh, w, few, rows):
            a.copy_(m.normal(g, *a.shape, dtype=t, std=0.3 + k))
        for a in (tokens, many):
            a.copy_(torch.randint(0, 700, a.shape, generator=g))
        tokens[k::5] = -100 if k % 2 else 3
        graph.replay()
        torch.cuda.synchronize()
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0)) for a, b in zip(out, want)), k

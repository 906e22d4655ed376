"""Refusals of the operators of a chain's stages (no GPU): the C entry points
return ROTOR_EINVAL before any device work, the binding raises ValueError."""
import contextlib
import ctypes
import itertools

import pytest
import torch

import xent_plan
from paper_1911_13214_amd import ops, rotor

FAKE = 0x10000
E = rotor.ROTOR_EINVAL


def test_dropout_refuses_bad_arguments():
    f = rotor.lib().rotor_dropout
    good = [0, 4, 8, FAKE, 8, None, 0, FAKE, 8, 0.1, 1, 2, None, None]
    for at, bad in [(0, 3), (0, -1), (1, -1), (2, 0), (3, None), (3, FAKE + 2), (4, 7), (5, FAKE), (7, None),
                    (7, FAKE + 1), (8, 7), (9, -0.1), (9, 1.1), (9, float("nan")), (12, FAKE + 4), (1, 1 << 60)]:
        a = list(good)
        a[at] = bad
        assert f(*a) == E, (at, bad)
    a = list(good)
    a[1] = 0  # no rows: nothing to do, whatever the pointers
    a[3] = a[7] = None
    assert f(*a) == rotor.ROTOR_OK


def test_embedding_refuses_bad_arguments():
    f = rotor.lib().rotor_embedding
    good = [1, 4, 10, 8, FAKE, 8, FAKE, 8, 1.0, FAKE, 8, None]
    for at, bad in [(0, 9), (1, -1), (1, 1 << 31), (2, 0), (2, 1 << 31), (3, 0), (4, None), (4, FAKE + 4), (5, 2),
                    (6, None), (6, FAKE + 1), (7, 7), (9, None), (10, 7)]:
        a = list(good)
        a[at] = bad
        assert f(*a) == E, (at, bad)
    b = rotor.lib().rotor_embedding_backward
    need = ctypes.c_uint64()
    assert rotor.lib().rotor_embedding_workspace_bytes(4, 10, 8, ctypes.byref(need)) == rotor.ROTOR_OK
    good = [1, 4, 10, 8, FAKE, 8, FAKE, 8, 1.0, -1, FAKE, 8, FAKE, need.value, None]
    for at, bad in [(0, 9), (1, -1), (2, 0), (3, 0), (4, None), (5, 3), (6, None), (7, 7), (9, -2), (9, 10),
                    (10, None), (11, 7), (12, None), (12, FAKE + 8), (13, need.value - 1)]:
        a = list(good)
        a[at] = bad
        assert b(*a) == E, (at, bad)
    w = rotor.lib().rotor_embedding_workspace_bytes
    assert w(-1, 10, 8, ctypes.byref(need)) == E and w(4, 10, 8, None) == E


def test_residual_norm_refuses_bad_arguments():
    lib = rotor.lib()
    base = dict(type=1, post=1, pre=2, rows=4, cols=8, gate_rows=2, gate_pitch=8, residual_scale=1.0, eps=1e-5,
                gate=FAKE)
    grads = ops._NormGrads(gate_pitch=8)
    need = ctypes.c_uint64()

    def fwd(how, x=FAKE, z=FAKE, y=FAKE, h=FAKE, stats=FAKE, zp=8):
        n = ops._Norm(**{**base, **how})
        return lib.rotor_residual_norm(ctypes.byref(n), x, 8, z, zp, y, 8, h, 8, stats, None)

    def bwd(how, dy=FAKE, dh=FAKE, y=FAKE, z=FAKE, stats=FAKE, dx=FAKE, dz=FAKE, g=grads, work=FAKE, less=0):
        n = ops._Norm(**{**base, **how})
        lib.rotor_residual_norm_workspace_bytes(ctypes.byref(n), ctypes.byref(need))
        return lib.rotor_residual_norm_backward(ctypes.byref(n), dy, 8, dh, 8, y, 8, z, 8, stats, dx, 8, dz, 8,
                                                ctypes.byref(g), work, need.value - less, None)

    for how in [dict(type=3), dict(post=3), dict(pre=-1), dict(rows=-1), dict(cols=0), dict(cols=16385),
                dict(gate_rows=3), dict(gate_rows=-1), dict(gate=None), dict(gate_pitch=7), dict(eps=-1.0),
                dict(post_weight=FAKE + 1), dict(post=0, post_weight=FAKE), dict(pre=0, pre_bias=FAKE)]:
        assert fwd(how) == E, how
        assert bwd(how) == E, how
    for kw in [dict(x=None), dict(x=FAKE + 1), dict(z=None), dict(zp=7), dict(y=None), dict(h=None),
               dict(stats=FAKE + 4)]:
        assert fwd({}, **kw) == E, kw
    assert fwd(dict(pre=0)) == E  # h without pre
    assert fwd(dict(post=0, gate_rows=0, gate=None, residual_scale=0.5), z=None, y=None) == E
    for kw in [dict(dh=None), dict(y=None), dict(z=None), dict(stats=None), dict(stats=FAKE + 8), dict(dx=None),
               dict(dz=None), dict(work=None), dict(work=FAKE + 4), dict(less=1)]:
        assert bwd({}, **kw) == E, kw
    assert bwd(dict(pre=0), dy=None, dh=None) == E
    assert bwd(dict(gate_rows=0, gate=None), g=ops._NormGrads(gate_pitch=8, gate=FAKE)) == E
    assert bwd({}, g=ops._NormGrads(gate_pitch=7, gate=FAKE)) == E


def test_the_binding_refuses_what_is_not_on_a_gpu():
    x = torch.zeros(2, 4)
    for call in (lambda: ops.dropout(x, 0.1, 1), lambda: ops.embedding(torch.zeros(2, dtype=torch.int64), x),
                 lambda: ops.embedding_backward(torch.zeros(2, dtype=torch.int64), x, 3),
                 lambda: ops.residual_norm(x, pre="rms"),
                 lambda: ops.residual_norm_backward(x, None, None, None, x),
                 lambda: ops.dropout([1.0], 0.1, 1)):
        with pytest.raises(ValueError, match="CUDA"):
            call()


def test_matrices_are_described_by_their_row_pitch():
    x = torch.zeros(6, 10)
    assert ops._matrix(x, "x") == (6, 10, 10)
    assert ops._matrix(x[:, :7], "x") == (6, 7, 10)
    assert ops._matrix(x[::2], "x") == (3, 10, 20)
    assert ops._matrix(x.view(2, 3, 10)[:, :, 2:5], "x") == (6, 3, 10)
    assert ops._matrix(x[0], "x") == (1, 10, 10)
    assert ops._matrix(x[:1, :7], "x") == (1, 7, 7)
    for bad in (x.t(), x[:, ::2], x.view(2, 3, 10)[:, :2], x[0].expand(6, 10), torch.zeros(()), torch.zeros(3, 0)):
        with pytest.raises(ValueError):
            ops._matrix(bad, "x")


def test_cross_entropy_refuses_bad_arguments():
    lib = rotor.lib()
    need = ctypes.c_uint64()

    def bytes_of(*a):
        return lib.rotor_xent_workspace_bytes(*a, ctypes.byref(need))

    for bad in [(5, 4, 8, 10, 1, 0), (1, -1, 8, 10, 1, 0), (1, (1 << 20) + 1, 8, 10, 1, 0), (1, 4, 0, 10, 1, 0),
                (1, 4, 65537, 10, 1, 1), (1, 4, 8, 0, 1, 1), (1, 4, 8, (1 << 26) + 1, 1, 1)]:
        assert bytes_of(*bad) == E, bad
    assert lib.rotor_xent_workspace_bytes(1, 4, 8, 10, 1, 0, None) == E
    assert bytes_of(1, 0, 8, 10, 1, 1) == rotor.ROTOR_OK and need.value == 0  # no tokens
    assert bytes_of(1, 4, 8, 10, 1, 0) == rotor.ROTOR_OK
    good = [1, 4, 8, 10, FAKE, 8, FAKE, 8, FAKE, -100, FAKE, FAKE, 1, FAKE, need.value, None]
    for at, bad in [(0, 5), (1, -1), (2, 0), (3, 0), (4, None), (4, FAKE + 8), (5, 7), (5, 12), (6, None), (6, FAKE + 2),
                    (7, 7), (7, (1 << 22) + 8), (8, None), (8, FAKE + 4), (10, None), (10, FAKE + 2), (11, None),
                    (13, None), (13, FAKE + 8), (14, need.value - 1)]:
        a = list(good)
        a[at] = bad
        assert lib.rotor_xent(*a) == E, (at, bad)
    assert bytes_of(1, 4, 8, 10, 1, 1) == rotor.ROTOR_OK
    good = [1, 4, 8, 10, FAKE, 8, FAKE, 8, FAKE, -100, FAKE, FAKE, FAKE, 8, FAKE, 8, 1, FAKE, need.value, None]
    for at, bad in [(0, 5), (1, -1), (2, 0), (3, 0), (4, None), (5, 7), (5, 12), (6, FAKE + 8), (7, 7), (8, None),
                    (10, None), (11, None), (12, FAKE + 1), (13, 7), (14, FAKE + 1), (15, 7), (15, (1 << 22) + 8),
                    (17, None), (18, need.value - 1)]:
        a = list(good)
        a[at] = bad
        assert lib.rotor_xent_backward(*a) == E, (at, bad)
    a = list(good)
    a[12] = a[14] = None  # no gradient wanted
    assert lib.rotor_xent_backward(*a) == E
    x = torch.zeros(2, 4)
    with pytest.raises(ValueError, match="CUDA"):
        ops.linear_cross_entropy(x, x, torch.zeros(2, dtype=torch.int64))


def test_cross_entropy_workspace_does_not_grow_with_the_logits():
    need = ctypes.c_uint64()
    # 2^20 tokens of 262144 rows would be 512 GiB of 16-bit logits
    for n, v in [(8192, 128000), (8192, 1 << 20), (65536, 262144), (1 << 20, 262144)]:
        assert rotor.lib().rotor_xent_workspace_bytes(1, n, 1024, v, 1, 1, ctypes.byref(need)) == rotor.ROTOR_OK
        piece = max(512 << 20, 4 * 256 * n)
        assert need.value < piece * 2 + 16 * n * 1024, (n, v, need.value)


def test_a_call_allocates_on_the_stream_it_is_given(monkeypatch):
    # Its results and scratch are written on that stream: blocks of another
    # one's pool may still be in use there.  Allocations are watched, kernels
    # and streams replaced.
    class Stream:
        device = torch.device("cpu")
        cuda_stream = 7

    now, seen, recorded = ["current"], [], []

    @contextlib.contextmanager
    def on(stream):
        before, now[0] = now[0], stream
        yield
        now[0] = before

    def watch(f):
        def alloc(*args, **kw):
            seen.append(now[0])
            return f(*args, **kw)
        return alloc

    given = Stream()
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now[0])
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, stream: recorded.append(stream))
    monkeypatch.setattr(torch.Tensor, "new_empty", watch(torch.Tensor.new_empty))
    monkeypatch.setattr(torch, "empty_like", watch(torch.empty_like))
    monkeypatch.setattr(ops, "_cuda", lambda t, what: t)
    monkeypatch.setattr(ops, "_call", lambda *args: None)
    x, t = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    stats, per = torch.zeros(4, 4), torch.zeros(4)
    calls = [lambda **kw: ops.dropout(x, 0.1, 1, **kw), lambda **kw: ops.embedding(t, x, **kw),
             lambda **kw: ops.embedding_backward(t, x, 9, **kw),
             lambda **kw: ops.residual_norm(x, x, pre="rms", **kw),
             lambda **kw: ops.residual_norm_backward(x, x, x, x, stats, pre="rms", **kw),
             lambda **kw: ops.linear_cross_entropy(x, x, t, **kw),
             lambda **kw: ops.linear_cross_entropy_backward(x, x, t, per, per, **kw)]
    for k, call in enumerate(calls):
        for kw, want in (({}, "current"), ({"stream": given}, given)):
            seen.clear()
            recorded.clear()
            call(**kw)
            assert seen and all(s is want for s in seen), (k, want, seen)
            # what is returned may be used and freed where the caller works
            assert ("current" in recorded) == bool(kw), (k, recorded)
    with pytest.raises(ValueError, match="stream"):
        given.device = torch.device("meta")
        calls[0](stream=given)


def test_more_workgroups_than_a_grid_holds_are_refused():
    # 2^20 along one index and 65535 along another
    f = rotor.lib().rotor_dropout
    per = 2048  # elements of a workgroup
    rows = (1 << 20) * 65535 * per // 8 + 1
    assert f(1, rows, 8, FAKE, 8, None, 0, FAKE, 8, 0.1, 1, 2, None, None) == E
    need = ctypes.c_uint64()
    assert rotor.lib().rotor_embedding_workspace_bytes(4, 10, 33553921, ctypes.byref(need)) == rotor.ROTOR_OK
    assert rotor.lib().rotor_embedding_backward(1, 4, 10, 33553921, FAKE, 8, FAKE, 33553921, 1.0, -1, FAKE, 33553921,
                                                FAKE, need.value, None) == E


def test_the_cross_entropys_plan_in_python_is_the_librarys():
    need = ctypes.c_uint64()
    sizes = [1, 3, 17, 33, 64, 65, 300, 2100, 9000, 70001], [1, 8, 63, 300, 1031, 4096, 65536], [1, 300, 24700, 128000]
    for type, n, d, v, aligned in itertools.product(range(3), *sizes, (0, 1)):
        for backward, plan in ((0, xent_plan.forward), (1, xent_plan.backward)):
            assert rotor.lib().rotor_xent_workspace_bytes(type, n, d, v, aligned, backward, ctypes.byref(need)) == 0
            assert plan(type, n, d, v, aligned)[0] == need.value, (type, n, d, v, aligned, backward)


def test_checked_cross_entropies_reach_every_product():
    # every product with both tiles, in every type; with the large ones an odd
    # and an even number of steps past the pipeline's first, and more tiles than
    # the 256 workgroups that run at once
    seen = set()
    for type, name in enumerate(("f32", "bf16", "f16")):
        for n, rows, cols, ignored in xent_plan.CHECKED:
            aligned = cols % 8 == 0
            live = round(n * (1 - ignored))
            runs = xent_plan.forward(type, n, cols, rows, aligned)[1] + \
                xent_plan.backward(type, n, cols, rows, aligned, live)[1]
            for what, side, steps, count in runs:
                seen.add((type, what, side))
                if side == 256 and steps > 8:
                    seen |= {(type, what, "odd" if steps % 2 else "even")} | \
                        ({(type, what, "several")} if count > 256 else set())
        for what, want in (("stats", (128, 256, "several")), ("prob", (128, 256, "several")),
                           ("dh", (128, 256, "several")), ("dw", (128, 256)), ("dw split", (128, 256))):
            for w in want:
                assert (type, what, w) in seen, (name, what, w)
            assert (type, what, "even") in seen or (type, what, "odd") in seen, (name, what)
        if type != xent_plan.F32:  # six products of as many steps each: an even number, where they are not split
            for what in ("stats", "prob", "dh", "dw"):
                assert {(type, what, "even"), (type, what, "odd")} <= seen, (name, what)
    assert {(1, "dw", "several"), (2, "dw", "several")} <= seen


def test_cross_entropy_workspace_is_within_the_documented_sum():
    need = ctypes.c_uint64()
    mib = 1 << 20
    sizes = [1, 17, 64, 65, 300, 2100, 8192, 65536, 262144, 1 << 20], [1, 63, 300, 1031, 4096, 65536], \
        [1, 300, 24700, 128000, 1 << 22]
    for type, n, d, v, aligned in itertools.product(range(3), *sizes, (0, 1)):
        pack = type == 0 or not aligned
        parts, dk = 3 if type == 0 else 1, -(-d // 64) * 64
        copy_h = 2 * parts * n * dk
        copy_w = max(128 * mib, 256 * 2 * parts * dk) if pack else 0
        small = 64 * (n + 256)  # per-token figures, each array's rounding to 256 bytes
        assert rotor.lib().rotor_xent_workspace_bytes(type, n, d, v, aligned, 0, ctypes.byref(need)) == 0
        rows = 16 if n <= 64 else 128  # few tokens' waves take as few as 16 rows
        assert need.value <= 8 * n * -(-v // rows) + small + (copy_h + copy_w if pack else 0), (type, n, d, v, aligned)
        assert rotor.lib().rotor_xent_workspace_bytes(type, n, d, v, aligned, 1, ctypes.byref(need)) == 0
        p = 256 * mib if n <= 64 else max(128 * mib, 256 * 2 * parts * n)
        skew = 512 * parts * (n + d) + 2 * parts * 64 * (n + d)
        assert need.value <= p + 2 * copy_h + skew + 4 * n * (d + 4) + 2 * 64 * mib + copy_w + small, \
            (type, n, d, v, aligned, need.value)

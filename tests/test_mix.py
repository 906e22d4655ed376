"""Refusals of the operators that mix tokens (no GPU): the C entry points
return ROTOR_EINVAL before any device work, the binding raises ValueError.  And
the plain implementation's gradients against automatic differentiation and
differences."""
import ctypes
import math

import pytest
import torch

import mix_model
import ops_model as m
from paper_1911_13214_amd import ops, rotor

FAKE = 0x10000
E = rotor.ROTOR_EINVAL
NAN, INF = float("nan"), float("inf")


def heads(p=FAKE, batch=4096, token=512, head=64):
    return rotor.Heads(p, batch, token, head)


# ---- head norms and rotation --------------------------------------------------------

F = (ctypes.c_double * 16)(*[0.5] * 16)
ROT = dict(type=1, norm=1, interleaved=0, position_bytes=8, batch=2, tokens=4, heads=4, kv_heads=2, width=32,
           rotary=32, eps=1e-5, frequencies=ctypes.addressof(F), positions=FAKE, position_batch=4, q_weight=FAKE,
           k_weight=FAKE)


def rotation(**kw):
    return rotor.Rotation(**{**ROT, **kw})


def test_rotation_refuses_bad_arguments():
    lib = rotor.lib()

    def fwd(how=None, **kw):
        t = [kw.get(x, heads()) for x in ("q", "k", "y", "z")]
        return lib.rotor_head_norm_rotate(rotation(**(how or {})), *t, None)

    bad_f = (ctypes.c_double * 16)(*[0.5] * 15 + [INF])
    for how in [dict(type=3), dict(type=-1), dict(norm=3), dict(norm=-1), dict(interleaved=2), dict(position_bytes=2),
                dict(batch=-1), dict(tokens=-1), dict(tokens=1 << 31), dict(heads=0), dict(kv_heads=-1),
                dict(width=0), dict(width=31), dict(width=258), dict(rotary=34), dict(rotary=3), dict(rotary=-2),
                dict(eps=-1.0), dict(eps=NAN), dict(frequencies=None), dict(frequencies=ctypes.addressof(bad_f)),
                dict(positions=FAKE + 4), dict(position_batch=-1), dict(q_weight=FAKE + 1), dict(k_weight=FAKE + 1),
                dict(norm=0), dict(batch=1 << 40)]:
        assert fwd(how) == E, how
    for x in ("q", "k", "y", "z"):
        for h in (None, heads(p=None), heads(p=FAKE + 1), heads(batch=-1), heads(token=-1), heads(head=-1),
                  heads(token=1 << 60)):
            assert fwd(**{x: h}) == E, x
    assert lib.rotor_head_norm_rotate(None, heads(), heads(), heads(), heads(), None) == E
    assert fwd(dict(tokens=0), q=None, k=None, y=None, z=None) == rotor.ROTOR_OK

    need = ctypes.c_uint64()
    assert lib.rotor_head_norm_rotate_workspace_bytes(rotation(), ctypes.byref(need)) == rotor.ROTOR_OK
    assert lib.rotor_head_norm_rotate_workspace_bytes(rotation(), None) == E
    assert lib.rotor_head_norm_rotate_workspace_bytes(rotation(width=3), ctypes.byref(need)) == E

    def back(how=None, **kw):
        t = [kw.get(x, heads()) for x in ("dy", "dz", "q", "k", "dq", "dk")]
        return lib.rotor_head_norm_rotate_backward(rotation(**(how or {})), *t, kw.get("dqw", FAKE),
                                                   kw.get("dkw", FAKE), kw.get("work", FAKE),
                                                   kw.get("size", need.value), None)

    for x in ("dy", "dz", "q", "k", "dq", "dk"):
        assert back(**{x: None}) == E and back(**{x: heads(p=FAKE + 1)}) == E, x
    for kw in (dict(dqw=FAKE + 1), dict(dkw=FAKE + 1), dict(work=None), dict(work=FAKE + 8), dict(size=need.value - 1)):
        assert back(**kw) == E, kw
    assert back(dict(norm=0, q_weight=None, k_weight=None)) == E  # a weight's gradient without a norm


def test_rotation_refuses_what_is_not_heads():
    x = torch.zeros(2, 3, 4, 32)
    with pytest.raises(ValueError):
        ops.head_norm_rotate(x)
    with pytest.raises(ValueError):
        ops.head_norm_rotate_backward(x, None, x)
    with pytest.raises(ValueError):
        ops._frequencies(8, 1e4, (1.0, 2.0))
    with pytest.raises(ValueError):
        ops._frequencies(4, 1e4, (1.0, INF))
    with pytest.raises(ValueError):
        ops._no_overlap(torch.zeros(4, 8).expand(3, 4, 8), "out")
    with pytest.raises(ValueError):
        ops._no_overlap(torch.zeros(40).as_strided((4, 8), (7, 1)), "out")
    t = torch.zeros(4, 5, 8)[:, 1:3, ::2].transpose(0, 1)
    assert ops._no_overlap(t, "out") is t


# ---- attention --------------------------------------------------------------------------

ATT = dict(type=1, position_bytes=8, length_bytes=4, batch=2, tokens=4, keys=8, heads=4, kv_heads=2, width=64,
           window=3, sinks=1, scale=0.125, positions=FAKE, lengths=FAKE)


def attention(**kw):
    return rotor.Attention(**{**ATT, **kw})


BAD = [dict(type=3), dict(type=-1), dict(batch=-1), dict(tokens=-1), dict(keys=-1), dict(heads=0), dict(kv_heads=0),
       dict(kv_heads=3), dict(kv_heads=8), dict(width=0), dict(width=4), dict(width=60), dict(width=136),
       dict(window=-1), dict(sinks=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN), dict(scale=INF),
       dict(positions=FAKE + 4), dict(position_bytes=3), dict(batch=1 << 21), dict(tokens=1 << 30), dict(keys=1 << 30),
       dict(heads=1 << 16, kv_heads=1)]
WRONG = [None, heads(p=None), heads(p=FAKE + 8), heads(batch=-8), heads(token=-8), heads(head=-8), heads(token=516),
         heads(head=68), heads(batch=4), heads(token=1 << 60)]


def test_attention_refuses_bad_arguments():
    f = rotor.lib().rotor_window_attention

    def fwd(how=None, lse=FAKE, **kw):
        return f(attention(**(how or {})), *[kw.get(x, heads()) for x in ("q", "k", "v", "out")], lse, FAKE, 1 << 20,
                 None)

    for how in BAD + [dict(lengths=FAKE + 2), dict(length_bytes=1)]:
        assert fwd(how) == E, how
    for x in ("q", "k", "v", "out"):
        for h in WRONG:
            assert fwd(**{x: h}) == E, (x, h and (h.p, h.batch, h.token, h.head))
    for x in ("k", "v"):  # 66 rows past 2^31 bytes
        assert fwd(**{x: heads(token=1 << 25)}) == E
    assert fwd(lse=FAKE + 2) == E
    # sums of the parts need their workspace
    how = dict(tokens=1, keys=1 << 20, window=0, positions=None, lengths=None)
    need = ctypes.c_uint64()
    w = rotor.lib().rotor_window_attention_workspace_bytes
    assert w(attention(**how), 0, ctypes.byref(need)) == rotor.ROTOR_OK and need.value > 0
    for work, size in ((None, need.value), (FAKE + 8, need.value), (FAKE, need.value - 1)):
        assert f(attention(**how), heads(), heads(), heads(), heads(), FAKE, work, size, None) == E
    assert w(attention(), 0, None) == E and w(attention(), 2, ctypes.byref(need)) == E
    assert w(attention(width=7), 0, ctypes.byref(need)) == E
    assert w(attention(), 1, ctypes.byref(need)) == E  # a step is of one token
    # nothing to do, whatever the pointers
    for how in (dict(batch=0), dict(tokens=0)):
        assert f(attention(**how), None, heads() if "tokens" in how else None, heads() if "tokens" in how else None, None,
                 None, None, 0, None) == rotor.ROTOR_OK


def test_attention_backward_refuses_bad_arguments():
    f = rotor.lib().rotor_window_attention_backward
    need = ctypes.c_uint64()
    w = rotor.lib().rotor_window_attention_backward_workspace_bytes
    assert w(attention(), ctypes.byref(need)) == rotor.ROTOR_OK and need.value > 0
    names = ("dout", "q", "k", "v", "out", "dq", "dk", "dv")

    def back(how=None, lse=FAKE, work=FAKE, size=need.value, **kw):
        t = [kw.get(x, heads()) for x in names]
        return f(attention(**(how or {})), *t[:5], lse, *t[5:], work, size, None)

    for how in BAD + [dict(lengths=FAKE + 2)]:
        assert back(how, size=1 << 40) == E, how
    for x in names:
        for h in WRONG:
            assert back(**{x: h}) == E, x
    for x in ("q", "dout"):  # a tile of rows past 2^31 bytes
        assert back(**{x: heads(head=1 << 29)}) == E
    for kw in (dict(lse=None), dict(lse=FAKE + 1), dict(work=None), dict(work=FAKE + 8), dict(size=need.value - 1)):
        assert back(**kw) == E, kw
    assert w(attention(), None) == E and w(attention(width=9), ctypes.byref(need)) == E
    assert w(attention(keys=1 << 24), ctypes.byref(need)) == E


def test_step_refuses_bad_arguments():
    f = rotor.lib().rotor_window_attention_step
    one = dict(tokens=1, lengths=None)

    def step(how=None, ring=0, **kw):
        t = [kw.get(x, heads()) for x in ("q", "k", "v", "kc", "vc", "out")]
        return f(attention(**{**one, **(how or {})}), *t[:5], ring, t[5], FAKE, 1 << 30, None)

    for how in BAD + [dict(tokens=2), dict(tokens=0), dict(keys=0), dict(positions=None), dict(lengths=FAKE)]:
        assert step(how) == E, how
    assert step(ring=2) == E and step(ring=-1) == E
    for how in (dict(window=0), dict(window=8), dict(sinks=6), dict(sinks=9)):
        assert step(how, ring=1) == E, how
    for x in ("q", "k", "v", "kc", "vc", "out"):
        for h in WRONG:
            if h is not None and h.token in (-8, 516, 1 << 60) and x in ("q", "k", "v", "out"):
                continue  # one token: its stride does not matter
            assert step(**{x: h}) == E, x


def test_attention_refuses_what_is_on_the_cpu():
    q = torch.zeros(2, 4, 4, 64)
    with pytest.raises(ValueError):
        ops.window_attention(q, q, q)
    with pytest.raises(ValueError):
        ops.window_attention_step(q[:, 0], q[:, 0], q[:, 0], q, q, torch.zeros(2, dtype=torch.int32))


def test_backward_workspaces_follow_their_documented_sums():
    """12 bytes a row (rows to 128), in float16 4 more for 32 rows, and sums of
    128 keys for each part."""
    w = rotor.lib().rotor_window_attention_backward_workspace_bytes
    need = ctypes.c_uint64()
    for how, parts in [(dict(tokens=1000, keys=1000, window=0), None), (dict(tokens=64, keys=64), 0)]:
        assert w(attention(**how), ctypes.byref(need)) == rotor.ROTOR_OK
        rows = -(-how["tokens"] * 2 // 128) * 128 * 2 * 2
        assert need.value >= 12 * rows
        if parts == 0:
            assert need.value <= 12 * rows + 5 * 256


# ---- the plain implementation --------------------------------------------------------------

def plain(q, k, v, window, sinks, scale, positions, lengths):
    """From the definition, row by row."""
    b, n, h, d = q.shape
    keys, g = k.shape[1], h // k.shape[2]
    out = []
    for x in range(b):
        for i in range(n):
            p = (keys - n if positions is None else int(positions[x])) + i
            end = keys if lengths is None else min(int(lengths[x]), keys)
            at = [j for j in range(keys) if 0 <= j <= p < end and (window is None or p - j < window or j < sinks)]
            for y in range(h):
                if not at:
                    out.append(torch.zeros(d, dtype=torch.float64))
                    continue
                s = torch.stack([scale * (q[x, i, y] * k[x, j, y // g]).sum() for j in at])
                out.append((torch.softmax(s, 0)[:, None] * v[x, at, y // g]).sum(0))
    return torch.stack(out).view(b, n, h, d)


@pytest.mark.parametrize("window,sinks,positions,lengths", [(None, 0, None, None), (3, 1, None, [7, 4]), (2, 0, [-2, 4], None),
                                                            (1, 2, [1, 3], [9, 5])])
def test_the_plain_attention(window, sinks, positions, lengths):
    g = torch.Generator().manual_seed(4)
    q, k, v, do = (m.normal(g, 2, n, h, 8) for n, h in ((5, 4), (9, 2), (9, 2), (5, 4)))
    positions = None if positions is None else torch.tensor(positions)
    lengths = None if lengths is None else torch.tensor(lengths)
    m.UNIT[torch.float64] = 2.0 ** -53
    try:
        val, _ = mix_model.attention(q, k, v, window, sinks, None, positions, lengths, do)
    finally:
        del m.UNIT[torch.float64]
    leaves = [x.clone().requires_grad_() for x in (q, k, v)]
    out = plain(*leaves, window, sinks, 8 ** -0.5, positions, lengths)
    assert torch.allclose(val["out"], out, atol=1e-13)
    for x, y in zip(torch.autograd.grad(out, leaves, do), ("dq", "dk", "dv")):
        assert torch.allclose(x, val[y], atol=1e-12)
    # differences along a direction
    with torch.no_grad():
        for i, name in enumerate(("dq", "dk", "dv")):
            way, args = m.normal(g, *leaves[i].shape), [x.detach() for x in leaves]
            f = [(plain(*[a + e * way if j == i else a for j, a in enumerate(args)], window, sinks, 8 ** -0.5, positions,
                        lengths) * do).sum() for e in (1e-5, -1e-5)]
            assert math.isclose(float(f[0] - f[1]) / 2e-5, float((val[name] * way).sum()), rel_tol=1e-6, abs_tol=1e-7)


@pytest.mark.parametrize("interleaved", [False, True])
def test_the_plain_rotation_keeps_lengths_and_distances(interleaved):
    g = torch.Generator().manual_seed(2)
    x, y = m.normal(g, 1, 1, 1, 16), m.normal(g, 1, 1, 1, 16)
    turn = lambda u, p: mix_model.rotation(u, None, "none", 0.0, torch.tensor([[p]]), 12, interleaved=interleaved)
    assert torch.allclose(turn(x, 77).norm(), x.norm()) and torch.equal(turn(x, 5)[..., 12:], x[..., 12:])
    a = (turn(x, 19) * turn(y, 12)).sum()
    assert torch.allclose((turn(x, 1007) * turn(y, 1000)).sum(), a) and torch.allclose(turn(turn(x, 4), -4), x)


def test_a_chain_with_attention_is_made_of_its_blocks():
    from paper_1911_13214_amd import stages as lm
    how = dict(heads=4, kv_heads=2, head_width=16, window=9, sinks=2)
    chain = lm.language_chain(3, 7, rows=11, width=32, device="cpu", attention=how)
    assert [type(f) for f in chain] == [lm.Embedding] + [lm.AttentionBlock] * 3 + [lm.Loss]
    a = chain[1].first
    assert a.enter.weight.shape == ((4 + 4) * 16, 32) and a.leave.weight.shape == (32, 64) and a.window == 9
    lm.set_lengths(chain, 5)
    assert all(f.first.lengths == 5 for f in chain[1:4])
    # seeded: the same again, and widths that do not depend on attention
    again = lm.language_chain(3, 7, rows=11, width=32, device="cpu", attention=how)
    assert all(torch.equal(x, y) for f, g in zip(chain, again) for x, y in zip(f.parameters(), g.parameters()))
    plain = lm.language_chain(3, 7, rows=11, width=32, device="cpu")
    assert [f.second[0].out_features for f in chain[1:4]] == [f.second[0].out_features for f in plain[1:4]]

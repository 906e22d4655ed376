"""Workloads of the operators of a language-model chain, as a training or
scoring program calls them.

The planner decides which stages of a chain keep their activations and which
run again; these four operators are the parts of such a chain around the
blocks' own products:

  "dropout"    y = r + keep * x / (1 - q), the mask drawn from a counter, and
               its gradient from the same counter
  "embedding"  y_i = s E[tok_i], and the table's gradient
  "norm"       y = a x + gate * post(z) and h = pre(y), and its gradients: the
               seam between a block and the next
  "xent"       projection onto the vocabulary and softmax cross entropy, and
               its gradients: the chain's loss

A case with train=False is the forward call alone (evaluation, scoring one
token); with train=True it is the forward and the backward call of one step,
and all gradients are outputs.  Every input is a function of the case and a
seed.  With ``own`` false, run() computes the same from elementary torch
operations in 32 bits.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}

# bounds of the drawn sizes, so that no drawn case costs more than the largest
# listed one of its operator
MOST_ELEMENTS = 8192 * 4096
MOST_TABLE = 65536 * 2048
MOST_PRODUCT = 8192 * 4096 * 128000


def listed():
    drop = dict(op="dropout", p=0.1, residual=False, train=False)
    emb = dict(op="embedding", scaled=True, padding=False, train=True)
    norm = dict(op="norm", post="rms", pre="rms", gate=0, biases=False, train=True)
    xent = dict(op="xent", ignored=0.0, train=True)
    return [
        # a small chain on a small batch: latency alone
        dict(drop, name="dropout-small", type="f32", rows=64, cols=1001),
        # the end of a block in training: dropout of its output onto the
        # residual, and the gradient
        dict(drop, name="dropout-residual", type="bf16", rows=8192, cols=4096, residual=True, train=True),
        # one token of a sequence being scored: latency alone
        dict(emb, name="embedding-token", type="f16", tokens=1, rows=32000, cols=1024, train=False),
        # a ragged batch with odd sizes and a padding token
        dict(emb, name="embedding-ragged", type="f32", tokens=5003, rows=50021, cols=1001, padding=True),
        # a training batch: eight sequences of 4096
        dict(emb, name="embedding-train", type="bf16", tokens=32768, rows=65536, cols=2048),
        # one token of a sequence being scored, a wide chain: latency alone
        dict(norm, name="norm-token", type="bf16", rows=1, cols=4096, train=False),
        # batch 4096, width 1024 as in the synthetic chains, LayerNorm with
        # biases before the block only
        dict(norm, name="norm-layer", type="f32", rows=4096, cols=1024, post="none", pre="layer", biases=True),
        # a training batch with a gate per sequence (eight of 2048), norms on
        # both sides
        dict(norm, name="norm-gated", type="bf16", rows=16384, cols=2048, gate=8),
        # one token scored against a whole vocabulary: the weights' bytes
        dict(xent, name="xent-token", type="bf16", tokens=1, rows=50021, cols=2048, train=False),
        # a small chain in 32 bits, odd sizes, some tokens without a target
        dict(xent, name="xent-f32", type="f32", tokens=1000, rows=10007, cols=1024, ignored=0.2),
        # a training batch of an ordinary chain, prompts without a target
        dict(xent, name="xent-train", type="bf16", tokens=4096, rows=32768, cols=2048, ignored=0.3),
        # the largest: a wide chain and a large vocabulary
        dict(xent, name="xent-large", type="bf16", tokens=8192, rows=128000, cols=4096),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """Half of the widths as chains have them (multiples of 64), half as they
    come, odd ones among them."""
    c = _log_int(rng, lo, hi)
    return max(64, c // 64 * 64) if rng.random() < 0.5 else c


def draw(rng):
    op = rng.choice(["dropout", "embedding", "norm", "xent", "xent"])
    c = dict(op=op, type=rng.choice(["f32", "bf16", "bf16", "f16"]), train=rng.random() < 0.7)
    if op == "dropout":
        c.update(rows=_log_int(rng, 1, 8192), cols=_width(rng, 16, 4096), residual=rng.random() < 0.5,
                 p=rng.choice([0.05, 0.1, 0.2, 0.5]))
        if c["type"] == "f32":
            c["rows"] = max(1, c["rows"] // 2)
    elif op == "embedding":
        c.update(tokens=_log_int(rng, 1, 32768), rows=_log_int(rng, 500, 65536), cols=_width(rng, 64, 2048),
                 scaled=rng.random() < 0.5, padding=rng.random() < 0.3)
        if c["type"] == "f32":
            c.update(tokens=(c["tokens"] + 1) // 2, rows=c["rows"] // 2)
    elif op == "norm":
        c.update(rows=_log_int(rng, 1, 16384), cols=_width(rng, 64, 4096), post=rng.choice(["none", "rms", "layer"]),
                 pre=rng.choice(["rms", "layer", "rms"]), gate=rng.choice([0, 1, 8]), biases=rng.random() < 0.3)
        c["rows"] = max(1, c["rows"] // (2 if c["type"] == "f32" else 1))
        while c["rows"] * c["cols"] * (2 if c["type"] == "f32" else 1) > MOST_ELEMENTS:
            c["rows"] = c["rows"] * 3 // 4
        if c["gate"] > 1:  # sequences of one length each
            c["rows"] = -(-c["rows"] // c["gate"]) * c["gate"]
            if c["rows"] * c["cols"] > MOST_ELEMENTS:
                c["rows"] -= c["gate"]
    else:
        c.update(tokens=_log_int(rng, 1, 8192), rows=_log_int(rng, 1000, 128000), cols=_width(rng, 64, 4096),
                 ignored=rng.choice([0.0, 0.1, 0.5]))
        most = MOST_PRODUCT // (16 if c["type"] == "f32" else 1)  # products in 32 bits take 16 times the time
        while c["tokens"] * c["rows"] * c["cols"] > most:
            c["tokens"] = c["tokens"] * 3 // 4
    return c


# ---- inputs ------------------------------------------------------------------

def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _token_shares(rows):
    """Shares of the tokens in text: Zipf's law with a flattened head."""
    w = 1.0 / (np.arange(rows, dtype=np.float64) + 2.7)
    return w / w.sum()


def _draw_tokens(case, n, gen, device):
    shares = torch.from_numpy(_token_shares(case["rows"])).to(device)
    edges = shares.cumsum(0)
    u = torch.rand(n, generator=gen, device=device, dtype=torch.float64)
    return torch.searchsorted(edges, u).clamp_(max=case["rows"] - 1)


def _inputs(case, seed):
    device = _device()
    gen = torch.Generator(device=device).manual_seed(1911 * 2 ** 20 + seed)
    dtype = TYPES[case["type"]]
    d = case["cols"]

    def normal(*shape, std=1.0, mean=0.0):
        return (torch.randn(shape, generator=gen, device=device) * std + mean).to(dtype)

    s = {"case": case}
    if case["op"] == "dropout":
        n = case["rows"]
        s.update(x=normal(n, d), seed=int(np.random.default_rng(seed).integers(1 << 62)), step=1000 + seed % 1000)
        s["residual"] = normal(n, d) if case["residual"] else None
        s["dy"] = normal(n, d, std=1e-2) if case["train"] else None
    elif case["op"] == "embedding":
        n = case["tokens"]
        s.update(tokens=_draw_tokens(case, n, gen, device), table=normal(case["rows"], d, std=0.02))
        s["scale"] = math.sqrt(d) if case["scaled"] else 1.0
        s["padding"] = 0 if case["padding"] else None  # the most frequent token, as a padded batch has it
        s["dy"] = normal(n, d, std=1e-2) if case["train"] else None
    elif case["op"] == "norm":
        n = case["rows"]
        s.update(x=normal(n, d, std=2.0), z=normal(n, d, std=0.7, mean=0.1))
        s["post_weight"] = normal(d, std=0.1, mean=1.0) if case["post"] != "none" else None
        s["pre_weight"] = normal(d, std=0.1, mean=1.0)
        s["post_bias"] = normal(d, std=0.1) if case["biases"] and case["post"] != "none" else None
        s["pre_bias"] = normal(d, std=0.1) if case["biases"] else None
        s["gate"] = normal(case["gate"], d, std=0.3, mean=0.5) if case["gate"] else None
        s.update(residual_scale=0.9, eps=1e-5)
        s["dy"] = normal(n, d, std=1e-2) if case["train"] else None
        s["dh"] = normal(n, d, std=1e-2) if case["train"] else None
    else:
        n = case["tokens"]
        w = torch.randn((case["rows"], d), generator=gen, device=device) * (1.0 / math.sqrt(d))
        t = _draw_tokens(case, n, gen, device)
        # normed activations that lean towards their target, as a model half
        # trained has them
        h = torch.randn((n, d), generator=gen, device=device) + 4.0 * w[t]
        s.update(h=h.to(dtype), w=w.to(dtype))
        skip = torch.rand(n, generator=gen, device=device) < case["ignored"]
        s["targets"] = torch.where(skip, -100, t)
        # the gradient of the mean over the tokens that have a target
        s["grad_loss"] = torch.full((n,), 1.0 / max(1, n - int(skip.sum())), device=device)
    return s


def prepare(case, seed):
    return _inputs(case, seed)


# ---- one pass ----------------------------------------------------------------

def run(state):
    return (_own if own else _plain)[state["case"]["op"]](state)


def _own_dropout(s):
    from paper_1911_13214_amd import ops
    p, seed, step = s["case"]["p"], s["seed"], s["step"]
    y = ops.dropout(s["x"], p, seed, step, residual=s["residual"])
    if not s["case"]["train"]:
        return y
    return y, ops.dropout(s["dy"], p, seed, step)


def _own_embedding(s):
    from paper_1911_13214_amd import ops
    y = ops.embedding(s["tokens"], s["table"], s["scale"])
    if not s["case"]["train"]:
        return y
    return y, ops.embedding_backward(s["tokens"], s["dy"], s["table"].shape[0], s["scale"], padding=s["padding"])


def _own_norm(s):
    from paper_1911_13214_amd import ops
    c = s["case"]
    how = dict(post=c["post"], post_weight=s["post_weight"], post_bias=s["post_bias"], gate=s["gate"],
               residual_scale=s["residual_scale"], pre=c["pre"], pre_weight=s["pre_weight"], pre_bias=s["pre_bias"],
               eps=s["eps"])
    y, h, stats = ops.residual_norm(s["x"], s["z"], **how)
    if not c["train"]:
        return y, h
    return (y, h), ops.residual_norm_backward(s["dy"], s["dh"], y, s["z"], stats, **how)


def _own_xent(s):
    from paper_1911_13214_amd import ops
    loss, lse = ops.linear_cross_entropy(s["h"], s["w"], s["targets"])
    if not s["case"]["train"]:
        return loss
    return loss, ops.linear_cross_entropy_backward(s["h"], s["w"], s["targets"], lse, s["grad_loss"])


_own = {"dropout": _own_dropout, "embedding": _own_embedding, "norm": _own_norm, "xent": _own_xent}


# ---- the plain forms -----------------------------------------------------------

_LOW = 0xFFFFFFFF


def _philox(groups, step, seed):
    """Philox4x32 with ten rounds (Salmon, Moraes, Dror, Shaw, 2011): the four
    32-bit words of every counter (group, step) under the key ``seed``."""
    c = [groups & _LOW, groups >> 32, torch.full_like(groups, step & _LOW), torch.full_like(groups, step >> 32)]
    k0, k1 = seed & _LOW, seed >> 32
    for _ in range(10):
        # 64-bit products wrap, their 64 bits are the right ones
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32 & _LOW) ^ c[1] ^ k0, b & _LOW, (a >> 32 & _LOW) ^ c[3] ^ k1, a & _LOW]
        k0, k1 = (k0 + 0x9E3779B9) & _LOW, (k1 + 0xBB67AE85) & _LOW
    return c


def _keep(n, p, step, seed, device):
    """Which of n elements are kept: 16 bits each, eight elements a counter."""
    words = _philox(torch.arange(-(-n // 8), device=device), step, seed)
    bits = torch.stack([half for w in words for half in (w & 0xFFFF, w >> 16)], 1).reshape(-1)[:n]
    return bits >= round(p * 65536)


def _plain_dropout(s):
    x, p = s["x"], s["case"]["p"]
    keep = _keep(x.numel(), p, s["step"], s["seed"], x.device).reshape(x.shape)
    scale = 65536 / (65536 - round(p * 65536))
    y = torch.where(keep, x.float() * scale, 0.0)
    if s["residual"] is not None:
        y = s["residual"].float() + y
    y = y.to(x.dtype)
    if not s["case"]["train"]:
        return y
    return y, torch.where(keep, s["dy"].float() * scale, 0.0).to(x.dtype)


def _plain_embedding(s):
    tokens, table = s["tokens"], s["table"]
    y = (table[tokens].float() * s["scale"]).to(table.dtype)
    if not s["case"]["train"]:
        return y
    g = torch.zeros(table.shape, dtype=torch.float32, device=table.device)
    g.index_add_(0, tokens, s["dy"].float() * s["scale"])
    if s["padding"] is not None:
        g[s["padding"]] = 0
    return y, g.to(table.dtype)


def _normed(kind, u, eps):
    """u normed, and the factor 1 / deviation of each row."""
    if kind == "none":
        return u, None
    if kind == "layer":
        u = u - u.mean(1, keepdim=True)
    r = 1.0 / torch.sqrt((u * u).mean(1, keepdim=True) + eps)
    return u * r, r


def _normed_grad(kind, n, r, d):
    """Gradient of the normed rows n with factor r, from that of n."""
    if kind == "none":
        return d
    if kind == "layer":
        d = d - d.mean(1, keepdim=True)
    return r * (d - n * (d * n).mean(1, keepdim=True))


def _scaled(n, weight, bias):
    if weight is not None:
        n = n * weight.float()
    return n if bias is None else n + bias.float()


def _plain_norm(s):
    c, dtype = s["case"], s["x"].dtype
    gate = None
    if s["gate"] is not None:  # one row of gates for each sequence
        gate = s["gate"].float().repeat_interleave(c["rows"] // c["gate"], 0)
    n1, r1 = _normed(c["post"], s["z"].float(), s["eps"])
    b = _scaled(n1, s["post_weight"], s["post_bias"])
    y = s["residual_scale"] * s["x"].float() + (b if gate is None else gate * b)
    n2, r2 = _normed(c["pre"], y, s["eps"])
    h = _scaled(n2, s["pre_weight"], s["pre_bias"])
    if not c["train"]:
        return y.to(dtype), h.to(dtype)
    dh = s["dh"].float()
    t = s["dy"].float() + _normed_grad(c["pre"], n2, r2, dh * s["pre_weight"].float())
    db = t if gate is None else gate * t
    weighted = db if s["post_weight"] is None else db * s["post_weight"].float()
    g = {"x": s["residual_scale"] * t, "z": _normed_grad(c["post"], n1, r1, weighted),
         "pre_weight": (dh * n2).sum(0)}
    if s["pre_bias"] is not None:
        g["pre_bias"] = dh.sum(0)
    if s["post_weight"] is not None:
        g["post_weight"] = (db * n1).sum(0)
    if s["post_bias"] is not None:
        g["post_bias"] = db.sum(0)
    if gate is not None:
        g["gate"] = (t * b).reshape(c["gate"], -1, c["cols"]).sum(1)
    return (y.to(dtype), h.to(dtype)), {k: v.to(dtype) for k, v in g.items()}


def _plain_xent(s):
    h, w, t = s["h"].float(), s["w"].float(), s["targets"]
    logits = h @ w.t()
    top = logits.amax(1, keepdim=True)
    e = torch.exp(logits - top)
    total = e.sum(1, keepdim=True)
    some = t >= 0
    at = t.clamp(min=0).unsqueeze(1)
    loss = (top + torch.log(total) - logits.gather(1, at)).squeeze(1)
    loss = torch.where(some, loss, 0.0)
    if not s["case"]["train"]:
        return loss
    p = e.div_(total)
    p.scatter_add_(1, at, torch.full_like(top, -1.0))
    p *= torch.where(some, s["grad_loss"], 0.0).unsqueeze(1)
    return loss, ((p @ w).to(s["h"].dtype), (p.t() @ h).to(s["w"].dtype))


_plain = {"dropout": _plain_dropout, "embedding": _plain_embedding, "norm": _plain_norm, "xent": _plain_xent}


# ---- what a pass cannot do without -------------------------------------------------

def work(case):
    es = 4 if case["type"] == "f32" else 2
    d, train = case["cols"], case["train"]
    if case["op"] == "dropout":
        n = case["rows"] * d
        arrays = 2 + case["residual"] + 2 * train
        return {"bytes": n * es * arrays, "flops": n * (1 + case["residual"] + train)}
    if case["op"] == "embedding":
        n, v = case["tokens"], case["rows"]
        distinct = -np.expm1(n * np.log1p(-_token_shares(v))).sum()  # expected
        fwd = 8 * n + (distinct + n) * d * es
        return {"bytes": int(fwd + train * (n + v) * d * es), "flops": n * d * (1 + 2 * train)}
    if case["op"] == "norm":
        n = case["rows"] * d
        # x, z in, y, h out; dy, dh, y, z in, dx, dz out
        return {"bytes": n * es * (4 + 6 * train), "flops": n * (12 + 24 * train)}
    n, v = case["tokens"], case["rows"]
    # h, w and targets in, losses out; gradients of h and w out; one product
    # forward, two more for the gradients
    return {"bytes": (n + v) * d * es * (1 + train) + 12 * n, "flops": 2 * n * v * d * (3 if train else 1)}


# ---- the definitions, in 64 bits -----------------------------------------------------

def _mask64(n, p, step, seed):
    """The kept elements again, with numpy's unsigned integers."""
    u32 = np.uint64(32)
    low = np.uint64(0xFFFFFFFF)
    i = np.arange((n + 7) // 8, dtype=np.uint64)
    x0, x1 = i & low, i >> u32
    x2 = np.full_like(i, step & 0xFFFFFFFF)
    x3 = np.full_like(i, step >> 32)
    for r in range(10):
        key0 = np.uint64(((seed & 0xFFFFFFFF) + r * 0x9E3779B9) % 2 ** 32)
        key1 = np.uint64(((seed >> 32) + r * 0xBB67AE85) % 2 ** 32)
        p0 = np.uint64(0xD2511F53) * x0
        p1 = np.uint64(0xCD9E8D57) * x2
        x0, x1, x2, x3 = (p1 >> u32) ^ x1 ^ key0, p1 & low, (p0 >> u32) ^ x3 ^ key1, p0 & low
    out = np.empty((i.size, 8), dtype=np.uint64)
    for k, word in enumerate((x0, x1, x2, x3)):
        out[:, 2 * k] = word % np.uint64(65536)
        out[:, 2 * k + 1] = word // np.uint64(65536)
    return out.reshape(-1)[:n] >= np.uint64(round(p * 65536))


def exact(case, seed):
    """What run() returns, from the definitions in 64 bits; gradients by
    automatic differentiation of the forward."""
    s = _inputs(case, seed)
    train = case["train"]
    f64 = torch.float64

    def leaf(t):
        return None if t is None else t.to(f64).requires_grad_(train)

    with torch.set_grad_enabled(train):
        if case["op"] == "dropout":
            n = s["x"].numel()
            keep = torch.from_numpy(_mask64(n, case["p"], s["step"], s["seed"])).to(s["x"].device)
            q = round(case["p"] * 65536) / 65536
            x = leaf(s["x"])
            y = x * keep.reshape(x.shape) / (1 - q)
            if s["residual"] is not None:
                y = y + s["residual"].to(f64)
            if not train:
                return y
            return y.detach(), torch.autograd.grad(y, x, s["dy"].to(f64))[0]
        if case["op"] == "embedding":
            table = s["table"].to(f64)
            y = table[s["tokens"]] * s["scale"]
            if not train:
                return y
            # the k-th occurrence of every token at once, then the tokens that
            # occur more often one by one
            g = torch.zeros_like(table)
            order = torch.argsort(s["tokens"], stable=True)
            sorted_tokens = s["tokens"][order]
            first = torch.searchsorted(sorted_tokens, sorted_tokens)
            nth = torch.arange(len(order), device=order.device) - first
            few = nth < 64
            dy = s["dy"].to(f64)
            for k in range(min(64, int(nth.max()) + 1)):
                at = order[nth == k]
                g[s["tokens"][at]] += dy[at]
            for v in torch.unique(sorted_tokens[~few]).tolist():
                g[v] = dy[s["tokens"] == v].sum(0)
            g *= s["scale"]
            if s["padding"] is not None:
                g[s["padding"]] = 0
            return y, g
        if case["op"] == "norm":
            names = ["x", "z", "pre_weight", "pre_bias", "post_weight", "post_bias", "gate"]
            v = {k: leaf(s[k]) for k in names}

            def norm(kind, u, w, b):
                if kind == "layer":
                    u = (u - u.mean(-1, keepdim=True)) / torch.sqrt(u.var(-1, unbiased=False, keepdim=True) + s["eps"])
                elif kind == "rms":
                    u = u / torch.sqrt(u.square().mean(-1, keepdim=True) + s["eps"])
                u = u if w is None else u * w
                return u if b is None else u + b

            out = norm(case["post"], v["z"], v["post_weight"], v["post_bias"])
            if v["gate"] is not None:
                out = (out.view(case["gate"], -1, case["cols"]) * v["gate"][:, None]).view(out.shape)
            y = s["residual_scale"] * v["x"] + out
            h = norm(case["pre"], y, v["pre_weight"], v["pre_bias"])
            if not train:
                return y, h
            present = [k for k in names if v[k] is not None]
            grads = torch.autograd.grad([y, h], [v[k] for k in present], [s["dy"].to(f64), s["dh"].to(f64)])
            return (y.detach(), h.detach()), dict(zip(present, grads))
        h, w = leaf(s["h"]), leaf(s["w"])
        rows = torch.nonzero(s["targets"] >= 0).squeeze(1)
        loss = torch.zeros(case["tokens"], dtype=f64, device=h.device)
        logits = h[rows] @ w.t()
        part = torch.logsumexp(logits, 1) - logits.gather(1, s["targets"][rows].unsqueeze(1)).squeeze(1)
        loss = loss.index_put((rows,), part)
        if not train:
            return loss
        return loss.detach(), torch.autograd.grad(loss, (h, w), s["grad_loss"].to(f64))

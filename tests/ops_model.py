"""Plain 64-bit implementations of the operators of a chain's stages, on the
CPU, and the comparison of 16- and 32-bit results with them."""
import numpy as np
import torch

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U32 = 2.0 ** -24  # unit roundoff of the 32-bit arithmetic
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
# half the spacing of the subnormal numbers of each type
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}


def close(out, ref, slack=0.0, what=""):
    """Every element of ``out`` within one rounding of its type of ``ref``
    (64 bits), plus ``slack`` (a number or a tensor): the error of the value
    before it is rounded."""
    got = out.detach().cpu().double()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    slack = slack if torch.is_tensor(slack) else torch.tensor(float(slack), dtype=torch.float64)
    bound = UNIT[out.dtype] * (ref.abs() + slack) + slack + TINY[out.dtype]
    err = (got - ref).abs()
    bad = ~(err <= bound)
    assert not bad.any(), (what, int(bad.sum()), float(err[bad].max()), float(bound[bad].min()),
                           torch.nonzero(bad)[:4].tolist())


def normal(gen, *shape, dtype=torch.float64, std=1.0, mean=0.0):
    """Seeded normal numbers, rounded to ``dtype``."""
    return (torch.randn(shape, generator=gen, dtype=torch.float64) * std + mean).to(dtype)


# ---- dropout -------------------------------------------------------------------

def philox(counter, key):
    """Philox4x32-10 in Python's integers: four 32-bit words."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def keep_mask(n, p, seed, step):
    """Which of n elements are kept."""
    low = 0xFFFFFFFF
    out = np.empty(-(-n // 8) * 8, dtype=bool)
    t = round(65536 * p)
    for g in range(-(-n // 8)):
        words = philox((g & low, g >> 32, step & low, step >> 32 & low), (seed & low, seed >> 32 & low))
        for e in range(8):
            out[8 * g + e] = (words[e // 2] >> (16 * (e % 2)) & 0xFFFF) >= t
    return torch.from_numpy(out[:n])


def dropout(x, p, seed, step, residual=None):
    t = round(65536 * p)
    keep = keep_mask(x.numel(), p, seed, step).reshape(x.shape)
    y = torch.where(keep, x.double() * (65536 / (65536 - t) if t < 65536 else 0.0), 0.0)
    return y if residual is None else residual.double() + y


# ---- embedding -----------------------------------------------------------------

def embedding(tokens, table, scale):
    rows = table.shape[0]
    ok = (tokens >= 0) & (tokens < rows)
    y = table.double()[tokens.clamp(0, rows - 1)] * scale
    y[~ok] = float("nan")
    return y


def embedding_grad(tokens, dy, rows, scale, padding=None):
    """The gradient, and the sum of its terms' magnitudes."""
    tokens, dy = tokens.reshape(-1), dy.double().reshape(-1, dy.shape[-1])
    ok = (tokens >= 0) & (tokens < rows)
    if padding is not None:
        ok &= tokens != padding
    g = torch.zeros(rows, dy.shape[1], dtype=torch.float64)
    m = torch.zeros_like(g)
    g.index_add_(0, tokens[ok], dy[ok] * scale)
    m.index_add_(0, tokens[ok], (dy[ok] * scale).abs())
    return g, m


# ---- residual norm ----------------------------------------------------------------

def norm(kind, u, weight, bias, eps):
    """The norm's output, the normed rows and 1 / deviation."""
    if kind == "none":
        return u, u, torch.ones_like(u[:, :1])
    mean = u.mean(1, keepdim=True) if kind == "layer" else 0.0
    r = 1.0 / torch.sqrt((u - mean).square().mean(1, keepdim=True) + eps)
    n = (u - mean) * r
    out = n if weight is None else n * weight
    return (out if bias is None else out + bias), n, r


def residual_norm(x, z, post, post_weight, post_bias, gate, residual_scale, pre, pre_weight, pre_bias, eps):
    y = residual_scale * x
    if z is not None:
        b = norm(post, z, post_weight, post_bias, eps)[0]
        if gate is not None:
            b = b * gate.reshape(-1, x.shape[1]).repeat_interleave(x.shape[0] // (gate.numel() // x.shape[1]), 0)
        y = y + b
    return y, norm(pre, y, pre_weight, pre_bias, eps)[0] if pre != "none" else None


# ---- cross entropy ---------------------------------------------------------------------

def cross_entropy(h, w, targets, ignore):
    """Loss and log-sum-exp of each token, NaN for targets outside w."""
    logits = h.double() @ w.double().t()
    lse = torch.logsumexp(logits, 1)
    some = targets != ignore
    bad = some & ((targets < 0) | (targets >= w.shape[0]))
    at = torch.where(some & ~bad, targets, 0)
    loss = torch.where(some, lse - logits.gather(1, at.unsqueeze(1)).squeeze(1), 0.0)
    return torch.where(bad, float("nan"), loss), lse


def cross_entropy_grad(h, w, targets, grad_loss, ignore):
    """P, the gradient of the logits, by the formula: (softmax - target) times
    each loss's gradient, 0 for tokens without a target; the sums of the
    magnitudes follow from it."""
    p = torch.softmax(h.double() @ w.double().t(), 1)
    some = targets != ignore
    p[some, targets[some]] -= 1.0
    return p * torch.where(some, grad_loss.double(), 0.0).unsqueeze(1)

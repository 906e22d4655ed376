"""Plain 64-bit implementations of the operators that mix a chain's tokens, on
the CPU, with bounds on the error of a computation in 32 bits whose
probabilities are rounded to the tensors' type."""
import math

import torch

import ops_model as m

U32 = m.U32


def visible(batch, tokens, keys, window, sinks, positions=None, lengths=None):
    """[batch, tokens, keys]: which keys a row sees."""
    off = torch.full((batch,), keys - tokens) if positions is None else positions.cpu().long()
    end = torch.full((batch,), keys) if lengths is None else lengths.cpu().long().clamp(0, keys)
    p = off[:, None, None] + torch.arange(tokens)[None, :, None]
    j = torch.arange(keys)[None, None]
    see = (j <= p) & (p < end[:, None, None]) & (p >= 0)
    if window is not None:
        see &= (p - j < window) | (j < sinks)
    return see


def attention(q, k, v, window=None, sinks=0, scale=None, positions=None, lengths=None, dout=None):
    """out and lse, and with dout the gradients dq, dk, dv: (values, bounds),
    dicts of 64-bit tensors.  Inputs are those of the call, on the CPU."""
    dtype = q.dtype
    unit, f16 = m.UNIT[dtype], dtype == torch.float16
    # probabilities and gradients of scores are rounded to 16 bits; in 32 bits
    # they are not rounded again
    round_p = unit if dtype != torch.float32 else 0.0
    b, n, h, d = q.shape
    keys, hk = k.shape[1], k.shape[2]
    g = h // hk
    scale = d ** -0.5 if scale is None else scale
    see = visible(b, n, keys, window, sinks, positions, lengths)[:, None]
    some = see.any(-1, keepdim=True)
    q, k, v = (x.double().permute(0, 2, 1, 3) for x in (q, k, v))
    some_row = some.expand(b, h, n, 1)
    # what a row without a place holds, and a key that no row sees, does not count
    q = torch.where(some_row, q, 0.0)
    seen_key = see.any(2)[:, 0].view(b, 1, keys, 1)
    k, v = torch.where(seen_key, k, 0.0), torch.where(seen_key, v, 0.0)
    kk, vv = k.repeat_interleave(g, 1), v.repeat_interleave(g, 1)
    s = scale * q @ kk.transpose(-1, -2)
    s = s.masked_fill(~see, -math.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.where(see, torch.exp(s - torch.where(some, lse.unsqueeze(-1), 0.0)), 0.0)
    out = p @ vv
    # relative error of a probability: its score (width products and the
    # rounding of the scale, in units of the sum of their magnitudes), the
    # exponential's argument, the sum over the keys, 32 more roundings
    size = (scale * q.abs() @ kk.abs().transpose(-1, -2)).masked_fill(~see, 0.0).amax(-1, keepdim=True)
    e = U32 * ((d + 16) * size + keys + 32)
    tiny = 2.0 ** -25 if f16 else 0.0  # of a probability below float16's normal numbers
    rough = p * (round_p + e) + tiny * see
    bound_out = rough @ vv.abs() + U32 * keys * (p @ vv.abs())
    back = lambda x: x.permute(0, 2, 1, 3).contiguous()
    val = {"out": back(out), "lse": lse.permute(0, 2, 1).contiguous()}
    err = {"out": back(bound_out), "lse": (e.squeeze(-1) + 8 * U32 * lse.abs().nan_to_num(posinf=0.0)).permute(0, 2, 1)}
    if dout is None:
        return val, err
    do = torch.where(some_row, dout.double().permute(0, 2, 1, 3), 0.0)
    dp = do @ vv.transpose(-1, -2)
    delta = (do * out).sum(-1, keepdim=True)
    ds = p * (dp - delta)
    # delta comes from out as it was rounded
    err_delta = (do.abs() * (unit * out.abs() + (1 + unit) * bound_out)).sum(-1, keepdim=True)
    err_delta = err_delta + U32 * (d + 2) * (do * out).abs().sum(-1, keepdim=True)
    err_dp = U32 * (d + 2) * (do.abs() @ vv.abs().transpose(-1, -2))
    err_ds = p * ((round_p + e) * (dp - delta).abs() + (1 + unit) * (1 + e) * (err_dp + err_delta)) * see
    if f16:
        # a gradient of a score is scaled so that its step below the normal
        # numbers is at most 2^-25 2^6 of the largest |do| of its rows, or of
        # those of the rows summed with it
        err_ds = err_ds + 2.0 ** -19 * do.abs().amax((-1, -2), keepdim=True) * see
    heads = lambda x: x.reshape(b, hk, g, *x.shape[2:]).sum(2)
    val["dq"] = back(scale * ds @ kk)
    val["dk"] = back(heads(scale * ds.transpose(-1, -2) @ q))
    val["dv"] = back(heads(p.transpose(-1, -2) @ do))
    many = U32 * (keys + n * g + 8)
    err["dq"] = back(scale * (err_ds + many * ds.abs()) @ kk.abs())
    err["dk"] = back(heads(scale * (err_ds + many * ds.abs()).transpose(-1, -2) @ q.abs()))
    err["dv"] = back(heads((rough + many * p).transpose(-1, -2) @ do.abs()))
    return val, err


def rotation(x, weight, norm, eps, positions, rotary, base=1e4, frequencies=None, interleaved=False):
    """Heads [batch, tokens, heads, width], normed, weighted and turned."""
    x = x.double()
    if norm == "layer":
        x = x - x.mean(-1, keepdim=True)
    if norm != "none":
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    if weight is not None:
        x = x * weight.double()
    if frequencies is None:
        frequencies = [base ** (-2.0 * i / rotary) for i in range(rotary // 2)]
    t = positions.double()[..., None, None] * torch.tensor(frequencies, dtype=torch.float64)
    a, b = (x[..., :rotary:2], x[..., 1:rotary:2]) if interleaved else \
        (x[..., :rotary // 2], x[..., rotary // 2:rotary])
    u, w = a * torch.cos(t) - b * torch.sin(t), b * torch.cos(t) + a * torch.sin(t)
    turned = torch.stack([u, w], -1).flatten(-2) if interleaved else torch.cat([u, w], -1)
    return torch.cat([turned, x[..., rotary:]], -1)

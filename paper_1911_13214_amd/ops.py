"""Operators of a language-model chain's stages, on the C ABI in
include/rotor.h: counter-based dropout, embedding lookup, the residual seam
between two blocks (norms, gate, residual scale), the cross entropy over a
vocabulary without its logits, and their gradients.

Argument checks, allocation and marshalling only: every operator runs in the
library's HIP kernels.  Tensors are CUDA tensors of one device and, where
floating-point, of one type (float32, bfloat16 or float16); a matrix may have
any row pitch, its last dimension is dense.  Calls enqueue on ``stream``
(default: the current one) and return at once; a tensor that was made on
another stream is the caller's to order and to keep (``record_stream``), and
so is the order of a result's use on another one.  What a call allocates,
results and scratch, comes from torch's caching allocator for the stream it
runs on; results are recorded for the caller's current stream as well.  Results
are allocated unless ``out`` is given.

``stages`` wraps these in autograd functions and modules."""
from __future__ import annotations

import ctypes
import functools

import torch

from . import rotor

TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
NORMS = {"none": 0, "rms": 1, "layer": 2}
NORM_MAX_COLS = 16384


class _Norm(ctypes.Structure):
    _fields_ = [("type", ctypes.c_int32), ("post", ctypes.c_int32), ("pre", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("gate_rows", ctypes.c_int64), ("gate_pitch", ctypes.c_int64), ("residual_scale", ctypes.c_double),
                ("eps", ctypes.c_double), ("post_weight", ctypes.c_void_p), ("post_bias", ctypes.c_void_p),
                ("gate", ctypes.c_void_p), ("pre_weight", ctypes.c_void_p), ("pre_bias", ctypes.c_void_p)]


class _NormGrads(ctypes.Structure):
    _fields_ = [("post_weight", ctypes.c_void_p), ("post_bias", ctypes.c_void_p), ("gate", ctypes.c_void_p),
                ("pre_weight", ctypes.c_void_p), ("pre_bias", ctypes.c_void_p), ("gate_pitch", ctypes.c_int64)]


# ---- checks --------------------------------------------------------------------

def _cuda(t, what):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{what} must be a CUDA tensor")
    return t


def _typed(t, what):
    """The C ABI's code of a floating-point tensor's type."""
    code = TYPES.get(_cuda(t, what).dtype)
    if code is None:
        raise ValueError(f"{what} must be float32, bfloat16 or float16, not {t.dtype}")
    return code


def _like(t, other, what, shape=None):
    """``t`` checked to have ``other``'s device and type, and a shape."""
    _cuda(t, what)
    if t.device != other.device or t.dtype != other.dtype:
        raise ValueError(f"{what} must be {other.dtype} on {other.device}")
    shape = other.shape if shape is None else shape
    if t.shape != shape:
        raise ValueError(f"{what} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    return t


def _matrix(t, what):
    """(rows, cols, pitch) of a tensor whose leading dimensions are rows."""
    shape = t.shape
    if not shape:
        raise ValueError(f"{what} needs at least one dimension")
    cols = shape[-1]
    if cols == 0:
        raise ValueError(f"{what} has no columns")
    rows = t.numel() // cols
    if t.is_contiguous():
        return rows, cols, cols
    if t.dim() == 1:
        t = t.unsqueeze(0)
    elif t.dim() > 2:
        try:
            t = t.view(rows, cols)
        except RuntimeError:
            raise ValueError(f"the leading dimensions of {what} must be one row pitch apart") from None
    pitch = t.stride(0) if rows > 1 else cols
    if (cols > 1 and t.stride(1) != 1) or pitch < cols:
        raise ValueError(f"{what} must have a dense last dimension and rows that do not overlap")
    return rows, cols, pitch


def _empty(like):
    """A dense tensor of another's shape, type and device."""
    return torch.empty_like(like, memory_format=torch.contiguous_format)


def _out(out, like, what, shape=None):
    if out is None:
        return _empty(like) if shape is None else like.new_empty(shape)
    return _like(out, like, what, shape)


def _ptr(t):
    return None if t is None else t.data_ptr()


@functools.lru_cache(maxsize=None)
def _entry(name):
    return getattr(rotor.lib(), name)


def _on(stream, f, *args, **kw):
    """A call on the stream it is given: that stream is the current one while
    it allocates and launches, since a block of another stream's pool may still
    be in use there.  Results are free to be used, and freed, on the caller's."""
    for t in args:
        if isinstance(t, torch.Tensor) and t.device != stream.device:
            raise ValueError(f"stream is one of {stream.device}, a tensor is on {t.device}")
    here = torch.cuda.current_stream(stream.device)
    with torch.cuda.stream(stream):
        out = f(*args, **kw)
    for t in out.values() if isinstance(out, dict) else out if isinstance(out, tuple) else (out,):
        if t is not None:
            t.record_stream(here)
    return out


def _call(name, device, *args):
    """One entry point of the library, on the device's current stream."""
    index = device.index
    raw = torch._C._cuda_getCurrentRawStream(index)
    if index == torch._C._cuda_getDevice():
        status = _entry(name)(*args, raw)
    else:
        with torch.cuda.device(device):
            status = _entry(name)(*args, raw)
    if status != rotor.ROTOR_OK:
        raise rotor.RotorError(status, name)


@functools.lru_cache(maxsize=4096)
def _workspace_bytes(name, *sizes):
    """Workspace of an entry point for these sizes (a function of them alone)."""
    need = ctypes.c_uint64()
    rotor._check(_entry(name)(*sizes, ctypes.byref(need)), name)
    return need.value


def _scratch(nbytes, like):
    """Device scratch of a call, returned to the allocator when it ends: what is
    allocated there next is used after it, on the same stream."""
    return like.new_empty(max(nbytes, 16), dtype=torch.uint8)


# ---- dropout ---------------------------------------------------------------------

def dropout(x, p, seed, step=0, residual=None, *, step_tensor=None, out=None, stream=None):
    """residual + keep * x / (1 - q), q = round(65536 p) / 65536, the mask a
    function of (seed, step) and the element's index alone: the same call on
    the gradient of the result (without residual) is the gradient of ``x``.

    ``seed``, ``step``: integers, taken modulo 2^64.  ``step_tensor``: an int64
    device tensor of one element added to ``step`` (for captured graphs).
    ``out`` may be ``x`` or ``residual``."""
    if stream is not None:
        return _on(stream, dropout, x, p, seed, step, residual, step_tensor=step_tensor, out=out)
    code = _typed(x, "x")
    if not 0.0 <= p <= 1.0:
        raise ValueError(f"p must lie in [0, 1], not {p}")
    if step_tensor is not None and (not isinstance(step_tensor, torch.Tensor) or step_tensor.device != x.device or
                                    step_tensor.dtype != torch.int64 or step_tensor.numel() != 1):
        raise ValueError("step_tensor must be one int64 on the device of x")
    y = _out(out, x, "out")
    if residual is not None:
        _like(residual, x, "residual")
    n = x.numel()
    if n == 0:
        return y
    if x.is_contiguous() and y.is_contiguous() and (residual is None or residual.is_contiguous()):
        rows, cols, xp, yp, rp = 1, n, n, n, n
    else:
        rows, cols, xp = _matrix(x, "x")
        _, _, yp = _matrix(y, "out")
        rp = _matrix(residual, "residual")[2] if residual is not None else cols
    _call("rotor_dropout", x.device, code, rows, cols, x.data_ptr(), xp, _ptr(residual), rp, y.data_ptr(), yp,
          p, seed & 0xFFFFFFFFFFFFFFFF, step & 0xFFFFFFFFFFFFFFFF, _ptr(step_tensor))
    return y


# ---- embedding -------------------------------------------------------------------

def _tokens(tokens, device):
    _cuda(tokens, "tokens")
    if tokens.dtype not in (torch.int64, torch.int32) or tokens.device != device or not tokens.is_contiguous():
        raise ValueError(f"tokens must be contiguous int64 or int32 on {device}")
    return tokens.element_size()


def embedding(tokens, table, scale=1.0, *, out=None, stream=None):
    """scale * table[tokens], of shape [*tokens.shape, cols].  A token outside
    the table gives a row of NaN."""
    if stream is not None:
        return _on(stream, embedding, tokens, table, scale, out=out)
    code = _typed(table, "table")
    if table.dim() != 2:
        raise ValueError("table must have two dimensions")
    size = _tokens(tokens, table.device)
    rows, cols, pitch = _matrix(table, "table")
    y = _out(out, table, "out", tokens.shape + (cols,))
    if tokens.numel() == 0:
        return y
    _call("rotor_embedding", table.device, code, tokens.numel(), rows, cols, tokens.data_ptr(), size,
          table.data_ptr(), pitch, scale, y.data_ptr(), _matrix(y, "out")[2])
    return y


def embedding_backward(tokens, grad, n_rows, scale=1.0, *, padding=None, out=None, stream=None):
    """Gradient [n_rows, cols] of the table from the gradient of
    ``embedding(tokens, table, scale)``: every row written, that of the token
    ``padding`` 0.  Bit for bit the same on every call."""
    if stream is not None:
        return _on(stream, embedding_backward, tokens, grad, n_rows, scale, padding=padding, out=out)
    code = _typed(grad, "grad")
    size = _tokens(tokens, grad.device)
    if grad.dim() < 1 or grad.shape[:-1] != tokens.shape:
        raise ValueError(f"grad must have shape {tuple(tokens.shape)} + (cols,)")
    n, (_, cols, pitch) = tokens.numel(), _matrix(grad, "grad")
    out = _out(out, grad, "out", (n_rows, cols))
    work = _scratch(_workspace_bytes("rotor_embedding_workspace_bytes", n, n_rows, cols), grad)
    _call("rotor_embedding_backward", grad.device, code, n, n_rows, cols, _ptr(tokens), size, _ptr(grad),
          pitch, scale, -1 if padding is None else padding, out.data_ptr(), _matrix(out, "out")[2], work.data_ptr(),
          work.numel())
    return out


# ---- residual norm ------------------------------------------------------------------

def _norm(x, z, post, post_weight, post_bias, gate, residual_scale, pre, pre_weight, pre_bias, eps):
    """The C ABI's description of a seam, checked against ``x``."""
    code = _typed(x, "x")
    if post not in NORMS or pre not in NORMS:
        raise ValueError(f"post and pre must be one of {tuple(NORMS)}")
    cols = x.shape[-1] if x.dim() else 0
    if not 1 <= cols <= NORM_MAX_COLS:
        raise ValueError(f"the last dimension must lie in [1, {NORM_MAX_COLS}]")
    if not eps >= 0.0:
        raise ValueError("eps must not be negative")
    rows = x.numel() // cols
    if z is None and (post != "none" or gate is not None):
        raise ValueError("post and gate need z")
    at = []
    for name, q, kind in (("post_weight", post_weight, post), ("post_bias", post_bias, post),
                          ("pre_weight", pre_weight, pre), ("pre_bias", pre_bias, pre)):
        if q is None:
            at.append(None)
            continue
        if kind == "none":
            raise ValueError(f"{name} without its norm")
        if not _like(q, x, name, (cols,)).is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        at.append(q.data_ptr())
    n = _Norm(code, NORMS[post], NORMS[pre], 0, rows, cols, 0, 0, residual_scale, eps, at[0], at[1], None, at[2], at[3])
    if gate is not None:
        g_rows, g_cols, n.gate_pitch = _matrix(_cuda(gate, "gate"), "gate")
        if gate.dtype != x.dtype or gate.device != x.device or g_cols != cols or g_rows < 1 or rows % g_rows:
            raise ValueError(f"gate must be {x.dtype} on {x.device}, [n, {cols}] with n dividing the {rows} rows")
        n.gate_rows, n.gate = g_rows, gate.data_ptr()
    return n


def residual_norm(x, z=None, *, post="none", post_weight=None, post_bias=None, gate=None, residual_scale=1.0,
                  pre="none", pre_weight=None, pre_bias=None, eps=1e-5, stats=True, stream=None):
    """y = residual_scale * x + gate * post(z) and h = pre(y): returns
    (y, h, stats), h None without ``pre``.

    ``post``, ``pre``: "none", "rms" or "layer", each with an optional weight
    and bias [cols]; ``gate``: [cols], or [..., cols] of n rows where n divides
    the rows of x (one row of gates for each run of rows / n adjacent rows);
    ``z`` None: no block, y = residual_scale * x (``x`` itself if that is 1).
    ``stats``: keep what the backward needs (16 bytes a row), or None is
    returned."""
    if stream is not None:
        return _on(stream, residual_norm, x, z, post=post, post_weight=post_weight, post_bias=post_bias, gate=gate,
                   residual_scale=residual_scale, pre=pre, pre_weight=pre_weight, pre_bias=pre_bias, eps=eps,
                   stats=stats)
    n = _norm(x, z, post, post_weight, post_bias, gate, residual_scale, pre, pre_weight, pre_bias, eps)
    xp = _matrix(x, "x")[2]
    zp = _matrix(_like(z, x, "z"), "z")[2] if z is not None else n.cols
    copy = z is not None or residual_scale != 1.0
    y = _empty(x) if copy else x
    h = _empty(x) if pre != "none" else None
    st = x.new_empty((n.rows, 4), dtype=torch.float32) if stats else None
    _call("rotor_residual_norm", x.device, ctypes.byref(n), x.data_ptr(), xp, _ptr(z), zp,
          y.data_ptr() if copy else None, n.cols, _ptr(h), n.cols, _ptr(st))
    return y, h, st


def residual_norm_backward(dy, dh, y, z, stats, *, post="none", post_weight=None, post_bias=None, gate=None,
                           residual_scale=1.0, pre="none", pre_weight=None, pre_bias=None, eps=1e-5, stream=None):
    """Gradients of residual_norm's arguments from those of y (``dy``, None:
    0) and h (``dh``, None without ``pre``), as a dict: "x", "z" and the
    parameters that are given."""
    if stream is not None:
        return _on(stream, residual_norm_backward, dy, dh, y, z, stats, post=post, post_weight=post_weight,
                   post_bias=post_bias, gate=gate, residual_scale=residual_scale, pre=pre, pre_weight=pre_weight,
                   pre_bias=pre_bias, eps=eps)
    lead = dy if dy is not None else dh
    if lead is None:
        raise ValueError("dy or dh is needed")
    n = _norm(lead, z, post, post_weight, post_bias, gate, residual_scale, pre, pre_weight, pre_bias, eps)
    if (dh is not None) != (pre != "none"):
        raise ValueError("dh goes with pre")
    if dh is not None:
        _like(dh, lead, "dh")
        _like(y, lead, "y")
    _cuda(stats, "stats")
    if stats.shape != (n.rows, 4) or stats.dtype != torch.float32 or not stats.is_contiguous() or \
            stats.device != lead.device:
        raise ValueError("stats must be what residual_norm returned")

    def matrix(t, what):
        return (None, n.cols) if t is None else (t.data_ptr(), _matrix(_like(t, lead, what), what)[2])

    g = {"x": _empty(lead)}
    if z is not None:
        g["z"] = _empty(lead)
    for name, q in (("pre_weight", pre_weight), ("pre_bias", pre_bias), ("post_weight", post_weight),
                    ("post_bias", post_bias), ("gate", gate)):
        if q is not None:
            g[name] = _empty(q)
    out = _NormGrads(gate_pitch=n.cols, **{k: g[k].data_ptr() for k in g if k not in ("x", "z")})
    need = ctypes.c_uint64()
    rotor._check(_entry("rotor_residual_norm_workspace_bytes")(ctypes.byref(n), ctypes.byref(need)),
                 "rotor_residual_norm_workspace_bytes")
    work = _scratch(need.value, lead)
    _call("rotor_residual_norm_backward", lead.device, ctypes.byref(n), *matrix(dy, "dy"), *matrix(dh, "dh"),
          *(matrix(y, "y") if dh is not None else (None, n.cols)), *matrix(z, "z"), stats.data_ptr(),
          g["x"].data_ptr(), n.cols, _ptr(g.get("z")), n.cols, ctypes.byref(out), work.data_ptr(), work.numel())
    return g


# ---- cross entropy ---------------------------------------------------------------------

XENT_MAX_TOKENS, XENT_MAX_COLS, XENT_MAX_ROWS = 1 << 20, 65536, 1 << 26


def _xent(h, w, targets, backward):
    """Checked sizes, pitches and workspace of a cross entropy."""
    code = _typed(h, "h")
    if h.dim() < 1 or w.dim() != 2 or h.shape[-1] != w.shape[1]:
        raise ValueError("h and w must have the same columns, w two dimensions")
    if _cuda(w, "w").dtype != h.dtype or w.device != h.device:
        raise ValueError(f"w must be {h.dtype} on {h.device}")
    if not isinstance(targets, torch.Tensor) or targets.dtype != torch.int64 or targets.device != h.device or \
            targets.shape != h.shape[:-1] or not targets.is_contiguous():
        raise ValueError(f"targets must be contiguous int64 on {h.device}, one for each row of h")
    n, cols, hp = _matrix(h, "h")
    rows, _, wp = _matrix(w, "w")
    if not 1 <= rows <= XENT_MAX_ROWS or n > XENT_MAX_TOKENS or cols > XENT_MAX_COLS:
        raise ValueError(f"at most {XENT_MAX_TOKENS} tokens, {XENT_MAX_COLS} columns, {XENT_MAX_ROWS} rows of w, and "
                         "at least one")
    aligned = int(not (cols % 8 or hp % 8 or wp % 8 or h.data_ptr() % 16 or w.data_ptr() % 16))
    need = _workspace_bytes("rotor_xent_workspace_bytes", code, n, cols, rows, aligned, backward)
    return code, n, cols, rows, hp, wp, aligned, _scratch(need, h)


def _per_token(t, targets, what):
    if not isinstance(t, torch.Tensor) or t.dtype != torch.float32 or t.device != targets.device or \
            t.shape != targets.shape or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous float32 on {targets.device}, shaped as targets")
    return t.data_ptr()


def linear_cross_entropy(h, w, targets, ignore=-100, *, stream=None):
    """Loss and log-sum-exp of each token, float32, shaped as ``targets``: the
    softmax cross entropy of the logits h w^T, which never exist whole.
    Tokens with target ``ignore`` have loss 0; other targets outside the rows
    of w give NaN."""
    if stream is not None:
        return _on(stream, linear_cross_entropy, h, w, targets, ignore)
    code, n, cols, rows, hp, wp, aligned, work = _xent(h, w, targets, 0)
    loss, lse = (torch.empty_like(targets, dtype=torch.float32) for _ in range(2))
    _call("rotor_xent", h.device, code, n, cols, rows, h.data_ptr(), hp, w.data_ptr(), wp, targets.data_ptr(),
          ignore, loss.data_ptr(), lse.data_ptr(), aligned, work.data_ptr(), work.numel())
    return loss, lse


def linear_cross_entropy_backward(h, w, targets, lse, grad_loss, ignore=-100, *, need_h=True, need_w=True,
                                  stream=None):
    """Gradients of h and w from those of the losses (float32, shaped as
    ``targets``) and the log-sum-exps of the forward; None where not needed."""
    if stream is not None:
        return _on(stream, linear_cross_entropy_backward, h, w, targets, lse, grad_loss, ignore, need_h=need_h,
                   need_w=need_w)
    if not (need_h or need_w):
        return None, None
    code, n, cols, rows, hp, wp, aligned, work = _xent(h, w, targets, 1)
    lse, grad_loss = _per_token(lse, targets, "lse"), _per_token(grad_loss, targets, "grad_loss")
    dh = _empty(h) if need_h else None
    dw = _empty(w) if need_w else None
    _call("rotor_xent_backward", h.device, code, n, cols, rows, h.data_ptr(), hp, w.data_ptr(), wp,
          targets.data_ptr(), ignore, lse, grad_loss, _ptr(dh), cols, _ptr(dw), cols, aligned, work.data_ptr(),
          work.numel())
    return dh, dw

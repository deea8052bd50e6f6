"""Tensor conveniences over the sequence operators' C ABI (device pointers and
streams only): the gated linear recurrence along the tokens, and the norms
before and after a block with its gate and scaled residual.

Activations are float32, float16 or bfloat16 tensors whose last axis is
consecutive in memory (the other axes may be strided: slices of a wider
projection need no copy); weights, states and statistics are contiguous
float32.  Every function runs on the current stream, or on ``stream``.
``gated_scan_train`` and ``residual_norm_train`` are the same operators as
autograd functions.
"""
from __future__ import annotations

import torch

from . import _seq_lib as _l
from ._seq_lib import SEQ_SCAN_CHUNK, SeqError  # noqa: F401
from .torch_api import _raw_device, _stream

_TYPES = {torch.float32: _l.SEQ_FP32, torch.float16: _l.SEQ_FP16, torch.bfloat16: _l.SEQ_BF16}
_fp32 = torch.float32


def _type_of(x: torch.Tensor, name: str, dims: int) -> int:
    kind = _TYPES.get(x.dtype)
    if kind is None or not x.is_cuda:
        raise TypeError(f"{name} must be a float32, float16 or bfloat16 GPU tensor")
    if x.dim() != dims:
        raise ValueError(f"{name} must have {dims} axes")
    here = _raw_device() if _raw_device is not None else torch.cuda.current_device()
    if x.get_device() != here:
        raise ValueError(f"{name} must be on the current device")
    return kind


def _activation(t: torch.Tensor, name: str, like: torch.Tensor) -> None:
    if t.dtype != like.dtype or t.device != like.device:
        raise TypeError(f"{name} must have the type and device of the other activations")
    if t.shape != like.shape:
        raise ValueError(f"{name} must have the shape {tuple(like.shape)}")


def _consecutive(t: torch.Tensor, name: str) -> None:
    if t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError(f"the last axis of {name} must be consecutive in memory")


def _weight(t, name: str, shape, like: torch.Tensor, dtype=_fp32):
    """Pointer of an optional contiguous tensor of weights or states."""
    if t is None:
        return None
    if t.dtype != dtype or t.device != like.device:
        raise TypeError(f"{name} must be {dtype} on the device of the activations")
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous with the shape {tuple(shape)}")
    return t.data_ptr()


def _strides(tensors, dims):
    """None where every tensor is contiguous, else the host array of the outer strides."""
    for t in tensors:
        if t is not None and not t.is_contiguous():
            break
    else:
        return None
    return _l.int64s([s for t in tensors for s in (t.stride()[:dims] if t is not None else (0,) * dims)])


def _workspace(nbytes: int, given, like: torch.Tensor, stream):
    """(tensor, pointer) of scratch memory: the caller's, or new memory of the current stream."""
    if nbytes == 0:
        return None, None
    if given is None:
        given = torch.empty(nbytes, dtype=torch.uint8, device=like.device)
        if stream is not None:  # it is given back to the current stream's pool while `stream` may still use it
            given.record_stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(int(stream)))
    elif given.device != like.device or not given.is_contiguous() or given.numel() * given.element_size() < nbytes:
        raise ValueError(f"workspace must be contiguous, of at least {nbytes} bytes, on the device of the activations")
    return given, given.data_ptr()


def gated_scan_saved(x: torch.Tensor) -> torch.Tensor:
    """New memory for the states that ``gated_scan`` saves for its gradient."""
    b, t, d = x.shape
    return torch.empty(b, -(-t // SEQ_SCAN_CHUNK), d, dtype=_fp32, device=x.device)


def gated_scan(x, r, g, rate, state=None, lengths=None, *, out=None, state_out=None, saved=None, workspace=None,
               stream=None):
    """The gated linear recurrence of each channel of (batch, tokens, channels):

        h_t = h_(t-1) + q_t (c_t - h_(t-1)),  q_t = rate sigmoid(r_t),  c_t = sigmoid(g_t) x_t

    Returns (y, state after the last token).  ``state`` (batch, channels) is
    the state before the first token, zeros if None; ``state_out`` may be
    ``state`` itself.  ``lengths`` (batch) int32 are the tokens that count:
    those behind leave the state and give 0.  ``saved`` (``gated_scan_saved``)
    is filled for ``gated_scan_backward``.
    """
    kind = _type_of(x, "x", 3)
    b, t, d = x.shape
    out = torch.empty((b, t, d), dtype=x.dtype, device=x.device) if out is None else out
    for v, name in ((r, "r"), (g, "g"), (out, "out")):
        _activation(v, name, x)
    for v, name in ((x, "x"), (r, "r"), (g, "g"), (out, "out")):
        _consecutive(v, name)
    state_out = torch.empty((b, d), dtype=_fp32, device=x.device) if state_out is None else state_out
    _, ws = _workspace(_l.lib.seq_scan_workspace_bytes(b, t, d, kind, 0), workspace, x, stream)
    if rate is None:
        raise TypeError("rate is missing")
    _l.check(_l.lib.seq_scan_forward(
        b, t, d, kind, x.data_ptr(), r.data_ptr(), g.data_ptr(), _strides((x, r, g, out), 2),
        _weight(rate, "rate", (d,), x), _weight(state, "state", (b, d), x),
        _weight(lengths, "lengths", (b,), x, torch.int32), out.data_ptr(), _weight(state_out, "state_out", (b, d), x),
        _weight(saved, "saved", (b, -(-t // SEQ_SCAN_CHUNK), d), x), ws, _stream(stream)), "seq_scan_forward")
    return out, state_out


def gated_scan_step(x, r, g, rate, state, *, out=None, stream=None):
    """One token (batch, channels) of ``gated_scan``; ``state`` is updated in place.  Returns y."""
    if x.dim() != 2 or r.dim() != 2 or g.dim() != 2:
        raise ValueError("x, r and g must have 2 axes")
    y, _ = gated_scan(x.unsqueeze(1), r.unsqueeze(1), g.unsqueeze(1), rate, state,
                      out=None if out is None else out.unsqueeze(1), state_out=state, stream=stream)
    return y.squeeze(1) if out is None else out


def gated_scan_backward(grad_out, x, r, g, rate, saved, lengths=None, *, grad_state=None, out=(None, None, None),
                        workspace=None, stream=None):
    """Gradient of ``gated_scan``: (dx, dr, dg, drate, dstate) from the
    gradients of y and of the state after the last token (None: zeros).
    ``out``: tensors for dx, dr and dg, slices of one buffer for example."""
    kind = _type_of(x, "x", 3)
    b, t, d = x.shape
    dx, dr, dg = (torch.empty((b, t, d), dtype=x.dtype, device=x.device) if v is None else v for v in out)
    named = ((grad_out, "grad_out"), (x, "x"), (r, "r"), (g, "g"), (dx, "dx"), (dr, "dr"), (dg, "dg"))
    for v, name in named:
        _activation(v, name, x)
        _consecutive(v, name)
    if rate is None or saved is None:
        raise TypeError("rate or saved is missing")
    drate = torch.empty(d, dtype=_fp32, device=x.device)
    dstate = torch.empty((b, d), dtype=_fp32, device=x.device)
    _, ws = _workspace(_l.lib.seq_scan_workspace_bytes(b, t, d, kind, 1), workspace, x, stream)
    _l.check(_l.lib.seq_scan_backward(
        b, t, d, kind, grad_out.data_ptr(), x.data_ptr(), r.data_ptr(), g.data_ptr(),
        _strides((grad_out, x, r, g, dx, dr, dg), 2), _weight(rate, "rate", (d,), x),
        _weight(saved, "saved", (b, -(-t // SEQ_SCAN_CHUNK), d), x), _weight(lengths, "lengths", (b,), x, torch.int32),
        _weight(grad_state, "grad_state", (b, d), x), dx.data_ptr(), dr.data_ptr(), dg.data_ptr(), drate.data_ptr(),
        dstate.data_ptr(), ws, _stream(stream)), "seq_scan_backward")
    return dx, dr, dg, drate, dstate


def residual_norm_stats(x: torch.Tensor) -> torch.Tensor:
    """New memory for the row statistics that ``residual_norm`` saves for its gradient."""
    return torch.empty((*x.shape[:-1], 2), dtype=_fp32, device=x.device)


def _rows(t):
    """A tensor as (rows, channels) without a copy."""
    if t is None or t.dim() == 2:
        return t
    return t.view(-1, t.shape[-1]) if t.dim() > 2 else t.view(1, -1)


def residual_norm(x, y=None, z=None, post=None, scale=None, pre=None, *, eps: float, out=None, normed=None, stats=None,
                  stream=None):
    """The end of a block and the beginning of the next one, over the last axis:

        o = x + scale post (y / rms(y)) silu(z),  n = pre o / rms(o)

    Returns (o, n).  Without ``y`` there is no block and o is x (the first norm
    of a model); ``z`` None: no gate; ``scale`` None: 1; ``pre`` None: n is
    None.  ``stats`` (``residual_norm_stats``) is filled for
    ``residual_norm_backward``.
    """
    shape = x.shape
    x2, y2, z2, o2, n2 = _rows(x), _rows(y), _rows(z), _rows(out), _rows(normed)
    kind = _type_of(x2, "x", 2)
    rows, d = x2.shape
    if y is not None and o2 is None:
        o2 = torch.empty((rows, d), dtype=x.dtype, device=x.device)
    if pre is not None and n2 is None:
        n2 = torch.empty((rows, d), dtype=x.dtype, device=x.device)
    tensors = (x2, y2, z2, o2, n2)
    for v, name in zip(tensors, ("x", "y", "z", "out", "normed")):
        if v is not None:
            _activation(v, name, x2)
            _consecutive(v, name)
    _l.check(_l.lib.seq_norm_forward(
        rows, d, kind, x2.data_ptr(), _ptr(y2), _ptr(z2), _strides(tensors, 1), _weight(post, "post", (d,), x2),
        _weight(scale, "scale", (d,), x2), _weight(pre, "pre", (d,), x2), eps, _ptr(o2), _ptr(n2),
        _weight(stats, "stats", (*shape[:-1], 2), x2), _stream(stream)), "seq_norm_forward")
    return (x if y is None else o2.view(shape) if out is None else out,
            None if pre is None else n2.view(shape) if normed is None else normed)


def _ptr(t):
    return None if t is None else t.data_ptr()


def residual_norm_backward(grad_out, grad_normed, x, y, z, post, scale, pre, stats, *, eps: float,
                           out=(None, None, None), workspace=None, stream=None):
    """Gradient of ``residual_norm``: (dx, dy, dz, dpost, dscale, dpre), None
    where the argument is.  ``grad_out`` may be None (zeros), ``grad_normed``
    is None where ``pre`` is.  ``out``: tensors for dx, dy and dz."""
    shape = x.shape
    go, gn, x2, y2, z2, dx, dy, dz = (_rows(v) for v in (grad_out, grad_normed, x, y, z, *out))
    kind = _type_of(x2, "x", 2)
    rows, d = x2.shape
    dx, dy, dz = (torch.empty((rows, d), dtype=x.dtype, device=x.device) if v is None and of is not None else v
                  for v, of in ((dx, x2), (dy, y2), (dz, z2)))
    tensors = (go, gn, x2, y2, z2, dx, dy, dz)
    for v, name in zip(tensors, ("grad_out", "grad_normed", "x", "y", "z", "dx", "dy", "dz")):
        if v is not None:
            _activation(v, name, x2)
            _consecutive(v, name)
    grads = [None if w is None else torch.empty(d, dtype=_fp32, device=x.device) for w in (post, scale, pre)]
    _, ws = _workspace(_l.lib.seq_norm_workspace_bytes(rows, d, kind), workspace, x2, stream)
    if stats is None:
        raise TypeError("stats is missing")
    _l.check(_l.lib.seq_norm_backward(
        rows, d, kind, _ptr(go), _ptr(gn), x2.data_ptr(), _ptr(y2), _ptr(z2), _strides(tensors, 1),
        _weight(post, "post", (d,), x2), _weight(scale, "scale", (d,), x2), _weight(pre, "pre", (d,), x2), eps,
        _weight(stats, "stats", (*shape[:-1], 2), x2), dx.data_ptr(), _ptr(dy), _ptr(dz), *map(_ptr, grads), ws,
        _stream(stream)), "seq_norm_backward")
    dx, dy, dz = (None if v is None else v.view(shape) if given is None else given for v, given in zip((dx, dy, dz), out))
    return (dx, dy, dz, *grads)


class _GatedScan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, r, g, rate, state, lengths):
        saved = gated_scan_saved(x)
        y, last = gated_scan(x, r, g, rate, state, lengths, saved=saved)
        ctx.save_for_backward(x, r, g, rate, saved, lengths)
        ctx.set_materialize_grads(False)
        return y, last

    @staticmethod
    def backward(ctx, grad_y, grad_last):
        x, r, g, rate, saved, lengths = ctx.saved_tensors
        grad_y = torch.zeros_like(x) if grad_y is None else grad_y if grad_y.stride(-1) == 1 else grad_y.contiguous()
        if grad_last is not None:
            grad_last = grad_last.contiguous()
        grads = gated_scan_backward(grad_y, x, r, g, rate, saved, lengths, grad_state=grad_last)
        return tuple(v if need else None for v, need in zip((*grads, None), ctx.needs_input_grad))


class _ResidualNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, y, z, post, scale, pre, eps):
        stats = residual_norm_stats(x)
        out, normed = residual_norm(x, y, z, post, scale, pre, eps=eps, stats=stats)
        ctx.save_for_backward(x, y, z, post, scale, pre, stats)
        ctx.eps = eps
        ctx.set_materialize_grads(False)
        return (normed,) if y is None else (out, normed) if pre is not None else (out,)

    @staticmethod
    def backward(ctx, *grads):
        x, y, z, post, scale, pre, stats = ctx.saved_tensors
        grad_out, grad_normed = None if y is None else grads[0], None if pre is None else grads[-1]
        if pre is not None and grad_normed is None:
            grad_normed = torch.zeros_like(x)
        grad_out, grad_normed = (None if v is None else v.contiguous() for v in (grad_out, grad_normed))
        found = residual_norm_backward(grad_out, grad_normed, x, y, z, post, scale, pre, stats, eps=ctx.eps)
        return tuple(v if need else None for v, need in zip((*found, None), ctx.needs_input_grad))


def gated_scan_train(x, r, g, rate, state=None, lengths=None):
    """``gated_scan`` with a gradient for x, r, g, rate and state: (y, state after the last token)."""
    return _GatedScan.apply(x, r, g, rate, state, lengths)


def residual_norm_train(x, y=None, z=None, post=None, scale=None, pre=None, *, eps: float):
    """``residual_norm`` with a gradient for every tensor: (o, n); n is None without ``pre``."""
    got = _ResidualNorm.apply(x, y, z, post, scale, pre, eps)
    return (x, got[0]) if y is None else (got[0], got[1] if pre is not None else None)

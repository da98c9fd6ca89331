"""The head operators of include/rrm.h on torch tensors: group normalisation with an activation, the gated feed-forward
block and the gated recurrence over frames, each with its backward pass.

Argument marshalling only, as in binding.py: sizes and strides come from the tensors, outputs and workspaces that are not
given are allocated by torch (on the stream the call runs on, so a captured call has its own), and everything else is the C
call.  Tensors must lie on the current device; what the library does not take raises RRMError before anything is launched."""
import contextlib
import ctypes

import torch

from . import binding as _b
from .binding import RRMError, NormDesc, FfDesc, ScanDesc, ACT, lib

_DTYPE = {torch.float32: 0, torch.bfloat16: 3, torch.float16: 4}


def _need(ok, what):
    if not ok:
        raise RRMError(what)


def _on_device(name, dtype, **tensors):
    """Every given tensor on the current device and of `dtype`."""
    for k, t in tensors.items():
        if t is None:
            continue
        _need(isinstance(t, torch.Tensor) and t.is_cuda and t.get_device() == torch.cuda.current_device(),
              f"{name}: {k} must be a tensor on the current CUDA device")
        _need(t.dtype == dtype, f"{name}: {k} must be {dtype}, is {t.dtype}")


def _dense(name, shape, **tensors):
    for k, t in tensors.items():
        _need(t is None or (tuple(t.shape) == tuple(shape) and t.is_contiguous()),
              f"{name}: {k} must be a contiguous tensor of shape {tuple(shape)}")


def _axis(name, t, first, last):
    """The stride that runs through axes first .. last - 1 of t as through one axis, innermost fastest (0: at most one element)."""
    step, span = 0, 1
    for i in reversed(range(first, last)):
        if t.shape[i] == 1:
            continue
        if span == 1:
            step = t.stride(i)
        _need(t.stride(i) == step * span and step > 0, f"{name}: the axes {first} to {last - 1} of a tensor of strides {t.stride()} are not one axis")
        span *= t.shape[i]
    return step


def _inner(name, t):
    _need(t.dim() >= 1 and (t.shape[-1] <= 1 or t.stride(-1) == 1), f"{name}: the last axis must be contiguous")


@contextlib.contextmanager
def _on_stream(stream):
    """The raw stream a call runs on; torch allocates for that stream meanwhile."""
    handle = _b._stream(stream)
    if stream is None or handle == torch.cuda.current_stream().cuda_stream:
        yield handle
    else:
        with torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(handle)):
            yield handle


def _workspace(name, fn, desc, backward):
    n = fn(ctypes.byref(desc), backward)
    if n < 0:
        _b._check(int(n), name)
    return torch.empty(n, dtype=torch.uint8, device="cuda") if n else None, n


# ---- group normalisation with an activation ------------------------------------------------------------------------

def _norm_desc(name, x, groups, act, eps):
    _need(isinstance(x, torch.Tensor) and x.dim() >= 2, f"{name}: x is [images, ..., channels]")
    _need(x.dtype in _DTYPE, f"{name}: x must be float32, bfloat16 or float16, is {x.dtype}")
    _need(act in ACT, f"{name}: unknown activation {act!r}")
    d = NormDesc()
    d.dtype, d.act, d.n, d.c, d.groups, d.eps = _DTYPE[x.dtype], ACT[act], x.shape[0], x.shape[-1], int(groups), float(eps)
    d.pixels = x[0].numel() // x.shape[-1] if x.numel() else 0
    return d


def _norm_strides(name, t):
    _inner(name, t)
    return (_axis(name, t, 1, t.dim() - 1), _axis(name, t, 0, 1)) if t.numel() else (0, 0)


def group_norm(x, groups, gamma=None, beta=None, eps=1e-5, act="none", y=None, stats=None, stream=None):
    """rrm_group_norm: (y, stats) of x [images, ..., channels].  gamma, beta: float32 [channels] or None.  stats [images,
    groups, 2] float32 = mean, 1 / sqrt(var + eps) for group_norm_backward.  y may be x."""
    name = "group_norm"
    d = _norm_desc(name, x, groups, act, eps)
    _on_device(name, x.dtype, x=x, y=y)
    _on_device(name, torch.float32, gamma=gamma, beta=beta, stats=stats)
    _dense(name, (d.c,), gamma=gamma, beta=beta)
    with _on_stream(stream) as handle:
        if y is None:
            y = torch.empty(x.shape, dtype=x.dtype, device="cuda")
        _need(y.shape == x.shape, f"{name}: y must have x's shape")
        if stats is None:
            stats = torch.empty(d.n, max(d.groups, 0), 2, dtype=torch.float32, device="cuda")
        _dense(name, (d.n, d.groups, 2), stats=stats)
        d.x_pixel, d.x_image = _norm_strides(name, x)
        d.y_pixel, d.y_image = _norm_strides(name, y)
        ws, n = _workspace(name, lib().rrm_group_norm_workspace, d, 0)
        _b._check(lib().rrm_group_norm(ctypes.byref(d), _b._ptr(x), _b._ptr(gamma), _b._ptr(beta), _b._ptr(y), _b._ptr(stats),
                                       _b._ptr(ws), n, handle), name)
    return y, stats


def group_norm_backward(x, dy, groups, gamma=None, beta=None, stats=None, eps=1e-5, act="none", dx=None, stream=None):
    """rrm_group_norm_backward: (dx, dgamma, dbeta) from dy = dL/dy and the forward call's x and stats."""
    name = "group_norm_backward"
    d = _norm_desc(name, x, groups, act, eps)
    _need(stats is not None, f"{name}: stats of the forward call are needed")
    _on_device(name, x.dtype, x=x, dy=dy, dx=dx)
    _on_device(name, torch.float32, gamma=gamma, beta=beta, stats=stats)
    _dense(name, (d.c,), gamma=gamma, beta=beta)
    _dense(name, (d.n, d.groups, 2), stats=stats)
    with _on_stream(stream) as handle:
        if dx is None:
            dx = torch.empty(x.shape, dtype=x.dtype, device="cuda")
        _need(dy.shape == x.shape and dx.shape == x.shape, f"{name}: dy and dx must have x's shape")
        dgamma = torch.empty(d.c, dtype=torch.float32, device="cuda")
        dbeta = torch.empty(d.c, dtype=torch.float32, device="cuda")
        d.x_pixel, d.x_image = _norm_strides(name, x)
        d.y_pixel, d.y_image = _norm_strides(name, dy)
        d.dx_pixel, d.dx_image = _norm_strides(name, dx)
        ws, n = _workspace(name, lib().rrm_group_norm_workspace, d, 1)
        _b._check(lib().rrm_group_norm_backward(ctypes.byref(d), _b._ptr(x), _b._ptr(dy), _b._ptr(gamma), _b._ptr(beta),
                                                _b._ptr(stats), _b._ptr(dx), _b._ptr(dgamma), _b._ptr(dbeta), _b._ptr(ws), n,
                                                handle), name)
    return dx, dgamma, dbeta


# ---- gated feed-forward block --------------------------------------------------------------------------------------

def _ff_desc(name, x, w_gate, w_up, b_gate, b_up, act):
    _need(isinstance(x, torch.Tensor) and x.dim() >= 1 and isinstance(w_gate, torch.Tensor) and w_gate.dim() == 2,
          f"{name}: x is [..., inputs], w_gate and w_up are [outputs, inputs]")
    _need(x.dtype in (torch.float32, torch.bfloat16), f"{name}: x must be float32 or bfloat16, is {x.dtype}")
    _need(act in ACT, f"{name}: unknown activation {act!r}")
    _on_device(name, x.dtype, x=x, w_gate=w_gate, w_up=w_up)
    _on_device(name, torch.float32, b_gate=b_gate, b_up=b_up)
    f, k = w_gate.shape
    _need(w_up.shape == w_gate.shape and x.shape[-1] == k, f"{name}: w_gate {tuple(w_gate.shape)}, w_up {tuple(w_up.shape)} and x {tuple(x.shape)} do not fit")
    _dense(name, (f,), b_gate=b_gate, b_up=b_up)
    d = FfDesc()
    d.dtype, d.act, d.k, d.f = _DTYPE[x.dtype], ACT[act], k, f
    d.m = x.numel() // k if k else 0
    d.ld_x = _rows(name, x)
    d.ld_w = _rows(name, w_gate)
    _need(_rows(name, w_up) == d.ld_w, f"{name}: w_gate and w_up must have the same row stride")
    d.unaligned = int(any(t.data_ptr() % 16 for t in (x, w_gate, w_up)))
    return d


def _rows(name, t):
    """Row stride of a tensor whose last axis is a row, 0 if there is at most one."""
    _inner(name, t)
    return _axis(name, t, 0, t.dim() - 1) if t.numel() else 0


def gated_ff(x, w_gate, w_up, b_gate=None, b_up=None, act="silu", y=None, stream=None):
    """rrm_gated_ff: y = act(x w_gate^T + b_gate) * (x w_up^T + b_up) for x [..., inputs] and weights [outputs, inputs];
    biases float32 or None."""
    name = "gated_ff"
    d = _ff_desc(name, x, w_gate, w_up, b_gate, b_up, act)
    _on_device(name, x.dtype, y=y)
    with _on_stream(stream) as handle:
        shape = x.shape[:-1] + (d.f,)
        if y is None:
            y = torch.empty(shape, dtype=x.dtype, device="cuda")
        _need(y.shape == shape, f"{name}: y must be {tuple(shape)}")
        d.ld_y = _rows(name, y)
        ws, n = _workspace(name, lib().rrm_gated_ff_workspace, d, 0)
        _b._check(lib().rrm_gated_ff(ctypes.byref(d), _b._ptr(x), _b._ptr(w_gate), _b._ptr(w_up), _b._ptr(b_gate), _b._ptr(b_up),
                                     _b._ptr(y), _b._ptr(ws), n, handle), name)
    return y


def gated_ff_backward(x, w_gate, w_up, dy, b_gate=None, b_up=None, act="silu", stream=None):
    """rrm_gated_ff_backward: (dx, dw_gate, dw_up, db_gate, db_up) from dy = dL/dy; a bias that is None has None."""
    name = "gated_ff_backward"
    d = _ff_desc(name, x, w_gate, w_up, b_gate, b_up, act)
    _on_device(name, x.dtype, dy=dy)
    _need(dy.shape == x.shape[:-1] + (d.f,), f"{name}: dy must be {tuple(x.shape[:-1] + (d.f,))}")
    d.ld_y = _rows(name, dy)
    with _on_stream(stream) as handle:
        new = lambda *shape, dtype=x.dtype: torch.empty(*shape, dtype=dtype, device="cuda")   # noqa: E731
        dx, dwg, dwu = new(*x.shape), new(d.f, d.k), new(d.f, d.k)
        dbg = None if b_gate is None else new(d.f, dtype=torch.float32)
        dbu = None if b_up is None else new(d.f, dtype=torch.float32)
        ws, n = _workspace(name, lib().rrm_gated_ff_workspace, d, 1)
        _b._check(lib().rrm_gated_ff_backward(ctypes.byref(d), _b._ptr(x), _b._ptr(w_gate), _b._ptr(w_up), _b._ptr(b_gate),
                                              _b._ptr(b_up), _b._ptr(dy), _b._ptr(dx), _b._ptr(dwg), _b._ptr(dwu), _b._ptr(dbg),
                                              _b._ptr(dbu), _b._ptr(ws), n, handle), name)
    return dx, dwg, dwu, dbg, dbu


def head_status(stream=None):
    """rrm_head_status: raises if a bounded device wait of a gated block ran out since the last call (synchronises the stream)."""
    _b._check(lib().rrm_head_status(_b._stream(stream)), "rrm_head_status")


# ---- gated recurrence over frames ----------------------------------------------------------------------------------

def _scan_desc(name, g, x, reset, lengths, **states):
    _need(isinstance(g, torch.Tensor) and isinstance(x, torch.Tensor) and g.dim() == 3 and g.shape == x.shape,
          f"{name}: g and x are [frames, streams, features]")
    _need(g.dtype in _DTYPE, f"{name}: g must be float32, bfloat16 or float16, is {g.dtype}")
    d = ScanDesc()
    d.dtype, d.frames, d.n, d.d = _DTYPE[g.dtype], *g.shape
    _on_device(name, g.dtype, g=g, x=x)
    _on_device(name, torch.float32, **states)
    _on_device(name, torch.int32, lengths=lengths)
    if reset is not None:
        _on_device(name, torch.bool if reset.dtype == torch.bool else torch.uint8, reset=reset)
    _dense(name, (d.n, d.d), **states)
    _dense(name, (d.n,), lengths=lengths)
    _dense(name, (d.frames, d.n), reset=reset)
    return d


def _scan_strides(name, t, like):
    _need(t.shape == like.shape, f"{name}: a tensor of shape {tuple(t.shape)} should have {tuple(like.shape)}")
    _inner(name, t)
    if not t.numel():
        return 0, 0
    frame, stream = _axis(name, t, 0, 1), _axis(name, t, 1, 2)
    if stream == 0:
        stream = t.shape[2]                     # one stream: any stride
    return (frame or stream * t.shape[1]), stream


def _scan_out(like):
    return torch.empty(like.shape, dtype=like.dtype, device="cuda")


def gated_scan(g, x, h0=None, reset=None, lengths=None, h=None, last=None, stream=None):
    """rrm_gated_scan: (h, last) of h_t = f_t h_{t-1} + (1 - f_t) x_t with f = sigmoid(g), for g, x [frames, streams,
    features].  h0, last: float32 [streams, features] (last may be h0).  reset: uint8 or bool [frames, streams], the state
    is dropped before such a frame.  lengths: int32 [streams]; rows of h behind a stream's last frame are left as they are
    (zeros in an h allocated here)."""
    name = "gated_scan"
    d = _scan_desc(name, g, x, reset, lengths, h0=h0, last=last)
    _on_device(name, g.dtype, h=h)
    with _on_stream(stream) as handle:
        if h is None:
            h, d.fill = _scan_out(g), 1
        if last is None:
            last = torch.empty(d.n, d.d, dtype=torch.float32, device="cuda")
        d.g_frame, d.g_stream = _scan_strides(name, g, g)
        d.x_frame, d.x_stream = _scan_strides(name, x, g)
        d.h_frame, d.h_stream = _scan_strides(name, h, g)
        ws, n = _workspace(name, lib().rrm_gated_scan_workspace, d, 0)
        _b._check(lib().rrm_gated_scan(ctypes.byref(d), _b._ptr(g), _b._ptr(x), _b._ptr(h0), _b._ptr(reset), _b._ptr(lengths),
                                       _b._ptr(h), _b._ptr(last), _b._ptr(ws), n, handle), name)
    return h, last


def gated_scan_backward(g, x, dh, h0=None, dlast=None, reset=None, lengths=None, dg=None, dx=None, stream=None):
    """rrm_gated_scan_backward: (dg, dx, dh0) from dh = dL/dh and dlast = dL/dlast (None: zeros); the other arguments as in
    the forward call.  dg and dx: both given or neither; their rows behind a stream's last frame as h's there."""
    name = "gated_scan_backward"
    d = _scan_desc(name, g, x, reset, lengths, h0=h0, dlast=dlast)
    _on_device(name, g.dtype, dh=dh, dg=dg, dx=dx)
    with _on_stream(stream) as handle:
        _need((dg is None) == (dx is None), f"{name}: give both dg and dx, or neither")
        if dg is None:
            dg, dx, d.fill = _scan_out(g), _scan_out(g), 1
        dh0 = torch.empty(d.n, d.d, dtype=torch.float32, device="cuda")
        for key, t in (("g", g), ("x", x), ("h", dh), ("dg", dg), ("dx", dx)):
            frame, row = _scan_strides(name, t, g)
            setattr(d, key + "_frame", frame)
            setattr(d, key + "_stream", row)
        ws, n = _workspace(name, lib().rrm_gated_scan_workspace, d, 1)
        _b._check(lib().rrm_gated_scan_backward(ctypes.byref(d), _b._ptr(g), _b._ptr(x), _b._ptr(h0), _b._ptr(reset),
                                                _b._ptr(lengths), _b._ptr(dh), _b._ptr(dlast), _b._ptr(dg), _b._ptr(dx),
                                                _b._ptr(dh0), _b._ptr(ws), n, handle), name)
    return dg, dx, dh0

"""Network operators (include/auvnet.h) on torch tensors: argument marshalling only.

``gate_scan`` and ``gate_scan_backward`` (gated linear recurrence along a trajectory, with the rollout's episode ends),
``group_norm`` and ``group_norm_backward`` (group norm with an activation, channels last) and ``dropout`` (mask drawn
from a counter, never stored) launch the library's CUDA kernels on the current (or given) stream and return without
waiting.  Outputs are allocated unless they are given; a raw state or gradient buffer given as an output is written in
place.  There is no CPU fallback.  Wrong arguments raise AuvError with the library's code and reason.
"""
from __future__ import annotations

import ctypes as C
import struct

import torch

from . import auvenv
from .auvenv import AUV_ERR_INVALID, AUV_ERR_SIZE, AUV_OK, AuvError

NET_DTYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
NET_ACT = {"none": 0, "relu": 1, "silu": 2, "tanh": 3}

EXPORTED = ("net_gate_scan_workspace_bytes", "net_gate_scan", "net_gate_scan_backward", "net_group_norm_workspace_bytes", "net_group_norm",
            "net_group_norm_backward", "net_dropout", "net_last_error")

# The argument blocks, field by field as in the header (native alignment).
_ROWS = "Pqq"
_SCAN = struct.Struct("@II3q" + 6 * _ROWS + "7PN")
_NORM = struct.Struct("@IIIf4q" + 4 * _ROWS + "7PN")
_DROP = struct.Struct("@4I3q" + 3 * _ROWS + "dQQ")
_NO_ROWS = (0, 0, 0)

_lib = None


def lib():
    """The library with the argument types of the network operators set (once)."""
    global _lib
    if _lib is None:
        L = auvenv.lib()
        for name in ("net_gate_scan", "net_gate_scan_backward", "net_group_norm", "net_group_norm_backward",
                     "net_dropout"):
            getattr(L, name).argtypes = [C.c_char_p, C.c_void_p]
            getattr(L, name).restype = C.c_int
        for name in ("net_gate_scan_workspace_bytes", "net_group_norm_workspace_bytes"):
            getattr(L, name).argtypes = [C.c_char_p, C.c_int]
            getattr(L, name).restype = C.c_size_t
        L.net_last_error.restype = C.c_char_p
        _lib = L
    return _lib


def _fail(code, msg):
    raise AuvError(code, msg)


def _call(fn, args, device, stream, scratch=()):
    """One call with `device` current.  `scratch`: what was allocated here for it."""
    current = torch.cuda.current_stream(device)
    s = current if stream is None else stream
    if stream is not None and stream.cuda_stream != current.cuda_stream:
        # memory allocated here belongs to the current stream: order its earlier use before the
        # call, and keep it from being handed out again until the call has run
        if scratch:
            s.wait_stream(current)
        for t in scratch:
            t.record_stream(s)
    if device.index == torch.cuda.current_device():
        rc = fn(args, s.cuda_stream)
    else:
        with torch.cuda.device(device):
            rc = fn(args, s.cuda_stream)
    if rc != AUV_OK:
        raise AuvError(rc, lib().net_last_error().decode())


def _activation(x, name):
    """Checks of the tensor that sets shape, type and device of a call."""
    if not isinstance(x, torch.Tensor) or x.dim() != 3:
        _fail(AUV_ERR_INVALID, f"{name} is not a tensor of three axes")
    if x.dtype not in NET_DTYPE:
        _fail(AUV_ERR_INVALID, f"{name}: type {x.dtype} is none of float32, bfloat16, float16")
    if not x.is_cuda:
        _fail(AUV_ERR_SIZE, f"{name} is not device memory")
    return _rows(x, name, x)


def _rows(t, name, like):
    """(pointer, outer, inner) of an activation of the shape, type and device of `like`."""
    if t is not like and (t.shape != like.shape or t.dtype != like.dtype or t.device != like.device):
        _fail(AUV_ERR_INVALID, f"{name}: {tuple(t.shape)} {t.dtype} on {t.device}, expected "
                               f"{tuple(like.shape)} {like.dtype} on {like.device}")
    outer, inner, last = t.stride()
    if last != 1 and t.shape[2] > 1:
        _fail(AUV_ERR_SIZE, f"{name}: channels are not contiguous (stride {last})")
    return t.data_ptr(), outer, inner


def _flat(t, name, shape, dtype, device):
    """Pointer of a contiguous array, 0 for None."""
    if t is None:
        return 0
    if t.shape != shape or t.dtype != dtype or t.device != device:
        _fail(AUV_ERR_INVALID, f"{name}: {tuple(t.shape)} {t.dtype} on {t.device}, expected "
                               f"{tuple(shape)} {dtype} on {device}")
    if not t.is_contiguous():
        _fail(AUV_ERR_SIZE, f"{name} is not contiguous")
    return t.data_ptr()


def _flags(t, name, shape, device):
    return _flat(t, name, shape, torch.bool if t is not None and t.dtype == torch.bool else torch.uint8, device)


def _call_with_workspace(fn, size_of, backward, form, fields, device, stream, scratch):
    """A call whose argument block ends in a workspace, allocated here if one is needed."""
    need = size_of(form.pack(*fields, 0, 0), backward)
    ws = 0
    if need:
        buf = torch.empty(need, dtype=torch.uint8, device=device)
        scratch.append(buf)
        ws = buf.data_ptr()
    _call(fn, form.pack(*fields, ws, need), device, stream, scratch)


def gate_scan(f, v, h0=None, *, done=None, done_prev=None, y=None, hT=None, stream=None):
    """Gated linear recurrence h[t] = a c[t] + (1 - a) v[t], a = sigmoid(f[t]), over f, v [T, N, D]; c[t] is h[t - 1], or
    0 where an episode ended before step t (done [T, N]: after the step; done_prev [N]: before step 0).  Returns
    (y [T, N, D], hT [N, D] fp32).  hT may be h0: a state updated in place."""
    scratch = []
    rf = _activation(f, "f")
    T, N, D = f.shape
    dev, f32 = f.device, torch.float32
    rv = _rows(v, "v", f)
    if y is None:
        y = torch.empty((T, N, D), dtype=f.dtype, device=dev)
        scratch.append(y)
    if hT is None:
        hT = torch.empty((N, D), dtype=f32, device=dev)
        scratch.append(hT)
    fields = (_SCAN.size, NET_DTYPE[f.dtype], T, N, D, *rf, *rv, *_rows(y, "y", f), *_NO_ROWS, *_NO_ROWS, *_NO_ROWS,
              _flat(h0, "h0", (N, D), f32, dev), _flat(hT, "hT", (N, D), f32, dev), 0, 0,
              _flags(done, "done", (T, N), dev), _flags(done_prev, "done_prev", (N,), dev))
    L = lib()
    _call_with_workspace(L.net_gate_scan, L.net_gate_scan_workspace_bytes, 0, _SCAN, fields, dev, stream, scratch)
    return y, hT


def gate_scan_backward(f, v, y, dy, h0=None, *, done=None, done_prev=None, dhT=None, df=None, dv=None, dh0=None,
                       stream=None):
    """Gradients (df, dv, dh0) of gate_scan from dy [T, N, D] and dhT [N, D] (None: zeros); y as gate_scan stored it,
    the other arguments as given to it."""
    scratch = []
    rf = _activation(f, "f")
    T, N, D = f.shape
    dev, f32 = f.device, torch.float32
    rv, ry, rdy = _rows(v, "v", f), _rows(y, "y", f), _rows(dy, "dy", f)
    if df is None:
        df = torch.empty((T, N, D), dtype=f.dtype, device=dev)
        scratch.append(df)
    if dv is None:
        dv = torch.empty((T, N, D), dtype=f.dtype, device=dev)
        scratch.append(dv)
    if dh0 is None:
        dh0 = torch.empty((N, D), dtype=f32, device=dev)
        scratch.append(dh0)
    fields = (_SCAN.size, NET_DTYPE[f.dtype], T, N, D, *rf, *rv, *ry, *rdy, *_rows(df, "df", f), *_rows(dv, "dv", f),
              _flat(h0, "h0", (N, D), f32, dev), 0, _flat(dhT, "dhT", (N, D), f32, dev),
              _flat(dh0, "dh0", (N, D), f32, dev), _flags(done, "done", (T, N), dev),
              _flags(done_prev, "done_prev", (N,), dev))
    L = lib()
    _call_with_workspace(L.net_gate_scan_backward, L.net_gate_scan_workspace_bytes, 1, _SCAN, fields, dev, stream, scratch)
    return df, dv, dh0


def _act(act):
    if act not in NET_ACT:
        _fail(AUV_ERR_INVALID, f"act {act!r} is none of {', '.join(NET_ACT)}")
    return NET_ACT[act]


def _groups(groups):
    if not isinstance(groups, int) or groups < 1:
        _fail(AUV_ERR_INVALID, f"groups {groups!r} is no positive number")
    return groups


def group_norm(x, groups, gamma=None, beta=None, *, eps=1e-5, act="none", y=None, mean=None, rstd=None, stream=None):
    """y = act(gamma (x - mean) rstd + beta) over x [B, S, C], mean and rstd of each instance's groups of C / groups
    channels over all S positions (groups = 1 and S = 1: layer norm).  act: "none", "relu", "silu" or "tanh".  Returns
    (y [B, S, C], mean [B, groups], rstd [B, groups])."""
    scratch = []
    rx = _activation(x, "x")
    B, S, Ch = x.shape
    dev, f32 = x.device, torch.float32
    if y is None:
        y = torch.empty((B, S, Ch), dtype=x.dtype, device=dev)
        scratch.append(y)
    if mean is None:
        mean = torch.empty((B, _groups(groups)), dtype=f32, device=dev)
        scratch.append(mean)
    if rstd is None:
        rstd = torch.empty((B, groups), dtype=f32, device=dev)
        scratch.append(rstd)
    head = (_NORM.size, NET_DTYPE[x.dtype], _act(act), eps, B, S, Ch, _groups(groups), *rx, *_rows(y, "y", x), *_NO_ROWS,
            *_NO_ROWS)
    ptrs = (_flat(gamma, "gamma", (Ch,), f32, dev), _flat(beta, "beta", (Ch,), f32, dev),
            _flat(mean, "mean", (B, groups), f32, dev), _flat(rstd, "rstd", (B, groups), f32, dev), 0, 0)
    L = lib()
    _call_with_workspace(L.net_group_norm, L.net_group_norm_workspace_bytes, 0, _NORM, head + ptrs, dev, stream, scratch)
    return y, mean, rstd


def group_norm_backward(x, groups, gamma, beta, mean, rstd, dy, *, act="none", dx=None, dgamma=None, dbeta=None,
                        stream=None):
    """Gradients (dx, dgamma, dbeta) of group_norm from dy [B, S, C]; mean and rstd as it returned them."""
    scratch = []
    rx = _activation(x, "x")
    B, S, Ch = x.shape
    dev, f32 = x.device, torch.float32
    rdy = _rows(dy, "dy", x)
    if dx is None:
        dx = torch.empty((B, S, Ch), dtype=x.dtype, device=dev)
        scratch.append(dx)
    if dgamma is None:
        dgamma = torch.empty(Ch, dtype=f32, device=dev)
        scratch.append(dgamma)
    if dbeta is None:
        dbeta = torch.empty(Ch, dtype=f32, device=dev)
        scratch.append(dbeta)
    head = (_NORM.size, NET_DTYPE[x.dtype], _act(act), 0.0, B, S, Ch, _groups(groups), *rx, *_NO_ROWS, *rdy,
            *_rows(dx, "dx", x))
    ptrs = (_flat(gamma, "gamma", (Ch,), f32, dev), _flat(beta, "beta", (Ch,), f32, dev),
            _flat(mean, "mean", (B, groups), f32, dev), _flat(rstd, "rstd", (B, groups), f32, dev),
            _flat(dgamma, "dgamma", (Ch,), f32, dev), _flat(dbeta, "dbeta", (Ch,), f32, dev))
    L = lib()
    _call_with_workspace(L.net_group_norm_backward, L.net_group_norm_workspace_bytes, 1, _NORM, head + ptrs, dev, stream,
                         scratch)
    return dx, dgamma, dbeta


def dropout(x, p, seed, draw, *, residual=None, shared=False, y=None, stream=None):
    """residual + (dropped ? 0 : x / (1 - p)) over x [T, N, D]; the mask is a function of (seed, draw) and the element's
    index, one for all T if shared.  The gradient by x is dropout(dy, p, seed, draw, shared=shared).  y may be x or
    residual."""
    scratch = []
    rx = _activation(x, "x")
    if y is None:
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        scratch.append(y)
    rr = _NO_ROWS if residual is None else _rows(residual, "residual", x)
    args = _DROP.pack(_DROP.size, NET_DTYPE[x.dtype], bool(shared), 0, *x.shape, *rx, *rr, *_rows(y, "y", x), p,
                      seed & 0xFFFFFFFFFFFFFFFF, draw & 0xFFFFFFFFFFFFFFFF)
    _call(lib().net_dropout, args, x.device, stream, scratch)
    return y

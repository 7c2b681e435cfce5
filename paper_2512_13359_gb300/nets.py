"""Network operators (include/auvnet.h) on torch tensors: argument marshalling only.

``gate_scan`` and ``gate_scan_backward`` (gated linear recurrence along a trajectory, with the rollout's episode ends),
``group_norm`` and ``group_norm_backward`` (group norm with an activation, channels last) and ``dropout`` (mask drawn
from a counter, never stored) launch the library's CUDA kernels on the current (or given) stream and return without
waiting.  Outputs are allocated unless they are given; a raw state or gradient buffer given as an output is written in
place.  There is no CPU fallback.  Wrong arguments raise AuvError with the library's code and reason.

Gradients are calls of their own: tensors that require gradients are taken as they are, and outputs carry no graph.

A given stream is the caller's to order, as with every call of the package: behind what made the inputs, and ahead of what
uses the outputs.  A call that allocates also makes it wait for the current stream, whose memory the allocations are; one
whose outputs are all given may not, so nothing should rest on that.
"""
from __future__ import annotations

import ctypes as C
import struct

import torch

from . import auvenv
from .auvenv import AUV_ERR_INVALID, AUV_ERR_SIZE, AUV_OK, AuvError

NET_DTYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
NET_ACT = {"none": 0, "relu": 1, "silu": 2, "tanh": 3}

EXPORTED = ("net_gate_scan_workspace_bytes", "net_gate_scan", "net_gate_scan_backward",
            "net_group_norm_workspace_bytes", "net_group_norm", "net_group_norm_backward", "net_dropout",
            "net_last_error")

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


def _call(fn, args, index, stream, scratch):
    """One call on device `index`.  `scratch`: what was allocated here for it."""
    if stream is None:
        handle = torch._C._cuda_getCurrentRawStream(index)
    else:
        handle = stream.cuda_stream
        current = torch.cuda.current_stream(index)
        if scratch and handle != current.cuda_stream:
            # memory allocated here belongs to the current stream: order its earlier use before the
            # call, and keep it from being handed out again until the call has run
            stream.wait_stream(current)
            for t in scratch:
                t.record_stream(stream)
    if index == torch.cuda.current_device():
        rc = fn(args, handle)
    else:
        with torch.cuda.device(index):
            rc = fn(args, handle)
    if rc != AUV_OK:
        raise AuvError(rc, lib().net_last_error().decode())


def _activation(x, name):
    """(shape, type, device) of the tensor that sets those of a call."""
    if not isinstance(x, torch.Tensor) or x.dim() != 3:
        _fail(AUV_ERR_INVALID, f"{name} is not a tensor of three axes")
    if x.dtype not in NET_DTYPE:
        _fail(AUV_ERR_INVALID, f"{name}: type {x.dtype} is none of float32, bfloat16, float16")
    if not x.is_cuda:
        _fail(AUV_ERR_SIZE, f"{name} is not device memory")
    return x.shape, x.dtype, x.get_device()


def _rows(t, name, like):
    """(pointer, outer, inner) of an activation of the (shape, type, device) `like`."""
    shape, dtype, index = like
    try:
        if t.shape != shape or t.dtype is not dtype or t.get_device() != index:
            _fail(AUV_ERR_INVALID, f"{name}: {tuple(t.shape)} {t.dtype} on {t.device}, expected "
                                   f"{tuple(shape)} {dtype} on device {index}")
    except AttributeError:
        _fail(AUV_ERR_INVALID, f"{name} is not a tensor")
    outer, inner, last = t.stride()
    if last != 1 and shape[2] > 1:
        _fail(AUV_ERR_SIZE, f"{name}: channels are not contiguous (stride {last})")
    return t.data_ptr(), outer, inner


def _flat(t, name, shape, dtype, index):
    """Pointer of a contiguous array, 0 for None."""
    if t is None:
        return 0
    try:
        if t.shape != shape or t.dtype is not dtype or t.get_device() != index:
            _fail(AUV_ERR_INVALID, f"{name}: {tuple(t.shape)} {t.dtype} on {t.device}, expected "
                                   f"{tuple(shape)} {dtype} on device {index}")
    except AttributeError:
        _fail(AUV_ERR_INVALID, f"{name} is not a tensor")
    if not t.is_contiguous():
        _fail(AUV_ERR_SIZE, f"{name} is not contiguous")
    return t.data_ptr()


def _flags(t, name, shape, index):
    if t is None:
        return 0
    return _flat(t, name, shape, torch.bool if getattr(t, "dtype", None) is torch.bool else torch.uint8, index)


def _new(shape, dtype, index, scratch):
    t = torch.empty(shape, dtype=dtype, device=index)
    scratch.append(t)
    return t


# What packing an argument block raises for a number that is none, or does not fit its field.  Caught in place, as are
# arrays that are no tensors: checks ahead and a function around the packing took 0.5 to 1 us of a call's 10.
_NO_NUMBER = (struct.error, OverflowError)


def _no_number(e):
    _fail(AUV_ERR_INVALID, f"an argument is no number, or too large: {e}")


def _call_with_workspace(fn, size_of, backward, form, fields, index, stream, scratch):
    """A call whose argument block ends in a workspace, allocated here if one is needed."""
    try:
        args = form.pack(*fields, 0, 0)
    except _NO_NUMBER as e:
        _no_number(e)
    need = size_of(args, backward)
    if need:
        args = form.pack(*fields, _new(need, torch.uint8, index, scratch).data_ptr(), need)
    _call(fn, args, index, stream, scratch)


def gate_scan(f, v, h0=None, *, done=None, done_prev=None, y=None, hT=None, stream=None):
    """Gated linear recurrence h[t] = a c[t] + (1 - a) v[t], a = sigmoid(f[t]), over f, v [T, N, D]; c[t] is h[t - 1], or
    0 where an episode ended before step t (done [T, N]: after the step; done_prev [N]: before step 0).  Returns
    (y [T, N, D], hT [N, D] fp32).  hT may be h0: a state updated in place."""
    scratch = []
    like = shape, dtype, index = _activation(f, "f")
    T, N, D = shape
    f32 = torch.float32
    if y is None:
        y = _new(shape, dtype, index, scratch)
    if hT is None:
        hT = _new((N, D), f32, index, scratch)
    fields = (_SCAN.size, NET_DTYPE[dtype], T, N, D, *_rows(f, "f", like), *_rows(v, "v", like), *_rows(y, "y", like),
              *_NO_ROWS, *_NO_ROWS, *_NO_ROWS, _flat(h0, "h0", (N, D), f32, index), _flat(hT, "hT", (N, D), f32, index),
              0, 0, _flags(done, "done", (T, N), index), _flags(done_prev, "done_prev", (N,), index))
    L = lib()
    if T < 32:                        # short sequences need no workspace
        _call(L.net_gate_scan, _SCAN.pack(*fields, 0, 0), index, stream, scratch)
    else:
        _call_with_workspace(L.net_gate_scan, L.net_gate_scan_workspace_bytes, 0, _SCAN, fields, index, stream, scratch)
    return y, hT


def gate_scan_backward(f, v, y, dy, h0=None, *, done=None, done_prev=None, dhT=None, df=None, dv=None, dh0=None,
                       stream=None):
    """Gradients (df, dv, dh0) of gate_scan from dy [T, N, D] and dhT [N, D] (None: zeros); y as gate_scan stored it,
    the other arguments as given to it."""
    scratch = []
    like = shape, dtype, index = _activation(f, "f")
    T, N, D = shape
    f32 = torch.float32
    if df is None:
        df = _new(shape, dtype, index, scratch)
    if dv is None:
        dv = _new(shape, dtype, index, scratch)
    if dh0 is None:
        dh0 = _new((N, D), f32, index, scratch)
    fields = (_SCAN.size, NET_DTYPE[dtype], T, N, D, *_rows(f, "f", like), *_rows(v, "v", like), *_rows(y, "y", like),
              *_rows(dy, "dy", like), *_rows(df, "df", like), *_rows(dv, "dv", like),
              _flat(h0, "h0", (N, D), f32, index), 0, _flat(dhT, "dhT", (N, D), f32, index),
              _flat(dh0, "dh0", (N, D), f32, index), _flags(done, "done", (T, N), index),
              _flags(done_prev, "done_prev", (N,), index))
    L = lib()
    if T < 32:
        _call(L.net_gate_scan_backward, _SCAN.pack(*fields, 0, 0), index, stream, scratch)
    else:
        _call_with_workspace(L.net_gate_scan_backward, L.net_gate_scan_workspace_bytes, 1, _SCAN, fields, index, stream,
                             scratch)
    return df, dv, dh0


def _norm_head(act, groups, channels):
    if act not in NET_ACT:
        _fail(AUV_ERR_INVALID, f"act {act!r} is none of {', '.join(NET_ACT)}")
    if not isinstance(groups, int) or groups < 1:
        _fail(AUV_ERR_INVALID, f"groups {groups!r} is no positive number")
    if channels % groups or groups > 1 << 31:
        _fail(AUV_ERR_INVALID, f"{channels} channels are no multiple of {groups} groups")
    return NET_ACT[act]


def group_norm(x, groups, gamma=None, beta=None, *, eps=1e-5, act="none", y=None, mean=None, rstd=None, stream=None):
    """y = act(gamma (x - mean) rstd + beta) over x [B, S, C], mean and rstd of each instance's groups of C / groups
    channels over all S positions (groups = 1 and S = 1: layer norm).  act: "none", "relu", "silu" or "tanh".  Returns
    (y [B, S, C], mean [B, groups], rstd [B, groups])."""
    scratch = []
    like = shape, dtype, index = _activation(x, "x")
    B, S, Ch = shape
    kind = _norm_head(act, groups, Ch)
    f32, stats = torch.float32, (B, groups)
    if y is None:
        y = _new(shape, dtype, index, scratch)
    if mean is None:
        mean = _new(stats, f32, index, scratch)
    if rstd is None:
        rstd = _new(stats, f32, index, scratch)
    fields = (_NORM.size, NET_DTYPE[dtype], kind, eps, B, S, Ch, groups, *_rows(x, "x", like), *_rows(y, "y", like),
              *_NO_ROWS, *_NO_ROWS, _flat(gamma, "gamma", (Ch,), f32, index), _flat(beta, "beta", (Ch,), f32, index),
              _flat(mean, "mean", stats, f32, index), _flat(rstd, "rstd", stats, f32, index), 0, 0)
    L = lib()
    if S * Ch <= 2048 * groups <= 1 << 26:      # small groups need no workspace
        try:
            args = _NORM.pack(*fields, 0, 0)
        except _NO_NUMBER as e:
            _no_number(e)
        _call(L.net_group_norm, args, index, stream, scratch)
    else:
        _call_with_workspace(L.net_group_norm, L.net_group_norm_workspace_bytes, 0, _NORM, fields, index, stream, scratch)
    return y, mean, rstd


def group_norm_backward(x, groups, gamma, beta, mean, rstd, dy, *, act="none", dx=None, dgamma=None, dbeta=None,
                        stream=None):
    """Gradients (dx, dgamma, dbeta) of group_norm from dy [B, S, C]; mean and rstd as it returned them."""
    scratch = []
    like = shape, dtype, index = _activation(x, "x")
    B, S, Ch = shape
    kind = _norm_head(act, groups, Ch)
    f32, stats = torch.float32, (B, groups)
    if dx is None:
        dx = _new(shape, dtype, index, scratch)
    if dgamma is None:
        dgamma = _new((Ch,), f32, index, scratch)
    if dbeta is None:
        dbeta = _new((Ch,), f32, index, scratch)
    fields = (_NORM.size, NET_DTYPE[dtype], kind, 0.0, B, S, Ch, groups, *_rows(x, "x", like), *_NO_ROWS,
              *_rows(dy, "dy", like), *_rows(dx, "dx", like), _flat(gamma, "gamma", (Ch,), f32, index),
              _flat(beta, "beta", (Ch,), f32, index), _flat(mean, "mean", stats, f32, index),
              _flat(rstd, "rstd", stats, f32, index), _flat(dgamma, "dgamma", (Ch,), f32, index),
              _flat(dbeta, "dbeta", (Ch,), f32, index))
    L = lib()
    _call_with_workspace(L.net_group_norm_backward, L.net_group_norm_workspace_bytes, 1, _NORM, fields, index, stream,
                         scratch)
    return dx, dgamma, dbeta


def dropout(x, p, seed, draw, *, residual=None, shared=False, y=None, stream=None):
    """residual + (dropped ? 0 : x / (1 - p)) over x [T, N, D]; the mask is a function of (seed, draw) and the element's
    index, one for all T if shared.  The gradient by x is dropout(dy, p, seed, draw, shared=shared).  y may be x or
    residual."""
    scratch = []
    like = shape, dtype, index = _activation(x, "x")
    if y is None:
        y = _new(shape, dtype, index, scratch)
    try:
        args = _DROP.pack(_DROP.size, NET_DTYPE[dtype], bool(shared), 0, *shape, *_rows(x, "x", like),
                          *(_NO_ROWS if residual is None else _rows(residual, "residual", like)), *_rows(y, "y", like), p,
                          seed & 0xFFFFFFFFFFFFFFFF, draw & 0xFFFFFFFFFFFFFFFF)
    except (*_NO_NUMBER, TypeError) as e:
        _no_number(e)
    _call(lib().net_dropout, args, index, stream, scratch)
    return y

"""Operators of a mixture-of-experts layer around the planner: binding of include/taot_layer.h.  Argument marshalling only.

In the order in which a layer runs them: `rms_norm` (residual's addition, RMS norm, 8-bit rows with scales), `route` (router
logits to the table that `Planner.plan` takes), `send` (rows to the send buffer by `Planner.dispatch`'s positions), `combine`
(weighted sum of the rows that came back); and `combine_backward`, `route_backward`, `rms_norm_backward`.  The gradient of
`send` is `combine` without weights.

Tensors are on one CUDA device, which need not be the current one; the kernels go to that device's current stream.  Rows may
be strided (their columns dense).  `out`: a dict returned by an earlier call (or a part of one), to reuse its tensors.

Nothing is recorded for automatic differentiation: the results need no gradient, whatever the arguments do.  A program that
differentiates calls the *_backward functions, in a torch.autograd.Function of its own for instance."""
from __future__ import annotations

import ctypes
from typing import Dict, Optional

import torch

from .binding import TaotError, _check, load_library

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_SCORES = {"softmax": 0, "sigmoid": 1}


class NormParams(ctypes.Structure):
    """taot_norm_params"""
    _fields_ = [("struct_size", ctypes.c_int32), ("dtype", ctypes.c_int32), ("N", ctypes.c_int64), ("D", ctypes.c_int32),
                ("group", ctypes.c_int32), ("eps", ctypes.c_float), ("reserved", ctypes.c_int32), ("ld_x", ctypes.c_int64),
                ("ld_residual", ctypes.c_int64), ("ld_h", ctypes.c_int64), ("ld_y", ctypes.c_int64), ("ld_q", ctypes.c_int64)]


class RouteParams(ctypes.Structure):
    """taot_route_params"""
    _fields_ = [("struct_size", ctypes.c_int32), ("dtype", ctypes.c_int32), ("L", ctypes.c_int64), ("T", ctypes.c_int64),
                ("E", ctypes.c_int32), ("k", ctypes.c_int32), ("score", ctypes.c_int32), ("groups", ctypes.c_int32),
                ("groups_kept", ctypes.c_int32), ("group_top", ctypes.c_int32), ("renormalise", ctypes.c_int32),
                ("scale", ctypes.c_float), ("ld_logits", ctypes.c_int64), ("ld_dlogits", ctypes.c_int64)]


class RowsParams(ctypes.Structure):
    """taot_rows_params"""
    _fields_ = [("struct_size", ctypes.c_int32), ("dtype", ctypes.c_int32), ("B", ctypes.c_int64), ("n", ctypes.c_int64),
                ("k", ctypes.c_int32), ("D", ctypes.c_int32), ("C", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("ld_rows", ctypes.c_int64), ("ld_tokens", ctypes.c_int64), ("ld_residual", ctypes.c_int64)]


_NORM_BYTES, _ROUTE_BYTES, _ROWS_BYTES = (ctypes.sizeof(t) for t in (NormParams, RouteParams, RowsParams))
_P, _I = ctypes.c_void_p, ctypes.c_int32
_ARGS = {                                        # behind the pointer to the params; the stream comes last
    "taot_rms_norm": [_P] * 8, "taot_rms_norm_backward": [_P] * 8, "taot_route": [_P] * 5, "taot_route_backward": [_P] * 4,
    "taot_send": [_I, _P, _P, _I, _P, _P, _P, _P, _P], "taot_combine": [_P] * 7, "taot_combine_backward": [_P] * 8,
}
_functions: Dict[str, object] = {}


def _function(name: str):
    fn = _functions.get(name)
    if fn is None:
        lib = load_library()
        proto = ctypes.CFUNCTYPE(ctypes.c_int, _P, *_ARGS[name], _P)
        fn = _functions[name] = proto((name, lib))
    return fn


def _stream_of(index: int) -> int:
    return torch.cuda.current_stream(index).cuda_stream


_stream_of = getattr(torch._C, "_cuda_getCurrentRawStream", _stream_of)      # the same without a stream object, which takes microseconds


def _at(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _type(t: torch.Tensor, name: str) -> int:
    code = _TYPES.get(t.dtype)
    if code is None:
        raise TaotError(f"{name}: expected float32, bfloat16 or float16, not {t.dtype}")
    return code


def _rows(t: torch.Tensor, name: str, shape, dtype, device) -> int:
    """Checks a tensor whose last dimension is a row; returns the distance between rows in elements."""
    if t.shape != shape or t.dtype != dtype or t.device != device:
        raise TaotError(f"{name}: expected a tensor {list(shape)} of {dtype} on {device}, not {list(t.shape)} of {t.dtype} on {t.device}")
    if t.is_contiguous():
        return shape[-1]
    stride = t.stride()
    if t.shape[-1] > 1 and stride[-1] != 1:
        raise TaotError(f"{name}: the columns of a row must be dense")
    ld, step = None, None
    for size, s in zip(reversed(t.shape[:-1]), reversed(stride[:-1])):
        if size == 1:
            continue
        if ld is None:
            ld = step = s
        elif s != step:
            raise TaotError(f"{name}: the rows must be evenly spaced")
        step = step * size
    ld = t.shape[-1] if ld is None else ld
    if ld < t.shape[-1]:
        raise TaotError(f"{name}: the rows overlap")
    return ld


def _dense(t: Optional[torch.Tensor], name: str, shape, dtype, device):
    if t is not None and (t.shape != shape or t.dtype != dtype or t.device != device or not t.is_contiguous()):
        raise TaotError(f"{name}: expected a contiguous tensor {list(shape)} of {dtype} on {device}")


def _start(t: torch.Tensor, name: str, dims: int) -> torch.device:
    if not t.is_cuda:
        raise TaotError(f"{name}: expected a CUDA tensor (there is no CPU path)")
    if t.dim() < dims:
        raise TaotError(f"{name}: expected at least {dims} dimensions")
    return t.device


def _call(device: torch.device, what: str, params, *args):
    """Calls an entry point with the device's current stream as its last argument, that device being current."""
    fn = _functions.get(what) or _function(what)
    if device.index == torch.cuda.current_device():
        rc = fn(ctypes.addressof(params), *args, _stream_of(device.index))
    else:
        with torch.cuda.device(device):
            rc = fn(ctypes.addressof(params), *args, _stream_of(device.index))
    if rc:
        _check(rc, what)


def _count(shape) -> int:
    n = 1
    for s in shape:
        n *= s
    return n


_MOST = (1 << 31) - 1


def _in_range(what: str, *values: int):
    """The structs' 32-bit fields: ctypes would cut off what does not fit."""
    for v in values:
        if not -_MOST <= v <= _MOST:
            raise TaotError(f"{what}: {v} is out of range")


def _take(out: Optional[Dict[str, torch.Tensor]], name: str, shape, dtype, device):
    """An output whose last dimension is a row, and the distance between rows: the caller's, checked, or a new one."""
    t = None if out is None else out.get(name)
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device), shape[-1]
    return t, _rows(t, name, shape, dtype, device)


def _take_dense(out: Optional[Dict[str, torch.Tensor]], name: str, shape, dtype, device) -> torch.Tensor:
    """A contiguous output: the caller's, checked, or a new one."""
    t = None if out is None else out.get(name)
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device)
    _dense(t, name, shape, dtype, device)
    return t


# ---------------------------------------------------------------------------------------------------------------------
# norm


def rms_norm(x: torch.Tensor, weight: torch.Tensor, eps: float = 1e-6, residual: Optional[torch.Tensor] = None,
             group: int = 0, want_y: bool = True, out: Optional[Dict[str, torch.Tensor]] = None) -> Dict[str, torch.Tensor]:
    """h = x + residual, y = h * rstd(h) * weight over the last dimension, through `taot_rms_norm`.

    group 32, 64, 128 or 256: also q [..., D] (float8_e4m3fn) and scales [..., ceil(D / group)], with y ~ q * scale;
    want_y False leaves y out then.  Returns y, rstd (for the backward pass), h (with a residual), q and scales.
    out may hold x or residual as "h", and x as "y"."""
    dev = _start(x, "x", 1)
    D = x.shape[-1]
    lead = x.shape[:-1]
    _in_range("rms_norm", D, group)
    if not want_y and not group:
        raise TaotError("rms_norm: nothing to write (want_y is False and group is 0)")
    code = _type(x, "x")
    _dense(weight, "weight", (D,), x.dtype, dev)
    shape, dtype = x.shape, x.dtype
    rstd = _take_dense(out, "rstd", lead, torch.float32, dev)
    h = y = q = scales = None
    ld_x, ld_res, ld_h, ld_y, ld_q = _rows(x, "x", shape, dtype, dev), 0, 0, 0, 0
    res = dict(rstd=rstd)
    if residual is not None:
        ld_res = _rows(residual, "residual", shape, dtype, dev)
        h, ld_h = _take(out, "h", shape, dtype, dev)
        res["h"] = h
    if want_y:
        y, ld_y = _take(out, "y", shape, dtype, dev)
        res["y"] = y
    if group:
        q, ld_q = _take(out, "q", shape, torch.float8_e4m3fn, dev)
        scales = _take_dense(out, "scales", lead + (-(-D // group) if group > 0 else 0,), torch.float32, dev)
        res["q"], res["scales"] = q, scales
    p = NormParams(_NORM_BYTES, code, _count(lead), D, group, eps, 0, ld_x, ld_res, ld_h, ld_y, ld_q)
    _call(dev, "taot_rms_norm", p, _at(x), _at(residual), _at(weight), _at(h), _at(y), _at(q), _at(scales), _at(rstd))
    return res


def rms_norm_backward(dy: torch.Tensor, h: torch.Tensor, weight: torch.Tensor, rstd: torch.Tensor,
                      dh: Optional[torch.Tensor] = None, want_dweight: bool = True,
                      out: Optional[Dict[str, torch.Tensor]] = None) -> Dict[str, torch.Tensor]:
    """Gradients of `rms_norm` through `taot_rms_norm_backward`: dx (of x and of the residual alike) and dweight (fp32).
    h: the call's h, or x where it had no residual; dh: what reaches h from elsewhere.  out may hold dy or dh as "dx"."""
    dev = _start(h, "h", 1)
    D = h.shape[-1]
    lead = h.shape[:-1]
    _in_range("rms_norm_backward", D)
    code = _type(h, "h")
    _dense(weight, "weight", (D,), h.dtype, dev)
    _dense(rstd, "rstd", lead, torch.float32, dev)
    p = NormParams(_NORM_BYTES, code, _count(lead), D, 0, 0.0, 0)
    p.ld_h = _rows(h, "h", h.shape, h.dtype, dev)
    p.ld_y = _rows(dy, "dy", h.shape, h.dtype, dev)
    if dh is not None:
        p.ld_residual = _rows(dh, "dh", h.shape, h.dtype, dev)
    dx, p.ld_x = _take(out, "dx", h.shape, h.dtype, dev)
    res = dict(dx=dx)
    ws = None
    if want_dweight:
        res["dweight"] = _take_dense(out, "dweight", (D,), torch.float32, dev)
        n = ctypes.c_size_t()
        _check(load_library().taot_rms_norm_backward_workspace(ctypes.byref(p), ctypes.byref(n)), "taot_rms_norm_backward_workspace")
        ws = torch.empty(n.value, dtype=torch.uint8, device=dev)     # of this call alone: its stream's allocator takes it back
    _call(dev, "taot_rms_norm_backward", p, _at(dy), _at(dh), _at(h), _at(weight), _at(rstd), _at(dx),
          _at(res.get("dweight")), _at(ws))
    return res


# ---------------------------------------------------------------------------------------------------------------------
# router


def _route_params(logits: torch.Tensor, k: int, score: str, renormalise: bool, scale: float):
    code = _type(logits, "logits")
    if score not in _SCORES:
        raise TaotError(f"score: expected one of {sorted(_SCORES)}, not {score!r}")
    lead = logits.shape[:-1]
    T = lead[-1]
    L = _count(lead[:-1])
    _in_range("route", logits.shape[-1], k)
    p = RouteParams(_ROUTE_BYTES, code, L, T, logits.shape[-1], k, _SCORES[score], 1, 1, 1, int(bool(renormalise)), scale)
    p.ld_logits = _rows(logits, "logits", logits.shape, logits.dtype, logits.device)
    return p, lead


def route(logits: torch.Tensor, k: int, score: str = "softmax", bias: Optional[torch.Tensor] = None, groups: int = 1,
          groups_kept: int = 1, group_top: int = 1, renormalise: bool = True, scale: float = 1.0,
          mask: Optional[torch.Tensor] = None, want_weights: bool = True,
          out: Optional[Dict[str, torch.Tensor]] = None) -> Dict[str, torch.Tensor]:
    """Routing of logits [T, E] or [L, T, E] through `taot_route`: topk [.., T, k] int32, as `Planner.plan` takes it, and
    weights [.., T, k] fp32.  bias [E] or [L, E] fp32 takes part in the choice only; mask [.., T] bool: False for padding."""
    dev = _start(logits, "logits", 2)
    p, lead = _route_params(logits, k, score, renormalise, scale)
    _in_range("route", groups, groups_kept, group_top)
    p.groups, p.groups_kept, p.group_top = groups, groups_kept, group_top
    if k < 1:
        raise TaotError(f"route: k = {k} is out of range")
    if bias is not None:
        if bias.dim() == 1 and p.L != 1:
            bias = bias.expand(p.L, -1).contiguous()
        _dense(bias, "bias", bias.shape, torch.float32, dev)
        if bias.dim() < 1 or bias.numel() != p.L * p.E or bias.shape[-1] != p.E:
            raise TaotError(f"bias: expected [{p.E}] or [{p.L}, {p.E}], not {list(bias.shape)}")
    _dense(mask, "mask", lead, torch.bool, dev)
    shape = lead + (k,)
    res = dict(topk=_take_dense(out, "topk", shape, torch.int32, dev))
    if want_weights:
        res["weights"] = _take_dense(out, "weights", shape, torch.float32, dev)
    _call(dev, "taot_route", p, _at(logits), _at(bias), _at(mask), _at(res["topk"]), _at(res.get("weights")))
    return res


def route_backward(logits: torch.Tensor, topk: torch.Tensor, dweights: torch.Tensor, score: str = "softmax",
                   renormalise: bool = True, scale: float = 1.0, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient of `route`'s weights with respect to the logits, of their type and shape, through `taot_route_backward`."""
    dev = _start(logits, "logits", 2)
    if topk.dim() < 1:
        raise TaotError("topk: expected at least 1 dimension")
    p, lead = _route_params(logits, topk.shape[-1], score, renormalise, scale)
    _dense(topk, "topk", lead + (p.k,), torch.int32, dev)
    _dense(dweights, "dweights", lead + (p.k,), torch.float32, dev)
    res = torch.empty(logits.shape, dtype=logits.dtype, device=dev) if out is None else out
    p.ld_dlogits = _rows(res, "out", logits.shape, logits.dtype, dev)
    _call(dev, "taot_route_backward", p, _at(logits), _at(topk), _at(dweights), _at(res))
    return res


# ---------------------------------------------------------------------------------------------------------------------
# rows to the send buffer and back


def _rows_params(perm: torch.Tensor, counts: Optional[torch.Tensor], D: int, code: int):
    dev = _start(perm, "perm", 2)
    shape = perm.shape
    lead, n, k = shape[:-2], shape[-2], shape[-1]
    _dense(perm, "perm", perm.shape, torch.int32, dev)
    _in_range("rows", k, D)
    p = RowsParams(_ROWS_BYTES, code, _count(lead), n, k, D, 0, 0)
    if counts is not None:
        if counts.dim() != len(lead) + 1 or counts.shape[-1] < 1:
            raise TaotError(f"counts: expected {list(lead)} + [C]")
        _dense(counts, "counts", lead + (counts.shape[-1],), torch.int32, dev)
        _in_range("counts", counts.shape[-1])
        p.C = counts.shape[-1]
    return p, lead, n, k, dev


def _info(out, lead, dev) -> torch.Tensor:
    """Status words, OR-ed into by the call: zeroed here unless the caller keeps them (as in the planner's stages)."""
    t = None if out is None else out.get("info")
    if t is None:
        return torch.zeros(lead, dtype=torch.int32, device=dev)
    _dense(t, "info", lead, torch.int32, dev)
    return t


def send(x: torch.Tensor, perm: torch.Tensor, counts: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None,
         out: Optional[Dict[str, torch.Tensor]] = None) -> Dict[str, torch.Tensor]:
    """Rows x [.., n, D] to the send buffers rows [.., n*k, D] by the positions perm [.., n, k], through `taot_send`.

    The leading dimensions are send buffers, e.g. layers and source ranks: `Planner.dispatch`'s perm as [L, R, T/R, k].
    counts [.., C], e.g. its send_counts [L, R, R]: only their sum's first rows of a buffer are in use, the others are left as
    they are.  x is of any type of 1, 2 or 4 bytes; scales [.., n, G] fp32 go the same way.
    Returns rows, scales (if given) and info [..]."""
    D = x.shape[-1] if x.dim() >= 2 else 0
    p, lead, n, k, dev = _rows_params(perm, counts, max(D, 1), 0)
    shape = lead + (n, D)
    p.ld_tokens = _rows(x, "x", shape, x.dtype, dev)
    if x.element_size() not in (1, 2, 4):
        raise TaotError(f"x: expected elements of 1, 2 or 4 bytes, not {x.dtype}")
    rows, p.ld_rows = _take(out, "rows", lead + (n * k, D), x.dtype, dev)
    res = dict(rows=rows, info=_info(out, lead, dev))
    cols = 0
    if scales is not None:
        if scales.dim() < 1:
            raise TaotError("scales: expected [.., n, G]")
        cols = scales.shape[-1]
        _in_range("scales", cols)
        _dense(scales, "scales", lead + (n, cols), torch.float32, dev)
        res["scales"] = _take_dense(out, "scales", lead + (n * k, cols), torch.float32, dev)
    _call(dev, "taot_send", p, x.element_size(), _at(x), _at(scales), cols, _at(perm),
          _at(counts), _at(res["rows"]), _at(res.get("scales")), _at(res["info"]))
    return res


def combine(y: torch.Tensor, perm: torch.Tensor, weights: Optional[torch.Tensor] = None, counts: Optional[torch.Tensor] = None,
            residual: Optional[torch.Tensor] = None, out: Optional[Dict[str, torch.Tensor]] = None) -> Dict[str, torch.Tensor]:
    """out [.., n, D] = residual + the sum over a token's entries of weights [.., n, k] times the rows of y [.., n*k, D] at
    their positions, through `taot_combine`.  perm and counts as in `send`.  Without weights (all one) it is the gradient of
    `send`.  Returns out and info [..]; out may hold the residual as "out"."""
    D = y.shape[-1] if y.dim() >= 2 else 0
    p, lead, n, k, dev = _rows_params(perm, counts, max(D, 1), _type(y, "y"))
    p.ld_rows = _rows(y, "y", lead + (n * k, D), y.dtype, dev)
    _dense(weights, "weights", perm.shape, torch.float32, dev)
    shape = lead + (n, D)
    if residual is not None:
        p.ld_residual = _rows(residual, "residual", shape, y.dtype, dev)
    into, p.ld_tokens = _take(out, "out", shape, y.dtype, dev)
    res = dict(out=into, info=_info(out, lead, dev))
    _call(dev, "taot_combine", p, _at(y), _at(perm), _at(counts), _at(weights), _at(residual), _at(res["out"]),
          _at(res["info"]))
    return res


def combine_backward(dout: torch.Tensor, perm: torch.Tensor, y: Optional[torch.Tensor] = None,
                     weights: Optional[torch.Tensor] = None, counts: Optional[torch.Tensor] = None,
                     want_dy: bool = True, out: Optional[Dict[str, torch.Tensor]] = None) -> Dict[str, torch.Tensor]:
    """Gradients of `combine` (that of the residual is dout) through `taot_combine_backward`: dy [.., n*k, D] for the rows and,
    with y, dweights [.., n, k] fp32.  Rows that are not in use are left as they are.  out may hold y as "dy".
    Returns dy, dweights and info [..]."""
    D = dout.shape[-1] if dout.dim() >= 2 else 0
    p, lead, n, k, dev = _rows_params(perm, counts, max(D, 1), _type(dout, "dout"))
    if not want_dy and y is None:
        raise TaotError("combine_backward: nothing to write (want_dy is False and y is not given)")
    p.ld_tokens = _rows(dout, "dout", lead + (n, D), dout.dtype, dev)
    _dense(weights, "weights", perm.shape, torch.float32, dev)
    rows = lead + (n * k, D)
    res = dict(info=_info(out, lead, dev))
    lds = []
    if y is not None:
        lds.append(_rows(y, "y", rows, dout.dtype, dev))
        res["dweights"] = _take_dense(out, "dweights", perm.shape, torch.float32, dev)
    if want_dy:
        res["dy"], ld = _take(out, "dy", rows, dout.dtype, dev)
        lds.append(ld)
    if len(set(lds)) > 1:
        raise TaotError("y and dy: their rows must be equally far apart")
    p.ld_rows = lds[0]
    _call(dev, "taot_combine_backward", p, _at(dout), _at(y), _at(perm), _at(counts), _at(weights),
          _at(res.get("dy")), _at(res.get("dweights")), _at(res["info"]))
    return res

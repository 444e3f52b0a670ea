"""ctypes binding of a routed expert block's operators (include/fff.h): the routing of tokens to experts, the
sum of a token's experts' rows, RMS norm, and activations kept in 8 bits, with their gradients.

Argument marshalling only, as in ``ops.py``: contiguous GPU tensors, everything computed by the library's HIP
kernels on the call's stream; results and scratch that the caller does not pass are allocated per call.
"""
from __future__ import annotations

import ctypes
from ctypes import c_float, c_int32, c_int64, c_size_t, c_void_p
from typing import NamedTuple

import torch

from .fff import _TORCH_DT, ACTS, FFF_F32, _dt, _raw_stream
from .ops import _INT32, _gpu, _lib, _like, _on_call, _rows, _run, _scratch, _sizes

SCORES = {"softmax": 0, "sigmoid": 1}
GROUP_SCORES = {"max": 0, "top2": 1}
PACK_BLOCK = 32  # columns of a packed row that share a scale


class FffRouteArgs(ctypes.Structure):
    """Mirror of ``fff_route_args`` in include/fff.h."""

    _fields_ = [
        ("logits", c_void_p), ("bias", c_void_p), ("ids", c_void_p), ("weights", c_void_p), ("n_tokens", c_int64),
        ("n_experts", c_int32), ("top_k", c_int32), ("n_groups", c_int32), ("top_groups", c_int32),
        ("x_dtype", c_int32), ("score", c_int32), ("group_score", c_int32), ("renormalise", c_int32),
        ("scale", c_float), ("hip_stream", c_void_p),
    ]


class FffRouteBackwardArgs(ctypes.Structure):
    """Mirror of ``fff_route_backward_args`` in include/fff.h."""

    _fields_ = [
        ("dweights", c_void_p), ("logits", c_void_p), ("ids", c_void_p), ("dlogits", c_void_p), ("n_tokens", c_int64),
        ("n_experts", c_int32), ("top_k", c_int32), ("x_dtype", c_int32), ("d_dtype", c_int32), ("score", c_int32),
        ("renormalise", c_int32), ("scale", c_float), ("hip_stream", c_void_p),
    ]


class FffCombineArgs(ctypes.Structure):
    """Mirror of ``fff_combine_args`` in include/fff.h."""

    _fields_ = [
        ("rows", c_void_p), ("weights", c_void_p), ("ids", c_void_p), ("residual", c_void_p), ("y", c_void_p),
        ("n_tokens", c_int64), ("hidden", c_int32), ("top_k", c_int32), ("rows_dtype", c_int32), ("y_dtype", c_int32),
        ("hip_stream", c_void_p),
    ]


class FffCombineBackwardArgs(ctypes.Structure):
    """Mirror of ``fff_combine_backward_args`` in include/fff.h."""

    _fields_ = [
        ("dy", c_void_p), ("rows", c_void_p), ("weights", c_void_p), ("ids", c_void_p), ("drows", c_void_p),
        ("dweights", c_void_p), ("n_tokens", c_int64), ("hidden", c_int32), ("top_k", c_int32), ("y_dtype", c_int32),
        ("rows_dtype", c_int32), ("drows_dtype", c_int32), ("hip_stream", c_void_p),
    ]


class FffRmsNormArgs(ctypes.Structure):
    """Mirror of ``fff_rms_norm_args`` in include/fff.h."""

    _fields_ = [
        ("x", c_void_p), ("residual", c_void_p), ("gamma", c_void_p), ("y", c_void_p), ("s", c_void_p),
        ("rstd", c_void_p), ("q", c_void_p), ("q_scale", c_void_p), ("n_tokens", c_int64), ("hidden", c_int32),
        ("x_dtype", c_int32), ("s_dtype", c_int32), ("y_dtype", c_int32), ("eps", c_float), ("hip_stream", c_void_p),
    ]


class FffRmsNormBackwardArgs(ctypes.Structure):
    """Mirror of ``fff_rms_norm_backward_args`` in include/fff.h."""

    _fields_ = [
        ("dy", c_void_p), ("s", c_void_p), ("rstd", c_void_p), ("gamma", c_void_p), ("ds_in", c_void_p),
        ("ds", c_void_p), ("dx", c_void_p), ("dgamma", c_void_p), ("n_tokens", c_int64), ("hidden", c_int32),
        ("x_dtype", c_int32), ("s_dtype", c_int32), ("y_dtype", c_int32), ("accumulate", c_int32),
        ("workspace", c_void_p), ("workspace_bytes", c_size_t), ("hip_stream", c_void_p),
    ]


class FffPackRowsArgs(ctypes.Structure):
    """Mirror of ``fff_pack_rows_args`` in include/fff.h."""

    _fields_ = [
        ("x", c_void_p), ("q", c_void_p), ("q_scale", c_void_p), ("n_rows", c_int64), ("hidden", c_int32),
        ("x_dtype", c_int32), ("hip_stream", c_void_p),
    ]


class FffUnpackRowsArgs(ctypes.Structure):
    """Mirror of ``fff_unpack_rows_args`` in include/fff.h."""

    _fields_ = [
        ("q", c_void_p), ("q_scale", c_void_p), ("dy", c_void_p), ("y", c_void_p), ("dx", c_void_p),
        ("n_rows", c_int64), ("hidden", c_int32), ("dy_dtype", c_int32), ("y_dtype", c_int32), ("dx_dtype", c_int32),
        ("act", c_int32), ("hip_stream", c_void_p),
    ]


class Packed(NamedTuple):
    """Rows in 8 bits: ``values`` float8_e4m3fn [rows, hidden] and ``scales`` float8_e8m0fnu
    [rows, ceil(hidden / 32)], a power of two for every 32 columns."""

    values: torch.Tensor
    scales: torch.Tensor


def _choice(names, v, what):
    if v in names:
        return names[v]
    if isinstance(v, str):
        raise ValueError(f"{what} must be one of {', '.join(names)}, got {v!r}")
    return int(v)


def _top_k(top_k, n_tokens):
    top_k = int(top_k)
    if top_k < 1:
        raise ValueError("top_k must be positive")
    if top_k * n_tokens >= 1 << 31:
        raise ValueError(f"{n_tokens} tokens with {top_k} entries each: there must be less than 2^31 entries")
    return top_k


def _out(t, what, index, like, shape, dtype=None, new=None):
    """A result and its pointer: ``t`` (checked; of ``dtype`` where that is given), or a tensor of the type ``new`` or
    ``dtype`` that is allocated as ``like`` is, of ``shape`` (``like``'s own where it is None)."""
    if t is None:
        dtype = new or dtype
        if shape is None:
            t = torch.empty_like(like) if dtype is like.dtype else torch.empty_like(like, dtype=dtype)
        else:
            t = like.new_empty(shape, dtype=dtype)
        return t, t.data_ptr()
    return t, _like(t, what, index, like.shape if shape is None else shape, dtype)


def _new_packed(x):
    """Packed rows for x's, and their pointers."""
    B, H = x.shape
    values = torch.empty_like(x, dtype=torch.float8_e4m3fn)
    scales = x.new_empty((B, -(-H // PACK_BLOCK)), dtype=torch.float8_e8m0fnu)
    return Packed(values, scales), values.data_ptr(), scales.data_ptr()


def _packed(packed, index, shape=None):
    """Pointers of packed rows (of ``shape``), and their shape."""
    try:
        values, scales = packed
    except (TypeError, ValueError):
        raise ValueError("packed must be a Packed: values and scales") from None
    if shape is None:
        shape = _rows(values, "packed values")
        index = values.get_device() if index is None else index
    return (_like(values, "packed values", index, shape, torch.float8_e4m3fn),
            _like(scales, "packed scales", index, (shape[0], -(-shape[1] // PACK_BLOCK)), torch.float8_e8m0fnu), shape)


@_on_call
def route(logits, top_k: int, *, bias=None, score="softmax", n_groups=1, top_groups=None, group_score="top2",
          renormalise=False, scale=1.0, ids=None, weights=None, stream=None):
    """Every token's ``top_k`` experts through ``fff_route``; returns (ids, weights), int32 and float32 [n_tokens, top_k].

    ``logits`` [n_tokens, n_experts].  Scores are the softmax over a token's experts or each one's
    sigmoid; experts are chosen by score + ``bias`` (float32 [n_experts]; without one by the logits), in
    falling order, the lower index where two are equal.  With ``n_groups`` > 1 a token chooses among the experts
    of its ``top_groups`` best groups, by their ``group_score``: "max", or "top2", the sum of the two best.
    Weights are the scores, with ``renormalise`` divided by the chosen ones' sum, times ``scale``.
    Experts with a logit of -inf or NaN are not chosen: entries without an expert have id -1 and weight 0.
    ``group_rows(ids, n_experts, n_trees=1)`` groups the entries for ``grouped_matmul``."""
    B, E = _rows(logits, "logits")
    device, at, top_k = logits.device, logits.get_device(), _top_k(top_k, B)
    n_groups = int(n_groups)
    top_groups = n_groups if top_groups is None else int(top_groups)
    if not 0 < top_groups <= n_groups <= _INT32:
        _sizes((n_groups, "n_groups"), (top_groups, "top_groups"))
    ids, ids_at = _out(ids, "ids", at, logits, (B, top_k), torch.int32)
    weights, weights_at = _out(weights, "weights", at, logits, (B, top_k), torch.float32)
    _run(_lib().fff_route, FffRouteArgs(
        logits.data_ptr(), _like(bias, "bias", at, (E,), torch.float32), ids_at, weights_at, B, E, top_k, n_groups, top_groups,
        _dt(logits, "logits"), _choice(SCORES, score, "score"), _choice(GROUP_SCORES, group_score, "group_score"),
        1 if renormalise else 0, scale, _raw_stream(device, stream)))
    return ids, weights


@_on_call
def route_backward(dweights, logits, ids, *, score="softmax", renormalise=False, scale=1.0, dlogits=None,
                   dlogits_dtype=None, stream=None):
    """Gradient of ``route``'s weights to its logits through ``fff_route_backward``; returns dlogits.

    ``dweights`` float32 and ``ids`` int32 [n_tokens, top_k]; ``score``, ``renormalise`` and ``scale`` are the
    forward's.  The choice has no gradient: groups and bias do not appear.  ``dlogits`` is allocated of
    ``dlogits_dtype`` or logits' type when not given."""
    B, K = _rows(dweights, "dweights")
    device, at = dweights.device, dweights.get_device()
    if dweights.dtype != torch.float32:
        raise ValueError(f"dweights must be torch.float32, got {dweights.dtype}")
    _gpu(logits, "logits", at)
    if _rows(logits, "logits")[0] != B:
        raise ValueError(f"logits must have {B} rows, got {logits.shape[0]}")
    _top_k(K, B)
    shape = logits.shape
    if ids is None:
        raise ValueError("ids are needed")
    dlogits, dlogits_at = _out(dlogits, "dlogits", at, logits, None, new=dlogits_dtype or logits.dtype)
    _run(_lib().fff_route_backward, FffRouteBackwardArgs(
        dweights.data_ptr(), logits.data_ptr(), _like(ids, "ids", at, (B, K), torch.int32), dlogits_at, B, shape[1], K,
        _dt(logits, "logits"), _dt(dlogits, "dlogits"),
        _choice(SCORES, score, "score"), int(bool(renormalise)), scale, _raw_stream(device, stream)))
    return dlogits


@_on_call
def combine(rows, top_k: int, weights=None, *, ids=None, residual=None, y=None, y_dtype=None, stream=None):
    """``y[t] = residual[t] + sum_j weights[t, j] * rows[t * top_k + j]`` through ``fff_combine``; returns y.

    ``rows`` [n_tokens * top_k, hidden]: the experts' (or, without ``weights``, a routing tree's leaves') rows in entry
    order, as ``grouped_matmul(..., y_index=order)`` leaves them.  Entries with a negative id in ``ids``
    take no part, whatever their row holds.  ``y`` may be ``residual``; else it is allocated, of ``y_dtype``,
    residual's or rows' type."""
    R, H = _rows(rows, "rows")
    device, at = rows.device, rows.get_device()
    top_k = int(top_k)
    if top_k < 1 or R % top_k:
        raise ValueError(f"rows must be n_tokens x top_k: got {R} rows for top_k = {top_k}")
    B = R // top_k
    _top_k(top_k, B)
    if y is None and residual is not None and y_dtype in (None, residual.dtype):
        y, y_at = _out(None, "y", at, _gpu(residual, "residual", at), None, residual.dtype)
    else:
        y, y_at = _out(y, "y", at, rows, (B, H), new=y_dtype or rows.dtype)
    _run(_lib().fff_combine, FffCombineArgs(
        rows.data_ptr(), _like(weights, "weights", at, (B, top_k), torch.float32),
        _like(ids, "ids", at, (B, top_k), torch.int32), _like(residual, "residual", at, (B, H), y.dtype), y_at,
        B, H, top_k, _dt(rows, "rows"), _dt(y, "y"), _raw_stream(device, stream)))
    return y


@_on_call
def combine_backward(dy, top_k: int, rows=None, weights=None, *, ids=None, drows=None, dweights=None, drows_dtype=None,
                     want=("drows", "dweights"), stream=None):
    """Gradients of ``combine`` through ``fff_combine_backward``; returns (drows, dweights).

    ``drows[t * top_k + j] = weights[t, j] * dy[t]`` (of ``drows_dtype``, rows' or dy's type; may be the buffer
    ``rows``) and ``dweights[t, j] = <dy[t], rows[t * top_k + j]>``, which needs ``rows``; both are 0 for
    entries whose id is negative.  dy itself is the residual's gradient.  Gradients named in ``want`` are allocated when
    not given (dweights only with ``rows``)."""
    B, H = _rows(dy, "dy")
    device, at, top_k = dy.device, dy.get_device(), _top_k(top_k, B)
    shape, drows_at, dweights_at = (B * top_k, H), None, None
    if drows is not None or "drows" in want:
        dtype = drows_dtype or (rows.dtype if rows is not None else dy.dtype)
        drows, drows_at = _out(drows, "drows", at, dy, shape, new=dtype)
    if dweights is not None or ("dweights" in want and rows is not None):
        dweights, dweights_at = _out(dweights, "dweights", at, dy, (B, top_k), torch.float32)
    _run(_lib().fff_combine_backward, FffCombineBackwardArgs(
        dy.data_ptr(), _like(rows, "rows", at, shape), _like(weights, "weights", at, (B, top_k), torch.float32),
        _like(ids, "ids", at, (B, top_k), torch.int32), drows_at, dweights_at, B, H, top_k, _dt(dy, "dy"),
        _dt(rows, "rows") if rows is not None else FFF_F32, _dt(drows, "drows") if drows is not None else FFF_F32,
        _raw_stream(device, stream)))
    return drows, dweights


@_on_call
def rms_norm(x, gamma=None, *, eps=1e-6, residual=None, y=None, s=None, rstd=None, packed=None, y_dtype=None,
             s_dtype=None, stats=True, pack=False, want_y=True, stream=None):
    """``s = residual + x``, then ``y = s / sqrt(mean(s^2) + eps) * gamma`` per row, through ``fff_rms_norm``.

    Returns (y, s, rstd, packed).  Without a residual s is x itself, unless an s or another ``s_dtype`` than x's is
    passed; ``s`` may be ``residual`` (the stream updated in place).  With ``pack`` (or a ``packed`` to write) y is
    also stored in 8 bits, for the backward pass; with ``want_y`` false in 8 bits alone (y is None).  With ``stats``
    false rstd is None unless passed.  Types of what is allocated: y as ``y_dtype`` or x; s as ``s_dtype``,
    residual or x."""
    B, H = shape = _rows(x, "x")
    device, at, f32 = x.device, x.get_device(), torch.float32
    summed = residual is not None or s is not None or s_dtype not in (None, x.dtype)
    if residual is not None and s_dtype is not None and s_dtype != residual.dtype:
        raise ValueError("residual and s share a dtype")
    s_dt = residual.dtype if residual is not None else s.dtype if s is not None else s_dtype or x.dtype
    if s_dt not in _TORCH_DT:
        raise ValueError(f"s must be float32 or bfloat16, got {s_dt}")
    q = q_scale = y_at = s_at = rstd_at = None
    residual_at = _like(residual, "residual", at, shape)
    if packed is not None:
        q, q_scale, _ = _packed(packed, at, shape)
    elif pack:
        packed, q, q_scale = _new_packed(x)
    if y is not None or want_y:
        y, y_at = _out(y, "y", at, x, None, new=y_dtype or x.dtype)
    elif packed is None:
        raise ValueError("neither y nor packed rows are wanted")
    if summed:
        s, s_at = _out(s, "s", at, x, None, s_dt)
    if stats or rstd is not None:
        rstd, rstd_at = _out(rstd, "rstd", at, x, (B,), f32)
    _run(_lib().fff_rms_norm, FffRmsNormArgs(
        x.data_ptr(), residual_at, _like(gamma, "gamma", at, (H,), f32), y_at, s_at, rstd_at, q, q_scale, B, H,
        _dt(x, "x"), _TORCH_DT[s_dt], _dt(y, "y") if y is not None else FFF_F32, eps, _raw_stream(device, stream)))
    return y, s if summed else x, rstd, packed


def rms_norm_backward_workspace_bytes(n_tokens: int, hidden: int) -> int:
    _sizes((hidden, "hidden"))
    return int(_lib().fff_rms_norm_backward_workspace_bytes(n_tokens, hidden))


@_on_call
def rms_norm_backward(dy, s, rstd, gamma=None, *, ds_in=None, ds=None, dx=None, dgamma=None, accumulate=False,
                      dx_dtype=None, workspace=None, want=("ds", "dx", "dgamma"), stream=None):
    """Gradients of ``rms_norm`` through ``fff_rms_norm_backward``; returns (ds, dx, dgamma).

    ``s`` and ``rstd`` are the forward's.  ``ds_in`` is the gradient that reaches s past the norm; ``ds``
    (of s's type; may be ``ds_in``) is the gradient of s and of the residual, ``dx`` the same for x: ds itself, unless
    a dx or another ``dx_dtype`` than ds's is passed.  Gradients named in ``want`` are allocated when not given;
    ``accumulate`` adds to dgamma, which must then be given."""
    B, H = shape = _rows(dy, "dy")
    device, at, f32 = dy.device, dy.get_device(), torch.float32
    if s is None or rstd is None:
        raise ValueError("s and rstd are needed")
    _like(s, "s", at, shape)
    alias = dx is None and dx_dtype in (None, s.dtype)  # dx is ds
    if alias and "dx" in want and "ds" not in want:
        want = tuple(want) + ("ds",)
    if accumulate and "dgamma" in want and dgamma is None:
        raise ValueError("accumulate adds to the dgamma that is given")
    ds_at = dx_at = dgamma_at = None
    if ds is not None or "ds" in want:
        ds, ds_at = _out(ds, "ds", at, s, None, s.dtype)
    if dx is not None or (not alias and "dx" in want):
        dx, dx_at = _out(dx, "dx", at, dy, None, new=dx_dtype or dy.dtype)
    if dgamma is not None or "dgamma" in want:
        dgamma, dgamma_at = _out(dgamma, "dgamma", at, dy, (H,), f32)
        if workspace is None:
            workspace = dy.new_empty(max(256, rms_norm_backward_workspace_bytes(B, H)), dtype=torch.uint8)
    _run(_lib().fff_rms_norm_backward, FffRmsNormBackwardArgs(
        dy.data_ptr(), s.data_ptr(), _like(rstd, "rstd", at, (B,), f32), _like(gamma, "gamma", at, (H,), f32),
        _like(ds_in, "ds_in", at, shape, s.dtype), ds_at, dx_at, dgamma_at, B, H,
        _dt(dx, "dx") if dx is not None else FFF_F32, _dt(s, "s"), _dt(dy, "dy"), int(bool(accumulate)),
        *_scratch(workspace, "workspace", at), _raw_stream(device, stream)))
    return ds, (ds if "dx" in want else None) if alias else dx, dgamma


@_on_call
def pack_rows(x, *, packed=None, stream=None):
    """x's rows in 8 bits through ``fff_pack_rows``: an activation kept for the backward pass; returns a ``Packed``.

    e4m3 values and a power of two for every 32 columns of a row: 8.25 bits a value, each within 2^-4 of
    itself (of its block's smallest steps where it is far below the block's largest)."""
    shape = _rows(x, "x")
    device, at = x.device, x.get_device()
    if packed is None:
        packed, q, q_scale = _new_packed(x)
    else:
        q, q_scale, _ = _packed(packed, at, shape)
    _run(_lib().fff_pack_rows, FffPackRowsArgs(x.data_ptr(), q, q_scale, shape[0], shape[1], _dt(x, "x"),
                                               _raw_stream(device, stream)))
    return packed


@_on_call
def _unpack_rows(values, packed, act, y, dtype, *, stream=None):
    q, q_scale, shape = _packed(packed, None)
    y, y_at = _out(y, "y", values.get_device(), values, None, new=dtype)
    _run(_lib().fff_unpack_rows, FffUnpackRowsArgs(
        q, q_scale, None, y_at, None, shape[0], shape[1], FFF_F32, _dt(y, "y"), FFF_F32, _choice(ACTS, act, "act"),
        _raw_stream(values.device, stream)))
    return y


def unpack_rows(packed, *, act="identity", y=None, dtype=torch.bfloat16, stream=None):
    """``act`` of the rows that ``packed`` holds, through ``fff_unpack_rows``; returns y (allocated of ``dtype``).

    With the identity the packed values themselves, exact in float32 (in bfloat16 for scales of 2^-124 and more): an input of
    ``grouped_weight_grad``.  With "gelu" or "gelu_tanh" the activation of a packed pre-activation."""
    try:
        values = packed[0]
    except (TypeError, IndexError):
        raise ValueError("packed must be a Packed: values and scales") from None
    return _unpack_rows(values, packed, act, y, dtype, stream=stream)


@_on_call
def activation_backward(dy, packed, act="gelu", *, dx=None, dx_dtype=None, y=None, keep_y=False, y_dtype=None,
                        stream=None):
    """``dx = dy * act'(z)`` from a packed pre-activation z, through ``fff_unpack_rows``.

    Returns dx (of ``dx_dtype`` or dy's type; may be the buffer ``dy``), or (dx, y) with ``keep_y`` (or a
    ``y``): y = act(z), of ``y_dtype`` or dy's type, the next product's input for its weight gradient."""
    shape = _rows(dy, "dy")
    device, at = dy.device, dy.get_device()
    q, q_scale, _ = _packed(packed, at, shape)
    dx, dx_at = _out(dx, "dx", at, dy, None, new=dx_dtype or dy.dtype)
    keep_y, y_at = keep_y or y is not None, None
    if keep_y:
        y, y_at = _out(y, "y", at, dy, None, new=y_dtype or dy.dtype)
    _run(_lib().fff_unpack_rows, FffUnpackRowsArgs(
        q, q_scale, dy.data_ptr(), y_at, dx_at, shape[0], shape[1], _dt(dy, "dy"),
        _dt(y, "y") if y is not None else FFF_F32, _dt(dx, "dx"), _choice(ACTS, act, "act"), _raw_stream(device, stream)))
    return (dx, y) if keep_y else dx

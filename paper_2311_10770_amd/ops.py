"""ctypes binding of the operators around the layer (include/fff.h): LayerNorm with its residual,
dropout and gradients, dropout alone, the grouping of entries by leaf, and the leaf experts'
products with their weight gradients.

Argument marshalling only, as in ``fff.py``: contiguous float32 or bfloat16 GPU tensors, everything
computed by the library's HIP kernels on the call's stream.  Results and scratch that the caller does
not pass are allocated per call, in the order of the call's stream (inside a captured graph, from
that graph's own memory), so no two calls and no two graphs share any.
"""
from __future__ import annotations

import contextlib
import ctypes
from ctypes import c_double, c_float, c_int32, c_int64, c_size_t, c_uint64, c_void_p

import torch

from .fff import _TORCH_DT, ACTS, FFF_F32, _check, _dt, _on_device, _raw_stream, load_library


class FffDropoutRng(ctypes.Structure):
    """Mirror of ``fff_dropout_rng`` in include/fff.h."""

    _fields_ = [("p", c_double), ("seed", c_uint64), ("offset", c_uint64), ("rng_offset", c_void_p)]


class FffLayerNormArgs(ctypes.Structure):
    """Mirror of ``fff_layer_norm_args`` in include/fff.h."""

    _fields_ = [
        ("x", c_void_p), ("residual", c_void_p), ("gamma", c_void_p), ("beta", c_void_p),
        ("y", c_void_p), ("s", c_void_p), ("mean", c_void_p), ("rstd", c_void_p),
        ("n_tokens", c_int64), ("hidden", c_int32), ("x_dtype", c_int32), ("s_dtype", c_int32), ("y_dtype", c_int32),
        ("eps", c_float), ("drop", FffDropoutRng), ("hip_stream", c_void_p),
    ]


class FffLayerNormBackwardArgs(ctypes.Structure):
    """Mirror of ``fff_layer_norm_backward_args`` in include/fff.h."""

    _fields_ = [
        ("dy", c_void_p), ("s", c_void_p), ("mean", c_void_p), ("rstd", c_void_p), ("gamma", c_void_p),
        ("ds_in", c_void_p), ("ds", c_void_p), ("dx", c_void_p), ("dgamma", c_void_p), ("dbeta", c_void_p),
        ("n_tokens", c_int64), ("hidden", c_int32), ("x_dtype", c_int32), ("s_dtype", c_int32), ("y_dtype", c_int32),
        ("accumulate", c_int32), ("drop", FffDropoutRng), ("workspace", c_void_p), ("workspace_bytes", c_size_t),
        ("hip_stream", c_void_p),
    ]


class FffDropoutArgs(ctypes.Structure):
    """Mirror of ``fff_dropout_args`` in include/fff.h."""

    _fields_ = [
        ("x", c_void_p), ("residual", c_void_p), ("y", c_void_p),
        ("n_tokens", c_int64), ("hidden", c_int32), ("x_dtype", c_int32), ("r_dtype", c_int32), ("y_dtype", c_int32),
        ("drop", FffDropoutRng), ("hip_stream", c_void_p),
    ]


class FffGroupRowsArgs(ctypes.Structure):
    """Mirror of ``fff_group_rows_args`` in include/fff.h."""

    _fields_ = [
        ("ids", c_void_p), ("order", c_void_p), ("offsets", c_void_p), ("bad_ids", c_void_p),
        ("n_entries", c_int64), ("n_ids", c_int32), ("n_trees", c_int32), ("first", c_int32),
        ("workspace", c_void_p), ("workspace_bytes", c_size_t), ("hip_stream", c_void_p),
    ]


class FffGroupedMatmulArgs(ctypes.Structure):
    """Mirror of ``fff_grouped_matmul_args`` in include/fff.h."""

    _fields_ = [
        ("x", c_void_p), ("w", c_void_p), ("offsets", c_void_p), ("x_index", c_void_p), ("y_index", c_void_p),
        ("y", c_void_p), ("z_out", c_void_p), ("z_in", c_void_p),
        ("n_entries", c_int64), ("x_rows", c_int64), ("y_rows", c_int64),
        ("n_groups", c_int32), ("k", c_int32), ("n", c_int32), ("x_div", c_int32), ("w_transposed", c_int32),
        ("x_dtype", c_int32), ("w_dtype", c_int32), ("y_dtype", c_int32), ("z_dtype", c_int32),
        ("act", c_int32), ("hip_stream", c_void_p),
    ]


class FffGroupedWeightGradArgs(ctypes.Structure):
    """Mirror of ``fff_grouped_weight_grad_args`` in include/fff.h."""

    _fields_ = [
        ("dy", c_void_p), ("x", c_void_p), ("offsets", c_void_p), ("dy_index", c_void_p), ("x_index", c_void_p),
        ("dw", c_void_p), ("n_entries", c_int64), ("dy_rows", c_int64), ("x_rows", c_int64),
        ("n_groups", c_int32), ("k", c_int32), ("n", c_int32), ("x_div", c_int32),
        ("dy_dtype", c_int32), ("x_dtype", c_int32), ("accumulate", c_int32),
        ("workspace", c_void_p), ("workspace_bytes", c_size_t), ("hip_stream", c_void_p),
    ]


def _gpu(t, what: str, device=None):
    """``t`` as a contiguous GPU tensor (on ``device``)."""
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{what} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{what} must be a GPU tensor")
    if device is not None and t.device != device:
        raise ValueError(f"{what} is on {t.device}, expected {device}")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return t


def _like(t, what, device, shape, dtype=None):
    """Pointer of an optional tensor of exactly ``shape`` (and ``dtype``), or None."""
    if t is None:
        return None
    _gpu(t, what, device)
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what} must be {list(shape)}, got {tuple(t.shape)}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{what} must be {dtype}, got {t.dtype}")
    return t.data_ptr()


def _index(t, what, device, n):
    """Pointer of an optional int32 tensor of n elements, or None."""
    if t is None:
        return None
    _gpu(t, what, device)
    if t.dtype != torch.int32 or t.numel() != n:
        raise ValueError(f"{what} must be int32 with {n} elements")
    return t.data_ptr()


def _on_stream(stream):
    """Allocations of a call on ``stream`` belong to that stream."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _set_rng(drop, p, seed, offset, rng_offset, device):
    p = float(p)
    if not 0.0 <= p < 1.0:
        raise ValueError("p must be in [0, 1)")
    if not (0 <= seed < 1 << 64 and 0 <= offset < 1 << 64):
        raise ValueError("seed and offset must fit 64 unsigned bits")
    drop.p, drop.seed, drop.offset = p, seed, offset
    if rng_offset is not None:
        _gpu(rng_offset, "rng_offset", device)
        if rng_offset.dtype != torch.int64 or rng_offset.numel() != 1:
            raise ValueError("rng_offset must be one int64")
        drop.rng_offset = rng_offset.data_ptr()


def _rows(x, what: str):
    _gpu(x, what)
    if x.dim() != 2:
        raise ValueError(f"{what} must be a 2-D tensor [n_tokens, hidden]")
    return x.shape


def _run(fn, args, device):
    with _on_device(device):
        _check(getattr(load_library(), fn)(ctypes.addressof(args)))


def layer_norm(x, gamma=None, beta=None, *, eps=1e-12, residual=None, p=0.0, seed=0, offset=0, rng_offset=None, y=None,
               s=None, mean=None, rstd=None, y_dtype=None, s_dtype=None, stats=True, stream=None):
    """``s = residual + drop(x)``, then ``y = (s - mean) * rstd * gamma + beta`` per row, through ``fff_layer_norm``.

    Returns (y, s, mean, rstd).  Without a residual and with p = 0, s is x itself.  With ``stats``
    false, mean and rstd are None unless passed.  ``s`` may be ``residual`` (the stream updated in
    place).  Types of what is allocated: y as ``y_dtype`` or x; s as ``s_dtype``, residual or x."""
    B, H = _rows(x, "x")
    device = x.device
    a = FffLayerNormArgs()
    summed = residual is not None or p > 0
    if not summed and s is not None:
        raise ValueError("s is x itself without a residual and dropout")
    if residual is not None and s_dtype is not None and s_dtype != residual.dtype:
        raise ValueError("residual and s share a dtype")
    s_dt = residual.dtype if residual is not None else s.dtype if s is not None else s_dtype or x.dtype
    with _on_device(device), _on_stream(stream):
        if y is None:
            y = torch.empty((B, H), dtype=y_dtype or x.dtype, device=device)
        if summed and s is None:
            s = torch.empty((B, H), dtype=s_dt, device=device)
        if stats and mean is None:
            mean = torch.empty(B, dtype=torch.float32, device=device)
        if stats and rstd is None:
            rstd = torch.empty(B, dtype=torch.float32, device=device)
    a.x = x.data_ptr()
    a.residual = _like(residual, "residual", device, (B, H))
    a.gamma = _like(gamma, "gamma", device, (H,), torch.float32)
    a.beta = _like(beta, "beta", device, (H,), torch.float32)
    a.y = _like(y, "y", device, (B, H))
    a.s = _like(s, "s", device, (B, H), s_dt)
    a.mean = _like(mean, "mean", device, (B,), torch.float32)
    a.rstd = _like(rstd, "rstd", device, (B,), torch.float32)
    a.n_tokens, a.hidden = B, H
    a.x_dtype, a.y_dtype = _dt(x, "x"), _dt(y, "y")
    a.s_dtype = _TORCH_DT.get(s_dt, -1)
    if a.s_dtype < 0:
        raise ValueError(f"s must be float32 or bfloat16, got {s_dt}")
    a.eps = eps
    if p or rng_offset is not None:
        _set_rng(a.drop, p, seed, offset, rng_offset, device)
    a.hip_stream = _raw_stream(device, stream)
    _run("fff_layer_norm", a, device)
    return y, s if summed else x, mean, rstd


def layer_norm_backward_workspace_bytes(n_tokens: int, hidden: int) -> int:
    return int(load_library().fff_layer_norm_backward_workspace_bytes(n_tokens, hidden))


def layer_norm_backward(dy, s, mean, rstd, gamma=None, *, ds_in=None, p=0.0, seed=0, offset=0, rng_offset=None, ds=None,
                        dx=None, dgamma=None, dbeta=None, accumulate=False, dx_dtype=None, workspace=None,
                        want=("ds", "dx", "dgamma", "dbeta"), stream=None):
    """Gradients of ``layer_norm`` through ``fff_layer_norm_backward``; returns (ds, dx, dgamma, dbeta).

    ``s``, ``mean`` and ``rstd`` are the forward's, ``p``, ``seed`` and ``offset`` its dropout's.
    ``ds_in`` is the gradient that reaches s past the norm; ``ds`` (of s's type; may be ``ds_in``) is
    the gradient of s and of the residual, ``dx`` (``dx_dtype`` or dy's type) that of x behind the
    dropout: ds itself where p = 0, unless a dx is passed.  Gradients named in ``want`` are allocated when
    not given; ``accumulate`` adds to dgamma and dbeta, which must then be given."""
    B, H = _rows(dy, "dy")
    device = dy.device
    a = FffLayerNormBackwardArgs()
    a.dy = dy.data_ptr()
    a.s = _like(s, "s", device, (B, H))
    a.mean = _like(mean, "mean", device, (B,), torch.float32)
    a.rstd = _like(rstd, "rstd", device, (B,), torch.float32)
    if s is None or mean is None or rstd is None:
        raise ValueError("s, mean and rstd are needed")
    alias = dx is None and p == 0  # dx is ds
    if alias and "dx" in want and "ds" not in want:
        want = tuple(want) + ("ds",)
    if accumulate and (("dgamma" in want and dgamma is None) or ("dbeta" in want and dbeta is None)):
        raise ValueError("accumulate adds to the dgamma and dbeta that are given")
    with _on_device(device), _on_stream(stream):
        if ds is None and "ds" in want:
            ds = torch.empty((B, H), dtype=s.dtype, device=device)
        if dx is None and not alias and "dx" in want:
            dx = torch.empty((B, H), dtype=dx_dtype or dy.dtype, device=device)
        if dgamma is None and "dgamma" in want:
            dgamma = torch.empty(H, dtype=torch.float32, device=device)
        if dbeta is None and "dbeta" in want:
            dbeta = torch.empty(H, dtype=torch.float32, device=device)
        if workspace is None and (dgamma is not None or dbeta is not None):
            workspace = torch.empty(max(256, layer_norm_backward_workspace_bytes(B, H)), dtype=torch.uint8, device=device)
    a.gamma = _like(gamma, "gamma", device, (H,), torch.float32)
    a.ds_in = _like(ds_in, "ds_in", device, (B, H), s.dtype)
    a.ds = _like(ds, "ds", device, (B, H), s.dtype)
    a.dx = _like(dx, "dx", device, (B, H))
    a.dgamma = _like(dgamma, "dgamma", device, (H,), torch.float32)
    a.dbeta = _like(dbeta, "dbeta", device, (H,), torch.float32)
    a.n_tokens, a.hidden = B, H
    a.y_dtype, a.s_dtype = _dt(dy, "dy"), _dt(s, "s")
    a.x_dtype = _dt(dx, "dx") if dx is not None else FFF_F32
    a.accumulate = int(bool(accumulate))
    if p or rng_offset is not None:
        _set_rng(a.drop, p, seed, offset, rng_offset, device)
    if workspace is not None:
        _gpu(workspace, "workspace", device)
        a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    a.hip_stream = _raw_stream(device, stream)
    _run("fff_layer_norm_backward", a, device)
    return ds, (ds if "dx" in want else None) if alias else dx, dgamma, dbeta


def dropout(x, p, seed, offset=0, *, rng_offset=None, residual=None, y=None, y_dtype=None, stream=None):
    """``y = residual + drop(x)`` (residual optional) through ``fff_dropout``; y may be x or residual.

    The gradient of x is ``dropout(dy, p, seed, offset)``: the mask is drawn again, never stored.
    Without a y it is allocated, of ``y_dtype`` or x's type."""
    B, H = _rows(x, "x")
    device = x.device
    a = FffDropoutArgs()
    if y is None:
        with _on_device(device), _on_stream(stream):
            y = torch.empty((B, H), dtype=y_dtype or x.dtype, device=device)
    a.x = x.data_ptr()
    a.residual = _like(residual, "residual", device, (B, H))
    a.y = _like(y, "y", device, (B, H))
    a.n_tokens, a.hidden = B, H
    a.x_dtype, a.y_dtype = _dt(x, "x"), _dt(y, "y")
    a.r_dtype = _dt(residual, "residual") if residual is not None else FFF_F32
    _set_rng(a.drop, p, seed, offset, rng_offset, device)
    a.hip_stream = _raw_stream(device, stream)
    _run("fff_dropout", a, device)
    return y


def group_rows_workspace_bytes(n_entries: int, n_ids: int, n_trees: int = 1) -> int:
    return int(load_library().fff_group_rows_workspace_bytes(n_entries, n_ids, n_trees))


def group_rows(ids, n_ids: int, *, first: int = 0, n_trees: int = 1, order=None, offsets=None, bad_ids=None,
               workspace=None, stream=None):
    """Entries by group through ``fff_group_rows``; returns (order, offsets), int32.

    ``ids``: int32, any shape, flattened to the entries (token by token, its trees together); entry e
    belongs to group (e % n_trees) * n_ids + ids[e] - first.  ``order`` holds the entries group by
    group, ``offsets`` [n_trees * n_ids + 1] where each group's stand.  For the leaves of a forward:
    ``group_rows(nodes_out[..., depth].contiguous(), 2**depth, first=2**depth - 1, n_trees=n_trees)``."""
    _gpu(ids, "ids")
    device, E = ids.device, ids.numel()
    if ids.dtype != torch.int32:
        raise ValueError("ids must be int32")
    if n_ids < 1 or n_trees < 1:
        raise ValueError("n_ids and n_trees must be positive")
    G = n_ids * n_trees
    with _on_device(device), _on_stream(stream):
        if order is None:
            order = torch.empty(E, dtype=torch.int32, device=device)
        if offsets is None:
            offsets = torch.empty(G + 1, dtype=torch.int32, device=device)
        if workspace is None:
            workspace = torch.empty(max(256, group_rows_workspace_bytes(E, n_ids, n_trees)), dtype=torch.uint8,
                                    device=device)
    a = FffGroupRowsArgs()
    a.ids = ids.data_ptr()
    a.order = _index(order, "order", device, E)
    a.offsets = _index(offsets, "offsets", device, G + 1)
    a.bad_ids = _index(bad_ids, "bad_ids", device, 1)
    a.n_entries, a.n_ids, a.n_trees, a.first = E, n_ids, n_trees, first
    _gpu(workspace, "workspace", device)
    a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    a.hip_stream = _raw_stream(device, stream)
    _run("fff_group_rows", a, device)
    return order, offsets


def _entries(x, index, x_div, what):
    """How many entries read x's rows."""
    return index.numel() if index is not None else x.shape[0] * x_div


def grouped_matmul(x, w, offsets, *, x_index=None, x_div=1, y=None, y_index=None, y_dtype=None, transpose_w=False,
                   act="identity", z_out=None, keep_z=False, z_in=None, stream=None):
    """Every entry's row times its group's matrix, through ``fff_grouped_matmul``.

    ``w`` [n_groups, n, k] gives ``act(x W_g^T)``, with ``transpose_w`` [n_groups, k, n] gives
    ``act(x W_g)``, for the entries offsets[g] .. offsets[g + 1] of each group.  Entry i reads row
    ``x_index[i] // x_div`` of x (i // x_div without an index) and writes row ``y_index[i]`` of y (i
    without).  ``keep_z`` (or a ``z_out``) also stores the product before the activation, in grouped
    order; with ``z_in`` the result is ``z * act'(z_in)``, the data gradient through the activation.
    Returns y, or (y, z) when z is kept.  y without an argument is allocated with a row per entry;
    its rows that no entry names are not written."""
    _gpu(x, "x")
    _gpu(w, "w", x.device)
    if x.dim() != 2 or w.dim() != 3:
        raise ValueError("x must be [rows, k] and w [n_groups, n, k] ([n_groups, k, n] with transpose_w)")
    if x_div < 1:
        raise ValueError("x_div must be positive")
    device = x.device
    G, N, K = (w.shape[0], w.shape[2], w.shape[1]) if transpose_w else w.shape
    if x.shape[1] != K:
        raise ValueError(f"x has rows of {x.shape[1]}, w takes {K}")
    E = _entries(x, x_index, x_div, "x")
    a = FffGroupedMatmulArgs()
    keep_z = keep_z or z_out is not None
    if keep_z and z_in is not None:
        raise ValueError("z_in makes a gradient: no z is kept")
    if y is None or (keep_z and z_out is None):
        with _on_device(device), _on_stream(stream):
            if y is None:
                y = torch.empty((E, N), dtype=y_dtype or x.dtype, device=device)
            if keep_z and z_out is None:
                z_out = torch.empty((E, N), dtype=y.dtype, device=device)
    _gpu(y, "y", device)
    if y.dim() != 2 or y.shape[1] != N:
        raise ValueError(f"y must have rows of {N}")
    a.x, a.w, a.y = x.data_ptr(), w.data_ptr(), y.data_ptr()
    if offsets is None:
        raise ValueError("offsets are needed")
    a.offsets = _index(offsets, "offsets", device, G + 1)
    a.x_index = _index(x_index, "x_index", device, E)
    a.y_index = _index(y_index, "y_index", device, E)
    a.z_out = _like(z_out, "z_out", device, (E, N))
    a.z_in = _like(z_in, "z_in", device, (E, N))
    z = z_out if z_out is not None else z_in
    a.n_entries, a.x_rows, a.y_rows = E, x.shape[0], y.shape[0]
    a.n_groups, a.k, a.n, a.x_div, a.w_transposed = G, K, N, x_div, int(bool(transpose_w))
    a.x_dtype, a.w_dtype, a.y_dtype = _dt(x, "x"), _dt(w, "w"), _dt(y, "y")
    a.z_dtype = _dt(z, "z") if z is not None else FFF_F32
    a.act = ACTS[act] if isinstance(act, str) else int(act)
    a.hip_stream = _raw_stream(device, stream)
    _run("fff_grouped_matmul", a, device)
    return (y, z_out) if keep_z else y


def grouped_weight_grad_workspace_bytes(n_entries: int, n_groups: int, k: int, n: int) -> int:
    return int(load_library().fff_grouped_weight_grad_workspace_bytes(n_entries, n_groups, k, n))


def grouped_weight_grad(dy, x, offsets, *, dy_index=None, x_index=None, x_div=1, dw=None, accumulate=False,
                        workspace=None, stream=None):
    """``dW_g = sum dy_i^T x_i`` over every group's entries, through ``fff_grouped_weight_grad``.

    Returns dw, float32 [n_groups, n, k] (zeros for groups without entries), added to with
    ``accumulate``.  Entry i reads row ``dy_index[i]`` of dy (i without) and ``x_index[i] // x_div`` of
    x (i // x_div without).  For a W used transposed, pass x as ``dy`` and dy as ``x``."""
    _gpu(dy, "dy")
    _gpu(x, "x", dy.device)
    if x.dim() != 2 or dy.dim() != 2:
        raise ValueError("dy must be [rows, n] and x [rows, k]")
    if x_div < 1:
        raise ValueError("x_div must be positive")
    if offsets is None or offsets.numel() < 2:
        raise ValueError("offsets must hold n_groups + 1 values")
    device = dy.device
    N, K, G = dy.shape[1], x.shape[1], offsets.numel() - 1
    E = dy_index.numel() if dy_index is not None else dy.shape[0]
    if accumulate and dw is None:
        raise ValueError("accumulate adds to the dw that is given")
    a = FffGroupedWeightGradArgs()
    need = grouped_weight_grad_workspace_bytes(E, G, K, N)
    if dw is None or (workspace is None and need):
        with _on_device(device), _on_stream(stream):
            if dw is None:
                dw = torch.empty((G, N, K), dtype=torch.float32, device=device)
            if workspace is None and need:
                workspace = torch.empty(need, dtype=torch.uint8, device=device)
    a.dy, a.x = dy.data_ptr(), x.data_ptr()
    a.offsets = _index(offsets, "offsets", device, G + 1)
    a.dy_index = _index(dy_index, "dy_index", device, E)
    a.x_index = _index(x_index, "x_index", device, E)
    a.dw = _like(dw, "dw", device, (G, N, K), torch.float32)
    a.n_entries, a.dy_rows, a.x_rows = E, dy.shape[0], x.shape[0]
    a.n_groups, a.k, a.n, a.x_div = G, K, N, x_div
    a.dy_dtype, a.x_dtype = _dt(dy, "dy"), _dt(x, "x")
    a.accumulate = int(bool(accumulate))
    if workspace is not None:
        _gpu(workspace, "workspace", device)
        a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    a.hip_stream = _raw_stream(device, stream)
    _run("fff_grouped_weight_grad", a, device)
    return dw

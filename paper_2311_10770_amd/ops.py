"""ctypes binding of the operators around the layer (include/fff.h): LayerNorm with its residual,
dropout and gradients, dropout alone, the grouping of entries by leaf, and the leaf experts'
products with their weight gradients.

Argument marshalling only, as in ``fff.py``: contiguous float32 or bfloat16 GPU tensors, everything
computed by the library's HIP kernels on the call's stream.  Results and scratch that the caller does
not pass are allocated per call, in the order of the call's stream (inside a captured graph, from
that graph's own memory), so no two calls and no two graphs share any.
"""
from __future__ import annotations

import ctypes
import functools
import inspect
from ctypes import c_double, c_float, c_int32, c_int64, c_size_t, c_uint64, c_void_p

import torch

from .fff import _TORCH_DT, ACTS, FFF_F32, _check, _dt, _raw_stream, load_library


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


_get_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_LIB = None


def _lib():
    global _LIB
    if _LIB is None:
        _LIB = load_library()
    return _LIB


_INT32 = (1 << 31) - 1  # the library's sizes: a larger one would arrive cut to its low 32 bits


def _sizes(*named):
    """Refuses sizes, as (value, name) pairs, that the library's 32 bits do not hold."""
    for v, what in named:
        if not -_INT32 - 1 <= v <= _INT32:
            raise ValueError(f"{what} must fit 32 bits, got {v}")


def _gpu(t, what: str, index=None):
    """``t`` as a contiguous GPU tensor (on GPU ``index``)."""
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{what} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{what} must be a GPU tensor")
    if index is not None and t.get_device() != index:
        raise ValueError(f"{what} is on {t.device}, expected cuda:{index}")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return t


def _like(t, what, index, shape, dtype=None):
    """Pointer of an optional tensor of exactly ``shape`` (and ``dtype``), or None."""
    if t is None:
        return None
    _gpu(t, what, index)
    if t.shape != shape:
        raise ValueError(f"{what} must be {list(shape)}, got {tuple(t.shape)}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{what} must be {dtype}, got {t.dtype}")
    return t.data_ptr()


def _index(t, what, index, n):
    """Pointer of an optional int32 tensor of n elements, or None."""
    if t is None:
        return None
    _gpu(t, what, index)
    if t.dtype != torch.int32 or t.numel() != n:
        raise ValueError(f"{what} must be int32 with {n} elements")
    return t.data_ptr()


def _scratch(t, what, index):
    """Pointer and bytes of an optional workspace."""
    if t is None:
        return None, 0
    _gpu(t, what, index)
    return t.data_ptr(), t.numel() * t.element_size()


def _on_call(fn):
    """Runs ``fn`` with its first tensor's GPU current, and ``stream`` too when one is given: allocations then
    belong to the call's stream."""
    name = next(iter(inspect.signature(fn).parameters))

    @functools.wraps(fn)
    def call(*args, stream=None, **kw):
        t = args[0] if args else kw.get(name)
        if not (isinstance(t, torch.Tensor) and t.is_cuda):
            return fn(*args, stream=None, **kw)  # refused there
        if stream is None:
            if t.get_device() == _get_device():
                return fn(*args, stream=None, **kw)
            with torch.cuda.device(t.device):
                return fn(*args, stream=None, **kw)
        if stream.device != t.device:
            raise ValueError(f"stream is on {stream.device}, the tensors on {t.device}")
        with torch.cuda.stream(stream):
            return fn(*args, stream=stream, **kw)

    return call


_NO_DROP = FffDropoutRng()


def _rng(p, seed, offset, rng_offset, index):
    p = float(p)
    if not 0.0 <= p < 1.0:
        raise ValueError("p must be in [0, 1)")
    if not (0 <= seed < 1 << 64 and 0 <= offset < 1 << 64):
        raise ValueError("seed and offset must fit 64 unsigned bits")
    at = None
    if rng_offset is not None:
        _gpu(rng_offset, "rng_offset", index)
        if rng_offset.dtype != torch.int64 or rng_offset.numel() != 1:
            raise ValueError("rng_offset must be one int64")
        at = rng_offset.data_ptr()
    return FffDropoutRng(p, seed, offset, at)


def _rows(x, what: str):
    _gpu(x, what)
    if x.dim() != 2:
        raise ValueError(f"{what} must be a 2-D tensor [n_tokens, hidden]")
    if x.shape[1] > _INT32:
        raise ValueError(f"{what} has rows of {x.shape[1]}: hidden must fit 32 bits")
    return x.shape


def _run(fn, args):
    rc = fn(ctypes.addressof(args))
    if rc:
        _check(rc)


def _describe(fn, args) -> str:
    buf = ctypes.create_string_buffer(256)
    _check(fn(ctypes.addressof(args), buf, len(buf)))
    return buf.value.decode()


@_on_call
def layer_norm(x, gamma=None, beta=None, *, eps=1e-12, residual=None, p=0.0, seed=0, offset=0, rng_offset=None, y=None,
               s=None, mean=None, rstd=None, y_dtype=None, s_dtype=None, stats=True, stream=None):
    """``s = residual + drop(x)``, then ``y = (s - mean) * rstd * gamma + beta`` per row, through ``fff_layer_norm``.

    Returns (y, s, mean, rstd).  Without a residual and with p = 0, s is x itself, unless an s or another
    ``s_dtype`` than x's is passed.  With ``stats`` false, mean and rstd are None unless passed.  ``s``
    may be ``residual`` (the stream updated in place).  Types of what is allocated: y as ``y_dtype`` or x;
    s as ``s_dtype``, residual or x."""
    B, H = shape = _rows(x, "x")
    device, at = x.device, x.get_device()
    summed = residual is not None or p > 0 or s is not None or s_dtype not in (None, x.dtype)
    if residual is not None and s_dtype is not None and s_dtype != residual.dtype:
        raise ValueError("residual and s share a dtype")
    s_dt = residual.dtype if residual is not None else s.dtype if s is not None else s_dtype or x.dtype
    if s_dt not in _TORCH_DT:
        raise ValueError(f"s must be float32 or bfloat16, got {s_dt}")
    if y is None:
        y = torch.empty(shape, dtype=y_dtype or x.dtype, device=device)
    if summed and s is None:
        s = torch.empty(shape, dtype=s_dt, device=device)
    if stats and mean is None:
        mean = torch.empty(B, dtype=torch.float32, device=device)
    if stats and rstd is None:
        rstd = torch.empty(B, dtype=torch.float32, device=device)
    f32 = torch.float32
    _run(_lib().fff_layer_norm, FffLayerNormArgs(
        x.data_ptr(), _like(residual, "residual", at, shape), _like(gamma, "gamma", at, (H,), f32),
        _like(beta, "beta", at, (H,), f32), _like(y, "y", at, shape), _like(s, "s", at, shape, s_dt),
        _like(mean, "mean", at, (B,), f32), _like(rstd, "rstd", at, (B,), f32), B, H, _dt(x, "x"), _TORCH_DT[s_dt],
        _dt(y, "y"), eps, _rng(p, seed, offset, rng_offset, at) if p or rng_offset is not None else _NO_DROP,
        _raw_stream(device, stream)))
    return y, s if summed else x, mean, rstd


def layer_norm_backward_workspace_bytes(n_tokens: int, hidden: int) -> int:
    _sizes((hidden, "hidden"))
    return int(_lib().fff_layer_norm_backward_workspace_bytes(n_tokens, hidden))


@_on_call
def layer_norm_backward(dy, s, mean, rstd, gamma=None, *, ds_in=None, p=0.0, seed=0, offset=0, rng_offset=None, ds=None,
                        dx=None, dgamma=None, dbeta=None, accumulate=False, dx_dtype=None, workspace=None,
                        want=("ds", "dx", "dgamma", "dbeta"), stream=None):
    """Gradients of ``layer_norm`` through ``fff_layer_norm_backward``; returns (ds, dx, dgamma, dbeta).

    ``s``, ``mean`` and ``rstd`` are the forward's, ``p``, ``seed`` and ``offset`` its dropout's.
    ``ds_in`` is the gradient that reaches s past the norm; ``ds`` (of s's type; may be ``ds_in``) is
    the gradient of s and of the residual, ``dx`` (``dx_dtype`` or dy's type) that of x behind the
    dropout: ds itself where p = 0, unless a dx or another ``dx_dtype`` than ds's is passed.
    Gradients named in ``want`` are allocated when not given; ``accumulate`` adds to dgamma and dbeta,
    which must then be given."""
    B, H = shape = _rows(dy, "dy")
    device, at, f32 = dy.device, dy.get_device(), torch.float32
    if s is None or mean is None or rstd is None:
        raise ValueError("s, mean and rstd are needed")
    _like(s, "s", at, shape)
    alias = dx is None and p == 0 and dx_dtype in (None, s.dtype)  # dx is ds
    if alias and "dx" in want and "ds" not in want:
        want = tuple(want) + ("ds",)
    if accumulate and (("dgamma" in want and dgamma is None) or ("dbeta" in want and dbeta is None)):
        raise ValueError("accumulate adds to the dgamma and dbeta that are given")
    if ds is None and "ds" in want:
        ds = torch.empty(shape, dtype=s.dtype, device=device)
    if dx is None and not alias and "dx" in want:
        dx = torch.empty(shape, dtype=dx_dtype or dy.dtype, device=device)
    if dgamma is None and "dgamma" in want:
        dgamma = torch.empty(H, dtype=f32, device=device)
    if dbeta is None and "dbeta" in want:
        dbeta = torch.empty(H, dtype=f32, device=device)
    if workspace is None and (dgamma is not None or dbeta is not None):
        workspace = torch.empty(max(256, layer_norm_backward_workspace_bytes(B, H)), dtype=torch.uint8, device=device)
    _run(_lib().fff_layer_norm_backward, FffLayerNormBackwardArgs(
        dy.data_ptr(), s.data_ptr(), _like(mean, "mean", at, (B,), f32), _like(rstd, "rstd", at, (B,), f32),
        _like(gamma, "gamma", at, (H,), f32), _like(ds_in, "ds_in", at, shape, s.dtype),
        _like(ds, "ds", at, shape, s.dtype), _like(dx, "dx", at, shape), _like(dgamma, "dgamma", at, (H,), f32),
        _like(dbeta, "dbeta", at, (H,), f32), B, H, _dt(dx, "dx") if dx is not None else FFF_F32, _dt(s, "s"),
        _dt(dy, "dy"), int(bool(accumulate)),
        _rng(p, seed, offset, rng_offset, at) if p or rng_offset is not None else _NO_DROP,
        *_scratch(workspace, "workspace", at), _raw_stream(device, stream)))
    return ds, (ds if "dx" in want else None) if alias else dx, dgamma, dbeta


@_on_call
def dropout(x, p, seed, offset=0, *, rng_offset=None, residual=None, y=None, y_dtype=None, stream=None):
    """``y = residual + drop(x)`` (residual optional) through ``fff_dropout``; y may be x or residual.

    The gradient of x is ``dropout(dy, p, seed, offset)``: the mask is drawn again, never stored.
    Without a y it is allocated, of ``y_dtype`` or x's type."""
    B, H = shape = _rows(x, "x")
    device, at = x.device, x.get_device()
    if y is None:
        y = torch.empty(shape, dtype=y_dtype or x.dtype, device=device)
    _run(_lib().fff_dropout, FffDropoutArgs(
        x.data_ptr(), _like(residual, "residual", at, shape), _like(y, "y", at, shape), B, H, _dt(x, "x"),
        _dt(residual, "residual") if residual is not None else FFF_F32, _dt(y, "y"), _rng(p, seed, offset, rng_offset, at),
        _raw_stream(device, stream)))
    return y


def group_rows_workspace_bytes(n_entries: int, n_ids: int, n_trees: int = 1) -> int:
    _sizes((n_ids, "n_ids"), (n_trees, "n_trees"))
    return int(_lib().fff_group_rows_workspace_bytes(n_entries, n_ids, n_trees))


@_on_call
def group_rows(ids, n_ids: int, *, first: int = 0, n_trees: int = 1, order=None, offsets=None, bad_ids=None,
               workspace=None, stream=None):
    """Entries by group through ``fff_group_rows``; returns (order, offsets), int32.

    ``ids``: int32, any shape, flattened to the entries (token by token, its trees together); entry e
    belongs to group (e % n_trees) * n_ids + ids[e] - first.  ``order`` holds the entries group by
    group, ``offsets`` [n_trees * n_ids + 1] where each group's stand.  For the leaves of a forward:
    ``group_rows(nodes_out[..., depth].contiguous(), 2**depth, first=2**depth - 1, n_trees=n_trees)``."""
    _gpu(ids, "ids")
    device, at, E = ids.device, ids.get_device(), ids.numel()
    if ids.dtype != torch.int32:
        raise ValueError("ids must be int32")
    if n_ids < 1 or n_trees < 1:
        raise ValueError("n_ids and n_trees must be positive")
    if max(n_ids, n_trees, abs(first)) > _INT32:
        _sizes((n_ids, "n_ids"), (n_trees, "n_trees"), (first, "first"))
    G = n_ids * n_trees
    if order is None:
        order = torch.empty(E, dtype=torch.int32, device=device)
    if offsets is None:
        offsets = torch.empty(G + 1, dtype=torch.int32, device=device)
    if workspace is None:
        need = group_rows_workspace_bytes(E, n_ids, n_trees)
        workspace = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    _run(_lib().fff_group_rows, FffGroupRowsArgs(
        ids.data_ptr(), _index(order, "order", at, E), _index(offsets, "offsets", at, G + 1),
        _index(bad_ids, "bad_ids", at, 1), E, n_ids, n_trees, first, *_scratch(workspace, "workspace", at),
        _raw_stream(device, stream)))
    return order, offsets


def _product(x, w, offsets, *, x_index=None, x_div=1, y=None, y_index=None, y_dtype=None, transpose_w=False,
             act="identity", z_out=None, keep_z=False, z_in=None, stream=None):
    """Checked arguments and results of a product."""
    _gpu(x, "x")
    device, at = x.device, x.get_device()
    _gpu(w, "w", at)
    if x.dim() != 2 or w.dim() != 3:
        raise ValueError("x must be [rows, k] and w [n_groups, n, k] ([n_groups, k, n] with transpose_w)")
    if x_div < 1:
        raise ValueError("x_div must be positive")
    if offsets is None:
        raise ValueError("offsets are needed")
    G, N, K = w.shape
    if transpose_w:
        N, K = K, N
    if x.shape[1] != K:
        raise ValueError(f"x has rows of {x.shape[1]}, w takes {K}")
    if max(G, K, N, x_div) > _INT32:
        _sizes((G, "the number of groups"), (K, "k"), (N, "n"), (x_div, "x_div"))
    E = x_index.numel() if x_index is not None else x.shape[0] * x_div
    keep_z = keep_z or z_out is not None
    if keep_z and z_in is not None:
        raise ValueError("z_in makes a gradient: no z is kept")
    if y is None:
        y = torch.empty((E, N), dtype=y_dtype or x.dtype, device=device)
    _gpu(y, "y", at)
    if y.dim() != 2 or y.shape[1] != N:
        raise ValueError(f"y must have rows of {N}")
    if keep_z and z_out is None:
        z_out = torch.empty((E, N), dtype=y.dtype, device=device)
    z = z_out if z_out is not None else z_in
    args = FffGroupedMatmulArgs(
        x.data_ptr(), w.data_ptr(), _index(offsets, "offsets", at, G + 1), _index(x_index, "x_index", at, E),
        _index(y_index, "y_index", at, E), y.data_ptr(), _like(z_out, "z_out", at, (E, N)), _like(z_in, "z_in", at, (E, N)),
        E, x.shape[0], y.shape[0], G, K, N, x_div, int(bool(transpose_w)), _dt(x, "x"), _dt(w, "w"), _dt(y, "y"),
        _dt(z, "z") if z is not None else FFF_F32, ACTS[act] if isinstance(act, str) else int(act),
        _raw_stream(device, stream))
    return args, (y, z_out) if keep_z else y


@_on_call
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
    args, out = _product(x, w, offsets, x_index=x_index, x_div=x_div, y=y, y_index=y_index, y_dtype=y_dtype,
                         transpose_w=transpose_w, act=act, z_out=z_out, keep_z=keep_z, z_in=z_in, stream=stream)
    _run(_lib().fff_grouped_matmul, args)
    return out


@_on_call
def describe_grouped_matmul(x, w, offsets, **kw) -> str:
    """The kernel and launch shape that ``grouped_matmul`` would use."""
    return _describe(_lib().fff_describe_grouped_matmul, _product(x, w, offsets, **kw)[0])


def grouped_weight_grad_workspace_bytes(n_entries: int, n_groups: int, k: int, n: int) -> int:
    _sizes((n_groups, "n_groups"), (k, "k"), (n, "n"))
    return int(_lib().fff_grouped_weight_grad_workspace_bytes(n_entries, n_groups, k, n))


def _weight_grad(dy, x, offsets, *, dy_index=None, x_index=None, x_div=1, dw=None, accumulate=False,
                 workspace=None, stream=None):
    """Checked arguments, result and scratch of a weight gradient."""
    _gpu(dy, "dy")
    device, at = dy.device, dy.get_device()
    _gpu(x, "x", at)
    if x.dim() != 2 or dy.dim() != 2:
        raise ValueError("dy must be [rows, n] and x [rows, k]")
    if x_div < 1:
        raise ValueError("x_div must be positive")
    if offsets is None or offsets.numel() < 2:
        raise ValueError("offsets must hold n_groups + 1 values")
    N, K, G = dy.shape[1], x.shape[1], offsets.numel() - 1
    if max(G, K, N, x_div) > _INT32:
        _sizes((G, "the number of groups"), (K, "k"), (N, "n"), (x_div, "x_div"))
    E = dy_index.numel() if dy_index is not None else dy.shape[0]
    if accumulate and dw is None:
        raise ValueError("accumulate adds to the dw that is given")
    if dw is None:
        dw = torch.empty((G, N, K), dtype=torch.float32, device=device)
    if workspace is None:
        need = grouped_weight_grad_workspace_bytes(E, G, K, N)
        workspace = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    args = FffGroupedWeightGradArgs(
        dy.data_ptr(), x.data_ptr(), _index(offsets, "offsets", at, G + 1), _index(dy_index, "dy_index", at, E),
        _index(x_index, "x_index", at, E), _like(dw, "dw", at, (G, N, K), torch.float32), E, dy.shape[0], x.shape[0],
        G, K, N, x_div, _dt(dy, "dy"), _dt(x, "x"), int(bool(accumulate)), *_scratch(workspace, "workspace", at),
        _raw_stream(device, stream))
    return args, dw, workspace


@_on_call
def grouped_weight_grad(dy, x, offsets, *, dy_index=None, x_index=None, x_div=1, dw=None, accumulate=False,
                        workspace=None, stream=None):
    """``dW_g = sum dy_i^T x_i`` over every group's entries, through ``fff_grouped_weight_grad``.

    Returns dw, float32 [n_groups, n, k] (zeros for groups without entries), added to with
    ``accumulate``.  Entry i reads row ``dy_index[i]`` of dy (i without) and ``x_index[i] // x_div`` of
    x (i // x_div without).  For a W used transposed, pass x as ``dy`` and dy as ``x``."""
    args, dw, _scratch_held = _weight_grad(dy, x, offsets, dy_index=dy_index, x_index=x_index, x_div=x_div, dw=dw,
                                           accumulate=accumulate, workspace=workspace, stream=stream)
    _run(_lib().fff_grouped_weight_grad, args)
    return dw


@_on_call
def describe_grouped_weight_grad(dy, x, offsets, **kw) -> str:
    """The kernel and launch shape that ``grouped_weight_grad`` would use."""
    args, _dw, _scratch_held = _weight_grad(dy, x, offsets, **kw)
    return _describe(_lib().fff_describe_grouped_weight_grad, args)

"""The operators around the layer in 64 bits, and how far fp32 arithmetic may be off (the tests' references).

Every bound counts roundings of U = 2^-24 (fp32, half a step) in any order of a sum of n terms (n U times the
sum of the terms' sizes), plus half a step of the output's type.
"""
from __future__ import annotations

import math

import numpy as np
import torch

U = 2.0 ** -24
F8 = torch.float64


def half_step(dtype) -> float:
    return torch.finfo(dtype).eps / 2


def philox_words(c0, c1, offset: int, seed: int) -> np.ndarray:
    """Philox4x32-10 at counters (c0, c1, offset low, offset high), key seed: uint64 array [..., 4]."""
    u, low = np.uint64, np.uint64(0xFFFFFFFF)
    c = [np.asarray(c0, u), np.asarray(c1, u), np.asarray(offset & 0xFFFFFFFF, u), np.asarray(offset >> 32, u)]
    c = list(np.broadcast_arrays(*c))
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        a, b = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = [(b >> u(32)) ^ c[1] ^ u(k[0]), b & low, (a >> u(32)) ^ c[3] ^ u(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, -1)


def kept(rows, H: int, p: float, seed: int, offset: int) -> torch.Tensor:
    """Which elements of the given rows (a count, or row numbers) dropout keeps."""
    rows = np.arange(rows) if isinstance(rows, int) else np.asarray(rows)
    blocks = np.arange((H + 3) // 4)
    w = philox_words(blocks[None, :], rows[:, None], offset, seed).reshape(len(rows), -1)[:, :H]
    return torch.from_numpy(w >= np.uint64(math.floor(p * 2.0 ** 32)))


def drop(v: torch.Tensor, p: float, seed: int, offset: int, rows=None) -> torch.Tensor:
    if p == 0:
        return v
    k = kept(v.shape[0] if rows is None else rows, v.shape[1], p, seed, offset)
    return torch.where(k, v / (1 - p), torch.zeros((), dtype=v.dtype))


def layer_norm(x, gamma, beta, eps, residual=None, p=0.0, seed=0, offset=0):
    """(y, s, mean, rstd) in float64 and the fp32 errors (y, s, mean, rstd) allowed before the stores."""
    x = x.cpu().to(F8)
    H = x.shape[1]
    d = drop(x, p, seed, offset)
    s = d + residual.cpu().to(F8) if residual is not None else d
    size = d.abs() + (residual.cpu().to(F8).abs() if residual is not None else 0)
    mean = s.mean(1, keepdim=True)
    var = (s - mean).square().mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    g = gamma.cpu().to(F8) if gamma is not None else torch.ones(H, dtype=F8)
    b = beta.cpu().to(F8) if beta is not None else torch.zeros(H, dtype=F8)
    y = (s - mean) * rstd * g + b
    summed = residual is not None or p > 0
    es = 3 * U * size if summed else torch.zeros_like(s)
    em = (H + 2) * U * s.abs().mean(1, keepdim=True) + es.mean(1, keepdim=True)
    ev = (H + 4) * U * var + 2 * ((s - mean).abs() * (es + em)).mean(1, keepdim=True) + ((es + em) ** 2).mean(1, keepdim=True)
    er = rstd * (ev / (var + eps) / 2 * 1.01 + 4 * U)
    ey = g.abs() * (rstd * (es + em + U * (s - mean).abs()) + (s - mean).abs() * er) * 1.01 + 4 * U * ((y - b).abs() + b.abs())
    return (y, s, mean[:, 0], rstd[:, 0]), (ey, es, em[:, 0], er[:, 0])


def layer_norm_backward(dy, s, mean, rstd, gamma, ds_in=None, p=0.0, seed=0, offset=0):
    """(ds, dx, dgamma, dbeta) in float64 and the fp32 errors allowed before the stores."""
    dy, s = dy.cpu().to(F8), s.cpu().to(F8)
    B, H = dy.shape
    mean, rstd = mean.cpu().to(F8)[:, None], rstd.cpu().to(F8)[:, None]
    gam = gamma.cpu().to(F8) if gamma is not None else torch.ones(H, dtype=F8)
    xh, g = (s - mean) * rstd, dy * gam
    exh = 3 * U * xh.abs()
    c1, c2 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    e1 = (H + 3) * U * g.abs().mean(1, keepdim=True)
    e2 = (H + 6) * U * (g * xh).abs().mean(1, keepdim=True)
    inner = g - c1 - xh * c2
    ei = U * g.abs() + e1 + xh.abs() * e2 + exh * c2.abs() + 4 * U * (g.abs() + c1.abs() + (xh * c2).abs())
    ds = rstd * inner
    eds = rstd * ei + 2 * U * ds.abs()
    if ds_in is not None:
        ds = ds + ds_in.cpu().to(F8)
        eds = eds + U * ds.abs()
    scale = 1 / (1 - p)
    dx = drop(ds, p, seed, offset)
    edx = eds * scale + 2 * U * dx.abs()
    dgamma, dbeta = (dy * xh).sum(0), dy.sum(0)
    egamma = (B + 6) * U * (dy * xh).abs().sum(0)
    ebeta = (B + 2) * U * dy.abs().sum(0)
    return (ds, dx, dgamma, dbeta), (eds, edx, egamma, ebeta)


def act(z: torch.Tensor, name: str) -> torch.Tensor:
    if name == "gelu":
        # z Phi(z) by erfc: torch's ndtr keeps only an absolute 5e-17 in the left tail (at -8.25 it gives
        # 5.6e-17 for 7.9e-17)
        return z * 0.5 * torch.erfc(-z * math.sqrt(0.5))
    if name == "gelu_tanh":
        # (1 + tanh u) / 2 = 1 / (1 + exp(-2u)); the tanh form cancels for negative z (1 + tanh u keeps an
        # absolute 1e-16 where the value itself falls below 1e-13), this one does not
        return z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
    return z.clone()


def act_grad(z: torch.Tensor, name: str) -> torch.Tensor:
    v = z.clone().requires_grad_(True)
    return torch.autograd.grad(act(v, name).sum(), v)[0]


def grouped(x, w, offsets, x_index=None, x_div=1, transpose_w=False, act_name="identity", z_in=None):
    """(y, z) in grouped order in float64 and the fp32 errors allowed before the stores; entries in no group: NaN."""
    x, w = x.cpu().to(F8), w.cpu().to(F8)
    offs = offsets.cpu().tolist()
    E = x_index.numel() if x_index is not None else x.shape[0] * x_div
    src = (x_index.cpu().long() if x_index is not None else torch.arange(E)).div(x_div, rounding_mode="floor")
    xs = torch.where(((src >= 0) & (src < x.shape[0]))[:, None], x[src.clamp(0, max(0, x.shape[0] - 1))], 0.0)
    K, N = x.shape[1], w.shape[2] if transpose_w else w.shape[1]
    z, ez = torch.full((E, N), math.nan, dtype=F8), torch.zeros((E, N), dtype=F8)
    for g, (a, b) in enumerate(zip(offs, offs[1:])):
        m = w[g] if transpose_w else w[g].T
        z[a:b] = xs[a:b] @ m
        ez[a:b] = (2 * K + 4) * U * (xs[a:b].abs() @ m.abs())  # 2 U a term: the matrix cores may truncate
    if z_in is not None:
        zi = z_in.cpu().to(F8)
        d = act_grad(zi, act_name)
        # the derivative's own error: z enters exp and erfc squared, a few roundings each, sizes up to 1 + |z|
        ed = (16 + 2 * zi ** 2) * U * (1 + zi.abs()) * torch.exp(-zi ** 2 / 2).clamp_min(1e-30) + 8 * U * d.abs()
        y = z * d
        return (y, z), (ez * d.abs() + z.abs() * ed + ez * ed + 2 * U * y.abs(), ez)
    y = act(z, act_name)
    slope = 1.0 if act_name == "identity" else 1.13  # the largest derivative of either GELU
    own = 0 if act_name == "identity" else (16 + 2 * z ** 2) * U * y.abs()
    return (y, z), (slope * ez + own, ez)


def weight_grad(dy, x, offsets, dy_index=None, x_index=None, x_div=1):
    """dw in float64 and the fp32 error allowed."""
    dy, x = dy.cpu().to(F8), x.cpu().to(F8)
    offs = offsets.cpu().tolist()
    E = dy_index.numel() if dy_index is not None else dy.shape[0]
    di = dy_index.cpu().long() if dy_index is not None else torch.arange(E)
    si = (x_index.cpu().long() if x_index is not None else torch.arange(E)).div(x_div, rounding_mode="floor")

    def rows(v, i):
        return torch.where(((i >= 0) & (i < v.shape[0]))[:, None], v[i.clamp(0, max(0, v.shape[0] - 1))], 0.0)

    dw = torch.zeros((len(offs) - 1, dy.shape[1], x.shape[1]), dtype=F8)
    ew = torch.zeros_like(dw)
    for g, (a, b) in enumerate(zip(offs, offs[1:])):
        if b > a:
            u, v = rows(dy, di[a:b]), rows(x, si[a:b])
            dw[g] = u.T @ v
            ew[g] = (2 * (b - a) + 4) * U * (u.abs().T @ v.abs())
    return dw, ew


def check(got: torch.Tensor, ref: torch.Tensor, err, what: str):
    """|got - ref| within the fp32 error and half a step of got's type (2 % slack for second-order terms)."""
    g = got.detach().cpu().to(F8)
    assert g.shape == ref.shape, (what, g.shape, ref.shape)
    tiny = torch.finfo(got.dtype).smallest_normal * half_step(got.dtype)
    lim = 1.02 * (err + half_step(got.dtype) * (ref.abs() + err)) + tiny
    bad = ~((g - ref).abs() <= lim)
    if bad.any():
        i = tuple(int(v) for v in bad.nonzero()[0])
        worst = ((g - ref).abs() / lim).nan_to_num(math.inf).max()
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {i}: {g[i]} for {ref[i]}, "
                             f"worst {float(worst):.3g} of the bound")

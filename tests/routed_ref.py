"""A routed expert block's operators in 64 bits, and how far fp32 arithmetic may be off (the tests' references).

Bounds count roundings of U = 2^-24 as tests/ops_ref.py does: n U times the sum of the terms' sizes for a sum of n
terms in any order.  An exponential of an fp32 argument a that was itself rounded once (a difference of two
logits) has a relative error of at most |a| U + 4 U.
"""
from __future__ import annotations

import math

import torch

from tests.ops_ref import F8, U, act, act_grad

NONE = -math.inf
F32_MAX = torch.finfo(torch.float32).max
TINY = 2.0 ** -126  # what fp32 exponentials may lose where they leave its normal numbers


def clean(logits):
    """Logits in 64 bits: -inf where there is no expert (NaN too), the largest fp32 value for +inf."""
    l = logits.cpu().to(F8)
    return torch.where(l > NONE, l.clamp(max=F32_MAX), NONE)


def scores(l, score):
    there = l > NONE
    if score == "sigmoid":
        return torch.where(there, 1 / (1 + torch.exp(-l)), 0.0)
    most = l.amax(1, keepdim=True)
    e = torch.where(there, torch.exp(l - torch.where(most > NONE, most, 0.0)), 0.0)
    total = e.sum(1, keepdim=True)
    return torch.where(total > 0, e / torch.where(total > 0, total, 1.0), 0.0)


def route(logits, top_k, bias=None, score="softmax", n_groups=1, top_groups=None, group_score="top2",
          renormalise=False, scale=1.0):
    """(ids, weights, the weights' fp32 error): token by token, expert by expert, from the definition."""
    l = clean(logits)
    s = scores(l, score)
    T, E = l.shape
    b = bias.cpu().to(F8) if bias is not None else None
    ids = torch.full((T, top_k), -1, dtype=torch.int32)
    weights, err = torch.zeros((T, top_k), dtype=F8), torch.zeros((T, top_k), dtype=F8)
    size, keep = E // n_groups, n_groups if top_groups is None else top_groups
    c = s + b if b is not None else l.clone()
    c = torch.where((l > NONE) & (c > NONE), c, NONE)  # a NaN compares false
    C, S, L = c.tolist(), s.tolist(), l.tolist()
    for t in range(T):
        allowed = range(E)
        if n_groups > 1:
            value = []
            for g in range(n_groups):
                live = [e for e in range(g * size, (g + 1) * size) if C[t][e] > NONE]
                by = [S[t][e] if bias is None and group_score == "top2" else C[t][e] for e in live]
                best = sorted(by, reverse=True)[:2 if group_score == "top2" else 1]
                value.append(sum(best) if best else NONE)
            order = sorted((g for g in range(n_groups) if value[g] > NONE), key=lambda g: (-value[g], g))[:keep]
            allowed = [e for g in sorted(order) for e in range(g * size, (g + 1) * size)]
        chosen = sorted((e for e in allowed if C[t][e] > NONE), key=lambda e: (-C[t][e], e))[:top_k]
        if not chosen:
            continue
        ids[t, :len(chosen)] = torch.tensor(chosen, dtype=torch.int32)
        top = max(L[t][e] for e in chosen)
        if renormalise:
            # shares of the chosen: each score over the largest one's, so that none of them underflows alone
            if score == "softmax":
                part = [math.exp(L[t][e] - top) for e in chosen]
            else:
                part = [math.exp(_log_sigmoid(L[t][e]) - _log_sigmoid(top)) for e in chosen]
            total = sum(part)
            w = [p / total for p in part]
            away = [top - L[t][e] for e in chosen]
            n = len(chosen)
        else:
            w = [S[t][e] for e in chosen]
            away = [max(L[t]) - L[t][e] if score == "softmax" else 0.0 for e in chosen]
            n = E if score == "softmax" else 1
        for j, (v, a) in enumerate(zip(w, away)):
            weights[t, j] = scale * v
            err[t, j] = abs(scale) * ((n + 16 + min(a, 200.0)) * U * v + TINY)
    return ids, weights, err


def _log_sigmoid(v):
    return v - math.log1p(math.exp(v)) if v < 0 else -math.log1p(math.exp(-v))


def route_backward(dweights, logits, ids, score="softmax", renormalise=False, scale=1.0):
    """dlogits in 64 bits by the formulas, and the fp32 error allowed before the store."""
    l, E = clean(logits), logits.shape[1]
    ids = ids.cpu().long()
    live = (ids >= 0) & (ids < E)
    at = ids.clamp(0, E - 1)
    live &= l.gather(1, at) > NONE
    dw = torch.where(live, scale * dweights.cpu().to(F8), 0.0)
    s = scores(l, score)
    chosen = torch.where(live, l.gather(1, at), NONE)
    K = ids.shape[1]

    def spread(v):
        return torch.zeros((l.shape[0], E), dtype=F8).scatter_add_(1, at, torch.where(live, v, 0.0))

    def away(most, of):  # of: logits that may be -inf
        return torch.where(of > NONE, (most - of).clamp(0, 200), 0.0)

    if renormalise:
        most = chosen.amax(1, keepdim=True)
        most = torch.where(most > NONE, most, 0.0)
        if score == "softmax":
            p = torch.where(live, torch.exp(chosen - most), 0.0)
        else:
            soft = torch.nn.functional.softplus
            p = torch.where(live, torch.exp((chosen - soft(chosen)) - (most - soft(most))).nan_to_num(0.0), 0.0)
        p = p / p.sum(1, keepdim=True).clamp(min=1e-300)
        D = (dw * p).sum(1, keepdim=True)
        g = p * (dw - D)
        rest = torch.where(l > NONE, 1 / (1 + torch.exp(l)), 0.0) if score == "sigmoid" else torch.ones_like(l)
        size = p * (dw.abs() + (dw.abs() * p).sum(1, keepdim=True))
        err = spread(size * (3 * K + 40 + 2 * away(most, chosen).amax(1, keepdim=True)) * U + TINY) * rest
        return spread(g) * rest, err
    d, da = spread(dw), spread(dw.abs())
    if score == "sigmoid":
        out = d * s * torch.where(l > NONE, 1 / (1 + torch.exp(l)), 0.0)
        return out, (K + 16) * U * da * s * torch.where(l > NONE, 1 / (1 + torch.exp(l)), 0.0) + TINY * da
    most = l.amax(1, keepdim=True)
    most = torch.where(most > NONE, most, 0.0)
    D, Da = (d * s).sum(1, keepdim=True), (da * s).sum(1, keepdim=True)
    n = E + K + 40 + 2 * away(most, l)
    # the sum D carries the exponentials' errors of the entries' own logits
    far = (da * s * away(most, l)).sum(1, keepdim=True)
    err = s * ((da + Da) * n + far) * U + TINY * (da + Da)
    return s * (d - D), err


def combine(rows, top_k, weights=None, ids=None, residual=None):
    """y in 64 bits and the fp32 error allowed."""
    R, H = rows.shape
    v = rows.cpu().to(F8).view(-1, top_k, H)
    w = weights.cpu().to(F8) if weights is not None else torch.ones(v.shape[:2], dtype=F8)
    if ids is not None:
        off = ids.cpu() < 0
        v, w = v.masked_fill(off[:, :, None], 0.0), w.masked_fill(off, 0.0)
    terms = w[:, :, None] * v
    y, size = terms.sum(1), terms.abs().sum(1)
    if residual is not None:
        r = residual.cpu().to(F8)
        y, size = y + r, size + r.abs()
    return y, (top_k + 2) * U * size


def combine_backward(dy, top_k, rows=None, weights=None, ids=None):
    """(drows, dweights) in 64 bits and the fp32 errors allowed."""
    dy = dy.cpu().to(F8)
    B, H = dy.shape
    w = weights.cpu().to(F8) if weights is not None else torch.ones((B, top_k), dtype=F8)
    off = ids.cpu() < 0 if ids is not None else torch.zeros((B, top_k), dtype=torch.bool)
    drows = torch.where(off[:, :, None], 0.0, w[:, :, None] * dy[:, None, :])
    out, err = [drows.view(B * top_k, H)], [U * drows.abs().view(B * top_k, H)]
    if rows is None:
        return out + [None], err + [None]
    terms = torch.where(off[:, :, None], 0.0, rows.cpu().to(F8).view(B, top_k, H) * dy[:, None, :])
    return out + [terms.sum(2)], err + [(H + 4) * U * terms.abs().sum(2)]


def rms_norm(x, gamma, eps, residual=None):
    """(y, s, rstd) in 64 bits and the fp32 errors allowed."""
    x = x.cpu().to(F8)
    H = x.shape[1]
    s = x + residual.cpu().to(F8) if residual is not None else x
    es = U * s.abs() if residual is not None else torch.zeros_like(s)
    var = s.square().mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    g = gamma.cpu().to(F8) if gamma is not None else torch.ones(H, dtype=F8)
    y = s * rstd * g
    ev = (H + 4) * U * var + 2 * (s.abs() * es).mean(1, keepdim=True) + (es ** 2).mean(1, keepdim=True)
    er = rstd * (ev / (var + eps) / 2 * 1.01 + 4 * U)
    ey = g.abs() * (rstd * es + s.abs() * er) * 1.01 + 4 * U * y.abs()
    return (y, s, rstd[:, 0]), (ey, es, er[:, 0])


def rms_norm_backward(dy, s, rstd, gamma, ds_in=None):
    """(ds, dgamma) in 64 bits and the fp32 errors allowed."""
    dy, s, rstd = dy.cpu().to(F8), s.cpu().to(F8), rstd.cpu().to(F8)[:, None]
    B, H = dy.shape
    gam = gamma.cpu().to(F8) if gamma is not None else torch.ones(H, dtype=F8)
    xh, g = s * rstd, dy * gam
    c2 = (g * xh).mean(1, keepdim=True)
    e2 = (H + 6) * U * (g * xh).abs().mean(1, keepdim=True)
    ds = rstd * (g - xh * c2)
    eds = rstd * (xh.abs() * e2 + 6 * U * (g.abs() + (xh * c2).abs())) + 2 * U * ds.abs()
    if ds_in is not None:
        ds = ds + ds_in.cpu().to(F8)
        eds = eds + U * ds.abs()
    return (ds, (dy * xh).sum(0)), (eds, (B + 6) * U * (dy * xh).abs().sum(0))


# the 127 finite magnitudes of e4m3, by code: seven bits of exponent (bias 7, 0: subnormal) and mantissa
E4M3 = [(m / 8 * 2.0 ** -6) if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127]


def scale_codes(x):
    """The scale bytes of x's rows: for every 32 columns the smallest exponent (at least -127) for which no
    finite value passes 448 times the power of two, + 127.  By integer comparisons of exact values."""
    x = x.cpu().to(F8)
    B, H = x.shape
    out = torch.zeros((B, -(-H // 32)), dtype=torch.uint8)
    for r in range(B):
        for b in range(out.shape[1]):
            v = x[r, 32 * b:32 * b + 32]
            v = v[torch.isfinite(v)].abs()
            most = float(v.max()) if v.numel() else 0.0
            p = max(-127, math.frexp(most)[1] - 10) if most else -127
            while most > 448 * 2.0 ** p:
                p += 1
            out[r, b] = p + 127
    return out


def pack(x):
    """(values, scale bytes): values in 64 bits as e4m3 holds them, NaN for what is not finite."""
    codes = scale_codes(x)
    x = x.cpu().to(F8)
    H = x.shape[1]
    scale = torch.exp2(codes.to(F8) - 127).repeat_interleave(32, 1)[:, :H]
    v = x.abs() / scale
    table = torch.tensor(E4M3, dtype=F8)
    i = torch.searchsorted(table, v.clamp(max=448), right=True) - 1  # the value at or below
    up = (i + 1).clamp(max=126)
    low, high = table[i], table[up]
    nearer = torch.where(v - low < high - v, i, torch.where(v - low > high - v, up, torch.where(i % 2 == 0, i, up)))
    out = torch.minimum(table[nearer], (1.875 * 2.0 ** 127) / scale)  # finite values stay finite in fp32: 2^128 is not
    return torch.where(torch.isfinite(x), torch.copysign(out, x), math.nan), codes


def unpack(values, codes):
    """The numbers that packed rows stand for, in 64 bits."""
    H = values.shape[1]
    c = codes.cpu().to(F8)
    scale = torch.where(c == 255, math.nan, torch.exp2(c - 127)).repeat_interleave(32, 1)[:, :H]
    return values.cpu().to(torch.float32).to(F8) * scale


def activations(z, name, dy=None):
    """(act(z), dy act'(z)) in 64 bits and the fp32 errors allowed, as tests/ops_ref.py derives them for the products."""
    y = act(z, name)
    ey = 0 * z if name == "identity" else (16 + 2 * z ** 2) * U * y.abs()
    if dy is None:
        return y, ey, None, None
    if name == "identity":
        return y, ey, dy, 0 * dy
    d = act_grad(z, name)
    ed = (16 + 2 * z ** 2) * U * (1 + z.abs()) * torch.exp(-z ** 2 / 2).clamp_min(1e-30) + 8 * U * d.abs()
    return y, ey, dy * d, dy.abs() * ed + 2 * U * (dy * d).abs()

"""The operators around the layer on the GPU against their definitions in 64 bits (tests/ops_ref.py)."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from tests import ops_ref as ref
from tests.conftest import flush_print

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SEED, OFFSET = 0x0123456789ABCDEF, (7 << 32) + 5


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _randn(gen, *shape, dtype="f32", mean=0.0):
    return (torch.randn(shape, generator=gen, device=DEV) + mean).to(DT[dtype])


# ------------------------------------------------------------------------------------------ layer norm

NORM_SHAPES = [(1, 1), (3, 2), (2, 3), (5, 4), (1, 8), (7, 31), (9, 100), (4, 255), (33, 256), (6, 257), (5, 300),
               (10, 512), (3, 519), (130, 768), (2, 769), (65, 1000), (17, 1024), (3, 1032), (5, 1536), (4, 2001),
               (9, 2048), (3, 2056), (7, 4096), (2, 4099), (3, 8192), (2, 8200), (3, 16384), (2, 16390), (2, 40001)]
NORM_TYPES = [("bf16", "bf16", "bf16"), ("f32", "f32", "f32"), ("bf16", "f32", "bf16"), ("f32", "bf16", "f32")]


@pytest.mark.parametrize("B,H", NORM_SHAPES)
@pytest.mark.parametrize("kind", ["plain", "residual", "residual_dropout", "dropout"])
def test_layer_norm(fff_lib, B, H, kind):
    for n, (xt, st, yt) in enumerate(NORM_TYPES):
        flush_print(f"[gpu] layer_norm {B}x{H} {kind} {xt}/{st}/{yt}")
        gen = _gen(100 * H + B + n)
        x = _randn(gen, B, H, dtype=xt, mean=0.5)
        residual = _randn(gen, B, H, dtype=st, mean=-2.0) if "residual" in kind else None
        gamma = _randn(gen, H, mean=1.0) if n != 1 else None
        beta = _randn(gen, H) if n != 2 else None
        p = 0.25 if "dropout" in kind else 0.0
        kw = {"p": p, "seed": SEED, "offset": OFFSET} if p else {}
        y, s, mean, rstd = fff_lib.layer_norm(x, gamma, beta, eps=1e-5, residual=residual, y_dtype=DT[yt],
                                              s_dtype=DT[st] if residual is None and p else None, **kw)
        want, err = ref.layer_norm(x, gamma, beta, 1e-5, residual, p, SEED, OFFSET)
        for got, w, e, what in zip((y, s, mean, rstd), want, err, ("y", "s", "mean", "rstd")):
            ref.check(got, w, e, f"{what} {B}x{H} {kind} {xt}/{st}/{yt}")
        if kind == "plain":
            assert s is x
        else:
            assert s.dtype == DT[st]


@pytest.mark.parametrize("B,H", NORM_SHAPES)
@pytest.mark.parametrize("kind", ["plain", "stream", "stream_dropout", "dropout"])
def test_layer_norm_backward(fff_lib, B, H, kind):
    for n, (xt, st, yt) in enumerate(NORM_TYPES):
        flush_print(f"[gpu] layer_norm_backward {B}x{H} {kind} {xt}/{st}/{yt}")
        gen = _gen(77 * H + B + n)
        s, dy = _randn(gen, B, H, dtype=st, mean=0.5), _randn(gen, B, H, dtype=yt)
        gamma = _randn(gen, H, mean=1.0) if n != 1 else None
        ds_in = _randn(gen, B, H, dtype=st) if "stream" in kind else None
        p = 0.4 if "dropout" in kind else 0.0
        wide = s.double()
        mean = wide.mean(1).float()
        rstd = (1 / torch.sqrt(wide.var(1, correction=0) + 1e-5)).float()
        kw = {"p": p, "seed": SEED, "offset": OFFSET} if p else {}
        got = fff_lib.layer_norm_backward(dy, s, mean, rstd, gamma, ds_in=ds_in, dx_dtype=DT[xt], **kw)
        want, err = ref.layer_norm_backward(dy, s, mean, rstd, gamma, ds_in, p, SEED, OFFSET)
        for v, w, e, what in zip(got, want, err, ("ds", "dx", "dgamma", "dbeta")):
            ref.check(v, w, e, f"{what} {B}x{H} {kind} {xt}/{st}/{yt}")
        again = fff_lib.layer_norm_backward(dy, s, mean, rstd, gamma, ds_in=ds_in, dx_dtype=DT[xt], **kw)
        assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("B,H,t", [(4097, 768, "bf16"), (2500, 100, "f32"), (700, 1024, "f32"), (1030, 4096, "bf16")])
def test_layer_norm_backward_many_rows(fff_lib, B, H, t):
    gen = _gen(B)
    s, dy, gamma = _randn(gen, B, H, dtype=t, mean=1.0), _randn(gen, B, H, dtype=t), _randn(gen, H, mean=1.0)
    wide = s.double()
    mean, rstd = wide.mean(1).float(), (1 / torch.sqrt(wide.var(1, correction=0) + 1e-5)).float()
    flush_print(f"[gpu] layer_norm_backward {B}x{H} {t}")
    got = fff_lib.layer_norm_backward(dy, s, mean, rstd, gamma)
    want, err = ref.layer_norm_backward(dy, s, mean, rstd, gamma)
    for v, w, e, what in zip(got, want, err, ("ds", "dx", "dgamma", "dbeta")):
        ref.check(v, w, e, what)
    # each gradient alone gives the same bits, and accumulate adds to what is there
    for name, full in zip(("ds", "dgamma", "dbeta"), (got[0], got[2], got[3])):
        one = fff_lib.layer_norm_backward(dy, s, mean, rstd, gamma, want=(name,))
        assert [v is not None for v in one].count(True) == 1
        assert torch.equal(next(v for v in one if v is not None), full), name
    dgamma, dbeta = torch.full((H,), 2.0, device=DEV), torch.full((H,), -3.0, device=DEV)
    fff_lib.layer_norm_backward(dy, s, mean, rstd, gamma, dgamma=dgamma, dbeta=dbeta, accumulate=True, want=())
    assert torch.equal(dgamma, got[2] + 2.0) and torch.equal(dbeta, got[3] - 3.0)


def test_layer_norm_no_rows(fff_lib):
    e = torch.empty((0, 64), device=DEV)
    y, s, mean, rstd = fff_lib.layer_norm(e)
    assert y.shape == (0, 64) and mean.numel() == 0
    g, b = torch.full((64,), 5.0, device=DEV), torch.full((64,), 5.0, device=DEV)
    fff_lib.layer_norm_backward(e, e, mean, rstd, dgamma=g, dbeta=b, accumulate=True)
    assert (g == 5).all() and (b == 5).all()
    fff_lib.layer_norm_backward(e, e, mean, rstd, dgamma=g, dbeta=b)
    assert (g == 0).all() and (b == 0).all()
    assert fff_lib.dropout(e, 0.5, 1).shape == (0, 64)


@pytest.mark.parametrize("H", [96, 768, 4096, 20000])
def test_layer_norm_rows_apart(fff_lib, H):
    """A row of infinities or NaN spoils no other; constant rows give beta (eps > 0); large means do not cancel."""
    gen = _gen(H)
    x = _randn(gen, 6, H)
    x[1, 3], x[2, 5], x[3] = math.inf, math.nan, 4.0
    x[4] += 1000.0
    beta = _randn(gen, H)
    flush_print(f"[gpu] layer_norm rows apart, {H}")
    y = fff_lib.layer_norm(x, None, beta, eps=1e-5)[0]
    assert torch.isnan(y[1]).all() and torch.isnan(y[2]).all()
    assert torch.equal(y[3], beta)
    ok = [0, 3, 4, 5]
    want, err = ref.layer_norm(x[ok], None, beta, 1e-5)
    ref.check(y[ok], want[0], err[0], "finite rows")


def test_layer_norm_stream_in_place(fff_lib):
    """s may be the residual's buffer, ds the buffer of ds_in: the same bits as apart."""
    for H in (100, 768, 1024, 20000):
        gen = _gen(H)
        x, r = _randn(gen, 37, H, dtype="bf16"), _randn(gen, 37, H)
        flush_print(f"[gpu] layer_norm in place, {H}")
        apart = fff_lib.layer_norm(x, residual=r, p=0.1, seed=3)
        stream = r.clone()
        inside = fff_lib.layer_norm(x, residual=stream, s=stream, p=0.1, seed=3)
        assert inside[1] is stream and all(torch.equal(a, b) for a, b in zip(apart, inside))
        dy, up = _randn(gen, 37, H, dtype="bf16"), _randn(gen, 37, H)
        a = fff_lib.layer_norm_backward(dy, apart[1], apart[2], apart[3], ds_in=up, p=0.1, seed=3)
        buf = up.clone()
        b = fff_lib.layer_norm_backward(dy, apart[1], apart[2], apart[3], ds_in=buf, ds=buf, p=0.1, seed=3)
        assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_layer_norm_matches_the_forward_prologue(fff_lib):
    """The normalised rows feed fff.forward as its own LayerNorm prologue would."""
    gen = _gen(5)
    x = _randn(gen, 200, 768, mean=0.3)
    gamma, beta = _randn(gen, 768, mean=1.0), _randn(gen, 768)
    w = [_randn(gen, 1, 127, 768) * 768 ** -0.5 for _ in range(2)]
    u = fff_lib.layer_norm(x, gamma, beta, eps=1e-5, stats=False)[0]
    nodes = [torch.empty((200, 1, 7), dtype=torch.int32, device=DEV) for _ in range(2)]
    a = fff_lib.forward(u, *w, 6, nodes_out=nodes[0])
    b = fff_lib.forward(x, *w, 6, norm="layernorm", norm_eps=1e-5, norm_gamma=gamma, norm_beta=beta, nodes_out=nodes[1])
    same = (nodes[0] == nodes[1]).all(2)[:, 0]
    assert same.float().mean() > 0.98
    torch.testing.assert_close(a[same], b[same], rtol=1e-4, atol=1e-4)


# --------------------------------------------------------------------------------------------- dropout


@pytest.mark.parametrize("B,H", [(1, 1), (1, 3), (3, 4), (2, 5), (5, 8), (333, 101), (7, 768), (64, 1024), (3, 4100),
                                 (2, 12289), (1000, 16)])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.999])
def test_dropout(fff_lib, B, H, p):
    for xt, rt, yt in (("f32", None, "f32"), ("bf16", "bf16", "bf16"), ("bf16", "f32", "f32"), ("f32", "bf16", "bf16")):
        gen = _gen(B + H)
        x = _randn(gen, B, H, dtype=xt)
        r = _randn(gen, B, H, dtype=rt) if rt else None
        flush_print(f"[gpu] dropout {B}x{H} p={p} {xt}/{rt}/{yt}")
        y = fff_lib.dropout(x, p, SEED, OFFSET, residual=r, y_dtype=DT[yt])
        d = ref.drop(x.cpu().double(), p, SEED, OFFSET)
        want = d + r.cpu().double() if rt else d
        ref.check(y, want, 3 * ref.U * (d.abs() + (r.cpu().double().abs() if rt else 0)), f"dropout {B}x{H} {p}")
        if not rt:
            assert torch.equal(y.cpu() != 0, ref.kept(B, H, p, SEED, OFFSET) if p else torch.ones(B, H, dtype=torch.bool))


def test_dropout_share_and_streams_of_numbers(fff_lib):
    ones = torch.ones((4096, 768), device=DEV)
    a, b, c = (fff_lib.dropout(ones, 0.1, 11, o) for o in (0, 0, 1))
    assert torch.equal(a, b)
    kept = (a != 0).double().mean().item()
    # 3.1 M draws: the share's standard deviation is sqrt(.09 / 3.1e6) = 1.7e-4; six of them
    assert abs(kept - 0.9) < 1.1e-3
    both = ((a != 0) & (c != 0)).double().mean().item()
    assert abs(both - 0.81) < 1.4e-3


def test_dropout_hides_what_it_drops(fff_lib):
    """A dropped infinity or NaN leaves 0; in place on x or on the residual gives the same bits."""
    x = torch.full((50, 100), math.nan, device=DEV)
    y = fff_lib.dropout(x, 0.3, 9)
    assert torch.equal(torch.isnan(y).cpu(), ref.kept(50, 100, 0.3, 9, 0))
    assert (y[~torch.isnan(y)] == 0).all()
    gen = _gen(1)
    x, r = _randn(gen, 50, 100, dtype="bf16"), _randn(gen, 50, 100, dtype="bf16")
    want = fff_lib.dropout(x, 0.3, 9, residual=r)
    for buf in (x.clone(), r.clone()):
        is_x = torch.equal(buf, x)
        got = fff_lib.dropout(buf if is_x else x, 0.3, 9, residual=r if is_x else buf, y=buf)
        assert torch.equal(got, want)


def test_keywords_and_streams_of_the_binding(fff_lib):
    x = _randn(_gen(3), 8, 64)
    want = fff_lib.dropout(x, 0.5, 7)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = fff_lib.dropout(x=x, p=0.5, seed=7, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    with pytest.raises(ValueError):
        fff_lib.dropout(x.t(), 0.5, 7)
    with pytest.raises(ValueError):
        fff_lib.dropout(x.half(), 0.5, 7)
    with pytest.raises(ValueError):
        fff_lib.dropout(x, 1.0, 7)
    with pytest.raises(ValueError):
        fff_lib.layer_norm(x, torch.ones(63, device=DEV))
    with pytest.raises(fff_lib.FffError):
        fff_lib.layer_norm(x, eps=-1.0)


def test_rows_past_four_billion_elements(fff_lib):
    """65552 rows of 65536: offsets and addresses past 32 bits (checked on sampled rows)."""
    B, H = 65552, 65536
    rows = [0, 1, 32767, 65535, 65536, B - 1]
    x = torch.empty((B, H), dtype=torch.bfloat16, device=DEV).normal_(generator=_gen(8))
    flush_print("[gpu] dropout past 2^32 elements")
    y = fff_lib.dropout(x, 0.1, SEED, OFFSET)
    d = ref.drop(x[rows].cpu().double(), 0.1, SEED, OFFSET, rows=rows)
    ref.check(y[rows], d, 2 * ref.U * d.abs(), "dropout")
    flush_print("[gpu] layer_norm past 2^32 elements")
    y = fff_lib.layer_norm(x, eps=1e-5, y=y)[0]
    want, err = ref.layer_norm(x[rows], None, None, 1e-5)
    ref.check(y[rows], want[0], err[0], "y")
    mean, rstd = torch.zeros(B, device=DEV), torch.ones(B, device=DEV)
    flush_print("[gpu] layer_norm_backward past 2^32 elements")
    ds = fff_lib.layer_norm_backward(y, x, mean, rstd, want=("ds",))[0]
    want, err = ref.layer_norm_backward(y[rows], x[rows], mean[rows], rstd[rows], None)
    ref.check(ds[rows], want[0], err[0], "ds")


# ------------------------------------------------------------------------------------------ group rows


def _group_ref(ids, n_ids, first, n_trees):
    ids = ids.cpu().numpy().astype(np.int64).ravel()
    local = ids - first
    ok = (local >= 0) & (local < n_ids)
    key = np.where(ok, np.arange(ids.size) % n_trees * n_ids + local, n_ids * n_trees)
    order = np.argsort(key, kind="stable")[:int(ok.sum())]
    offsets = np.concatenate(([0], np.cumsum(np.bincount(key, minlength=n_ids * n_trees + 1)[:-1])))
    return order.astype(np.int32), offsets.astype(np.int32), int((~ok).sum())


@pytest.mark.parametrize("E,n_ids,n_trees,first", [
    (1, 1, 1, 0), (1, 2048, 1, 2047), (2, 3, 2, -5), (63, 7, 1, 0), (64, 64, 1, 63), (65, 2, 1, 1), (1000, 1, 1, 0),
    (1023, 33, 3, 100), (1025, 256, 1, 255), (4096, 512, 8, 511), (5000, 32768, 1, 32767), (40000, 32768, 1, 32767), (16384, 64, 1, 63), (16384, 1024, 1, 0), (16383, 1025, 1, 0),
    (30000, 16384, 1, 0), (16384, 2048, 1, 2047), (2000000, 1000, 3, 0),
    (16385, 5, 1, 0), (40001, 4096, 8, 4095), (70000, 100, 1, -50), (300000, 2, 1, 0), (524288, 512, 8, 511)])
def test_group_rows(fff_lib, E, n_ids, n_trees, first):
    gen = _gen(E)
    for kind in ("uniform", "one", "strays"):
        if kind == "uniform":
            ids = torch.randint(0, n_ids, (E,), generator=gen, device=DEV) + first
        elif kind == "one":
            ids = torch.full((E,), first + n_ids - 1, device=DEV)
        else:
            ids = torch.randint(-2, n_ids + 2, (E,), generator=gen, device=DEV) + first
            ids[::7] = -2 ** 31
            ids[3::11] = 2 ** 31 - 1
        ids = ids.to(torch.int32)
        order, offsets, strays = _group_ref(ids, n_ids, first, n_trees)
        flush_print(f"[gpu] group_rows {E} entries, {n_trees} x {n_ids}, {kind}")
        got = torch.full((E,), -9, dtype=torch.int32, device=DEV)
        bad = torch.zeros(1, dtype=torch.int32, device=DEV)
        o, f = fff_lib.group_rows(ids, n_ids, first=first, n_trees=n_trees, order=got, bad_ids=bad)
        assert np.array_equal(f.cpu().numpy(), offsets)
        assert np.array_equal(o[:order.size].cpu().numpy(), order)
        assert (o[order.size:] == -9).all(), "entries behind the last group are left as they were"
        assert int(bad) == strays


def test_group_rows_nothing(fff_lib):
    for n_ids in (5, 2048, 16384):
        order, offsets = fff_lib.group_rows(torch.empty((0, 2), dtype=torch.int32, device=DEV), n_ids, n_trees=2)
        assert order.numel() == 0 and torch.equal(offsets.cpu(), torch.zeros(2 * n_ids + 1, dtype=torch.int32))


# ------------------------------------------------------------------------------------- grouped products


def _groups(gen, E, G, kind):
    """Offsets [G + 1] of E entries: ragged, all in one group, or with rows behind the last group."""
    if kind == "one":
        sizes = torch.zeros(G, dtype=torch.int64)
        sizes[G // 2] = E
    else:
        n = E - E // 5 if kind == "tail" else E
        pick = torch.randint(0, G, (n,), generator=gen, device=DEV).cpu()
        if G > 2:
            pick[pick == 1] = 0  # group 1 stays empty
        sizes = torch.bincount(pick, minlength=G)
    return torch.cat((torch.zeros(1, dtype=torch.int64), sizes.cumsum(0))).to(torch.int32).to(DEV)


PRODUCTS = [  # entries, groups, k, n
    (1, 1, 1, 1), (1, 5, 16, 16), (2, 3, 7, 5), (3, 2, 64, 33), (8, 64, 512, 96), (9, 3, 100, 130), (17, 1, 65, 64),
    (40, 70, 64, 72), (64, 4, 40, 1), (100, 3, 1, 65), (130, 2, 96, 257), (200, 7, 129, 100), (257, 1, 256, 256),
    (300, 33, 72, 264), (515, 2, 320, 520), (700, 5, 264, 136), (1000, 3, 203, 300), (33, 2, 2050, 40), (5, 4, 4096, 24),
    (1300, 1, 64, 512), (16, 1, 768, 1000), (1600, 600, 48, 40)]


@pytest.mark.parametrize("E,G,K,N", PRODUCTS)
@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("transpose", [False, True])
def test_grouped_matmul(fff_lib, E, G, K, N, t, transpose):
    gen = _gen(E * 7 + G + K + N)
    w = _randn(gen, G, *((K, N) if transpose else (N, K)), dtype=t) * K ** -0.5
    for kind in ("ragged", "one", "tail"):
        offsets = _groups(gen, E, G, kind)
        used = int(offsets[-1])
        x = _randn(gen, E, K, dtype=t)
        flush_print(f"[gpu] grouped_matmul {E}x{G} k={K} n={N} {t} transpose={transpose} {kind}")
        for yt in ("f32", "bf16"):
            y = torch.full((E, N), -7.0, dtype=DT[yt], device=DEV)
            got = fff_lib.grouped_matmul(x, w, offsets, y=y, transpose_w=transpose)
            (want, _), (err, _) = ref.grouped(x, w, offsets, transpose_w=transpose)
            assert got is y
            ref.check(y[:used], want[:used], err[:used], f"y {yt}")
            assert (y[used:] == -7).all(), "rows behind the last group are left as they were"


@pytest.mark.parametrize("E,G,K,N", PRODUCTS)
@pytest.mark.parametrize("t,yt,zt", [("bf16", "bf16", "bf16"), ("bf16", "f32", "f32"), ("f32", "f32", "f32"), ("f32", "bf16", "f32")])
def test_grouped_matmul_epilogues(fff_lib, E, G, K, N, t, yt, zt):
    """Gathered rows (two entries a row), scattered results, the activation with z kept, and its gradient."""
    gen = _gen(E + G + 3 * K + N)
    offsets = _groups(gen, E, G, "ragged")
    rows = (E + 1) // 2
    x = _randn(gen, rows, K, dtype=t)
    w = _randn(gen, G, N, K, dtype=t) * K ** -0.5
    order = torch.randperm(E, generator=gen, device=DEV).to(torch.int32)
    for act in ("identity", "gelu", "gelu_tanh"):
        flush_print(f"[gpu] grouped_matmul {E}x{G} k={K} n={N} {t}/{yt}/{zt} {act}")
        z_out = torch.full((E, N), -7.0, dtype=DT[zt], device=DEV)
        y = torch.full((E + 3, N), -7.0, dtype=DT[yt], device=DEV)
        got = fff_lib.grouped_matmul(x, w, offsets, x_index=order, x_div=2, y=y, y_index=order, act=act, z_out=z_out)
        assert got[0] is y and got[1] is z_out
        (want, wz), (err, ez) = ref.grouped(x, w, offsets, order, 2, act_name=act)
        ref.check(z_out, wz, ez, "z")
        ref.check(y[order.long()], want, err, "y")
        assert (y[E:] == -7).all()
        # the gradient's form: W read transposed, times the derivative at a given z
        dy = _randn(gen, E, N, dtype=t)
        z_in = _randn(gen, E, K, dtype=zt) * 2
        dz = fff_lib.grouped_matmul(dy, w, offsets, x_index=order, transpose_w=True, act=act, z_in=z_in, y_dtype=DT[yt])
        (want, _), (err, _) = ref.grouped(dy, w, offsets, order, transpose_w=True, act_name=act, z_in=z_in)
        ref.check(dz, want, err, "dz")


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("E,G,K,N", [(5, 3, 64, 48), (300, 4, 72, 100), (600, 2, 256, 256), (40, 2, 33, 20)])
def test_grouped_bad_values_stay_in_bounds(fff_lib, E, G, K, N, t):
    """Indices outside x read zeros, outside y store nothing; offsets are clamped, falling ones are empty."""
    gen = _gen(E)
    x, w = _randn(gen, E, K, dtype=t), _randn(gen, G, N, K, dtype=t)
    offsets = _groups(gen, E, G, "ragged")
    xi, yi = (torch.randperm(E, generator=gen, device=DEV).to(torch.int32) for _ in range(2))
    xi[0], xi[1 % E], yi[2 % E] = -1, E, 2 ** 31 - 1
    flush_print(f"[gpu] grouped_matmul bad indices {E}x{G} {t}")
    y = torch.full((E, N), -7.0, device=DEV)
    fff_lib.grouped_matmul(x, w, offsets, x_index=xi, y=y, y_index=yi)
    (want, _), (err, _) = ref.grouped(x, w, offsets, xi)
    full, lim = torch.full((E, N), -7.0, dtype=torch.float64), torch.zeros((E, N), dtype=torch.float64)
    for i, d in enumerate(yi.tolist()):
        if 0 <= d < E:
            full[d], lim[d] = want[i], err[i]
    ref.check(y, full, lim, "y")
    dy = _randn(gen, E, N, dtype=t)
    dw = fff_lib.grouped_weight_grad(dy, x, offsets, dy_index=yi, x_index=xi)
    ref.check(dw, *ref.weight_grad(dy, x, offsets, yi, xi), "dw")
    bad = offsets.clone()
    bad[0], bad[-1] = -5, E + 1000
    flush_print(f"[gpu] grouped_matmul clamped offsets {E}x{G} {t}")
    good = offsets.clone()
    good[-1] = E
    a = fff_lib.grouped_matmul(x, w, bad)
    assert torch.equal(a, fff_lib.grouped_matmul(x, w, good))
    assert torch.equal(fff_lib.grouped_weight_grad(dy, x, bad), fff_lib.grouped_weight_grad(dy, x, good))
    bad = torch.tensor([E] + [0] * G, dtype=torch.int32, device=DEV)  # falls: every group empty
    y = torch.full((E, N), -7.0, device=DEV)
    fff_lib.grouped_matmul(x, w, bad, y=y)
    assert (y == -7).all()
    assert (fff_lib.grouped_weight_grad(dy, x, bad) == 0).all()


@pytest.mark.parametrize("E,G,K,N", PRODUCTS)
@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_grouped_weight_grad(fff_lib, E, G, K, N, t):
    gen = _gen(E + 5 * G + K + N)
    for kind in ("ragged", "one", "tail"):
        offsets = _groups(gen, E, G, kind)
        rows = (E + 2) // 3
        dy, x = _randn(gen, E, N, dtype=t), _randn(gen, rows, K, dtype=t)
        order = torch.randperm(E, generator=gen, device=DEV).to(torch.int32)
        flush_print(f"[gpu] grouped_weight_grad {E}x{G} k={K} n={N} {t} {kind}")
        dw = fff_lib.grouped_weight_grad(dy, x, offsets, dy_index=order, x_index=order, x_div=3)
        want, err = ref.weight_grad(dy, x, offsets, order, order, 3)
        ref.check(dw, want, err, "dw")
        assert torch.equal(dw, fff_lib.grouped_weight_grad(dy, x, offsets, dy_index=order, x_index=order, x_div=3))
        base = _randn(gen, G, N, K)
        got = fff_lib.grouped_weight_grad(dy, x, offsets, dy_index=order, x_index=order, x_div=3, dw=base.clone(),
                                          accumulate=True)
        ref.check(got, want + base.cpu().double(), err + ref.U * (want.abs() + base.cpu().double().abs()), "accumulated")


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("E,G,K,N", [(20, 4, 64, 40), (20, 4, 61, 33), (900, 3, 128, 256), (900, 3, 61, 33)])
def test_grouped_entries_without_a_row_beside_infinities(fff_lib, E, G, K, N, t):
    """Entries without a row give 0 and add nothing, whatever the operand beside them holds."""
    gen = _gen(E + K)
    flush_print(f"[gpu] grouped products, entries without a row {E} x {G}: {K} -> {N} {t}")
    x, dy = _randn(gen, E, K, dtype=t).to(DEV), _randn(gen, E, N, dtype=t).to(DEV)
    w = torch.full((G, N, K), math.inf, dtype=x.dtype, device=DEV)
    cuts = torch.linspace(0, E, G + 1).to(torch.int32).to(DEV)
    none = torch.arange(E, dtype=torch.int32) % 3 == 1
    index = torch.where(none, -1, torch.arange(E, dtype=torch.int32)).to(DEV)
    for transpose in (False, True):
        y = fff_lib.grouped_matmul(x, w.transpose(1, 2).contiguous() if transpose else w, cuts, x_index=index,
                                   transpose_w=transpose)
        assert (y[none.to(DEV)] == 0).all() and not torch.isfinite(y[~none.to(DEV)]).any()
    full = x.clone()
    full[none.to(DEV)] = math.nan
    zero_dy, zero_x = dy.clone(), x.clone()
    zero_dy[none.to(DEV)] = 0
    zero_x[none.to(DEV)] = 0
    want = fff_lib.grouped_weight_grad(zero_dy, zero_x, cuts)
    assert torch.isfinite(want).all()
    assert torch.equal(fff_lib.grouped_weight_grad(dy, full, cuts, dy_index=index), want)
    full = dy.clone()
    full[none.to(DEV)] = math.inf
    assert torch.equal(fff_lib.grouped_weight_grad(full, x, cuts, x_index=index), want)


def test_grouped_offsets_that_name_entries_again(fff_lib):
    """Offsets that rise and fall over many groups: more tiles than the launch holds, every access in bounds."""
    E, G, K, N = 300, 5000, 32, 40
    x, w = torch.ones((E, K), device=DEV), torch.ones((G, N, K), device=DEV)
    offsets = torch.tensor([0, E] * (G // 2) + [0], dtype=torch.int32, device=DEV)
    flush_print("[gpu] grouped_matmul offsets that name entries again")
    for t in (torch.float32, torch.bfloat16):
        for transpose in (False, True):
            wt = w.transpose(1, 2).contiguous() if transpose else w
            y = fff_lib.grouped_matmul(x.to(t), wt.to(t), offsets, transpose_w=transpose)
            assert (y == K).all()  # every group gives the same rows
    dw = fff_lib.grouped_weight_grad(torch.ones((E, N), device=DEV), x, offsets)
    assert (dw[0::2] == E).all() and (dw[1::2] == 0).all()


def test_grouped_weight_grad_of_more_groups_than_a_launch_holds(fff_lib):
    flush_print("[gpu] grouped_weight_grad of 2^24 groups")
    x = torch.ones((3, 1), device=DEV)
    dw = torch.full((1 << 24, 1, 1), 7.0, device=DEV)
    with pytest.raises(fff_lib.FffError):
        fff_lib.grouped_weight_grad(x, x, torch.zeros((1 << 24) + 1, dtype=torch.int32, device=DEV), dw=dw)
    assert (dw == 7).all()
    offsets = torch.full(((1 << 23) + 1,), 3, dtype=torch.int32, device=DEV)
    offsets[0] = 0
    dw = fff_lib.grouped_weight_grad(x, x, offsets)
    assert dw[0, 0, 0] == 3 and (dw[1:] == 0).all()


@pytest.mark.parametrize("K,N", [(4096, 4104), (4100, 4099)])
@pytest.mark.parametrize("E", [40, 700])
def test_grouped_past_four_billion_elements(fff_lib, E, K, N):
    """The last of 300 groups, rows behind 2^20 of x, y and dy: every matrix holds more than 2^32 elements."""
    G, B, gen, bf = 300, (1 << 20) + E, _gen(E + K), torch.bfloat16
    offsets = torch.zeros(G + 1, dtype=torch.int32, device=DEV)
    offsets[G] = E
    index = (B - 1 - torch.randperm(E, generator=gen, device=DEV)).to(torch.int32)
    x, dy = torch.empty((B, K), dtype=bf, device=DEV), torch.empty((B, N), dtype=bf, device=DEV)
    near_x, near_w = _randn(gen, E, K, dtype="bf16"), _randn(gen, 1, N, K, dtype="bf16") * K ** -0.5
    near_dy = _randn(gen, E, N, dtype="bf16")
    x[B - E:], dy[B - E:] = near_x, near_dy
    ends, at = torch.tensor([0, E], dtype=torch.int32, device=DEV), (index - (B - E)).to(torch.int32)
    (want, _), (err, _) = ref.grouped(near_x, near_w, ends, at)
    for transpose in (False, True):
        w = torch.empty((G, K, N) if transpose else (G, N, K), dtype=bf, device=DEV)
        w[G - 1] = near_w[0].T if transpose else near_w[0]
        y = torch.empty((B, N), dtype=bf, device=DEV)
        flush_print(f"[gpu] grouped_matmul past 2^32 elements, {E} entries {K} -> {N}, transposed {transpose}")
        fff_lib.grouped_matmul(x, w, offsets, x_index=index, y=y, y_index=index, transpose_w=transpose)
        ref.check(y[index.long()], want, err, "y")
        del w, y
    flush_print(f"[gpu] grouped_weight_grad past 2^32 elements, {E} entries {K} -> {N}")
    dw = fff_lib.grouped_weight_grad(dy, x, offsets, dy_index=index, x_index=index)
    want, err = ref.weight_grad(near_dy, near_x, ends, at, at)
    ref.check(dw[G - 1:], want, err, "dw")
    assert (dw[0] == 0).all() and (dw[G - 2] == 0).all()


def test_grouped_no_entries(fff_lib):
    w = torch.ones((3, 4, 8), device=DEV)
    e8, e4, off = torch.empty((0, 8), device=DEV), torch.empty((0, 4), device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV)
    assert fff_lib.grouped_matmul(e8, w, off).shape == (0, 4)
    assert (fff_lib.grouped_weight_grad(e4, e8, off) == 0).all()
    dw = torch.full((3, 4, 8), 2.0, device=DEV)
    assert (fff_lib.grouped_weight_grad(e4, e8, off, dw=dw, accumulate=True) == 2).all()


@pytest.mark.parametrize("E,G,K,N,t", [(5000, 3, 512, 768, "bf16"), (3000, 1, 1024, 1024, "bf16"), (4100, 8, 256, 512, "f32"),
                                       (6000, 1, 136, 72, "bf16"), (9000, 2, 64, 65, "f32")])
def test_grouped_large(fff_lib, E, G, K, N, t):
    """Sizes of the large tiles and of long sums split over several workgroups."""
    gen = _gen(E)
    offsets = _groups(gen, E, G, "ragged")
    order = torch.randperm(E, generator=gen, device=DEV).to(torch.int32)
    x, w, dy = _randn(gen, E, K, dtype=t), _randn(gen, G, N, K, dtype=t) * K ** -0.5, _randn(gen, E, N, dtype=t)
    flush_print(f"[gpu] grouped large {E}x{G} {K} {N} {t}")
    y, z = fff_lib.grouped_matmul(x, w, offsets, x_index=order, act="gelu", keep_z=True)
    (want, wz), (err, ez) = ref.grouped(x, w, offsets, order, act_name="gelu")
    ref.check(y, want, err, "y")
    ref.check(z, wz, ez, "z")
    dx = fff_lib.grouped_matmul(dy, w, offsets, transpose_w=True)
    (want, _), (err, _) = ref.grouped(dy, w, offsets, transpose_w=True)
    ref.check(dx, want, err, "dx")
    dw = fff_lib.grouped_weight_grad(dy, x, offsets, x_index=order)
    ref.check(dw, *ref.weight_grad(dy, x, offsets, None, order), "dw")


# ------------------------------------------------------------------------ streams, graphs, whole steps


def _step(fff, t, drop):
    """One training step of a block of leaf experts behind a routing tree, every tensor of it."""
    B, H, F, depth, p = t["x"].shape[0], t["x"].shape[1], t["w1"].shape[1], t["depth"], 0.1
    leaves = 1 << depth
    u, _, mean, rstd = fff.layer_norm(t["x"], t["gamma"], t["beta"], eps=1e-5, y_dtype=t["w1"].dtype)
    nodes = torch.empty((B, 1, depth + 1), dtype=torch.int32, device=u.device)
    fff.forward(u, t["tree"], t["tree"], depth, nodes_out=nodes, act="identity")
    order, offsets = fff.group_rows(nodes[..., depth].contiguous(), leaves, first=leaves - 1)
    h, z = fff.grouped_matmul(u, t["w1"], offsets, x_index=order, act="gelu", keep_z=True)
    f = torch.empty((B, H), dtype=u.dtype, device=u.device)
    fff.grouped_matmul(h, t["w2"], offsets, y=f, y_index=order)
    y, s, mean2, rstd2 = fff.layer_norm(f, t["gamma"], t["beta"], eps=1e-5, residual=t["x"], p=p, **drop)
    ds, df, dgamma2, dbeta2 = fff.layer_norm_backward(t["dy"], s, mean2, rstd2, t["gamma"], ds_in=t["ds"],
                                                      dx_dtype=u.dtype, p=p, **drop)
    dz = fff.grouped_matmul(df, t["w2"], offsets, x_index=order, transpose_w=True, act="gelu", z_in=z)
    dw2 = fff.grouped_weight_grad(df, h, offsets, dy_index=order)
    dw1 = fff.grouped_weight_grad(dz, u, offsets, x_index=order)
    du = torch.empty((B, H), dtype=u.dtype, device=u.device)
    fff.grouped_matmul(dz, t["w1"], offsets, y=du, y_index=order, transpose_w=True)
    dx, _, dgamma1, dbeta1 = fff.layer_norm_backward(du, t["x"], mean, rstd, t["gamma"], ds_in=ds)
    return {"y": y, "s": s, "dx": dx, "dw1": dw1, "dw2": dw2, "dgamma1": dgamma1, "dbeta1": dbeta1, "dgamma2": dgamma2,
            "dbeta2": dbeta2, "leaves": nodes[:, 0, depth]}


def _step_inputs(seed, B=300, H=128, F=192, depth=3, t="f32"):
    gen = _gen(seed)
    G = 1 << depth
    return {"x": _randn(gen, B, H), "gamma": _randn(gen, H, mean=1.0), "beta": _randn(gen, H), "depth": depth,
            "tree": _randn(gen, 1, 2 * G - 1, H, dtype=t) * H ** -0.5, "w1": _randn(gen, G, F, H, dtype=t) * H ** -0.5,
            "w2": _randn(gen, G, H, F, dtype=t) * F ** -0.5, "dy": _randn(gen, B, H, dtype=t), "ds": _randn(gen, B, H)}


def _step_ref(t, leaves, seed, offset, p=0.1):
    """The same step in float64 by autograd, along the device's routing."""
    leaf = leaves.cpu().long() - ((1 << t["depth"]) - 1)
    v = {k: t[k].cpu().double().requires_grad_(True) for k in ("x", "w1", "w2")}
    g1, b1, g2, b2 = (t[k].cpu().double().requires_grad_(True) for k in ("gamma", "beta", "gamma", "beta"))

    def norm(s, g, b):
        var, mean = torch.var_mean(s, 1, correction=0, keepdim=True)
        return (s - mean) / torch.sqrt(var + 1e-5) * g + b

    u = norm(v["x"], g1, b1)
    h = ref.act(torch.matmul(v["w1"][leaf], u[:, :, None])[..., 0], "gelu")
    f = torch.matmul(v["w2"][leaf], h[:, :, None])[..., 0]
    s = v["x"] + ref.drop(f, p, seed, offset)
    y = norm(s, g2, b2)
    loss = (y * t["dy"].cpu().double()).sum() + (s * t["ds"].cpu().double()).sum()
    grads = torch.autograd.grad(loss, [v["x"], v["w1"], v["w2"], g1, b1, g2, b2])
    names = ("dx", "dw1", "dw2", "dgamma1", "dbeta1", "dgamma2", "dbeta2")
    return {"y": y.detach(), "s": s.detach(), **dict(zip(names, grads))}, loss


def test_expert_block_step(fff_lib):
    """Forward and backward of a whole block, each operator fed by the others, against float64 autograd.

    fp32 through a chain of five products and norms of width <= 192: relative norms within
    100 x 192 U = 1.2e-3 of each tensor at worst; a wrong row, mask or term is off by far more."""
    t = _step_inputs(3)
    flush_print("[gpu] expert block step")
    got = _step(fff_lib, t, {"seed": SEED, "offset": OFFSET})
    want, _ = _step_ref(t, got["leaves"], SEED, OFFSET)
    for k, w in want.items():
        rel = (got[k].cpu().double() - w).norm() / w.norm()
        flush_print(f"[gpu] {k}: {float(rel):.2e}")
        assert rel < 100 * 192 * ref.U, k


def test_expert_block_step_gradient_against_differences(fff_lib):
    """The device's gradients against central differences of the float64 loss along the device's routing and mask."""
    t = _step_inputs(4, B=40, H=64, F=48, depth=2)
    got = _step(fff_lib, t, {"seed": SEED, "offset": OFFSET})
    gen = torch.Generator().manual_seed(1)
    for name, grad in (("x", "dx"), ("w1", "dw1"), ("w2", "dw2")):
        d = torch.randn(t[name].shape, generator=gen, dtype=torch.float64)
        losses = []
        for sign in (1, -1):
            moved = dict(t)
            moved[name] = t[name].cpu().double() + sign * 1e-5 * d
            losses.append(float(_step_ref(moved, got["leaves"], SEED, OFFSET)[1].detach()))
        slope = (losses[0] - losses[1]) / 2e-5
        dot = float((got[grad].cpu().double() * d).sum())
        # fp32 gradients: each term within 2e-4 of its size; the differences' own error is ~1e-8
        assert abs(slope - dot) <= 2e-4 * float((got[grad].cpu().double() * d).abs().sum()) + 1e-5, name


def test_other_stream(fff_lib):
    """Work goes to the stream it is given; results and scratch belong to that stream."""
    t = _step_inputs(5, t="bf16")
    want = _step(fff_lib, t, {"seed": 1})
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = _step(fff_lib, t, {"seed": 1})
    side.synchronize()
    assert all(torch.equal(got[k], want[k]) for k in want)
    x, r = _randn(_gen(1), 64, 768), _randn(_gen(2), 64, 768)
    torch.cuda.synchronize()
    a = fff_lib.layer_norm(x, residual=r, p=0.1, seed=2, stream=side)
    d = fff_lib.dropout(x, 0.1, 2, residual=r, stream=side)
    b = fff_lib.layer_norm_backward(x, a[1], a[2], a[3], ds_in=r, stream=side)
    side.synchronize()
    assert torch.equal(a[1], d)
    assert all(torch.equal(u, v) for u, v in zip(b, fff_lib.layer_norm_backward(x, a[1], a[2], a[3], ds_in=r)))


def test_captured_step_draws_new_masks(fff_lib):
    """A whole step in a graph: each replay equals the eager step at its rng offset, with eager steps between."""
    for t in (_step_inputs(6), _step_inputs(7, B=700, H=256, F=512, depth=2, t="bf16")):
        count = torch.zeros(1, dtype=torch.int64, device=DEV)
        drop = {"seed": 5, "offset": 10, "rng_offset": count}
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            _step(fff_lib, t, drop)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            inside = _step(fff_lib, t, drop)
        seen = []
        for n in (0, 1, 1 << 33, 2):
            count.fill_(n)
            graph.replay()
            torch.cuda.synchronize()
            eager = _step(fff_lib, t, {"seed": 5, "offset": 10 + n})
            torch.cuda.synchronize()
            for k in eager:
                assert torch.equal(inside[k], eager[k]), (k, n)
            seen.append(inside["s"].clone())
        assert not torch.equal(seen[0], seen[1])


def test_two_graphs_share_no_scratch(fff_lib):
    """Two captured backward passes replayed at once on two streams give their own results."""
    ins = [[_randn(_gen(20 + i), 900, 512, dtype="bf16") for _ in range(2)] for i in range(2)]
    offsets = torch.tensor([0, 300, 300, 900], dtype=torch.int32, device=DEV)
    ids = [torch.randint(0, 64, (5000,), generator=_gen(i), device=DEV).to(torch.int32) for i in range(2)]
    stats = torch.zeros(900, device=DEV), torch.ones(900, device=DEV)

    def work(i):
        return [*fff_lib.layer_norm_backward(*ins[i], *stats), fff_lib.grouped_weight_grad(*ins[i], offsets),
                *fff_lib.group_rows(ids[i], 64)]

    want = [work(i) for i in range(2)]
    torch.cuda.synchronize()
    graphs, outs, streams = [], [], [torch.cuda.Stream() for _ in range(2)]
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(work(i))
        graphs.append(g)
    for _ in range(3):
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert all(torch.equal(a, b) for a, b in zip(outs[i], want[i]))


def test_captured_long_forms_and_sums(fff_lib):
    """The forms of several launches in a graph, adding to gradients, against eager calls between the replays."""
    gen = _gen(31)
    E, G = 50000, 300
    ids = torch.randint(-1, G, (E,), generator=gen, device=DEV).to(torch.int32)
    x, dy = _randn(gen, 3000, 256, dtype="bf16"), _randn(gen, 3000, 136, dtype="bf16")
    offsets = torch.tensor([0, 2900, 2950], dtype=torch.int32, device=DEV)
    long = [_randn(gen, 3, 20000) for _ in range(3)]
    gamma, stats = _randn(gen, 20000), (torch.zeros(3, device=DEV), torch.ones(3, device=DEV))
    assert fff_lib.grouped_weight_grad_workspace_bytes(3000, 2, 256, 136) > 0

    def sums():
        return {"bad": torch.zeros(1, dtype=torch.int32, device=DEV), "dw": torch.ones((2, 136, 256), device=DEV),
                "dgamma": torch.ones(20000, device=DEV), "dbeta": torch.ones(20000, device=DEV)}

    def work(t):
        out = [*fff_lib.group_rows(ids, G, bad_ids=t["bad"])]
        out[0] = out[0][:E - int((ids < 0).sum())] if not torch.cuda.is_current_stream_capturing() else out[0]
        fff_lib.grouped_weight_grad(dy, x, offsets, dw=t["dw"], accumulate=True)
        out += fff_lib.layer_norm_backward(long[0], long[1], *stats, gamma, ds_in=long[2], dgamma=t["dgamma"],
                                           dbeta=t["dbeta"], accumulate=True, p=0.5, seed=3)[:2]
        return out

    flush_print("[gpu] long forms and sums in a graph")
    mine, eager = sums(), sums()
    work(sums())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        inside = work(mine)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        want = work(eager)
        torch.cuda.synchronize()
        assert torch.equal(inside[0][:want[0].numel()], want[0])
        assert all(torch.equal(a, b) for a, b in zip(inside[1:], want[1:]))
        assert all(torch.equal(mine[k], eager[k]) for k in mine)
    assert int(mine["bad"]) == 3 * int((ids < 0).sum())


@pytest.mark.parametrize("H", [768, 20000])
def test_in_place_equals_out_of_place(fff_lib, H):
    """The stream and its gradient written over their inputs, rows in registers and long ones, with dropout."""
    gen = _gen(H)
    x, r, dy, up = (_randn(gen, 5, H) for _ in range(4))
    drop = {"p": 0.3, "seed": 11, "offset": 4}
    flush_print(f"[gpu] layer_norm in place, {H}")
    want = fff_lib.layer_norm(x, residual=r, **drop)
    got = fff_lib.layer_norm(x, residual=r, s=r, **drop)
    assert got[1] is r and all(torch.equal(a, b) for a, b in zip(got, want))
    want = fff_lib.layer_norm_backward(dy, *want[1:], ds_in=up, **drop)
    got = fff_lib.layer_norm_backward(dy, *got[1:], ds_in=up, ds=up, **drop)
    assert got[0] is up and all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("E,G,K,N,t", [(9, 4, 72, 40, "bf16"), (700, 5, 61, 47, "f32"), (700, 5, 64, 128, "bf16"),
                                       (6000, 6, 256, 512, "bf16"), (6000, 6, 72, 264, "f32")])
def test_grouped_entries_and_groups_apart(fff_lib, E, G, K, N, t):
    """NaN in one entry's row or one group's matrix stays with that entry and that group."""
    gen = _gen(E + N)
    flush_print(f"[gpu] grouped products with NaN, {E} x {G}: {K} -> {N} {t}")
    offsets = torch.linspace(0, E, G + 1).to(torch.int32).to(DEV)
    x, dy, w = _randn(gen, E, K, dtype=t), _randn(gen, E, N, dtype=t), _randn(gen, G, N, K, dtype=t)
    for transpose in (False, True):
        wt = w.transpose(1, 2).contiguous() if transpose else w.clone()
        clean = fff_lib.grouped_matmul(x, wt, offsets, act="gelu", transpose_w=transpose)
        wt[1] = math.nan
        xn = x.clone()
        xn[0], xn[E - 1] = math.nan, math.inf
        got = fff_lib.grouped_matmul(xn, wt, offsets, act="gelu", transpose_w=transpose)
        hit = torch.zeros(E, dtype=torch.bool, device=DEV)
        hit[0] = hit[E - 1] = True
        hit[int(offsets[1]):int(offsets[2])] = True
        assert torch.equal(got[~hit], clean[~hit]) and not torch.isfinite(got[0]).any()
        assert torch.isnan(got[int(offsets[1]):int(offsets[2])]).all()
    clean = fff_lib.grouped_weight_grad(dy, x, offsets)
    xn = x.clone()
    xn[int(offsets[1])] = math.nan
    got = fff_lib.grouped_weight_grad(dy, xn, offsets)
    rest = [g for g in range(G) if g != 1]
    assert torch.equal(got[rest], clean[rest]) and torch.isnan(got[1]).all()


def test_training_step_of_the_tree_block(fff_lib):
    """x + drop(FFF(LN(x))) and its gradients: the layer's own forward and backward between the new operators."""
    B, H, depth = 64, 64, 3
    gen = _gen(9)
    x, gamma, beta = _randn(gen, B, H), _randn(gen, H, mean=1.0), _randn(gen, H)
    w = [_randn(gen, 1, 15, H) * H ** -0.5 for _ in range(2)]
    dy = _randn(gen, B, H)
    u, _, mean, rstd = fff_lib.layer_norm(x, gamma, beta, eps=1e-5)
    nodes = torch.empty((B, 1, depth + 1), dtype=torch.int32, device=DEV)
    logits = torch.empty((B, 1, depth + 1), device=DEV)
    f = fff_lib.forward(u, *w, depth, nodes_out=nodes, logits_out=logits)
    y = fff_lib.dropout(f, 0.1, SEED, OFFSET, residual=x)
    df = fff_lib.dropout(dy, 0.1, SEED, OFFSET)
    du, dwi, dwo = fff_lib.backward(u, *w, depth, 1, df, nodes[..., depth].contiguous(), logits)
    dx, _, dgamma, dbeta = fff_lib.layer_norm_backward(du, x, mean, rstd, gamma, ds_in=dy)
    v = [a.cpu().double().requires_grad_(True) for a in (x, gamma, beta, *w)]
    var, m = torch.var_mean(v[0], 1, correction=0, keepdim=True)
    un = (v[0] - m) / torch.sqrt(var + 1e-5) * v[1] + v[2]
    path = nodes.cpu().long()[:, 0]
    z = torch.matmul(v[3][0][path], un[:, :, None])
    fn = (ref.act(z, "gelu") * v[4][0][path]).sum(1)
    yn = v[0] + ref.drop(fn, 0.1, SEED, OFFSET)
    grads = torch.autograd.grad((yn * dy.cpu().double()).sum(), v)
    for name, a, b in zip(("y", "dx", "dgamma", "dbeta", "dw_in", "dw_out"), (y, dx, dgamma, dbeta, dwi, dwo),
                          (yn.detach(), *grads)):
        rel = (a.cpu().double() - b).norm() / b.norm()
        # chains of three sums of at most 64 terms, a factor of a hundred for conditioning
        assert rel < 100 * 64 * ref.U, (name, float(rel))


@pytest.mark.parametrize("t,E", [("f32", 1 << 18), ("bf16", 1 << 18), ("f32", 16)])
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh"])
def test_activations_stored_in_fp32_are_as_exact_as_fp32_allows(fff_lib, t, E, act):
    """Root mean square errors over z ~ N(0, 1) against the least that the formulas' own fp32 roundings leave.

    z Phi(z) from a correctly rounded Phi, and the derivative as the sum of correctly rounded Phi and z phi, are
    the ideals (evaluated here).  A value may have twice that variance: as much again from what Phi is
    computed of (the polynomial, or the exponential and the reciprocal).  The derivative of the tanh form has one more
    such operand, u' beside u, and may have 2.5 times it.  The product before the activation is exact (k = 1, W = 1)."""
    n = 1 << 14 if E == 16 else 1  # few entries take the kernel for them, here over many columns
    z = _randn(_gen(12), E, 1, dtype=t)
    ones = torch.ones((1, n, 1), dtype=DT[t], device=DEV)
    if E == 16:
        z, ones = torch.ones((E, 1), device=DEV), _randn(_gen(12), 1, n, 1)
    offsets = torch.tensor([0, E], dtype=torch.int32, device=DEV)
    flush_print(f"[gpu] {act} in fp32, {E} x {n} {t}")
    y, zs = fff_lib.grouped_matmul(z, ones, offsets, act=act, keep_z=True, y_dtype=torch.float32)
    assert torch.equal(zs, (z.float() @ ones[0].float().T))
    unit = fff_lib.grouped_matmul(torch.ones_like(z), torch.ones_like(ones), offsets, act=act, z_in=zs, y_dtype=torch.float32)
    v = zs.cpu().double()
    share = ref.act(v, act) / v  # Phi, or the logistic of 2 u
    slope = ref.act_grad(v, act)

    def rms(got, want):
        return float(((got.double() - want) / ref.U).square().mean().sqrt())

    least = rms((v * share.float().double()).float(), v * share)
    assert rms(y.cpu(), v * share) <= math.sqrt(2) * least
    least = rms((share.float().double() + (slope - share).float().double()).float(), slope)
    assert rms(unit.cpu(), slope) <= math.sqrt(2 if act == "gelu" else 2.5) * least


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("E", [16, 4096])
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh"])
def test_activations_far_out(fff_lib, t, E, act):
    """Where either GELU is z or 0 to every bit, up to the largest numbers: its derivative is 1 or 0, nothing overflows."""
    far = torch.tensor([20.0, 1e4, 1e10, 6e18, 8e18, 1e20, 1.5e38, 3e38], device=DEV).repeat(E // 8)[:, None]
    one, offsets = torch.ones((1, 1, 1), dtype=DT[t], device=DEV), torch.tensor([0, E], dtype=torch.int32, device=DEV)
    for yt in ("f32", "bf16"):
        for sign in (1, -1):
            z = (sign * far).to(DT[t])
            flush_print(f"[gpu] {act} far out, {E} {t}/{yt} {sign}")
            y = fff_lib.grouped_matmul(z, one, offsets, act=act, y_dtype=DT[yt])
            assert torch.equal(y, z.to(DT[yt]) if sign > 0 else torch.zeros_like(y))
            d = fff_lib.grouped_matmul(torch.ones_like(z), one, offsets, act=act, z_in=z, y_dtype=DT[yt])
            assert torch.equal(d, torch.full_like(d, float(sign > 0)))
    # a positive infinity is itself, a NaN stays one
    z = torch.tensor([math.inf, math.nan], device=DEV).repeat(E // 2)[:, None].to(DT[t])
    for yt in ("f32", "bf16"):
        y = fff_lib.grouped_matmul(z, one, offsets, act=act, y_dtype=DT[yt])
        assert (y[0::2] == math.inf).all() and torch.isnan(y[1::2]).all()
        assert torch.isnan(fff_lib.grouped_matmul(torch.ones_like(z), one, offsets, act=act, z_in=z)[1::2]).all()


def test_two_graphs_of_long_forms_share_no_scratch(fff_lib):
    """As above at sizes where all three operators need scratch: two graphs replayed at once, eager calls beside them."""
    E, G = 50000, 300
    ids = [torch.randint(0, G, (E,), generator=_gen(40 + i), device=DEV).to(torch.int32) for i in range(2)]
    rows = [(_randn(_gen(50 + i), 3000, 136, dtype="bf16"), _randn(_gen(60 + i), 3000, 256, dtype="bf16")) for i in range(2)]
    norm = [[_randn(_gen(70 + i), 900, 512, dtype="bf16") for _ in range(2)] for i in range(2)]
    offsets = torch.tensor([0, 2900, 3000], dtype=torch.int32, device=DEV)
    stats = torch.zeros(900, device=DEV), torch.ones(900, device=DEV)
    assert fff_lib.group_rows_workspace_bytes(E, G) > 0
    assert fff_lib.grouped_weight_grad_workspace_bytes(3000, 2, 256, 136) > 0
    assert fff_lib.layer_norm_backward_workspace_bytes(900, 512) > 0
    plan = fff_lib.describe_grouped_weight_grad(*rows[0], offsets)
    assert "splits=1 " not in plan, plan

    def work(i):
        return [*fff_lib.group_rows(ids[i], G), fff_lib.grouped_weight_grad(*rows[i], offsets),
                *fff_lib.layer_norm_backward(*norm[i], *stats)]

    flush_print("[gpu] two graphs of long forms")
    want = [work(i) for i in range(2)]
    torch.cuda.synchronize()
    graphs, outs, streams = [], [], [torch.cuda.Stream() for _ in range(2)]
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(work(i))
        graphs.append(g)
    for _ in range(4):
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        eager = work(0)
        torch.cuda.synchronize()
        for i in range(2):
            assert all(torch.equal(a, b) for a, b in zip(outs[i], want[i]))
        assert all(torch.equal(a, b) for a, b in zip(eager, want[0]))


@pytest.mark.parametrize("H", [(1 << 26) + 5, 1 << 24])
def test_layer_norm_backward_sums_of_very_long_rows(fff_lib, H):
    """dgamma and dbeta of more columns than one launch has threads for, and of as many as its workgroups take at once."""
    gen = _gen(H)
    dy, s = (torch.empty((1, H), dtype=torch.bfloat16, device=DEV).normal_(generator=gen) for _ in range(2))
    mean, rstd = torch.full((1,), 0.25, device=DEV), torch.full((1,), 2.0, device=DEV)  # (s - mean) rstd: one rounding
    dgamma, dbeta = torch.full((H,), 1.0, device=DEV), torch.full((H,), 1.0, device=DEV)
    flush_print(f"[gpu] layer_norm_backward sums of {H} columns")
    out = fff_lib.layer_norm_backward(dy, s, mean, rstd, want=("dgamma", "dbeta"))
    want = dy.double() * (s.double() - 0.25) * 2
    assert torch.equal(out[3], dy[0].float())
    assert ((out[2].double() - want[0]).abs() <= 2.02 * ref.U * want[0].abs()).all()  # of the difference, of the product
    fff_lib.layer_norm_backward(dy, s, mean, rstd, dgamma=dgamma, dbeta=dbeta, accumulate=True, want=())
    assert torch.equal(dgamma, out[2] + 1) and torch.equal(dbeta, out[3] + 1)


@pytest.mark.parametrize("p", [0.0, 0.1])
@pytest.mark.parametrize("H", [96, 20000])
def test_layer_norm_backward_dx_has_the_type_that_is_asked_for(fff_lib, H, p):
    """The branch's gradient in the branch's type, with dropout and without; ds itself only where both are one."""
    gen = _gen(H)
    for st in ("f32", "bf16"):
        s, dy, up = _randn(gen, 9, H, dtype=st), _randn(gen, 9, H, dtype="bf16"), _randn(gen, 9, H, dtype=st)
        mean, rstd = torch.zeros(9, device=DEV), torch.ones(9, device=DEV)
        kw = {"ds_in": up, "p": p, "seed": SEED, "offset": OFFSET} if p else {"ds_in": up}
        want, err = ref.layer_norm_backward(dy, s, mean, rstd, None, up, p, SEED, OFFSET)
        for xt in ("f32", "bf16"):
            for names in (("ds", "dx"), ("dx",), ("ds", "dx", "dgamma", "dbeta")):
                flush_print(f"[gpu] layer_norm_backward 9x{H} stream {st} branch {xt} p={p} {names}")
                got = fff_lib.layer_norm_backward(dy, s, mean, rstd, dx_dtype=DT[xt], want=names, **kw)
                assert got[1].dtype == DT[xt]
                ref.check(got[1], want[1], err[1], "dx")
                if "ds" in names:
                    assert got[0].dtype == DT[st] and (got[0] is got[1]) == (p == 0 and st == xt)
                    ref.check(got[0], want[0], err[0], "ds")
        free = fff_lib.layer_norm_backward(dy, s, mean, rstd, **kw)  # no type asked for
        assert free[1].dtype == (DT[st] if p == 0 else torch.bfloat16)


def test_sizes_past_32_bits_are_refused(fff_lib):
    """Not handed on as their low 32 bits: the trees, ids and divisors of calls that would be in order, and long rows."""
    ids = torch.zeros(8, dtype=torch.int32, device=DEV)
    x, w = torch.ones((4, 8), device=DEV), torch.ones((1, 8, 8), device=DEV)
    offsets = torch.tensor([0, 4], dtype=torch.int32, device=DEV)
    wide = torch.empty((1, (1 << 32) + 8), dtype=torch.bfloat16, device=DEV)
    flush_print("[gpu] sizes past 32 bits")
    for call in (lambda: fff_lib.group_rows(ids, 4, first=1 << 32), lambda: fff_lib.group_rows(ids, 4, first=-(1 << 32)),
                 lambda: fff_lib.group_rows(ids, (1 << 32) + 4), lambda: fff_lib.group_rows(ids, 4, n_trees=(1 << 32) + 1),
                 lambda: fff_lib.grouped_matmul(x, w, offsets, x_index=ids[:4], x_div=(1 << 32) + 1),
                 lambda: fff_lib.grouped_weight_grad(x, x, offsets, x_index=ids[:4], x_div=(1 << 32) + 1),
                 lambda: fff_lib.layer_norm(wide), lambda: fff_lib.dropout(wide, 0.1, 1),
                 lambda: fff_lib.layer_norm_backward(wide, wide, x[0, :1].clone(), x[0, :1].clone())):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("H", [1, 30, 100, 250, 768, 1000, 2001, 4099, 12289, 20000])
def test_layer_norm_backward_of_constant_rows_of_any_size(fff_lib, H):
    """xh is 0 in them, however large the value times 1 / sqrt(eps) would be: ds = rstd (g - mean(g))."""
    s = torch.tensor([0.0, 2.0 ** 100, -(2.0 ** 112), 2.0 ** 20], device=DEV)[:, None].repeat(1, H)
    dy = torch.zeros_like(s)
    dy[:, 0] = 1.0
    flush_print(f"[gpu] layer_norm_backward of constant rows, {H}")
    y, _, mean, rstd = fff_lib.layer_norm(s, eps=2.0 ** -40)
    assert (y == 0).all() and torch.equal(mean, s[:, 0]) and (rstd == 2.0 ** 20).all()
    ds, _, dgamma, dbeta = fff_lib.layer_norm_backward(dy, s, mean, rstd)
    want = 2.0 ** 20 * (dy.double() - dy.double().mean(1, keepdim=True))
    assert ((ds.double() - want).abs() <= 3 * ref.U * 2.0 ** 20).all()  # of the mean, of the difference, of the product
    assert (dgamma == 0).all() and torch.equal(dbeta, dy.sum(0))


@pytest.mark.parametrize("H", [100, 768, 20000])
def test_layer_norm_stream_has_the_type_that_is_asked_for(fff_lib, H):
    """A stream that starts from a branch in another type, or in a buffer of the caller's, with dropout and without."""
    gen = _gen(H)
    x = _randn(gen, 7, H, dtype="bf16", mean=0.5)
    flush_print(f"[gpu] layer_norm 7x{H}, a stream of its own type")
    for p in (0.0, 0.3):
        kw = {"p": p, "seed": SEED, "offset": OFFSET} if p else {}
        want, err = ref.layer_norm(x, None, None, 1e-5, None, p, SEED, OFFSET)
        y, s, mean, rstd = fff_lib.layer_norm(x, eps=1e-5, s_dtype=torch.float32, **kw)
        assert s.dtype == torch.float32
        for got, w, e, what in zip((y, s, mean, rstd), want, err, ("y", "s", "mean", "rstd")):
            ref.check(got, w, e, what)
        for dt in (torch.float32, torch.bfloat16):
            buf = torch.full((7, H), 9.0, dtype=dt, device=DEV)
            got = fff_lib.layer_norm(x, eps=1e-5, s=buf, **kw)
            assert got[1] is buf and torch.equal(buf, s.to(dt)) and torch.equal(got[0], y)
    assert fff_lib.layer_norm(x, s_dtype=torch.bfloat16)[1] is x and fff_lib.layer_norm(x)[1] is x
    with pytest.raises(fff_lib.FffError):
        fff_lib.layer_norm(x, s=x)

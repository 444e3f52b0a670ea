"""A routed expert block's operators on the GPU against their definitions in 64 bits (tests/routed_ref.py)."""
from __future__ import annotations

import math

import pytest
import torch

from tests import ops_ref
from tests import routed_ref as ref
from tests.conftest import flush_print

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
INF, NAN = math.inf, math.nan


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _randn(gen, *shape, dtype="f32", mean=0.0, scale=1.0):
    return (torch.randn(shape, generator=gen, device=DEV) * scale + mean).to(DT[dtype])


# --------------------------------------------------------------------------------------------- routing


def _check_route(fff, logits, k, what, **kw):
    ids, w = fff.route(logits, k, **kw)
    want, weights, err = ref.route(logits, k, **kw)
    assert torch.equal(ids.cpu(), want), f"{what}: ids differ at {(ids.cpu() != want).nonzero()[:3].tolist()}"
    ops_ref.check(w, weights, err, f"{what}: weights")
    again = fff.route(logits, k, **kw)
    assert torch.equal(again[0], ids) and torch.equal(again[1], w)
    return ids, w


ROUTE_SIZES = [(1, 1, 1), (3, 2, 1), (5, 3, 3), (2, 7, 4), (33, 8, 2), (1, 64, 2), (17, 63, 5), (130, 64, 8), (9, 65, 64),
               (5, 100, 10), (70, 128, 4), (257, 255, 3), (19, 256, 8), (1, 256, 8), (4, 257, 16), (3, 511, 64), (6, 512, 6),
               (2, 1000, 20), (3, 1024, 8), (2, 1025, 9), (2, 4096, 33), (1, 5000, 2), (1, 32768, 64)]


@pytest.mark.parametrize("T,E,k", ROUTE_SIZES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route(fff_lib, T, E, k, score):
    for n, (t, renormalise, with_bias) in enumerate([("f32", True, False), ("bf16", False, True), ("f32", False, True),
                                                     ("bf16", True, False)]):
        flush_print(f"[gpu] route {T}x{E} top {k} {score} {t} renormalise={renormalise} bias={with_bias}")
        gen = _gen(13 * T + E + n)
        logits = _randn(gen, T, E, dtype=t, scale=1.5)
        bias = _randn(gen, E, scale=0.1) if with_bias else None
        _check_route(fff_lib, logits, k, f"{T}x{E}", score=score, bias=bias, renormalise=renormalise, scale=2.5)


@pytest.mark.parametrize("T,E,k,G,keep", [(40, 8, 2, 4, 2), (40, 12, 3, 3, 1), (70, 64, 6, 8, 3), (33, 60, 5, 5, 5), (50, 30, 4, 15, 4),
                                          (25, 256, 8, 8, 4), (9, 256, 8, 256, 9), (20, 21, 2, 7, 2), (5, 1024, 8, 32, 6),
                                          (3, 2048, 10, 1024, 5), (2, 4100, 9, 41, 7), (1, 160, 6, 8, 3)])
@pytest.mark.parametrize("group_score", ["max", "top2"])
def test_route_groups(fff_lib, T, E, k, G, keep, group_score):
    for n, (t, score, with_bias) in enumerate([("f32", "sigmoid", True), ("bf16", "softmax", False),
                                               ("f32", "softmax", True), ("bf16", "sigmoid", False)]):
        flush_print(f"[gpu] route {T}x{E} top {k}, {keep} of {G} groups by {group_score}, {score} {t} bias={with_bias}")
        gen = _gen(7 * T + E + n)
        logits = _randn(gen, T, E, dtype=t, scale=1.5)
        logits[0, : E // 2] = -INF  # whole groups without an expert
        if T > 1:
            logits[1] = -INF
        bias = _randn(gen, E, scale=0.1) if with_bias else None
        _check_route(fff_lib, logits, k, f"{T}x{E}", score=score, bias=bias, n_groups=G, top_groups=keep,
                     group_score=group_score, renormalise=n % 2 == 0)


@pytest.mark.parametrize("T,E,k,G,keep", [
    (70, 64, 14, 8, 5), (67, 256, 16, 16, 9), (66, 100, 11, 1, 1), (65, 33, 16, 1, 1), (65, 17, 9, 1, 1), (69, 64, 16, 4, 1),
    (40, 256, 24, 1, 1), (37, 64, 30, 1, 1), (33, 512, 32, 32, 20), (35, 500, 17, 1, 1), (34, 128, 20, 32, 12), (38, 256, 8, 32, 5),
    (21, 1024, 6, 64, 9), (20, 256, 40, 64, 30), (19, 128, 64, 32, 32), (36, 96, 32, 1, 1), (39, 72, 25, 18, 9), (45, 50, 8, 5, 5)])
def test_route_many_picks(fff_lib, T, E, k, G, keep):
    """Less than two lanes a pick, and groups over 16, 32 and 64 lanes; some tokens with few experts, some with equal ones."""
    for n, (t, score, with_bias, group_score) in enumerate([
            ("f32", "sigmoid", True, "top2"), ("bf16", "softmax", False, "max"), ("f32", "softmax", True, "max"),
            ("bf16", "sigmoid", True, "top2")]):
        flush_print(f"[gpu] route {T}x{E} top {k}, {keep} of {G} groups by {group_score}, {score} {t} bias={with_bias}")
        gen = _gen(11 * T + E + n)
        logits = _randn(gen, T, E, dtype=t, scale=1.5)
        logits[2::5] = torch.randint(-2, 3, logits[2::5].shape, generator=gen, device=DEV).to(logits.dtype)
        logits[3::5, : E - k // 2] = -INF  # less than k
        logits[4::5, ::2] = NAN
        bias = _randn(gen, E, scale=0.1) if with_bias else None
        _check_route(fff_lib, logits, k, f"{T}x{E}", score=score, bias=bias, n_groups=G, top_groups=keep,
                     group_score=group_score, renormalise=n % 2 == 0)
        if with_bias:  # equal and nearly equal sums
            _check_route(fff_lib, logits, k, f"{T}x{E}", score=score, bias=torch.zeros_like(bias), n_groups=G, top_groups=keep,
                         group_score=group_score)


@pytest.mark.parametrize("E", [6, 64, 200, 256, 1000, 3000])
def test_route_ties_go_to_the_lowest_index(fff_lib, E):
    """Equal logits under equal biases, many of them: integers in bf16, all equal, and equal sums in 64 bits."""
    gen, k = _gen(E), 6
    for name, logits in (("all equal", torch.full((5, E), 0.5, device=DEV)),
                         ("integers", torch.randint(-2, 3, (40, E), generator=gen, device=DEV).float()),
                         ("lowest values", torch.full((3, E), torch.finfo(torch.float32).min, device=DEV))):
        for t in ("f32", "bf16"):
            l = logits.clamp(min=torch.finfo(DT[t]).min).to(DT[t])
            for kw in ({}, {"bias": torch.zeros(E, device=DEV)}, {"bias": torch.full((E,), 0.25, device=DEV), "score": "sigmoid"},
                       {"score": "sigmoid", "n_groups": 2, "top_groups": 1}, {"n_groups": 2, "top_groups": 1, "group_score": "max"},
                       {"bias": (torch.arange(E, device=DEV) % 3).float(), "score": "sigmoid", "renormalise": True}):
                flush_print(f"[gpu] route ties, {name} {E} {t} {sorted(kw)}")
                _check_route(fff_lib, l, k, f"{name} {E}", **kw)


@pytest.mark.parametrize("E", [16, 64, 256, 500, 2000])
def test_route_zeros_and_infinities_of_either_type(fff_lib, E):
    """0 and -0 are equal, in any order; several infinite logits share a softmax, above the largest finite one."""
    gen = _gen(E + 4)
    logits = torch.where(torch.rand((6, E), generator=gen, device=DEV) < 0.5, 0.0, -0.0)
    logits[1] = -logits[1].abs() - 1.0
    logits[1, ::3], logits[1, 1::3] = 0.0, -0.0
    logits[2, 3] = logits[2, 9] = logits[2, 10] = INF
    logits[3, 3], logits[3, 5] = torch.finfo(torch.bfloat16).max, INF
    logits[4], logits[4, 7] = -INF, INF
    logits[5, 2:] = torch.finfo(torch.bfloat16).min
    for t in ("f32", "bf16"):
        for score in ("softmax", "sigmoid"):
            for kw in ({}, {"renormalise": True}, {"n_groups": 2, "top_groups": 1, "group_score": "max"}, {"n_groups": 4, "top_groups": 2},
                       {"bias": torch.zeros(E, device=DEV)}):
                flush_print(f"[gpu] route zeros and infinities {E} {t} {score} {sorted(kw)}")
                ids, w = _check_route(fff_lib, logits.to(DT[t]), 5, f"{E} {t}", score=score, **kw)
                assert torch.isfinite(w).all()


@pytest.mark.parametrize("E", [4, 100, 600, 2000])
def test_route_small_scores_keep_their_shares(fff_lib, E):
    """Renormalised sigmoids that fp32 holds no more beside one that it does, far below 0."""
    for top in (-21.0, -50.0, -59.0, -70.0, -200.0):
        logits = torch.full((3, E), -1e4, device=DEV)
        logits[:, 1], logits[:, 2] = top, torch.tensor([top - 1.0, top - 40.0, top - 60.0], device=DEV)
        flush_print(f"[gpu] route small scores {E} from {top}")
        _, w = _check_route(fff_lib, logits, 2, f"{E} from {top}", score="sigmoid", renormalise=True)
        assert (w > 0).all()
        dw = torch.tensor([[0.0, 1.0]] * 3, device=DEV)
        ids = torch.tensor([[1, 2]] * 3, dtype=torch.int32, device=DEV)
        got = fff_lib.route_backward(dw, logits, ids, score="sigmoid", renormalise=True)
        want, err = ref.route_backward(dw, logits, ids, score="sigmoid", renormalise=True)
        ops_ref.check(got, want, err, f"gradient {E} from {top}")


@pytest.mark.parametrize("E,G", [(64, 1), (256, 8), (100, 5), (3000, 1)])
def test_route_order_of_close_choices(fff_lib, E, G):
    """Choices closer to each other than fp32 resolves: a bias that takes back what the score differs by, to 1e-9."""
    gen = _gen(E + 1)
    for score in ("sigmoid", "softmax"):
        logits = _randn(gen, 1, E)
        s = ref.scores(ref.clean(logits), score)[0]
        bias = (0.7 - s).float()  # sums within 2^-25 of each other, no two alike
        logits = logits.repeat(20, 1)
        flush_print(f"[gpu] route close choices {E} {score}")
        _check_route(fff_lib, logits, 8, f"close {E} {score}", score=score, bias=bias.to(DEV), n_groups=G,
                     top_groups=max(1, G // 2))


@pytest.mark.parametrize("E", [40, 64, 256, 700, 2500])
def test_route_masked_and_not_finite(fff_lib, E):
    gen = _gen(E + 2)
    logits = _randn(gen, 9, E)
    logits[0] = -INF
    logits[1, 3:] = -INF                        # fewer experts than asked for
    logits[2] = NAN
    logits[3, ::2] = NAN
    logits[4, 5] = logits[4, 9] = INF
    logits[5] = torch.finfo(torch.float32).min  # a mask by the lowest value leaves a row of equal experts
    logits[5, 7] = 0.0
    logits[6] = -3000.0 - torch.arange(E, device=DEV) % 7
    logits[7] = torch.finfo(torch.float32).max
    bias = _randn(gen, E, scale=0.1)
    bias[2], bias[4], bias[11] = NAN, -INF, INF
    for score in ("softmax", "sigmoid"):
        for renormalise in (False, True):
            for b in (None, bias):
                for kw in ({}, {"n_groups": 4, "top_groups": 2} if E % 4 == 0 else {}):
                    flush_print(f"[gpu] route not finite {E} {score} {renormalise} bias={b is not None} {kw}")
                    ids, w = _check_route(fff_lib, logits, 5, f"masked {E}", score=score, renormalise=renormalise, bias=b, **kw)
                    assert (ids[0] == -1).all() and (w[0] == 0).all() and (ids[2] == -1).all() and (ids[1, 3:] == -1).all()


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (3, 2, 2), (40, 8, 2), (7, 63, 4), (65, 64, 4), (9, 65, 64), (33, 100, 10),
                                   (130, 256, 8), (1, 256, 8), (5, 511, 3), (3, 1024, 7), (2, 3000, 16), (1, 32768, 64)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [False, True])
def test_route_backward(fff_lib, T, E, k, score, renormalise):
    for n, (t, dt) in enumerate([("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")]):
        flush_print(f"[gpu] route_backward {T}x{E} top {k} {score} renormalise={renormalise} {t}/{dt}")
        gen = _gen(3 * T + E + n)
        logits, dw = _randn(gen, T, E, dtype=t, scale=1.5), _randn(gen, T, k)
        ids, _ = fff_lib.route(logits, min(k, E), score=score, renormalise=renormalise)
        ids = ids[:, torch.randperm(k, device=DEV, generator=gen)].contiguous()
        got = fff_lib.route_backward(dw, logits, ids, score=score, renormalise=renormalise, scale=2.5, dlogits_dtype=DT[dt])
        want, err = ref.route_backward(dw, logits, ids, score, renormalise, 2.5)
        ops_ref.check(got, want, err, f"dlogits {T}x{E}")
        assert got.dtype == DT[dt]


@pytest.mark.parametrize("E", [30, 64, 256, 900])
def test_route_backward_any_ids(fff_lib, E):
    """Ids out of range, an expert twice, masked experts, rows without any; large logits that saturate."""
    gen = _gen(E + 3)
    logits, dw = _randn(gen, 8, E), _randn(gen, 8, 6)
    ids = torch.randint(0, E, (8, 6), generator=gen, device=DEV).to(torch.int32)
    ids[0, 1], ids[0, 4], ids[0, 5] = ids[0, 0], E, -7
    ids[1] = -1
    ids[2] = ids[2, 0]
    ids[3, 0], ids[3, 1] = 2 ** 31 - 1, -2 ** 31
    logits[4] = -INF
    logits[5, ids[5, 2].long()] = -INF
    logits[5, ids[5, 3].long()] = NAN
    logits[6] *= 40
    logits[7] = -2000.0 - torch.arange(E, device=DEV) % 3
    for score in ("softmax", "sigmoid"):
        for renormalise in (False, True):
            flush_print(f"[gpu] route_backward any ids {E} {score} {renormalise}")
            got = fff_lib.route_backward(dw, logits, ids, score=score, renormalise=renormalise)
            want, err = ref.route_backward(dw, logits, ids, score, renormalise)
            ops_ref.check(got, want, err, f"dlogits {E} {score} {renormalise}")
            assert (got[4] == 0).all()


# --------------------------------------------------------------------------------------------- combine

COMBINE_SIZES = [(1, 1, 1), (2, 3, 5), (7, 2, 8), (5, 4, 31), (33, 1, 64), (9, 8, 100), (4, 5, 129), (6, 6, 256), (3, 2, 257),
                 (17, 3, 519), (11, 8, 768), (3, 16, 1001), (5, 2, 1024), (2, 9, 2056), (8, 8, 4096), (1, 4, 8200), (2, 70, 40),
                 (1, 1, 16384), (300, 4, 96),
                 # many tokens: lanes a token
                 (8200, 3, 20), (8193, 1, 127), (4099, 5, 200), (4096, 2, 129), (2050, 5, 520), (2049, 6, 1001), (515, 6, 1100),
                 (513, 4, 2051), (600, 1, 4099), (512, 3, 2048)]


@pytest.mark.parametrize("T,k,H", COMBINE_SIZES)
def test_combine(fff_lib, T, k, H):
    for n, (rt, yt, weighted, dropped, residual) in enumerate([
            ("bf16", "bf16", True, True, True), ("f32", "f32", True, False, False), ("bf16", "f32", False, True, True),
            ("f32", "bf16", True, True, False), ("bf16", "bf16", False, False, False)]):
        flush_print(f"[gpu] combine {T}x{k}x{H} {rt}/{yt} weighted={weighted} dropped={dropped} residual={residual}")
        gen = _gen(T + 10 * k + 100 * H + n)
        rows = _randn(gen, T * k, H, dtype=rt)
        weights = _randn(gen, T, k) if weighted else None
        ids = torch.randint(-2, 5, (T, k), generator=gen, device=DEV).to(torch.int32) if dropped else None
        if dropped:
            rows[ids.flatten() < 0] = NAN
        res = _randn(gen, T, H, dtype=yt) if residual else None
        y = fff_lib.combine(rows, k, weights, ids=ids, residual=res, y_dtype=DT[yt])
        want, err = ref.combine(rows, k, weights, ids, res)
        ops_ref.check(y, want, err, f"combine {T}x{k}x{H}")
        if residual:
            stream = res.clone()
            assert fff_lib.combine(rows, k, weights, ids=ids, residual=stream, y=stream) is stream
            assert torch.equal(stream, y)


@pytest.mark.parametrize("T,k,H", COMBINE_SIZES)
def test_combine_backward(fff_lib, T, k, H):
    for n, (yt, rt, dt, weighted, dropped) in enumerate([
            ("bf16", "bf16", "bf16", True, True), ("f32", "f32", "f32", True, False), ("bf16", "f32", "bf16", False, True),
            ("f32", "bf16", "f32", True, True)]):
        flush_print(f"[gpu] combine_backward {T}x{k}x{H} {yt}/{rt}/{dt} weighted={weighted} dropped={dropped}")
        gen = _gen(T + 10 * k + 100 * H + n)
        dy, rows = _randn(gen, T, H, dtype=yt), _randn(gen, T * k, H, dtype=rt)
        weights = _randn(gen, T, k) if weighted else None
        ids = torch.randint(-2, 5, (T, k), generator=gen, device=DEV).to(torch.int32) if dropped else None
        if dropped:
            rows[ids.flatten() < 0] = NAN
        got = fff_lib.combine_backward(dy, k, rows, weights, ids=ids, drows_dtype=DT[dt])
        want, err = ref.combine_backward(dy, k, rows, weights, ids)
        for v, w, e, what in zip(got, want, err, ("drows", "dweights")):
            ops_ref.check(v, w, e, f"{what} {T}x{k}x{H}")
        # each gradient alone, and the rows' gradient in their own buffer: the same bits
        alone = fff_lib.combine_backward(dy, k, None, weights, ids=ids, drows_dtype=DT[dt])
        assert torch.equal(alone[0], got[0]) and alone[1] is None
        alone = fff_lib.combine_backward(dy, k, rows, weights, ids=ids, want=("dweights",))
        assert alone[0] is None and torch.equal(alone[1], got[1])
        if rt == dt:
            inside = rows.clone()
            again = fff_lib.combine_backward(dy, k, inside, weights, ids=ids, drows=inside)
            assert again[0] is inside and torch.equal(inside, got[0]) and torch.equal(again[1], got[1])


@pytest.mark.parametrize("T,k,H", [(3, 2, 2563), (5, 1, 4099), (2, 4, 8191), (1, 1, 2049)])
def test_combine_backward_long_rows_in_place(fff_lib, T, k, H):
    """Rows that several waves share, with a part of a vector at their end: the gradient written over them changes no
    sum that another wave is still forming."""
    for dt in ("bf16", "f32"):
        flush_print(f"[gpu] combine_backward in place {T}x{k}x{H} {dt}")
        gen = _gen(T + 10 * k + 100 * H)
        dy, rows, weights = _randn(gen, T, H, dtype=dt), _randn(gen, T * k, H, dtype=dt), _randn(gen, T, k)
        want, err = ref.combine_backward(dy, k, rows, weights, None)
        got = fff_lib.combine_backward(dy, k, rows, weights)
        for _ in range(8):
            inside = rows.clone()
            again = fff_lib.combine_backward(dy, k, inside, weights, drows=inside)
            for v, o, w, e, what in zip(again, got, want, err, ("drows", "dweights")):
                ops_ref.check(v, w, e, f"{what} {T}x{k}x{H}")
                assert torch.equal(v, o)


def test_combine_rows_apart(fff_lib):
    """NaN in a row that takes part spoils its own token's column alone; a weight of 0 does not hide it."""
    for H in (40, 77, 512):
        rows, w = torch.ones((12, H), device=DEV), torch.ones((4, 3), device=DEV)
        rows[4, 3], w[1, 1] = NAN, 0.0
        rows[11, H - 1] = INF
        flush_print(f"[gpu] combine rows apart {H}")
        y = fff_lib.combine(rows, 3, w)
        bad = torch.zeros((4, H), dtype=torch.bool, device=DEV)
        bad[1, 3], bad[3, H - 1] = True, True
        assert torch.equal(~torch.isfinite(y), bad) and (y[~bad][:H] == 3).all()


# -------------------------------------------------------------------------------------------- RMS norm

RMS_SHAPES = [(1, 1), (3, 2), (2, 3), (5, 4), (1, 8), (7, 31), (3, 33), (9, 100), (4, 255), (33, 256), (6, 257), (5, 300),
              (10, 512), (3, 519), (130, 768), (2, 769), (65, 1000), (17, 1024), (3, 1032), (5, 1536), (4, 2001), (9, 2048),
              (3, 2056), (7, 4096), (2, 4099), (3, 8192), (2, 8200), (3, 16384), (2, 16390), (2, 40001)]
RMS_TYPES = [("bf16", "bf16", "bf16"), ("f32", "f32", "f32"), ("bf16", "f32", "bf16"), ("f32", "bf16", "f32")]


def _codes(packed):
    return packed.values.view(torch.uint8), packed.scales.view(torch.uint8)


@pytest.mark.parametrize("B,H", RMS_SHAPES)
@pytest.mark.parametrize("residual", [False, True])
def test_rms_norm(fff_lib, B, H, residual):
    for n, (xt, st, yt) in enumerate(RMS_TYPES):
        flush_print(f"[gpu] rms_norm {B}x{H} {xt}/{st}/{yt} residual={residual}")
        gen = _gen(100 * H + B + n)
        x = _randn(gen, B, H, dtype=xt, mean=0.5)
        res = _randn(gen, B, H, dtype=st, mean=-1.0) if residual else None
        gamma = _randn(gen, H, mean=1.0) if n != 1 else None
        y, s, rstd, packed = fff_lib.rms_norm(x, gamma, eps=1e-5, residual=res, y_dtype=DT[yt])
        want, err = ref.rms_norm(x, gamma, 1e-5, res)
        for got, w, e, what in zip((y, s, rstd), want, err, ("y", "s", "rstd")):
            ops_ref.check(got, w, e, f"{what} {B}x{H} {xt}/{st}/{yt}")
        assert packed is None and (residual or s is x)
        # the 8-bit copy is the fp32 y's; it changes nothing else, nor does leaving y out
        fine, s2, rstd2, packed = fff_lib.rms_norm(x, gamma, eps=1e-5, residual=res, y_dtype=torch.float32, pack=True)
        assert torch.equal(s2, s) and torch.equal(rstd2, rstd) and torch.equal(fine.to(DT[yt]), y)
        values, codes = ref.pack(fine)
        assert torch.equal(packed.values.float().cpu().double(), values)
        assert torch.equal(_codes(packed)[1].cpu(), codes)
        none, _, _, only = fff_lib.rms_norm(x, gamma, eps=1e-5, residual=res, pack=True, want_y=False, stats=False)
        assert none is None and all(torch.equal(a, b) for a, b in zip(_codes(only), _codes(packed)))
        if residual:
            stream = res.clone()
            inside = fff_lib.rms_norm(x, gamma, eps=1e-5, residual=stream, s=stream, y_dtype=DT[yt])
            assert inside[1] is stream and torch.equal(stream, s) and torch.equal(inside[0], y)


@pytest.mark.parametrize("B,H", RMS_SHAPES)
@pytest.mark.parametrize("stream", [False, True])
def test_rms_norm_backward(fff_lib, B, H, stream):
    for n, (xt, st, yt) in enumerate(RMS_TYPES):
        flush_print(f"[gpu] rms_norm_backward {B}x{H} {xt}/{st}/{yt} stream={stream}")
        gen = _gen(77 * H + B + n)
        s, dy = _randn(gen, B, H, dtype=st, mean=0.5), _randn(gen, B, H, dtype=yt)
        gamma = _randn(gen, H, mean=1.0) if n != 1 else None
        ds_in = _randn(gen, B, H, dtype=st) if stream else None
        rstd = (1 / torch.sqrt(s.double().square().mean(1) + 1e-5)).float()
        ds, dx, dgamma = fff_lib.rms_norm_backward(dy, s, rstd, gamma, ds_in=ds_in, dx_dtype=DT[xt])
        want, err = ref.rms_norm_backward(dy, s, rstd, gamma, ds_in)
        for got, w, e, what in zip((ds, dx, dgamma), (want[0], want[0], want[1]), (err[0], err[0], err[1]), ("ds", "dx", "dgamma")):
            ops_ref.check(got, w, e, f"{what} {B}x{H} {xt}/{st}/{yt}")
        assert (dx is ds) == (xt == st)
        again = fff_lib.rms_norm_backward(dy, s, rstd, gamma, ds_in=ds_in, dx_dtype=DT[xt])
        assert all(torch.equal(a, b) for a, b in zip((ds, dx, dgamma), again))
        if stream:
            inside = ds_in.clone()
            assert fff_lib.rms_norm_backward(dy, s, rstd, gamma, ds_in=inside, ds=inside)[0] is inside
            assert torch.equal(inside, ds)


@pytest.mark.parametrize("B,H,t", [(4097, 768, "bf16"), (2500, 100, "f32"), (700, 1024, "f32"), (1030, 4096, "bf16"), (3, 20000, "f32")])
def test_rms_norm_backward_many_rows(fff_lib, B, H, t):
    gen = _gen(B)
    s, dy, gamma = _randn(gen, B, H, dtype=t, mean=1.0), _randn(gen, B, H, dtype=t), _randn(gen, H, mean=1.0)
    rstd = (1 / torch.sqrt(s.double().square().mean(1) + 1e-5)).float()
    flush_print(f"[gpu] rms_norm_backward {B}x{H} {t}")
    got = fff_lib.rms_norm_backward(dy, s, rstd, gamma)
    want, err = ref.rms_norm_backward(dy, s, rstd, gamma)
    for v, w, e, what in zip((got[0], got[2]), want, err, ("ds", "dgamma")):
        ops_ref.check(v, w, e, what)
    for name, full in (("ds", got[0]), ("dgamma", got[2])):
        one = fff_lib.rms_norm_backward(dy, s, rstd, gamma, want=(name,))
        assert [v is not None for v in one].count(True) == 1
        assert torch.equal(next(v for v in one if v is not None), full), name
    dgamma = torch.full((H,), 2.0, device=DEV)
    fff_lib.rms_norm_backward(dy, s, rstd, gamma, dgamma=dgamma, accumulate=True, want=())
    assert torch.equal(dgamma, got[2] + 2.0)


@pytest.mark.parametrize("H", [96, 768, 4096, 20000])
def test_rms_norm_rows_apart(fff_lib, H):
    """A row of infinities or NaN spoils no other; a row of zeros stays one (eps > 0)."""
    gen = _gen(H)
    x = _randn(gen, 6, H)
    x[1, 3], x[2, 5], x[3] = INF, NAN, 0.0
    flush_print(f"[gpu] rms_norm rows apart, {H}")
    y, _, _, packed = fff_lib.rms_norm(x, None, eps=1e-5, pack=True)
    assert torch.isnan(y[2]).all() and torch.isnan(y[1, 3]) and (y[3] == 0).all()
    ok = [0, 3, 4, 5]
    want, err = ref.rms_norm(x[ok], None, 1e-5)
    ops_ref.check(y[ok], want[0], err[0], "finite rows")
    assert torch.equal(packed.values.float()[ok].cpu().double(), ref.pack(y[ok])[0])


def test_no_rows(fff_lib):
    e = torch.empty((0, 64), device=DEV)
    y, s, rstd, packed = fff_lib.rms_norm(e, pack=True)
    assert y.shape == (0, 64) and rstd.numel() == 0 and packed.scales.shape == (0, 2)
    g = torch.full((64,), 5.0, device=DEV)
    fff_lib.rms_norm_backward(e, e, rstd, dgamma=g, accumulate=True)
    assert (g == 5).all()
    fff_lib.rms_norm_backward(e, e, rstd, dgamma=g)
    assert (g == 0).all()
    ids, w = fff_lib.route(e, 4)
    assert ids.shape == (0, 4) and w.shape == (0, 4)
    assert fff_lib.route_backward(w, e, ids).shape == (0, 64)
    assert fff_lib.combine(e, 4, w).shape == (0, 64)
    drows, dw = fff_lib.combine_backward(e, 4, e, w)
    assert drows.shape == (0, 64) and dw.shape == (0, 4)
    assert fff_lib.unpack_rows(fff_lib.pack_rows(e)).shape == (0, 64)
    assert fff_lib.activation_backward(e, packed).shape == (0, 64)


# --------------------------------------------------------------------------------------- 8-bit rows

PACK_SHAPES = [(1, 1), (3, 7), (5, 8), (2, 31), (4, 32), (9, 33), (1, 40), (6, 63), (7, 100), (333, 101), (17, 256), (65, 300),
               (3, 1000), (40, 1024), (2, 4099), (5, 8192), (1, 70001)]


@pytest.mark.parametrize("B,H", PACK_SHAPES)
@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_pack_and_unpack(fff_lib, B, H, t):
    flush_print(f"[gpu] pack {B}x{H} {t}")
    gen = _gen(B + H)
    x = (_randn(gen, B, H) * torch.exp(3 * _randn(gen, B, H))).to(DT[t])
    packed = fff_lib.pack_rows(x)
    values, codes = ref.pack(x)
    assert torch.equal(packed.values.float().cpu().double(), values) and torch.equal(_codes(packed)[1].cpu(), codes)
    back = ref.unpack(packed.values, codes)
    for dt in (torch.float32, torch.bfloat16):
        assert torch.equal(fff_lib.unpack_rows(packed, dtype=dt).cpu().double(), back), dt
    y = torch.full((B, H), NAN, device=DEV)
    assert fff_lib.unpack_rows(packed, y=y) is y and torch.equal(y.cpu().double(), back)


def test_pack_every_value(fff_lib):
    """Every e4m3 value comes back as it is, and every number half way between two goes to the even code, at every scale."""
    table = torch.tensor(ref.E4M3, dtype=torch.float64)
    between = (table[1:] + table[:-1]) / 2
    v = torch.cat((table, between, between * (1 + 2.0 ** -20), between * (1 - 2.0 ** -20)))
    v = torch.cat((v, -v))
    blocks = torch.zeros((-(-v.numel() // 31), 32), dtype=torch.float64)
    blocks[:, 0] = 448.0  # the block's scale
    blocks[:, 1:].reshape(-1)
    flat = torch.zeros(blocks.shape[0] * 31, dtype=torch.float64)
    flat[:v.numel()] = v
    blocks[:, 1:] = flat.view(-1, 31)
    flush_print("[gpu] pack every value")
    for power in (-126, -100, -9, 0, 1, 60, 118):
        x = (blocks * 2.0 ** power).float()
        packed = fff_lib.pack_rows(x.to(DEV))
        values, codes = ref.pack(x)
        assert (codes == 127 + power).all()
        assert torch.equal(packed.values.float().cpu().double(), values), power
        assert torch.equal(_codes(packed)[1].cpu(), codes)


def test_pack_extremes(fff_lib):
    """Blocks of zeros, of the largest and of denormal numbers, with infinities and NaN among them."""
    f = torch.finfo(torch.float32)
    x = torch.zeros((12, 70))
    x[1] = f.max
    x[2, 3] = f.tiny
    x[3] = torch.arange(70) * 2.0 ** -149
    x[4, 5], x[4, 40] = INF, NAN
    x[4, 6], x[4, 41] = 3.0, -5.0
    x[5], x[6] = INF, NAN
    x[7] = -0.0
    x[8, 0], x[8, 1] = 2.0 ** 100, 2.0 ** -100
    x[9, 64:] = 448.5
    x[10] = f.min
    x[11] = torch.linspace(-1e-37, 1e-37, 70)
    flush_print("[gpu] pack extremes")
    packed = fff_lib.pack_rows(x.to(DEV))
    values, codes = ref.pack(x)
    got = packed.values.float().cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(values)) and torch.equal(got.nan_to_num(), values.nan_to_num())
    assert torch.equal(_codes(packed)[1].cpu(), codes)
    back = fff_lib.unpack_rows(packed, dtype=torch.float32).cpu().double()
    assert torch.equal(back.nan_to_num(), ref.unpack(packed.values, codes).nan_to_num())
    # any scale byte, as another program may have written it
    every = torch.arange(256, dtype=torch.uint8).repeat(3, 1)
    ones = torch.full((3, 256 * 32), 1.5).to(torch.float8_e4m3fn)
    back = fff_lib.unpack_rows(type(packed)(ones.to(DEV), every.to(DEV).view(torch.float8_e8m0fnu)), dtype=torch.float32)
    want = ref.unpack(ones, every)
    assert torch.equal(back.cpu().double().nan_to_num(), want.nan_to_num()) and torch.isnan(back[:, -32:]).all()


def test_unpack_every_byte_at_every_scale(fff_lib):
    """All 256 values at all 256 scales, as other programs may write them: exact, to infinity where fp32 ends."""
    values = torch.arange(256, dtype=torch.uint8).repeat(256, 1).view(torch.float8_e4m3fn)
    codes = torch.arange(256, dtype=torch.uint8)[:, None].repeat(1, 8)
    flush_print("[gpu] unpack every byte at every scale")
    packed = fff_lib.Packed(values.to(DEV), codes.to(DEV).view(torch.float8_e8m0fnu))
    want = ref.unpack(values, codes).float()
    for dt in (torch.float32, torch.bfloat16):
        got = fff_lib.unpack_rows(packed, dtype=dt).cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(got.nan_to_num(7.0), want.to(dt).nan_to_num(7.0))


@pytest.mark.parametrize("B,H", PACK_SHAPES)
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "identity"])
def test_activation_from_packed_rows(fff_lib, B, H, act):
    for t, dt in (("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")):
        flush_print(f"[gpu] activation of packed rows {B}x{H} {act} {t}/{dt}")
        gen = _gen(B + H)
        packed = fff_lib.pack_rows(_randn(gen, B, H, scale=2.0))
        dy = _randn(gen, B, H, dtype=t)
        z = ref.unpack(packed.values, _codes(packed)[1])
        y, ey, dx, edx = ref.activations(z, act, dy.cpu().double())
        got = fff_lib.unpack_rows(packed, act=act, dtype=DT[dt])
        ops_ref.check(got, y, ey, f"act {B}x{H} {act}")
        d, again = fff_lib.activation_backward(dy, packed, act, dx_dtype=DT[dt], keep_y=True, y_dtype=DT[dt])
        ops_ref.check(d, dx, edx, f"slope {B}x{H} {act}")
        assert torch.equal(again, got)
        assert torch.equal(fff_lib.activation_backward(dy, packed, act, dx_dtype=DT[dt]), d)
        if t == dt:
            inside = dy.clone()
            assert fff_lib.activation_backward(inside, packed, act, dx=inside) is inside and torch.equal(inside, d)


def test_activation_of_far_packed_values(fff_lib):
    """Large pre-activations keep finite activations and gradients, as their formulas do."""
    z = torch.tensor([[0.0, -0.0, 5.0, -5.0, 12.0, -12.0, 40.0, -40.0, 1e6, -1e6, 1e19, -1e19, 1e30, -1e30, 1e38, -1e38]], device=DEV)
    z = z.T.contiguous()  # a block each
    packed = fff_lib.pack_rows(z)
    want = ref.unpack(packed.values, _codes(packed)[1])
    for act in ("gelu", "gelu_tanh"):
        flush_print(f"[gpu] far packed values {act}")
        dx, y = fff_lib.activation_backward(torch.ones_like(z), packed, act, keep_y=True)
        assert torch.isfinite(y).all() and torch.isfinite(dx).all()
        assert torch.allclose(y.cpu().double(), torch.where(want > 0, want, 0.0) if act else want, atol=1e-4, rtol=1e-5)
        assert torch.allclose(dx.cpu().double()[2:], (want[2:] > 0).double(), atol=1e-4)


def test_past_four_billion_elements(fff_lib):
    """Rows behind element 2^32: packed, read back, normalised and combined as the same rows alone."""
    B, H = (1 << 18) + 3, 16400
    gen = _gen(9)
    x = torch.zeros((B, H), dtype=torch.bfloat16, device=DEV)
    tail = _randn(gen, 4, H, dtype="bf16")
    x[-4:] = tail
    flush_print("[gpu] past 2^32 elements: pack")
    packed, alone = fff_lib.pack_rows(x), fff_lib.pack_rows(tail)
    assert all(torch.equal(a[-4:], b) for a, b in zip(_codes(packed), _codes(alone)))
    y = fff_lib.unpack_rows(packed, act="gelu")
    assert torch.equal(y[-4:], fff_lib.unpack_rows(alone, act="gelu")) and (y[:4] == 0).all()
    del packed, y
    flush_print("[gpu] past 2^32 elements: rms_norm")
    y, _, rstd, packed = fff_lib.rms_norm(x, pack=True)
    want = fff_lib.rms_norm(tail, pack=True)
    assert torch.equal(y[-4:], want[0]) and torch.equal(rstd[-4:], want[2])
    assert all(torch.equal(a[-4:], b) for a, b in zip(_codes(packed), _codes(want[3])))
    del y, packed
    flush_print("[gpu] past 2^32 elements: combine")
    x = x[3:]
    x = x.contiguous() if x.data_ptr() % 16 else x
    y = fff_lib.combine(x, 2)
    assert torch.equal(y[-2:], fff_lib.combine(tail, 2))
    drows, _ = fff_lib.combine_backward(y, 2)
    assert torch.equal(drows[-4:], y[-2:].repeat_interleave(2, 0)) and (drows[:4] == 0).all()


# ------------------------------------------------------------------------ streams, graphs, whole steps


def _block(fff, t):
    """A routed expert block forward and backward, with its kept activations in 8 bits.  t: its tensors."""
    k, E, out = t["k"], t["router"].shape[1], {}
    T = t["x"].shape[0]
    all_rows = torch.tensor([0, T], dtype=torch.int32, device=DEV) if "all" not in t else t["all"]
    u, s, rstd, u8 = fff.rms_norm(t["x"], t["gamma"], eps=1e-5, residual=t["stream"], pack=True)
    logits = fff.grouped_matmul(u, t["router"], all_rows, y_dtype=torch.float32)
    if t.get("mask") is not None:
        logits.masked_fill_(t["mask"][:, None], -INF)
    ids, w = fff.route(logits, k, bias=t["bias"], score="sigmoid", n_groups=t["groups"], top_groups=t["keep"],
                       renormalise=True, scale=2.0)
    order, offsets = fff.group_rows(ids, E)
    h, z = fff.grouped_matmul(u, t["up"], offsets, x_index=order, x_div=k, act="gelu", keep_z=True)
    z8 = fff.pack_rows(z)
    rows = torch.full((T * k, u.shape[1]), NAN, dtype=u.dtype, device=DEV)  # nothing in entries without an expert
    fff.grouped_matmul(h, t["down"], offsets, y=rows, y_index=order)
    y = fff.combine(rows, k, w, ids=ids, residual=s)
    # backward
    drows, dw = fff.combine_backward(t["dy"], k, rows, w, ids=ids)
    dh = fff.grouped_matmul(drows, t["down"], offsets, x_index=order, transpose_w=True)
    dz, h8 = fff.activation_backward(dh, z8, "gelu", keep_y=True)
    ddown = fff.grouped_weight_grad(drows, h8, offsets, dy_index=order)
    dup = fff.grouped_weight_grad(dz, fff.unpack_rows(u8, dtype=u.dtype), offsets, x_index=order, x_div=k)
    du_rows = torch.full((T * k, u.shape[1]), NAN, dtype=u.dtype, device=DEV)
    fff.grouped_matmul(dz, t["up"], offsets, y=du_rows, y_index=order, transpose_w=True)
    dlogits = fff.route_backward(dw, logits, ids, score="sigmoid", renormalise=True, scale=2.0, dlogits_dtype=u.dtype)
    drouter = fff.grouped_weight_grad(dlogits, u, all_rows)
    du = fff.combine(du_rows, k, ids=ids, residual=fff.grouped_matmul(dlogits, t["router"], all_rows, transpose_w=True))
    ds, dx, dgamma = fff.rms_norm_backward(du, s, rstd, t["gamma"], ds_in=t["dy"])
    out = {"y": y, "ids": ids, "w": w, "dx": dx, "dgamma": dgamma, "drouter": drouter, "dup": dup, "ddown": ddown,
           "u8": u8.values.view(torch.uint8), "us": u8.scales.view(torch.uint8), "z8": z8.values.view(torch.uint8),
           "zs": z8.scales.view(torch.uint8), "order": order, "offsets": offsets}
    return out


def _block_inputs(seed, T=37, H=48, F=80, E=12, k=3, dtype="f32", masked=True):
    gen = _gen(seed)
    t = {"x": _randn(gen, T, H, dtype=dtype), "stream": _randn(gen, T, H, dtype=dtype), "gamma": _randn(gen, H, mean=1.0, scale=0.2),
         "router": _randn(gen, 1, E, H, dtype=dtype, scale=H ** -0.5), "bias": _randn(gen, E, scale=0.05),
         "up": _randn(gen, E, F, H, dtype=dtype, scale=H ** -0.5), "down": _randn(gen, E, H, F, dtype=dtype, scale=F ** -0.5),
         "dy": _randn(gen, T, H, dtype=dtype), "k": k, "groups": 4, "keep": 2,
         "all": torch.tensor([0, T], dtype=torch.int32, device=DEV),
         "mask": (torch.arange(T, device=DEV) % 7 == 3) if masked else None}
    t["router"] = t["router"].view(1, E, H)
    return t


def _block_fp64(t, got):
    """The block by torch's own derivatives in 64 bits, with the device's choices and kept activations."""
    f8 = torch.float64
    c = {n: t[n].cpu().to(f8) for n in ("x", "stream", "gamma", "router", "bias", "up", "down", "dy")}
    leaf = {n: c[n].clone().requires_grad_(True) for n in ("x", "gamma", "router", "up", "down")}
    k, T, H = t["k"], *t["x"].shape
    s = c["stream"] + leaf["x"]
    u = s / torch.sqrt(s.square().mean(1, keepdim=True) + 1e-5) * leaf["gamma"]
    l = u @ leaf["router"][0].T
    ids = got["ids"].cpu().long()
    live = ids >= 0
    p = torch.where(live, torch.sigmoid(l.gather(1, ids.clamp(min=0))), 0.0)
    w = 2.0 * p / p.sum(1, keepdim=True).clamp(min=1e-300)
    order, count = got["order"].cpu().long(), int(got["offsets"][-1])
    u8, z8 = (ref.unpack(got[a].view(torch.float8_e4m3fn), got[b]) for a, b in (("u8", "us"), ("z8", "zs")))
    kept = torch.zeros((T * k, z8.shape[1]), dtype=f8)
    kept[order[:count]] = z8[:count]
    slope = ops_ref.act_grad(kept, "gelu")

    class Up(torch.autograd.Function):
        # the first product and GELU, whose derivatives see the kept activations
        @staticmethod
        def forward(ctx, row, up, row8, slope):
            ctx.save_for_backward(up, row8, slope)
            return ops_ref.act(up @ row, "gelu")

        @staticmethod
        def backward(ctx, g):
            up, row8, slope = ctx.saved_tensors
            return up.T @ (g * slope), torch.outer(g * slope, row8), None, None

    class Down(torch.autograd.Function):
        @staticmethod
        def forward(ctx, h, down, z8):
            ctx.save_for_backward(down, z8)
            return down @ h

        @staticmethod
        def backward(ctx, g):
            down, z8 = ctx.saved_tensors
            return down.T @ g, torch.outer(g, ops_ref.act(z8, "gelu")), None

    y = []
    for i in range(T):
        acc = s[i]
        for j in range(k):
            if live[i, j]:
                e = int(ids[i, j])
                h = Up.apply(u[i], leaf["up"][e], u8[i], slope[i * k + j])
                acc = acc + w[i, j] * Down.apply(h, leaf["down"][e], kept[i * k + j])
        y.append(acc)
    y = torch.stack(y)
    (y * c["dy"]).sum().backward()
    return {"y": y.detach(), "w": w.detach(), "dx": leaf["x"].grad, "dgamma": leaf["gamma"].grad,
            "drouter": leaf["router"].grad, "dup": leaf["up"].grad, "ddown": leaf["down"].grad}


@pytest.mark.parametrize("T", [1, 37])
def test_routed_block_step(fff_lib, T):
    """Norm, routing, grouping, the experts, the sum and every gradient, against 64-bit derivatives.

    The longest chain of fp32 sums has 3 x 80 + 4 x 48 terms and a handful of factors, 500 U or 3e-5 of a
    result's largest terms: 1e-4 in the 2-norm of each output."""
    t = _block_inputs(T, T=T)
    flush_print(f"[gpu] routed block step, {T} tokens")
    got = _block(fff_lib, t)
    want = _block_fp64(t, got)
    assert (got["ids"][t["mask"]] == -1).all() and (got["ids"][~t["mask"]] >= 0).all()
    for n, v in want.items():
        g = got[n].cpu().double().view(v.shape)
        assert torch.isfinite(g).all(), n
        assert (g - v).norm() <= 1e-4 * v.norm() + 1e-12, (n, float((g - v).norm() / v.norm()))


def test_routed_block_in_a_graph(fff_lib):
    """The whole block captured, replayed on new inputs between eager calls, and twice at once on two streams."""
    ins = [_block_inputs(i, T=300, H=256, F=512, E=32, dtype="bf16") for i in range(2)]
    flush_print("[gpu] routed block in a graph")
    want = [_block(fff_lib, t) for t in ins]
    torch.cuda.synchronize()
    graphs, outs, streams = [], [], [torch.cuda.Stream() for _ in range(2)]
    for t in ins:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(_block(fff_lib, t))
        graphs.append(g)

    def same(a, b):
        # entries behind the last group's are left as they were
        n = int(b["offsets"][-1])
        for name in b:
            x, y = a[name], b[name]
            if name in ("order", "z8", "zs"):
                x, y = x[:n], y[:n]
            assert torch.equal(x, y), name

    for _ in range(3):
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        eager = _block(fff_lib, ins[1])
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            same(a, b)
        same(eager, want[1])
    swapped = {n: v.clone() if torch.is_tensor(v) else v for n, v in ins[0].items()}
    for n, v in ins[1].items():
        if torch.is_tensor(v):
            ins[0][n].copy_(v)
    graphs[0].replay()
    torch.cuda.synchronize()
    same(outs[0], want[1])
    for n, v in swapped.items():
        if torch.is_tensor(v):
            ins[0][n].copy_(v)


def test_routed_operators_on_a_stream(fff_lib):
    """A call on another stream runs behind that stream's work, on results that it alone wrote."""
    gen = _gen(5)
    logits, rows, dy = _randn(gen, 5000, 64), _randn(gen, 20000, 256), _randn(gen, 5000, 256)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    flush_print("[gpu] routed operators on a stream")
    with torch.cuda.stream(side):
        l2, r2, d2 = logits * 2, rows * 2, dy * 2
    ids, w = fff_lib.route(l2, 4, stream=side)
    dl = fff_lib.route_backward(w, l2, ids, stream=side)
    y = fff_lib.combine(r2, 4, w, ids=ids, stream=side)
    drows, dw = fff_lib.combine_backward(d2, 4, r2, w, stream=side)
    n, _, rstd, packed = fff_lib.rms_norm(y, pack=True, stream=side)
    ds = fff_lib.rms_norm_backward(d2, y, rstd, stream=side)
    z = fff_lib.unpack_rows(packed, act="gelu", stream=side)
    g = fff_lib.activation_backward(d2, fff_lib.pack_rows(y, stream=side), stream=side)
    side.synchronize()
    got = (ids, w, dl, y, drows, dw, n, rstd, ds[0], ds[2], z, g)
    ids, w = fff_lib.route(logits * 2, 4)
    y = fff_lib.combine(rows * 2, 4, w, ids=ids)
    n, _, rstd, packed = fff_lib.rms_norm(y, pack=True)
    ds = fff_lib.rms_norm_backward(dy * 2, y, rstd)
    want = (ids, w, fff_lib.route_backward(w, logits * 2, ids), y, *fff_lib.combine_backward(dy * 2, 4, rows * 2, w), n, rstd, ds[0],
            ds[2], fff_lib.unpack_rows(packed, act="gelu"), fff_lib.activation_backward(dy * 2, fff_lib.pack_rows(y)))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_trees_rows_are_added(fff_lib):
    """The rows of a token's trees, without weights: the step that the leaf experts' products leave open."""
    gen = _gen(8)
    T, trees, depth, H = 50, 3, 3, 64
    ids = torch.randint(0, 2 ** depth, (T, trees), generator=gen, device=DEV).to(torch.int32)
    w, x = _randn(gen, trees * 2 ** depth, H, H, scale=0.1), _randn(gen, T, H)
    order, offsets = fff_lib.group_rows(ids, 2 ** depth, n_trees=trees)
    rows = fff_lib.grouped_matmul(x, w, offsets, x_index=order, x_div=trees, y_index=order)
    flush_print("[gpu] trees' rows added")
    y = fff_lib.combine(rows, trees, residual=x)
    c = ids.cpu().long() + torch.arange(trees) * 2 ** depth
    want = x.cpu().double() + torch.einsum("tkhi,ti->th", w.cpu().double()[c], x.cpu().double())
    assert (y.cpu().double() - want).norm() <= 1e-5 * want.norm()  # sums of 64 terms: 66 U of them


def test_refusals_of_the_binding(fff_lib):
    x = torch.zeros((6, 40), device=DEV)
    packed = fff_lib.pack_rows(x)
    ids, w = fff_lib.route(x, 2)
    bad = [
        lambda: fff_lib.route(x.half(), 2), lambda: fff_lib.route(x[:, ::2], 2), lambda: fff_lib.route(x.view(-1), 2),
        lambda: fff_lib.route(x, 0), lambda: fff_lib.route(x, 2, bias=x[0].bfloat16()), lambda: fff_lib.route(x, 2, bias=x[0, :3]),
        lambda: fff_lib.route(x, 2, score="relu"), lambda: fff_lib.route(x, 2, group_score="top3"),
        lambda: fff_lib.route(x, 2, ids=ids.long()), lambda: fff_lib.route(x, 2, weights=w.bfloat16()),
        lambda: fff_lib.route(x, 3, ids=ids), lambda: fff_lib.route(x, 1 << 33), lambda: fff_lib.route(x, 2, n_groups=1 << 40),
        lambda: fff_lib.route_backward(w.bfloat16(), x, ids), lambda: fff_lib.route_backward(w, x[:5].contiguous(), ids),
        lambda: fff_lib.route_backward(w, x, ids[:, :1].contiguous()), lambda: fff_lib.route_backward(w, x, None),
        lambda: fff_lib.combine(x, 4), lambda: fff_lib.combine(x, 0), lambda: fff_lib.combine(x, 2, w),
        lambda: fff_lib.combine(x, 2, residual=x), lambda: fff_lib.combine(x, 3, residual=x[:2].bfloat16(), y_dtype=torch.float32),
        lambda: fff_lib.combine(x, 2, ids=ids.float()), lambda: fff_lib.combine_backward(x, 2, x), lambda: fff_lib.combine_backward(x, 0),
        lambda: fff_lib.rms_norm(x, x[0, :5]), lambda: fff_lib.rms_norm(x, want_y=False),
        lambda: fff_lib.rms_norm(x, residual=x[:3]), lambda: fff_lib.rms_norm(x, packed=fff_lib.pack_rows(x[:3])),
        lambda: fff_lib.rms_norm(x, residual=x, s_dtype=torch.bfloat16), lambda: fff_lib.rms_norm_backward(x, None, None),
        lambda: fff_lib.rms_norm_backward(x, x, w[:, 0]), lambda: fff_lib.rms_norm_backward(x, x, x[:, 0].contiguous(), accumulate=True),
        lambda: fff_lib.unpack_rows(type(packed)(x, packed.scales)), lambda: fff_lib.unpack_rows(type(packed)(packed.values, x)),
        lambda: fff_lib.unpack_rows(packed, dtype=torch.float16), lambda: fff_lib.unpack_rows(type(packed)(packed.values.cpu(), packed.scales)),
        lambda: fff_lib.unpack_rows(type(packed)(packed.values, packed.scales.cpu())),
        lambda: fff_lib.activation_backward(x[:5].contiguous(), packed), lambda: fff_lib.pack_rows(x.double()),
        lambda: fff_lib.pack_rows(x, packed=x), lambda: fff_lib.route(x.cpu(), 2), lambda: fff_lib.combine(x, 2, w.cpu()),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print(f"call {i} was not refused")
    for call in (lambda: fff_lib.route(x, 41), lambda: fff_lib.route(x, 2, n_groups=7), lambda: fff_lib.route(x, 2, top_groups=2),
                 lambda: fff_lib.route(x, 2, scale=INF), lambda: fff_lib.rms_norm(x, eps=-1.0),
                 lambda: fff_lib.combine(x, 2, y=x[:3]), lambda: fff_lib.rms_norm(x, y=x)):
        with pytest.raises(fff_lib.FffError):
            call()

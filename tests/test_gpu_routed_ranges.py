"""A routed expert block's operators at the far ends of their ranges, against their definitions in 64 bits (tests/routed_ref.py)."""
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


@pytest.mark.parametrize("E", [4, 100, 300, 600, 2000])
@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_route_shares_of_sigmoids_far_apart(fff_lib, E, t):
    """Renormalised sigmoids whose exponential leaves fp32 beside one near 0: their shares are normal fp32 numbers, and so
    are the shares' gradients.  The references' bounds are absolute below 2^-126 alone."""
    seconds = torch.tensor([-30.0, -70.0, -85.0, -87.0, -88.5, -89.0, -90.0, -95.0, -100.0, -105.0], device=DEV)
    for top in (-25.0, -20.0, -19.875, -19.5, -15.0, -8.0, -3.0, -0.5, 0.0, 3.0):
        logits = torch.full((len(seconds), E), -1e4, device=DEV)
        logits[:, 1], logits[:, 2], logits[:, 3] = top, seconds, seconds - 2
        logits = logits.to(DT[t])
        flush_print(f"[gpu] route shares far apart {E} {t} from {top}")
        ids, w = fff_lib.route(logits, 3, score="sigmoid", renormalise=True, scale=2.0)
        want, weights, err = ref.route(logits, 3, score="sigmoid", renormalise=True, scale=2.0)
        assert torch.equal(ids.cpu(), want)
        ops_ref.check(w, weights, err, f"{E} from {top}: weights")
        dw = torch.tensor([0.5, 1.0, -2.0], device=DEV).repeat(len(seconds), 1)
        got = fff_lib.route_backward(dw, logits, ids, score="sigmoid", renormalise=True, scale=2.0, dlogits_dtype=torch.float32)
        d, derr = ref.route_backward(dw, logits, ids, score="sigmoid", renormalise=True, scale=2.0)
        ops_ref.check(got, d, derr, f"{E} from {top}: gradient")


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "identity"])
def test_activation_of_every_byte_at_every_scale(fff_lib, act):
    """All 256 values at all 256 scales, as other programs may write them, infinities among them: what the formulas give
    in IEEE arithmetic (+inf from +inf; NaN from NaN, from -inf and for the derivative of either), the same in each type."""
    values = torch.arange(256, dtype=torch.uint8).repeat(256, 1).view(torch.float8_e4m3fn)
    codes = torch.arange(256, dtype=torch.uint8)[:, None].repeat(1, 8)
    packed = fff_lib.Packed(values.to(DEV), codes.to(DEV).view(torch.float8_e8m0fnu))
    flush_print(f"[gpu] {act} of every byte at every scale")
    z = ref.unpack(values, codes).float()  # infinite where fp32 ends
    finite, up = torch.isfinite(z), z == math.inf
    assert up.sum() > 100 and (z == -math.inf).sum() > 100
    y, ey, dx, edx = ref.activations(torch.where(finite, z, 0.0).double(), act, torch.ones(z.shape, dtype=torch.float64))
    # |y| = |z| Phi(z) for z < 0 is below 0.4 exp(-z^2 / 2) (Phi(z) < phi(z) / |z|): where that exponential leaves the normal
    # numbers of fp32, from -13.3 on, and is lost, y is off by 0.4 times 2^-126 at most
    ey = ey + 0.4 * ref.TINY
    for dt in (torch.float32, torch.bfloat16):
        got = fff_lib.unpack_rows(packed, act=act, dtype=dt).cpu()
        slope, again = (v.cpu() for v in fff_lib.activation_backward(torch.ones(z.shape, dtype=dt, device=DEV), packed, act, keep_y=True))
        assert torch.equal(torch.isnan(got), torch.isnan(again)) and torch.equal(got.nan_to_num(7.0), again.nan_to_num(7.0))
        assert (got[up] == math.inf).all()
        if act == "identity":
            assert torch.equal(got[~torch.isnan(z)], z.to(dt)[~torch.isnan(z)]) and (slope == 1).all()
        else:
            assert torch.isnan(got[~finite & ~up]).all() and torch.isnan(slope[~finite]).all()
        assert torch.isnan(got[torch.isnan(z)]).all()
        ops_ref.check(torch.where(finite, got, 0.0), y, ey, f"{act} {dt}")
        ops_ref.check(torch.where(finite, slope, dx.to(dt)), dx, edx, f"slope of {act} {dt}")


def test_activation_beside_a_far_block(fff_lib):
    """A block's activations have the same bits whatever its neighbours' scales."""
    gen = torch.Generator(device=DEV).manual_seed(3)
    for H in (96, 100, 1024):
        z = torch.randn((40, H), generator=gen, device=DEV) * 3
        far = z.clone()
        far[::3] = 3e38
        flush_print(f"[gpu] activation beside a far block {H}")
        a, b = fff_lib.pack_rows(z), fff_lib.pack_rows(far)
        near = torch.arange(40, device=DEV) % 3 != 0
        for act in ("gelu", "gelu_tanh"):
            for dt in (torch.float32, torch.bfloat16):
                dy = torch.ones((40, H), dtype=dt, device=DEV)
                for u, v in zip(fff_lib.activation_backward(dy, a, act, keep_y=True), fff_lib.activation_backward(dy, b, act, keep_y=True)):
                    assert torch.equal(u[near], v[near])
                assert torch.equal(v[~near], fff_lib.unpack_rows(b, dtype=dt)[~near])


def test_an_unknown_activation_is_refused(fff_lib):
    """By the error type and the list of names that an unknown score is refused with."""
    x = torch.zeros((3, 40), device=DEV)
    packed = fff_lib.pack_rows(x)
    for call in (lambda: fff_lib.unpack_rows(packed, act="relu"), lambda: fff_lib.activation_backward(x, packed, "relu")):
        with pytest.raises(ValueError, match="act must be one of gelu.*relu"):
            call()
    for act in ("gelu", "gelu_erf", "gelu_tanh", "identity", 0, 1, 2):
        assert (fff_lib.unpack_rows(packed, act=act) == 0).all()


def _tokens_alone(fff, logits, tail, k, what, **kw):
    """route and route_backward of `logits`, whose last rows are `tail`, against `tail` alone."""
    n = tail.shape[0]
    flush_print(f"[gpu] {what}: route")
    ids, w = fff.route(logits, k, **kw)
    one, v = fff.route(tail, k, **kw)
    assert torch.equal(ids[-n:], one) and torch.equal(w[-n:], v)
    assert torch.equal(ids[:4], fff.route(logits[:4].contiguous(), k, **kw)[0])
    del w
    kw = {key: kw[key] for key in ("score", "renormalise") if key in kw}
    dw = torch.zeros(ids.shape, device=DEV)
    dw[-n:] = torch.arange(n * k, device=DEV).view(n, k) % 5 - 1.5
    flush_print(f"[gpu] {what}: route_backward")
    d = fff.route_backward(dw, logits, ids, **kw)
    assert torch.equal(d[-n:], fff.route_backward(dw[-n:].contiguous(), tail, one, **kw)) and (d[:4] == 0).all()
    assert (d[-n:] != 0).any()


def test_route_past_a_launch(fff_lib):
    """More tokens than a launch holds at 16 lanes each: 2^23 workgroups of 16."""
    T, gen = (1 << 27) + 37, torch.Generator(device=DEV).manual_seed(5)
    tail = torch.randn((41, 2), generator=gen, device=DEV).bfloat16()
    logits = torch.zeros((T, 2), dtype=torch.bfloat16, device=DEV)
    logits[-41:] = tail
    _tokens_alone(fff_lib, logits, tail, 2, "past a launch", score="softmax")


@pytest.mark.parametrize("E", [1024, 2048])
def test_route_past_four_billion_logits(fff_lib, E):
    T, gen = (1 << 32) // E + 5, torch.Generator(device=DEV).manual_seed(E)
    tail = torch.randn((7, E), generator=gen, device=DEV).bfloat16()
    logits = torch.zeros((T, E), dtype=torch.bfloat16, device=DEV)
    logits[:, E // 3] = 1.0
    logits[-7:] = tail
    _tokens_alone(fff_lib, logits, tail, 3, f"past 2^32 logits of {E}", score="sigmoid", renormalise=True)
    _tokens_alone(fff_lib, logits, tail, 1, f"past 2^32 logits of {E}", score="softmax")


@pytest.mark.parametrize("H", [1024, 1001, 16400])
def test_rms_norm_past_four_billion_elements(fff_lib, H):
    """Rows held in registers and longer ones, both directions: as the same rows alone."""
    B, gen = (1 << 32) // H + 6, torch.Generator(device=DEV).manual_seed(H)
    x = torch.zeros((B, H), dtype=torch.bfloat16, device=DEV)
    tail = torch.randn((5, H), generator=gen, device=DEV).bfloat16()
    gamma = torch.rand(H, generator=gen, device=DEV) + 0.5
    x[-5:] = tail
    flush_print(f"[gpu] past 2^32 elements of {H}: rms_norm")
    y, s, rstd, packed = fff_lib.rms_norm(x, gamma, pack=True)
    want = fff_lib.rms_norm(tail, gamma, pack=True)
    assert torch.equal(y[-5:], want[0]) and torch.equal(rstd[-5:], want[2]) and (y[:4] == 0).all()
    for a, b in zip(packed, want[3]):
        assert torch.equal(a.view(torch.uint8)[-5:], b.view(torch.uint8))
    del packed
    dy = y  # zeros but for the last rows
    flush_print(f"[gpu] past 2^32 elements of {H}: rms_norm_backward")
    ds, _, dgamma = fff_lib.rms_norm_backward(dy, x, rstd, gamma, ds_in=x)
    alone = fff_lib.rms_norm_backward(want[0], tail, want[2], gamma, ds_in=tail)
    assert torch.equal(ds[-5:], alone[0]) and (ds[:4] == 0).all()
    # five products and sums of them in some order, each of fp32, on both sides
    xh = tail.double() * want[2].double()[:, None]
    assert ((dgamma - alone[2]).double().abs() <= 2 * (5 + 6) * ops_ref.U * (want[0].double() * xh).abs().sum(0)).all()


def test_activation_gradient_past_four_billion_elements(fff_lib):
    for H in (1024, 1001):
        B, gen = (1 << 32) // H + 6, torch.Generator(device=DEV).manual_seed(H)
        z = torch.zeros((B, H), dtype=torch.bfloat16, device=DEV)
        tail = torch.randn((5, H), generator=gen, device=DEV).bfloat16()
        z[-5:] = tail
        flush_print(f"[gpu] past 2^32 elements of {H}: activation_backward")
        packed, alone = fff_lib.pack_rows(z), fff_lib.pack_rows(tail)
        dx, y = fff_lib.activation_backward(z, packed, "gelu", keep_y=True)
        want = fff_lib.activation_backward(tail, alone, "gelu", keep_y=True)
        assert torch.equal(dx[-5:], want[0]) and torch.equal(y[-5:], want[1])
        assert (dx[:4] == 0).all() and (y[:4] == 0).all()


@pytest.mark.parametrize("k,H", [(2, 1024), (3, 1001), (1, 4096)])
def test_combine_gradient_past_four_billion_elements(fff_lib, k, H):
    """The kernel of many tokens, at the lanes of each row length."""
    T, gen = (1 << 32) // (H * k) + 5, torch.Generator(device=DEV).manual_seed(H)
    rows = torch.zeros((T * k, H), dtype=torch.bfloat16, device=DEV)
    tail = torch.randn((3 * k, H), generator=gen, device=DEV).bfloat16()
    rows[-3 * k:] = tail
    w = torch.rand((T, k), generator=gen, device=DEV)
    flush_print(f"[gpu] past 2^32 elements of {k} x {H}: combine")
    dy = fff_lib.combine(rows, k, w)
    assert torch.equal(dy[-3:], fff_lib.combine(tail, k, w[-3:].contiguous()))
    flush_print(f"[gpu] past 2^32 elements of {k} x {H}: combine_backward")
    drows, dw = fff_lib.combine_backward(dy, k, rows, w)
    d = dy[-3:].double()
    want = (w[-3:].double()[:, :, None] * d[:, None]).view(3 * k, H)
    ops_ref.check(drows[-3 * k:], want.cpu(), (ops_ref.U * want.abs()).cpu(), "drows")
    terms = d[:, None] * tail.double().view(3, k, H)
    ops_ref.check(dw[-3:], terms.sum(2).cpu(), ((H + 4) * ops_ref.U * terms.abs().sum(2)).cpu(), "dweights")
    assert (drows[:4] == 0).all() and (dw[:4] == 0).all()


@pytest.mark.parametrize("E", [5, 100, 600, 2000])
@pytest.mark.parametrize("renormalise", [False, True])
def test_route_gradient_of_saturated_sigmoids(fff_lib, E, renormalise):
    """1 - s of logits whose exponential leaves fp32: large gradients of the weights make normal numbers of it."""
    logits = torch.full((6, E), -1e4, device=DEV)
    logits[:, 3] = torch.tensor([80.0, 87.0, 88.5, 89.0, 90.0, 92.0], device=DEV)
    logits[:, 1] = logits[:, 3] - 1
    ids = torch.tensor([[3, 1]] * 6, dtype=torch.int32, device=DEV)
    dw = torch.tensor([[1.0, -1.0]] * 6, device=DEV)
    flush_print(f"[gpu] gradient of saturated sigmoids {E} renormalise={renormalise}")
    got = fff_lib.route_backward(dw, logits, ids, score="sigmoid", renormalise=renormalise, scale=1e9)
    want, err = ref.route_backward(dw, logits, ids, score="sigmoid", renormalise=renormalise, scale=1e9)
    # 1 - s is off by its own roundings, which the references' bounds count relative to it, and by two halves of fp32's
    # smallest step, 2^-149, where it has fewer bits: a factor of what the weights' gradients come to, 1e9 at most
    if not renormalise:
        err = err - ref.TINY * 1e9 * (want != 0)
        assert (err >= 0).all()
    ops_ref.check(got, want, err + 1e9 * 2.0 ** -149 * (want != 0), f"{E}")
    assert (got[:, [1, 3]] != 0).all()

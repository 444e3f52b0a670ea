"""A routed expert block's operators without a GPU: struct layouts, refusals, and the references' own pins."""
import ctypes
import math
import subprocess

import pytest
import torch

import paper_2311_10770_amd as fff
from paper_2311_10770_amd import build as native_build
from paper_2311_10770_amd import fff as binding
from paper_2311_10770_amd import routed
from tests import routed_ref as ref
from tests.conftest import ROOT

INVALID, UNSUPPORTED, WORKSPACE, OK = (binding.FFF_ERR_INVALID_ARG, binding.FFF_ERR_UNSUPPORTED,
                                       binding.FFF_ERR_WORKSPACE, binding.FFF_OK)
P = 1 << 32  # an aligned fake device address; validation never dereferences it
INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module")
def lib():
    if not binding.LIB_PATH.exists():
        native_build.build_lib("libfff.so")
    return binding.load_library()


@pytest.mark.parametrize("cls,cname", [
    (routed.FffRouteArgs, "fff_route_args"), (routed.FffRouteBackwardArgs, "fff_route_backward_args"),
    (routed.FffCombineArgs, "fff_combine_args"), (routed.FffCombineBackwardArgs, "fff_combine_backward_args"),
    (routed.FffRmsNormArgs, "fff_rms_norm_args"), (routed.FffRmsNormBackwardArgs, "fff_rms_norm_backward_args"),
    (routed.FffPackRowsArgs, "fff_pack_rows_args"), (routed.FffUnpackRowsArgs, "fff_unpack_rows_args")])
def test_struct_layout_matches_c(tmp_path, cls, cname):
    fields = [f[0] for f in cls._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "fff.h"\nint main(void){\n'
                   + f'printf("%zu\\n", sizeof({cname}));\n'
                   + "".join(f'printf("%zu\\n", offsetof({cname}, {f}));\n' for f in fields) + "return 0;}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-I", str(ROOT / "include"), str(src), "-o", str(exe)], check=True)
    vals = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert vals == [ctypes.sizeof(cls)] + [getattr(cls, f).offset for f in fields]


def _refused(lib, fn, cls, base, over, code):
    a = cls()
    for k, v in {**base, **over}.items():
        setattr(a, k, v)
    assert getattr(lib, fn)(ctypes.addressof(a)) == code
    assert lib.fff_last_hip_error() == 0


ROUTE = dict(logits=P, bias=2 * P, ids=3 * P, weights=4 * P, n_tokens=5, n_experts=12, top_k=3, n_groups=4,
             top_groups=2, score=1, group_score=1, renormalise=1, scale=1.0)


@pytest.mark.parametrize("over,code", [
    (dict(n_tokens=-1), INVALID), (dict(n_tokens=1 << 31), INVALID), (dict(n_tokens=1 << 30), INVALID),
    (dict(n_experts=0), INVALID), (dict(top_k=0), INVALID), (dict(top_k=13), INVALID), (dict(n_groups=5), INVALID),
    (dict(n_groups=0), INVALID), (dict(top_groups=0), INVALID), (dict(top_groups=5), INVALID), (dict(x_dtype=2), INVALID),
    (dict(score=2), INVALID), (dict(score=-1), INVALID), (dict(group_score=2), INVALID), (dict(renormalise=2), INVALID),
    (dict(scale=INF), INVALID), (dict(scale=NAN), INVALID), (dict(logits=None), INVALID), (dict(ids=None), INVALID),
    (dict(weights=None), INVALID), (dict(logits=P + 4), INVALID), (dict(bias=P + 4), INVALID), (dict(ids=P + 2), INVALID),
    (dict(weights=P + 1), INVALID), (dict(ids=P), INVALID), (dict(ids=4 * P + 56), INVALID), (dict(weights=2 * P), INVALID),
    (dict(n_experts=32772, n_groups=1, top_groups=1), UNSUPPORTED), (dict(n_experts=1000, top_k=65), UNSUPPORTED),
    (dict(n_experts=2048, n_groups=2048), UNSUPPORTED)])
def test_route_refusals(lib, over, code):
    _refused(lib, "fff_route", routed.FffRouteArgs, ROUTE, over, code)


ROUTE_BWD = dict(dweights=P, logits=2 * P, ids=3 * P, dlogits=4 * P, n_tokens=5, n_experts=12, top_k=3, scale=1.0)


@pytest.mark.parametrize("over,code", [
    (dict(n_tokens=-1), INVALID), (dict(n_tokens=1 << 30), INVALID), (dict(n_experts=0), INVALID), (dict(top_k=0), INVALID),
    (dict(x_dtype=2), INVALID), (dict(d_dtype=3), INVALID), (dict(score=2), INVALID), (dict(renormalise=-1), INVALID),
    (dict(scale=NAN), INVALID), (dict(dweights=None), INVALID), (dict(logits=None), INVALID), (dict(ids=None), INVALID),
    (dict(dlogits=None), INVALID), (dict(logits=P + 8), INVALID), (dict(dlogits=P + 8), INVALID), (dict(ids=P + 2), INVALID),
    (dict(dlogits=2 * P), INVALID), (dict(dlogits=P - 16), INVALID), (dict(n_experts=40000), UNSUPPORTED),
    (dict(top_k=65), UNSUPPORTED)])
def test_route_backward_refusals(lib, over, code):
    _refused(lib, "fff_route_backward", routed.FffRouteBackwardArgs, ROUTE_BWD, over, code)


COMBINE = dict(rows=P, weights=2 * P, ids=3 * P, residual=4 * P, y=5 * P, n_tokens=5, hidden=20, top_k=3)


@pytest.mark.parametrize("over,code", [
    (dict(n_tokens=-1), INVALID), (dict(n_tokens=1 << 30), INVALID), (dict(hidden=0), INVALID), (dict(top_k=0), INVALID),
    (dict(rows_dtype=2), INVALID), (dict(y_dtype=2), INVALID), (dict(rows=None), INVALID), (dict(y=None), INVALID),
    (dict(rows=P + 8), INVALID), (dict(residual=P + 8), INVALID), (dict(y=P + 8), INVALID), (dict(weights=P + 2), INVALID),
    (dict(ids=P + 2), INVALID), (dict(y=P), INVALID), (dict(y=2 * P), INVALID), (dict(y=4 * P + 16), INVALID),
    (dict(residual=P, y=P), INVALID), (dict(hidden=2 ** 31 - 1, n_tokens=2 ** 31 - 1, top_k=1), INVALID)])
def test_combine_refusals(lib, over, code):
    _refused(lib, "fff_combine", routed.FffCombineArgs, COMBINE, over, code)


COMBINE_BWD = dict(dy=P, rows=2 * P, weights=3 * P, ids=4 * P, drows=5 * P, dweights=6 * P, n_tokens=5, hidden=20, top_k=3)


@pytest.mark.parametrize("over,code", [
    (dict(n_tokens=-1), INVALID), (dict(hidden=0), INVALID), (dict(top_k=0), INVALID), (dict(y_dtype=2), INVALID),
    (dict(rows_dtype=2), INVALID), (dict(drows_dtype=2), INVALID), (dict(dy=None), INVALID), (dict(rows=None), INVALID),
    (dict(dy=P + 8), INVALID), (dict(rows=P + 8), INVALID), (dict(drows=P + 8), INVALID), (dict(dweights=P + 2), INVALID),
    (dict(drows=P), INVALID), (dict(drows=2 * P + 16), INVALID), (dict(drows=2 * P, rows_dtype=1), INVALID),
    (dict(dweights=2 * P), INVALID), (dict(dweights=5 * P), INVALID), (dict(drows=2 * P, weights=2 * P), INVALID)])
def test_combine_backward_refusals(lib, over, code):
    _refused(lib, "fff_combine_backward", routed.FffCombineBackwardArgs, COMBINE_BWD, over, code)


RMS = dict(x=P, residual=2 * P, gamma=3 * P, y=4 * P, s=5 * P, rstd=6 * P, q=7 * P, q_scale=8 * P, n_tokens=4, hidden=100,
           eps=1e-6)


@pytest.mark.parametrize("over,code", [
    (dict(n_tokens=-1), INVALID), (dict(n_tokens=1 << 32), INVALID), (dict(hidden=0), INVALID), (dict(x_dtype=2), INVALID),
    (dict(s_dtype=2), INVALID), (dict(y_dtype=2), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=NAN), INVALID),
    (dict(eps=INF), INVALID), (dict(x=None), INVALID), (dict(y=None, q=None, q_scale=None), INVALID),
    (dict(q=None), INVALID), (dict(q_scale=None), INVALID), (dict(x=P + 8), INVALID), (dict(residual=P + 8), INVALID),
    (dict(gamma=P + 4), INVALID), (dict(y=P + 8), INVALID), (dict(s=P + 8), INVALID), (dict(rstd=P + 2), INVALID),
    (dict(q=P + 8), INVALID), (dict(q_scale=P + 8), INVALID), (dict(y=P), INVALID), (dict(y=5 * P), INVALID),
    (dict(s=P), INVALID), (dict(s=2 * P + 16), INVALID), (dict(q=4 * P), INVALID), (dict(q_scale=7 * P + 384), INVALID),
    (dict(q=2 * P), INVALID), (dict(rstd=3 * P), INVALID), (dict(x=2 * P, s=2 * P), INVALID)])
def test_rms_norm_refusals(lib, over, code):
    _refused(lib, "fff_rms_norm", routed.FffRmsNormArgs, RMS, over, code)


RMS_BWD = dict(dy=P, s=2 * P, rstd=3 * P, gamma=4 * P, ds_in=5 * P, ds=6 * P, dx=7 * P, dgamma=8 * P, n_tokens=4, hidden=100,
               workspace=9 * P, workspace_bytes=1 << 24)


@pytest.mark.parametrize("over,code", [
    (dict(n_tokens=-1), INVALID), (dict(n_tokens=1 << 32), INVALID), (dict(hidden=0), INVALID), (dict(x_dtype=2), INVALID),
    (dict(s_dtype=2), INVALID), (dict(y_dtype=2), INVALID), (dict(accumulate=2), INVALID), (dict(dy=None), INVALID),
    (dict(s=None), INVALID), (dict(rstd=None), INVALID), (dict(dy=P + 8), INVALID), (dict(ds=P + 8), INVALID),
    (dict(dgamma=P + 8), INVALID), (dict(ds=P), INVALID), (dict(ds=5 * P + 16), INVALID), (dict(dx=5 * P), INVALID),
    (dict(dx=6 * P), INVALID), (dict(dgamma=4 * P), INVALID), (dict(dy=5 * P, ds=5 * P), INVALID),
    (dict(workspace=None), WORKSPACE), (dict(workspace_bytes=64), WORKSPACE), (dict(workspace=9 * P + 16), INVALID),
    (dict(workspace=P), INVALID)])
def test_rms_norm_backward_refusals(lib, over, code):
    _refused(lib, "fff_rms_norm_backward", routed.FffRmsNormBackwardArgs, RMS_BWD, over, code)


PACK = dict(x=P, q=2 * P, q_scale=3 * P, n_rows=4, hidden=100)


@pytest.mark.parametrize("over", [
    dict(n_rows=-1), dict(n_rows=1 << 32), dict(hidden=0), dict(x_dtype=2), dict(x=None), dict(q=None), dict(q_scale=None),
    dict(x=P + 8), dict(q=P + 8), dict(q_scale=P + 8), dict(q=P), dict(q_scale=P + 16), dict(q_scale=2 * P)])
def test_pack_rows_refusals(lib, over):
    _refused(lib, "fff_pack_rows", routed.FffPackRowsArgs, PACK, over, INVALID)


UNPACK = dict(q=P, q_scale=2 * P, dy=3 * P, y=4 * P, dx=5 * P, n_rows=4, hidden=100)


@pytest.mark.parametrize("over", [
    dict(n_rows=-1), dict(n_rows=1 << 32), dict(hidden=0), dict(dy_dtype=2), dict(y_dtype=2), dict(dx_dtype=2), dict(act=3),
    dict(act=-1), dict(q=None), dict(q_scale=None), dict(dy=None), dict(q=P + 8), dict(q_scale=P + 8), dict(dy=P + 8),
    dict(y=P + 8), dict(dx=P + 8), dict(y=P), dict(dx=P), dict(dx=4 * P), dict(dx=3 * P + 16), dict(dx=3 * P, dx_dtype=1),
    dict(y=3 * P), dict(y=2 * P)])
def test_unpack_rows_refusals(lib, over):
    _refused(lib, "fff_unpack_rows", routed.FffUnpackRowsArgs, UNPACK, over, INVALID)


def test_no_rows_is_no_work(lib):
    for fn, cls, sizes in (("fff_route", routed.FffRouteArgs, dict(n_experts=4, top_k=2, n_groups=1, top_groups=1)),
                           ("fff_route_backward", routed.FffRouteBackwardArgs, dict(n_experts=4, top_k=2)),
                           ("fff_combine", routed.FffCombineArgs, dict(hidden=4, top_k=2)),
                           ("fff_combine_backward", routed.FffCombineBackwardArgs, dict(hidden=4, top_k=2)),
                           ("fff_rms_norm", routed.FffRmsNormArgs, dict(hidden=4)),
                           ("fff_rms_norm_backward", routed.FffRmsNormBackwardArgs, dict(hidden=4)),
                           ("fff_pack_rows", routed.FffPackRowsArgs, dict(hidden=4)),
                           ("fff_unpack_rows", routed.FffUnpackRowsArgs, dict(hidden=4))):
        a = cls()
        for k, v in sizes.items():
            setattr(a, k, v)
        assert getattr(lib, fn)(ctypes.addressof(a)) == OK, fn
        assert getattr(lib, fn)(None) == INVALID, fn
    assert lib.fff_rms_norm_backward_workspace_bytes(-1, 4) == 0
    assert lib.fff_rms_norm_backward_workspace_bytes(4, 0) == 0
    assert lib.fff_rms_norm_backward_workspace_bytes(4, 100) > 0


def test_binding_wants_gpu_tensors():
    x = torch.zeros(4, 8)
    packed = fff.Packed(torch.zeros(4, 8).to(torch.float8_e4m3fn), torch.zeros(4, 1).to(torch.float8_e8m0fnu))
    for call in (lambda: fff.route(x, 2), lambda: fff.route_backward(x, x, x), lambda: fff.combine(x, 2),
                 lambda: fff.combine_backward(x, 2), lambda: fff.rms_norm(x), lambda: fff.rms_norm_backward(x, x, x),
                 lambda: fff.pack_rows(x), lambda: fff.unpack_rows(packed), lambda: fff.unpack_rows(3),
                 lambda: fff.activation_backward(x, packed), lambda: fff.rms_norm(None)):
        with pytest.raises(ValueError):
            call()


# -------------------------------------------------------------------------------- the references' pins


def test_reference_route_closed_forms():
    l = torch.tensor([[0.0, math.log(3.0), 0.0, math.log(4.0)], [NAN, -INF, NAN, -INF], [1.0, INF, -INF, INF]])
    ids, w, _ = ref.route(l, 3)
    assert ids.tolist() == [[3, 1, 0], [-1, -1, -1], [1, 3, 0]]
    assert torch.allclose(w[0], torch.tensor([4 / 9, 3 / 9, 1 / 9], dtype=torch.float64))
    assert w[1].tolist() == [0, 0, 0] and w[2].tolist() == [0.5, 0.5, 0.0]
    ids, w, _ = ref.route(l[:1], 2, renormalise=True, scale=7.0)
    assert torch.allclose(w[0], torch.tensor([4.0, 3.0], dtype=torch.float64))
    ids, w, _ = ref.route(torch.zeros(1, 6), 3, bias=torch.tensor([0.0, 0.1, -INF, NAN, 0.1, -0.5]), score="sigmoid")
    assert ids.tolist() == [[1, 4, 0]] and w.tolist() == [[0.5, 0.5, 0.5]]
    # groups of two: by the largest (4 > 3 > 2) and by the sum of two (3 + 2.9)
    l = torch.tensor([[4.0, -9.0, 3.0, 2.9, 2.0, 1.0]])
    assert ref.route(l, 2, n_groups=3, top_groups=1, group_score="max")[0].tolist() == [[0, 1]]
    assert ref.route(l, 2, score="sigmoid", n_groups=3, top_groups=1)[0].tolist() == [[2, 3]]
    # scores that underflow keep their shares
    w = ref.route(torch.tensor([[-2000.0, -2000.0, -INF]]), 3, score="sigmoid", renormalise=True)[1]
    assert w.tolist() == [[0.5, 0.5, 0.0]]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [False, True])
def test_reference_route_gradient_against_differences(score, renormalise):
    gen = torch.Generator().manual_seed(3)
    l = torch.randn(4, 9, generator=gen, dtype=torch.float64)
    l[1, 4], l[2] = -INF, -INF
    ids = torch.tensor([[3, 0, 7], [1, -1, 8], [0, 1, 2], [5, 5, 99]], dtype=torch.int32)  # an expert twice, an id out of range
    dw = torch.randn(4, 3, generator=gen, dtype=torch.float64)

    def loss(v):
        live = (ids >= 0) & (ids < 9)
        s = ref.scores(v, score)
        w = torch.where(live, s.gather(1, ids.clamp(0, 8).long()), 0.0)
        if renormalise:
            w = w / w.sum(1, keepdim=True).clamp(min=1e-300)
        return (1.5 * w * dw).sum()

    got, err = ref.route_backward(dw, l, ids, score, renormalise, 1.5)
    assert (err >= 0).all() and torch.isfinite(err).all()
    for t in range(4):
        for e in range(9):
            if l[t, e] == -INF:
                assert got[t, e] == 0
                continue
            h = torch.zeros_like(l)
            h[t, e] = 1e-5
            assert abs((loss(l + h) - loss(l - h)) / 2e-5 - got[t, e]) < 1e-8


def test_reference_combine_gradient_against_differences():
    gen = torch.Generator().manual_seed(4)
    rows, w = torch.randn(6, 5, generator=gen, dtype=torch.float64), torch.randn(2, 3, generator=gen, dtype=torch.float64)
    dy, ids = torch.randn(2, 5, generator=gen, dtype=torch.float64), torch.tensor([[1, -1, 2], [0, 0, 0]])
    (drows, dweights), _ = ref.combine_backward(dy, 3, rows, w, ids)

    def loss(r, v):
        return (ref.combine(r, 3, v, ids)[0] * dy).sum()

    for v, g, call in ((rows, drows, lambda r: loss(r, w)), (w, dweights, lambda v: loss(rows, v))):
        for i in range(v.numel()):
            h = torch.zeros_like(v)
            h.view(-1)[i] = 1e-5
            assert abs((call(v + h) - call(v - h)) / 2e-5 - g.reshape(-1)[i]) < 1e-8


def test_reference_rms_norm_gradient_against_differences():
    gen = torch.Generator().manual_seed(5)
    s, g = torch.randn(3, 7, generator=gen, dtype=torch.float64), torch.randn(7, generator=gen, dtype=torch.float64)
    dy, up = (torch.randn(3, 7, generator=gen, dtype=torch.float64) for _ in range(2))
    rstd = ref.rms_norm(s, g, 1e-3)[0][2]
    (ds, dgamma), _ = ref.rms_norm_backward(dy, s, rstd, g, up)

    def loss(v, gamma):
        return (ref.rms_norm(v, gamma, 1e-3)[0][0] * dy).sum() + (v * up).sum()

    for v, got, call in ((s, ds, lambda v: loss(v, g)), (g, dgamma, lambda v: loss(s, v))):
        for i in range(v.numel()):
            h = torch.zeros_like(v)
            h.view(-1)[i] = 1e-5
            assert abs((call(v + h) - call(v - h)) / 2e-5 - got.reshape(-1)[i]) < 1e-7
    assert torch.allclose(ref.rms_norm(torch.full((1, 5), 3.0), None, 0.0)[0][0], torch.ones(1, 5, dtype=torch.float64))


def test_reference_pack_against_torch():
    """The reference's e4m3 values against torch's conversion, and its scales' defining property."""
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    assert codes.tolist() == ref.E4M3
    gen = torch.Generator().manual_seed(6)
    x = torch.randn(40, 77, generator=gen) * torch.exp(4 * torch.randn(40, 1, generator=gen))
    x[3, :32], x[4, 5], x[5, 40], x[6, 64:] = 0.0, INF, NAN, torch.tensor(448.0)
    x[7, 0], x[8, 0], x[9, 0] = 448 * 4.0, 449 * 4.0, 1e-40
    values, scale = ref.pack(x)
    by = torch.exp2(scale.double() - 127).repeat_interleave(32, 1)[:, :77]
    v = (x.double() / by).float()
    fine = torch.isfinite(x)
    assert torch.equal(v[fine].to(torch.float8_e4m3fn).double(), values[fine]) and torch.isnan(values[~fine]).all()
    most = torch.where(fine, x.double().abs(), 0.0)
    assert (most <= 448 * by).all()
    for b in range(3):
        top, p = most[:, 32 * b:32 * b + 32].amax(1), torch.exp2(scale[:, b].double() - 127)
        assert ((top > 448 * p / 2) | (scale[:, b] == 0)).all()
    assert scale[7, 0] == 129 and scale[8, 0] == 130 and scale[3, 0] == 0
    assert torch.equal(torch.exp2(scale.double() - 127).float(), scale.view(torch.float8_e8m0fnu).float())
    top = ref.pack(torch.tensor([[torch.finfo(torch.float32).max, -1.9 * 2.0 ** 127, 1.8 * 2.0 ** 127]]))
    assert top[0].tolist() == [[240.0, -240.0, 224.0]] and top[1].tolist() == [[247]]
    # half a step of e4m3, or of the scale's smallest one
    back = ref.unpack(values, scale)
    assert ((back - x.double()).abs()[fine] <= torch.maximum(x.double().abs() / 16, by * 2.0 ** -10)[fine]).all()

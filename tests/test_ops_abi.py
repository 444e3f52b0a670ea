"""The operators around the layer without a GPU: struct layouts, refusals, and the references' own pins."""
import ctypes
import subprocess

import numpy as np
import pytest
import torch

import paper_2311_10770_amd as fff
from paper_2311_10770_amd import build as native_build
from paper_2311_10770_amd import fff as binding
from paper_2311_10770_amd import ops
from tests import ops_ref as ref
from tests.conftest import ROOT

INVALID, UNSUPPORTED, WORKSPACE, OK = (binding.FFF_ERR_INVALID_ARG, binding.FFF_ERR_UNSUPPORTED,
                                       binding.FFF_ERR_WORKSPACE, binding.FFF_OK)
P = 1 << 32  # an aligned fake device address; validation never dereferences it


@pytest.fixture(scope="module")
def lib():
    if not binding.LIB_PATH.exists():
        native_build.build_lib("libfff.so")
    return binding.load_library()


@pytest.mark.parametrize("cls,cname", [
    (ops.FffDropoutRng, "fff_dropout_rng"), (ops.FffLayerNormArgs, "fff_layer_norm_args"),
    (ops.FffLayerNormBackwardArgs, "fff_layer_norm_backward_args"), (ops.FffDropoutArgs, "fff_dropout_args"),
    (ops.FffGroupRowsArgs, "fff_group_rows_args"), (ops.FffGroupedMatmulArgs, "fff_grouped_matmul_args"),
    (ops.FffGroupedWeightGradArgs, "fff_grouped_weight_grad_args")])
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


def _fill(cls, base, over):
    a = cls()
    for k, v in {**base, **over}.items():
        if k in ("p", "rng_offset"):
            setattr(a.drop, k, v)
        else:
            setattr(a, k, v)
    return a


def _refused(lib, fn, a, code):
    assert getattr(lib, fn)(ctypes.addressof(a)) == code
    assert lib.fff_last_hip_error() == 0


NORM = dict(x=P, residual=2 * P, gamma=3 * P, beta=4 * P, y=5 * P, s=6 * P, mean=7 * P, rstd=8 * P, n_tokens=4,
            hidden=100, eps=1e-5)


@pytest.mark.parametrize("over", [
    dict(n_tokens=-1), dict(n_tokens=1 << 32), dict(hidden=0), dict(x_dtype=2), dict(s_dtype=-1), dict(y_dtype=7),
    dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(p=1.0), dict(p=-0.1), dict(p=float("nan")),
    dict(rng_offset=P + 4), dict(x=None), dict(y=None), dict(x=P + 8), dict(residual=P + 2), dict(gamma=P + 4),
    dict(beta=P + 4), dict(y=P + 8), dict(s=P + 2), dict(mean=P + 2), dict(rstd=P + 1),
    dict(y=P), dict(y=P + 16), dict(y=2 * P), dict(y=3 * P), dict(s=5 * P + 1584), dict(s=P), dict(s=2 * P + 16),
    dict(mean=8 * P + 12), dict(mean=P), dict(rstd=4 * P), dict(rng_offset=5 * P), dict(hidden=2 ** 31 - 1, n_tokens=2 ** 32 - 1)])
def test_layer_norm_refusals(lib, over):
    _refused(lib, "fff_layer_norm", _fill(ops.FffLayerNormArgs, NORM, over), INVALID)


def test_no_tokens_is_no_work(lib):
    for fn, cls in (("fff_layer_norm", ops.FffLayerNormArgs), ("fff_dropout", ops.FffDropoutArgs)):
        a = cls()
        a.hidden = 8
        assert getattr(lib, fn)(ctypes.addressof(a)) == OK
        assert getattr(lib, fn)(None) == INVALID
    a = ops.FffLayerNormBackwardArgs()
    a.hidden = 8
    assert lib.fff_layer_norm_backward(ctypes.addressof(a)) == OK
    a = ops.FffGroupedMatmulArgs()
    a.n_groups = a.k = a.n = a.x_div = 1
    assert lib.fff_grouped_matmul(ctypes.addressof(a)) == OK
    for fn in ("fff_layer_norm_backward", "fff_group_rows", "fff_grouped_matmul", "fff_grouped_weight_grad"):
        assert getattr(lib, fn)(None) == INVALID


NORM_BWD = dict(dy=P, s=2 * P, mean=3 * P, rstd=4 * P, gamma=5 * P, ds_in=6 * P, ds=7 * P, dx=8 * P, dgamma=9 * P,
                dbeta=10 * P, n_tokens=4, hidden=100, workspace=11 * P, workspace_bytes=1 << 24)


@pytest.mark.parametrize("over,code", [
    (dict(n_tokens=-1), INVALID), (dict(n_tokens=1 << 32), INVALID), (dict(hidden=0), INVALID), (dict(x_dtype=2), INVALID),
    (dict(s_dtype=3), INVALID), (dict(y_dtype=-1), INVALID), (dict(accumulate=2), INVALID), (dict(p=1.0), INVALID),
    (dict(dy=None), INVALID), (dict(s=None), INVALID), (dict(mean=None), INVALID), (dict(rstd=None), INVALID),
    (dict(dy=P + 4), INVALID), (dict(ds=P + 4), INVALID), (dict(dgamma=P + 4), INVALID), (dict(ds=P), INVALID),
    (dict(ds=2 * P), INVALID), (dict(ds=6 * P + 16), INVALID), (dict(dx=6 * P), INVALID), (dict(dx=7 * P), INVALID),
    (dict(dgamma=10 * P), INVALID), (dict(dgamma=5 * P), INVALID), (dict(workspace=None), WORKSPACE),
    (dict(workspace_bytes=64), WORKSPACE), (dict(workspace=11 * P + 16), INVALID), (dict(workspace=P), INVALID)])
def test_layer_norm_backward_refusals(lib, over, code):
    _refused(lib, "fff_layer_norm_backward", _fill(ops.FffLayerNormBackwardArgs, NORM_BWD, over), code)


DROP = dict(x=P, residual=2 * P, y=3 * P, n_tokens=4, hidden=100, p=0.1)


@pytest.mark.parametrize("over", [
    dict(n_tokens=-1), dict(n_tokens=1 << 32), dict(hidden=0), dict(x_dtype=2), dict(r_dtype=2), dict(y_dtype=2), dict(p=1.0),
    dict(p=-1e-9), dict(x=None), dict(y=None), dict(x=P + 4), dict(residual=P + 4), dict(y=P + 4), dict(y=P + 16),
    dict(y=P, x_dtype=1), dict(y=2 * P, r_dtype=1), dict(rng_offset=3 * P + 8)])
def test_dropout_refusals(lib, over):
    _refused(lib, "fff_dropout", _fill(ops.FffDropoutArgs, DROP, over), INVALID)


def test_in_place_is_for_one_input(lib):
    """The buffer that may be written in place must not be another input too, whatever that one's type."""
    for x_dtype in (0, 1):
        _refused(lib, "fff_layer_norm", _fill(ops.FffLayerNormArgs, NORM, dict(x=2 * P, s=2 * P, x_dtype=x_dtype)), INVALID)
        _refused(lib, "fff_layer_norm_backward",
                 _fill(ops.FffLayerNormBackwardArgs, NORM_BWD, dict(dy=6 * P, ds=6 * P, y_dtype=x_dtype)), INVALID)
    _refused(lib, "fff_dropout", _fill(ops.FffDropoutArgs, DROP, dict(residual=P, y=P, r_dtype=1)), INVALID)
    _refused(lib, "fff_dropout", _fill(ops.FffDropoutArgs, DROP, dict(residual=P, y=P, x_dtype=1)), INVALID)


GROUP = dict(ids=P, order=2 * P, offsets=3 * P, bad_ids=4 * P, n_entries=100000, n_ids=16, n_trees=2, first=15,
             workspace=5 * P, workspace_bytes=1 << 24)


@pytest.mark.parametrize("over,code", [
    (dict(n_entries=-1), INVALID), (dict(n_entries=1 << 31), INVALID), (dict(n_ids=0), INVALID), (dict(n_trees=0), INVALID),
    (dict(n_ids=32768), UNSUPPORTED), (dict(n_ids=2 ** 31 - 1, n_trees=2 ** 31 - 1), UNSUPPORTED),
    (dict(ids=None), INVALID), (dict(order=None), INVALID), (dict(offsets=None), INVALID), (dict(ids=P + 2), INVALID),
    (dict(order=P), INVALID), (dict(offsets=2 * P), INVALID), (dict(bad_ids=2 * P + 4), INVALID),
    (dict(workspace=None), WORKSPACE), (dict(workspace_bytes=8), WORKSPACE), (dict(workspace=5 * P + 4), INVALID),
    (dict(workspace=P), INVALID)])
def test_group_rows_refusals(lib, over, code):
    _refused(lib, "fff_group_rows", _fill(ops.FffGroupRowsArgs, GROUP, over), code)


PRODUCT = dict(x=P, w=2 * P, offsets=3 * P, x_index=4 * P, y_index=5 * P, y=6 * P, z_out=7 * P, n_entries=10, x_rows=10,
               y_rows=10, n_groups=3, k=20, n=30, x_div=1)


@pytest.mark.parametrize("over,code", [
    (dict(n_entries=-1), INVALID), (dict(n_entries=1 << 31), INVALID), (dict(n_groups=0), INVALID), (dict(k=0), INVALID),
    (dict(n=0), INVALID), (dict(n=1 << 28), INVALID), (dict(k=1 << 28), INVALID), (dict(x_div=0), INVALID),
    (dict(x_dtype=2), INVALID), (dict(w_dtype=2), INVALID),
    (dict(y_dtype=2), INVALID), (dict(z_dtype=2), INVALID), (dict(act=3), INVALID), (dict(w_transposed=2), INVALID),
    (dict(x_rows=-1), INVALID), (dict(x_rows=0), INVALID), (dict(x_index=None, x_rows=9), INVALID), (dict(y_index=None, y_rows=9), INVALID),
    (dict(x_rows=1 << 31), INVALID), (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(offsets=None), INVALID),
    (dict(y=None), INVALID), (dict(z_in=8 * P), INVALID), (dict(x=P + 4), INVALID), (dict(w=P + 4), INVALID),
    (dict(offsets=P + 2), INVALID), (dict(x_index=P + 2), INVALID), (dict(y=P), INVALID), (dict(y=2 * P + 16), INVALID),
    (dict(z_out=6 * P + 16), INVALID), (dict(z_out=None, z_in=6 * P), INVALID), (dict(y=3 * P), INVALID),
    (dict(x_dtype=1), UNSUPPORTED), (dict(w_dtype=1), UNSUPPORTED),
    (dict(n_groups=2 ** 31 - 1, k=2 ** 31 - 1, n=2 ** 31 - 1), INVALID)])
def test_grouped_matmul_refusals(lib, over, code):
    _refused(lib, "fff_grouped_matmul", _fill(ops.FffGroupedMatmulArgs, PRODUCT, over), code)


GRAD = dict(dy=P, x=2 * P, offsets=3 * P, dy_index=4 * P, x_index=5 * P, dw=6 * P, n_entries=10, dy_rows=10, x_rows=10,
            n_groups=3, k=20, n=30, x_div=1, workspace=7 * P, workspace_bytes=1 << 30)


@pytest.mark.parametrize("over,code", [
    (dict(n_entries=-1), INVALID), (dict(n_entries=1 << 31), INVALID), (dict(n_groups=0), INVALID), (dict(k=0), INVALID),
    (dict(n=0), INVALID), (dict(x_div=0), INVALID), (dict(dy_dtype=2), INVALID), (dict(x_dtype=2), INVALID),
    (dict(accumulate=2), INVALID), (dict(dy=None), INVALID), (dict(x=None), INVALID), (dict(offsets=None), INVALID),
    (dict(dw=None), INVALID), (dict(x_rows=0), INVALID), (dict(dy_rows=0), INVALID), (dict(dy=P + 4), INVALID), (dict(dw=P + 4), INVALID), (dict(dy_index=None, dy_rows=9), INVALID),
    (dict(x_index=None, x_rows=9), INVALID), (dict(dw=P), INVALID), (dict(dw=2 * P + 32), INVALID), (dict(dw=4 * P), INVALID),
    (dict(dy_dtype=1), UNSUPPORTED)])
def test_grouped_weight_grad_refusals(lib, over, code):
    _refused(lib, "fff_grouped_weight_grad", _fill(ops.FffGroupedWeightGradArgs, GRAD, over), code)


def test_workspace_sizes(lib):
    assert lib.fff_layer_norm_backward_workspace_bytes(-1, 8) == 0
    assert lib.fff_layer_norm_backward_workspace_bytes(4, 0) == 0
    assert lib.fff_layer_norm_backward_workspace_bytes(65536, 768) >= 2 * 4 * 768
    assert lib.fff_group_rows_workspace_bytes(-1, 8, 1) == 0
    assert lib.fff_group_rows_workspace_bytes(10, 32768, 2) == 0
    assert lib.fff_grouped_weight_grad_workspace_bytes(10, 0, 8, 8) == 0
    assert lib.fff_grouped_weight_grad_workspace_bytes(-1, 1, 8, 8) == 0


def test_binding_refuses_before_the_library():
    x = torch.zeros((4, 8))
    for call in (lambda: fff.layer_norm(x), lambda: fff.dropout(x, 0.1, 1), lambda: fff.layer_norm_backward(x, x, x, x),
                 lambda: fff.group_rows(torch.zeros(4, dtype=torch.int32), 2),
                 lambda: fff.grouped_matmul(x, torch.zeros((1, 3, 8)), None),
                 lambda: fff.grouped_weight_grad(x, x, None)):
        with pytest.raises(ValueError):
            call()


def test_generator_known_answers():
    """The published known-answer vectors of Philox4x32-10."""
    full = 2 ** 64 - 1
    for c0, c1, offset, seed, want in (
            (0, 0, 0, 0, (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
            (2 ** 32 - 1, 2 ** 32 - 1, full, full, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
            (0x243F6A88, 0x85A308D3, 0x0370734413198A2E, 0x299F31D0A4093822,
             (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))):
        assert tuple(int(v) for v in ref.philox_words(c0, c1, offset, seed)) == want


def test_references_agree_with_autograd():
    gen = torch.Generator().manual_seed(0)
    x, g, b, dy, up = (torch.randn(s, generator=gen, dtype=torch.float64) for s in ((6, 24), (24,), (24,), (6, 24), (6, 24)))
    v = [t.clone().requires_grad_(True) for t in (x, g, b)]
    (y, s, mean, rstd), _ = ref.layer_norm(x, g, b, 1e-5)
    yt = torch.nn.functional.layer_norm(v[0], (24,), v[1], v[2], 1e-5)
    torch.testing.assert_close(y, yt.detach(), rtol=1e-12, atol=1e-12)
    want = torch.autograd.grad((yt * dy).sum() + (v[0] * up).sum(), v)
    (ds, dx, dg, db), _ = ref.layer_norm_backward(dy, s, mean, rstd, g, up)
    for a, w in zip((ds, dg, db), want):
        torch.testing.assert_close(a, w, rtol=1e-10, atol=1e-10)
    assert torch.equal(dx, ds)
    z = torch.linspace(-9, 9, 400, dtype=torch.float64)
    torch.testing.assert_close(ref.act(z, "gelu"), torch.nn.functional.gelu(z), rtol=1e-9, atol=1e-12)
    torch.testing.assert_close(ref.act(z, "gelu_tanh"), torch.nn.functional.gelu(z, approximate="tanh"), rtol=1e-9, atol=1e-12)


def test_plain_and_reference_masks_agree():
    """The mask is the generator's words against floor(p 2^32), row by row, whatever the width."""
    a, b = ref.kept(5, 10, 0.3, 7, 9), ref.kept(5, 64, 0.3, 7, 9)
    assert torch.equal(a, b[:, :10])
    assert torch.equal(ref.kept([4], 10, 0.3, 7, 9), a[4:])
    assert abs(float(ref.kept(400, 400, 0.3, 7, 9).double().mean()) - 0.7) < 6 * np.sqrt(0.21 / 160000)


def test_descriptions_check_what_the_calls_check(lib):
    buf = ctypes.create_string_buffer(64)
    for fn, cls, base, bad in (("fff_describe_grouped_matmul", ops.FffGroupedMatmulArgs, PRODUCT, dict(k=0)),
                               ("fff_describe_grouped_weight_grad", ops.FffGroupedWeightGradArgs, GRAD, dict(dw=P))):
        call = getattr(lib, fn)
        assert call(None, buf, len(buf)) == INVALID
        a = _fill(cls, base, bad)
        assert call(ctypes.addressof(a), buf, len(buf)) == INVALID
        a = _fill(cls, base, dict(n_entries=0, accumulate=1) if "dw" in base else dict(n_entries=0))
        assert call(ctypes.addressof(a), buf, len(buf)) == OK and buf.value == b"none"
        assert call(ctypes.addressof(a), None, 0) == OK
    assert lib.fff_last_hip_error() == 0


@pytest.mark.parametrize("call", [
    lambda: fff.layer_norm_backward_workspace_bytes(4, (1 << 32) + 8),
    lambda: fff.group_rows_workspace_bytes(100000, (1 << 32) + 16), lambda: fff.group_rows_workspace_bytes(100000, 16, 1 << 32 | 1),
    lambda: fff.grouped_weight_grad_workspace_bytes(100000, (1 << 32) + 1, 64, 64),
    lambda: fff.grouped_weight_grad_workspace_bytes(100000, 1, (1 << 32) + 64, 64),
    lambda: fff.grouped_weight_grad_workspace_bytes(100000, 1, 64, -(1 << 32) + 64)])
def test_sizes_past_32_bits_are_refused(lib, call):
    """ctypes would hand on their low 32 bits."""
    with pytest.raises(ValueError):
        call()

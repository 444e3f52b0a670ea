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

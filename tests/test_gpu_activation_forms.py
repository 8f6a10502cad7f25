"""An activation and its slope are the same values whatever call computes them: few rows, tiles, parts of a split sum, the activation's gradient alone."""
import math

import pytest
import torch

import paper_2608_15211_b200 as terra
from tests._block import act, act_slope, held

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16
VALUES = [0.0, -0.0, 1e-3, -1e-3, 0.7, -0.7, 3.0, -3.0, 8.0, -8.0, 12.5, -12.5, 40.0, -40.0, 90.0, -90.0, 200.0, -200.0, 6e4, -6e4, math.inf, -math.inf, math.nan, 1.0]


def same(a, b):
    return torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(0.0, posinf=1.0, neginf=-1.0), b.nan_to_num(0.0, posinf=1.0, neginf=-1.0)) \
        and torch.equal(a.isinf(), b.isinf())


@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("activation", ["relu", "silu", "gelu", "gelu_tanh"])
def test_values_far_out_and_infinities(activation, dtype):
    z = torch.tensor(VALUES, device="cuda")
    n = len(VALUES)
    # x = 0, so that the bias is z itself: few rows, tiles of one CTA and of two, a sum in parts
    outs = [terra.terra_linear_fwd(torch.zeros(rows, n_in, device="cuda", dtype=dtype), torch.zeros(n, n_in, device="cuda", dtype=dtype), bias=z, activation=activation)[0]
            for rows, n_in in ((1, 64), (8, 72), (16, 64), (300, 64), (40, 8192))]
    assert all(same(o, outs[0][:1].expand_as(o)) for o in outs)
    finite = z.isfinite()
    ref = act(z.double(), activation)[finite]
    held(activation, outs[0][0][finite], ref, ref.abs() * 1.2e-5 + 2.0 ** -120, dtype)       # (the tail's polynomial is 9e-6 off; silu(-90) is 0)
    at = outs[0][0]
    assert at[n - 4] == math.inf and at[n - 2].isnan()
    assert at[n - 3] == 0 if activation in ("relu", "gelu") else at[n - 3].isnan()


@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("activation", ["relu", "silu", "gelu", "gelu_tanh"])
def test_slopes_far_out_and_infinities(activation, dtype):
    z = torch.tensor(VALUES, device="cuda").to(dtype)
    n = len(VALUES)
    for rows in (1, 300):
        z_in, one = z.expand(rows, n).contiguous(), torch.ones(rows, n, device="cuda", dtype=dtype)
        alone = terra.terra_activation_bwd(z_in, one, activation)
        dx, _, _ = terra.terra_linear_bwd(z_in, torch.eye(n, device="cuda", dtype=dtype), one, z_in=z_in, activation=activation, need_dw=False, need_dbias=False)
        tail = terra.terra_activation_bwd(z_in.flatten()[:n - 1].contiguous(), one.flatten()[:n - 1].contiguous(), activation)      # the last ones by themselves
        assert same(dx, alone) and same(alone, alone[:1].expand_as(alone)) and same(tail, alone[0, :n - 1])
    finite = z.isfinite()
    held("slope", alone[0][finite], act_slope(z.double(), activation)[finite], 2e-5, dtype)
    assert alone[0, n - 4] == 1 and alone[0, n - 3] == 0 and (activation == "relu" or alone[0, n - 2].isnan())

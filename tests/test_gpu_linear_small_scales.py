"""Products of 8-bit operands whose scales' product lies below fp32's normal numbers while the result does not."""
import pytest
import torch

import paper_2608_15211_b200 as terra
from tests._block import EPS32, held

pytestmark = pytest.mark.gpu


# few rows; tiles of one CTA and of two; a sum in parts
@pytest.mark.parametrize("rows,n_in,n_out", [(4, 1024, 96), (100, 1024, 4096), (600, 1024, 512), (40, 16384, 64)])
def test_the_scales_are_not_multiplied_first(rows, n_in, n_out):
    g = torch.Generator(device="cuda").manual_seed(rows)
    x, w = (torch.randint(200, 449, s, generator=g, device="cuda").float().to(torch.float8_e4m3fn) for s in ((rows, n_in), (n_out, n_in)))
    xs = torch.full((rows,), 1.37 * 2.0 ** -100, device="cuda")
    ws = (torch.rand(n_out, generator=g, device="cuda") + 1) * 2.0 ** -46          # the product of the two has 3 bits left in fp32
    ref = (x.double() @ w.double().t()) * xs.double()[:, None] * ws.double()
    assert ref.min() > 2.0 ** -126
    y = terra.terra_linear_fwd_e4m3(x, xs, w, ws, dtype=torch.bfloat16)
    held("y", y, ref, ref * (256 + 32) * 2 * EPS32, torch.bfloat16)

"""The 8-bit norm hands the backward call what it needs."""
import pytest
import torch

import paper_2608_15211_b200 as terra
from paper_2608_15211_b200.build import build


@pytest.mark.gpu
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("rows,channels,dtype", [(1, 8, torch.bfloat16), (300, 96, torch.float16), (77, 1001, torch.bfloat16), (33, 16384, torch.bfloat16)])
def test_the_eight_bit_norm_can_be_differentiated(rows, channels, dtype, residual):
    g = torch.Generator(device="cuda").manual_seed(rows)
    n = lambda: torch.randn(rows, channels, generator=g, device="cuda").to(dtype)
    x, r, dy, w = n(), n() if residual else None, n(), 1 + 0.1 * torch.randn(channels, generator=g, device="cuda")
    _, h, want = terra.terra_rms_norm_fwd(x, w, residual=r)
    rstd = torch.full((rows,), -7.0, device="cuda")
    y, scale, h8 = terra.terra_rms_norm_fwd_e4m3(x, w, residual=r, rstd=rstd)
    assert torch.equal(rstd, want) and torch.equal(h8, h)           # the same sums in the same order
    plain = terra.terra_rms_norm_fwd_e4m3(x, w, residual=r)
    assert torch.equal(plain[0].view(torch.uint8), y.view(torch.uint8)) and torch.equal(plain[1], scale)
    for got, ref in zip(terra.terra_rms_norm_bwd(h8, w, rstd, dy), terra.terra_rms_norm_bwd(h, w, want, dy)):
        assert torch.equal(got, ref)


def test_refusals():
    build()
    x, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.ones(64)
    for bad in (torch.ones(3), torch.ones(4, dtype=torch.float64)):
        with pytest.raises(ValueError, match="rstd must be torch.float32 with 4 elements"):
            terra.terra_rms_norm_fwd_e4m3(x, w, rstd=bad)
    with pytest.raises(ValueError, match="CUDA tensors"):
        terra.terra_rms_norm_fwd_e4m3(x, w, rstd=torch.ones(4))

"""Rows quantised to 8-bit integers: 127 x / max rounded to the nearest whole number, ties to the even one, by every kernel that does it and whatever the row's scale."""
import zlib

import pytest
import torch

import paper_2608_15211_b200 as terra

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


def nearest(x):
    """127 x / max of the row to the nearest whole number, and where that is a tie.  In 64 bits 127 |x|, its remainder and what is left of it are exact: a
    remainder is shorter than its operands, and x has 11 bits at most."""
    a = 127 * x.double().abs()
    most = x.double().abs().amax(1, keepdim=True).clamp(min=2.0 ** -200)           # (a row of zeros keeps them)
    rest = torch.fmod(a, most)
    q = (a - rest) / most
    tie = 2 * rest == most
    q = q + ((2 * rest > most) | (tie & (q % 2 == 1)))
    return torch.where(x < 0, -q, q).to(torch.int8), tie


# channels: vectors of 8 in one and in several a thread, one to a warp and to a block; 2 and 1 at a time; rows longer than a block holds, by 8 and by 1
CHANNELS = [(700, 8), (300, 96), (64, 2048), (32, 4096), (9, 16384), (301, 130), (77, 1001), (40, 6001), (12, 16400), (7, 16385), (5, 65535)]


@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("rows,channels", CHANNELS)
def test_ties_go_to_even(rows, channels, dtype):
    g = torch.Generator(device="cuda").manual_seed(zlib.crc32(repr((rows, channels)).encode()))
    x = torch.randn(rows, channels, generator=g, device="cuda").to(dtype)
    # 127 X / M of whole numbers is a tie where X = M / 2, whatever M is, and for M = 127 k (a scale of k, in bf16 a power of two) where X is an odd multiple of k / 2
    x[0::3, 1::3] = x[0::3].abs().amax(1, keepdim=True) / 2 * (torch.randint(0, 2, x[0::3, 1::3].shape, generator=g, device="cuda") * 2 - 1).to(dtype)
    k = 2 * torch.randint(1, 9, (len(x[1::3]), 1), generator=g, device="cuda") if dtype == F16 else 2 ** torch.randint(1, 9, (len(x[1::3]), 1), generator=g, device="cuda")
    x[1::3] = (k // 2 * torch.randint(-253, 254, x[1::3].shape, generator=g, device="cuda")).to(dtype)
    x[1::3, channels // 2] = (127 * k[:, 0]).to(dtype)
    q, scale = terra.terra_quantize_i8(x)
    want, tie = nearest(x)
    assert tie.sum() > rows * channels // 8 and (want[tie] % 2 == 0).all()
    assert torch.equal(q, want)
    assert torch.equal(scale, x.float().abs().amax(1).double().div(127).float())


@pytest.mark.parametrize("channels", [96, 1001, 16400, 16385])
@pytest.mark.parametrize("exponent", [-133, -127, -120, -101, -99, -61, -59, 59, 61, 99, 101, 120, 124])
def test_scales_far_out(exponent, channels):
    # bf16's whole range: values of 16 steps either way of which the largest is 2^exponent times 15, rounded as the type has them
    g = torch.Generator(device="cuda").manual_seed(channels)
    x = torch.randint(-15, 16, (64, channels), generator=g, device="cuda").double()
    x[:, 3] = torch.randint(1, 16, (64,), generator=g, device="cuda").double()
    x[::4] *= x[::4].abs() <= x[::4, 3:4].abs()        # (rows whose largest value is another one each)
    x = (x * 2.0 ** exponent).to(BF16)
    x[0] = 0
    assert x.isfinite().all() and (x[1:].abs().amax(1) > 0).all()
    q, scale = terra.terra_quantize_i8(x)
    want, tie = nearest(x)
    assert tie.any() and torch.equal(q, want) and scale[0] == 0

"""The group norm at the ends of its sizes."""
import pytest
import torch

import paper_2608_15211_b200 as terra
import tests.test_gpu_group_norm as cases
from tests.test_gpu_group_norm import check_forward

pytestmark = pytest.mark.gpu


def test_more_than_2_31_groups():
    # 65535 samples of 32769 groups: more than a grid's first dimension takes
    samples, channels = 65535, 32769
    assert samples * channels > 2 ** 31
    x = torch.empty(samples, 2, channels, device="cuda", dtype=torch.bfloat16).normal_()
    w, b = 1 + 0.1 * torch.randn(channels, device="cuda"), torch.randn(channels, device="cuda")
    ends = [slice(0, 2), slice(32766, 32768), slice(samples - 2, samples)]
    parts = [x[s].clone() for s in ends]
    y, stats = terra.terra_group_norm_fwd(x, w, b, channels, activation="silu", y=x)
    for s, part in zip(ends, parts):
        check_forward(part, w, b, channels, 1e-5, "silu", y[s], stats[s])
    assert stats[..., 1].min() > 0
    del x, y, stats, parts
    torch.cuda.empty_cache()           # 50 GB


# samples in shared memory: at a time by smaller clusters, in two turns, nearly all of an SM's, a group to a channel
@pytest.mark.parametrize("samples,tokens,channels,groups", [(16, 280, 960, 4), (64, 371, 256, 1), (100, 1720, 96, 2), (32, 88, 1784, 2), (2, 2804, 1904, 1904), (100, 64, 1264, 4), (3, 4189, 640, 32)])
def test_samples_in_shared_memory(samples, tokens, channels, groups):
    cases.test_forward(samples, tokens, channels, groups, torch.bfloat16)
    cases.test_backward(samples, tokens, channels, groups, torch.float16)


@pytest.mark.parametrize("tokens", [40, 3000, 50000])
def test_sums_of_squares_beyond_the_range(tokens):
    # deviations of 2^63: four of their squares are more than fp32 holds; of 2^53 in the next group 2^22 of them would be
    x = torch.zeros(1, tokens, 16, device="cuda", dtype=torch.bfloat16)
    x[:, 0::2, :8], x[:, 1::2, :8] = 2.0 ** 63, -2.0 ** 63
    x[:, 0::2, 8:], x[:, 1::2, 8:] = 2.0 ** 53, -2.0 ** 53
    w, b = torch.ones(16, device="cuda"), torch.linspace(-1, 1, 16, device="cuda")
    y, stats = terra.terra_group_norm_fwd(x, w, b, 2)
    assert stats[0, 0, 1] == 0 and torch.equal(y[0, :, :8], b[:8].to(torch.bfloat16).expand(tokens, 8))
    # means of 0 within the joinings' roundings of values of that size
    assert stats[0, 0, 0].abs() <= 2.0 ** 63 * 64 * 2.0 ** -24 and stats[0, 1, 0].abs() <= 2.0 ** 53 * 64 * 2.0 ** -24
    assert abs(stats[0, 1, 1].item() * 2.0 ** 53 - 1) <= 2.0 ** -17

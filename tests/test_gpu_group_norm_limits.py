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

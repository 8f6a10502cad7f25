"""The group norm at the ends of its sizes."""
import pytest
import torch

import paper_2608_15211_b200 as terra
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

"""The group norm where the deviations are far from 1: statistics up to rstd = 1e19 and down to 1e-19, against the formulas in 64 bits."""
import zlib

import pytest
import torch

import paper_2608_15211_b200 as terra
from tests._block import EPS32, act_slope, held
from tests.test_gpu_group_norm import check_forward, moments, per_channel
from tests.test_gpu_gated import fenced

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16

# samples that clusters hold in registers and in shared memory, three launches; vectors of 8, 2 and 1 channels
SHAPES = [(2, 2048, 96, 8), (2, 4096, 640, 32), (1, 60001, 64, 16), (3, 4000, 130, 5), (3, 9, 1001, 7), (1, 9000, 31, 1), (2, 6, 64, 32)]


def make(samples, tokens, channels, exponent):
    g = torch.Generator(device="cuda").manual_seed(zlib.crc32(repr((samples, tokens, channels)).encode()))
    n = lambda *s: torch.randn(s, generator=g, device="cuda")
    x = (n(samples, tokens, channels) + n(samples, 1, channels)).double() * 2.0 ** exponent
    return x.to(BF16), 1 + 0.1 * n(channels), 0.3 * n(channels), n(samples, tokens, channels)


@pytest.mark.parametrize("exponent", [-63, -47, -43, -20, 20, 43, 53, 62])
@pytest.mark.parametrize("samples,tokens,channels,groups", SHAPES)
def test_backward(samples, tokens, channels, groups, exponent):
    x, w, b, dy = make(samples, tokens, channels, exponent)
    v, mean, var, rstd = moments(x, groups, 0.0)
    # an upstream gradient that goes along with n: the mean of their product is about 8, no rounding's rest
    dy = (dy + 8 * ((v - mean) * rstd).flatten(2)).to(BF16)
    stats = torch.stack((mean[:, 0, :, 0], rstd[:, 0, :, 0]), -1).float()
    assert stats.isfinite().all() and (exponent > -63 or stats[..., 1].max() > 5e18)
    dx, ok = fenced(x.shape, BF16)
    got = terra.terra_group_norm_bwd(x, w, b, stats, dy, activation="silu", d_x=dx)
    assert ok() and got[0].data_ptr() == dx.data_ptr()
    # the formula with the given mean and rstd; the bounds are those of values about 1, relative to rstd
    mean, rstd = (per_channel(stats[:, None, :, None, i].double(), channels) for i in (0, 1))
    n = (x.double() - mean) * rstd
    z = n * w.double() + b.double()
    off_z = (n * w.double()).abs() * 4 * EPS32 + (z.abs() + b.double().abs()) * 2 * EPS32 + (w.double() * rstd).abs() * mean.abs() * EPS32
    g = dy.double() * act_slope(z, "silu")
    off_g = dy.double().abs() * (off_z * 1.1 + 2e-5 + 2 * EPS32)
    many = 64 * EPS32                  # of a sum: chains of up to 2^12 terms in a thread, then pairwise; of their magnitudes' sum
    held("d_bias", got[2], g.sum((0, 1)), off_g.sum((0, 1)) + g.abs().sum((0, 1)) * many, torch.float32)
    held("d_weight", got[1], (g * n).sum((0, 1)), (off_g * n.abs()).sum((0, 1)) + (g * n).abs().sum((0, 1)) * many, torch.float32)
    group = lambda t: per_channel(t.unflatten(2, (groups, -1)).mean((1, 3), keepdim=True), channels)
    gw, off_gw = g * w.double(), off_g * w.double().abs()
    level, along = group(gw), group(gw * n)
    ref = rstd * (gw - level - n * along)
    mags = gw.abs() + group(gw.abs()) + n.abs() * group((gw * n).abs())
    off = rstd * (off_gw + group(off_gw) + n.abs() * group(off_gw * n.abs()) + mags * (many + 6 * EPS32) + off_z * along.abs() * 4)
    # (of a result in fp32 and its terms below the normal numbers some steps of 2^-149 are lost)
    held("d_x", dx, ref, off + 2.0 ** -146, BF16)


@pytest.mark.parametrize("exponent", [-47, -43, 43, 50])
@pytest.mark.parametrize("samples,tokens,channels,groups", SHAPES)
def test_forward(samples, tokens, channels, groups, exponent):
    # (at 2^50 the largest of these groups' squared deviations add up to 2^100 x 960016)
    x, w, b, _ = make(samples, tokens, channels, exponent)
    y, stats = terra.terra_group_norm_fwd(x, w, b, groups, eps=0.0, activation="silu")
    check_forward(x, w, b, groups, 0.0, "silu", y, stats)

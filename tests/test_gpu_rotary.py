"""Rotary positions of queries and keys against the formula in 64 bits."""
import pytest
import torch

import paper_2608_15211_b200 as terra
from paper_2608_15211_b200.workloads import small_config
from tests._block import frequencies, grid_positions, held, rotate

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16
# the reduced angle (up to pi) rounded to fp32, cos and sin to two units, two products and a sum: below 2^-20 of |a| + |b|
REL = 2.0 ** -20


def inputs(cfg, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + cfg.H * cfg.W)
    shape = (cfg.B, cfg.H, cfg.W, cfg.heads, cfg.head_dim)
    return [torch.randn(shape, generator=g, device="cuda").to(dtype) for _ in range(3)]


def wanted(cfg, x, freq, row_pairs, layout, scale, inverse, positions=None):
    pos = (grid_positions(cfg) if positions is None else positions.reshape(-1, 2).cpu()).double()
    by_row = torch.arange(len(freq)) < row_pairs
    angle = torch.where(by_row, pos[:, :1], pos[:, 1:]) * freq * (-1 if inverse else 1)
    x64 = x.double().cpu().reshape(-1, cfg.heads, cfg.head_dim)
    size = rotate(x64.abs(), torch.full_like(angle, 0.25 * torch.pi), layout, 2 ** 0.5 * abs(scale))     # second of a pair: (|a| + |b|) scale
    pairs = len(freq)
    first, second = (slice(0, pairs), slice(pairs, 2 * pairs)) if layout == "half" else (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2))
    size[..., first] = size[..., second].clone()
    size[..., 2 * pairs:] = 0
    return rotate(x64, angle, layout, scale).reshape(x.shape), size.reshape(x.shape)


CASES = [  # B, H, W, heads, d, shift_h, shift_w, rot, row_pairs, dtype
    (1, 1, 1, 1, 32, 0, 0, 32, 0, BF16), (2, 5, 7, 3, 32, 2, 3, 32, 8, BF16), (1, 13, 9, 2, 64, 4, 4, 32, 8, F16), (1, 3, 70, 5, 128, 0, 8, 128, 32, BF16),
    (1, 6, 11, 2, 32, 1, 2, 20, 5, BF16), (1, 6, 11, 2, 64, 1, 2, 22, 11, F16), (1, 4, 5, 1, 128, 0, 0, 126, 1, BF16), (1, 9, 9, 2, 32, 0, 0, 2, 1, BF16),
    (1, 2, 3, 131, 32, 1, 1, 32, 8, BF16), (1, 3, 5, 3, 128, 1, 1, 110, 20, BF16), (1, 3, 5, 2, 64, 0, 1, 36, 18, F16), (2, 3, 4, 2, 32, 1, 0, 6, 1, BF16), (3, 40, 30, 6, 32, 4, 4, 16, 4, F16), (1, 1, 700, 4, 64, 0, 0, 48, 0, BF16),
]


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c[:9])))
def test_turns(case, layout):
    B, H, W, heads, d, sh, sw, rot, row_pairs, dtype = case
    cfg = small_config("rot", B, H, W, heads, d, 8, sh, sw)
    q, k, v = inputs(cfg, dtype)
    freq = frequencies(rot, row_pairs)
    desc = terra.make_desc(cfg, dtype=dtype)
    for scale, inverse in ((1.0, False), (1.25, True)):
        qo, ko = terra.terra_rotary(desc, q, k, freq.cuda(), row_pairs=row_pairs, layout=layout, scale=scale, inverse=inverse)
        for name, got, x in (("q", qo, q), ("k", ko, k)):
            ref, size = wanted(cfg, x, freq, row_pairs, layout, scale, inverse)
            held(name, got.cpu(), ref, size * REL, dtype)
            assert torch.equal(got[..., rot:], x[..., rot:])
        # alone, in place, and in place on the packed tensor: the same bits
        assert torch.equal(terra.terra_rotary(desc, q, None, freq.cuda(), row_pairs=row_pairs, layout=layout, scale=scale, inverse=inverse)[0], qo)
        q2, k2 = q.clone(), k.clone()
        terra.terra_rotary(desc, q2, k2, freq.cuda(), row_pairs=row_pairs, layout=layout, scale=scale, inverse=inverse, q_out=q2, k_out=k2)
        assert torch.equal(q2, qo) and torch.equal(k2, ko)
        packed = torch.stack((q, k, v), 3).contiguous()
        assert terra.terra_rotary_packed(desc, packed, freq.cuda(), row_pairs=row_pairs, layout=layout, scale=scale, inverse=inverse).data_ptr() == packed.data_ptr()
        assert torch.equal(packed, torch.stack((qo, ko, v), 3))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_given_positions_far_from_the_origin(layout):
    cfg = small_config("far", 3, 1, 17, 2, 64, 8, 0, 0)
    q, k, _ = inputs(cfg, BF16, 5)
    pos = torch.randint(-(2 ** 31), 2 ** 31 - 1, (3, 1, 17, 2), dtype=torch.int32)
    pos[0, 0, 0] = torch.tensor([2 ** 31 - 1, -(2 ** 31)])
    freq = frequencies(64, 16)
    qo, ko = terra.terra_rotary(terra.make_desc(cfg), q, k, freq.cuda(), row_pairs=16, layout=layout, positions=pos.cuda())
    for got, x in ((qo, q), (ko, k)):
        ref, size = wanted(cfg, x, freq, 16, layout, 1.0, False, pos)
        held("far", got.cpu(), ref, size * (REL + 2.0 ** 31 * 2.0 ** -52), BF16)


def test_back_and_forth_and_the_gradient():
    cfg = small_config("grad", 1, 5, 6, 2, 32, 8, 2, 1)
    q, k, g = inputs(cfg, F16, 9)
    freq = frequencies(32, 8).cuda()
    desc = terra.make_desc(cfg, dtype=F16)
    turn = lambda x, inverse: terra.terra_rotary(desc, x, None, freq, row_pairs=8, inverse=inverse)[0]
    back = turn(turn(q, False), True)
    assert (back.double() - q.double()).abs().max() <= 4 * 2.0 ** -11 * q.double().abs().max()
    # <turn(q), g> = <q, turn back(g)>: the transpose is the inverse
    a, b = (turn(q, False).double() * g.double()).sum(), (q.double() * turn(g, True).double()).sum()
    assert abs(a - b) <= 2 * 2.0 ** -11 * (q.double().abs() * g.double().abs()).sum() * 2


def test_only_position_differences_matter_to_scores_inside_a_window():
    # tokens of the window over the longitude seam: the scores are those of the same tokens on the unrolled grid
    cfg = small_config("seam", 1, 4, 16, 1, 32, 8, 0, 4)
    q, k, _ = inputs(cfg, F16, 3)
    freq = frequencies(32, 8).cuda()
    qo, ko = terra.terra_rotary(terra.make_desc(cfg, dtype=F16), q, k, freq, row_pairs=8)
    cols = [(v + 4) % 16 for v in range(8, 16)]                     # window 1 of the shifted frame
    plain = small_config("plain", 1, 4, 8, 1, 32, 8, 0, 0)
    qp, kp = terra.terra_rotary(terra.make_desc(plain, dtype=F16), q[:, :, cols].contiguous(), k[:, :, cols].contiguous(), freq, row_pairs=8)
    s = torch.einsum("uvd,xyd->uvxy", qo[0][:, cols, 0].double(), ko[0][:, cols, 0].double())
    p = torch.einsum("uvd,xyd->uvxy", qp[0, :, :, 0].double(), kp[0, :, :, 0].double())
    bound = 4 * 2.0 ** -11 * torch.einsum("uvd,xyd->uvxy", qp[0, :, :, 0].double().abs(), kp[0, :, :, 0].double().abs()).max() * 2
    assert (s - p).abs().max() <= bound

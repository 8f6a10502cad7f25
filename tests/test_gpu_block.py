"""A whole pre-norm Transformer block of the library's calls, forward and backward, and its 8-bit serving form, against the formulas in 64 bits."""
import math

import pytest
import torch

import paper_2608_15211_b200 as terra
from paper_2608_15211_b200.workloads import small_config
from tests._block import act, frequencies, grid_positions, rotate
from tests._brute import rolled_geometry

pytestmark = pytest.mark.gpu
EPS, ROW_PAIRS = 1e-6, 8


def parameters(cfg, hidden, dtype):
    g = torch.Generator().manual_seed(cfg.H * cfg.W)
    C = cfg.heads * cfg.head_dim
    n = lambda *s: torch.randn(s, generator=g)
    p = {"n1": 1 + 0.1 * n(C), "n2": 1 + 0.1 * n(C), "bias": 0.1 * n((2 * cfg.window - 1) ** 2, cfg.heads)}
    for name, a, b in (("qkv", C, 3 * C), ("o", C, C), ("up", C, hidden), ("down", hidden, C)):
        p["w_" + name], p["b_" + name] = (n(b, a) / math.sqrt(a)).to(dtype), 0.1 * n(b)
    x, d = n(cfg.B, cfg.H, cfg.W, C).to(dtype), n(cfg.B, cfg.H, cfg.W, C).to(dtype)
    return {k: v.cuda() for k, v in p.items()}, x.cuda(), d.cuda()


def forward(cfg, desc, freq, p, x):
    C = cfg.heads * cfg.head_dim
    s = {}
    s["y1"], _, s["r1"] = terra.terra_rms_norm_fwd(x, p["n1"], eps=EPS)
    qkv, _ = terra.terra_linear_fwd(s["y1"], p["w_qkv"], bias=p["b_qkv"])
    s["qkv"] = terra.terra_rotary_packed(desc, qkv.view(cfg.B, cfg.H, cfg.W, 3, cfg.heads, cfg.head_dim), freq, row_pairs=ROW_PAIRS)
    s["o"], s["lse"] = terra.terra_swin_attn_fwd_packed(desc, s["qkv"], p["bias"])
    branch, _ = terra.terra_linear_fwd(s["o"].view(cfg.B, cfg.H, cfg.W, C), p["w_o"], bias=p["b_o"])
    s["y2"], s["h"], s["r2"] = terra.terra_rms_norm_fwd(branch, p["n2"], residual=x, eps=EPS)
    s["a"], s["z"] = terra.terra_linear_fwd(s["y2"], p["w_up"], bias=p["b_up"], activation="gelu", keep_z=True)
    out, _ = terra.terra_linear_fwd(s["a"], p["w_down"], bias=p["b_down"], residual=s["h"])
    return out, s


def backward(cfg, desc, freq, p, x, s, d):
    C = cfg.heads * cfg.head_dim
    g = {}
    dz, g["w_down"], g["b_down"] = terra.terra_linear_bwd(s["a"], p["w_down"], d, z_in=s["z"], activation="gelu")
    dy2, g["w_up"], g["b_up"] = terra.terra_linear_bwd(s["y2"], p["w_up"], dz)
    dh, g["n2"] = terra.terra_rms_norm_bwd(s["h"], p["n2"], s["r2"], dy2, d_h=d)
    o = s["o"].view(cfg.B, cfg.H, cfg.W, C)
    do, g["w_o"], g["b_o"] = terra.terra_linear_bwd(o, p["w_o"], dh)
    dqkv, g["bias"] = terra.terra_swin_attn_bwd_packed(desc, s["qkv"], p["bias"], s["o"], s["lse"], do.view_as(s["o"]))
    terra.terra_rotary_packed(desc, dqkv, freq, row_pairs=ROW_PAIRS, inverse=True)
    dy1, g["w_qkv"], g["b_qkv"] = terra.terra_linear_bwd(s["y1"], p["w_qkv"], dqkv.view(cfg.B, cfg.H, cfg.W, 3 * C))
    g["x"], g["n1"] = terra.terra_rms_norm_bwd(x, p["n1"], s["r1"], dy1, d_h=dh)
    return g


def formula(cfg, freq, p, x):
    """The block in fp64, with attention over all tokens under the windows' membership mask."""
    C, N = cfg.heads * cfg.head_dim, cfg.H * cfg.W
    norm = lambda h, w: h * (h.square().mean(-1, keepdim=True) + EPS).rsqrt() * w
    y1 = norm(x, p["n1"])
    qkv = (y1 @ p["w_qkv"].t() + p["b_qkv"]).view(cfg.B, N, 3, cfg.heads, cfg.head_dim)
    pos = grid_positions(cfg)[:N].double()
    angle = torch.where(torch.arange(len(freq)) < ROW_PAIRS, pos[:, :1], pos[:, 1:]) * freq
    win, lab, a, b = (torch.from_numpy(t).reshape(-1) for t in rolled_geometry(cfg.H, cfg.W, cfg.window, cfg.shift_h, cfg.shift_w, cfg.periodic_h, cfg.periodic_w))
    allowed = (win[:, None] == win) & (lab[:, None] == lab)
    w = cfg.window
    row = ((a[:, None] - a + w - 1) * (2 * w - 1) + b[:, None] - b + w - 1).clamp(0, (2 * w - 1) ** 2 - 1)
    outs = []
    for i in range(cfg.B):
        q, k = (rotate(qkv[i, :, j], angle, "half", 1.0) for j in (0, 1))
        s = torch.einsum("nhd,mhd->hnm", q, k) / math.sqrt(cfg.head_dim) + p["bias"][row].permute(2, 0, 1)
        outs.append(torch.einsum("hnm,mhd->nhd", s.masked_fill(~allowed, -math.inf).softmax(-1), qkv[i, :, 2]).reshape(cfg.H, cfg.W, C))
    h = torch.stack(outs) @ p["w_o"].t() + p["b_o"] + x
    y2 = norm(h, p["n2"])
    return act(y2 @ p["w_up"].t() + p["b_up"], "gelu") @ p["w_down"].t() + p["b_down"] + h


# A path through the block has at most 12 tensors that are rounded to 16 bits, each by half a step of each value at most; their contributions to a
# result's 2-norm add up to less than 12 half steps of it, and as much again for sums in which larger terms cancel
@pytest.mark.parametrize("case,dtype", [(("block_w8", 2, 12, 20, 2, 32, 8, 4, 4, 0, 1), torch.bfloat16), (("block_w16", 1, 20, 24, 2, 64, 16, 8, 8, 0, 1), torch.float16)],
                         ids=["w8_bf16", "w16_fp16"])
def test_block(case, dtype):
    cfg = small_config(*case)
    p, x, d = parameters(cfg, 176, dtype)
    freq = frequencies(cfg.head_dim, ROW_PAIRS)
    desc = terra.make_desc(cfg, dtype=dtype)
    out, saved = forward(cfg, desc, freq.cuda(), p, x)
    got = backward(cfg, desc, freq.cuda(), p, x, saved, d)
    terra.terra_swin_check()
    leaves = {k: v.double().cpu().requires_grad_() for k, v in {**p, "x": x}.items()}
    ref = formula(cfg, freq, leaves, leaves["x"])
    grads = dict(zip(leaves, torch.autograd.grad(ref, list(leaves.values()), d.double().cpu())))
    bound = 24 * (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -11)
    off = lambda a, b: ((a.double().cpu() - b).norm() / b.norm()).item()
    assert off(out, ref.detach()) <= bound
    for name, g in grads.items():
        assert off(got[name].reshape(g.shape), g) <= bound, name


def test_block_served_in_eight_bits():
    cfg = small_config("block8", 1, 12, 20, 2, 64, 8, 4, 4, 0, 1)
    p, x, _ = parameters(cfg, 256, torch.bfloat16)
    quantised = {}
    for name in ("w_qkv", "w_up"):
        scale = p[name].float().abs().amax(1) / 448
        quantised[name] = ((p[name].float() / scale[:, None]).to(torch.float8_e4m3fn), scale)
    y1, s1, h1 = terra.terra_rms_norm_fwd_e4m3(x, p["n1"], eps=EPS)
    qkv = terra.terra_linear_fwd_e4m3(y1, s1, *quantised["w_qkv"], bias=p["b_qkv"])
    y2, s2, h2 = terra.terra_rms_norm_fwd_e4m3(x, p["n2"], residual=x, eps=EPS)
    up = terra.terra_linear_fwd_e4m3(y2, s2, *quantised["w_up"], bias=p["b_up"], activation="gelu")
    assert h1.data_ptr() == x.data_ptr() and h2.data_ptr() != x.data_ptr()
    for got, name, h, n, a in ((qkv, "qkv", x, "n1", "none"), (up, "up", 2 * x.double(), "n2", "gelu")):
        h = h.double()
        y = h * (h.square().mean(-1, keepdim=True) + EPS).rsqrt() * p[n].double()
        ref = act(y @ p["w_" + name].double().t() + p["b_" + name].double(), a)
        # either operand is off by at most 2^-4 of each value: sqrt(2) 2^-4 of the product's 2-norm were they in phase; the bias and gelu add nothing
        assert (got.double() - ref).norm() <= 2 ** 0.5 * 2.0 ** -4 * ref.norm()

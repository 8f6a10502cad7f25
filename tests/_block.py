"""The operators around the attention written out in 64 bits, and the bounds that the kernels' results are held to."""
import math

import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}      # half the smallest subnormal step
EPS32 = 2.0 ** -24


def held(name, got, ref, extra, dtype):
    """|got - ref| <= a rounding to `dtype` + extra (the error before it, which the rounding may enlarge by its own share)."""
    assert got.dtype == dtype, (name, got.dtype)
    assert tuple(got.shape) == tuple(ref.shape), (name, got.shape, ref.shape)
    got, extra = got.double(), extra if torch.is_tensor(extra) else torch.full_like(ref, extra)
    allowed = (ref.abs() + extra) * HALF_STEP[dtype] + extra + TINY[dtype]
    off = (got - ref).abs()
    bad = ~(off <= allowed)
    assert not bad.any(), (f"{name}: {int(bad.sum())} of {bad.numel()} off, first at {bad.nonzero()[0].tolist()}: got {got[bad][0].item()!r}, "
                           f"want {ref[bad][0].item()!r} +- {allowed[bad][0].item():.3g}")


def act(z, name):
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))          # slope 0 at 0
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu":
        return 0.5 * z * torch.erfc(-z * math.sqrt(0.5))
    if name == "gelu_tanh":
        return z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
    return z


def act_slope(z, name):
    z = z.detach().clone().requires_grad_()
    return torch.autograd.grad(act(z, name).sum(), z)[0] if name != "none" else torch.ones_like(z)


def frequencies(rot, row_pairs, base=10000.0):
    out = []
    for n in (row_pairs, rot // 2 - row_pairs):
        out += [base ** (-i / n) for i in range(n)]
    return torch.tensor(out, dtype=torch.float64)


def rotate(x, angle, layout, scale):
    """x [tokens, heads, d], angle [tokens, pairs], all fp64."""
    pairs = angle.shape[1]
    y = x.clone()
    for p in range(pairs):
        i, j = (p, p + pairs) if layout == "half" else (2 * p, 2 * p + 1)
        c, s = angle[:, p, None].cos() * scale, angle[:, p, None].sin() * scale
        y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., i] * s + x[..., j] * c
    return y


def grid_positions(cfg):
    """[tokens, 2] row and column in the shifted frame."""
    u = (torch.arange(cfg.H) - cfg.shift_h) % cfg.H
    v = (torch.arange(cfg.W) - cfg.shift_w) % cfg.W
    return torch.stack((u[:, None].expand(cfg.H, cfg.W), v[None].expand(cfg.H, cfg.W)), -1).reshape(1, -1, 2).expand(cfg.B, -1, 2).reshape(-1, 2)

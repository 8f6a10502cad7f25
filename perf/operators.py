"""Performance cases of what stands around the window attention in a Transformer block: the root-mean-square norm with the
residual's addition, the product with bias, activation and residual, and the rotary positions of queries and keys.

A case is one call as a block makes it on a token grid: `rows` tokens of `channels` (norm), `rows` tokens from `n_in` to `n_out`
features (linear), or the queries and keys of the grid of a descriptor (rotary).  The listed sizes are the repository's own
configurations (`workloads.CONFIGS`) and the patch products of the paper's 93 variables; `draw` gives more of the same ranges.

`own` false computes the operators from elementary torch operations in 32 bits (angles in 64), rounded once at the end.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
_E4M3 = torch.float8_e4m3fn
_E4M3_MAX = 448.0
_EPS = 1e-6


def _norm(name, call, rows, channels, dtype="bf16", residual=True):
    out = {} if name is None else {"name": name}
    out.update(op="norm", call=call, rows=rows, channels=channels, dtype=dtype, residual=residual)
    return out


def _linear(name, call, rows, n_in, n_out, dtype="bf16", activation="none", residual=False, keep_z=False):
    out = {} if name is None else {"name": name}
    out.update(op="linear", call=call, rows=rows, n_in=n_in, n_out=n_out, dtype=dtype, activation=activation, residual=residual,
               keep_z=keep_z)
    return out


def _rotary(name, B, H, W, heads, head_dim, rot, shift, layout, axial, far=False, scale=1.0, inverse=False, dtype="bf16"):
    out = {} if name is None else {"name": name}
    out.update(op="rotary", B=B, H=H, W=W, heads=heads, head_dim=head_dim, rot=rot, shift=shift, layout=layout, axial=axial, far=far,
               scale=scale, inverse=inverse, dtype=dtype)
    return out


def listed():
    return [
        # the norm before the attention of a small forecaster that answers a request: launch and latency
        _norm("norm_cfg1", "forward", 32 * 64, 3 * 32),
        # inference of the medium model: the residual stream is added up and the next product's operand comes out in 8 bits
        _norm("norm_e4m3_tv_medium", "e4m3", 288 * 544, 32 * 128),
        # a training step with 32 x 32 windows at head dim 64: the norm's backward, joined with the residual stream's gradient
        _norm("norm_backward_cfg4", "backward", 256 * 512, 12 * 64),
        # a shallow stage with 8 x 8 windows, positions by latitude and longitude
        _rotary("rotary_cfg2", 1, 128, 256, 6, 32, 32, 4, "half", True),
        # the medium model's queries and keys, half of each head turned, frequencies stretched for a longer range
        _rotary("rotary_tv_medium", 1, 288, 544, 32, 128, 64, 4, "interleaved", True, scale=1.1),
        # the conditioning vector (lead time) of two rollout samples: all weights for two rows
        _linear("linear_two_rows", "forward", 2, 4096, 8192, dtype="fp16", activation="silu"),
        # patch recovery of 93 variables x 2 x 2 points on the fine grid: rows of 744 bytes come out
        _linear("linear_patch_out", "forward", 1020 * 2160, 256, 372, dtype="fp16"),
        # training on the global grid at patch 4: the widening product keeps what its activation is taken of
        _linear("linear_cfg3_up", "forward", 510 * 1080, 384, 1536, activation="gelu", keep_z=True),
        # the medium model's output projection onto the residual stream
        _linear("linear_tv_medium_out", "forward", 288 * 544, 4096, 4096, residual=True),
        # inference of the medium model in 8 bits: the widening product
        _linear("linear_e4m3_tv_medium_up", "e4m3", 288 * 544, 4096, 16384, activation="gelu"),
        # training on a shallow stage: the narrowing product's gradients, through the activation before it
        _linear("linear_backward_cfg2", "backward", 128 * 256, 768, 192, dtype="fp16", activation="gelu_tanh"),
        # the small model's narrowing product, backward
        _linear("linear_backward_tv_small", "backward", 288 * 544, 4096, 1024, activation="gelu"),
    ]


def _log_int(rng, low, high):
    return max(low, min(high, round(math.exp(rng.uniform(math.log(low), math.log(high))))))


def draw(rng):
    """Another call of these ranges: 1 to 10^6 tokens, 32 to 8192 channels in heads of 32, 64 and 128 or, one time in four, any number."""
    while True:
        dtype = rng.choice(["bf16", "bf16", "fp16"])
        rows = _log_int(rng, 1, 1000000)

        def features():
            if rng.random() < 0.25:
                return _log_int(rng, 8, 4096)
            width = rng.choice([32, 64, 128])
            return width * _log_int(rng, 1, 8192 // width)

        op = rng.choice(["norm", "rotary", "linear", "linear"])
        if op == "norm":
            case = _norm(None, rng.choice(["forward", "e4m3", "backward"]), rows, features(), dtype, rng.random() < 0.7)
        elif op == "rotary":
            head_dim = rng.choice([32, 64, 128])
            B = rng.choice([1, 1, 2])
            H = rng.choice([1, _log_int(rng, 1, 1000)])
            W = max(1, rows // (B * H))
            case = _rotary(None, B, H, W, _log_int(rng, 1, 4096 // head_dim), head_dim, rng.choice([head_dim, head_dim // 2, 2 * rng.randint(1, head_dim // 2)]),
                           rng.choice([0, 4, 16]), rng.choice(["half", "interleaved"]), rng.random() < 0.6, rng.random() < 0.3,
                           rng.choice([1.0, 1.2]), rng.random() < 0.4, dtype)
        else:
            call = rng.choice(["forward", "forward", "e4m3", "backward", "backward"])
            n_in, n_out = features(), features()
            if call == "e4m3":
                n_in = max(16, n_in // 16 * 16)
            case = _linear(None, call, rows, n_in, n_out, dtype, rng.choice(["none", "relu", "silu", "gelu", "gelu_tanh"]),
                           call != "backward" and rng.random() < 0.4, call == "forward" and rng.random() < 0.4)
        cost = work(case)
        if cost["flops"] <= 6e12 and cost["bytes"] <= 6e9:       # a fraction of the largest listed ones
            return case


def prepare(case, seed):
    """Activations N(0, 1) with a few channels ten times as wide, as residual streams have them; weights N(0, 1 / n_in)."""
    c = SimpleNamespace(**case)
    dtype = _DTYPES[c.dtype]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape, dtype=dtype):
        return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)

    s = SimpleNamespace(**case)
    if c.op == "norm":
        s.x = normal(c.rows, c.channels)
        s.x[:, ::37] *= 10
        s.weight = 1 + 0.1 * normal(c.channels, dtype=torch.float32)
        s.r = normal(c.rows, c.channels) if c.residual else None
        if c.call == "backward":
            s.d_y = normal(c.rows, c.channels)
            s.rstd = torch.rsqrt(s.x.float().square().mean(1) + _EPS)
    elif c.op == "rotary":
        from paper_2608_15211_b200 import make_desc
        s.desc = make_desc(SimpleNamespace(B=c.B, H=c.H, W=c.W, heads=c.heads, head_dim=c.head_dim, window=8, shift_h=c.shift, shift_w=c.shift,
                                           periodic_h=0, periodic_w=1), dtype=dtype)
        shape = (c.B, c.H, c.W, c.heads, c.head_dim)
        s.q, s.k = normal(*shape), normal(*shape)
        pairs = c.rot // 2
        s.row_pairs = pairs // 2 if c.axial else 0
        p = torch.arange(pairs, device="cuda", dtype=torch.float64)
        own_axis = torch.where(p < s.row_pairs, p, p - s.row_pairs)
        length = torch.where(p < s.row_pairs, s.row_pairs, pairs - s.row_pairs)
        s.inv_freq = 10000.0 ** (-own_axis / length)
        s.positions = None
        if c.far:                     # positions as a program counts them, up to ten million steps from the origin
            s.positions = torch.randint(0, 10000000, (c.B, c.H, c.W, 2), generator=gen, device="cuda", dtype=torch.int32)
    else:
        s.bias = 0.1 * normal(c.n_out, dtype=torch.float32)
        w = normal(c.n_out, c.n_in, dtype=torch.float32) / math.sqrt(c.n_in)
        s.r = normal(c.rows, c.n_out) if c.residual else None
        if c.call == "e4m3":
            x = normal(c.rows, c.n_in)
            s.x_scale = (x.abs().amax(1).float() / _E4M3_MAX).clamp(min=1e-12)
            s.x = (x / s.x_scale[:, None].to(dtype)).clamp(-_E4M3_MAX, _E4M3_MAX).to(_E4M3)
            s.w_scale = w.abs().amax(1) / _E4M3_MAX
            s.w = (w / s.w_scale[:, None]).clamp(-_E4M3_MAX, _E4M3_MAX).to(_E4M3)
        else:
            s.x, s.w = normal(c.rows, c.n_in), w.to(dtype)
        if c.call == "backward":
            s.d_z = normal(c.rows, c.n_out)
            s.z_in = None if c.activation == "none" else normal(c.rows, c.n_in)
    return s


def _cdf(z):
    return 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))


def _tanh_argument(z):
    return math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)


def _act(z, name):
    if name == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "gelu":
        return z * _cdf(z)
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(_tanh_argument(z)))
    return z


def _act_slope(z, name):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "silu":
        sig = 1 / (1 + torch.exp(-z))
        return sig * (1 + z * (1 - sig))
    if name == "gelu":
        return _cdf(z) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        t = torch.tanh(_tanh_argument(z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def _norm_plain(s):
    dtype = _DTYPES[s.dtype]
    if s.call == "backward":
        h, g = s.x.float(), s.d_y.float()
        n = h * s.rstd[:, None]
        gw = g * s.weight
        dx = s.rstd[:, None] * (gw - n * (gw * n).mean(1, keepdim=True))
        if s.r is not None:
            dx = dx + s.r.float()
        return dx.to(dtype), (g * n).sum(0)
    h = s.x.float()
    if s.r is not None:
        h = h + s.r.float()
    rstd = torch.rsqrt(h.square().mean(1) + _EPS)
    y = h * rstd[:, None] * s.weight
    if s.call == "forward":
        return y.to(dtype), h.to(dtype), rstd
    scale = y.abs().amax(1) / _E4M3_MAX
    return (y / torch.where(scale > 0, scale, torch.ones_like(scale))[:, None]).to(_E4M3), scale, h.to(dtype)


def _positions(s, wide=torch.float64):
    """Row and column positions [B, H, W] of the grid's tokens in the frame that the windows tile."""
    if s.positions is not None:
        return s.positions[..., 0].to(wide), s.positions[..., 1].to(wide)
    u = (torch.arange(s.H, device="cuda") - s.shift) % s.H
    v = (torch.arange(s.W, device="cuda") - s.shift) % s.W
    return u.to(wide)[None, :, None].expand(s.B, s.H, s.W), v.to(wide)[None, None, :].expand(s.B, s.H, s.W)


def _rotary_plain(s, wide=torch.float32):
    dtype = _DTYPES[s.dtype]
    pairs = s.rot // 2
    u, v = _positions(s)
    by_row = torch.arange(pairs, device="cuda") < s.row_pairs
    angle = torch.where(by_row, u[..., None], v[..., None]) * s.inv_freq
    cos, sin = (angle.cos() * s.scale).to(wide)[..., None, :], (angle.sin() * s.scale).to(wide)[..., None, :]
    if s.inverse:
        sin = -sin

    def turn(x):
        x = x.to(wide)
        head, rest = x[..., : s.rot], x[..., s.rot:]
        if s.layout == "half":
            a, b = head[..., :pairs], head[..., pairs:]
            turned = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
        else:
            a, b = head[..., 0::2], head[..., 1::2]
            turned = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
        return torch.cat((turned, rest), -1)

    q, k = turn(s.q), turn(s.k)
    return (q.to(dtype), k.to(dtype)) if wide is torch.float32 else (q, k)


def _linear_plain(s):
    dtype = _DTYPES[s.dtype]
    if s.call == "backward":
        g, w = s.d_z.float(), s.w.float()
        dx = g @ w
        if s.z_in is not None:
            dx = dx * _act_slope(s.z_in.float(), s.activation)
        return dx.to(dtype), g.t() @ s.x.float(), g.sum(0)
    z = s.x.float() @ s.w.float().t()
    if s.call == "e4m3":
        z = z * s.x_scale[:, None] * s.w_scale
    z = z + s.bias
    y = _act(z, s.activation)
    if s.r is not None:
        y = y + s.r.float()
    return (y.to(dtype), z.to(dtype)) if s.keep_z else y.to(dtype)


def run(s):
    if not own:
        return {"norm": _norm_plain, "rotary": _rotary_plain, "linear": _linear_plain}[s.op](s)
    import paper_2608_15211_b200 as terra
    if s.op == "norm":
        if s.call == "backward":
            return terra.terra_rms_norm_bwd(s.x, s.weight, s.rstd, s.d_y, d_h=s.r)
        if s.call == "forward":
            return terra.terra_rms_norm_fwd(s.x, s.weight, residual=s.r, eps=_EPS)
        return terra.terra_rms_norm_fwd_e4m3(s.x, s.weight, residual=s.r, eps=_EPS)
    if s.op == "rotary":
        return terra.terra_rotary(s.desc, s.q, s.k, s.inv_freq, row_pairs=s.row_pairs, layout=s.layout, scale=s.scale, positions=s.positions,
                                  inverse=s.inverse)
    if s.call == "backward":
        return terra.terra_linear_bwd(s.x, s.w, s.d_z, z_in=s.z_in, activation=s.activation)
    if s.call == "e4m3":
        return terra.terra_linear_fwd_e4m3(s.x, s.x_scale, s.w, s.w_scale, bias=s.bias, residual=s.r, activation=s.activation, dtype=_DTYPES[s.dtype])
    y, z = terra.terra_linear_fwd(s.x, s.w, bias=s.bias, residual=s.r, activation=s.activation, keep_z=s.keep_z)
    return (y, z) if s.keep_z else y


def work(case):
    """Each input read once and each output written once; a product's 2 rows n_in n_out operations, twice that backward."""
    c = SimpleNamespace(**case)
    if c.op == "norm":
        n = c.rows * c.channels
        if c.call == "backward":
            return {"bytes": 2 * n * (3 + c.residual) + 4 * c.rows + 8 * c.channels, "flops": 9 * n}
        return {"bytes": n * (2 + 4 * c.residual + (2 if c.call == "forward" else 1)) + 4 * c.rows + 4 * c.channels, "flops": 5 * n}
    if c.op == "rotary":
        tokens = c.B * c.H * c.W
        n = 2 * tokens * c.heads
        return {"bytes": 4 * n * c.head_dim + 8 * tokens * c.far + 4 * c.rot, "flops": 3 * n * c.rot}
    product = 2 * c.rows * c.n_in * c.n_out
    weights = c.n_in * c.n_out
    if c.call == "backward":
        return {"bytes": 2 * c.rows * (2 * c.n_in + c.n_out + c.n_in * (c.activation != "none")) + 6 * weights + 4 * c.n_out, "flops": 2 * product}
    if c.call == "e4m3":
        return {"bytes": c.rows * (c.n_in + 2 * c.n_out * (1 + c.residual) + 4) + weights + 8 * c.n_out, "flops": product}
    return {"bytes": 2 * c.rows * (c.n_in + c.n_out * (1 + c.residual + c.keep_z)) + 2 * weights + 4 * c.n_out, "flops": product}


def exact(case, seed):
    s = prepare(case, seed)
    if s.op == "norm":
        x, w = s.x.double(), s.weight.double()
        r = s.r.double() if s.r is not None else 0.0
        if s.call == "backward":
            d, g, rs = x.shape[1], s.d_y.double(), s.rstd.double().unsqueeze(1)
            along = torch.einsum("ij,j,ij->i", g, w, x).unsqueeze(1)
            return rs * g * w - x * rs ** 3 * along / d + r, torch.einsum("ij,ij,ik->j", g, x, rs)
        h = x + r
        length = (torch.einsum("ij,ij->i", h, h) / x.shape[1] + _EPS).sqrt()
        y = h / length.unsqueeze(1) * w
        if s.call == "forward":
            return y, h, 1 / length
        scale = torch.maximum(y.amax(1), -y.amin(1)) / _E4M3_MAX
        return y / scale.clamp(min=1e-300).unsqueeze(1), scale, h
    if s.op == "rotary":
        u, v = _positions(s)
        pairs = s.rot // 2
        angle = torch.cat((u[..., None] * s.inv_freq[: s.row_pairs], v[..., None] * s.inv_freq[s.row_pairs:]), -1)
        turn = torch.polar(torch.full_like(angle, s.scale), -angle if s.inverse else angle).unsqueeze(-2)
        out = []
        for x in (s.q, s.k):
            y = x.double()
            halves = (slice(0, pairs), slice(pairs, s.rot)) if s.layout == "half" else (slice(0, s.rot, 2), slice(1, s.rot, 2))
            z = torch.complex(y[..., halves[0]], y[..., halves[1]]) * turn
            y[..., halves[0]], y[..., halves[1]] = z.real, z.imag
            out.append(y)
        return tuple(out)
    if s.call == "backward":
        g = s.d_z.double()
        dx = torch.einsum("mo,oi->mi", g, s.w.double())
        if s.z_in is not None:
            z = s.z_in.double().requires_grad_()
            dx = torch.autograd.grad(_act64(z, s.activation), z, dx)[0]
        return dx, torch.einsum("mo,mi->oi", g, s.x.double()), g.sum(0)
    x, w = s.x.double(), s.w.double()
    if s.call == "e4m3":
        x, w = x * s.x_scale.double().unsqueeze(1), w * s.w_scale.double().unsqueeze(1)
    z = torch.addmm(s.bias.double(), x, w.t())
    del x, w
    y = _act64(z, s.activation)
    if s.r is not None:
        y = y + s.r
    return (y, z) if s.keep_z else y


def _act64(z, name):
    f = torch.nn.functional
    return {"none": lambda t: t, "relu": f.relu, "silu": f.silu, "gelu": f.gelu, "gelu_tanh": lambda t: f.gelu(t, approximate="tanh")}[name](z)

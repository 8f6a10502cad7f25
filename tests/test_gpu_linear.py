"""The products with bias, activation and residual, in 16 and 8 bits, and their backward, against the formulas in 64 bits."""
import zlib

import pytest
import torch

import paper_2608_15211_b200 as terra
from tests._block import EPS32, act, act_slope, held

pytestmark = pytest.mark.gpu
BF16, F16, E4M3 = torch.bfloat16, torch.float16, torch.float8_e4m3fn
ACTS = ["none", "relu", "silu", "gelu", "gelu_tanh"]

# rows, n_in, n_out: one row, fewer than a tile, tiles and a bit, features that are no multiple of 8 (padded rows) or of 4 (rows of odd bytes), long sums
SHAPES = [(1, 64, 32), (1, 8, 8), (3, 13, 5), (7, 46, 70), (8, 8192, 24), (9, 72, 40), (17, 96, 288), (128, 64, 128), (129, 200, 100), (256, 64, 256), (300, 384, 130), (513, 72, 372), (257, 1024, 514),
          (1000, 33, 31), (2048, 96, 96), (2, 4096, 1024), (5, 2048, 40), (700, 256, 744), (1500, 520, 1)]


def ints(g, *shape, dtype=BF16):
    return torch.randint(-2, 3, shape, generator=g, device="cuda").to(dtype)


def gen(*key):
    return torch.Generator(device="cuda").manual_seed(zlib.crc32(repr(key).encode()))


@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("rows,n_in,n_out", SHAPES)
def test_whole_numbers_are_exact(rows, n_in, n_out, dtype):
    # every partial sum is a whole number below 2^24, so the order does not matter and only the last rounding is left
    g = gen(rows, n_in, n_out)
    x, w, r, dz = ints(g, rows, n_in, dtype=dtype), ints(g, n_out, n_in, dtype=dtype), ints(g, rows, n_out, dtype=dtype), ints(g, rows, n_out, dtype=dtype)
    b = ints(g, n_out, dtype=torch.float32)
    z64 = x.double() @ w.double().t()
    y, z = terra.terra_linear_fwd(x, w)
    assert z is None and torch.equal(y, z64.to(dtype))
    y, z = terra.terra_linear_fwd(x, w, bias=b, residual=r, activation="relu", keep_z=True)
    assert torch.equal(z, (z64 + b).to(dtype)) and torch.equal(y, ((z64 + b).clamp(min=0) + r).to(dtype))
    dx, dw, db = terra.terra_linear_bwd(x, w, dz)
    assert torch.equal(dx, (dz.double() @ w.double()).to(dtype))
    assert torch.equal(dw, (dz.double().t() @ x.double()).float()) and torch.equal(db, dz.double().sum(0).float())
    # single outputs are the same bits
    for i, only in enumerate(("need_dx", "need_dw", "need_dbias")):
        one = terra.terra_linear_bwd(x, w, dz, **{n: n == only for n in ("need_dx", "need_dw", "need_dbias")})
        assert torch.equal(one[i], (dx, dw, db)[i]) and [t is None for t in one] == [j != i for j in range(3)]
    x8, w8 = x.to(E4M3), w.to(E4M3)
    xs, ws = 2.0 ** torch.randint(-3, 4, (rows,), generator=g, device="cuda").float(), 2.0 ** torch.randint(-3, 4, (n_out,), generator=g, device="cuda").float()
    y = terra.terra_linear_fwd_e4m3(x8, xs, w8, ws, bias=b, residual=r, activation="relu", dtype=dtype)
    assert torch.equal(y, ((z64 * xs.double()[:, None] * ws.double() + b).clamp(min=0) + r).to(dtype))


@pytest.mark.parametrize("activation", ACTS)
@pytest.mark.parametrize("rows,n_in,n_out,dtype", [(3, 40, 24, BF16), (300, 96, 384, BF16), (129, 33, 50, F16), (600, 256, 96, F16)])
def test_activations(rows, n_in, n_out, dtype, activation):
    g = gen(rows, activation)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")
    x, w, r, b = n(rows, n_in).to(dtype), (2 * n(n_out, n_in) / n_in ** 0.5).to(dtype), n(rows, n_out).to(dtype), 0.3 * n(n_out)
    z64 = x.double() @ w.double().t() + b.double()
    # truncated sums: each step of 16 may lose a unit of what is there
    off = (x.double().abs() @ w.double().abs().t()) * (n_in / 16 + 4) * 2 * EPS32 + b.double().abs() * EPS32
    y, z = terra.terra_linear_fwd(x, w, bias=b, residual=r, activation=activation, keep_z=True)
    held("z", z, z64, off, dtype)
    ref = act(z64, activation)
    # slopes are at most 1.13; the tail's polynomial is 9e-6 off, exp2 and the reciprocal 2^-21
    own = 0 if activation in ("none", "relu") else 1.2e-5
    held("y", y, ref + r.double(), 1.2 * off + ref.abs() * own + z64.abs() * 2.0 ** -21 + r.double().abs() * EPS32, dtype)
    # the gradient through the activation before the product
    dz, z_in = n(rows, n_out).to(dtype), (2 * n(rows, n_in)).to(dtype)
    h = act(z_in.double(), activation).to(dtype)
    dx, dw, db = terra.terra_linear_bwd(h, w, dz, z_in=z_in, activation=activation)
    slope = act_slope(z_in.double(), activation)
    plain = dz.double() @ w.double()
    off = (dz.double().abs() @ w.double().abs()) * (n_out / 16 + 4) * 2 * EPS32
    held("d_x", dx, plain * slope, 1.2 * off + plain.abs() * (2e-5 if own else 0), dtype)
    mag = dz.double().abs().t() @ h.double().abs()
    held("d_w", dw, dz.double().t() @ h.double(), mag * (rows / 16 + 4) * 2 * EPS32, torch.float32)
    held("d_bias", db, dz.double().sum(0), dz.double().abs().sum(0) * (rows / 8 + 16) * EPS32, torch.float32)
    if activation != "none":
        dy = n(rows, n_in).to(dtype)
        held("d_z", terra.terra_activation_bwd(z_in, dy, activation), dy.double() * slope, dy.double().abs() * (2e-5 if own else 0), dtype)


def test_activations_far_out():
    z = torch.tensor([0.0, -0.0, 1e-3, -1e-3, 3.0, -3.0, 8.0, -8.0, 40.0, -40.0, 200.0, -200.0, 6e4, -6e4, 3e38, -3e38], device="cuda").to(BF16)
    one, eye = torch.ones_like(z)[None], torch.eye(16, device="cuda", dtype=BF16)
    for activation in ACTS[1:]:
        y, _ = terra.terra_linear_fwd(z[None], eye, activation=activation)
        ref = act(z.double(), activation)
        held(activation, y[0], ref, ref.abs() * 1.2e-5 + 2.0 ** -120, BF16)
        held("slope " + activation, terra.terra_activation_bwd(z[None], one, activation)[0], act_slope(z.double().clamp(-1e3, 1e3), activation), 2e-5, BF16)
        nan = terra.terra_linear_fwd(torch.full((1, 16), float("nan"), device="cuda", dtype=BF16), eye, activation=activation)[0]
        assert nan.isnan().all()


def test_eight_bit_operands():
    g = gen("e4m3")
    n = lambda *s: torch.randn(s, generator=g, device="cuda")
    x, w = n(300, 400), n(200, 400)
    xs, ws = x.abs().amax(1) / 448, w.abs().amax(1) / 448
    x8, w8 = (x / xs[:, None]).to(E4M3), (w / ws[:, None]).to(E4M3)
    y = terra.terra_linear_fwd_e4m3(x8, xs, w8, ws, activation="gelu", dtype=F16)
    a, b = x8.double() * xs.double()[:, None], w8.double() * ws.double()[:, None]
    z = a @ b.t()
    off = (a.abs() @ b.abs().t()) * (400 / 32 + 6) * 2 * EPS32
    held("y", y, act(z, "gelu"), 1.2 * off + z.abs() * 1.2e-5, F16)


@pytest.mark.parametrize("n_in,n_out", [(72, 100), (128, 256), (256, 96), (1024, 320)])      # rows by the warps; by the copy engine, two tiles a warp and one
def test_rows_do_not_meet_and_given_buffers(n_in, n_out):
    g = gen("rows", n_in)
    x, w, r = ints(g, 300, n_in), ints(g, n_out, n_in), ints(g, 300, n_out)
    y, z = terra.terra_linear_fwd(x, w, residual=r, activation="gelu", keep_z=True)
    bad = x.clone()
    bad[17], bad[299, 3] = float("nan"), float("inf")
    yb, _ = terra.terra_linear_fwd(bad, w, residual=r, activation="gelu")
    rest = [i for i in range(300) if i not in (17, 299)]
    assert torch.equal(yb[rest], y[rest]) and yb[17].isnan().all()
    over = r.clone()
    y2, z2 = terra.terra_linear_fwd(x, w, residual=over, activation="gelu", y=over, z=torch.empty_like(r))
    assert y2.data_ptr() == over.data_ptr() and torch.equal(over, y) and torch.equal(z2, z)
    dz, z_in = ints(g, 300, n_out), ints(g, 300, n_in)
    dx, dw, db = terra.terra_linear_bwd(x, w, dz, z_in=z_in, activation="silu")
    over = z_in.clone()
    ws = torch.empty(terra.terra_linear_workspace_bytes(300, n_in, n_out, "bwd"), dtype=torch.uint8, device="cuda")
    got = terra.terra_linear_bwd(x, w, dz, z_in=over, activation="silu", d_x=over, d_w=torch.empty_like(dw), d_bias=torch.empty_like(db), workspace=ws)
    assert got[0].data_ptr() == over.data_ptr() and all(torch.equal(a, b) for a, b in zip(got, (dx, dw, db)))


def test_leading_dimensions():
    g = gen("grid")
    x, w = ints(g, 2, 3, 5, 64), ints(g, 96, 64)
    y, z = terra.terra_linear_fwd(x, w, keep_z=True)
    assert y.shape == z.shape == (2, 3, 5, 96) and torch.equal(y.reshape(30, 96), terra.terra_linear_fwd(x.reshape(30, 64), w)[0])


def test_long_sum_over_rows():
    # the weight gradient over 70001 rows stays near fp32's own rounding
    g = gen("long")
    x, dz = torch.randn(70001, 40, generator=g, device="cuda").to(BF16), torch.randn(70001, 72, generator=g, device="cuda").to(BF16)
    w = torch.zeros(72, 40, device="cuda", dtype=BF16)
    _, dw, db = terra.terra_linear_bwd(x, w, dz, need_dx=False)
    want = dz.double().t() @ x.double()
    assert (dw.double() - want).norm() <= 4e-6 * want.norm()
    assert (db.double() - dz.double().sum(0)).norm() <= 1e-6 * dz.double().sum(0).norm()


@pytest.mark.parametrize("n", [1, 7, 8, 9, 2047, 2048, 2049, 2055, 16 * 148 * 2048 + 13])       # a last vector that is not whole, one block and a bit, every block twice
def test_an_activation_alone(n):
    g = gen("alone", n)
    z, dy = (torch.randn(n, generator=g, device="cuda").to(BF16) for _ in range(2))
    mem = torch.full((n + 16,), -7.0, device="cuda", dtype=BF16)
    d_z = mem[8:8 + n]
    assert terra.terra_activation_bwd(z, dy, "silu", d_z=d_z) is d_z
    held("d_z", d_z, dy.double() * act_slope(z.double(), "silu"), dy.double().abs() * 2e-5, BF16)
    assert (mem[:8] == -7).all() and (mem[8 + n:] == -7).all()
    terra.terra_activation_bwd(z, dy, "silu", d_z=dy)       # over the gradient
    assert torch.equal(dy, d_z)


@pytest.mark.parametrize("e4m3", [False, True], ids=["16", "e4m3"])
@pytest.mark.parametrize("rows,n_in,n_out", [(1, 16384, 64), (3, 4096, 372), (6, 1000, 5001), (2, 40, 65536), (4, 4094, 300), (5, 4095, 257), (8, 1, 1), (7, 2052, 17), (8, 8192, 1030)])
def test_few_rows_are_exact_and_do_not_meet(rows, n_in, n_out, e4m3):
    g = gen("few", rows, n_in, e4m3)
    x, w, r = ints(g, rows, n_in), ints(g, n_out, n_in), ints(g, rows, n_out, dtype=F16)
    b = torch.randint(-4, 5, (n_out,), generator=g, device="cuda").float()
    mem = torch.full((rows * n_out + 16,), -7.0, device="cuda", dtype=F16)
    y = mem[8:8 + rows * n_out].view(rows, n_out)

    def call(x, r):
        if not e4m3:
            return terra.terra_linear_fwd(x.to(F16), w.to(F16), bias=b, residual=r, activation="relu", y=y)[0]
        xs = torch.full((rows,), 2.0, device="cuda")
        return terra.terra_linear_fwd_e4m3((x / 2).to(E4M3), xs, w.to(E4M3), torch.ones(n_out, device="cuda"), bias=b, residual=r, activation="relu", dtype=F16, y=y)

    # whole numbers (halves, in 8 bits): the sums are exact, only the last rounding is left
    ref = torch.relu(x.double() @ w.double().t() + b.double()) + r.double()
    held("y", call(x, r), ref, 0, F16)
    assert (mem[:8] == -7).all() and (mem[8 + rows * n_out:] == -7).all()
    first = y.clone()
    if rows > 1:                                       # a row of NaN stays with itself
        bad = x.clone()
        bad[-1] = float("nan")
        call(bad, r)
        assert torch.equal(y[:-1], first[:-1]) and y[-1].isnan().all()
    w[-1] = float("nan")                               # and an output's weights with that output
    call(x, r)
    assert torch.equal(y[:, :-1], first[:, :-1]) and y[:, -1].isnan().all()

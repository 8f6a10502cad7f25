"""Root-mean-square norm with the residual's addition, its 8-bit output and its backward, against the formulas in 64 bits."""
import pytest
import torch

import paper_2608_15211_b200 as terra
from tests._block import EPS32, held

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16
# A row's sum of squares: at most 32 values in a thread, 5 + 31 additions over threads, then a quotient, a root and two products
REL = 2.0 ** -18

# rows, channels: one thread's vector, rows of 2 to 512 threads, odd channels (single elements), one row and odd numbers of rows
SHAPES = [(1, 8), (7, 1), (33, 96), (5, 13), (64, 128), (2048, 96), (129, 384), (70, 768), (9, 1024), (3, 1040), (5, 1001), (11, 4096), (2, 4097), (3, 8192), (2, 16384), (1, 16383), (37, 372), (6, 1860), (9, 2002), (4, 5000), (3, 8190), (2, 16380)]


def draw(rows, channels, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(100 * channels + rows + seed)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")
    x, r = n(rows, channels).to(dtype), n(rows, channels).to(dtype)
    x[:, ::7] *= 8
    return x, r, 1 + 0.2 * n(channels), n(rows, channels).to(dtype), n(rows, channels).to(dtype)


def formula(x, r, w, eps):
    h = x.double() + (r.double() if r is not None else 0)
    rstd = (h.square().mean(-1, keepdim=True) + eps).rsqrt()
    return h, rstd, h * rstd * w.double()


@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("rows,channels", SHAPES)
def test_forward(rows, channels, dtype):
    x, r, w, _, _ = draw(rows, channels, dtype)
    for res in (r, None):
        y, h, rstd = terra.terra_rms_norm_fwd(x, w, residual=res, eps=1e-5)
        rh, rr, ry = formula(x, res, w, 1e-5)
        held("h", h, rh, rh.abs() * EPS32, dtype)
        held("rstd", rstd, rr[:, 0], rr[:, 0] * REL, torch.float32)
        held("y", y, ry, ry.abs() * REL, dtype)
    assert h.data_ptr() == x.data_ptr()          # without a residual the sum is x


@pytest.mark.parametrize("rows,channels,dtype", [(1, 8, BF16), (33, 96, BF16), (129, 384, F16), (9, 1024, BF16), (5, 13, F16), (5, 1001, BF16), (11, 4096, BF16), (3, 8192, F16), (2, 16383, BF16)])
def test_eight_bits(rows, channels, dtype):
    x, r, w, _, _ = draw(rows, channels, dtype)
    if rows > 2:
        x[1] = 0
        r[1] = 0
    y, scale, h = terra.terra_rms_norm_fwd_e4m3(x, w, residual=r, eps=1e-5)
    rh, _, ry = formula(x, r, w, 1e-5)
    held("h", h, rh, rh.abs() * EPS32, dtype)
    top = ry.abs().amax(1)
    held("scale", scale, top / 448, top * REL, torch.float32)
    assert y.dtype == torch.float8_e4m3fn and y.shape == x.shape
    want = ry / torch.where(scale > 0, scale, 1.0).double()[:, None]
    # half a step: 2^-4 of the value, below 2^-6 the subnormals' 2^-10
    assert ((y.double() - want).abs() <= torch.maximum(want.abs() * 2.0 ** -4, torch.tensor(2.0 ** -10)) + want.abs() * REL).all()
    if rows > 2:
        assert scale[1] == 0 and not y[1].double().any()


@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("rows,channels", SHAPES + [(4500, 40), (3001, 104), (2500, 33)])
def test_backward(rows, channels, dtype):
    x, dh, w, dy, _ = draw(rows, channels, dtype, 1)
    rstd = (x.float().square().mean(1) + 1e-5).rsqrt()
    n, g, rs = x.double() * rstd.double()[:, None], dy.double() * w.double(), rstd.double()[:, None]
    want = rs * (g - n * (g * n).mean(1, keepdim=True))
    size = rs * (g.abs() + n.abs() * (g * n).abs().mean(1, keepdim=True))
    terms = dy.double() * n
    for d in (dh, None):
        dx, dw = terra.terra_rms_norm_bwd(x, w, rstd, dy, d_h=d)
        dd = d.double() if d is not None else torch.zeros_like(want)
        held("d_x", dx, want + dd, size * REL + dd.abs() * EPS32, dtype)
        # a chain of at most rows + 64 additions, each of which rounds what is there
        held("d_weight", dw, terms.sum(0), terms.abs().sum(0) * (rows + 64) * EPS32, torch.float32)


def test_gradients_are_those_of_the_forward():
    x, r, w, dy, _ = draw(3, 24, BF16, 2)
    x64, r64, w64 = (t.double().requires_grad_() for t in (x, r, w))
    h = x64 + r64
    y = h * (h.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * w64
    gx, gw = torch.autograd.grad((y * dy.double()).sum(), (x64, w64))
    _, h16, rstd = terra.terra_rms_norm_fwd(x, w, residual=r, eps=1e-5)
    dx, dw = terra.terra_rms_norm_bwd(h16, w, rstd, dy)
    # h is kept with 8 bits: each of its roundings moves n by half a step
    assert (dx.double() - gx).abs().max() <= 4 * 2.0 ** -8 * gx.abs().max()
    assert (dw.double() - gw).abs().max() <= 4 * 2.0 ** -8 * (dy.double() * y.detach()).abs().sum(0).max()


def test_outputs_over_inputs_and_given_buffers():
    x, r, w, dy, dh = draw(70, 192, BF16)
    y, h, rstd = terra.terra_rms_norm_fwd(x, w, residual=r)
    x2, r2 = x.clone(), r.clone()
    y2, h2, _ = terra.terra_rms_norm_fwd(x2, w, residual=r2, h=r2, y=x2)
    assert y2.data_ptr() == x2.data_ptr() and torch.equal(y2, y) and torch.equal(r2, h)
    plain, _, _ = terra.terra_rms_norm_fwd(x, w)
    x2 = x.clone()
    y2, h2, _ = terra.terra_rms_norm_fwd(x2, w, y=x2)
    assert torch.equal(y2, plain) and h2 is None             # the sum, x, is gone
    dx, dw = terra.terra_rms_norm_bwd(h, w, rstd, dy, d_h=dh)
    ws = torch.empty(terra.terra_rms_norm_workspace_bytes(70, 192), dtype=torch.uint8, device="cuda")
    for over in ("d_y", "d_h"):
        t = {"d_y": dy.clone(), "d_h": dh.clone()}
        dx2, dw2 = terra.terra_rms_norm_bwd(h, w, rstd, t["d_y"], d_h=t["d_h"], d_x=t[over], workspace=ws)
        assert dx2.data_ptr() == t[over].data_ptr() and torch.equal(dx2, dx) and torch.equal(dw2, dw)


def test_rows_that_are_no_numbers():
    x, r, w, _, _ = draw(6, 64, BF16)
    x[1, 5] = float("nan")
    x[2, 7] = float("inf")
    x[3] = 0
    y, _, rstd = terra.terra_rms_norm_fwd(x, w)
    good = [0, 4, 5]
    assert torch.equal(y[good], terra.terra_rms_norm_fwd(x[good].contiguous(), w)[0])       # rows do not meet
    assert y[1].isnan().all() and rstd[2] == 0 and y[2, 7].isnan() and not y[2, 8:].any() and not y[3].any()
    y8, scale, _ = terra.terra_rms_norm_fwd_e4m3(x, w)
    assert scale[1].isnan() and y8[1].double().isnan().all() and scale[3] == 0
    assert torch.equal(y8[good].view(torch.uint8), terra.terra_rms_norm_fwd_e4m3(x[good].contiguous(), w)[0].view(torch.uint8))


def test_tiny_rows_in_eight_bits():
    x = torch.full((2, 16), 1.0, dtype=BF16, device="cuda")
    w = torch.full((16,), 2.0 ** -126, device="cuda")
    w[3] = 2.0 ** -127
    y, scale, _ = terra.terra_rms_norm_fwd_e4m3(x, w, eps=0.0)
    want = w.double() / scale.double()[0]
    assert scale[0] > 0 and ((y[0].double() - want).abs() <= want * 2.0 ** -4).all()

"""Products whose sum over the features is long: exact on whole numbers by every way to memory, and, on data whose terms have one sign, as near to the formula
in 64 bits as a sum that leaves the matrix units every 128 steps is."""
import pytest
import torch

import paper_2608_15211_b200 as terra

pytestmark = pytest.mark.gpu
BF16, F16, E4M3 = torch.bfloat16, torch.float16, torch.float8_e4m3fn
STEPS = 128                            # in a row, at most: 32 stages of 4

# rows and outputs: tiles of two CTAs and of one, each whole and in parts, outputs by the copy engine and by the warps; the second sum ends inside 16 bytes
WAYS = [(2560, 2048), (2560, 2051), (100, 19200), (100, 19201), (300, 520), (300, 515), (100, 2000)]


def ints(g, *shape, dtype):
    return torch.randint(-2, 3, shape, generator=g, device="cuda").to(dtype)


def product(a, b):
    """a b' in 64 bits."""
    z = torch.zeros(a.shape[0], b.shape[0], dtype=torch.float64, device="cuda")
    for k in range(0, a.shape[1], 4096):
        z += a[:, k:k + 4096].double() @ b[:, k:k + 4096].double().t()
    return z


@pytest.mark.parametrize("length", [16512, 16507])
@pytest.mark.parametrize("rows,n", WAYS)
def test_whole_numbers_are_exact(rows, n, length):
    g = torch.Generator(device="cuda").manual_seed(rows + n + length)
    x, w, r, b = ints(g, rows, length, dtype=BF16), ints(g, n, length, dtype=BF16), ints(g, rows, n, dtype=BF16), ints(g, n, dtype=torch.float32)
    zz = product(x, w)
    y, z = terra.terra_linear_fwd(x, w, bias=b, residual=r, activation="relu", keep_z=True)
    assert torch.equal(z, (zz + b).to(BF16)) and torch.equal(y, ((zz + b).clamp(min=0) + r).to(BF16))
    y, _ = terra.terra_linear_fwd(x.to(F16), w.to(F16))
    assert torch.equal(y, zz.to(F16))
    xs, ws = torch.full((rows,), 0.5, device="cuda"), torch.full((n,), 4.0, device="cuda")
    y = terra.terra_linear_fwd_e4m3(x.to(E4M3), xs, w.to(E4M3), ws, bias=b, residual=r)
    assert torch.equal(y, (2 * zz + b + r).to(BF16))
    dx, _, _ = terra.terra_linear_bwd(r, w.t().contiguous(), x, z_in=r, activation="relu", need_dw=False, need_dbias=False)
    assert torch.equal(dx, (zz * (r > 0)).to(BF16))
    terra.terra_swin_check()


def held_before_the_rounding(call, z, allowed, dtype):
    """A residual of -round(z) leaves the sum's own error: what is left of it is rounded to a fraction of itself."""
    r = (-z).to(dtype)
    left = call(r).double()
    off = (left - r.double() - z).abs()
    assert (off <= allowed * z + left.abs() * 2.0 ** -8 + 2.0 ** -24).all(), (off / z).max().item()


# A step may cut off two units (2^-23) of the sum as it stands, which is half of the whole on average: 2^-23 of the whole a step.  What leaves the matrix
# units is added up in fp32, half a unit each: 32 times at most, and as many parts.
@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("rows,n,length", [(2560, 2048, 4096), (2560, 2048, 65536), (100, 19200, 16512), (300, 520, 65536), (2560, 2051, 8200)])
def test_terms_of_one_sign(rows, n, length, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows + n)
    x = torch.randn(rows, length, generator=g, device="cuda").abs().to(dtype)
    w = (torch.randn(n, length, generator=g, device="cuda").abs() / length ** 0.5).to(dtype)
    z = product(x, w)
    allowed = (STEPS + 32) * 2.0 ** -23
    held_before_the_rounding(lambda r: terra.terra_linear_fwd(x, w, residual=r)[0], z, allowed, dtype)
    # the input gradient has no residual: its mean error, in which the roundings (independent, half a step at most each) leave less than 2^-11 / sqrt(outputs)
    dx, _, _ = terra.terra_linear_bwd(torch.zeros(rows, n, dtype=dtype, device="cuda"), w.t().contiguous(), x, need_dw=False, need_dbias=False)
    noise = 4 * torch.finfo(dtype).eps / 2 / z.numel() ** 0.5
    assert abs((dx.double() - z).sum() / z.sum()) <= allowed + noise
    if dtype == F16:
        w8, x8 = (w * length ** 0.5).to(E4M3), x.to(E4M3)
        xs, ws = torch.ones(rows, device="cuda"), torch.full((n,), 2.0 ** -8, device="cuda")
        z = product(x8, w8) * 2.0 ** -8
        held_before_the_rounding(lambda r: terra.terra_linear_fwd_e4m3(x8, xs, w8, ws, residual=r, dtype=F16), z, allowed, F16)


# Few rows: 16 steps in a row, then 32 sums of a warp and those of 16 warps in fp32
@pytest.mark.parametrize("rows,n", [(1, 300), (8, 520)])
def test_terms_of_one_sign_few_rows(rows, n):
    g = torch.Generator(device="cuda").manual_seed(rows)
    x, w = torch.randn(rows, 65536, generator=g, device="cuda").abs().to(F16), (torch.randn(n, 65536, generator=g, device="cuda").abs() / 256).to(F16)
    allowed = (16 + 32 + 16) * 2.0 ** -23
    held_before_the_rounding(lambda r: terra.terra_linear_fwd(x, w, residual=r)[0], product(x, w), allowed, F16)
    x8, w8 = x.to(E4M3), (w * 256).to(E4M3)
    xs, ws = torch.ones(rows, device="cuda"), torch.full((n,), 2.0 ** -8, device="cuda")
    held_before_the_rounding(lambda r: terra.terra_linear_fwd_e4m3(x8, xs, w8, ws, residual=r, dtype=F16), product(x8, w8) * 2.0 ** -8, allowed, F16)

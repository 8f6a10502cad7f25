"""Products in 8-bit integers whose sums are split over the GPU: exact however large the parts are that cancel."""
import zlib

import pytest
import torch

import paper_2608_15211_b200 as terra

pytestmark = pytest.mark.gpu
BF16, F16, I8 = torch.bfloat16, torch.float16, torch.int8

# few tiles and long sums: outputs that are multiples of 4 and not, few and many parts, sums of padded rows; short ones beside them
SHAPES = [(40, 16384, 96), (40, 16384, 43), (300, 65536, 40), (130, 8192, 258), (33, 5000, 64), (9, 40001, 24), (1000, 32768, 12), (20, 640, 32)]


def cancelling(rows, n_in, n_out):
    """x [rows, n_in], w [n_out, n_in]: the second half of a sum is the first with the other sign but for one term, which is what is left: -254 .. 254."""
    g = torch.Generator(device="cuda").manual_seed(zlib.crc32(repr((rows, n_in, n_out)).encode()))
    i = lambda low, high, *s: torch.randint(low, high, s, generator=g, device="cuda")
    half = n_in // 2
    x, w = torch.zeros(rows, n_in, device="cuda", dtype=torch.int64), i(-127, 128, n_out, n_in)
    w[:, :half] = i(90, 128, n_out, half)              # parts of one sign: about 12000 a term
    x[:, :half] = i(90, 126, rows, half)
    w[:, half:2 * half], x[:, half:2 * half] = w[:, :half], -x[:, :half]
    left = i(0, half, rows)
    x[torch.arange(rows, device="cuda"), half + left] += i(0, 2, rows) * 3 - 2     # two less or one more
    d = x.double() @ w.double().t()
    assert d.abs().max() <= 254 and d.abs().min() > 0
    return x.to(I8), w.to(I8), d


@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("rows,n_in,n_out", SHAPES)
def test_product(rows, n_in, n_out, dtype):
    x, w, d = cancelling(rows, n_in, n_out)
    xs, ws = torch.ones(rows, device="cuda"), torch.ones(n_out, device="cuda")
    assert torch.equal(terra.terra_linear_fwd_i8(x, xs, w, ws, dtype=dtype), d.to(dtype))
    # the bias and the residual, and the same rows few at a time: the same bits
    b, r = torch.full((n_out,), 0.5, device="cuda"), torch.full((rows, n_out), -2.0, device="cuda", dtype=dtype)
    y = terra.terra_linear_fwd_i8(x, xs, w, ws, bias=b, residual=r, activation="relu", dtype=dtype)
    assert torch.equal(y, ((d + 0.5).clamp(min=0) - 2).to(dtype))
    assert torch.equal(terra.terra_linear_fwd_i8(x[:8], xs[:8], w, ws, bias=b, residual=r[:8], activation="relu", dtype=dtype), y[:8])


@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("rows,n_in,n_out", SHAPES)
def test_gated_product(rows, n_in, n_out, dtype):
    x, w, d = cancelling(rows, n_in, 2 * n_out)
    xs, ws = torch.full((rows,), 0.25, device="cuda"), torch.full((2 * n_out,), 0.5, device="cuda")
    y = terra.terra_gated_fwd_i8(x, xs, w, ws, activation="relu", dtype=dtype)
    assert torch.equal(y, (d[:, :n_out].clamp(min=0) * d[:, n_out:] / 64).to(dtype))       # (below 2^16 in whole numbers: exact in fp32)
    assert torch.equal(terra.terra_gated_fwd_i8(x[:8], xs[:8], w, ws, activation="relu", dtype=dtype), y[:8])

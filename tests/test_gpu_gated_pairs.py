"""Which gate row goes with which up row: weights that are not finite reach the outputs that the formula says, and no others."""
import pytest
import torch

import paper_2608_15211_b200 as terra

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.mark.parametrize("bad", [float("inf"), float("nan")], ids=["inf", "nan"])
@pytest.mark.parametrize("half", ["gate", "up"])
@pytest.mark.parametrize("rows,n_in,n_out", [(8, 96, 72), (300, 96, 72), (300, 64, 392), (130, 96, 51), (40, 4096, 72), (300, 2304, 200)])
def test_bad_rows_of_weights(rows, n_in, n_out, half, bad):
    g = torch.Generator(device="cuda").manual_seed(rows + n_out)
    ints = lambda *s: torch.randint(1, 3, s, generator=g, device="cuda") * (torch.randint(0, 2, s, generator=g, device="cuda") * 2 - 1)
    x, w = ints(rows, n_in).to(BF16), ints(2 * n_out, n_in).to(BF16)
    clean, _ = terra.terra_gated_fwd(x, w, activation="silu")
    at = [j for j in (0, 9, 33, 40, n_out - 1) if j < n_out]
    w[torch.tensor(at) + (n_out if half == "up" else 0), torch.arange(len(at)) + 5] = bad
    y, z = terra.terra_gated_fwd(x, w, activation="silu", keep_z=True)
    # an infinite weight of a value that is not 0 makes its sum infinite, of the value's sign
    z64 = x.double() @ w.double().t()
    gate, up = z64.chunk(2, 1)
    kind = lambda t: t.isnan() * 3 + t.isposinf() * 1 + t.isneginf() * 2
    assert (kind(z64)[:, torch.tensor(at) + (n_out if half == "up" else 0)] > 0).all() and torch.equal(kind(z), kind(z64))
    rest = [j for j in range(n_out) if j not in at]
    assert torch.equal(y[:, rest], clean[:, rest])
    ref = gate * torch.sigmoid(gate) * up              # silu(-inf) is -inf 0: NaN, as in the formula
    assert torch.equal(y[:, at].isfinite(), ref[:, at].isfinite())
    if half == "up":
        # a finite gate that is not 0: infinite, of the product's sign.  (Below -87 the gate's sigmoid is less than fp32's smallest normal number, e^-87 = 2^-125.5,
        # and silu of it may be 0 there: NaN.)
        sure = (gate[:, at] != 0) & (gate[:, at] > -87)
        assert sure.any()
        assert torch.equal(kind(y[:, at])[sure], kind(ref[:, at])[sure])

"""Products whose blocks work on several tiles each: two tiles of shared memory a warp in turn (short sums with a residual, a slope or a costly activation), the
residual of the next tile under way, columns of tiles that are partly empty; and the accuracy that the weight gradient leaves the matrix units early for."""
import pytest
import torch

import paper_2608_15211_b200 as terra
from tests._block import EPS32, act, act_slope, held
from tests._host_program import run_host_program

BF16, F16 = torch.bfloat16, torch.float16

# rows, n_in, n_out: 157 x 3 tiles of 256 x 256 for 74 pairs of SMs; a last row of tiles of 101 rows, a last column of 8 outputs; narrow tiles and sums of
# eight stages; sums of one; the same of the input gradient
FORWARD = [(40000, 256, 768), (40037, 128, 520), (60013, 512, 96), (30011, 64, 1032), (60013, 96, 512)]
GRADIENT = [(60013, 512, 96), (40037, 520, 128), (60013, 96, 512)]
SHAPES = FORWARD + [s for s in GRADIENT if s not in FORWARD]


def ints(g, *shape, dtype):
    return torch.randint(-2, 3, shape, generator=g, device="cuda").to(dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("rows,n_in,n_out", SHAPES)
def test_whole_numbers_are_exact(rows, n_in, n_out, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows)
    x, w, r, b = ints(g, rows, n_in, dtype=dtype), ints(g, n_out, n_in, dtype=dtype), ints(g, rows, n_out, dtype=dtype), ints(g, n_out, dtype=torch.float32)
    dz, z_in = ints(g, rows, n_out, dtype=dtype), ints(g, rows, n_in, dtype=dtype)
    zz = (x.double() @ w.double().t() + b).float()
    want = (zz.clamp(min=0) + r).to(dtype)
    for residual in (r, r.clone()):                    # a new output, and one over the residual
        y = None if residual is r else residual
        got, _ = terra.terra_linear_fwd(x, w, bias=b, residual=residual, activation="relu", y=y)
        assert torch.equal(got, want)
    y, z = terra.terra_linear_fwd(x, w, bias=b, residual=r, activation="relu", keep_z=True)
    assert torch.equal(y, want) and torch.equal(z, zz.to(dtype))
    want = (dz.double() @ w.double() * (z_in > 0)).to(dtype)
    for over in (None, z_in.clone()):
        dx, _, _ = terra.terra_linear_bwd(x, w, dz, z_in=z_in if over is None else over, activation="relu", d_x=over, need_dw=False, need_dbias=False)
        assert torch.equal(dx, want)
    terra.terra_swin_check()


@pytest.mark.gpu
@pytest.mark.parametrize("activation", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("rows,n_in,n_out,dtype", [(40000, 256, 768, BF16), (40037, 128, 520, F16), (40037, 520, 128, BF16), (60013, 96, 512, F16)])
def test_costly_activations(rows, n_in, n_out, dtype, activation):
    g = torch.Generator(device="cuda").manual_seed(n_in)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")
    x, w, r, b = n(rows, n_in).to(dtype), (2 * n(n_out, n_in) / n_in ** 0.5).to(dtype), n(rows, n_out).to(dtype), 0.3 * n(n_out)
    z64 = x.double() @ w.double().t() + b.double()
    off = (x.double().abs() @ w.double().abs().t()) * (n_in / 16 + 4) * 2 * EPS32 + b.double().abs() * EPS32
    ref = act(z64, activation)
    near = 1.2 * off + ref.abs() * 1.2e-5 + z64.abs() * 2.0 ** -21         # slopes up to 1.13, the tail's polynomial 9e-6, exp2 and the reciprocal 2^-21
    y, _ = terra.terra_linear_fwd(x, w, bias=b, activation=activation)     # no residual: both tiles in turn, a store of one under way
    held("y", y, ref, near, dtype)
    y, z = terra.terra_linear_fwd(x, w, bias=b, activation=activation, keep_z=True)      # z in the second tile
    held("y beside z", y, ref, near, dtype)
    held("z", z, z64, off, dtype)
    over = r.clone()
    y, _ = terra.terra_linear_fwd(x, w, bias=b, residual=over, activation=activation, y=over)
    held("y over the residual", y, ref + r.double(), near + r.double().abs() * EPS32, dtype)
    dz, z_in = n(rows, n_out).to(dtype), (2 * n(rows, n_in)).to(dtype)
    dx, _, _ = terra.terra_linear_bwd(x, w, dz, z_in=z_in, activation=activation, need_dw=False, need_dbias=False)
    plain = dz.double() @ w.double()
    off = (dz.double().abs() @ w.double().abs()) * (n_out / 16 + 4) * 2 * EPS32
    held("d_x", dx, plain * act_slope(z_in.double(), activation), 1.2 * off + plain.abs() * 2e-5, dtype)
    terra.terra_swin_check()


def test_the_shapes_give_every_block_several_tiles(tmp_path):
    out = run_host_program(tmp_path, """
#include "block_kernels.h"
int main(int, char** a) {
    for (int i = 1; a[i]; i += 4) {
        const long long rows = atoll(a[i + 1]);
        const int n_in = atoi(a[i + 2]), n_out = atoi(a[i + 3]);
        const LinearPlan p = a[i][0] == 'f' ? plan_linear(kLinearForward, false, rows, n_out, n_in) : plan_linear(kLinearInput, false, rows, n_in, n_out);
        std::printf("%d %d %d %d\\n", p.pair, p.splits, p.k_blocks, p.m_tiles * p.n_tiles);
    }
    const LinearPlan w = plan_linear(kLinearWeights, false, 2048, 2048, 20011);
    std::printf("%d", w.kb_per_split);
}
""", *[v for s in FORWARD for v in ("f", *s)], *[v for s in GRADIENT for v in ("d", *s)]).split("\n")
    for line in out[:-1]:
        pair, splits, stages, tiles = map(int, line.split())
        assert pair == 1 and splits == 1 and stages <= 8 and tiles >= 2 * 74, line
    assert len(out) == len(FORWARD) + len(GRADIENT) + 1 and int(out[-1]) >= 64


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "fp16"])
def test_weight_gradient_leaves_the_matrix_units_early(dtype):
    # 20011 rows in parts of at least 64 stages.  A chunk of n steps of 16 N(0, 1) terms: the running sum after step i is 4 sqrt(i) on average, a step cuts off
    # half a unit of it at its mean, 0.36 2^-23 of it (the mean of unit over value is 0.72), all of one sign: 0.36 2^-23 sum(sqrt(i)) / sqrt(n) = 0.24 n 2^-23 of
    # the chunk.  Signs of different chunks are independent, so that is the sum's share too: n = 16: 4.6e-7, and 64 would be 1.8e-6.  The 79 additions of chunks
    # in fp32, each half a unit at most, 0.29 of one on average: sqrt(79 / 2) 0.29 0.72 2^-23 = 1.6e-7.  Together 4.9e-7; a quarter is left for both models.
    g = torch.Generator(device="cuda").manual_seed(3)
    x, dz = torch.randn(20011, 2048, generator=g, device="cuda").to(dtype), torch.randn(20011, 2048, generator=g, device="cuda").to(dtype)
    w = torch.zeros(2048, 2048, device="cuda", dtype=dtype)
    _, dw, _ = terra.terra_linear_bwd(x, w, dz, need_dx=False, need_dbias=False)
    want = dz.double().t() @ x.double()
    assert (dw.double() - want).norm() <= 6e-7 * want.norm()

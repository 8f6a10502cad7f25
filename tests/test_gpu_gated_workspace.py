"""The backward through a gate in exactly the workspace that terra_linear_workspace_bytes gives for it: right, and nothing is written behind it."""
import pytest
import torch

import paper_2608_15211_b200 as terra

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


# sums that would be split had they the room, and ones that are; padded rows
@pytest.mark.parametrize("rows,n_in,n_out", [(79, 152, 704), (312, 136, 1216), (275, 720, 1144), (487, 2752, 3936), (2153, 856, 6016), (880, 1605, 3960), (40, 64, 4096), (200, 96, 8192), (2838, 32, 1408)])
def test_exact_workspace(rows, n_in, n_out):
    g = torch.Generator(device="cuda").manual_seed(rows)
    ints = lambda *s: torch.randint(-2, 3, s, generator=g, device="cuda").to(BF16)
    x, w, d, z = ints(rows, n_in), ints(n_out, n_in), ints(rows, n_out), ints(rows, 2 * n_in)
    need = terra.terra_linear_workspace_bytes(rows, n_in, n_out, "bwd")
    memory = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
    dz, dw, db = terra.terra_linear_bwd_gated(x, w, d, z, activation="relu", workspace=memory[:need])
    assert (memory[need:] == 0x5a).all()
    dy, gate, up = d.double() @ w.double(), z.double()[:, :n_in], z.double()[:, n_in:]      # (whole numbers below 2^24: exact in any order)
    assert torch.equal(dz, torch.cat((dy * up * (gate > 0), dy * gate.clamp(min=0)), 1).to(BF16))
    assert torch.equal(dw.double(), d.double().t() @ x.double()) and torch.equal(db.double(), d.double().sum(0))
    again = terra.terra_linear_bwd_gated(x, w, d, z, activation="relu", workspace=memory)
    assert all(torch.equal(a, b) for a, b in zip(again, (dz, dw, db)))

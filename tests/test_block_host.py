"""What the norm, product and rotary entry points refuse on the host, before any CUDA call, and the host-side helpers."""
import ctypes
import math

import pytest
import torch

import paper_2608_15211_b200 as terra
from paper_2608_15211_b200 import binding
from paper_2608_15211_b200.build import build

INVALID, UNSUPPORTED, ALIGNMENT, WORKSPACE = 1, 2, 3, 4
P = 0x10000          # a pointer that is never followed: the call is refused before


@pytest.fixture(scope="module")
def lib():
    build()
    return binding.load_library()


def norm(rows=4, channels=64, eps=1e-6, dtype=0):
    return ctypes.byref(terra.terra_norm_desc(rows, channels, eps, dtype))


def linear(rows=4, n_in=64, n_out=32, activation=0, dtype=0):
    return ctypes.byref(terra.terra_linear_desc(rows, n_in, n_out, activation, dtype))


def grid(heads=2, head_dim=32, B=1, H=4, W=4, shift=0, dtype=0):
    return ctypes.byref(terra.terra_swin_desc(B, H, W, heads, head_dim, 4, shift, shift, 0, 1, 0.0, dtype))


def rotary(rot_dim=32, layout=0, row_pairs=8, inverse=0, scale=1.0):
    return ctypes.byref(terra.terra_rotary_desc(rot_dim, layout, row_pairs, inverse, scale))


BAD_NORM = [(dict(rows=0), INVALID), (dict(rows=-1), INVALID), (dict(channels=0), INVALID), (dict(channels=16385), UNSUPPORTED), (dict(eps=-1e-6), INVALID),
            (dict(eps=math.nan), INVALID), (dict(eps=math.inf), INVALID), (dict(dtype=2), INVALID)]


@pytest.mark.parametrize("kw,status", BAD_NORM, ids=str)
def test_norm_descriptors(lib, kw, status):
    n = ctypes.c_size_t()
    assert lib.terra_rms_norm_fwd(norm(**kw), P, None, P, None, P, None, None) == status
    assert lib.terra_rms_norm_fwd_e4m3(norm(**kw), P, None, P, None, P, P, None, None) == status
    assert lib.terra_rms_norm_bwd(norm(**kw), P, P, P, P, None, P, P, P, 1 << 30, None) == status
    assert lib.terra_rms_norm_workspace_bytes(norm(**kw), ctypes.byref(n)) == status


def test_norm_arguments(lib):
    d = norm()
    fwd = [P, P, P, 2 * P, 3 * P, P]                       # x, residual, weight, h, y, rstd
    for i, status in ((0, INVALID), (2, INVALID), (4, INVALID)):
        assert lib.terra_rms_norm_fwd(d, *[None if j == i else p for j, p in enumerate(fwd)], None) == status
    for i in range(6):
        assert lib.terra_rms_norm_fwd(d, *[p + 8 if j == i else p for j, p in enumerate(fwd)], None) == ALIGNMENT
    assert lib.terra_rms_norm_fwd(d, P, P, P, P, P, P, None) == INVALID                      # y over h
    assert lib.terra_rms_norm_fwd_e4m3(d, P, P, P, 2 * P, 3 * P, None, None, None) == INVALID
    assert lib.terra_rms_norm_fwd_e4m3(d, P, P, P, 2 * P, 3 * P, P + 4, None, None) == ALIGNMENT
    bwd = [P, P, P, P, P, 2 * P, P]                        # h, weight, rstd, d_y, d_h, d_x, d_weight
    for i in (0, 1, 2, 3, 5, 6):
        assert lib.terra_rms_norm_bwd(d, *[None if j == i else p for j, p in enumerate(bwd)], P, 1 << 30, None) == INVALID
    for i in range(7):
        assert lib.terra_rms_norm_bwd(d, *[p + 2 if j == i else p for j, p in enumerate(bwd)], P, 1 << 30, None) == ALIGNMENT
    need = terra.terra_rms_norm_workspace_bytes(4, 64)
    assert lib.terra_rms_norm_bwd(d, *bwd, P, need - 1, None) == WORKSPACE and lib.terra_rms_norm_bwd(d, *bwd, None, need, None) == WORKSPACE
    assert lib.terra_rms_norm_bwd(d, *bwd, P + 4, need, None) == ALIGNMENT
    assert lib.terra_rms_norm_workspace_bytes(d, None) == INVALID and lib.terra_rms_norm_fwd(None, *fwd, None) == INVALID


BAD_LINEAR = [(dict(rows=0), INVALID), (dict(rows=2 ** 31 - 1023), INVALID), (dict(n_in=0), INVALID), (dict(n_out=-3), INVALID), (dict(n_in=65537), UNSUPPORTED),
              (dict(n_out=65537), UNSUPPORTED), (dict(activation=5), INVALID), (dict(activation=-1), INVALID), (dict(dtype=7), INVALID)]


@pytest.mark.parametrize("kw,status", BAD_LINEAR, ids=str)
def test_linear_descriptors(lib, kw, status):
    n = ctypes.c_size_t()
    assert lib.terra_linear_fwd(linear(**kw), P, P, None, None, P, None, P, 1 << 40, None) == status
    assert lib.terra_linear_fwd_e4m3(linear(**kw), P, P, P, P, None, None, P, P, 1 << 40, None) == status
    assert lib.terra_linear_bwd(linear(**kw), P, P, P, None, P, P, P, P, 1 << 40, None) == status
    assert lib.terra_linear_workspace_bytes(linear(**kw), 0, ctypes.byref(n)) == status


def test_linear_arguments(lib):
    d = linear()
    fwd = [P, P, P, P, 2 * P, 3 * P]                       # x, w, bias, residual, y, z
    for i in (0, 1, 4):
        assert lib.terra_linear_fwd(d, *[None if j == i else p for j, p in enumerate(fwd)], P, 1 << 30, None) == INVALID
    for i in range(6):
        assert lib.terra_linear_fwd(d, *[p + 8 if j == i else p for j, p in enumerate(fwd)], P, 1 << 30, None) == ALIGNMENT
    assert lib.terra_linear_fwd(d, P, P, P, P, P, P, P, 1 << 30, None) == INVALID             # y over z
    e = [P, P, P, P, P, P, 2 * P]                          # x8, x_scale, w8, w_scale, bias, residual, y
    for i in (0, 1, 2, 3, 6):
        assert lib.terra_linear_fwd_e4m3(d, *[None if j == i else p for j, p in enumerate(e)], P, 1 << 30, None) == INVALID
    for i in range(7):
        assert lib.terra_linear_fwd_e4m3(d, *[p + 1 if j == i else p for j, p in enumerate(e)], P, 1 << 30, None) == ALIGNMENT
    bwd = [P, P, P, P, 2 * P, 3 * P, 4 * P]                # x, w, d_z, z_in, d_x, d_w, d_bias
    for i in (0, 1, 2):
        assert lib.terra_linear_bwd(d, *[None if j == i else p for j, p in enumerate(bwd)], P, 1 << 30, None) == INVALID
    for i in range(7):
        assert lib.terra_linear_bwd(d, *[p + 4 if j == i else p for j, p in enumerate(bwd)], P, 1 << 30, None) == ALIGNMENT
    assert lib.terra_linear_bwd(d, P, P, P, None, None, None, None, P, 1 << 30, None) == INVALID
    need = terra.terra_linear_workspace_bytes(4, 64, 32, "bwd")
    assert need > 0 and lib.terra_linear_bwd(d, *bwd, P, need - 1, None) == WORKSPACE and lib.terra_linear_bwd(d, *bwd, P + 8, need, None) == ALIGNMENT
    odd = linear(rows=16, n_in=63)
    need = terra.terra_linear_workspace_bytes(16, 63, 32)
    assert need > 0 and lib.terra_linear_fwd(odd, *fwd, None, 0, None) == WORKSPACE and lib.terra_linear_fwd(odd, *fwd, P, need - 1, None) == WORKSPACE
    n = ctypes.c_size_t()
    assert lib.terra_linear_workspace_bytes(d, 3, ctypes.byref(n)) == INVALID and lib.terra_linear_workspace_bytes(d, 0, None) == INVALID
    for bad in ((0, 1, 0), (8, 9, 0), (8, 1, 3)):
        assert lib.terra_activation_bwd(*bad, P, P, P, None) == INVALID
    assert lib.terra_activation_bwd(8, 1, 0, P, None, P, None) == INVALID and lib.terra_activation_bwd(8, 1, 0, P, P, P + 2, None) == ALIGNMENT


@pytest.mark.parametrize("kw", [dict(rot_dim=0), dict(rot_dim=31), dict(rot_dim=34), dict(layout=2), dict(layout=-1), dict(row_pairs=-1), dict(row_pairs=17),
                                dict(scale=math.nan), dict(scale=math.inf)], ids=str)
def test_rotary_descriptors(lib, kw):
    assert lib.terra_rotary(grid(), rotary(**kw), P, None, P, P, P, P, None) == INVALID
    assert lib.terra_rotary_packed(grid(), rotary(**kw), P, None, P, None) == INVALID


def test_rotary_arguments(lib):
    a = [P, P, P, P, P, P]                                 # inv_freq, positions, q, k, q_out, k_out
    for i in (0, 2, 3, 4, 5):
        assert lib.terra_rotary(grid(), rotary(), *[None if j == i else p for j, p in enumerate(a)], None) == INVALID
    for i in range(6):
        assert lib.terra_rotary(grid(), rotary(), *[p + 8 if j == i else p for j, p in enumerate(a)], None) == ALIGNMENT
    assert lib.terra_rotary(grid(head_dim=48), rotary(), *a, None) == UNSUPPORTED and lib.terra_rotary(grid(heads=0), rotary(), *a, None) == INVALID
    assert lib.terra_rotary(None, rotary(), *a, None) == INVALID and lib.terra_rotary(grid(), None, *a, None) == INVALID
    assert lib.terra_rotary_packed(grid(), rotary(), P, None, None, None) == INVALID and lib.terra_rotary_packed(None, rotary(), P, None, P, None) == INVALID
    assert lib.terra_rotary_packed(grid(), rotary(), P, None, P + 8, None) == ALIGNMENT


def test_workspaces_hold_what_the_shapes_ask_for(lib):
    # padded rows of x and w, or of d_z too; and 16-byte rows need none of it
    assert terra.terra_linear_workspace_bytes(100000, 93, 512) >= 100000 * 192 + 512 * 192
    assert terra.terra_linear_workspace_bytes(100000, 96, 512) == 0
    assert terra.terra_linear_workspace_bytes(100000, 100, 512, "fwd_e4m3") >= 100000 * 112 + 512 * 112
    assert terra.terra_linear_workspace_bytes(100000, 96, 93, "bwd") >= 100000 * 192
    assert terra.terra_rms_norm_workspace_bytes(1, 8) >= 32


def test_the_binding_refuses(lib):
    x, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.ones(64)
    for call in (lambda: terra.terra_rms_norm_fwd(x, w), lambda: terra.terra_linear_fwd(x, x), lambda: terra.terra_linear_bwd(x, x, torch.zeros(4, 4, dtype=torch.bfloat16)),
                 lambda: terra.terra_activation_bwd(x, x, "relu")):
        with pytest.raises(ValueError, match="CUDA tensors"):
            call()
    with pytest.raises(ValueError, match="last dimension"):
        terra.terra_rms_norm_fwd(x, torch.ones(32))
    with pytest.raises(ValueError, match="bfloat16 or torch.float16"):
        terra.terra_rms_norm_fwd(x.float(), w)
    with pytest.raises(ValueError, match="weight must be torch.float32"):
        terra.terra_rms_norm_fwd(x, w.bfloat16())
    with pytest.raises(ValueError, match="residual must be torch.bfloat16"):
        terra.terra_rms_norm_fwd(x, w, residual=x.half())
    with pytest.raises(ValueError, match="w must be"):
        terra.terra_linear_fwd(x, w)
    with pytest.raises(ValueError, match="w must be torch.bfloat16"):
        terra.terra_linear_fwd(x, x.half())
    with pytest.raises(ValueError, match="activation must be one of"):
        terra.terra_linear_fwd(x, x, activation="tanh")
    with pytest.raises(ValueError, match="bf16 or fp16"):
        terra.terra_linear_fwd_e4m3(x, w, x, w, dtype=torch.float32)
    with pytest.raises(ValueError, match="x must be torch.float8_e4m3fn"):
        terra.terra_linear_fwd_e4m3(x, w, x, w)
    d = binding.terra_swin_desc(1, 2, 2, 1, 32, 2, 0, 0, 0, 1, 0.0, 0)
    q = torch.zeros(1, 2, 2, 1, 32, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="layout must be one of"):
        terra.terra_rotary(d, q, q, torch.ones(16, dtype=torch.float64), layout="quarter")
    with pytest.raises(ValueError, match="inv_freq must be torch.float64"):
        terra.terra_rotary(d, q, q, torch.ones(16))
    with pytest.raises(ValueError, match="CUDA tensors"):
        terra.terra_rotary(d, q, q, torch.ones(16, dtype=torch.float64))


def test_rotary_frequencies():
    f, scale = terra.rotary_frequencies(32, row_pairs=8, device="cpu")
    assert f.dtype == torch.float64 and scale == 1.0 and torch.equal(f[:8], f[8:]) and f[0] == 1 and abs(f[7] - 10000 ** (-7 / 8)) < 1e-15
    g, _ = terra.rotary_frequencies(32, row_pairs=8, scaling="linear", factor=4, device="cpu")
    assert torch.allclose(g * 4, f, rtol=1e-15)
    b, _ = terra.rotary_frequencies(64, scaling="base", factor=4, device="cpu")
    plain, _ = terra.rotary_frequencies(64, device="cpu")
    assert b[0] == plain[0] and abs(b[-1] * 4 / plain[-1] - 1) < 1e-12
    p, scale = terra.rotary_frequencies(128, scaling="parts", factor=8, length=4096, device="cpu")
    plain, _ = terra.rotary_frequencies(128, device="cpu")
    turns = 4096 * plain / (2 * math.pi)
    assert abs(scale - (1 + 0.1 * math.log(8))) < 1e-15
    assert torch.equal(p[turns >= 32], plain[turns >= 32]) and torch.allclose(p[turns <= 1] * 8, plain[turns <= 1], rtol=1e-15)
    between = (turns > 1) & (turns < 32)
    assert between.any() and ((p < plain) & (p > plain / 8))[between].all()
    one, _ = terra.rotary_frequencies(2, scaling="base", factor=2, device="cpu")
    assert one.tolist() == [1.0]
    for bad in (dict(rot_dim=0), dict(rot_dim=3), dict(rot_dim=4, row_pairs=3), dict(rot_dim=4, factor=0.5), dict(rot_dim=4, base=0), dict(rot_dim=4, scaling="parts"),
                dict(rot_dim=4, scaling="other")):
        with pytest.raises(ValueError):
            terra.rotary_frequencies(**bad, device="cpu")


def test_outputs_over_inputs_that_others_still_read(lib):
    d = linear()
    Q, R, S = 2 * P, 3 * P, 4 * P                          # x, w, residual at P, Q, R
    for y, z in ((P, S), (Q, S), (S, P), (S, Q), (S, R), (S, S)):
        assert lib.terra_linear_fwd(d, P, Q, None, R, y, z, None, 0, None) == INVALID
    for y in (P, Q):
        assert lib.terra_linear_fwd_e4m3(d, P, S, Q, S, None, R, y, None, 0, None) == INVALID
    for d_x in (R, Q):
        assert lib.terra_linear_bwd(d, P, Q, R, None, d_x, S, None, P, 1 << 30, None) == INVALID
    for y8 in (P, Q):                                      # (8 bits over 16)
        assert lib.terra_rms_norm_fwd_e4m3(norm(), P, Q, R, None, y8, S, None, None) == INVALID
    for q_out, k_out in ((Q, R), (R, P), (R, R)):
        assert lib.terra_rotary(grid(), rotary(), S, None, P, Q, q_out, k_out, None) == INVALID

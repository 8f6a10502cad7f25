"""The norm, product and rotary calls as programs use them: captured and replayed, on several streams at once, from several threads, on tensors of more
than 2^31 values; and the product over a seeded sweep of sizes and options."""
import random
import threading

import pytest
import torch

import paper_2608_15211_b200 as terra
from paper_2608_15211_b200.workloads import small_config
from tests._block import frequencies

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


def ints(g, *shape, dtype=BF16):
    return torch.randint(-2, 3, shape, generator=g, device="cuda").to(dtype)


def calls(seed):
    """Every entry point on small tensors, as functions without arguments that return tensors."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")
    x, r, w, gy = n(300, 96).to(BF16), n(300, 96).to(BF16), 1 + 0.1 * n(96), n(300, 96).to(BF16)
    rstd = (x.float().square().mean(1) + 1e-6).rsqrt()
    wt, b, dz, z = n(200, 96).to(BF16), n(200), n(300, 200).to(BF16), n(300, 96).to(BF16)
    odd, few, long = n(130, 93).to(BF16), n(2, 96).to(BF16), n(40, 4096).to(BF16)
    wodd, wlong = n(50, 93).to(BF16), n(64, 4096).to(BF16)
    x8, w8, xs, ws = x.to(torch.float8_e4m3fn), wt.to(torch.float8_e4m3fn), n(300).abs(), n(200).abs()
    cfg = small_config("use", 1, 10, 30, 1, 32, 8, 4, 4)
    desc, freq = terra.make_desc(cfg), frequencies(32, 8).cuda()
    q, k = n(1, 10, 30, 1, 32).to(BF16), n(1, 10, 30, 1, 32).to(BF16)
    return [lambda: terra.terra_rms_norm_fwd(x, w, residual=r), lambda: terra.terra_rms_norm_fwd_e4m3(x, w, residual=r)[1:],
            lambda: terra.terra_rms_norm_bwd(x, w, rstd, gy, d_h=r), lambda: terra.terra_linear_fwd(x, wt, bias=b, activation="gelu", keep_z=True),
            lambda: terra.terra_linear_bwd(x, wt, dz, z_in=z, activation="silu"), lambda: (terra.terra_linear_fwd(odd, wodd)[0],),
            lambda: (terra.terra_linear_fwd(few, wt)[0],), lambda: (terra.terra_linear_fwd(long, wlong)[0],),
            lambda: (terra.terra_linear_fwd_e4m3(x8, xs, w8, ws, bias=b),), lambda: (terra.terra_activation_bwd(z, x, "gelu_tanh"),),
            lambda: terra.terra_rotary(desc, q, k, freq, row_pairs=8)]


def test_captured_and_replayed():
    fs = calls(1)
    want = [[t.clone() for t in f()] for f in fs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            got = [f() for f in fs]
        for _ in range(3):
            for ts in got:
                for t in ts:
                    t.zero_()
            graph.replay()
        side.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(s, t) for s, t in zip(a, b))
    terra.terra_swin_check()


def test_streams_and_threads_at_once():
    jobs = [calls(seed) for seed in (1, 2, 3)]
    want = [[[t.clone() for t in f()] for f in fs] for fs in jobs]
    torch.cuda.synchronize()
    bad = []

    def work(fs, ref):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(20):
                got = [f() for f in fs]
                stream.synchronize()
                bad.extend(i for i, (a, b) in enumerate(zip(got, ref)) if not all(torch.equal(s, t) for s, t in zip(a, b)))

    threads = [threading.Thread(target=work, args=j) for j in zip(jobs, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad
    terra.terra_swin_check()


def test_results_do_not_depend_on_what_the_workspace_holds():
    g = torch.Generator(device="cuda").manual_seed(5)
    x, w, dz = ints(g, 2000, 93), ints(g, 200, 93), ints(g, 2000, 200)
    want = terra.terra_linear_bwd(x, w, dz)
    for fill in (0, 255, 127):
        ws = torch.full((terra.terra_linear_workspace_bytes(2000, 93, 200, "bwd"),), fill, dtype=torch.uint8, device="cuda")
        assert all(torch.equal(a, b) for a, b in zip(terra.terra_linear_bwd(x, w, dz, workspace=ws), want))
        ws = torch.full((terra.terra_linear_workspace_bytes(2000, 93, 200),), fill, dtype=torch.uint8, device="cuda")
        assert torch.equal(terra.terra_linear_fwd(x, w, workspace=ws)[0], terra.terra_linear_fwd(x, w)[0])


def test_nothing_is_written_beside_the_outputs():
    g = torch.Generator(device="cuda").manual_seed(6)
    for rows, n_in, n_out in ((300, 96, 40), (257, 72, 372), (131, 33, 31), (3, 64, 50), (513, 128, 288)):
        x, w, dz, r = ints(g, rows, n_in), ints(g, n_out, n_in), ints(g, rows, n_out), ints(g, rows, n_out)

        def framed(*shape, dtype):
            n = torch.Size(shape).numel()
            whole = torch.full((n + 512,), 7, dtype=dtype, device="cuda")
            return whole, whole[256:256 + n].view(shape)

        y, z, dx, dw, db = framed(rows, n_out, dtype=BF16), framed(rows, n_out, dtype=BF16), framed(rows, n_in, dtype=BF16), framed(n_out, n_in, dtype=torch.float32), framed(n_out, dtype=torch.float32)
        terra.terra_linear_fwd(x, w, residual=r, activation="relu", y=y[1], z=z[1])
        terra.terra_linear_bwd(x, w, dz, d_x=dx[1], d_w=dw[1], d_bias=db[1])
        for whole, inner in (y, z, dx, dw, db):
            assert (whole[:256] == 7).all() and (whole[256 + inner.numel():] == 7).all()


@pytest.mark.parametrize("seed", range(48))
def test_product_sweep(seed):
    # whole numbers: exact whatever the tiles, the splits and the way to memory are
    rng = random.Random(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    pick = lambda low, high: round(low * (high / low) ** rng.random())
    rows, n_in, n_out = pick(1, 6000), pick(1, 3000), pick(1, 1500)
    if rng.random() < 0.7:
        n_in, n_out = -(-n_in // 8) * 8, -(-n_out // 8) * 8
    dtype, activation = rng.choice([BF16, F16]), rng.choice(["none", "relu"])
    f = (lambda t: t.clamp(min=0)) if activation == "relu" else (lambda t: t)
    x, w, dz, z_in = ints(g, rows, n_in, dtype=dtype), ints(g, n_out, n_in, dtype=dtype), ints(g, rows, n_out, dtype=dtype), ints(g, rows, n_in, dtype=dtype)
    r = ints(g, rows, n_out, dtype=dtype) if rng.random() < 0.5 else None
    b = ints(g, n_out, dtype=torch.float32) if rng.random() < 0.5 else None
    keep = rng.random() < 0.5
    zz = x.double() @ w.double().t() + (b.double() if b is not None else 0)
    y, z = terra.terra_linear_fwd(x, w, bias=b, residual=r, activation=activation, keep_z=keep)
    assert torch.equal(y, (f(zz) + (r.double() if r is not None else 0)).to(dtype))
    assert z is None if not keep else torch.equal(z, zz.to(dtype))
    dx, dw, db = terra.terra_linear_bwd(x, w, dz, z_in=z_in if activation == "relu" else None, activation=activation)
    slope = (z_in.double() > 0) if activation == "relu" else 1
    assert torch.equal(dx, (dz.double() @ w.double() * slope).to(dtype))
    assert torch.equal(dw, (dz.double().t() @ x.double()).float()) and torch.equal(db, dz.double().sum(0).float())
    xs, ws = 2.0 ** torch.randint(-2, 3, (rows,), generator=g, device="cuda").float(), 2.0 ** torch.randint(-2, 3, (n_out,), generator=g, device="cuda").float()
    y8 = terra.terra_linear_fwd_e4m3(x.to(torch.float8_e4m3fn), xs, w.to(torch.float8_e4m3fn), ws, bias=b, residual=r, activation=activation, dtype=dtype)
    z8 = x.double() @ w.double().t() * xs.double()[:, None] * ws.double() + (b.double() if b is not None else 0)
    assert torch.equal(y8, (f(z8) + (r.double() if r is not None else 0)).to(dtype))
    terra.terra_swin_check()


def test_more_than_two_to_the_31_values():
    g = torch.Generator(device="cuda").manual_seed(7)
    rows, c = 270000, 8192                                   # 2.2e9 values
    x, w = ints(g, rows, 64), ints(g, c, 64)
    y, _ = terra.terra_linear_fwd(x, w)
    some = torch.cat((torch.arange(0, 300, device="cuda"), torch.arange(rows - 300, rows, device="cuda"), torch.tensor([2 ** 31 // c, 2 ** 31 // c - 1], device="cuda")))
    ref = (x[some].double() @ w.double().t()).to(BF16)
    assert torch.equal(y[some], ref)
    dx = terra.terra_linear_bwd(x, w, y)[0]             # (reads y back; its sums are no longer exact)
    want = y[some].double() @ w.double()
    assert ((dx[some].double() - want).abs() <= want.abs() * 2.0 ** -8 + 2.0 ** -12 * (y[some].double().abs() @ w.double().abs())).all()
    del dx
    weight = 1 + torch.rand(c, generator=g, device="cuda")
    n, h, rstd = terra.terra_rms_norm_fwd(y, weight, residual=y)
    small, h_small, rstd_small = terra.terra_rms_norm_fwd(y[some].contiguous(), weight, residual=y[some].contiguous())
    assert torch.equal(n[some], small) and torch.equal(h[some], h_small) and torch.equal(rstd[some], rstd_small)
    dx, _ = terra.terra_rms_norm_bwd(h, weight, rstd, n)
    assert torch.equal(dx[some], terra.terra_rms_norm_bwd(h_small, weight, rstd_small, small)[0])
    del n, h, dx
    cfg = small_config("far", 1, 300, 900, 64, 128, 8, 4, 4)
    freq = frequencies(128, 32).cuda()
    q = y.view(1, 300, 900, 64, 128)
    turned, _ = terra.terra_rotary(terra.make_desc(cfg), q, None, freq, row_pairs=32)
    last = small_config("last", 1, 1, 900, 64, 128, 8, 0, 0)
    at = torch.stack((torch.full((900,), 295), (torch.arange(900) - 4) % 900), -1).view(1, 1, 900, 2).int().cuda()
    alone, _ = terra.terra_rotary(terra.make_desc(last), q[:, 299:].contiguous(), None, freq, row_pairs=32, positions=at)
    assert torch.equal(turned[:, 299:], alone)


@pytest.mark.parametrize("activation", ["silu", "gelu", "gelu_tanh"])
def test_slopes_are_the_forward_s_differences(activation):
    # (act(z + t) - act(z - t)) / 2 t for t = 1 / 16: off by a rounding of either value (half a step of fp16) and by t^2 / 6 of the third derivative, below 2
    t = 1 / 16
    z = (torch.arange(-96, 97, device="cuda") / 16).to(F16)[None]
    eye = torch.eye(193, device="cuda", dtype=F16)
    up, _ = terra.terra_linear_fwd(z + t, eye, activation=activation)
    down, _ = terra.terra_linear_fwd(z - t, eye, activation=activation)
    slope = terra.terra_activation_bwd(z, torch.ones_like(z), activation).double()
    allowed = 2.0 ** -11 * (up.double().abs() + down.double().abs()) / (2 * t) + t * t / 6 * 2 + 2.0 ** -11 * slope.abs() + 1e-5
    assert ((up.double() - down.double()) / (2 * t) - slope).abs().le(allowed).all()


def test_norm_gradient_is_the_forward_s_difference():
    # along a direction e: sum of g (y(x + t e) - y(x - t e)) / 2 t against the backward call's <d_x, e>
    g = torch.Generator(device="cuda").manual_seed(3)
    x, e, gy = (torch.randn(2000, 64, generator=g, device="cuda") for _ in range(3))
    w = 1 + 0.2 * torch.randn(64, generator=g, device="cuda")
    t = 1 / 64
    up, down, x, gy = (x + t * e).to(F16), (x - t * e).to(F16), x.to(F16), gy.to(F16)
    step = (up.double() - down.double()) / (2 * t)           # the step that was taken, after rounding
    y1, y0 = (terra.terra_rms_norm_fwd(v, w)[0].double() for v in (up, down))
    rstd = terra.terra_rms_norm_fwd(x, w)[2]
    dx, _ = terra.terra_rms_norm_bwd(x, w, rstd, gy)
    taken, said = (gy.double() * (y1 - y0) / (2 * t)).sum(), (dx.double() * step).sum()
    # each difference has two roundings of y (half a step of values up to 2^-11 |y|, of random sign: they add in squares), dx one; the curvature t^2 |e|^3
    size = (gy.double().square() * (y1.square() + y0.square())).sum().sqrt() * 2.0 ** -11 / (2 * t)
    curved = t * t * (gy.double().abs() * e.double().abs().pow(3)).sum() * 4 / 8
    assert abs(taken - said) <= 4 * size + (dx.double() * step).square().sum().sqrt() * 2.0 ** -11 * 4 + curved


def test_products_gradients_are_exact_differences():
    # the product is linear in x and in w: with whole numbers the differences are exact
    g = torch.Generator(device="cuda").manual_seed(4)
    x, w, dz, ex, ew = ints(g, 50, 40), ints(g, 24, 40), ints(g, 50, 24), ints(g, 50, 40), ints(g, 24, 40)
    y = lambda a, b: terra.terra_linear_fwd(a, b)[0].double()
    dx, dw, _ = terra.terra_linear_bwd(x, w, dz)
    exact = lambda t: bool((t.abs() <= 256).all())           # whole numbers that bf16 holds
    assert exact(y(x, w)) and exact(y(x + ex, w)) and exact(y(x, w + ew)) and exact(dx.double())
    assert ((y(x + ex, w) - y(x, w)) * dz.double()).sum() == (dx.double() * ex.double()).sum()
    assert ((y(x, w + ew) - y(x, w)) * dz.double()).sum() == (dw.double() * ew.double()).sum()

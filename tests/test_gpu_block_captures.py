"""The norm, product and rotary calls behind what is no kernel of this library in a captured graph: copies, fills, other streams; each as the first call there."""
import pytest
import torch

import paper_2608_15211_b200 as terra
from tests.test_gpu_block_use import calls

pytestmark = pytest.mark.gpu


def firsts(seed):
    """Each entry point on inputs that a copy in the graph brings, as (buffers to copy from, buffers to copy to, call)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
    out = []
    for rows, n_in, n_out in ((300, 96, 200), (3, 96, 200), (300, 93, 50), (40, 4096, 64), (2000, 256, 256)):
        src, w, dz = n(rows, n_in), n(n_out, n_in), n(rows, n_out)
        x = torch.empty_like(src)
        out.append((src, x, lambda x=x, w=w: terra.terra_linear_fwd(x, w, activation="gelu")[:1]))
        out.append((src, x, lambda x=x, w=w, dz=dz: terra.terra_linear_bwd(x, w, dz, z_in=x, activation="silu")))
    src, w = n(300, 96), 1 + 0.1 * torch.randn(96, generator=g, device="cuda")
    x = torch.empty_like(src)
    out.append((src, x, lambda x=x, w=w: terra.terra_rms_norm_fwd(x, w)[::2]))
    return out


@pytest.mark.parametrize("before", ["copy", "fill and copy", "two streams"])
def test_behind_other_nodes(before):
    for src, x, call in firsts(7):
        x.copy_(src)
        want = [t.clone() for t in call()]
        x.zero_()
        main, side = torch.cuda.Stream(), torch.cuda.Stream()
        main.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(main):
            with torch.cuda.graph(graph, stream=main):
                if before == "two streams":
                    side.wait_stream(main)
                    half = x.shape[0] // 2
                    x[:half].copy_(src[:half])
                    with torch.cuda.stream(side):
                        x[half:].copy_(src[half:])
                    main.wait_stream(side)
                else:
                    if before == "fill and copy":
                        x.zero_()
                    x.copy_(src)
                got = call()
            for _ in range(3):
                x.fill_(3)
                for t in got:
                    t.zero_()
                graph.replay()
                main.synchronize()
                assert all(torch.equal(a, b) for a, b in zip(got, want))
    terra.terra_swin_check()


def test_two_graphs_in_turn_and_at_once():
    # graphs of one pool share their workspaces, so they run one after the other; graphs of pools of their own may run at once
    for pool in (torch.cuda.graph_pool_handle(), None):
        graphs = []
        for seed in (1, 2):
            fs = calls(seed)
            want = [[t.clone() for t in f()] for f in fs]
            stream = torch.cuda.Stream()
            stream.wait_stream(torch.cuda.current_stream())
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.stream(stream), torch.cuda.graph(graph, stream=stream, pool=pool):
                got = [f() for f in fs]
            graphs.append((graph, stream, got, want, fs))
        for _ in range(5):
            for graph, stream, got, want, _ in graphs:
                with torch.cuda.stream(stream):
                    graph.replay()
                if pool is not None:
                    stream.synchronize()
                    assert all(torch.equal(s, t) for a, b in zip(got, want) for s, t in zip(a, b))
            torch.cuda.synchronize()
        if pool is None:
            for _, _, got, want, _ in graphs:
                assert all(torch.equal(s, t) for a, b in zip(got, want) for s, t in zip(a, b))
    terra.terra_swin_check()

"""GPU: a recorded propagation replayed after a call on a larger graph, for which the context's workspaces grew."""
import pytest
import torch

import paper_2305_03152_amd as spp

pytestmark = pytest.mark.gpu


def _ring(ctx, N, d, **kw):
    rp = torch.arange(N + 1, dtype=torch.int64, device="cuda") * d
    col = ((torch.arange(N, device="cuda").unsqueeze(1) + torch.arange(1, d + 1, device="cuda")) % N).sort(1).values.to(torch.int32).reshape(-1)
    return spp.Graph(ctx, rp, col, in_lists=True, **kw)


@pytest.mark.parametrize("kind", ["blocks", "chunked", "general"])
def test_propagation_replayed_after_a_larger_graph_s(kind):
    d = 10
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = spp.Context(0)
        graphs = [(N, _ring(ctx, N, d, chunked=kind == "chunked")) for N in (10_000, 300_000)]
        T = torch.arange(300, dtype=torch.int32, device="cuda")
        p0 = [torch.linspace(0, 1, N, device="cuda") for N, _ in graphs]
        t = [torch.linspace(1, 0, N * d, device="cuda") for N, _ in graphs]

        def call(k, sync):
            if kind == "general":
                return spp.vip_propagate_general(ctx, graphs[k][1], p0[k], t[k], 2, sync=sync)
            return spp.vip_propagate(ctx, graphs[k][1], T, 64, (3, 2, 4), sync=sync)

        want = call(0, True)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            recorded = call(0, False)
        large = call(1, True)
        filled = [torch.full((size,), float("nan"), device="cuda") for size in (1 << 14, 1 << 16, 1 << 18, 1 << 20) for _ in range(6)]
        for k in range(4):
            print("[case]", kind, k, flush=True)
            recorded.zero_()
            graph.replay()
            torch.cuda.synchronize()
            # the sums of a vertex may be added up in another order: the last bit of a result
            assert torch.allclose(recorded, want, rtol=3e-7, atol=0) and torch.allclose(call(1, True), large, rtol=3e-7, atol=0)
        assert all(bool(torch.isnan(f).all()) for f in filled)
        ctx.close()

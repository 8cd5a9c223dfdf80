"""GPU: operators on gathered rows recorded into graphs: every replay gives what an eager call gives, also after calls that
need more of the context's memory, and a context's first call may be a recorded one."""
import pytest
import torch

import paper_2305_03152_amd as spp

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _lists(c, n, D, H, groups, dtype, seed):
    gen = torch.Generator(DEV).manual_seed(seed)
    items = []
    for k in range(groups):
        rows = spp.mx4_quantize(c, torch.randn(n, D, generator=gen, device=DEV))
        items.append((rows, n, torch.tensor([n], dtype=torch.int64, device=DEV), torch.randn(n, H, generator=gen, device=DEV).to(dtype), k))
    return spp.RowLists(items)


def _change(lists, k):
    for j, (rows, n, count, y, _) in enumerate(lists.lists):
        y.copy_(torch.randn(y.shape, generator=torch.Generator(DEV).manual_seed(100 * k + j), device=DEV))
        count.fill_(n - 37 * k - j)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_gradient_replayed_after_a_call_that_needs_more_memory(dtype):
    D, H = 100, 172
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c = spp.Context(0, side)
        lists, large = _lists(c, 900, D, H, 2, dtype, 1), _lists(c, 30_000, 256, 512, 3, dtype, 2)
        out = torch.empty(2, H, D, device=DEV)
        spp.mx4_weight_grad(c, lists, H, D, groups=2, out=out)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            spp.mx4_weight_grad(c, lists, H, D, groups=2, out=out, sync=False)
        want_large = spp.mx4_weight_grad(c, large, 512, 256, groups=3)               # the workspace grows
        filled = [torch.full((size,), float("nan"), device=DEV) for size in (1 << 18, 1 << 20, 1 << 22) for _ in range(4)]
        for k in range(4):
            print("[case]", dtype, k, flush=True)
            _change(lists, k)
            out.zero_()
            graph.replay()
            side.synchronize()
            got = out.clone()
            assert torch.equal(got, spp.mx4_weight_grad(c, lists, H, D, groups=2)) and float(got.abs().max()) > 0
            assert torch.equal(want_large, spp.mx4_weight_grad(c, large, 512, 256, groups=3))
        assert all(bool(torch.isnan(f).all()) for f in filled)
        c.close()


@pytest.mark.parametrize("mode", ["global", "thread_local", "relaxed"])
def test_gradient_recorded_as_a_context_s_first_calls(mode):
    """A small gradient, then one for which the workspace grows, both in one recording that allocates on the way."""
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ref, c = spp.Context(0, side), spp.Context(0, side)
        small, large = _lists(ref, 900, 100, 172, 2, torch.bfloat16, 3), _lists(ref, 20_000, 768, 1024, 1, torch.bfloat16, 4)
        a, b = torch.empty(2, 172, 100, device=DEV), torch.empty(1, 1024, 768, device=DEV)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side, capture_error_mode=mode):
            spp.mx4_weight_grad(c, small, 172, 100, groups=2, out=a, sync=False)
            spp.mx4_weight_grad(c, large, 1024, 768, out=b, sync=False)
        for k in range(4):
            print("[case]", mode, k, flush=True)
            _change(small, k)
            _change(large, k)
            a.zero_()
            b.zero_()
            graph.replay()
            side.synchronize()
            assert torch.equal(a, spp.mx4_weight_grad(ref, small, 172, 100, groups=2))
            assert torch.equal(b, spp.mx4_weight_grad(ref, large, 1024, 768))
            assert torch.equal(b, spp.mx4_weight_grad(c, large, 1024, 768))                  # the context's eager calls go on
        c.close()
        ref.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_is_not_recorded(bits):
    """Replays of a recorded step would repeat its bias corrections: refused, nothing is recorded, and steps go on as before."""
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c = spp.Context(0, side)
        g = torch.randn(1000, device=DEV)
        p, q = torch.ones(1000, device=DEV), torch.ones(1000, device=DEV)
        opt, ref = spp.AdamW(c, [p], state_bits=bits, lr=1e-2), spp.AdamW(c, [q], state_bits=bits, lr=1e-2)
        opt.step([g])
        ref.step([g])
        graph, extra = torch.cuda.CUDAGraph(), torch.zeros(1, device=DEV)
        with torch.cuda.graph(graph, stream=side):
            extra.add_(1)
            with pytest.raises(spp.SppError, match="repeat step 2"):
                opt.step([g], sync=False)
        assert opt.t == 1
        for k in range(3):
            graph.replay()
            side.synchronize()
            assert torch.equal(p, q) and float(extra) == k + 1
            opt.step([g])
            ref.step([g])
        assert torch.equal(p, q) and opt.t == 4
        c.close()

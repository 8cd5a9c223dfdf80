"""The weight gradient of very many rows: sums in fp32 are of a bounded number of rows, whatever the matrix's size, and these sums are added in 64 bits.

With a matrix of as many tiles as the GPU has CUs a group's rows are one run: its result has to be the sum, in 64 bits, of the results of its
stretches, each a call of its own, rounded once.  These are equalities, not bounds."""
import numpy as np
import pytest
import torch

import paper_2305_03152_amd as spp

pytestmark = pytest.mark.gpu
DEV = "cuda"
STRETCH = {torch.bfloat16: 32768, torch.float16: 16384, torch.float32: 10912}       # rows of a sum in fp32
CHUNK = {torch.bfloat16: 64, torch.float16: 32, torch.float32: 32}                  # lists are cut into so many
FORMATS = {"mx4": (spp.mx4_quantize, spp.mx4_weight_grad), "fp8": (spp.fp8_quantize, spp.fp8_weight_grad)}


@pytest.fixture(scope="module")
def ctx():
    c = spp.Context(0)
    yield c
    c.close()


def _one_run(D, H):
    """Tiles of 256 x 256 as many as CUs: a run."""
    if -(-D // 256) * -(-H // 256) < torch.cuda.get_device_properties(0).multi_processor_count:
        pytest.skip("more CUs than tiles")


def _data(ctx, fmt, n, D, H, dtype, alike, seed=1):
    gen = torch.Generator(DEV).manual_seed(seed)
    few = 1 if alike else 5003
    rows = FORMATS[fmt][0](ctx, torch.rand(few, D, generator=gen, device=DEV) + 0.5)
    ys = (torch.rand(few, H, generator=gen, device=DEV) + 0.5).to(dtype)
    at = torch.arange(n, device=DEV) * 7919 % few
    return rows[at].contiguous(), ys[at].contiguous()


@pytest.mark.parametrize("fmt", ["mx4", "fp8"])
@pytest.mark.parametrize("alike", [True, False])
@pytest.mark.parametrize("dtype", list(STRETCH))
def test_a_run_is_the_sum_of_its_stretches(ctx, dtype, alike, fmt):
    D = H = 4096
    _one_run(D, H)
    grad, L = FORMATS[fmt][1], STRETCH[dtype]
    n = 4 * L + 777
    x, y = _data(ctx, fmt, n, D, H, dtype, alike)
    got = grad(ctx, [(x, n, None, y)], H, D)[0]
    want = torch.zeros(H, D, dtype=torch.float64, device=DEV)
    for a in range(0, n, L):
        want += grad(ctx, [(x[a:a + L], min(L, n - a), None, y[a:a + L])], H, D)[0]
    assert torch.equal(got, want.float())
    if alike:                                  # and is right: 1024 additions, each off by at most 2^-23 of what it adds, and 64 bits behind that
        exact = n * y[:1].double().T @ (FORMATS[fmt][1](ctx, [(x[:1], 1, None, torch.ones(1, H, device=DEV))], H, D)[0][:1].double())
        assert float((got / exact - 1).abs().max()) <= 1024 * 2.0 ** -23 + 2.0 ** -24


@pytest.mark.parametrize("dtype", list(STRETCH))
def test_stretches_over_lists_and_groups(ctx, dtype):
    """Lists that end inside chunks, a count on the device, a second group that begins within a stretch; the same bits in buffers of any room."""
    D = H = 4096
    _one_run(D, H)
    L, chunk = STRETCH[dtype], CHUNK[dtype]
    sizes = [L // 3 + 5, L + 100, 0, L // 2 + 1]
    x, y = _data(ctx, "fp8", sum(sizes), D, H, dtype, False)
    parts, a = [], 0
    for n in sizes:
        parts.append((x[a:a + n], y[a:a + n]))
        a += n
    def chunks(n):
        return -(-n // chunk)
    first = L - chunk * chunks(sizes[0])       # rows of the second list that the first stretch has
    def grad(items, groups=1):
        return spp.fp8_weight_grad(ctx, [(p[0].contiguous(), len(p[0]), None, p[1], g) for p, g in items], H, D, groups=groups)
    cut = (parts[1][0][:first], parts[1][1][:first]), (parts[1][0][first:], parts[1][1][first:])
    one = grad([(parts[0], 0), (cut[0], 0)])[0].double() + grad([(cut[1], 0), (parts[2], 0)])[0].double()
    two = grad([(parts[3], 0)])[0]
    got = grad([(parts[0], 0), (parts[1], 0), (parts[2], 0), (parts[3], 1)], 2)
    assert torch.equal(got[0], one.float()) and torch.equal(got[1], two)
    room = []
    for (px, py), n, g in zip(parts, sizes, (0, 0, 0, 1)):
        cap = n + 3 * L // 2
        bx, by = torch.full((cap, px.shape[1]), 255, dtype=torch.uint8, device=DEV), torch.full((cap, H), float("nan"), dtype=dtype, device=DEV)
        bx[:n], by[:n] = px, py
        room.append((bx, cap, torch.tensor([n], dtype=torch.int64, device=DEV), by, g))
    assert torch.equal(spp.fp8_weight_grad(ctx, room, H, D, groups=2), got)


@pytest.mark.parametrize("dtype", list(STRETCH))
@pytest.mark.parametrize("few", [1, 130, 3000])
def test_few_rows_in_very_much_room(ctx, dtype, few):
    """Room for runs longer than a stretch, and rows for one: as in buffers that just hold them."""
    D, H, cap = 700, 4000, 700_000 if dtype != torch.float32 else 250_000
    x, y = _data(ctx, "fp8", few, D, H, dtype, False)
    bx, by = torch.full((cap, x.shape[1]), 255, dtype=torch.uint8, device=DEV), torch.full((cap, H), float("nan"), dtype=dtype, device=DEV)
    bx[:few], by[:few] = x, y
    got = spp.fp8_weight_grad(ctx, [(bx, cap, torch.tensor([few], dtype=torch.int64, device=DEV), by)], H, D)
    assert torch.equal(got, spp.fp8_weight_grad(ctx, [(x, few, None, y)], H, D))


@pytest.mark.parametrize("dtype", list(STRETCH))
@pytest.mark.parametrize("D,H,groups", [(1000, 1001, 1), (2049, 300, 3), (129, 4000, 2), (2000, 2000, 5)])
def test_whole_numbers_over_several_runs_and_stretches(ctx, dtype, D, H, groups):
    """Rows of 0, 1 and 2 and gradients up to 3: sums of a stretch are below 2^24 and exact, the result is the exact sum rounded once."""
    n = int(2.2e9 // (H * (4 if dtype == torch.float32 else 2)))
    gen = torch.Generator(DEV).manual_seed(D)
    pool = spp.fp8_quantize(ctx, torch.randint(0, 3, (4001, D), generator=gen, device=DEV).float())
    ys = torch.randint(-1, 4, (4001, H), generator=gen, device=DEV).to(dtype)
    at = torch.arange(n, device=DEV) * 6007 % 4001
    x, y = pool[at].contiguous(), ys[at].contiguous()
    cuts = [0] + sorted(int(n * (k + 0.37) / (2 * groups)) for k in range(2 * groups - 1)) + [n]
    items = [(x[a:b].contiguous(), b - a, None, y[a:b], k // 2) for k, (a, b) in enumerate(zip(cuts, cuts[1:]))]
    got = spp.fp8_weight_grad(ctx, items, H, D, groups=groups)
    values, yd = spp.fp8_dequantize(ctx, pool, D).double(), ys.double()
    for g in range(groups):
        a, b = cuts[2 * g], cuts[2 * g + 2]
        times = torch.bincount(at[a:b], minlength=4001).double().unsqueeze(1)
        assert torch.equal(got[g], ((yd * times).T.contiguous() @ values).float()), g

"""The weight gradient where its result can be known exactly, or to what its smallest operands allow."""
import numpy as np
import pytest
import torch

import mx4_reference as R
import paper_2305_03152_amd as spp

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def ctx():
    c = spp.Context(0)
    yield c
    c.close()


def test_tiny_fp32_gradients_count_to_the_smallest_bf16(ctx):
    """dY of every magnitude down to the smallest fp32, X = 2^20: 24 bits are exact from 2^-110 on, below that what lies under
    2^-133 is cut off.  One row, so that nothing else rounds but the subnormal sum, which 2^20 keeps away."""
    D = H = 64
    rng = np.random.default_rng(1)
    bits = rng.integers(0, 1 << 23, (130, H), dtype=np.int64) | (np.minimum(np.arange(130), 60)[:, None].astype(np.int64) << 23)
    bits[61:] = rng.integers(1, 1 << 23, (69, H))                                     # subnormal
    y = bits.astype(np.uint32).view(np.float32) * np.where(rng.random((130, H)) < 0.5, -1, 1).astype(np.float32)
    rows = np.zeros((1, R.row_bytes(D)), np.uint8)
    rows[:, :32], rows[:, 32:34] = 0x22, 127 + 20
    row = torch.from_numpy(rows).to(DEV)
    for k in range(len(y)):
        got = spp.mx4_weight_grad(ctx, [(row, 1, None, torch.from_numpy(y[k:k + 1]).to(DEV))], H, D)[0].double().cpu().numpy() / 2.0 ** 20
        want = y[k].astype(np.float64)[:, None]
        off = np.abs(got - want)
        assert (off[np.abs(want[:, 0]) >= 2.0 ** -110] == 0).all() and (off < 2.0 ** -133).all()


def test_an_x_beyond_fp32_is_infinite(ctx):
    rows = np.zeros((2, R.row_bytes(32)), np.uint8)
    rows[0, :16], rows[0, 16] = 0x42, 254                        # 2^127 and 2^128 in turn
    y = torch.tensor([[1e-10], [1.0]], device=DEV)
    g = spp.mx4_weight_grad(ctx, [(torch.from_numpy(rows).to(DEV), 2, None, y)], 1, 32)[0, 0].cpu()
    assert torch.isinf(g[1::2]).all() and torch.isfinite(g[0::2]).all()


# every shape of tile: D up to 64, 128 and more, H up to 64, 128, 192 and 256 of a tile; few rows and many; lists over several groups
SHAPES = [(D, H) for D in (33, 64, 65, 128, 160, 700) for H in (7, 64, 65, 128, 129, 192, 193, 256, 300)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D,H", SHAPES)
def test_whole_numbers_are_added_exactly(ctx, dtype, D, H):
    """X of whole numbers up to 12, dY up to 4: sums below 2^24 are exact in any order, so that a chunk or a run lost, doubled or
    counted to another group shows.  Many rows in lists of uneven lengths, some counted on the device, behind them NaN."""
    rng = np.random.default_rng(D * 1000 + H)
    groups, nb = 3, -(-D // 32)
    want = torch.zeros(groups, H, D, dtype=torch.float64)
    items = []
    for j, n in enumerate([0, 1, 63, 64, 65, 7001, 2, 9000, 129, 0, 8191, 1000]):
        rows = np.zeros((n + 40, R.row_bytes(D)), np.uint8)
        rows[:, :16 * nb] = rng.integers(0, 256, (n + 40, 16 * nb))
        rows[:, 16 * nb:17 * nb] = 128
        rows[n:, 16 * nb:17 * nb] = 255
        y = torch.full((n + 40, H), float("nan"), dtype=dtype, device=DEV)
        y[:n] = torch.from_numpy(rng.integers(-4, 5, (n, H))).to(DEV, dtype)
        g = (5 * j) % groups if j != 6 else 2
        want[g] += y[:n].double().cpu().T @ torch.from_numpy(R.values(rows[:n], D))
        on_device = j % 2 == 0
        items.append((torch.from_numpy(rows).to(DEV), n + 40 if on_device else n, torch.tensor([n], device=DEV) if on_device else None, y, g))
    assert float(want.abs().max()) < 2 ** 24
    assert torch.equal(spp.mx4_weight_grad(ctx, items, H, D, groups=groups).double().cpu(), want)
    for n in (1, 63, 128, 129, 5000):                            # one list: straight into dW, or in runs
        x, y = items[5][0][:n], items[5][3][:n]
        one = y.double().cpu().T @ torch.from_numpy(R.values(x.cpu().numpy(), D))
        assert torch.equal(spp.mx4_weight_grad(ctx, [(x, n, None, y)], H, D)[0].double().cpu(), one), n

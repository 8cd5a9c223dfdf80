"""The weight gradient's runs: how the rows of all lists are cut does not depend on the room that the buffers have."""
import numpy as np
import pytest
import torch

import mx4_reference as R
import paper_2305_03152_amd as spp

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def ctx():
    c = spp.Context(0)
    yield c
    c.close()


def _list(rng, n, D, H, dtype):
    nb = -(-D // 32)
    rows = rng.integers(0, 256, (n, R.row_bytes(D))).astype(np.uint8)
    rows[:, 16 * nb:17 * nb] = rng.integers(120, 130, (n, nb))
    return torch.from_numpy(rows).to(DEV), torch.from_numpy(rng.standard_normal((n, H))).to(DEV, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("counts,groups,D,H,room", [([100], 1, 100, 172, (128, 129, 1000)), ([1], 1, 768, 1024, (100, 129, 5000)), ([64], 1, 32, 32, (65, 200, 4000)),
                                                    ([128], 1, 128, 256, (129, 100_000)), ([129], 1, 128, 256, (200, 100_000)), ([3000], 1, 128, 256, (3001, 6000, 300_000)),
                                                    ([2] * 64, 1, 768, 1024, (3, 40, 900)), ([5, 0, 70, 1, 0, 300], 4, 96, 200, (301, 5000)),
                                                    ([700] * 24, 8, 100, 172, (701, 9000)), ([20_000], 1, 400, 130, (20_001, 90_000))])
def test_the_same_rows_give_the_same_bits_in_buffers_of_any_room(ctx, dtype, counts, groups, D, H, room):
    rng = np.random.default_rng(sum(counts) + 3 * D + H)
    lists = [_list(rng, n, D, H, dtype) for n in counts]
    want = spp.mx4_weight_grad(ctx, [(x, n, None, y, j % groups) for j, (n, (x, y)) in enumerate(zip(counts, lists))], H, D, groups=groups)
    assert float(want.abs().max()) > 0
    for cap in room:
        items = []
        for j, (n, (x, y)) in enumerate(zip(counts, lists)):
            bx = torch.full((cap, x.shape[1]), 255, dtype=torch.uint8, device=DEV)
            by = torch.full((cap, H), float("nan"), dtype=dtype, device=DEV)
            bx[:n], by[:n] = x, y
            items.append((bx, cap, torch.tensor([n], dtype=torch.int64, device=DEV), by, j % groups))
        assert torch.equal(spp.mx4_weight_grad(ctx, items, H, D, groups=groups), want), cap

"""The 4-bit product where W's operands are read step by step or X's scales share a register: whole numbers, exactly.

Codes are any, scales 2^-2 to 2^2 by block: values are multiples of 2^-3, terms of 2^-6, and the terms' magnitudes of a sum add up to less
than 2^18 (checked), so that sums in fp32, 24 bits, are exact in any order: the result is the exact sum, rounded once."""
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


def _rows(rng, n, D):
    nb = -(-D // 32)
    rows = np.zeros((n, R.row_bytes(D)), np.uint8)
    codes = rng.integers(0, 256, (n, nb * 16)).astype(np.uint8)
    if D % 32:
        codes[:, D // 2 + D % 2:] = 0
        if D % 2:
            codes[:, D // 2] &= 15
    rows[:, :16 * nb] = codes
    rows[:, 16 * nb:17 * nb] = rng.integers(125, 130, (n, nb))
    return rows


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n,D,H,ld", [(1, 257, 321, 321), (300, 300, 501, 501), (131, 384, 330, 333), (1000, 353, 1001, 1001), (40, 384, 321, 640), (200000, 768, 321, 384),
                                      (200100, 641, 400, 448), (197000, 750, 300, 320)])
def test_sums_of_whole_numbers(ctx, dtype, n, D, H, ld):
    rng = np.random.default_rng(n + D + H)
    pool = _rows(rng, min(n, 1511), D)
    at = rng.integers(0, len(pool), n)
    w = _rows(rng, H, D)
    buf = torch.full((n * ld + 64,), 7.0, dtype=dtype, device=DEV)
    y = buf.as_strided((n, H), (ld, 1))
    rows = torch.from_numpy(pool).to(DEV)[torch.from_numpy(at).to(DEV)].contiguous()
    spp.mx4_product(ctx, rows, torch.from_numpy(w).to(DEV), D, out=y)
    x, v = R.values(pool, D), R.values(w, D)
    assert (np.abs(x) @ np.abs(v).T).max() < 2.0 ** 18 and (x * 8 == np.round(x * 8)).all() and (v * 8 == np.round(v * 8)).all()
    want = torch.from_numpy(x @ v.T).to(DEV, dtype)[torch.from_numpy(at).to(DEV)]
    assert torch.equal(y, want)
    keep = torch.ones(buf.numel(), dtype=torch.bool, device=DEV)
    keep.as_strided((n, H), (ld, 1)).fill_(False)
    assert (buf[keep] == 7).all()

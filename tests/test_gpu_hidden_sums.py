"""The layers on hidden rows add in fp32 whatever the type of their results: whole numbers whose large terms cancel each other.

In groups of eight neighbouring columns a row of X has 448 twice, which W multiplies by 448 and by -448 (times a power of two), and a small
number, which W multiplies by another.  At most 32 groups of a row hold anything: all terms are whole multiples of one power of two and their magnitudes
add up to less than 2^24 of it, so that sums in fp32 are exact in any order and what is left of each group is the small term alone.
The product is then the exact sum rounded once, half a step; of the gated layer and its gradient the sums G and U are exact and only
the activation's own bound and the roundings behind it remain (fp8_reference.activation).
"""
import numpy as np
import pytest
import torch

import fp8_reference as R
import paper_2305_03152_amd as spp

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = [torch.float32, torch.float16, torch.bfloat16]
STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
GROUPS = 32
# every form of a kernel: W in LDS as codes or values, one sixteen of rows or two, few rows and many, W in registers, both by way of LDS
SHAPES = [(1, 16, 8), (5, 8, 40), (300, 256, 256), (70000, 256, 256), (70000, 172, 100), (70000, 172, 86), (3000, 100, 64), (2000, 300, 47), (2000, 512, 64), (600, 640, 128),
          (900, 640, 300), (700, 512, 512), (400, 1024, 47), (900, 1024, 130), (70, 1100, 40), (70, 4096, 24)]


@pytest.fixture(scope="module")
def ctx():
    c = spp.Context(0)
    yield c
    c.close()


def _cancelling(n, D, H, size):
    """X [n, D] and W [H, D] as packed rows and as values; W's are multiples of `size`, a power of two."""
    rng = np.random.default_rng(n + 3 * D + 7 * H)
    x, w = np.zeros((n, D)), np.zeros((H, D))
    groups = D // 8
    role = np.concatenate([8 * g + rng.permutation(8)[:3] for g in range(groups)]).reshape(groups, 3)
    w[:, role[:, 0]], w[:, role[:, 1]] = 448.0, -448.0
    w[:, role[:, 2]] = rng.integers(1, 4, (H, groups))
    some = rng.random((n, groups)).argsort(1)[:, :GROUPS]
    held = np.zeros((n, groups), bool)
    np.put_along_axis(held, some, True, 1)
    x[:, role[:, 0]] = x[:, role[:, 1]] = 448.0 * held
    x[:, role[:, 2]] = held * rng.integers(-3, 4, (n, groups))
    rows, packed = R.quantize(x), R.quantize(w * size)
    assert (R.values(packed, D) == w * size).all() and (R.values(rows[:100], D) == x[:100]).all()
    assert np.abs(x[:100]).dot(np.abs(w).T).max() < 2 ** 24
    return rows, packed, x, w * size


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,D,H", SHAPES)
def test_small_terms_beside_large_ones_that_cancel(ctx, dtype, n, D, H):
    rows, w, x, wv = _cancelling(n, D, H, 1.0)
    y = spp.fp8_product(ctx, torch.from_numpy(rows).to(DEV), torch.from_numpy(w).to(DEV), D, dtype=dtype)
    assert torch.equal(y.cpu(), torch.from_numpy(x @ wv.T).to(dtype))


@pytest.mark.parametrize("act", ["silu", "gelu", "sigmoid"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,D,H", [(n, D, -(-H // 2)) for n, D, H in SHAPES if n < 70000 or D < 256])
def test_the_gated_layer_and_its_gradient_of_the_same(ctx, dtype, act, n, D, H):
    rows, w, x, wv = _cancelling(n, D, 2 * H, 2.0 ** -4)
    xd, wd = torch.from_numpy(rows).to(DEV), torch.from_numpy(w).to(DEV)
    g, u = x @ wv[:H].T, x @ wv[H:].T
    f, d, _, _, bf, bd = R.activation(act, g)
    dy = torch.from_numpy(np.random.default_rng(n).standard_normal((n, H))).to(dtype)
    dp = torch.full((n, 2 * H), float("nan"), dtype=dtype, device=DEV)
    y = spp.fp8_gated(ctx, xd, wd, D, activation=act, dtype=dtype)
    spp.fp8_gated_grad(ctx, [(xd, n, None, dy.to(DEV))], [(xd, n, None, dp)], wd, D, activation=act)
    dy = dy.double().numpy()
    # the activation's bound, a product's rounding each (two for dG), the rounding to the type, half of fp16's smallest step
    for got, want, bound in ((y, f * u, bf * np.abs(u) + np.abs(f * u) * 2.0 ** -24), (dp[:, :H], dy * u * d, np.abs(dy * u) * bd + np.abs(dy * u * d) * 2.0 ** -23),
                             (dp[:, H:], dy * f, np.abs(dy) * bf + np.abs(dy * f) * 2.0 ** -24)):
        got = got.double().cpu().numpy()
        bound = bound + STEP[dtype] * (np.abs(want) + bound) + (2.0 ** -25 if dtype == torch.float16 else 2.0 ** -126)
        bad = ~(np.abs(got - want) <= bound)
        assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3], got[bad][:3], want[bad][:3])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D,H", [(64, 40), (256, 200), (300, 600), (1024, 300), (1100, 30)])
def test_values_beyond_fp32_are_infinite(ctx, dtype, D, H):
    """Scale byte 254, which quantising does not give: 448 2^127 and its kin count as infinite whatever they are multiplied by, in their row only; 1.5 2^127 does not."""
    n, at = 20, R.code_bytes(D)
    rows, w = R.quantize(np.ones((n, D))), R.quantize(np.full((H, D), 2.0 ** -100))
    rows[:, at] = 127
    rows[:, :D] = 0x38                                         # ones
    rows[3, at], rows[3, 1:min(D, 128)], rows[3, 0] = 254, 0, 0x7E     # 448 2^127
    rows[7, at], rows[7, 1:min(D, 128)], rows[7, 0] = 254, 0, 0xFE
    rows[9, at], rows[9, 1:min(D, 128)], rows[9, 0] = 254, 0, 0x3C     # 1.5 2^127
    y = spp.fp8_product(ctx, torch.from_numpy(rows).to(DEV), torch.from_numpy(w).to(DEV), D, dtype=dtype).double().cpu()
    assert bool((y[3] == float("inf")).all()) and bool((y[7] == -float("inf")).all())
    rest = [k for k in range(n) if k not in (3, 7, 9)]
    assert bool(torch.isfinite(y[rest]).all())
    want = torch.tensor(1.5 * 2.0 ** 27 + max(0, D - 128) * 2.0 ** -100, dtype=torch.float64).to(dtype).double()
    assert bool((y[9] == want).all())

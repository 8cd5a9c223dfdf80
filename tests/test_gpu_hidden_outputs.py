"""The layers on hidden rows with many outputs: more blocks of columns than divide an XCD's CUs evenly, more than it has, and the most there can be.

Tolerances as in the tests of fewer outputs: terms are exact, sums round in fp32 (fp8_reference), what is written is rounded once, half a step."""
import numpy as np
import pytest
import torch

import fp8_reference as R
import paper_2305_03152_amd as spp

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = [torch.float32, torch.float16, torch.bfloat16]
STEP = {torch.float32: 0.0, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


@pytest.fixture(scope="module")
def ctx():
    c = spp.Context(0)
    yield c
    c.close()


def _close(got, want, bound, dtype):
    got = got.double().cpu().numpy()
    bound = bound + STEP[dtype] * (np.abs(want) + bound) + (2.0 ** -25 if dtype == torch.float16 else 0)
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,D,H", [(1, 100, 65536), (40, 33, 65535), (700, 1024, 8200), (1100, 300, 12001), (9000, 600, 2176), (300, 1100, 9000)])
def test_product(ctx, dtype, n, D, H):
    rng = np.random.default_rng(n + D + H)
    pool = R.quantize(rng.standard_normal((min(n, 211), D)))
    at = rng.integers(0, len(pool), n)
    w = R.quantize(rng.standard_normal((H, D)) * D ** -0.5)
    y = torch.full((n + 1, H), 7.0, dtype=dtype, device=DEV)
    spp.fp8_product(ctx, torch.from_numpy(pool[at]).to(DEV), torch.from_numpy(w).to(DEV), D, out=y[:n])
    assert (y[n] == 7).all()
    want, bound = R.sums(R.values(pool, D), R.values(w, D))
    first = np.array([np.flatnonzero(at == k)[0] if (at == k).any() else -1 for k in range(len(pool))])
    there = first >= 0
    _close(y[torch.from_numpy(first[there]).to(DEV)], want[there], bound[there], dtype)
    assert torch.equal(y[:n], y[torch.from_numpy(first[at]).to(DEV)])          # equal rows have equal results, wherever they are


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,D,H", [(1, 100, 32768), (40, 33, 32767), (500, 1024, 4200), (3000, 1024, 2816), (5000, 600, 2176), (300, 1100, 4500)])
def test_gated_layer_and_its_gradient(ctx, dtype, n, D, H):
    rng = np.random.default_rng(n + D + H + 1)
    pool = R.quantize(rng.standard_normal((min(n, 97), D)))
    at = rng.integers(0, len(pool), n)
    w = R.quantize(rng.standard_normal((2 * H, D)) * D ** -0.5)
    dpool = torch.from_numpy(rng.standard_normal((len(pool), H))).to(dtype)
    x, v = R.values(pool, D), R.values(w, D)
    xd, wd, dy = torch.from_numpy(pool[at]).to(DEV), torch.from_numpy(w).to(DEV), dpool[torch.from_numpy(at)].to(DEV)
    first = np.array([np.flatnonzero(at == k)[0] if (at == k).any() else -1 for k in range(len(pool))])
    there = first >= 0
    one, every = torch.from_numpy(first[there]).to(DEV), torch.from_numpy(first[at]).to(DEV)
    y = spp.fp8_gated(ctx, xd, wd, D, activation="gelu", dtype=dtype)
    want, bound = R.gated(x, v[:H], v[H:], "gelu")
    _close(y[one], want[there], bound[there], dtype)
    assert torch.equal(y, y[every])
    dp = torch.full((n + 1, 2 * H), 7.0, dtype=dtype, device=DEV)
    spp.fp8_gated_grad(ctx, [(xd, n, None, dy)], [(xd, n, None, dp[:n])], wd, D, activation="gelu")
    want, bound = R.gated_grad(x, v[:H], v[H:], dpool.double().numpy(), "gelu")
    _close(dp[one], want[there], bound[there], dtype)
    assert torch.equal(dp[:n], dp[every]) and (dp[n] == 7).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,D,H", [(3, 33, 65536), (500, 200, 20001)])
def test_weight_gradient(ctx, dtype, n, D, H):
    rng = np.random.default_rng(n)
    rows = R.quantize(rng.standard_normal((n, D)))
    y = torch.from_numpy(rng.standard_normal((n, H))).to(dtype)
    g = spp.fp8_weight_grad(ctx, [(torch.from_numpy(rows).to(DEV), n, None, y.to(DEV))], H, D)[0]
    x, v = R.values(rows, D), y.double().numpy()
    _close(g, v.T @ x, 3 * n * 2.0 ** -23 * (np.abs(v).T @ np.abs(x)), torch.float32)

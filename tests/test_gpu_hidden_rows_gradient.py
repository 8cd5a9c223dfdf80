"""The gradient of a layer's rows: a product by the transpose of the values that the layer read.

An E4M3's relative step is the same under any power of two as scale, down to 2^-6 of it, and the largest value of a block is above 224 of its scale and at most
448: a value of at least 2^-6 / 224 = 1/14336 of its new block's largest is held as it is, one below moves by at most half of the smallest step, 2^-10 of the
scale, 1/229376 of the largest."""
import numpy as np
import pytest
import torch

import fp8_reference as R
import paper_2305_03152_amd as spp

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def ctx():
    c = spp.Context(0)
    yield c
    c.close()


def _transposed(ctx, w, D):
    return spp.fp8_quantize(ctx, spp.fp8_dequantize(ctx, w, D).T.contiguous())


@pytest.mark.parametrize("H,D,spread", [(256, 256, 1.0), (512, 172, 1.0), (47, 100, 3.0), (1, 300, 1.0), (300, 1, 6.0), (1100, 640, 2.0)])
def test_the_transpose_has_the_values_that_the_layer_read(ctx, H, D, spread):
    rng = np.random.default_rng(H + D)
    wf = torch.from_numpy(rng.standard_normal((H, D)) * np.exp2(rng.standard_normal((H, 1)) * spread)).float().to(DEV)
    w = spp.fp8_quantize(ctx, wf)
    was = R.values(w.cpu().numpy(), D).T
    now = R.values(_transposed(ctx, w, D).cpu().numpy(), H)
    for a in range(0, H, 128):
        top = np.abs(was[:, a:a + 128]).max(1, keepdims=True)
        v, n = was[:, a:a + 128], now[:, a:a + 128]
        keeps = np.abs(v) * 14336 >= top
        assert (n[keeps] == v[keeps]).all() and (np.abs(n - v) * 229376 <= top).all()


@pytest.mark.parametrize("n,D,H", [(300, 256, 256), (500, 172, 100), (70, 100, 1024), (40, 64, 2048)])
def test_rows_gradient_of_a_gated_layer(ctx, n, D, H):
    """dX = dP W with dP as 8 bits hold it and the layer's own W, within what the sums round and the smallest weights move."""
    rng = np.random.default_rng(n + D + H)
    x = spp.fp8_quantize(ctx, torch.from_numpy(rng.standard_normal((n, D))).float().to(DEV))
    w = spp.fp8_quantize(ctx, torch.from_numpy(rng.standard_normal((2 * H, D)) * D ** -0.5).float().to(DEV))
    dy = torch.from_numpy(rng.standard_normal((n, H))).float().to(DEV)
    dp = torch.empty(n, 2 * H, device=DEV)
    spp.fp8_gated_grad(ctx, [(x, n, None, dy)], [(x, n, None, dp)], w, D)
    held = spp.fp8_quantize(ctx, dp)
    dx = spp.fp8_product(ctx, held, _transposed(ctx, w, D), 2 * H, dtype=torch.float32).double().cpu().numpy()
    p, v = R.values(held.cpu().numpy(), 2 * H), R.values(w.cpu().numpy(), D)
    moved = np.abs(v).max() / 229376
    assert (np.abs(dx - p @ v) <= 2 * H * 2.0 ** -23 * (np.abs(p) @ np.abs(v)) + moved * np.abs(p).sum(1, keepdims=True)).all()


def test_more_outputs_than_a_row_has_columns(ctx):
    """2H = 6000: no row of so many columns; two stretches of them, added."""
    n, D, H, cut = 50, 40, 3000, 4096
    with pytest.raises(spp.SppError):
        spp.fp8_row_bytes(2 * H)
    rng = np.random.default_rng(3)
    w = spp.fp8_quantize(ctx, torch.from_numpy(rng.standard_normal((2 * H, D))).float().to(DEV))
    dp = torch.from_numpy(rng.standard_normal((n, 2 * H))).float().to(DEV)
    dx, want, size = 0.0, 0.0, 0.0
    for a, b in ((0, cut), (cut, 2 * H)):
        held = spp.fp8_quantize(ctx, dp[:, a:b])
        dx = dx + spp.fp8_product(ctx, held, _transposed(ctx, w[a:b], D), b - a, dtype=torch.float32).double().cpu().numpy()
        p, v = R.values(held.cpu().numpy(), b - a), R.values(w[a:b].cpu().numpy(), D)
        want, size = want + p @ v, size + (b - a) * 2.0 ** -23 * (np.abs(p) @ np.abs(v)) + np.abs(v).max() / 229376 * np.abs(p).sum(1, keepdims=True)
    assert (np.abs(dx - want) <= size).all()

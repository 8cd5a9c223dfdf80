"""The layers on hidden rows in 8 bits, gated or not, and their gradients against sums in 64 bits, over lists, groups, types and strides.

Tolerances.  The product of two E4M3 has 8 bits and a scale is a power of two: the terms are exact and only the sums round, K terms each
addition of which is off by at most 2^-23 of what it adds, and for results of 16 bits the terms' alignment.  What these and the
activation's own roundings make of a gated layer is worked out beside the definitions (fp8_reference.py).  Rounding to 16 bits adds half a step: 2^-8 of the value in bf16, 2^-11 in fp16 or
half of the smallest step, 2^-25; to fp32 2^-24, which the bounds hold already.
"""
import numpy as np
import pytest
import torch

import fp8_reference as R
import paper_2305_03152_amd as spp

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = [torch.float32, torch.float16, torch.bfloat16]
STEP = {torch.float32: 0.0, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
SIZES = [(1, 1, 1), (1, 256, 256), (2, 32, 47), (15, 33, 64), (16, 100, 172), (17, 128, 65), (127, 96, 63), (128, 160, 128), (129, 172, 100),
         (255, 256, 47), (257, 300, 172), (700, 768, 512), (65, 1024, 40), (63, 1100, 130), (130, 4096, 24), (1, 1024, 512), (5, 1, 550),
         (3000, 31, 33), (600, 640, 129), (400, 512, 257), (300, 896, 96)]


@pytest.fixture(scope="module")
def ctx():
    c = spp.Context(0)
    yield c
    c.close()


def _rows(rng, n, D, size=1.0, spread=1.0):
    x = rng.standard_normal((n, D)) * size * np.exp2(rng.standard_normal((n, 1)) * spread)
    return R.quantize(x) if n else np.zeros((0, R.row_bytes(D)), np.uint8)


def _dev(rows):
    return torch.from_numpy(rows).to(DEV)


def _close(got, want, bound, dtype):
    got = got.double().cpu().numpy()
    bound = bound + STEP[dtype] * (np.abs(want) + bound) + (2.0 ** -25 if dtype == torch.float16 else 0)
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (int(bad.sum()), float(np.abs(got - want)[bad].max()), np.argwhere(bad)[:4])


def _bits(dtype):
    return 32 if dtype == torch.float32 else 16


def _split(w, H, D):
    v = R.values(w, D)
    return v[:H], v[H:]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,D,H", SIZES)
def test_product_of_one_list(ctx, dtype, n, D, H):
    rng = np.random.default_rng(n * 7 + D * 3 + H)
    rows, w = _rows(rng, n, D), _rows(rng, H, D, D ** -0.5)
    y = spp.fp8_product(ctx, _dev(rows), _dev(w), D, out=torch.full((n, H), float("nan"), dtype=dtype, device=DEV))
    _close(y, *R.sums(R.values(rows, D), R.values(w, D), _bits(dtype)), dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,D,H", SIZES)
def test_gated_layer_of_one_list_and_its_gradient(ctx, dtype, n, D, H):
    rng = np.random.default_rng(n * 7 + D * 3 + H + 1)
    rows, w = _rows(rng, n, D), _rows(rng, 2 * H, D, D ** -0.5)
    x, (wg, wu) = R.values(rows, D), _split(w, H, D)
    act = ("silu", "gelu", "sigmoid")[(n + D + H) % 3]
    dy = torch.from_numpy(rng.standard_normal((n, H))).to(dtype)
    xd, wd, dyd = _dev(rows), _dev(w), dy.to(DEV)
    dp = torch.full((n, 2 * H), float("nan"), dtype=dtype, device=DEV)
    y = spp.fp8_gated(ctx, xd, wd, D, activation=act, out=torch.full((n, H), float("nan"), dtype=dtype, device=DEV))
    _close(y, *R.gated(x, wg, wu, act, _bits(dtype)), dtype)
    spp.fp8_gated_grad(ctx, [(xd, n, None, dyd)], [(xd, n, None, dp)], wd, D, activation=act)
    _close(dp, *R.gated_grad(x, wg, wu, dy.double().numpy(), act, _bits(dtype)), dtype)
    assert torch.equal(dyd.cpu(), dy)


@pytest.mark.parametrize("act", ["silu", "gelu", "sigmoid"])
def test_activations_over_their_range(ctx, act):
    """g from -200 to 200 in one column, exactly: X holds g and 1 in two columns, W picks them."""
    D, H = 16, 8
    g = np.concatenate([np.arange(-448, 449) * 0.25 * 0.5, np.linspace(-6, 6, 97), np.exp2(np.arange(-60.0, 7.0)), -np.exp2(np.arange(-60.0, 7.0))])
    x = np.zeros((len(g), D))
    x[:, 0] = g
    rows = R.quantize(x)
    other = np.zeros((len(g), D))
    other[:, 0] = R.values(rows, D)[:, 0]
    w = np.zeros((2 * H, D))
    w[:H, 0] = 1.0
    w[H:, 0] = 1.0                                         # u = g too
    w = R.quantize(w)
    xv, (wg, wu) = R.values(rows, D), _split(w, H, D)
    y = spp.fp8_gated(ctx, _dev(rows), _dev(w), D, activation=act, dtype=torch.float32)
    _close(y, *R.gated(xv, wg, wu, act), torch.float32)
    dy, dp = torch.ones(len(g), H, device=DEV), torch.empty(len(g), 2 * H, device=DEV)
    xd = _dev(rows)
    spp.fp8_gated_grad(ctx, [(xd, len(g), None, dy)], [(xd, len(g), None, dp)], _dev(w), D, activation=act)
    _close(dp, *R.gated_grad(xv, wg, wu, np.ones((len(g), H)), act), torch.float32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,D,H", [(1, 1, 1), (1, 128, 256), (2, 32, 47), (31, 33, 64), (33, 100, 172), (63, 128, 129), (64, 96, 128), (65, 160, 127),
                                   (129, 100, 256), (700, 256, 47), (1500, 768, 300), (300, 1100, 130), (4000, 31, 33), (20000, 256, 512), (130, 4096, 24),
                                   (200, 17, 90), (3000, 64, 200)])
def test_weight_gradient_of_one_list(ctx, dtype, n, D, H):
    rng = np.random.default_rng(n * 7 + D * 3 + H + 2)
    rows = _rows(rng, n, D)
    y = torch.from_numpy(rng.standard_normal((n, H))).to(dtype)
    g = spp.fp8_weight_grad(ctx, [(_dev(rows), n, None, y.to(DEV))], H, D)
    x, v = R.values(rows, D), y.double().numpy()
    assert g.shape == (1, H, D)
    _close(g[0], v.T @ x, 3 * n * 2.0 ** -23 * (np.abs(v).T @ np.abs(x)), torch.float32)


def _many(rng, lists, groups, D, H, dtype, pad=0, offset=0):
    """Lists whose capacity exceeds their count, on the device for some; what lies behind the count must not matter."""
    items, plain = [], []
    for j in range(lists):
        cap = int(rng.integers(0, 400)) if j % 7 else int(rng.integers(0, 3))
        n = int(rng.integers(0, cap + 1)) if j % 5 else 0
        rows = _rows(rng, cap, D)
        rows[n:] = 255                                        # NaN codes and scales
        on_device = j % 2 == 0 or n == cap
        count = torch.tensor([n if j % 4 else (n if n < cap else cap + 17)], dtype=torch.int64, device=DEV) if on_device else None
        items.append((_dev(rows), cap if on_device else n, count, None, int(rng.integers(0, groups))))
        plain.append((rows[:n], n))
    return items, plain


def _matrices(rng, items, plain, H, dtype, pad, offset, fill=None):
    """A matrix for each list, its rows apart, NaN where nothing is to be read or written."""
    out, bufs = [], []
    for it, (_, n) in zip(items, plain):
        cap = it[0].shape[0]
        buf = torch.full((offset + cap * (H + pad) + 16,), float("nan"), dtype=dtype, device=DEV)
        y = torch.as_strided(buf, (cap, H), (H + pad, 1), offset)
        if fill is not None:
            y[:n] = torch.from_numpy(rng.standard_normal((n, H)) * fill).to(DEV, dtype)
        out.append((it[0], it[1], it[2], y, it[4]))
        bufs.append(buf)
    return out, bufs


def _untouched(items, bufs, plain, H, pad, offset):
    for it, buf, (_, n) in zip(items, bufs, plain):
        keep = torch.ones(buf.numel(), dtype=torch.bool, device=DEV)
        if n:
            keep.as_strided((n, H), (H + pad, 1), offset).fill_(False)
        assert torch.isnan(buf[keep]).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lists,groups,D,H,pad,offset", [(1, 1, 128, 256, 0, 0), (64, 1, 256, 96, 0, 0), (64, 64, 100, 48, 8, 8), (24, 8, 172, 100, 0, 0),
                                                         (9, 3, 50, 77, 3, 1), (3, 5, 32, 130, 0, 0), (12, 2, 600, 200, 24, 16), (5, 2, 1030, 65, 1, 0)])
def test_lists_and_groups(ctx, dtype, lists, groups, D, H, pad, offset):
    rng = np.random.default_rng(lists * 100 + groups + D)
    bare, plain = _many(rng, lists, groups, D, H, dtype)
    w1, w2 = _rows(rng, groups * H, D, D ** -0.5), _rows(rng, groups * 2 * H, D, D ** -0.5)
    d1, d2 = _dev(w1).view(groups, H, -1), _dev(w2).view(groups, 2 * H, -1)
    w1, w2 = w1.reshape(groups, H, -1), w2.reshape(groups, 2 * H, -1)
    items, bufs = _matrices(rng, bare, plain, H, dtype, pad, offset)
    spp.fp8_product_multi(ctx, spp.RowLists(items), d1, D)
    for (rows, n), it in zip(plain, items):
        _close(it[3][:n], *R.sums(R.values(rows, D), R.values(w1[it[4]], D), _bits(dtype)), dtype)
    _untouched(items, bufs, plain, H, pad, offset)
    items, bufs = _matrices(rng, bare, plain, H, dtype, pad, offset)
    spp.fp8_gated_multi(ctx, spp.RowLists(items), d2, D, activation="silu")
    for (rows, n), it in zip(plain, items):
        _close(it[3][:n], *R.gated(R.values(rows, D), *_split(w2[it[4]], H, D), "silu", _bits(dtype)), dtype)
    _untouched(items, bufs, plain, H, pad, offset)
    dys, dybufs = _matrices(rng, bare, plain, H, dtype, pad, offset, 1.0)
    dps, dpbufs = _matrices(rng, bare, plain, 2 * H, dtype, pad, offset)
    lists_dy, lists_dp = spp.RowLists(dys), spp.RowLists(dps)
    spp.fp8_gated_grad(ctx, lists_dy, lists_dp, d2, D, activation="silu")
    want, size, K = np.zeros((groups, 2 * H, D)), np.zeros((groups, 2 * H, D)), 1
    for (rows, n), dy, dp in zip(plain, dys, dps):
        x, v = R.values(rows, D), dy[3][:n].double().cpu().numpy()
        _close(dp[3][:n], *R.gated_grad(x, *_split(w2[dy[4]], H, D), v, "silu", _bits(dtype)), dtype)
        p = dp[3][:n].double().cpu().numpy()
        want[dp[4]] += p.T @ x
        size[dp[4]] += np.abs(p).T @ np.abs(x)
        K += 3 * n
    _untouched(dps, dpbufs, plain, 2 * H, pad, offset)
    _untouched(dys, dybufs, plain, H, pad, offset)
    grad = spp.fp8_weight_grad(ctx, lists_dp, 2 * H, D, groups=groups)
    _close(grad, want, K * 2.0 ** -23 * size, torch.float32)
    empty = [g for g in range(groups) if not any(it[4] == g and n for (_, n), it in zip(plain, dps))]
    assert all(int(grad[g].count_nonzero()) == 0 for g in empty)
    assert torch.equal(grad, spp.fp8_weight_grad(ctx, dps, 2 * H, D, groups=groups))


def test_nan_and_infinities_stay_in_their_rows(ctx):
    rng = np.random.default_rng(5)
    n, D, H = 200, 200, 80
    rows, w = _rows(rng, n, D), _rows(rng, 2 * H, D, D ** -0.5)
    rows[17, 208] = 255                                       # a block's scale
    rows[40, 150] = 0x7F                                      # one code
    w[33, 3] = 0xFF
    y = spp.fp8_product(ctx, _dev(rows), _dev(w), D, dtype=torch.float32).cpu()
    nan = torch.zeros(n, 2 * H, dtype=torch.bool)
    nan[17], nan[40], nan[:, 33] = True, True, True
    assert torch.equal(torch.isnan(y), nan)
    both = nan[:, :H] | nan[:, H:]
    for act in ("silu", "gelu", "sigmoid"):
        y = spp.fp8_gated(ctx, _dev(rows), _dev(w), D, activation=act, dtype=torch.float32).cpu()
        assert torch.equal(torch.isnan(y), both)
        dy, dp = torch.ones(n, H, device=DEV), torch.empty(n, 2 * H, device=DEV)
        xd = _dev(rows)
        spp.fp8_gated_grad(ctx, [(xd, n, None, dy)], [(xd, n, None, dp)], _dev(w), D, activation=act)
        dp = dp.cpu()
        assert torch.equal(torch.isnan(dp[:, :H]), both) and torch.equal(torch.isnan(dp[:, H:]), nan[:, :H])
    g = spp.fp8_weight_grad(ctx, [(_dev(rows), n, None, torch.ones(n, H, device=DEV))], H, D)[0].cpu()
    column = torch.zeros(D, dtype=torch.bool)
    column[:128] = True                                       # the block of row 17
    column[150] = True
    assert torch.equal(torch.isnan(g), column.expand(H, D))
    for dtype in TYPES:
        v = torch.from_numpy(rng.standard_normal((n, H))).to(dtype)
        v[5, 7], v[6, 8], v[90, 9] = float("inf"), float("nan"), -float("inf")
        clean = _rows(rng, n, D)
        clean[[5, 6, 90], :D] = 0x38                          # ones: infinite sums keep their sign
        d = spp.fp8_weight_grad(ctx, [(_dev(clean), n, None, v.to(DEV))], H, D)[0].cpu()
        with np.errstate(invalid="ignore"):
            want = torch.from_numpy(v.double().numpy().T @ R.values(clean, D))
        assert torch.equal(torch.isnan(d), torch.isnan(want)) and torch.equal(torch.isinf(d), torch.isinf(want))
        assert torch.equal(torch.sign(d[torch.isinf(d)]).double(), torch.sign(want[torch.isinf(want)]))


@pytest.mark.parametrize("act", ["silu", "gelu", "sigmoid"])
def test_gradients_against_differences(ctx, act):
    """Of sum(R * layer(X, W)) by single values of W and X, central differences in 64 bits: their own error is a sixth of the step's square
    times a third derivative, and a rounding of the sum over the step."""
    rng = np.random.default_rng(11)
    n, D, H = 60, 70, 20
    rows, w = _rows(rng, n, D), _rows(rng, 2 * H, D, D ** -0.5)
    x, (wg, wu) = R.values(rows, D), _split(w, H, D)
    r = torch.from_numpy(rng.standard_normal((n, H))).float()
    xd, dp = _dev(rows), torch.empty(n, 2 * H, device=DEV)
    spp.fp8_gated_grad(ctx, [(xd, n, None, r.to(DEV))], [(xd, n, None, dp)], _dev(w), D, activation=act)
    dw = spp.fp8_weight_grad(ctx, [(xd, n, None, dp)], 2 * H, D)[0].cpu().double().numpy()
    dx = dp.double().cpu().numpy() @ np.concatenate([wg, wu])
    r = r.double().numpy()
    def loss(x, wg, wu):
        return float((r * R.gated(x, wg, wu, act)[0]).sum())
    h = 2.0 ** -14
    for k in range(30):
        j, d = int(rng.integers(0, 2 * H)), int(rng.integers(0, D))
        both = np.concatenate([wg, wu])
        up, down = both.copy(), both.copy()
        up[j, d] += h
        down[j, d] -= h
        slope = (loss(x, up[:H], up[H:]) - loss(x, down[:H], down[H:])) / (2 * h)
        assert abs(slope - dw[j, d]) <= 1e-5 * (1 + np.abs(x[:, d]).max() ** 3 * n), (j, d, slope, dw[j, d])
        i = int(rng.integers(0, n))
        up, down = x.copy(), x.copy()
        up[i, d] += h
        down[i, d] -= h
        slope = (loss(up, wg, wu) - loss(down, wg, wu)) / (2 * h)
        assert abs(slope - dx[i, d]) <= 1e-4 * (1 + np.abs(x[i]).max() ** 2), (i, d, slope, dx[i, d])


def test_a_long_list_beyond_32_bits_of_bytes(ctx):
    """Y of 4.6 GB and dP of 9.2: rows far behind 2^31 bytes, and a gradient that only they give."""
    n, D, H = 9_000_000, 32, 256
    rng = np.random.default_rng(3)
    rows = torch.zeros(n, spp.fp8_row_bytes(D), dtype=torch.uint8, device=DEV)
    pick = torch.tensor([0, 4_194_304, 8_388_608, n - 2, n - 1], device=DEV)
    few = _rows(rng, len(pick), D)
    rows[pick] = _dev(few)
    w = _rows(rng, 2 * H, D, D ** -0.5)
    x, (wg, wu) = R.values(few, D), _split(w, H, D)
    y = spp.fp8_product(ctx, rows, _dev(w)[:H], D)
    _close(y[pick], *R.sums(x, wg, 16), torch.bfloat16)
    assert int(y[1:4_194_304].count_nonzero()) == 0
    spp.fp8_gated(ctx, rows, _dev(w), D, out=y)
    _close(y[pick], *R.gated(x, wg, wu, "silu", 16), torch.bfloat16)
    assert int(y[1:4_194_304].count_nonzero()) == 0
    y.fill_(1.0)
    dp = torch.full((n, 2 * H), 7.0, dtype=torch.bfloat16, device=DEV)
    spp.fp8_gated_grad(ctx, [(rows, n, None, y)], [(rows, n, None, dp)], _dev(w), D)
    want, bound = R.gated_grad(x, wg, wu, np.ones((len(pick), H)), "silu", 16)
    _close(dp[pick], want, bound, torch.bfloat16)
    assert int(dp[1:4_194_304].count_nonzero()) == 0 and int(dp[-3].count_nonzero()) == 0
    p = dp[pick].double().cpu().numpy()
    g = spp.fp8_weight_grad(ctx, [(rows, n, None, dp)], 2 * H, D)[0]
    _close(g, p.T @ x, 3 * len(pick) * 2.0 ** -23 * (np.abs(p).T @ np.abs(x)), torch.float32)


def _step(c, x, wf, rows, w, lists, dys, dps, dw, D, H, act):
    """A gated layer's training step: its input and weights to 8 bits, forward, backward, the weights' gradient."""
    spp.fp8_quantize(c, x, out=rows, sync=False)
    spp.fp8_quantize(c, wf, out=w, sync=False)
    spp.fp8_gated_multi(c, lists, w, D, activation=act, sync=False)
    spp.fp8_gated_grad(c, dys, dps, w, D, activation=act, sync=False)
    spp.fp8_weight_grad(c, dps, 2 * H, D, out=dw, sync=False)


@pytest.mark.parametrize("D,H", [(128, 64), (300, 47), (1024, 130), (1200, 40)])
def test_recorded_into_a_graph_and_replayed(ctx, D, H):
    rng = np.random.default_rng(8)
    n = 900
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c = spp.Context(0, side)
        x, wf = torch.randn(n, D, device=DEV), torch.randn(2 * H, D, device=DEV) * D ** -0.5
        rows, w = spp.fp8_quantize(c, x), spp.fp8_quantize(c, wf)
        y, dy = (torch.randn(n, H, device=DEV).to(torch.bfloat16) for _ in range(2))
        dp = torch.zeros(n, 2 * H, dtype=torch.bfloat16, device=DEV)
        dw = torch.empty(1, 2 * H, D, device=DEV)
        count = torch.tensor([n], dtype=torch.int64, device=DEV)
        lists, dys, dps = (spp.RowLists([(rows, n, count, v)]) for v in (y, dy, dp))
        args = (c, x, wf, rows, w, lists, dys, dps, dw, D, H, "gelu")
        _step(*args)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            _step(*args)
        for k in range(4):
            x.copy_(torch.from_numpy(rng.standard_normal((n, D))))
            count.fill_(n - 100 * k)
            y.zero_()
            dp.zero_()
            graph.replay()
            side.synchronize()
            got = y.clone(), dp.clone(), dw.clone()
            y.zero_()
            dp.zero_()
            _step(*args)
            side.synchronize()
            assert torch.equal(got[0], y) and torch.equal(got[1], dp) and torch.equal(got[2], dw)
            assert int(y[n - 100 * k:].count_nonzero()) == 0 and int(dp[n - 100 * k:].count_nonzero()) == 0 and int(y[:n - 100 * k].count_nonzero()) > 0
    c.close()


def test_two_layers_forward_and_backward(ctx):
    """Gathered rows in 4 bits through the first layer, its output in 8 bits through a gated layer and an output layer, and back, as a training
    step does; each piece is what 64 bits give for its own inputs, and the whole is near a model in 64 bits."""
    rng = np.random.default_rng(21)
    n, D0, D, H, C = 500, 100, 64, 96, 24
    feats = torch.from_numpy(rng.standard_normal((n, D0))).float().to(DEV)
    w0 = torch.from_numpy(rng.standard_normal((D, D0))).float().to(DEV) * D0 ** -0.5
    # weights that 8 bits hold exactly, under a scale by rows or by columns: eighths up to one
    w1 = torch.from_numpy(rng.integers(-8, 9, (2 * H, D)) / 8).float().to(DEV)
    w2 = torch.from_numpy(rng.integers(-8, 9, (C, H)) / 8).float().to(DEV)
    h0 = spp.mx4_product(ctx, spp.mx4_quantize(ctx, feats, sync=False), spp.mx4_quantize(ctx, w0, sync=False), D0, dtype=torch.float32, sync=False)
    x1 = spp.fp8_quantize(ctx, h0, sync=False)
    q1, q2 = spp.fp8_quantize(ctx, w1, sync=False), spp.fp8_quantize(ctx, w2, sync=False)
    a1 = spp.fp8_gated(ctx, x1, q1, D, dtype=torch.float32, sync=False)
    x2 = spp.fp8_quantize(ctx, a1, sync=False)
    out = spp.fp8_product(ctx, x2, q2, H, dtype=torch.float32, sync=False)
    dout = torch.from_numpy(rng.standard_normal((n, C))).float().to(DEV)
    dw2 = spp.fp8_weight_grad(ctx, [(x2, n, None, dout)], C, H, sync=False)[0]
    da1 = spp.fp8_product(ctx, spp.fp8_quantize(ctx, dout, sync=False), spp.fp8_quantize(ctx, w2.T.contiguous(), sync=False), C, dtype=torch.float32, sync=False)
    dp = torch.empty(n, 2 * H, device=DEV)
    grads = spp.RowLists([(x1, n, None, dp)])
    spp.fp8_gated_grad(ctx, [(x1, n, None, da1)], grads, q1, D, sync=False)
    dw1 = spp.fp8_weight_grad(ctx, grads, 2 * H, D, sync=False)[0]
    dx1 = spp.fp8_product(ctx, spp.fp8_quantize(ctx, dp, sync=False), spp.fp8_quantize(ctx, w1.T.contiguous(), sync=False), 2 * H, dtype=torch.float32)

    f = lambda t: t.double().cpu().numpy()
    v1, v2 = R.values(x1.cpu().numpy(), D), R.values(x2.cpu().numpy(), H)
    assert (R.values(q1.cpu().numpy(), D) == f(w1)).all() and (R.values(q2.cpu().numpy(), H) == f(w2)).all()
    _close(a1, *R.gated(v1, f(w1)[:H], f(w1)[H:], "silu"), torch.float32)
    _close(out, *R.sums(v2, f(w2)), torch.float32)
    _close(dw2, f(dout).T @ v2, 3 * n * 2.0 ** -23 * (np.abs(f(dout)).T @ np.abs(v2)), torch.float32)
    _close(dp, *R.gated_grad(v1, f(w1)[:H], f(w1)[H:], f(da1), "silu"), torch.float32)
    _close(dw1, f(dp).T @ v1, 3 * n * 2.0 ** -23 * (np.abs(f(dp)).T @ np.abs(v1)), torch.float32)
    # the rows' gradients come from gradients in 8 bits: each off by at most 2^-4 of itself, or of the smallest normal code, 2^-6 of a
    # scale that is below a 224th of the row's largest
    for got, d, w in ((da1, f(dout), f(w2)), (dx1, f(dp), f(w1))):
        off = 2.0 ** -4 * np.maximum(np.abs(d), 2.0 ** -6 / 224 * np.abs(d).max(1, keepdims=True))
        assert (np.abs(f(got) - d @ w) <= off @ np.abs(w) + d.shape[1] * 2.0 ** -22 * (np.abs(d) @ np.abs(w))).all()


def test_no_lists_and_empty_lists(ctx):
    D, H = 64, 32
    w = spp.fp8_quantize(ctx, torch.randn(2 * H, D, device=DEV))
    spp.fp8_product_multi(ctx, [], w, D)
    spp.fp8_gated_multi(ctx, [], w, D)
    spp.fp8_gated_grad(ctx, [], [], w, D)
    assert int(spp.fp8_weight_grad(ctx, [], H, D, groups=3, out=torch.full((3, H, D), 5.0, device=DEV)).count_nonzero()) == 0
    none = torch.zeros(0, spp.fp8_row_bytes(D), dtype=torch.uint8, device=DEV)
    y, p = torch.zeros(0, H, device=DEV), torch.zeros(0, 2 * H, device=DEV)
    spp.fp8_gated_multi(ctx, [(none, 0, None, y)] * 3, w, D)
    spp.fp8_gated_grad(ctx, [(none, 0, None, y)] * 3, [(none, 0, None, p)] * 3, w, D)
    assert int(spp.fp8_weight_grad(ctx, [(none, 0, None, p)] * 3, 2 * H, D, out=torch.full((1, 2 * H, D), 5.0, device=DEV)).count_nonzero()) == 0
    some, zero = torch.zeros(9, spp.fp8_row_bytes(D), dtype=torch.uint8, device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV)
    out, wide = torch.full((9, H), 3.0, device=DEV), torch.full((9, 2 * H), 3.0, device=DEV)
    spp.fp8_product_multi(ctx, [(some, 9, zero, wide)], w, D)
    spp.fp8_gated_multi(ctx, [(some, 9, zero, out)], w, D)
    spp.fp8_gated_grad(ctx, [(some, 9, zero, out)], [(some, 9, zero, wide)], w, D)
    assert (out == 3).all() and (wide == 3).all()


def test_on_a_stream_that_is_not_the_current_one():
    """The context's stream does the work and owns what the calls allocate; the caller orders the streams."""
    side = torch.cuda.Stream()
    c = spp.Context(0, side)
    n, D, H = 5000, 128, 64
    x, wf = torch.randn(n, D, device=DEV), torch.randn(2 * H, D, device=DEV) * 0.1
    side.wait_stream(torch.cuda.current_stream())
    rows, w = spp.fp8_quantize(c, x, sync=False), spp.fp8_quantize(c, wf, sync=False)
    y = spp.fp8_gated(c, rows, w, D, sync=False)
    z = spp.fp8_product(c, rows, w, D, sync=False)
    g = spp.fp8_weight_grad(c, [(rows, n, None, z)], 2 * H, D, sync=False)
    back = spp.fp8_dequantize(c, rows, D, sync=False)
    torch.cuda.current_stream().wait_stream(side)
    v, wv = R.values(rows.cpu().numpy(), D), R.values(w.cpu().numpy(), D)
    assert torch.equal(back.double().cpu(), torch.from_numpy(v))
    _close(z, *R.sums(v, wv, 16), torch.bfloat16)
    _close(y, *R.gated(v, wv[:H], wv[H:], "silu", 16), torch.bfloat16)
    p = z.double().cpu().numpy()
    _close(g[0], p.T @ v, 3 * n * 2.0 ** -23 * (np.abs(p).T @ np.abs(v)), torch.float32)
    c.close()


@pytest.mark.parametrize("D,H,n", [(100, 256, 500), (33, 47, 100), (700, 300, 200), (1000, 70, 300), (256, 64, 3), (160, 512, 400), (1100, 20, 70)])
def test_what_lies_behind_the_scales_does_not_matter(ctx, D, H, n):
    rng = np.random.default_rng(D + H)
    rows, w = _rows(rng, n, D), _rows(rng, 2 * H, D, D ** -0.5)
    x, (wg, wu) = R.values(rows, D), _split(w, H, D)
    behind = R.code_bytes(D) + -(-D // 128)
    rows[:, behind:] = 255
    w[:, behind:] = 255
    xd, wd = _dev(rows), _dev(w)
    _close(spp.fp8_product(ctx, xd, wd[:H], D, dtype=torch.float32), *R.sums(x, wg), torch.float32)
    y = spp.fp8_gated(ctx, xd, wd, D, dtype=torch.float32)
    _close(y, *R.gated(x, wg, wu, "silu"), torch.float32)
    g = spp.fp8_weight_grad(ctx, [(xd, n, None, y)], H, D)[0]
    v = y.double().cpu().numpy()
    _close(g, v.T @ x, 3 * n * 2.0 ** -23 * (np.abs(v).T @ np.abs(x)), torch.float32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,D,H,pad,offset", [(300, 32, 255, 0, 0), (130, 64, 513, 0, 0), (300, 64, 500, 0, 0), (12800, 32, 300, 0, 0), (12801, 32, 301, 0, 1),
                                              (700, 200, 1001, 0, 0), (700, 200, 1001, 3, 5), (300, 700, 500, 0, 3), (300, 500, 999, 1, 1), (5000, 40, 64, 64, 0),
                                              (5000, 40, 64, 1, 0), (70, 96, 2, 0, 0), (4000, 128, 1, 0, 0), (33000, 256, 256, 0, 0), (270000, 32, 64, 0, 0),
                                              (1100000, 32, 5, 0, 0), (20000, 1024, 192, 64, 0)])
def test_rows_of_any_length_and_address(ctx, dtype, n, D, H, pad, offset):
    """Rows that are lines, rows that are not, rows with gaps, of all three layers; nothing between or behind the rows is touched."""
    rng = np.random.default_rng(n + 3 * D + 7 * H + pad)
    pool = _rows(rng, min(n, 5003), D)
    rows, w = pool[rng.integers(0, len(pool), n)], _rows(rng, 2 * H, D, D ** -0.5)
    xd, wd = _dev(rows), _dev(w)
    pick = np.unique(np.concatenate([np.arange(min(n, 300)), np.arange(max(0, n - 300), n), rng.integers(0, n, 300)]))
    at = torch.from_numpy(pick).to(DEV)
    x, (wg, wu) = R.values(rows[pick], D), _split(w, H, D)
    whole, wt = spp.fp8_dequantize(ctx, xd, D), spp.fp8_dequantize(ctx, wd, D)
    def matrix(cols):
        buf = torch.full((offset + n * (cols + pad) + 64,), 7.0, dtype=dtype, device=DEV)
        return buf, torch.as_strided(buf, (n, cols), (cols + pad, 1), offset)
    def between(buf, cols):
        keep = torch.ones(buf.numel(), dtype=torch.bool, device=DEV)
        keep.as_strided((n, cols), (cols + pad, 1), offset).fill_(False)
        assert (buf[keep] == 7).all()
    def near(got, full):
        assert torch.allclose(got.float(), full, rtol=2.0 ** -7, atol=1e-4 * float(full.abs().max()))       # every row is where it belongs
    g, u = whole @ wt[:H].T, whole @ wt[H:].T
    buf, y = matrix(H)
    spp.fp8_product(ctx, xd, wd[:H], D, out=y)
    _close(y[at], *R.sums(x, wg, _bits(dtype)), dtype)
    near(y, g)
    between(buf, H)
    buf, y = matrix(H)
    spp.fp8_gated(ctx, xd, wd, D, out=y)
    _close(y[at], *R.gated(x, wg, wu, "silu", _bits(dtype)), dtype)
    s = torch.sigmoid(g)
    near(y, g * s * u)
    between(buf, H)
    buf, dy = matrix(H)
    dy[:] = torch.randn(n, H, generator=torch.Generator(DEV).manual_seed(n), device=DEV).to(dtype)
    pbuf, dp = matrix(2 * H)
    spp.fp8_gated_grad(ctx, [(xd, n, None, dy)], [(xd, n, None, dp)], wd, D)
    _close(dp[at], *R.gated_grad(x, wg, wu, dy[at].double().cpu().numpy(), "silu", _bits(dtype)), dtype)
    near(dp, torch.cat([dy.float() * u * s * (1 + g * (1 - s)), dy.float() * g * s], 1))
    between(pbuf, 2 * H)
    between(buf, H)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("further", [0, 1])
@pytest.mark.parametrize("n,D,H", [(70, 100, 70), (70, 700, 300), (33, 1000, 47)])
def test_rows_of_results_gigabytes_apart(ctx, dtype, further, n, D, H):
    """33 rows within 2^31 bytes by a hair, and not by a hair: offsets of 32 bits from a tile's first row, and of 64."""
    es = torch.empty(0, dtype=dtype).element_size()
    ld = (2 ** 31 - 1) // (33 * es) + further
    rng = np.random.default_rng(D + H)
    rows, w = _rows(rng, n, D), _rows(rng, 2 * H, D, D ** -0.5)
    x, (wg, wu) = R.values(rows, D), _split(w, H, D)
    xd, wd = _dev(rows), _dev(w)
    buf = torch.full((n * ld,), 7.0, dtype=dtype, device=DEV)
    y, p = buf.as_strided((n, H), (ld, 1)), buf.as_strided((n, 2 * H), (ld, 1), H)
    spp.fp8_product(ctx, xd, wd[:H], D, out=y)
    _close(y, *R.sums(x, wg, _bits(dtype)), dtype)
    spp.fp8_gated(ctx, xd, wd, D, out=y)
    _close(y, *R.gated(x, wg, wu, "silu", _bits(dtype)), dtype)
    dy = torch.from_numpy(rng.standard_normal((n, H))).to(dtype)
    y.copy_(dy)
    spp.fp8_gated_grad(ctx, [(xd, n, None, y)], [(xd, n, None, p)], wd, D)
    _close(p, *R.gated_grad(x, wg, wu, dy.double().numpy(), "silu", _bits(dtype)), dtype)
    assert torch.equal(y.cpu(), dy)
    g = spp.fp8_weight_grad(ctx, [(xd, n, None, p)], 2 * H, D)[0]
    v = p.double().cpu().numpy()
    _close(g, v.T @ x, 3 * n * 2.0 ** -23 * (np.abs(v).T @ np.abs(x)), torch.float32)
    y.fill_(7.0)
    p.fill_(7.0)
    assert all(bool((part == 7).all()) for part in buf.split(1 << 28))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D,H", [(300, 70), (300, 700), (640, 47), (1200, 70)])
def test_scales_that_quantising_does_not_give(ctx, dtype, D, H):
    """A scale of 2^-127 to 2^113, and NaN: a value below 2^-126 may count as zero, which moves a sum by as much times the other factor."""
    rng = np.random.default_rng(D)
    n, at = 40, R.code_bytes(D)
    rows, w = _rows(rng, n, D), _rows(rng, H, D, D ** -0.5)
    rows[0, at:at + 2] = 0
    rows[1, at + 1] = 255
    rows[2, at] = 240
    rows[3, at:at + 3] = (1, 2, 3)
    rows[4, at:at + 3] = (9, 127, 0)
    w[5, at:at + 2] = 0
    w[6, at + 2] = 255
    xd, wd = _dev(rows), _dev(w)
    x, wv = R.values(rows, D), R.values(w, D)
    y = spp.fp8_product(ctx, xd, wd, D, dtype=dtype)
    assert y[1].isnan().all() and y[:, 6].isnan().all()
    keep, cols = np.arange(n) != 1, np.arange(H) != 6
    x, wv = x[keep], wv[cols]
    want, bound = R.sums(x, wv, _bits(dtype))
    lost = 2.0 ** -126 * (np.abs(wv).sum(1)[None] + np.abs(x).sum(1)[:, None])
    _close(y.cpu()[keep][:, cols], want, bound + lost + 2.0 ** -126, dtype)
    v = torch.from_numpy(rng.standard_normal((n, H))).to(dtype)
    v[1] = 0
    clean = rows.copy()
    clean[1] = 0
    g = spp.fp8_weight_grad(ctx, [(_dev(clean), n, None, v.to(DEV))], H, D)[0]
    v = v.double().numpy()
    x = R.values(clean, D)
    _close(g, v.T @ x, 3 * n * 2.0 ** -23 * (np.abs(v).T @ np.abs(x)) + 2.0 ** -126 * (1 + np.abs(v).sum(0)[:, None]), torch.float32)


def test_the_same_rows_under_several_matrices_and_in_several_lists(ctx):
    """One hidden matrix, a list for each of five groups, and the same list three times: as separate calls."""
    rng = np.random.default_rng(21)
    n, D, H, G = 333, 160, 70, 5
    xd, w = _dev(_rows(rng, n, D)), _dev(_rows(rng, G * 2 * H, D, D ** -0.5)).view(G, 2 * H, -1)
    groups = [0, 1, 2, 3, 4, 2, 2]
    y = [torch.zeros(n, H, dtype=torch.bfloat16, device=DEV) for _ in groups]
    dy = [torch.randn(n, H, device=DEV).to(torch.bfloat16) for _ in groups]
    p = [torch.zeros(n, 2 * H, dtype=torch.bfloat16, device=DEV) for _ in groups]
    spp.fp8_gated_multi(ctx, [(xd, n, None, v, g) for v, g in zip(y, groups)], w, D)
    spp.fp8_gated_grad(ctx, [(xd, n, None, v, g) for v, g in zip(dy, groups)], [(xd, n, None, v, g) for v, g in zip(p, groups)], w, D)
    one = torch.empty(n, 2 * H, dtype=torch.bfloat16, device=DEV)
    for j, g in enumerate(groups):
        assert torch.equal(y[j], spp.fp8_gated(ctx, xd, w[g].contiguous(), D))
        spp.fp8_gated_grad(ctx, [(xd, n, None, dy[j])], [(xd, n, None, one)], w[g].contiguous(), D)
        assert torch.equal(p[j], one)
    dw = spp.fp8_weight_grad(ctx, [(xd, n, None, v, g) for v, g in zip(p, groups)], 2 * H, D, groups=G)
    x = R.values(xd.cpu().numpy(), D)
    for g in range(G):
        v = np.concatenate([p[j].double().cpu().numpy() for j in range(len(groups)) if groups[j] == g])
        xs = np.concatenate([x] * groups.count(g))
        _close(dw[g], v.T @ xs, 3 * len(v) * 2.0 ** -23 * (np.abs(v).T @ np.abs(xs)), torch.float32)


def test_two_contexts_at_once(ctx):
    """Two streams work at the same time, each context with a workspace of its own: as one after the other."""
    sides = [torch.cuda.Stream() for _ in range(2)]
    cs = [spp.Context(0, s) for s in sides]
    n, D, H = 30000, 200, 150
    x = [torch.randn(n, D, device=DEV) for _ in cs]
    wf = [torch.randn(2 * H, D, device=DEV) * D ** -0.5 for _ in cs]
    dy = torch.randn(n, H, device=DEV)
    def step(c, k, dp):
        rows, w = spp.fp8_quantize(c, x[k], sync=False), spp.fp8_quantize(c, wf[k], sync=False)
        y = spp.fp8_gated(c, rows, w, D, dtype=torch.float32, sync=False)
        spp.fp8_gated_grad(c, [(rows, n, None, dy)], [(rows, n, None, dp)], w, D, sync=False)
        return rows, w, y, dp, spp.fp8_weight_grad(c, [(rows, n, None, dp)], 2 * H, D, sync=False)
    torch.cuda.synchronize()
    want = []
    for k in range(2):
        want.append(step(ctx, k, torch.empty(n, 2 * H, device=DEV)))
        ctx.sync()
    dps = [torch.empty(n, 2 * H, device=DEV) for _ in range(8)]
    torch.cuda.synchronize()
    got = [step(cs[j % 2], j % 2, dps[j]) for j in range(8)]
    for s in sides:
        s.synchronize()
    for j, g in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(g, want[j % 2]))
    for c in cs:
        c.close()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D,H", [(172, 100), (100, 86), (128, 256), (300, 47), (500, 64)])
def test_the_same_bits_for_few_rows_and_for_many(ctx, dtype, D, H):
    """A row's results do not depend on how many other rows the call has, whatever form its kernel takes for them."""
    rng = np.random.default_rng(D + H)
    n = 70000
    xd, w = _dev(_rows(rng, 4096, D)), _dev(_rows(rng, 2 * H, D, D ** -0.5))
    xd = xd.repeat(-(-n // 4096), 1)[:n].contiguous()
    dy = torch.randn(n, H, generator=torch.Generator(DEV).manual_seed(1), device=DEV).to(dtype)
    def results(count):
        dp = torch.full((count, 2 * H), float("nan"), dtype=dtype, device=DEV)
        spp.fp8_gated_grad(ctx, [(xd[:count], count, None, dy[:count])], [(xd[:count], count, None, dp)], w, D)
        return spp.fp8_product(ctx, xd[:count], w[:H], D, dtype=dtype), spp.fp8_gated(ctx, xd[:count], w, D, dtype=dtype), dp
    want = results(n)
    assert not any(bool(t.isnan().any()) for t in want)
    for count in (1, 3, 100, 4000, 20000, 40000, 66000):
        for got, t in zip(results(count), want):
            assert torch.equal(got, t[:count]), count

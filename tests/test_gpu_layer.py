"""The product of MXFP4 rows with weights and its gradient against sums in 64 bits, over lists, groups, types and strides.

Tolerances.  The product of two values in MXFP4 has 6 bits at most and a value in MXFP4 times an fp32 cut in pieces of bf16 is exact
piece by piece: only the sums round.  Adding K terms in fp32 in any order, each addition off by at most 2^-23 of its result
(cut off rather than rounded), is off by at most K 2^-23 sum|term|; an fp32 gradient has three terms a row.  Rounding the sum to
16 bits adds half a step: 2^-8 of it in bf16 (8 significant bits), 2^-11 in fp16 or half of the smallest step, 2^-25.
"""
import numpy as np
import pytest
import torch

import mx4_reference as R
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


def _rows(rng, n, D, spread=4):
    nb = -(-D // 32)
    rows = np.zeros((n, R.row_bytes(D)), np.uint8)
    codes = rng.integers(0, 256, (n, nb * 16)).astype(np.uint8)
    if D % 32:                                                    # as the quantiser leaves the last block
        codes[:, D // 2 + D % 2:] = 0
        if D % 2:
            codes[:, D // 2] &= 15
    rows[:, :16 * nb] = codes
    rows[:, 16 * nb:17 * nb] = rng.integers(125 - spread, 125 + spread, (n, nb))
    return rows


def _close(got, want, size, K, dtype):
    got = got.double().cpu().numpy()
    bound = K * 2.0 ** -23 * size
    bound = bound + STEP[dtype] * (np.abs(want) + bound) + (2.0 ** -25 if dtype == torch.float16 else 0)
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (int(bad.sum()), float(np.abs(got - want)[bad].max()), np.argwhere(bad)[:4])


def _product(rows, w, D):
    x, v = R.values(rows, D), R.values(w, D)
    return x @ v.T, np.abs(x) @ np.abs(v).T


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,D,H", [(1, 1, 1), (1, 128, 256), (2, 32, 47), (15, 33, 64), (16, 100, 172), (17, 128, 65), (127, 96, 63),
                                   (128, 160, 128), (129, 100, 256), (255, 256, 47), (257, 300, 172), (700, 768, 1024), (65, 1024, 40),
                                   (63, 1100, 130), (130, 4096, 24), (1, 768, 1024), (5, 1, 1100), (3000, 31, 33)])
def test_product_of_one_list(ctx, dtype, n, D, H):
    rng = np.random.default_rng(n * 7 + D * 3 + H)
    rows, w = _rows(rng, n, D), _rows(rng, H, D)
    y = spp.mx4_product(ctx, torch.from_numpy(rows).to(DEV), torch.from_numpy(w).to(DEV), D, dtype=dtype)
    want, size = _product(rows, w, D)
    _close(y, want, size, D, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,D,H", [(1, 1, 1), (1, 128, 256), (2, 32, 47), (31, 33, 64), (33, 100, 172), (63, 128, 129), (64, 96, 128),
                                   (65, 160, 127), (129, 100, 256), (700, 256, 47), (1500, 768, 300), (300, 1100, 130), (4000, 31, 33),
                                   (20000, 128, 256), (130, 4096, 24)])
def test_gradient_of_one_list(ctx, dtype, n, D, H):
    rng = np.random.default_rng(n * 7 + D * 3 + H + 1)
    rows = _rows(rng, n, D)
    y = torch.from_numpy(rng.standard_normal((n, H))).to(dtype)
    g = spp.mx4_weight_grad(ctx, [(torch.from_numpy(rows).to(DEV), n, None, y.to(DEV))], H, D)
    x, v = R.values(rows, D), y.double().numpy()
    assert g.shape == (1, H, D)
    _close(g[0], v.T @ x, np.abs(v).T @ np.abs(x), 3 * n, torch.float32)


def _many(rng, lists, groups, D, H, dtype, pad=0, offset=0):
    """Lists whose capacity exceeds their count, on the device for some; what lies behind the count must not matter."""
    items, plain = [], []
    for j in range(lists):
        cap = int(rng.integers(0, 400)) if j % 7 else int(rng.integers(0, 3))
        n = int(rng.integers(0, cap + 1)) if j % 5 else 0
        rows = _rows(rng, cap, D)
        if cap > n:
            rows[n:] = 255                                        # NaN scales
        buf = torch.full((offset + cap * (H + pad) + 16,), float("nan"), dtype=dtype, device=DEV)
        y = torch.as_strided(buf, (cap, H), (H + pad, 1), offset)
        y[:n] = torch.from_numpy(rng.standard_normal((n, H))).to(DEV, dtype)
        on_device = j % 2 == 0 or n == cap
        count = torch.tensor([n if j % 4 else (n if n < cap else cap + 17)], dtype=torch.int64, device=DEV) if on_device else None
        items.append((torch.from_numpy(rows).to(DEV), cap if on_device else n, count, y, int(rng.integers(0, groups))))
        plain.append((rows[:n], n))
    return items, plain


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lists,groups,D,H,pad,offset", [(1, 1, 128, 256, 0, 0), (64, 1, 128, 96, 0, 0), (64, 64, 100, 48, 8, 8), (24, 8, 100, 172, 0, 0),
                                                         (9, 3, 50, 77, 3, 1), (3, 5, 32, 130, 0, 0), (12, 2, 600, 200, 24, 16)])
def test_lists_and_groups_both_ways(ctx, dtype, lists, groups, D, H, pad, offset):
    rng = np.random.default_rng(lists * 100 + groups + D)
    items, plain = _many(rng, lists, groups, D, H, dtype, pad, offset)
    w = _rows(rng, groups * H, D)
    wt = torch.from_numpy(w).to(DEV).view(groups, H, -1)
    # the gradient first: the product overwrites y
    grad = spp.mx4_weight_grad(ctx, items, H, D, groups=groups)
    want, size, K = np.zeros((groups, H, D)), np.zeros((groups, H, D)), 1
    for (rows, n), it in zip(plain, items):
        x, v = R.values(rows, D), it[3][:n].double().cpu().numpy()
        want[it[4]] += v.T @ x
        size[it[4]] += np.abs(v).T @ np.abs(x)
        K += 3 * n
    _close(grad, want, size, K, torch.float32)
    empty = [g for g in range(groups) if not any(it[4] == g and n for (_, n), it in zip(plain, items))]
    assert all(int(grad[g].count_nonzero()) == 0 for g in empty)
    again = spp.mx4_weight_grad(ctx, spp.RowLists(items), H, D, groups=groups)
    assert torch.equal(grad, again)
    before = [it[3].clone() for it in items]
    held = [torch.as_strided(it[3], (max(it[3].shape[0] - 1, 0), pad), (H + pad, 1), it[3].storage_offset() + H).clone() for it in items if pad]
    spp.mx4_product_multi(ctx, spp.RowLists(items), wt, D)
    for (rows, n), it, b in zip(plain, items, before):
        want, size = _product(rows, w.reshape(groups, H, -1)[it[4]], D)
        _close(it[3][:n], want, size, D, dtype)
        assert torch.equal(torch.isnan(it[3][n:]), torch.isnan(b[n:])) and torch.isnan(it[3][n:]).all()
    after = [torch.as_strided(it[3], (max(it[3].shape[0] - 1, 0), pad), (H + pad, 1), it[3].storage_offset() + H) for it in items if pad]
    assert all(torch.equal(torch.isnan(a), torch.isnan(b)) for a, b in zip(held, after))


def test_nan_scales_and_infinities_stay_in_their_rows(ctx):
    rng = np.random.default_rng(5)
    n, D, H = 200, 100, 80
    rows, w = _rows(rng, n, D), _rows(rng, H, D)
    rows[17, 16 * 4 + 2] = 255
    w[33, 16 * 4] = 255
    y = spp.mx4_product(ctx, torch.from_numpy(rows).to(DEV), torch.from_numpy(w).to(DEV), D, dtype=torch.float32).cpu()
    nan = torch.zeros(n, H, dtype=torch.bool)
    nan[17], nan[:, 33] = True, True
    assert torch.equal(torch.isnan(y), nan)
    for dtype in TYPES:
        g = torch.zeros(n, H, dtype=dtype)
        g[:] = torch.from_numpy(rng.standard_normal((n, H)))
        g[5, 7], g[6, 8], g[90, 9] = float("inf"), float("nan"), -float("inf")
        clean = _rows(rng, n, D)
        clean[[5, 6, 90], :64] = 0x22                             # ones: infinite sums keep their sign
        d = spp.mx4_weight_grad(ctx, [(torch.from_numpy(clean).to(DEV), n, None, g.to(DEV))], H, D)[0].cpu()
        x = R.values(clean, D)
        with np.errstate(invalid="ignore"):
            want = torch.from_numpy(g.double().numpy().T @ x)
        assert torch.equal(torch.isnan(d), torch.isnan(want)) and torch.equal(torch.isinf(d), torch.isinf(want))
        assert torch.equal(torch.sign(d[torch.isinf(d)]).double(), torch.sign(want[torch.isinf(want)]))


def test_gradient_against_differences(ctx):
    """sum(G * product(X, W)) is linear in each value of W: its slope between two codes is dW there, exactly in 64 bits."""
    rng = np.random.default_rng(11)
    n, D, H = 300, 70, 20
    rows, w = _rows(rng, n, D, 1), _rows(rng, H, D, 1)
    g = torch.from_numpy(rng.integers(-4, 5, (n, H)).astype(np.float32))
    dev = torch.from_numpy(rows).to(DEV)
    grad = spp.mx4_weight_grad(ctx, [(dev, n, None, g.to(DEV))], H, D)[0].cpu().double()
    def loss(wt):
        y = spp.mx4_product(ctx, dev, torch.from_numpy(wt).to(DEV), D, dtype=torch.float32)
        return float((g.double() * y.double().cpu()).sum())
    base = loss(w)
    for h, d in ((0, 0), (3, 31), (7, 32), (19, 69), (11, 40)):
        other = w.copy()
        byte, shift = d // 2, 4 * (d % 2)
        code = (int(w[h, byte]) >> shift) & 15
        other[h, byte] = (int(w[h, byte]) & ~(15 << shift)) | ((code ^ 9) << shift)
        step = R.values(other, D)[h, d] - R.values(w, D)[h, d]
        if step:
            # y has D terms of at most 6*6*4: exact in fp32 here, as multiples of 2^-8 below 2^16
            assert (loss(other) - base) / step == pytest.approx(float(grad[h, d]), abs=1e-9 * n)


def test_a_long_list_beyond_32_bits_of_bytes(ctx):
    """Y of 4.6 GB: rows far behind 2^31 bytes, and a gradient that only they give."""
    n, D, H = 9_000_000, 32, 256
    rng = np.random.default_rng(3)
    rows = torch.zeros(n, spp.mx4_row_bytes(D), dtype=torch.uint8, device=DEV)
    pick = torch.tensor([0, 4_194_304, 8_388_608, n - 2, n - 1], device=DEV)
    few = _rows(rng, len(pick), D)
    rows[pick] = torch.from_numpy(few).to(DEV)
    w = _rows(rng, H, D)
    y = spp.mx4_product(ctx, rows, torch.from_numpy(w).to(DEV), D)
    want, size = _product(few, w, D)
    _close(y[pick], want, size, D, torch.bfloat16)
    assert int(y[1:4_194_304].count_nonzero()) == 0
    y.fill_(1.0)
    g = spp.mx4_weight_grad(ctx, [(rows, n, None, y)], H, D)[0]
    x = R.values(few, D)
    _close(g, np.broadcast_to(x.sum(0), (H, D)), np.broadcast_to(np.abs(x).sum(0), (H, D)), len(pick), torch.float32)


def test_recorded_into_a_graph_and_replayed(ctx):
    rng = np.random.default_rng(8)
    n, D, H = 900, 128, 256
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c = spp.Context(0, side)
        x = torch.randn(n, D, device=DEV)
        wf = torch.randn(H, D, device=DEV) * 0.1
        rows, w = spp.mx4_quantize(c, x), spp.mx4_quantize(c, wf)
        y = torch.empty(n, H, dtype=torch.bfloat16, device=DEV)
        dw = torch.empty(1, H, D, device=DEV)
        count = torch.tensor([n], dtype=torch.int64, device=DEV)
        lists = spp.RowLists([(rows, n, count, y)])
        def work():
            spp.mx4_quantize(c, x, out=rows, sync=False)
            spp.mx4_quantize(c, wf, out=w, sync=False)
            spp.mx4_product_multi(c, lists, w, D, sync=False)
            spp.mx4_weight_grad(c, lists, H, D, out=dw, sync=False)
        work()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            work()
        for k in range(4):
            x.copy_(torch.from_numpy(rng.standard_normal((n, D))))
            count.fill_(n - 100 * k)
            y.zero_()
            graph.replay()
            side.synchronize()
            got = y.clone(), dw.clone()
            y.zero_()
            work()
            side.synchronize()
            assert torch.equal(got[0], y) and torch.equal(got[1], dw) and int(y[n - 100 * k:].count_nonzero()) == 0
    c.close()


def test_a_training_step_of_the_layer_on_gathered_rows(ctx):
    """Sample, gather rows in 4 bits, product, gradient, AdamW, weights quantised again: the loss falls, and each piece is what
    64 bits give for it."""
    import workloads.synth as S
    cfg = S.TINY
    g = S.make_graph(cfg, "cpu")
    T = S.local_training_set(cfg, S.make_training_set(cfg, "cpu"))
    lo, hi = cfg.bounds()
    G = spp.Graph(ctx, g.rowptr.to(DEV), g.col.to(DEV))
    x = S.feature_block(cfg, 0, cfg.N, "cpu")
    rows = spp.mx4_quantize(ctx, x.to(DEV))
    remote = torch.cat([rows[:lo], rows[hi:]]).cpu().pin_memory()
    local = rows[lo:hi].contiguous()
    H = 47
    truth = torch.randn(H, cfg.D, generator=torch.Generator().manual_seed(1)).to(DEV) / cfg.D ** 0.5
    wf = torch.zeros(H, cfg.D, device=DEV)
    opt = spp.AdamW(ctx, [wf], state_bits=8, lr=0.02, weight_decay=0.0)
    bufs = [spp.MFGBuffers(DEV, cfg.B, cfg.fanouts, cfg.N) for _ in range(2)]
    out = [torch.empty(b.node_ids.numel(), local.shape[1], dtype=torch.uint8, device=DEV) for b in bufs]
    y = [torch.empty(o.shape[0], H, dtype=torch.float32, device=DEV) for o in out]
    lists = spp.RowLists([(o, o.shape[0], b.n_final_device, v) for o, b, v in zip(out, bufs, y)])
    losses = []
    for step in range(60):
        spp.sample_mfg_multi(ctx, G, [(b_seeds.to(DEV), 2 * step + k, b) for k, (b_seeds, b) in enumerate(zip([T[:64], T[64:128]], bufs))],
                             cfg.fanouts, 4, sync=False)
        spp.gather_features_multi(ctx, None, local, cfg.N, lo, hi, remote, [(b.node_ids, o.shape[0], b.n_final_device, o) for b, o in zip(bufs, out)],
                                  sync=False)
        spp.mx4_product_multi(ctx, lists, spp.mx4_quantize(ctx, wf, sync=False), cfg.D, sync=False)
        loss, total = 0.0, 0
        for b, o, v in zip(bufs, out, y):
            n = int(b.n_final_device)
            d = v[:n] - x.to(DEV)[b.node_ids[:n].long()] @ truth.T
            loss, total = loss + float(d.square().sum()), total + n
            v[:n] = 2 * d
        losses.append(loss / total / H)
        dw = spp.mx4_weight_grad(ctx, lists, H, cfg.D, sync=False)
        opt.step([dw[0] / total], sync=False)
    ctx.sync()
    # features off by at most a sixth or so and weights in 4 bits: what is left is their rounding, far below the start
    assert losses[-1] < 0.1 * losses[0], (losses[0], losses[-1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,D,H,pad,offset", [(300, 32, 255, 0, 0), (130, 64, 513, 0, 0), (300, 64, 500, 0, 0), (12800, 32, 300, 0, 0), (12801, 32, 301, 0, 1),
                                              (700, 200, 1001, 0, 0), (700, 200, 1001, 3, 5), (300, 700, 500, 0, 3), (300, 500, 999, 1, 1), (5000, 40, 64, 64, 0),
                                              (5000, 40, 64, 1, 0), (70, 96, 2, 0, 0), (4000, 128, 1, 0, 0), (33000, 128, 256, 0, 0), (270000, 32, 64, 0, 0),
                                              (1100000, 32, 5, 0, 0)])
def test_rows_of_y_of_any_length_and_address(ctx, dtype, n, D, H, pad, offset):
    """Rows that are lines, rows that are put together (whole, or 64 columns at a time, their columns dealt out or not), rows
    with gaps; nothing between or behind them is touched."""
    rng = np.random.default_rng(n + 3 * D + 7 * H + pad)
    rows, w = _rows(rng, n, D), _rows(rng, H, D)
    buf = torch.full((offset + n * (H + pad) + 64,), 7.0, dtype=dtype, device=DEV)
    y = torch.as_strided(buf, (n, H), (H + pad, 1), offset)
    spp.mx4_product(ctx, torch.from_numpy(rows).to(DEV), torch.from_numpy(w).to(DEV), D, out=y)
    pick = np.unique(np.concatenate([np.arange(min(n, 400)), np.arange(max(0, n - 300), n), rng.integers(0, n, 600)]))
    want, size = _product(rows[pick], w, D)
    _close(y[torch.from_numpy(pick).to(DEV)], want, size, D, dtype)
    full = torch.from_numpy(R.values(rows, D)).to(DEV).float() @ torch.from_numpy(R.values(w, D)).to(DEV).float().T
    assert torch.allclose(y.float(), full, rtol=2.0 ** -7, atol=1e-4 * float(full.abs().max()))       # every row is where it belongs
    keep = torch.ones(buf.numel(), dtype=torch.bool, device=DEV)
    keep.as_strided((n, H), (H + pad, 1), offset).fill_(False)
    assert (buf[keep] == 7).all()


@pytest.mark.parametrize("D,H,n", [(100, 256, 500), (33, 47, 100), (700, 300, 200), (1000, 70, 300), (128, 64, 3), (160, 1024, 400)])
def test_what_lies_behind_the_scales_does_not_matter(ctx, D, H, n):
    rng = np.random.default_rng(D + H)
    rows, w = _rows(rng, n, D), _rows(rng, H, D)
    want, size = _product(rows, w, D)
    nb = -(-D // 32)
    rows[:, 17 * nb:] = 255
    w[:, 17 * nb:] = 255
    y = spp.mx4_product(ctx, torch.from_numpy(rows).to(DEV), torch.from_numpy(w).to(DEV), D, dtype=torch.float32)
    _close(y, want, size, D, torch.float32)
    g = spp.mx4_weight_grad(ctx, [(torch.from_numpy(rows).to(DEV), n, None, y)], H, D)[0]
    x, v = R.values(rows, D), y.double().cpu().numpy()
    _close(g, v.T @ x, np.abs(v).T @ np.abs(x), 3 * n, torch.float32)


def test_no_lists_and_empty_lists(ctx):
    D, H = 64, 32
    w = spp.mx4_quantize(ctx, torch.randn(H, D, device=DEV))
    spp.mx4_product_multi(ctx, [], w, D)
    g = spp.mx4_weight_grad(ctx, [], H, D, groups=3, out=torch.full((3, H, D), 5.0, device=DEV))
    assert int(g.count_nonzero()) == 0
    none = torch.zeros(0, spp.mx4_row_bytes(D), dtype=torch.uint8, device=DEV)
    y = torch.zeros(0, H, device=DEV)
    spp.mx4_product_multi(ctx, [(none, 0, None, y)] * 3, w, D)
    g = spp.mx4_weight_grad(ctx, [(none, 0, None, y)] * 3, H, D, out=torch.full((1, H, D), 5.0, device=DEV))
    assert int(g.count_nonzero()) == 0
    some = torch.zeros(9, spp.mx4_row_bytes(D), dtype=torch.uint8, device=DEV)
    out = torch.full((9, H), 3.0, device=DEV)
    zero = torch.zeros(1, dtype=torch.int64, device=DEV)
    spp.mx4_product_multi(ctx, [(some, 9, zero, out)], w, D)
    assert (out == 3).all()


def test_on_a_stream_that_is_not_the_current_one():
    """The context's stream does the work and owns what the calls allocate; the caller orders the streams."""
    side = torch.cuda.Stream()
    c = spp.Context(0, side)
    x = torch.randn(5000, 128, device=DEV)
    wf = torch.randn(256, 128, device=DEV)
    side.wait_stream(torch.cuda.current_stream())
    rows, w = spp.mx4_quantize(c, x, sync=False), spp.mx4_quantize(c, wf, sync=False)
    y = spp.mx4_product(c, rows, w, 128, sync=False)
    g = spp.mx4_weight_grad(c, [(rows, 5000, None, y)], 256, 128, sync=False)
    opt = spp.AdamW(c, [wf], state_bits=8)
    opt.step([g[0]], sync=False)
    m, v = opt.state(sync=False)
    back = spp.mx4_dequantize(c, rows, 128, sync=False)
    torch.cuda.current_stream().wait_stream(side)
    want = back.double() @ torch.from_numpy(R.values(w.cpu().numpy(), 128)).to(DEV).T
    assert (y.double() - want).abs().max() <= 2.0 ** -8 * want.abs().max() + 1e-3
    assert torch.allclose(g[0].double(), y.double().T @ back.double(), rtol=1e-4, atol=1e-2)
    assert torch.isfinite(m[0]).all() and float(m[0].abs().max()) > 0
    c.close()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D,H,ld", [(385, 320, 320), (512, 300, 320), (640, 255, 256), (768, 192, 192), (700, 260, 384)])
def test_many_wide_rows_in_lists_of_any_length(ctx, dtype, D, H, ld):
    """Enough wide rows that a wavefront takes more of them at a time: lists that end inside its rows, inside a workgroup's and with
    them, one whose count is on the device and below its room, two groups; nothing between or behind the rows is touched."""
    rng = np.random.default_rng(D + H)
    sizes = [(0, 0), (1, 1), (47, 47), (48, 48), (49, 49), (383, 383), (384, 384), (385, 385), (100, 0), (70000, 61234), (200001, 200001)]
    pool = _rows(rng, 4099, D)
    w = _rows(rng, 2 * H, D).reshape(2, H, -1)
    items, plain = [], []
    for j, (cap, n) in enumerate(sizes):
        rows = pool[rng.integers(0, len(pool), cap)]
        rows[n:] = 255
        buf = torch.full((cap * ld + 64,), 7.0, dtype=dtype, device=DEV)
        y = torch.as_strided(buf, (cap, H), (ld, 1))
        count = torch.tensor([n], dtype=torch.int64, device=DEV) if cap != n or j % 2 else None
        items.append((torch.from_numpy(rows).to(DEV), cap, count, y, j % 2))
        plain.append((rows, n, buf))
    spp.mx4_product_multi(ctx, spp.RowLists(items), torch.from_numpy(w).to(DEV), D)
    wv = torch.from_numpy(R.values(w.reshape(2 * H, -1), D)).to(DEV).float().view(2, H, D)
    for (rows, n, buf), it in zip(plain, items):
        if n:
            pick = np.unique(np.concatenate([np.arange(min(n, 400)), np.arange(max(0, n - 400), n), rng.integers(0, n, 400)]))
            want, size = _product(rows[pick], w[it[4]], D)
            _close(it[3][torch.from_numpy(pick).to(DEV)], want, size, D, dtype)
            for at in range(0, n, 50000):
                part = rows[at:min(n, at + 50000)]
                full = torch.from_numpy(R.values(part, D)).to(DEV).float() @ wv[it[4]].T
                assert torch.allclose(it[3][at:at + len(part)].float(), full, rtol=2.0 ** -7, atol=1e-4 * float(full.abs().max()))
        keep = torch.ones(buf.numel(), dtype=torch.bool, device=DEV)
        if n:
            keep.as_strided((n, H), (ld, 1)).fill_(False)
        assert (buf[keep] == 7).all()

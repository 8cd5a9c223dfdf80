"""Hidden rows in 8 bits against their definition, bit for bit: every code and scale, every 16-bit value, borders, odd widths, strides."""
import numpy as np
import pytest
import torch

import fp8_reference as R
import paper_2305_03152_amd as spp

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def ctx():
    c = spp.Context(0)
    yield c
    c.close()


def _check(ctx, x):
    rows = spp.fp8_quantize(ctx, x.to(DEV))
    want = R.quantize(x.double().numpy())
    got = rows.cpu().numpy()
    assert got.shape == want.shape and (got == want).all(), np.argwhere(got != want)[:5]
    return rows


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,D", [(1, 1), (1, 256), (3, 7), (5, 16), (9, 17), (64, 32), (65, 33), (31, 48), (40, 64), (33, 65), (17, 100), (300, 128), (16, 129),
                                 (50, 172), (1000, 256), (7, 300), (11, 1024), (5, 1100), (3, 2048), (2, 2049), (3, 4095), (2, 4096), (2000, 40)])
def test_rows_of_any_width(ctx, dtype, n, D):
    rng = np.random.default_rng(n * 5000 + D)
    x = torch.from_numpy(rng.standard_normal((n, D)) * np.exp2(rng.integers(-12, 12, (n, 1)))).to(dtype)
    rows = _check(ctx, x)
    v = R.values(rows.cpu().numpy(), D)
    for out in TYPES:
        back = spp.fp8_dequantize(ctx, rows, D, dtype=out)
        assert torch.equal(back.cpu(), torch.from_numpy(v).to(out))


def test_every_code_under_every_scale(ctx):
    """Values of every code and scale byte, 255 among them, as each type: what lies between is the type's own rounding."""
    D = 256
    rows = np.zeros((256, R.row_bytes(D)), np.uint8)
    rows[:, :256] = np.arange(256)
    rows[:, 256] = rows[:, 257] = np.arange(256)
    v = torch.from_numpy(R.values(rows, D))
    for out in TYPES:
        back = spp.fp8_dequantize(ctx, torch.from_numpy(rows).to(DEV), D, dtype=out).cpu()
        want = v.to(torch.float32).to(out)                             # (fp32 holds all values of scales up to 246, or gives infinity)
        assert torch.equal(torch.isnan(back), torch.isnan(want))
        ok = ~torch.isnan(want)
        assert torch.equal(back[ok], want[ok])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_every_16_bit_value(ctx, dtype):
    """In rows of their own neighbours, in shuffled rows, and each beside a large value: all finite values, signs, subnormals, NaN."""
    every = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(dtype)
    for x in (every.view(512, 128), every[torch.randperm(65536, generator=torch.Generator().manual_seed(1))].view(256, 256)):
        _check(ctx, x)
    x = torch.zeros(65536, 16, dtype=dtype)
    x[:, 3] = every
    _check(ctx, x)


def test_borders_between_codes_and_between_scales(ctx):
    """fp32 values half way between two codes and one step to either side, under scales from the least to the most."""
    mid = (R.MAGNITUDES[1:] + R.MAGNITUDES[:-1]) / 2
    at = np.concatenate([mid, R.MAGNITUDES])
    rng = np.random.default_rng(2)
    blocks = []
    for e in (-117, -100, -30, -1, 0, 7, 60, 118, 119):
        v = (at * 2.0 ** e).astype(np.float32)
        for near in (v, np.nextafter(v, np.float32(np.inf)), np.nextafter(v, np.float32(0))):
            near = np.concatenate([near, np.zeros(-len(near) % 127, np.float32)]).reshape(-1, 127)
            block = np.concatenate([near, np.full((len(near), 1), 448.0 * 2.0 ** e, np.float32)], 1)
            blocks.append(block * rng.choice([-1, 1], block.shape).astype(np.float32))
    _check(ctx, torch.from_numpy(np.concatenate(blocks)))
    # the largest value of a block just at, above and below 448 times a power of two; the smallest and largest there are
    tops = []
    for e in list(range(-130, 120, 7)) + [118, 119]:
        t = np.float32(448.0 * 2.0 ** e)
        tops += [t, np.nextafter(t, np.float32(np.inf)), np.nextafter(t, np.float32(0))]
    tops += [np.float32(v) for v in (0.0, -0.0, 1e-45, 1.1754942e-38, 1.1754944e-38, 3.4028235e38, 3.2e38)]
    x = np.zeros((len(tops), 130), np.float32)
    x[:, 5] = tops
    x[:, 7] = -np.array(tops) / 3
    x[:, 129] = np.array(tops)[::-1]
    _check(ctx, torch.from_numpy(x))


@pytest.mark.parametrize("dtype", TYPES)
def test_what_is_not_finite_is_nan_and_leaves_its_block_alone(ctx, dtype):
    rng = np.random.default_rng(4)
    x = torch.from_numpy(rng.standard_normal((200, 300))).to(dtype)
    x[3, 5], x[3, 200], x[7, 0], x[9, 299], x[11, 128:256], x[13, 127] = float("nan"), float("inf"), -float("inf"), float("nan"), float("inf"), torch.finfo(dtype).max
    rows = _check(ctx, x)
    back = spp.fp8_dequantize(ctx, rows, 300).cpu()
    assert torch.equal(torch.isnan(back), ~torch.isfinite(x))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D,pad,offset", [(256, 8, 0), (256, 3, 1), (100, 28, 4), (33, 0, 1), (128, 128, 8), (16, 5, 3), (1, 2, 1)])
def test_strides_counts_and_what_lies_between(ctx, dtype, D, pad, offset):
    rng = np.random.default_rng(D + pad)
    n, cap = 77, 90
    buf = torch.from_numpy(rng.standard_normal(offset + cap * (D + pad) + 9)).to(dtype)
    dev = buf.to(DEV)
    x = torch.as_strided(dev, (cap, D), (D + pad, 1), offset)
    out = torch.full((cap, spp.fp8_row_bytes(D)), 0xAB, dtype=torch.uint8, device=DEV)
    count = torch.tensor([n], dtype=torch.int64, device=DEV)
    spp.fp8_quantize(ctx, x, out=out, n_device=count)
    want = R.quantize(torch.as_strided(buf, (cap, D), (D + pad, 1), offset)[:n].double().numpy())
    assert (out[:n].cpu().numpy() == want).all() and (out[n:] == 0xAB).all()
    into = torch.full((offset + cap * (D + pad) + 9,), 7.0, dtype=dtype, device=DEV)
    spp.fp8_dequantize(ctx, out, D, out=torch.as_strided(into, (cap, D), (D + pad, 1), offset), n_device=count)
    got = torch.as_strided(into, (cap, D), (D + pad, 1), offset)
    assert torch.equal(got[:n].cpu(), torch.from_numpy(R.values(want, D)).to(dtype)) and (got[n:] == 7).all()
    keep = torch.ones(into.numel(), dtype=torch.bool, device=DEV)
    keep.as_strided((cap, D), (D + pad, 1), offset).fill_(False)
    assert (into[keep] == 7).all()


@pytest.mark.parametrize("count", [-3, 0, 10, 1000])
def test_counts_outside_the_buffers(ctx, count):
    x = torch.randn(10, 40, device=DEV)
    out = torch.full((10, spp.fp8_row_bytes(40)), 0xAB, dtype=torch.uint8, device=DEV)
    spp.fp8_quantize(ctx, x, out=out, n_device=torch.tensor([count], dtype=torch.int64, device=DEV))
    n = min(max(count, 0), 10)
    assert (out[:n].cpu().numpy() == R.quantize(x[:n].double().cpu().numpy())).all() and (out[n:] == 0xAB).all()


def test_empty(ctx):
    rows = spp.fp8_quantize(ctx, torch.zeros(0, 40, device=DEV))
    assert rows.shape == (0, 64) and spp.fp8_dequantize(ctx, rows, 40).shape == (0, 40)


def test_rows_behind_32_bits_of_bytes(ctx):
    """x of 5.2 GB, rows of 2.7 GB: the last rows are where they belong."""
    n, D = 10_200_000, 256
    x = torch.zeros(n, D, dtype=torch.bfloat16, device=DEV)
    pick = torch.tensor([0, 4_194_303, 4_194_304, 8_388_608, n - 9, n - 1], device=DEV)
    few = torch.from_numpy(np.random.default_rng(6).standard_normal((len(pick), D))).to(torch.bfloat16)
    x[pick] = few.to(DEV)
    rows = spp.fp8_quantize(ctx, x)
    want = R.quantize(few.double().numpy())
    assert (rows[pick].cpu().numpy() == want).all()
    x.fill_(3.0)
    spp.fp8_dequantize(ctx, rows, D, out=x)
    assert torch.equal(x[pick].cpu(), torch.from_numpy(R.values(want, D)).to(torch.bfloat16))
    assert int(x.count_nonzero()) == int(x[pick].count_nonzero())

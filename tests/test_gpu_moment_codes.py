"""The 8-bit moments at the edges of their codes: where a value becomes the next code, what becomes zero, what never does.

The run's largest value is the largest code's, so that the scale is 1 and every value here is exact."""
import numpy as np
import pytest
import torch

import paper_2305_03152_amd as spp

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def ctx():
    c = spp.Context(0)
    yield c
    c.close()


def _held(ctx, m, v):
    opt = spp.AdamW(ctx, [torch.zeros(len(m), device=DEV)], state_bits=8)
    opt.load([torch.from_numpy(m).to(DEV)], [torch.from_numpy(v).to(DEV)], 1)
    a, b = opt.state()
    return a[0].cpu().numpy(), b[0].cpu().numpy()


def _codes(steps):
    c = np.arange(16 * steps)
    return (2.0 ** (c // steps - 15.0) * (1 + c % steps / steps))


def _nearest(x, codes):
    """The nearest code, of two the even one; as the first code what 0 is taken as."""
    j = np.searchsorted(codes, x).clip(1, len(codes) - 1)
    down, up = x - codes[j - 1], codes[j] - x
    return np.where((up < down) | ((up == down) & (j % 2 == 0)), j, j - 1)


def test_every_boundary_between_two_codes_of_m(ctx):
    """Half way between two codes and the neighbours in fp32 of that, with both signs; the first boundary is 1.0625 * 2^-15."""
    codes = _codes(8)
    half = ((codes[:-1] + codes[1:]) / 2).astype(np.float32)
    assert half[0] == np.float32(1.0625 * 2.0 ** -15)
    x = np.concatenate([half, np.nextafter(half, np.float32(0)), np.nextafter(half, np.float32(9)), codes.astype(np.float32),
                        np.array([0.5, 0.5625, 0.75, 0.99], np.float32) * np.float32(2.0 ** -15)])
    x = np.concatenate([x, -x])
    x = np.concatenate([x, np.zeros(-len(x) % 255, np.float32)]).reshape(-1, 255)
    m = np.concatenate([np.full((len(x), 1), 1.875, np.float32), x], 1).ravel()
    got, _ = _held(ctx, m, np.zeros_like(m))
    code = np.where(np.abs(m) < 2.0 ** -15, 0, _nearest(np.abs(m).astype(np.float64), codes))
    want = np.where(code == 0, 0.0, np.copysign(codes[code], m))
    assert np.array_equal(got.astype(np.float64), want)
    assert (got[np.abs(m) == np.float32(1.0625 * 2.0 ** -15)] == 0).all()
    assert (np.abs(got[np.abs(m) == np.nextafter(np.float32(1.0625 * 2.0 ** -15), np.float32(1))]) == 1.125 * 2.0 ** -15).all()


def test_a_second_moment_above_zero_is_never_zero(ctx):
    """Squares of codes come back as they are; what lies below code 1, down to the smallest fp32, is code 1; zero is zero."""
    codes = _codes(16)
    codes[0] = 0
    small = np.array([2.0 ** -149, 1e-40, 1e-30, 1e-12, (2.0 ** -15) ** 2, (1.03 * 2.0 ** -15) ** 2, 0.0, 0.0], np.float32)
    v = np.concatenate([(codes * codes).astype(np.float32), [np.float32(1.9375 ** 2)], small, np.zeros(255 - len(small), np.float32)])
    v[255], v[256] = v[256], v[255]                                    # each run of 256 has the largest
    assert len(v) == 512 and v[255] == v[256] == np.float32(1.9375 ** 2)
    _, got = _held(ctx, np.zeros_like(v), v)
    assert np.array_equal(got[:256], v[:256])
    least = np.float32((1.0625 * 2.0 ** -15) ** 2)
    assert (got[257:263] == least).all() and (got[263:] == 0).all()


def test_runs_of_tiny_first_moments_hold_zeros(ctx):
    m = np.zeros(512, np.float32)
    m[:256], m[256:] = 2.0 ** -101, 2.0 ** -100
    got, _ = _held(ctx, m, np.ones_like(m))
    assert (got[:256] == 0).all() and np.abs(got[256:] / 2.0 ** -100 - 1).max() <= 2.0 ** -22

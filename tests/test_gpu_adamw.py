"""One AdamW step over many tensors against 64 bits, with the moments in 32 and in 8 bits.

Tolerances, u = 2^-24 a rounding to fp32.  m' has three roundings and two rounded coefficients: 4u(|b1 m| + |(1-b1) g|).  v' has four
and two, all of one sign: 5u v', to which 2^-149 is added where a square leaves the normal range.  The update
U = step m' / den: the error of m' and a relative 3u of den (half of v's, the root, the factor, the sum), the quotient, the step
and its product: 4u(|b1 m| + |(1-b1) g|) step/den + 8u|U|.  p' adds the decay, its rounding and that of the difference:
4u(|p| + |U|).  A parameter in bf16 (8 significant bits) is rounded to it: 2^-8.
"""
import numpy as np
import pytest
import torch

import mx4_reference as R
import paper_2305_03152_amd as spp

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
HYPER = dict(lr=1e-2, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)


@pytest.fixture(scope="module")
def ctx():
    c = spp.Context(0)
    yield c
    c.close()


def _check(p0, g, m0, v0, t, p1, m1=None, v1=None, lr=None, hyper=HYPER):
    """p1 (and m1, v1 where they are given in 32 bits) against the step in 64 bits from p0, m0, v0."""
    lr = hyper["lr"] if lr is None else lr
    (b1, b2), eps, wd = hyper["betas"], hyper["eps"], hyper["weight_decay"]
    f = [a.double().cpu().numpy().ravel() for a in (p0, g, m0, v0)]
    p, m, v = R.adamw(*f, t, lr, b1, b2, eps, wd)
    terms = b1 * np.abs(f[2]) + (1 - b1) * np.abs(f[1])
    if m1 is not None:
        assert (np.abs(m1.double().cpu().numpy().ravel() - m) <= 4 * U * terms + 2.0 ** -149).all()
        assert (np.abs(v1.double().cpu().numpy().ravel() - v) <= 5 * U * v + 3 * 2.0 ** -149).all()
    step, den = lr / (1 - b1 ** t), np.sqrt(v) / np.sqrt(1 - b2 ** t) + eps
    up = step * np.abs(m) / den
    bound = 4 * U * terms * step / den + 8 * U * up + 4 * U * (np.abs(f[0]) + up)
    if p0.dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * (np.abs(p) + bound)
    bad = ~(np.abs(p1.double().cpu().numpy().ravel() - p) <= bound)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3].tolist())
    return m, v, terms


def _tensors(sizes, ptype, gtype, seed, scale=0.01):
    gen = torch.Generator().manual_seed(seed)
    p = [(torch.randn(n, generator=gen) * 0.1).to(DEV, ptype) for n in sizes]
    g = [(torch.randn(n, generator=gen) * scale).to(DEV, gtype) for n in sizes]
    return p, g


SIZES = [[1], [3, 4, 5], [255, 256, 257, 0, 511], [2047, 2048, 2049, 1], [100_003, 64, 7], [17] * 64, list(range(1, 200)), [33_000] * 70 + [1]]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("ptype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("gtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("sizes", SIZES, ids=[str(len(s)) + "x" + str(max(s)) for s in SIZES])
def test_steps_against_64_bits(ctx, bits, ptype, gtype, sizes):
    p, _ = _tensors(sizes, ptype, gtype, 1)
    opt = spp.AdamW(ctx, p, state_bits=bits, **HYPER)
    for t in range(1, 4):
        _, g = _tensors(sizes, ptype, gtype, 10 * t)
        p0 = [a.clone() for a in p]
        m0, v0 = [[a.clone() for a in s] for s in opt.state()]
        opt.step(g)
        m1, v1 = opt.state()
        assert opt.t == t
        for j in range(len(sizes)):
            m, v, terms = _check(p0[j], g[j], m0[j], v0[j], t, p[j], *((m1[j], v1[j]) if bits == 32 else ()))
            if bits == 8 and sizes[j]:
                _check_small(m, v, 4 * U * terms, m1[j], v1[j])


def _check_small(m, v, off, m1, v1):
    """What 8 bits hold against the moments: half a code's step, 2^-4 of m and 2^-5 of sqrt(v), below the smallest code the
    codes themselves; 16u more for the roundings of scale, ratio and value, and `off`, what m' itself is off by in fp32 (its terms
    may cancel)."""
    n = len(m)
    pad = -n % 256
    def blocks(a):
        return np.pad(np.asarray(a, np.float64), (0, pad)).reshape(-1, 256)
    m, v, off, m1, v1 = blocks(m), blocks(v), blocks(off).max(1, keepdims=True), blocks(m1.double().cpu().numpy()), blocks(v1.double().cpu().numpy())
    top = np.abs(m).max(1, keepdims=True)
    least = top / 1.875 * 2.0 ** -15
    assert (np.abs(m1 - m) <= np.abs(m) * (2.0 ** -4 + 16 * U) + least * 1.25 + off).all()
    # a value well above the smallest code keeps its sign and half a step
    big = np.abs(m) > 4 * least
    assert (np.abs(m1 - m)[big] <= np.abs(m)[big] * (2.0 ** -4 + 16 * U) + (off + 0 * m)[big]).all()
    r, r1 = np.sqrt(v), np.sqrt(v1)
    least = r.max(1, keepdims=True) / 1.9375 * 2.0 ** -15
    assert (np.abs(r1 - r) <= r * (2.0 ** -5 + 16 * U) + least * 1.25).all()
    assert ((v1 > 0) == (v > 0)).all()
    assert (np.abs(np.abs(m1).max(1) - top[:, 0]) <= top[:, 0] * 16 * U + off[:, 0]).all()              # the largest is held as it is


def test_moments_in_8_bits_are_loaded_and_read_back(ctx):
    """Every code stands for itself: values that 8 bits can hold come back as they are, others as the nearest."""
    c = np.arange(256)
    m = (2.0 ** (np.maximum(c % 128, 1) // 8 - 15.0) * (1 + np.maximum(c % 128, 1) % 8 / 8)) * np.where(c >= 128, -1, 1) * (c % 128 > 0)
    r = 2.0 ** (np.maximum(c, 1) // 16 - 15.0) * (1 + np.maximum(c, 1) % 16 / 16) * (c > 0)
    m, v = torch.from_numpy(m).float().to(DEV), torch.from_numpy(r * r).float().to(DEV)
    opt = spp.AdamW(ctx, [torch.zeros(256, device=DEV)], state_bits=8)
    opt.load([m], [v], 5)
    m1, v1 = opt.state()
    # scale is the largest times a rounded 1/1.875 (1/1.9375): the ratio to a code is off by at most 3u, v by 6u and the root's u
    assert opt.t == 5 and ((m1[0] - m).abs() <= 4 * U * m.abs()).all() and ((v1[0] - v).abs() <= 8 * U * v).all()
    far = torch.tensor([0.0, float("nan"), float("inf"), -float("inf"), -1.0, 1.0] + [0.5] * 250, device=DEV)
    opt.load([far], [far], 0)
    m1, v1 = opt.state()
    assert (m1[0][1:4] == 0).all() and (v1[0][:5] == 0).all() and abs(float(m1[0][5]) - 1) < 4 * U and abs(float(v1[0][5]) - 1) < 8 * U


@pytest.mark.parametrize("bits", [32, 8])
def test_elements_without_a_finite_gradient_stay(ctx, bits):
    n = 1000
    p, g = _tensors([n], torch.float32, torch.float32, 2)
    opt = spp.AdamW(ctx, p, state_bits=bits, **HYPER)
    opt.step([g[0].clone()])
    ctx.totals(reset=True)
    p0, (m0, v0) = p[0].clone(), [a[0].clone() for a in opt.state()]
    bad = torch.tensor([0, 255, 256, 700, 999], device=DEV)
    g[0][bad] = torch.tensor([float("nan"), float("inf"), -float("inf"), 1e30, float("nan")], device=DEV)
    opt.step(g)
    m1, v1 = opt.state()
    assert opt.skipped() == 5 and torch.isfinite(p[0]).all() and torch.isfinite(m1[0]).all() and torch.isfinite(v1[0]).all()
    assert torch.equal(p[0][bad], p0[bad])
    rest = torch.ones(n, dtype=torch.bool, device=DEV)
    rest[bad] = False
    _check(p0[rest], g[0][rest], m0[rest], v0[rest], 2, p[0][rest])
    if bits == 32:
        assert torch.equal(m1[0][bad], m0[bad]) and torch.equal(v1[0][bad], v0[bad])
    else:                                                            # held again under the block's new scale
        assert ((m1[0][bad] - m0[bad]).abs() <= m0[bad].abs() * 2.0 ** -3.9).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_zero_tiny_and_large_gradients(ctx, bits):
    g = torch.tensor([0.0, 1e-45, 1e-30, 1e-20, 1e-10, 1.0, 1e10, 1e18, -1e18, -0.0] * 60, device=DEV)
    p = torch.ones_like(g)
    opt = spp.AdamW(ctx, [p], state_bits=bits, **HYPER)
    p0 = p.clone()
    opt.step([g])
    _check(p0, g, torch.zeros_like(g), torch.zeros_like(g), 1, p)
    opt2 = spp.AdamW(ctx, [torch.zeros(300, device=DEV)], state_bits=bits, **HYPER)
    for _ in range(3):
        opt2.step([torch.zeros(300, device=DEV)])
    m, v = opt2.state()
    assert int(opt2.params[0].count_nonzero()) == 0 and int(m[0].count_nonzero()) == 0 and int(v[0].count_nonzero()) == 0


@pytest.mark.parametrize("bits", [32, 8])
def test_views_at_odd_addresses_and_shapes(ctx, bits):
    buf = torch.randn(10_007, device=DEV)
    gbuf = torch.randn(10_009, device=DEV).bfloat16()
    p, g = buf[3:3 + 7 * 1001].view(7, 1001), gbuf[1:1 + 7 * 1001].view(7, 1001)
    keep, p0 = buf.clone(), p.clone()
    opt = spp.AdamW(ctx, [p], state_bits=bits, **HYPER)
    opt.step([g])
    _check(p0, g, torch.zeros_like(p0), torch.zeros_like(p0), 1, p)
    assert torch.equal(buf[:3], keep[:3]) and torch.equal(buf[3 + 7007:], keep[3 + 7007:])
    assert opt.state()[0][0].shape == (7, 1001)


@pytest.mark.parametrize("bits", [32, 8])
def test_a_tensor_beyond_32_bits_of_bytes(ctx, bits):
    n = 1_200_000_003                                                # 4.8 GB of parameters
    p = torch.zeros(n, device=DEV)
    g = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    pick = torch.tensor([0, 536_870_912, 1_073_741_824, n - 2, n - 1], device=DEV)
    g[pick] = 0.5
    opt = spp.AdamW(ctx, [p], state_bits=bits, **HYPER)
    opt.step([g])
    z = torch.zeros(len(pick))
    _check(z, g[pick], z, z, 1, p[pick])
    assert int(p.count_nonzero()) == len(pick)


def test_many_steps_in_8_bits_go_where_32_bits_go(ctx):
    """A quadratic with widely differing curvatures: both forms reach its minimum."""
    n = 4096
    curve = torch.exp2(torch.linspace(-6, 6, n, device=DEV))
    goal = torch.randn(n, generator=torch.Generator().manual_seed(3)).to(DEV)
    for bits in (32, 8):
        p = torch.zeros(n, device=DEV)
        opt = spp.AdamW(ctx, [p], state_bits=bits, lr=0.02, betas=(0.9, 0.99), weight_decay=0.0)
        for _ in range(600):
            opt.step([curve * (p - goal)], sync=False)
        ctx.sync()
        # steps of lr do not fall: what is left is a few of them
        assert float((p - goal).abs().max()) < 0.2, bits

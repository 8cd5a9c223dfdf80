"""Which gradients of a gated layer are refused for lying over the outputs' gradients that they are made from, without a GPU.

The check comes before that of the activation: a call with an activation that there is not says which of the two it ran into, and never launches."""
import ctypes as C
import os
import random

import pytest

import paper_2305_03152_amd as spp
from paper_2305_03152_amd import api


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(spp.LIB_PATH):
        from paper_2305_03152_amd import build
        build.build()
    return spp.load_library()


@pytest.fixture(scope="module")
def refused(lib):
    """Whether dP [n, 2H] at `p` with a row every `pld` elements is refused for dY [n, H] at `y` with one every `yld`; fp32."""
    buf = (C.c_char * 65536)()
    ctx = C.cast(buf, C.c_void_p)
    def call(y, yld, p, pld, n=10, H=16):
        a, g = api._RowList(), api._RowList()
        for r, at, ld in ((a, y, yld), (g, p, pld)):
            for k, v in dict(d_rows=0x1000, n=n, d_n=None, d_y=0x100000 + 4 * at, ld=ld, group=0).items():
                setattr(r, k, v)
        assert lib.spp_fp8_gated_grad(ctx, (api._RowList * 1)(a), (api._RowList * 1)(g), 1, 0x8000, 1, 128, H, 0, 99, 0) == -1
        text = lib.spp_last_error().decode()
        assert ("overlaps" in text) != ("activation" in text), text
        return "overlaps" in text
    return call


def test_the_same_matrix_and_a_shifted_one(refused):
    assert refused(0, 32, 0, 32)                               # the very pointer
    assert refused(0, 16, 0, 32) and refused(100, 16, 0, 32) and refused(0, 16, 159, 32) and refused(319, 16, 0, 32)
    assert not refused(0, 16, 160, 32) and not refused(320, 16, 0, 32)
    assert refused(0, 16, 15, 32, n=1) and not refused(0, 16, 16, 32, n=1) and refused(31, 16, 0, 32, n=1) and not refused(32, 1000, 0, 1000, n=1)
    assert not refused(0, 16, 0, 32, n=0)


def test_columns_side_by_side_in_one_buffer(refused):
    assert not refused(0, 48, 16, 48) and not refused(32, 48, 0, 48) and not refused(0, 50, 17, 50)
    assert refused(0, 47, 16, 47) and refused(0, 48, 15, 48) and refused(31, 48, 0, 48) and refused(0, 48, 17, 48)
    assert not refused(0, 48, 17, 48, n=1)                     # whose last columns would reach into the next row's


def test_several_lists(lib, refused):
    def lists(*rows):
        arr = (api._RowList * len(rows))()
        for r, (at, ld) in zip(arr, rows):
            for k, v in dict(d_rows=0x1000, n=10, d_n=None, d_y=0x100000 + 4 * at, ld=ld, group=0).items():
                setattr(r, k, v)
        return arr
    buf = (C.c_char * 65536)()
    def call(dy, dp):
        assert lib.spp_fp8_gated_grad(C.cast(buf, C.c_void_p), lists(*dy), lists(*dp), 2, 0x8000, 1, 128, 16, 0, 99, 0) == -1
        return lib.spp_last_error().decode()
    assert "activation" in call([(0, 16), (160, 16)], [(320, 32), (640, 32)])
    assert "activation" in call([(0, 16), (0, 16)], [(320, 32), (640, 32)])             # one dY for two lists
    assert "gradient of list 0 overlaps the dY of list 1" in call([(0, 16), (400, 16)], [(320, 32), (640, 32)])


def test_against_every_byte(refused):
    rng = random.Random(1)
    said = [0, 0]
    for _ in range(4000):
        H, n = rng.randint(1, 6), rng.randint(0, 9)
        yld, pld = H + rng.choice([0, 0, 1, 2 * H, rng.randint(0, 40)]), 2 * H + rng.choice([0, 0, 1, H, rng.randint(0, 40)])
        if rng.random() < 0.4:
            yld = pld = max(yld, pld)
        y, p = rng.randint(0, 300), rng.randint(0, 300)
        a = {y + i * yld + k for i in range(n) for k in range(H)}
        b = {p + i * pld + k for i in range(n) for k in range(2 * H)}
        assert refused(y, yld, p, pld, n, H) == bool(a & b), (H, n, y, yld, p, pld)
        said[bool(a & b)] += 1
    assert min(said) > 500, said

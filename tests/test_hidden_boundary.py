"""What the operators on hidden rows refuse, without a GPU: codes and texts from the C interface, exceptions from the binding."""
import ctypes as C
import os
import re

import numpy as np
import pytest
import torch

import fp8_reference as R
import paper_2305_03152_amd as spp
from paper_2305_03152_amd import api
from test_operator_binding import Says, Stub, _refused

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(spp.LIB_PATH):
        from paper_2305_03152_amd import build
        build.build()
    return spp.load_library()


@pytest.fixture()
def fake_ctx():
    """Zeroed memory in the place of a context: every refusal below comes before the library looks into it."""
    buf = (C.c_char * 65536)()
    return C.cast(buf, C.c_void_p), buf


def _text(lib):
    return lib.spp_last_error().decode()


def test_row_bytes(lib):
    widths = (1, 16, 17, 47, 100, 128, 129, 172, 256, 1024, 2048, 2049, 4096)
    assert [spp.fp8_row_bytes(D) for D in widths] == [32, 32, 48, 64, 128, 144, 160, 192, 272, 1040, 2064, 2096, 4128]
    assert all(spp.fp8_row_bytes(D) == R.row_bytes(D) for D in range(1, 4097))
    for D in (0, -1, 4097):
        assert lib.spp_fp8_row_bytes(D) == -1
        with pytest.raises(spp.SppError):
            spp.fp8_row_bytes(D)


def test_quantize_refusals(lib, fake_ctx):
    ctx, _ = fake_ctx
    ok = (0x1000, 0, 10, None, 64, 64, 0x2000)
    def call(c=ctx, **kw):
        names = ("x", "type", "n", "d_n", "D", "ld", "rows")
        a = dict(zip(names, ok)) | kw
        assert lib.spp_fp8_dequantize(c, a["rows"], a["n"], a["d_n"], a["D"], a["x"], a["type"], a["ld"], 0) == -1
        assert "spp_fp8_dequantize" in _text(lib)
        assert lib.spp_fp8_quantize(c, a["x"], a["type"], a["n"], a["d_n"], a["D"], a["ld"], a["rows"], 0) == -1
        assert "spp_fp8_quantize" in _text(lib)
        return _text(lib)
    assert "null" in call(c=None)
    assert "type" in call(type=3) and "type" in call(type=-1)
    assert "D =" in call(D=0) and "D =" in call(D=5000)
    assert "n =" in call(n=-1) and "n =" in call(n=1 << 31)
    assert "ld" in call(ld=63)
    assert "null" in call(x=None) and "null" in call(rows=None)
    assert "aligned" in call(rows=0x2008) and "aligned" in call(x=0x1002)


def _list(**kw):
    a = api._RowList()
    for k, v in (dict(d_rows=0x1000, n=10, d_n=None, d_y=0x4000, ld=64, group=0) | kw).items():
        setattr(a, k, v)
    return a


def test_layer_refusals(lib, fake_ctx):
    ctx, _ = fake_ctx
    wide = (api._RowList * 65)(*[_list(ld=128, d_y=0x9000)] * 65)
    def call(item=None, n_lists=1, c=ctx, w=0x8000, groups=1, D=128, H=64, type=2, null=False):
        arr = (api._RowList * 65)(*[item or _list()] * 65)
        p = None if null else arr
        assert lib.spp_fp8_weight_grad(c, p, n_lists, groups, D, H, type, w, 0) == -1 and "spp_fp8_weight_grad" in _text(lib)
        assert lib.spp_fp8_gated(c, p, n_lists, w, groups, D, H, type, 0, 0) == -1 and "spp_fp8_gated:" in _text(lib)
        assert lib.spp_fp8_gated_grad(c, p, wide, n_lists, w, groups, D, H, type, 0, 0) == -1 and "spp_fp8_gated_grad" in _text(lib)
        assert lib.spp_fp8_product(c, p, n_lists, w, groups, D, H, type, 0) == -1 and "spp_fp8_product" in _text(lib)
        return _text(lib)
    assert "null" in call(c=None) and "null" in call(w=None)
    assert "lists" in call(n_lists=65) and "lists" in call(n_lists=-1) and "lists" in call(null=True)
    assert "groups" in call(groups=0) and "groups" in call(groups=65)
    assert "D =" in call(D=0) and "D =" in call(D=4097) and "H =" in call(H=0) and "H =" in call(H=65537)
    assert "type" in call(type=7)
    assert "list 0" in call(_list(n=-1)) and "list 0" in call(_list(n=1 << 31)) and "ld" in call(_list(ld=63))
    assert "group" in call(_list(group=1)) and "group" in call(_list(group=-1))
    assert "null" in call(_list(d_rows=None)) and "null" in call(_list(d_y=None))
    assert "aligned" in call(_list(d_rows=0x1008)) and "aligned" in call(_list(d_y=0x4001)) and "aligned" in call(_list(d_n=0x3004))
    assert "aligned" in call(w=0x8002)


def test_gated_refusals(lib, fake_ctx):
    ctx, _ = fake_ctx
    def call(grad=None, null=False, H=64, act=0, lists=None, n=1):
        a = lists or (api._RowList * 1)(_list(ld=max(H, 64)))
        g = None if null else (api._RowList * n)(*[grad or _list(ld=2 * H, d_y=0x9000)] * n)
        assert lib.spp_fp8_gated_grad(ctx, a, g, n, 0x8000, 2, 128, H, 2, act, 0) == -1
        return _text(lib)
    assert "null" in call(null=True)
    assert "H =" in call(H=32769)
    assert "activation" in call(act=3) and "activation" in call(act=-1)
    assert "ld" in call(_list(ld=127, d_y=0x9000)) and "null" in call(_list(ld=128, d_y=None))
    assert "aligned" in call(_list(ld=128, d_y=0x9001))
    for other in (dict(d_rows=0x1010), dict(n=9), dict(d_n=0x3000), dict(group=1)):
        assert "not the list's" in call(_list(ld=128, d_y=0x9000, **other))
    assert lib.spp_fp8_gated(ctx, (api._RowList * 1)(_list()), 1, 0x8000, 1, 128, 64, 2, 5, 0) == -1 and "activation" in _text(lib)


@pytest.fixture()
def no_library(monkeypatch):
    real = api.fp8_row_bytes
    for D in (32, 64, 128, 200):
        real(D)                                                      # kept by its cache
    def called():
        raise AssertionError("the library was called")
    monkeypatch.setattr(api, "load_library", called)


def _rows(n, D=64, **kw):
    return Says((n, api.fp8_row_bytes(D)), dtype=torch.uint8, **kw)


def test_tensors_that_are_not_on_the_gpu_are_refused(no_library):
    c, cpu, cpu_rows = Stub(), torch.zeros(4, 64), torch.zeros(4, 80, dtype=torch.uint8)
    gpu, rows, w = Says((4, 64)), _rows(4), _rows(64)
    _refused("x must be", lambda: api.fp8_quantize(c, cpu, out=rows))
    _refused("out must be", lambda: api.fp8_quantize(c, gpu, out=cpu_rows))
    _refused("rows must be", lambda: api.fp8_dequantize(c, cpu_rows, 64, out=gpu))
    _refused("out must be", lambda: api.fp8_dequantize(c, rows, 64, out=cpu))
    _refused("rows of list 0", lambda: api.fp8_product(c, cpu_rows, w, 64, out=gpu))
    _refused("y of list 0", lambda: api.fp8_product(c, rows, w, 64, out=cpu))
    _refused("weights must be", lambda: api.fp8_gated(c, rows, torch.zeros(128, 80, dtype=torch.uint8), 64, out=gpu))
    _refused("weights must be", lambda: api.fp8_gated_grad(c, [(rows, 4, None, gpu)], [(rows, 4, None, Says((4, 128)))], torch.zeros(128, 80, dtype=torch.uint8), 64))
    _refused("out must be", lambda: api.fp8_weight_grad(c, [(rows, 4, None, gpu)], 64, 64, out=torch.zeros(1, 64, 64)))


def test_shapes_types_and_sizes_that_do_not_fit_are_refused(no_library):
    c, rows, y, p = Stub(), _rows(9), Says((9, 32)), Says((9, 64))
    w = Says((2, 64, 80), dtype=torch.uint8)
    lists, grads = api.RowLists([(rows, 9, None, y, 1)]), api.RowLists([(rows, 9, None, p, 1)])
    _refused("float32, float16 or bfloat16", lambda: api.fp8_quantize(c, Says((4, 64), dtype=torch.float64), out=_rows(4)))
    _refused("2-D", lambda: api.fp8_quantize(c, Says((64,)), out=_rows(4)))
    _refused("too small", lambda: api.fp8_quantize(c, Says((10, 64)), out=rows))
    _refused("rows of 80 bytes", lambda: api.fp8_quantize(c, Says((4, 64)), out=_rows(4, 128)))
    _refused("too small", lambda: api.fp8_dequantize(c, rows, 64, out=Says((8, 64))))
    _refused("64 columns", lambda: api.fp8_dequantize(c, rows, 64, out=Says((9, 32))))
    _refused("rows of 144 bytes", lambda: api.fp8_dequantize(c, rows, 128, out=Says((9, 128))))
    _refused("not of 128 columns", lambda: api.fp8_product_multi(c, lists, Says((2, 32, 144), dtype=torch.uint8), 128))
    _refused("31 outputs", lambda: api.fp8_product_multi(c, lists, Says((2, 31, 80), dtype=torch.uint8), 64))
    _refused("group 1 of 1", lambda: api.fp8_product_multi(c, lists, Says((32, 80), dtype=torch.uint8), 64))
    _refused("groups, rows, row bytes", lambda: api.fp8_product_multi(c, lists, Says((1, 2, 32, 80), dtype=torch.uint8), 64))
    _refused("weight must be", lambda: api.fp8_product(c, rows, w, 64, out=y))
    _refused("weight must be", lambda: api.fp8_gated(c, rows, w, 64, out=y))
    _refused("both factors", lambda: api.fp8_gated_multi(c, lists, Says((2, 63, 80), dtype=torch.uint8), 64))
    _refused("33 outputs", lambda: api.fp8_gated_multi(c, lists, Says((2, 66, 80), dtype=torch.uint8), 64))
    _refused("group 1 of 1", lambda: api.fp8_gated_multi(c, lists, Says((64, 80), dtype=torch.uint8), 64))
    for f in (lambda a: api.fp8_gated_multi(c, lists, w, 64, activation=a), lambda a: api.fp8_gated_grad(c, lists, grads, w, 64, activation=a)):
        _refused("activation", lambda: f("relu"))
        _refused("activation", lambda: f(None))
    _refused("a list for each", lambda: api.fp8_gated_grad(c, lists, [], w, 64))
    _refused("64 outputs", lambda: api.fp8_gated_grad(c, lists, lists, w, 64))
    _refused("type of lists", lambda: api.fp8_gated_grad(c, lists, [(rows, 9, None, Says((9, 64), dtype=torch.float16), 1)], w, 64))
    _refused("33 outputs", lambda: api.fp8_weight_grad(c, lists, 33, 64, groups=2, out=Says((2, 33, 64))))
    _refused("group 1 of 1", lambda: api.fp8_weight_grad(c, lists, 32, 64, out=Says((1, 32, 64))))
    _refused("groups \\* H \\* D", lambda: api.fp8_weight_grad(c, lists, 32, 64, groups=2, out=Says((1, 32, 64))))
    # rows in 4 bits are not rows in 8
    four = api.RowLists([(Says((9, 48), dtype=torch.uint8), 9, None, y)])
    _refused("not of 64 columns", lambda: api.fp8_product_multi(c, four, Says((32, 80), dtype=torch.uint8), 64))


def test_constants_match_the_header():
    text = open(os.path.join(ROOT, "include", "spp.h")).read()
    enums = {k: int(v) for k, v in re.findall(r"\b(SPP_(?:T_)?[A-Z0-9_]+)\s*=\s*(\d+)", text)}
    for name in ("SPP_SILU", "SPP_GELU", "SPP_SIGMOID", "SPP_T_MX4", "SPP_T_LAYER"):
        assert enums[name] == getattr(api, name), name


def test_the_definition_of_a_row():
    """The tests' own definition at values worked out by hand: 448 = 1.75 * 2^8 fits scale 1, 449 takes scale 2, 304 is half way between
    288 and 320 under scale 1 and goes to the even code, under scale 2 too; 2^-9 is the smallest code."""
    x = np.zeros((3, 200))
    x[0, :4] = [448, 304, 2.0 ** -9, -2.0 ** -10]
    x[1, :3] = [449, 304, -1]
    x[2, 199] = np.inf
    rows = R.quantize(x)
    assert list(rows[0, :4]) == [0x7E, 0x7A, 0x01, 0x80] and rows[0, 208] == 127
    assert R.values(rows, 200)[0, 1] == 320 and R.values(rows, 200)[1, 0] == 448 and rows[1, 208] == 128
    assert rows[2, 199] == 0x7F and list(rows[2, 208:]) == [10, 10] + [0] * 14 and list(rows[0, 200:208]) == [0] * 8
    table = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert (table == R.MAGNITUDES).all()

"""What the operators on gathered rows refuse, without a GPU: codes and texts from the C interface, exceptions from the binding."""
import ctypes as C
import os
import re

import pytest
import torch

import paper_2305_03152_amd as spp
from paper_2305_03152_amd import api

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
    assert [spp.mx4_row_bytes(D) for D in (1, 32, 33, 100, 128, 256, 768, 4096)] == [32, 32, 48, 80, 80, 144, 416, 2176]
    for D in (0, -1, 4097):
        assert lib.spp_mx4_row_bytes(D) == -1
        with pytest.raises(spp.SppError):
            spp.mx4_row_bytes(D)


def test_quantize_refusals(lib, fake_ctx):
    ctx, _ = fake_ctx
    ok = (0x1000, 0, 10, None, 64, 64, 0x2000)
    def call(c=ctx, **kw):
        names = ("x", "type", "n", "d_n", "D", "ld", "rows")
        a = dict(zip(names, ok)) | kw
        assert lib.spp_mx4_dequantize(c, a["rows"], a["n"], a["d_n"], a["D"], a["x"], a["type"], a["ld"], 0) == -1
        rc = lib.spp_mx4_quantize(c, a["x"], a["type"], a["n"], a["d_n"], a["D"], a["ld"], a["rows"], 0)
        assert rc == -1
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


def test_product_and_gradient_refusals(lib, fake_ctx):
    ctx, _ = fake_ctx
    def call(item=None, n_lists=1, c=ctx, w=0x8000, groups=1, D=128, H=64, type=2, null=False):
        arr = (api._RowList * 65)(*[item or _list()] * 65)
        p = None if null else arr
        assert lib.spp_mx4_weight_grad(c, p, n_lists, groups, D, H, type, w, 0) == -1
        assert lib.spp_mx4_product(c, p, n_lists, w, groups, D, H, type, 0) == -1
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


def test_adamw_refusals(lib, fake_ctx):
    ctx, _ = fake_ctx
    def call(c=ctx, n_tensors=1, bits=8, t=1, hyper=(1e-3, 0.9, 0.999, 1e-8, 0.0), null=False, none=False, **kw):
        a = api._AdamwTensor()
        for k, v in (dict(d_p=0x1000, d_g=0x2000, d_m=0x3000, d_v=0x4000, d_scale=0x5000, n=8, p_type=0, g_type=2) | kw).items():
            setattr(a, k, v)
        h = api._AdamwHyper(*hyper)
        assert lib.spp_adamw_step(c, None if null else C.byref(a), n_tensors, bits, None if none else C.byref(h), t, 0) == -1
        return _text(lib)
    assert "null" in call(c=None) and "null" in call(null=True) and "null" in call(none=True)
    assert "tensors" in call(n_tensors=-1) and "bits" in call(bits=16)
    assert "n =" in call(n=-1) and "n =" in call(n=(1 << 34) + 1)
    assert "types" in call(p_type=1) and "types" in call(g_type=3)
    for name in ("d_p", "d_g", "d_m", "d_v", "d_scale"):
        assert "null" in call(**{name: None})
    assert "aligned" in call(d_p=0x1002) and "aligned" in call(d_g=0x2001) and "aligned" in call(bits=32, d_m=0x3002) and "aligned" in call(d_scale=0x5002)
    for bad in ((1e-3, 1.0, 0.9, 1e-8, 0), (1e-3, -0.1, 0.9, 1e-8, 0), (1e-3, 0.9, 1.0, 1e-8, 0), (1e-3, 0.9, 0.999999999, 1e-8, 0), (1e-3, 0.9, float("nan"), 1e-8, 0)):
        assert "betas" in call(hyper=bad)
    for bad in ((-1e-3, 0.9, 0.9, 1e-8, 0), (float("inf"), 0.9, 0.9, 1e-8, 0), (1e-3, 0.9, 0.9, 0.0, 0), (1e-3, 0.9, 0.9, float("nan"), 0),
                (1e-3, 0.9, 0.9, 1e-8, -1.0), (1e-3, 0.9, 0.9, 1e-60, 0)):
        assert "eps" in call(hyper=bad)
    assert "step" in call(t=0)
    for f in (lib.spp_adamw_load, lib.spp_adamw_values):
        a = api._AdamwTensor(d_m=0x3000, d_v=0x4000, d_scale=None, n=8)
        p = (C.c_void_p * 1)(0x1000)
        assert f(ctx, C.byref(a), 1, p, p, 0) == -1 and "null" in _text(lib)
        assert f(ctx, C.byref(a), 1, None, p, 0) == -1 and f(None, C.byref(a), 1, p, p, 0) == -1 and f(ctx, C.byref(a), -1, p, p, 0) == -1


def test_the_binding_refuses_what_is_not_on_the_gpu():
    x = torch.zeros(4, 64)
    rows = torch.zeros(4, 48, dtype=torch.uint8)
    for call in (lambda: spp.mx4_quantize(None, x), lambda: spp.mx4_dequantize(None, rows, 64), lambda: spp.RowLists([(rows, 4, None, x)]),
                 lambda: spp.mx4_product(None, rows, rows, 64)):
        with pytest.raises((spp.SppError, AttributeError)):
            call()


def test_constants_and_layouts_match_the_header(tmp_path):
    import subprocess
    text = open(os.path.join(ROOT, "include", "spp.h")).read()
    defines = {k: int(v) for k, v in re.findall(r"#define\s+(SPP_[A-Z0-9_]+)\s+(\d+)\b", text)}
    for name in ("SPP_MAX_ROW_LISTS", "SPP_MX4_MAX_COLS", "SPP_MAX_HIDDEN", "SPP_ADAMW_BLOCK"):
        assert defines[name] == getattr(api, name), name
    enums = {k: int(v) for k, v in re.findall(r"\b(SPP_(?:T_)?[A-Z0-9_]+)\s*=\s*(\d+)", text)}
    for name in ("SPP_T_MX4", "SPP_T_LAYER", "SPP_T_ADAMW", "SPP_F32", "SPP_F16", "SPP_BF16"):
        assert enums[name] == getattr(api, name), name
    c = tmp_path / "s.c"
    c.write_text('#include "spp.h"\n#include <stdio.h>\nint main(void){printf("%zu %zu %zu\\n", sizeof(spp_row_list), sizeof(spp_adamw_tensor), '
                 'sizeof(spp_adamw_hyper));return 0;}\n')
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(c), "-o", str(tmp_path / "s")], check=True)
    out = subprocess.run([str(tmp_path / "s")], check=True, capture_output=True, text=True).stdout.split()
    assert [int(v) for v in out] == [C.sizeof(api._RowList), C.sizeof(api._AdamwTensor), C.sizeof(api._AdamwHyper)]

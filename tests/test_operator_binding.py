"""What the binding of the operators on gathered rows takes and refuses, without a GPU: tensors that only say what they are."""
import pytest
import torch

from paper_2305_03152_amd import api


class Says:
    """What the binding asks of a tensor."""
    def __init__(self, shape, strides=None, dtype=torch.float32, is_cuda=True, ptr=0x1000):
        self.t = torch.empty(4096, dtype=dtype).as_strided(shape, strides) if strides else torch.empty(shape, dtype=dtype, device="meta")
        self.shape, self.dtype, self.is_cuda, self.ptr = self.t.shape, dtype, is_cuda, ptr
    def __getattr__(self, name):
        return getattr(self.t, name)
    def data_ptr(self):
        return self.ptr


@pytest.mark.parametrize("strides", [(200, 1), (0, 0), (1, 5), (1, 1)])
def test_a_list_without_rows_is_taken_however_it_is_laid_out(strides):
    y = Says((0, 200), strides)
    lists = api.RowLists([(Says((0, 32), dtype=torch.uint8), 0, None, y), (Says((9, 32), dtype=torch.uint8), 9, None, Says((9, 200)))])
    assert [(a.n, a.ld) for a in lists._arr] == [(0, 200), (9, 200)]


def test_rows_that_are_not_contiguous_are_refused():
    rows = Says((2, 32), dtype=torch.uint8)
    for y in (Says((5, 1), (1, 7)), Says((1, 8), (99, 1)), Says((0, 0), (1, 1))):
        api._matrix(y, None, "y")
    for shape, strides in (((2, 5), (5, 2)), ((2, 5), (4, 1)), ((1, 5), (5, 2))):
        with pytest.raises(api.SppError, match="rows are contiguous"):
            api.RowLists([(rows, 1, None, Says(shape, strides))])


class Stub:
    """In the place of a context; what a call is refused for comes before the library is called."""
    _h, device, stream = None, 0, None


@pytest.fixture()
def no_library(monkeypatch):
    real = api.mx4_row_bytes
    for D in (32, 64, 128, 200):
        real(D)                                                      # kept by its cache
    def called():
        raise AssertionError("the library was called")
    monkeypatch.setattr(api, "load_library", called)


def _rows(n, D=64, **kw):
    return Says((n, api.mx4_row_bytes(D)), dtype=torch.uint8, **kw)


def _refused(text, call):
    with pytest.raises(api.SppError, match=text):
        call()


def test_tensors_that_are_not_on_the_gpu_are_refused(no_library):
    c, cpu, cpu_rows = Stub(), torch.zeros(4, 64), torch.zeros(4, 48, dtype=torch.uint8)
    gpu, rows = Says((4, 64)), _rows(4)
    count = torch.zeros(1, dtype=torch.int64)
    _refused("x must be", lambda: api.mx4_quantize(c, cpu, out=rows))
    _refused("out must be", lambda: api.mx4_quantize(c, gpu, out=cpu_rows))
    _refused("n_device must be", lambda: _call_with(api.mx4_quantize, c, gpu, out=rows, n_device=count))
    _refused("rows must be", lambda: api.mx4_dequantize(c, cpu_rows, 64, out=gpu))
    _refused("out must be", lambda: api.mx4_dequantize(c, rows, 64, out=cpu))
    _refused("rows of list 0", lambda: api.RowLists([(cpu_rows, 4, None, gpu)]))
    _refused("y of list 0", lambda: api.RowLists([(rows, 4, None, cpu)]))
    _refused("n_device of list 0", lambda: api.RowLists([(rows, 4, count, gpu)]))
    _refused("rows of list 0", lambda: api.mx4_product(c, cpu_rows, _rows(64), 64, out=gpu))
    _refused("weights must be", lambda: api.mx4_product(c, rows, torch.zeros(64, 48, dtype=torch.uint8), 64, out=gpu))
    _refused("y of list 0", lambda: api.mx4_product(c, rows, _rows(64), 64, out=cpu))
    _refused("out must be", lambda: api.mx4_weight_grad(c, [(rows, 4, None, gpu)], 64, 64, out=torch.zeros(1, 64, 64)))
    _refused("parameter 0", lambda: api.AdamW(c, [cpu]))


def _call_with(f, *args, **kw):
    """The count is looked at while the library's arguments are put together: it has one here that does nothing."""
    class Lib:
        def __getattr__(self, name):
            return lambda *a: 0
    was, api.load_library = api.load_library, lambda: Lib()
    try:
        return f(*args, **kw)
    finally:
        api.load_library = was


def test_shapes_types_and_sizes_that_do_not_fit_are_refused(no_library):
    c, rows, y, w = Stub(), _rows(9), Says((9, 32)), Says((2, 32, 48), dtype=torch.uint8)
    lists = api.RowLists([(rows, 9, None, y, 1)])
    _refused("float32, float16 or bfloat16", lambda: api.mx4_quantize(c, Says((4, 64), dtype=torch.float64), out=_rows(4)))
    _refused("2-D", lambda: api.mx4_quantize(c, Says((64,)), out=_rows(4)))
    _refused("too small", lambda: api.mx4_quantize(c, Says((10, 64)), out=rows))
    _refused("rows of 48 bytes", lambda: api.mx4_quantize(c, Says((4, 64)), out=_rows(4, 128)))
    _refused("too small", lambda: api.mx4_dequantize(c, rows, 64, out=Says((8, 64))))
    _refused("64 columns", lambda: api.mx4_dequantize(c, rows, 64, out=Says((9, 32))))
    _refused("rows of 80 bytes", lambda: api.mx4_dequantize(c, rows, 128, out=Says((9, 128))))
    _refused("at most 64", lambda: api.RowLists([(rows, 9, None, y)] * 65))
    _refused("n exceeds", lambda: api.RowLists([(rows, 10, None, y)]))
    _refused("n exceeds", lambda: api.RowLists([(rows, 9, None, Says((8, 32)))]))
    _refused("n exceeds", lambda: api.RowLists([(rows, -1, None, y)]))
    _refused("group -1", lambda: api.RowLists([(rows, 9, None, y, -1)]))
    _refused("unlike list 0", lambda: api.RowLists([(rows, 9, None, y), (rows, 9, None, Says((9, 33)))]))
    _refused("unlike list 0", lambda: api.RowLists([(rows, 9, None, y), (rows, 9, None, Says((9, 32), dtype=torch.float16))]))
    _refused("unlike list 0", lambda: api.RowLists([(rows, 9, None, y), (_rows(9, 128), 9, None, y)]))
    _refused("n_device of list 0", lambda: api.RowLists([(rows, 9, Says((2,), dtype=torch.int64), y)]))
    _refused("n_device of list 0", lambda: api.RowLists([(rows, 9, Says((1,), dtype=torch.int32), y)]))
    _refused("not of 128 columns", lambda: api.mx4_product_multi(c, lists, Says((2, 32, 80), dtype=torch.uint8), 128))
    _refused("31 outputs", lambda: api.mx4_product_multi(c, lists, Says((2, 31, 48), dtype=torch.uint8), 64))
    _refused("group 1 of 1", lambda: api.mx4_product_multi(c, lists, Says((32, 48), dtype=torch.uint8), 64))
    _refused("groups, H, row bytes", lambda: api.mx4_product_multi(c, lists, Says((1, 2, 32, 48), dtype=torch.uint8), 64))
    _refused("weight must be", lambda: api.mx4_product(c, rows, w, 64, out=y))
    _refused("33 outputs", lambda: api.mx4_weight_grad(c, lists, 33, 64, groups=2, out=Says((2, 33, 64))))
    _refused("group 1 of 1", lambda: api.mx4_weight_grad(c, lists, 32, 64, out=Says((1, 32, 64))))
    _refused("groups \\* H \\* D", lambda: api.mx4_weight_grad(c, lists, 32, 64, groups=2, out=Says((1, 32, 64))))
    _refused("state_bits", lambda: api.AdamW(c, [], state_bits=16))
    for p in (Says((4,), dtype=torch.float16), Says((4, 4), (1, 4))):
        _refused("parameter 0", lambda: api.AdamW(c, [p]))


def test_a_step_s_gradients_are_looked_at(no_library):
    opt = api.AdamW(Stub(), [])
    opt.params = [Says((6,))]
    a = api._AdamwTensor()
    opt._items = [[a, opt.params[0], 6, torch.float32, 0x1000, None, lambda: 0x1000, lambda: 6, lambda: True]]
    for g in (torch.zeros(6), Says((5,)), Says((6,), dtype=torch.float64), Says((6,), (2,)), Says((6,), dtype=torch.int32)):
        _refused("a gradient must be", lambda: opt.step([g]))
    _refused("one gradient per parameter", lambda: opt.step([]))
    _refused("one m and one v", lambda: opt.load([], [], 0))
    _refused("one m and one v", lambda: opt.load([Says((6,))], [Says((6,))], -1))
    _refused("m 0 must be", lambda: opt.load([torch.zeros(6)], [Says((6,))], 0))
    _refused("moments 0", lambda: opt.load([Says((6,))], [Says((7,))], 0))
    assert opt.t == 0

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

"""AdamW over parameters that were given other memory after the optimiser was made: refused unless the state still fits.
Without a GPU: tensors that only say what they are, and a library that must not be called."""
import ctypes as C

import pytest
import torch

from paper_2305_03152_amd import api


class Says:
    """What the binding asks of a tensor."""
    def __init__(self, n, dtype=torch.float32, contiguous=True, is_cuda=True):
        self.n, self.dtype, self.contiguous, self.is_cuda, self.shape = n, dtype, contiguous, is_cuda, (n,)
    def numel(self):
        return self.n
    def is_contiguous(self):
        return self.contiguous
    def data_ptr(self):
        return 0x1000


class Called(Exception):
    pass


def _optimiser(monkeypatch, bits):
    def called():
        raise Called
    monkeypatch.setattr(api, "load_library", called)
    monkeypatch.setattr(api, "_new", lambda ctx, shape, dtype: Says(shape[0]))
    opt = api.AdamW.__new__(api.AdamW)
    ctx = C.c_void_p()
    opt.ctx = type("Ctx", (), {"_h": ctx})()
    opt.state_bits, opt.t, opt.lr, opt.betas, opt.eps, opt.weight_decay = bits, 0, 1e-3, (0.9, 0.999), 1e-8, 0.0
    opt.params = [Says(100), Says(64)]
    opt._arr = (api._AdamwTensor * 2)()
    opt._items = []
    for a, p in zip(opt._arr, opt.params):
        a.n, a.p_type = p.n, api.SPP_F32
        opt._items.append([a, p, p.n, p.dtype, p.data_ptr(), None, lambda p=p: p.data_ptr(), p.numel, p.is_contiguous])
    opt._hyper = api._AdamwHyper()
    opt._args = None, None
    opt._state, opt._views = [], ([], [])
    return opt


CHANGES = [dict(n=99), dict(n=101), dict(n=0), dict(dtype=torch.bfloat16), dict(dtype=torch.float64), dict(contiguous=False), dict(is_cuda=False)]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("change", CHANGES, ids=str)
def test_a_parameter_that_changed_is_refused(monkeypatch, bits, change):
    opt = _optimiser(monkeypatch, bits)
    grads = [Says(100), Says(64)]
    for _ in range(2):
        with pytest.raises(Called):                              # as it was: the library's business
            opt.step(grads)
    for k, v in change.items():
        setattr(opt.params[0], k, v)
    if opt.params[0].is_cuda:                                    # at the address that it had (host memory lies elsewhere)
        with pytest.raises(api.SppError, match="no longer"):
            opt.step(grads)
    if bits == 8:
        with pytest.raises(api.SppError, match="no longer"):
            opt.state()
    opt.params[0].data_ptr = lambda: 0x2000
    with pytest.raises(api.SppError, match="no longer"):
        opt.step(grads)
    n = opt.params[0].n
    with pytest.raises(api.SppError, match="no longer"):
        opt.load([Says(n), Says(64)], [Says(n), Says(64)], 3)
    assert opt.t == 0


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_a_parameter_in_other_memory_of_its_size_is_stepped_there(bits):
    import paper_2305_03152_amd as spp
    ctx = spp.Context(0)
    p, q, g = (torch.ones(1000, device="cuda") for _ in range(3))
    opt, ref = spp.AdamW(ctx, [p], state_bits=bits, lr=1e-2), spp.AdamW(ctx, [q], state_bits=bits, lr=1e-2)
    opt.step([g])
    ref.step([g])
    old = p.data
    p.data = p.data.clone()
    kept = old.clone()
    opt.step([g])
    ref.step([g])
    assert torch.equal(p, q) and torch.equal(old, kept)
    p.data = torch.ones(500, device="cuda")
    with pytest.raises(spp.SppError, match="no longer"):
        opt.step([g])
    ctx.close()

"""Calls of the row operators that are refused on the host, before a device is looked at."""
import ctypes

import pytest
import torch

import paper_2512_06547_b200 as a3po
from paper_2512_06547_b200 import build as a3po_build

INVAL, UNSUP, WSP = -1, -2, -3
ONE, ODD, ODD2 = ctypes.c_void_p(256), ctypes.c_void_p(257), ctypes.c_void_p(258)    # never dereferenced
F32, BF16, RMS, LAYER = 0, 1, 0, 1


@pytest.fixture(scope="module")
def lib():
    a3po_build.build()
    return a3po.load_library()


def test_norm_fwd_refusals(lib):
    def call(x=ONE, gamma=ONE, beta=None, n=4, h=8, dt=BF16, kind=LAYER, eps=1e-6, y=ONE, mean=ONE, rstd=ONE):
        return lib.a3po_norm_fwd(x, gamma, beta, None, n, h, dt, kind, eps, y, mean, rstd, None)
    assert call(x=None) == INVAL and call(gamma=None) == INVAL and call(y=None) == INVAL
    assert call(n=-1) == INVAL and call(h=0) == INVAL and call(eps=-1.0) == INVAL and call(eps=float("nan")) == INVAL
    assert call(kind=RMS) == INVAL                       # an RMS norm reports no mean
    assert call(kind=2) == UNSUP and call(dt=5) == UNSUP and call(n=1 << 31) == UNSUP
    assert call(x=ODD) == UNSUP and call(dt=F32, x=ODD2) == UNSUP and call(rstd=ODD2) == UNSUP


def test_norm_bwd_refusals(lib):
    size = a3po.a3po_norm_bwd_workspace_bytes(4, 8)
    def call(x=ONE, mean=ONE, rstd=ONE, gy=ONE, n=4, h=8, dt=BF16, kind=LAYER, gx=ONE, gg=ONE, gb=ONE, ws=ONE, nb=size):
        return lib.a3po_norm_bwd(x, ONE, mean, rstd, None, gy, n, h, dt, kind, gx, gg, gb, 0, ws, nb, None)
    assert call(x=None) == INVAL and call(rstd=None) == INVAL and call(gy=None) == INVAL and call(gx=None) == INVAL
    assert call(gg=None) == INVAL and call(mean=None) == INVAL and call(kind=RMS) == INVAL
    assert call(ws=None) == WSP and call(nb=size - 1) == WSP and call(ws=ctypes.c_void_p(264)) == WSP
    assert call(gx=ODD) == UNSUP and call(gb=ODD2) == UNSUP


def test_dropout_refusals(lib):
    def call(x=ONE, n=4, h=8, dt=BF16, p=0.5, rng=ONE, y=ONE):
        return lib.a3po_dropout_fwd(x, None, None, n, h, dt, p, rng, y, None)
    assert call(p=-0.1) == INVAL and call(p=1.5) == INVAL and call(p=float("nan")) == INVAL and call(rng=None) == INVAL
    assert call(x=None) == INVAL and call(y=None) == INVAL and call(h=-3) == INVAL
    assert call(rng=ctypes.c_void_p(260)) == UNSUP and call(x=ODD) == UNSUP and call(dt=9) == UNSUP
    assert lib.a3po_dropout_bwd(ONE, None, 4, 8, BF16, 2.0, ONE, ONE, None) == INVAL


def test_join_refusals(lib):
    def fwd(res=ONE, r=ONE, p=0.5, rng=ONE, n=4):
        return lib.a3po_dropout_norm_fwd(ONE, res, p, rng, ONE, None, None, n, 8, BF16, RMS, 1e-6, r, ONE, None, None, None)
    assert fwd(res=None) == INVAL and fwd(r=None) == INVAL and fwd(rng=None) == INVAL and fwd(p=7.0) == INVAL
    assert fwd(n=-2) == INVAL
    size = a3po.a3po_norm_bwd_workspace_bytes(4, 8)
    def bwd(gres=ONE, p=0.5, nb=size):
        return lib.a3po_dropout_norm_bwd(ONE, p, ONE, ONE, None, ONE, None, ONE, None, 4, 8, BF16, RMS, gres, ONE, ONE,
                                         None, 0, ONE, nb, None)
    assert bwd(gres=None) == INVAL and bwd(p=-1.0) == INVAL and bwd(nb=0) == WSP


def test_workspace_sizes():
    f = a3po.a3po_norm_bwd_workspace_bytes
    assert f(-1, 8) == 0 and f(4, 0) == 0
    assert 0 < f(0, 64) <= f(1, 64) <= f(1000, 64) <= f(1 << 20, 64)
    assert f(1 << 20, 4096) <= 32 << 20


def test_binding_checks_shapes_and_types():
    """The Python layer refuses before the library is called (CPU tensors are refused too)."""
    x = torch.zeros(2, 8)
    with pytest.raises(TypeError, match="CUDA device"):
        a3po.a3po_norm_fwd(x, torch.ones(8), torch.zeros(2, 8))
    with pytest.raises(TypeError):
        a3po.a3po_dropout_fwd(x.half(), 0.1, None, x)


def test_binding_refuses_tensors_of_another_device(monkeypatch):
    """The kernels run on the current device's stream; a tensor elsewhere is refused (stand-ins: no GPU is needed)."""
    from paper_2512_06547_b200 import binding

    class Stand:
        is_cuda = True
        device = "cuda:1"
        def __init__(self, index): self.index = index
        def get_device(self): return self.index
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    binding._here(Stand(0), None, Stand(0))
    with pytest.raises(ValueError, match="current device"):
        binding._here(Stand(0), Stand(1))

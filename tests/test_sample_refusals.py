"""Calls of the sampling operator that are refused on the host, before a device is looked at."""
import ctypes

import pytest
import torch

import paper_2512_06547_b200 as a3po
from paper_2512_06547_b200 import build as a3po_build

INVAL, UNSUP, WSP = -1, -2, -3
ONE, ODD = ctypes.c_void_p(256), ctypes.c_void_p(257)    # never dereferenced
F32, BF16 = 0, 1


@pytest.fixture(scope="module")
def lib():
    a3po_build.build()
    return a3po.load_library()


def test_refusals(lib):
    n, v = 8, 1000
    wb = a3po.a3po_sample_workspace_bytes(n, v)
    assert wb > 0 and a3po.a3po_sample_workspace_bytes(-1, v) == 0 and a3po.a3po_sample_workspace_bytes(n, 0) == 0
    assert a3po.a3po_sample_workspace_bytes(200 * n, v) > wb

    def call(logits=ONE, ld=v, n=n, v=v, dt=F32, t=None, k=None, p=None, mp=None, u=ONE, token=ONE, logp=None, klp=None,
             kept=None, ws=ONE, wbytes=1 << 40):
        return lib.a3po_sample(logits, ld, None, n, v, dt, t, k, p, mp, u, token, logp, klp, kept, ws, wbytes, None)

    assert call(logits=None) == INVAL and call(u=None) == INVAL and call(token=None) == INVAL
    assert call(n=-1) == INVAL and call(v=0) == INVAL and call(ld=v - 1) == INVAL
    assert call(dt=5) == UNSUP and call(logits=ODD) == UNSUP and call(n=1 << 31) == UNSUP
    for name in ("t", "k", "p", "mp", "u", "token", "logp", "klp", "kept"):
        assert call(**{name: ctypes.c_void_p(258)}) == UNSUP, name
    # rows with filters have to fit the shared memory of a cluster
    for dt, most in ((F32, 393216), (BF16, 786432)):
        assert call(dt=dt, v=most + 1, ld=most + 1, k=ONE) == UNSUP
        assert call(dt=dt, v=most + 1, ld=most + 1, k=ONE, ws=None) == UNSUP
        assert call(dt=dt, v=most, ld=most, k=ONE, ws=None) == WSP
        assert call(dt=dt, v=most + 1, ld=most + 1, ws=None) == WSP
    assert call(ws=None) == WSP and call(ws=ctypes.c_void_p(264)) == WSP and call(wbytes=wb - 1) == WSP


def test_python_side_refusals(lib):
    x = torch.zeros(4, 10)
    one = torch.zeros(4)
    with pytest.raises(TypeError):
        a3po.a3po_sample(x, one, one.int(), torch.zeros(4096, dtype=torch.uint8))     # not on a GPU
    with pytest.raises(ValueError):
        a3po.a3po_sample(x[0], one, one.int(), torch.zeros(4096, dtype=torch.uint8))
    with pytest.raises(TypeError):
        a3po.a3po_sample(x.half(), one, one.int(), torch.zeros(4096, dtype=torch.uint8))

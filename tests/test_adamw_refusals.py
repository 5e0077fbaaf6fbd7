"""Calls of the AdamW step that are refused on the host, before a device is looked at."""
import ctypes

import pytest
import torch

import paper_2512_06547_b200 as a3po
from paper_2512_06547_b200 import build as a3po_build
from paper_2512_06547_b200.optimizer import AdamW

INVAL, UNSUP, WSP = -1, -2, -3
ONE = 256    # an address that is never dereferenced
F32, BF16 = 0, 1


@pytest.fixture(scope="module")
def lib():
    a3po_build.build()
    return a3po.load_library()


def test_refusals(lib):
    wb = a3po.a3po_adamw_workspace_bytes(1)
    assert wb > 0 and a3po.a3po_adamw_workspace_bytes(-1) == 0 and a3po.a3po_adamw_workspace_bytes(5000) > wb

    def call(weight=ONE, master=ONE, grad=ONE, m=ONE, v=ONE, ms=ONE, vs=ONE, n=100, count=1, wdt=BF16, gdt=F32, bits=8, b1=0.9,
             b2=0.95, eps=1e-8, clip=1.0, lr=ONE, step=ONE, norm=ONE, ws=ONE, wbytes=wb, table=True):
        t = (a3po.A3poAdamWTensor * 1)(a3po.A3poAdamWTensor(weight, master, grad, m, v, ms, vs, n, 0.0))
        return lib.a3po_adamw_step(ctypes.addressof(t) if table else None, count, wdt, gdt, bits, b1, b2, eps, clip, lr, step,
                                   norm, ws, wbytes, None)

    assert call(count=-1) == INVAL and call(table=False) == INVAL and call(lr=None) == INVAL and call(step=None) == INVAL
    assert call(weight=None) == INVAL and call(grad=None) == INVAL and call(m=None) == INVAL and call(v=None) == INVAL
    assert call(ms=None) == INVAL and call(vs=None) == INVAL and call(n=-1) == INVAL
    for bad in (dict(b1=1.0), dict(b1=-0.1), dict(b2=1.0), dict(b2=float("nan")), dict(eps=0.0), dict(clip=-1.0),
                dict(clip=float("nan"))):
        assert call(**bad) == INVAL, bad
    assert call(wdt=F32) == INVAL                    # fp32 weights are their own masters
    assert call(wdt=4) == UNSUP and call(gdt=4) == UNSUP and call(bits=16) == UNSUP
    assert call(lr=258) == UNSUP and call(step=260) == UNSUP and call(norm=258) == UNSUP
    assert call(weight=257) == UNSUP and call(master=258) == UNSUP and call(grad=258) == UNSUP and call(ms=258) == UNSUP
    assert call(m=258, bits=32) == UNSUP and call(m=257, ws=None) == WSP       # bytes may start anywhere
    assert call(n=1 << 42) == UNSUP
    assert call(ws=None) == WSP and call(ws=264) == WSP and call(wbytes=wb - 1) == WSP
    one = ctypes.c_void_p(256)
    assert lib.a3po_adamw_state_values(None, one, 4, 1, one, None) == INVAL
    assert lib.a3po_adamw_state_values(one, one, -1, 1, one, None) == INVAL
    assert lib.a3po_adamw_state_values(one, ctypes.c_void_p(258), 4, 1, one, None) == UNSUP


def test_python_side_refusals(lib):
    with pytest.raises(TypeError):
        AdamW([torch.zeros(4)])                       # not on a GPU
    with pytest.raises(TypeError):
        AdamW([torch.zeros(4, dtype=torch.float16)])
    with pytest.raises(ValueError):
        AdamW([], state_bits=16)

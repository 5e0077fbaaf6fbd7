"""Calls of the gated feed-forward block that are refused on the host, before a device is looked at."""
import ctypes

import pytest
import torch

import paper_2512_06547_b200 as a3po
from paper_2512_06547_b200 import build as a3po_build

INVAL, UNSUP, WSP = -1, -2, -3
ONE, ODD = ctypes.c_void_p(256), ctypes.c_void_p(264)    # never dereferenced
F32, BF16 = 0, 1
N, H, F = 64, 64, 128


@pytest.fixture(scope="module")
def lib():
    a3po_build.build()
    return a3po.load_library()


def test_forward_refusals(lib):
    kb = a3po.a3po_gated_ffn_kept_bytes(N, F, BF16)
    wb = a3po.a3po_gated_ffn_workspace_bytes(N, H, F, BF16, False, False)
    def call(x=ONE, wgu=ONE, wd=ONE, n=N, h=H, f=F, dt=BF16, act=0, y=ONE, kept=ONE, kbytes=kb, ws=ONE, wbytes=wb, mask=None):
        return lib.a3po_gated_ffn_fwd(x, wgu, wd, mask, n, h, f, dt, act, y, kept, kbytes, ws, wbytes, None, None)
    assert call(x=None) == INVAL and call(wgu=None) == INVAL and call(wd=None) == INVAL and call(y=None) == INVAL
    assert call(n=-1) == INVAL and call(h=0) == INVAL and call(f=-8) == INVAL
    assert call(dt=3) == UNSUP and call(act=2) == UNSUP and call(x=ODD) == UNSUP and call(wd=ODD) == UNSUP
    assert call(y=ODD) == UNSUP and call(n=(1 << 31) - 1) == UNSUP
    assert call(kept=ODD) == WSP and call(kbytes=kb - 1) == WSP
    assert call(ws=None) == WSP and call(ws=ODD) == WSP and call(wbytes=wb - 1) == WSP
    assert call(mask=ONE) == WSP                           # with a row mask the call needs more


def test_backward_refusals(lib):
    kb = a3po.a3po_gated_ffn_kept_bytes(N, F, BF16)
    wb = a3po.a3po_gated_ffn_workspace_bytes(N, H, F, BF16, False, True)
    def call(x=ONE, kept=ONE, kbytes=kb, gy=ONE, gx=ONE, ggu=ONE, gd=ONE, gdt=BF16, acc=0, wbytes=wb, dt=BF16):
        return lib.a3po_gated_ffn_bwd(x, ONE, ONE, None, kept, kbytes, gy, N, H, F, dt, 0, gx, ggu, gd, gdt, acc, ONE,
                                      wbytes, None, None)
    assert call(x=None) == INVAL and call(kept=None) == INVAL and call(gy=None) == INVAL and call(gx=None) == INVAL
    assert call(ggu=None) == INVAL and call(gd=None) == INVAL
    assert call(acc=1) == UNSUP                            # adding to bf16 gradients would round every time
    assert call(gdt=7) == UNSUP and call(dt=F32) == UNSUP and call(gx=ODD) == UNSUP and call(ggu=ODD) == UNSUP
    assert call(kbytes=kb - 1) == WSP and call(wbytes=wb - 1) == WSP


def test_sizes():
    k, w = a3po.a3po_gated_ffn_kept_bytes, a3po.a3po_gated_ffn_workspace_bytes
    assert k(-1, 8, BF16) == 0 and k(4, 0, BF16) == 0 and w(-1, 8, 8, BF16, 0, 0) == 0 and w(1 << 40, 8, 8, BF16, 0, 0) == 0
    assert 6 * N * F <= k(N, F, BF16) <= k(N + 200, F, BF16) and k(N, F, F32) >= 8 * N * F
    assert w(N, H, F, BF16, 0, 0) >= 2 * N * F and w(N, H, F, BF16, 0, 1) >= 4 * N * F
    assert w(0, H, F, BF16, 0, 1) > 0 and w(0, H, F, BF16, 1, 0) > 0 and w(0, 3, 5, BF16, 1, 0) > 0
    assert w(N, H, F, BF16, 1, 1) >= w(N, H, F, BF16, 0, 1) and w(N, H, F, F32, 0, 1) >= 12 * N * F


def test_binding_checks_shapes_and_types():
    x, wgu, wd = torch.zeros(4, 8), torch.zeros(32, 8), torch.zeros(8, 16)
    with pytest.raises(TypeError, match="CUDA device"):
        a3po.a3po_gated_ffn_fwd(x, wgu, wd, x, torch.zeros(256, dtype=torch.uint8))

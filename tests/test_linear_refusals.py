"""Calls of the linear operator that are refused on the host, before a device is looked at."""
import ctypes

import pytest
import torch

import paper_2512_06547_b200 as a3po
from paper_2512_06547_b200 import build as a3po_build

INVAL, UNSUP, WSP = -1, -2, -3
ONE, ODD = ctypes.c_void_p(256), ctypes.c_void_p(264)    # never dereferenced
F32, BF16, NONE, SILU = 0, 1, 2, 0
N, K, M = 64, 64, 128


@pytest.fixture(scope="module")
def lib():
    a3po_build.build()
    return a3po.load_library()


def test_forward_refusals(lib):
    kb, wb = a3po.a3po_linear_kept_bytes(N, M, BF16, SILU), a3po.a3po_linear_workspace_bytes(N, K, M, BF16, SILU)
    assert kb >= 4 * N * M and wb > 0 and a3po.a3po_linear_kept_bytes(N, M, BF16, NONE) == 0
    assert a3po.a3po_linear_kept_bytes(-1, M, BF16, SILU) == 0 and a3po.a3po_linear_workspace_bytes(N, 0, M, BF16, SILU) == 0

    def call(x=ONE, w=ONE, bias=None, res=None, mask=None, n=N, k=K, m=M, dt=BF16, act=SILU, y=ONE, ydt=BF16, kept=ONE, kbytes=kb,
             ws=ONE, wbytes=wb):
        return lib.a3po_linear_fwd(x, w, bias, res, mask, n, k, m, dt, act, y, ydt, kept, kbytes, ws, wbytes, None, None)

    assert call(x=None) == INVAL and call(w=None) == INVAL and call(y=None) == INVAL
    assert call(n=-1) == INVAL and call(k=0) == INVAL and call(m=-8) == INVAL
    assert call(dt=3) == UNSUP and call(act=3) == UNSUP and call(ydt=3) == UNSUP and call(dt=F32, ydt=BF16) == UNSUP
    assert call(x=ODD) == UNSUP and call(w=ODD) == UNSUP and call(bias=ODD) == UNSUP and call(res=ODD) == UNSUP
    assert call(y=ODD) == UNSUP and call(n=(1 << 31) - 1) == UNSUP and call(m=65535 * 32 + 8) == UNSUP
    assert call(kept=ODD) == WSP and call(kbytes=kb - 1) == WSP
    assert call(act=NONE, kept=ODD, ws=None) == WSP          # without an activation `kept` is not looked at
    assert call(ws=None) == WSP and call(ws=ODD) == WSP and call(wbytes=wb - 1) == WSP
    assert call(mask=ONE) == WSP                             # with a row mask the call needs more
    assert call(k=63, x=ctypes.c_void_p(258), ws=None) == WSP and call(k=63, x=ctypes.c_void_p(257)) == UNSUP


def test_backward_refusals(lib):
    kb = a3po.a3po_linear_kept_bytes(N, M, BF16, SILU)
    wb = a3po.a3po_linear_workspace_bytes(N, K, M, BF16, SILU, False, True)

    def call(x=ONE, w=ONE, mask=None, kept=ONE, kbytes=kb, gy=ONE, n=N, act=SILU, gx=ONE, gw=ONE, gdt=BF16, gb=ONE, acc=0, dt=BF16,
             wbytes=wb):
        return lib.a3po_linear_bwd(x, w, mask, kept, kbytes, gy, n, K, M, dt, act, gx, gw, gdt, gb, acc, ONE, wbytes, None, None)

    assert call(gx=None, gw=None, gb=None) == INVAL and call(gy=None) == INVAL and call(kept=None) == INVAL
    assert call(x=None) == INVAL and call(w=None) == INVAL
    assert call(gdt=7) == UNSUP and call(dt=F32, gdt=BF16) == UNSUP and call(acc=1) == UNSUP
    assert call(gy=ODD) == UNSUP and call(gx=ODD) == UNSUP and call(gw=ODD) == UNSUP and call(gb=ctypes.c_void_p(258)) == UNSUP
    assert call(kept=ODD) == WSP and call(kbytes=kb - 1) == WSP and call(wbytes=wb - 1) == WSP and call(mask=ONE) == WSP


def test_python_side_refusals(lib):
    x, w, y = torch.zeros(4, 8), torch.zeros(6, 8), torch.zeros(4, 6)
    ws = torch.zeros(4096, dtype=torch.uint8)
    with pytest.raises(TypeError):
        a3po.a3po_linear_fwd(x, w, y, ws)                                  # not on a GPU
    with pytest.raises(ValueError):
        a3po.a3po_linear_fwd(x, torch.zeros(6, 9), y, ws)
    with pytest.raises(TypeError):
        a3po.a3po_linear_fwd(x.half(), w.half(), y, ws)
    with pytest.raises(ValueError):
        a3po.a3po_linear_bwd(x, w[0], y, x, w, ws)


def test_gated_block_refuses_no_activation(lib):
    wb = a3po.a3po_gated_ffn_workspace_bytes(N, K, M, BF16, False, False)
    assert lib.a3po_gated_ffn_fwd(ONE, ONE, ONE, None, N, K, M, BF16, NONE, ONE, None, 0, ONE, wb, None, None) == UNSUP

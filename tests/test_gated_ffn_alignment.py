"""Where the rows of the feed-forward block may start: at any element on the FP32 pipes (fp32, or H or F not a multiple of 8),
whose kernels move elements, and at 16-byte boundaries on the tensor cores."""
import ctypes

import pytest
import torch

import paper_2512_06547_b200 as a3po
from paper_2512_06547_b200 import build as a3po_build

UNSUP, WSP = -2, -3
F32, BF16 = 0, 1
ptr = ctypes.c_void_p     # never dereferenced: every call is refused, for its workspace if for nothing else
ONE = ptr(256)


@pytest.fixture(scope="module")
def lib():
    a3po_build.build()
    return a3po.load_library()


def calls(lib, h, f, dt, grad_dt):
    n = 5
    kb = a3po.a3po_gated_ffn_kept_bytes(n, f, dt)
    def fwd(x=ONE, wgu=ONE, wd=ONE, y=ONE):
        return lib.a3po_gated_ffn_fwd(x, wgu, wd, None, n, h, f, dt, 0, y, ONE, kb, ONE, 1, None, None)
    def bwd(x=ONE, wgu=ONE, wd=ONE, gy=ONE, gx=ONE, ggu=ONE, gd=ONE):
        return lib.a3po_gated_ffn_bwd(x, wgu, wd, None, ONE, kb, gy, n, h, f, dt, 0, gx, ggu, gd, grad_dt, 0, ONE, 1, None, None)
    return fwd, bwd


@pytest.mark.parametrize("h,f,dt,at,off", [(63, 64, BF16, 258, 257), (64, 63, BF16, 264, 259), (64, 64, F32, 260, 258),
                                           (3, 5, F32, 264, 257)])
def test_fp32_pipes_take_rows_at_any_element(lib, h, f, dt, at, off):
    fwd, bwd = calls(lib, h, f, dt, dt)
    for call, names in ((fwd, ("x", "wgu", "wd", "y")), (bwd, ("x", "wgu", "wd", "gy", "gx", "ggu", "gd"))):
        for name in names:
            assert call(**{name: ptr(at)}) == WSP, name          # got as far as the workspace
            assert call(**{name: ptr(off)}) == UNSUP, name       # not at an element
    fwd, bwd = calls(lib, 63, 64, BF16, F32)                     # fp32 weight gradients of bf16 weights
    assert bwd(ggu=ptr(260)) == WSP and bwd(gd=ptr(258)) == UNSUP


def test_tensor_cores_want_16_bytes(lib):
    fwd, bwd = calls(lib, 64, 64, BF16, BF16)
    for name in ("x", "wgu", "wd", "y"):
        assert fwd(**{name: ptr(264)}) == UNSUP and fwd(**{name: ptr(272)}) == WSP
    for name in ("x", "wgu", "wd", "gy", "gx", "ggu", "gd"):
        assert bwd(**{name: ptr(264)}) == UNSUP and bwd(**{name: ptr(272)}) == WSP


@pytest.mark.gpu
@pytest.mark.parametrize("n,h,f,dt", [(37, 33, 65, "bf16"), (20, 64, 100, "bf16"), (70, 40, 64, "f32"), (1, 3, 5, "f32")])
def test_values_do_not_depend_on_the_start(n, h, f, dt):
    """The same kernels on the same values: bit for bit what 16-byte aligned buffers give."""
    td, code = (torch.float32, F32) if dt == "f32" else (torch.bfloat16, BF16)
    gen = torch.Generator(device="cuda").manual_seed(5)
    def place(t, shift):
        raw = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
        part = raw[shift:shift + t.numel()].view(t.shape)
        part.copy_(t)
        return part
    base = [torch.randn(*s, generator=gen, device="cuda").to(td) for s in ((n, h), (2 * f, h), (h, f), (n, h))]
    mask = (torch.arange(n, device="cuda") % 3 != 1).to(torch.uint8)
    ws = a3po.new_workspace(max(a3po.a3po_gated_ffn_workspace_bytes(n, h, f, code, True, b) for b in (False, True)))
    seen = []
    for shift in (0, 1):
        x, wgu, wd, gy = (place(t, shift) for t in base)
        outs = [place(torch.full(s, 9.0, device="cuda").to(d), shift)
                for s, d in (((n, h), td), ((n, h), td), ((2 * f, h), torch.float32), ((h, f), torch.float32))]
        assert (outs[0].data_ptr() % 16 != 0) == bool(shift)
        kept = a3po.new_workspace(a3po.a3po_gated_ffn_kept_bytes(n, f, code))
        a3po.a3po_gated_ffn_fwd(x, wgu, wd, outs[0], ws, row_mask=mask, kept=kept)
        a3po.a3po_gated_ffn_bwd(x, wgu, wd, kept, gy, outs[1], outs[2], outs[3], ws, row_mask=mask)
        seen.append([o.clone() for o in outs])
    assert all(torch.equal(a, b) for a, b in zip(*seen))

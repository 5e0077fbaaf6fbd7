"""Rows longer than the row operators' 32-bit column arithmetic holds are refused on the host."""
import ctypes

import pytest

import paper_2512_06547_b200 as a3po
from paper_2512_06547_b200 import build as a3po_build

UNSUP = -2
ONE = ctypes.c_void_p(256)    # never dereferenced: every call is refused
F32, BF16, RMS, LAYER = 0, 1, 0, 1


@pytest.fixture(scope="module")
def lib():
    a3po_build.build()
    return a3po.load_library()


@pytest.mark.parametrize("h", [(1 << 30) + 1, (1 << 31) - 8192, (1 << 31) - 7, (1 << 31) - 1])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_too_long_rows(lib, h, dt):
    assert lib.a3po_norm_fwd(ONE, ONE, None, None, 1, h, dt, RMS, 1e-6, ONE, None, ONE, None) == UNSUP
    assert lib.a3po_dropout_norm_fwd(ONE, ONE, 0.5, ONE, ONE, None, None, 1, h, dt, LAYER, 1e-6, ONE, ONE, ONE, ONE, None) == UNSUP
    assert lib.a3po_dropout_fwd(ONE, None, None, 1, h, dt, 0.5, ONE, ONE, None) == UNSUP
    assert lib.a3po_dropout_bwd(ONE, None, 1, h, dt, 0.5, ONE, ONE, None) == UNSUP
    big = a3po.a3po_norm_bwd_workspace_bytes(1, h)
    assert lib.a3po_norm_bwd(ONE, ONE, ONE, ONE, None, ONE, 1, h, dt, LAYER, ONE, ONE, ONE, 0, ONE, big, None) == UNSUP
    assert lib.a3po_dropout_norm_bwd(ONE, 0.5, ONE, ONE, None, ONE, None, ONE, None, 1, h, dt, RMS, ONE, ONE, ONE, None, 0, ONE,
                                     big, None) == UNSUP

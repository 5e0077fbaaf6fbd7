"""An RMS norm with a beta: its backward gives the beta's gradient, and no caller loses it.  (Host side; the values are
tests/test_gpu_norm_beta.py.)"""
import ctypes

import pytest
import torch

import paper_2512_06547_b200 as a3po
from paper_2512_06547_b200 import build as a3po_build
from paper_2512_06547_b200.policy_tail import PolicyTail

INVAL, WSP = -1, -3
ONE = ctypes.c_void_p(256)    # never dereferenced: every call below is refused, for its workspace if for nothing else
BF16, RMS = 1, 0


@pytest.fixture(scope="module")
def lib():
    a3po_build.build()
    return a3po.load_library()


def test_backward_takes_the_beta_gradient_of_an_rms_norm(lib):
    small = a3po.a3po_norm_bwd_workspace_bytes(4, 8) - 1
    def norm(mean, grad_beta):
        return lib.a3po_norm_bwd(ONE, ONE, mean, ONE, None, ONE, 4, 8, BF16, RMS, ONE, ONE, grad_beta, 0, ONE, small, None)
    def join(mean, grad_beta):
        return lib.a3po_dropout_norm_bwd(ONE, 0.5, ONE, ONE, mean, ONE, None, ONE, None, 4, 8, BF16, RMS, ONE, ONE, ONE,
                                         grad_beta, 0, ONE, small, None)
    for call in (norm, join):
        assert call(None, ONE) == WSP and call(None, None) == WSP      # got as far as the workspace
        assert call(ONE, ONE) == INVAL and call(ONE, None) == INVAL    # an RMS norm has no mean


def test_policy_tail_does_not_lose_a_beta(lib):
    n, h, f, v = 4, 8, 16, 10
    params = {"beta_in": torch.zeros(h)}
    batch = {"mask": torch.ones(n, dtype=torch.uint8)}
    with pytest.raises(ValueError, match="beta"):
        PolicyTail(n, h, f, v, torch.float32, device="cpu")(torch.zeros(n, h), params, batch)
    tail = PolicyTail(n, h, f, v, torch.float32, beta=True, device="cpu")
    assert {"beta_in", "beta_out"} <= set(tail.grads)
    with pytest.raises(TypeError, match="CUDA device"):                # past the check, to the first operator
        tail(torch.zeros(n, h), dict(params, gamma_in=torch.ones(h)), batch)
    assert "beta_in" not in PolicyTail(n, h, f, v, torch.float32, device="cpu").grads

"""Sampling, the linear operator and AdamW beyond 2^31 elements: what lies there is what a small call makes of the same values."""
import numpy as np
import pytest
import torch

import paper_2512_06547_b200 as a3po
from paper_2512_06547_b200.optimizer import AdamW

pytestmark = pytest.mark.gpu
DEV = "cuda"
FAR = (1 << 31) + 4096


def draw(x, u, **kw):
    n, v = x.shape
    token, n_kept = (torch.empty(n, dtype=torch.int32, device=DEV) for _ in range(2))
    logp, kept_logp = (torch.empty(n, device=DEV) for _ in range(2))
    ws = a3po.new_workspace(a3po.a3po_sample_workspace_bytes(n, v), DEV)
    a3po.a3po_sample(x, u, token, ws, logp=logp, kept_logp=kept_logp, n_kept=n_kept, **kw)
    return token, n_kept, logp, kept_logp


def test_rows_of_logits_far_apart():
    v, ld = 50001, FAR // 2 + 3
    gen = torch.Generator(device=DEV).manual_seed(1)
    small = (torch.randn(3, v, generator=gen, device=DEV) * 2).bfloat16()
    buf = torch.empty(2 * ld + v, dtype=torch.bfloat16, device=DEV)
    far = buf.as_strided((3, v), (ld, 1))
    far.copy_(small)
    u = torch.tensor([0.1, 0.5, 0.97], device=DEV)
    fill = lambda x, t: torch.full((3,), x, dtype=t, device=DEV)
    for kw in ({}, dict(top_k=fill(40, torch.int32)), dict(top_p=fill(0.9, torch.float32), min_p=fill(0.001, torch.float32))):
        for a, b in zip(draw(far, u, **kw), draw(small, u, **kw)):
            # (the segments begin elsewhere: sums in another order)
            assert torch.equal(a, b) if a.dtype is torch.int32 else torch.allclose(a, b, rtol=0, atol=1e-6)


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("act", [a3po.A3PO_ACT_NONE, a3po.A3PO_ACT_SILU])
def test_linear_rows_past_2_31(masked, act):
    n, k, m, last = FAR // 8192 + 500, 8192, 16, 700
    gen = torch.Generator(device=DEV).manual_seed(2)
    randn = lambda *s: torch.randn(*s, generator=gen, device=DEV).bfloat16()
    x = torch.zeros(n, k, dtype=torch.bfloat16, device=DEV)
    x[-last:] = randn(last, k)
    w, gy, bias = randn(m, k) * k ** -0.5, randn(n, m), randn(m)
    mask = None
    if masked:
        mask = (torch.rand(n, generator=gen, device=DEV) < 0.5).to(torch.uint8)

    def both(x, gy, mask):
        n = x.shape[0]
        dt = a3po.A3PO_BF16
        y, gx, gw = torch.empty(n, m, dtype=torch.bfloat16, device=DEV), torch.empty_like(x), torch.empty(m, k, device=DEV)
        kept = a3po.new_workspace(a3po.a3po_linear_kept_bytes(n, m, dt, act), DEV) if act != a3po.A3PO_ACT_NONE else None
        ws = a3po.new_workspace(max(a3po.a3po_linear_workspace_bytes(n, k, m, dt, act, masked, bwd) for bwd in (False, True)), DEV)
        a3po.a3po_linear_fwd(x, w, y, ws, bias=bias, row_mask=mask, kept=kept, activation=act)
        a3po.a3po_linear_bwd(x, w, gy, gx, gw, ws, kept=kept, row_mask=mask, activation=act)
        return y[-last:], gx[-last:], gw

    tail = both(x[-last:].contiguous(), gy[-last:].contiguous(), None if mask is None else mask[-last:].contiguous())
    y, gx, gw = both(x, gy, mask)
    torch.cuda.synchronize()
    # one contraction over k (over m) either way, whose sums may be cut up differently: fp32 sums of at most 8192 terms, one rounding
    assert torch.allclose(y.float(), tail[0].float(), rtol=2.0 ** -7, atol=2e-3)
    assert torch.allclose(gx.float(), tail[1].float(), rtol=2.0 ** -7, atol=2e-3)
    # The rows before the last are zeros of x: they add nothing.  700 products of numbers around 1: 2^-24 of their sum each way; with
    # an activation either dz, an operand, is rounded by half a bf16 step, 2^-8 of it, and may be rounded the other way where the
    # fp32 z differ in their last bit: 2^-7 |dz|^T |x| between the two, |dz| <= 1.13 |gy|.
    bound = 2e-2 + 2.0 ** -12 * tail[2].abs()
    if act != a3po.A3PO_ACT_NONE:
        on = torch.ones(last, device=DEV) if mask is None else mask[-last:].float()
        bound = bound + 1.13 * 2.0 ** -7 * (gy[-last:].float().abs() * on[:, None]).T @ x[-last:].float().abs()
    assert bool(((gw - tail[2]).abs() <= bound).all())


@pytest.mark.parametrize("bits", [8, 32])
def test_adamw_past_2_31_elements(bits):
    tail = 256 * 5 + 77
    n = FAR // 256 * 256 + tail
    gen = torch.Generator(device=DEV).manual_seed(3)
    w = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    g = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    w[-tail:] = torch.randn(tail, generator=gen, device=DEV).bfloat16()
    g[-tail:] = torch.randn(tail, generator=gen, device=DEV).bfloat16()
    ws, gs = w[-tail:].clone(), g[-tail:].clone()
    large, small = (AdamW([t], lr=1e-2, state_bits=bits) for t in (w, ws))
    for _ in range(2):
        large.step([g])
        small.step([gs])
    torch.cuda.synchronize()
    assert torch.equal(w[-tail:], ws) and torch.equal(large.m[0][-tail:], small.m[0]) and torch.equal(large.v[0][-tail:], small.v[0])
    assert not bool(w[:n - tail:65537].any())
    assert abs(float(large.grad_norm) - float(small.grad_norm)) <= 1e-6 * float(small.grad_norm)

"""RMS norm with a beta: gradients of the rows, gamma and beta against the fp64 definition, alone, as the join and as part of
the policy's tail.  Tolerances are those of tests/test_gpu_row_ops.py and tests/test_gpu_policy_tail.py."""
import numpy as np
import pytest
import torch

import paper_2512_06547_b200 as a3po
from oracle import a3po_oracle as orc
from oracle import operators_oracle as ops
from paper_2512_06547_b200 import workloads
from paper_2512_06547_b200.policy_tail import PolicyTail
from tests.helpers import rel_fro, to_np64
from tests.test_gpu_guard_bands import Guarded
from tests.test_gpu_policy_tail import gradients, reference
from tests.test_gpu_row_ops import Case, check_norm_bwd, check_norm_fwd, rng_words

pytestmark = pytest.mark.gpu
DEV = "cuda"


# every form of the backward: narrow rows, one block a row (16-byte and element-wise rows), the re-reading one
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,h", [(1, 1), (9, 64), (70, 96), (130, 512), (33, 1003), (37, 2048), (9, 4100), (5, 8200), (4, 16384),
                                 (3, 16392)])
@pytest.mark.parametrize("join", [False, True])
def test_rms_norm_with_beta(n, h, dt, join):
    c = Case(n, h, dt, 11 * n + h, masked=0.25 if n > 2 else 0.0, scale=1.5, shift=0.5)
    G = Guarded()
    y, rstd = G.new("y", (n, h), c.td, 9.0), G.new("rstd", (n,), torch.float32, 9.0)
    a3po.a3po_norm_fwd(c.x, c.gamma, y, rstd, beta=c.beta, eps=1e-5, row_mask=c.mask)
    check_norm_fwd(c, c.x, y, None, rstd, c.beta, False, float(np.float32(1e-5)))
    gx, gg, gb = G.new("grad_x", (n, h), c.td, 9.0), G.new("grad_gamma", (h,), torch.float32, 9.0), G.new("grad_beta", (h,),
                                                                                                    torch.float32, 9.0)
    ws = G.new("ws", (a3po.a3po_norm_bwd_workspace_bytes(n, h),), torch.uint8, 0xFF)
    def run(accumulate, gbeta):
        if join:
            a3po.a3po_dropout_norm_bwd(c.x, 0.25, rng_words(), c.gamma, rstd, c.gy, gx, torch.empty_like(gx), gg, ws,
                                       grad_r=c.gr, grad_beta=gbeta, accumulate_grad_w=accumulate, row_mask=c.mask)
        else:
            a3po.a3po_norm_bwd(c.x, c.gamma, rstd, c.gy, gx, gg, ws, grad_beta=gbeta, accumulate_grad_w=accumulate,
                               row_mask=c.mask)
        G.check("backward")
    run(False, gb)
    check_norm_bwd(c, c.x, None, rstd, c.gy, c.gr if join else None, False, gx, gg, gb)
    before = gg.clone(), gb.clone()
    run(True, gb)                                          # adding a value to itself is exact
    assert torch.equal(gg, 2 * before[0]) and torch.equal(gb, 2 * before[1])
    run(False, None)                                       # not wanted: the rest within the same bounds
    check_norm_bwd(c, c.x, None, rstd, c.gy, c.gr if join else None, False, gx, gg, None)
    assert torch.equal(gb, 2 * before[1])


def test_infinite_gradient_sums_do_not_reach_an_uncentred_row():
    """mean(gx) has no part in an RMS norm, also where it is not finite: two gradients whose sum overflows fp32 leave the
    row's gradient finite."""
    n, h = 3, 64
    x, gamma = torch.ones(n, h, device=DEV), torch.ones(h, device=DEV)
    x[:, 1::2] = -1.0                                      # gx xhat cancels where gx does not
    gy = torch.full((n, h), 1.5e37, device=DEV)
    rstd, gx = torch.ones(n, device=DEV), torch.empty_like(x)
    gg, gb, ws = torch.empty(h, device=DEV), torch.empty(h, device=DEV), a3po.new_workspace(a3po.a3po_norm_bwd_workspace_bytes(n, h))
    a3po.a3po_norm_bwd(x, gamma, rstd, gy, gx, gg, ws, grad_beta=gb)
    assert torch.equal(gx, gy) and torch.equal(gb, 3 * gy[0])


@pytest.mark.parametrize("name,kw,f", [("tiny", {}, 192),
                                       ("1p5b", dict(V=2048 + 8, n_prompts=1, group=2, row_len=150, len_lo=60, len_hi=150), 520)])
def test_tail_of_rms_norms_with_beta(name, kw, f):
    wl = workloads.make_workload(name, DEV, **kw)
    n, h, v = wl.N, wl.H, wl.V
    td = torch.bfloat16 if wl.dtype == "bf16" else torch.float32
    gen = np.random.default_rng(17)
    new = lambda *s, k=1.0, c=0.0: torch.from_numpy((gen.standard_normal(s) * k + c).astype(np.float32)).to(td).to(DEV)
    r0 = new(n, h, k=1.5)
    mask = torch.from_numpy(wl.mask).to(DEV)
    r0_np = np.where((wl.mask != 0)[:, None], to_np64(r0), 0.0)
    r0[mask == 0] = float("nan")
    params = {"gamma_in": new(h, k=0.1, c=1.0), "beta_in": new(h, k=0.1), "w_gate_up": new(2 * f, h, k=h ** -0.5),
              "w_down": new(h, f, k=f ** -0.5), "gamma_out": new(h, k=0.1, c=1.0), "beta_out": new(h, k=0.1), "w": wl.w}
    p_np = {k: to_np64(t) for k, t in params.items()}
    keep = np.ones((n, h))
    s = reference(r0_np, p_np, wl, False, "silu", keep)
    behav = workloads.behav_logp_from(s["logp"], wl.behav_noise)
    terms = orc.loss_terms(s["logp"], behav, wl.versions, wl.current_version, wl.adv, wl.mask, wl.clip_eps)
    adv = np.where(terms["margin"] > 2e-2 * terms["r"], wl.adv, 0.0).astype(np.float32)   # tokens off the clip bounds
    g_ref = orc.loss_bwd(s["logp"], behav, wl.versions, wl.current_version, adv, wl.mask, wl.clip_eps)
    grads_ref, gr0_ref = gradients(r0_np, p_np, wl, False, "silu", keep, s, g_ref)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    batch = dict(targets=dev(wl.targets), behav_logp=dev(behav), versions=dev(wl.versions),
                 current_version=wl.current_version, adv=dev(adv), mask=mask, clip_eps=wl.clip_eps)
    out = PolicyTail(n, h, f, v, td, beta=True)(r0, params, batch)
    torch.cuda.synchronize()
    assert int(out["status"].item()) == 0 and set(out["grads"]) == set(params)
    tol = 1.8e-2 if wl.dtype == "bf16" else 1e-4
    for k, got in out["grads"].items():
        assert rel_fro(to_np64(got), grads_ref[k]) <= tol, (k, rel_fro(to_np64(got), grads_ref[k]))
    assert rel_fro(to_np64(out["grad_r0"]), gr0_ref) <= tol

"""The operators as they are used together: norm -> gated feed-forward -> dropout + add + norm -> LM head and loss, and
back, against the fp64 definitions chained the same way.

Tolerances are those of the path (tests/helpers.py): log-probs 2e-3 for bf16 inputs (1e-4 for fp32 ones, whose hidden
rows come out of a chain of fp32 operators), gradients 1e-2 relative Frobenius (1e-4 for fp32) plus, for bf16, the
roundings of the intermediate rows a, y, r1, hidden and their gradients: each at most 2^-8 / sqrt(3) in rms relative to
itself, ten of them in the longest chain: sqrt(10) 2^-8 / sqrt(3) = 7.2e-3, so 1.8e-2 in all."""
import numpy as np
import pytest
import torch

import paper_2512_06547_b200 as a3po
from oracle import a3po_oracle as orc
from oracle import operators_oracle as ops
from paper_2512_06547_b200 import workloads
from paper_2512_06547_b200.policy_tail import PolicyTail
from tests.helpers import rel_fro, to_np64

pytestmark = pytest.mark.gpu
DEV = "cuda"
SEED, OFFSET = 77, 5


def reference(r0, p, wl, layer, act, keep):
    mask = wl.mask
    beta = lambda k: p.get(k)
    a, mean0, rstd0 = ops.norm_fwd(r0, p["gamma_in"], beta("beta_in"), layer, 1e-6, mask)
    y = ops.gated_ffn_fwd(a, p["w_gate_up"], p["w_down"], act, mask)
    r1 = ops.dropout(y, keep, r0, mask)
    hidden, mean1, rstd1 = ops.norm_fwd(r1, p["gamma_out"], beta("beta_out"), layer, 1e-6, mask)
    logp, _ = orc.token_logprobs_fwd(hidden, p["w"], wl.targets, row_mask=mask)
    return dict(a=a, mean0=mean0, rstd0=rstd0, y=y, r1=r1, hidden=hidden, mean1=mean1, rstd1=rstd1, logp=logp)


def gradients(r0, p, wl, layer, act, keep, s, g_logp):
    gh, gw = orc.token_logprobs_bwd(s["hidden"], p["w"], wl.targets, g_logp)
    gr1, ggo, gbo = ops.norm_bwd(s["r1"], p["gamma_out"], s["mean1"], s["rstd1"], gh, layer, wl.mask)
    ga, ggu, gd = ops.gated_ffn_bwd(s["a"], p["w_gate_up"], p["w_down"], gr1 * keep, act, wl.mask)
    gr0, ggi, gbi = ops.norm_bwd(r0, p["gamma_in"], s["mean0"], s["rstd0"], ga, layer, wl.mask)
    return {"w": gw, "gamma_out": ggo, "beta_out": gbo, "w_gate_up": ggu, "w_down": gd, "gamma_in": ggi, "beta_in": gbi}, gr0 + gr1


@pytest.mark.parametrize("name,kw,f,layer,act", [
    ("tiny", {}, 192, True, "gelu_tanh"),
    ("tiny", {}, 192, False, "silu"),
    ("1p5b", dict(V=4096 + 40, n_prompts=1, group=2, row_len=192, len_lo=60, len_hi=192), 1024 + 72, False, "silu"),
    ("1p5b", dict(V=2048 + 8, n_prompts=1, group=2, row_len=11, len_lo=5, len_hi=9), 520, True, "gelu_tanh")])
def test_tail_against_the_definitions(name, kw, f, layer, act):
    wl = workloads.make_workload(name, DEV, **kw)
    n, h, v = wl.N, wl.H, wl.V
    bf16 = wl.dtype == "bf16"
    td = torch.bfloat16 if bf16 else torch.float32
    gen = np.random.default_rng(91)
    new = lambda *s, k=1.0, c=0.0: torch.from_numpy((gen.standard_normal(s) * k + c).astype(np.float32)).to(td).to(DEV)
    r0 = new(n, h, k=1.5)
    dev_mask = torch.from_numpy(wl.mask).to(DEV)
    r0_np = np.where((wl.mask != 0)[:, None], to_np64(r0), 0.0)
    r0[dev_mask == 0] = float("nan")
    params = {"gamma_in": new(h, k=0.1, c=1.0), "w_gate_up": new(2 * f, h, k=h ** -0.5), "w_down": new(h, f, k=f ** -0.5),
              "gamma_out": new(h, k=0.1, c=1.0), "w": wl.w}
    if layer:
        params.update(beta_in=new(h, k=0.1), beta_out=new(h, k=0.1))
    p_np = {k: to_np64(t) for k, t in params.items()}
    drop = 0.125
    keep = ops.dropout_factors(n, h, drop, SEED, OFFSET)
    s = reference(r0_np, p_np, wl, layer, act, keep)
    behav = workloads.behav_logp_from(s["logp"], wl.behav_noise)
    terms = orc.loss_terms(s["logp"], behav, wl.versions, wl.current_version, wl.adv, wl.mask, wl.clip_eps)
    # tokens near a clip bound may take either branch when their log-prob is off by its tolerance: left out by advantage 0
    adv = np.where(terms["margin"] > 2e-2 * terms["r"], wl.adv, 0.0).astype(np.float32)
    args = (s["logp"], behav, wl.versions, wl.current_version, adv, wl.mask, wl.clip_eps)
    loss_ref, _ = orc.loss_fwd(*args)
    g_ref = orc.loss_bwd(*args)
    grads_ref, gr0_ref = gradients(r0_np, p_np, wl, layer, act, keep, s, g_ref)

    tail = PolicyTail(n, h, f, v, td, kind=a3po.A3PO_NORM_LAYER if layer else a3po.A3PO_NORM_RMS,
                      activation=a3po.A3PO_ACT_SILU if act == "silu" else a3po.A3PO_ACT_GELU_TANH, dropout_p=drop)
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(DEV)
    batch = dict(targets=dev(wl.targets), behav_logp=dev(behav), versions=dev(wl.versions),
                 current_version=wl.current_version, adv=dev(adv), mask=dev_mask, clip_eps=wl.clip_eps)
    rng = torch.tensor([SEED, OFFSET], dtype=torch.int64, device=DEV)
    out = tail(r0, params, batch, rng)
    torch.cuda.synchronize()
    assert int(out["status"].item()) == 0
    valid = wl.mask != 0
    # bf16: the hidden rows carry the roundings of the chain (each about 2^-9 of a row), and a logit is a sum of H of
    # their products with weights of 1 / sqrt(H): off by about sqrt(4) 2^-9 |hidden| / sqrt(H) ~ 4e-3 in rms, 5 sigma
    assert np.max(np.abs(to_np64(out["logp"]) - s["logp"])[valid]) <= (2e-2 if bf16 else 1e-4)
    assert abs(float(out["loss"].item()) - loss_ref) <= (2e-2 if bf16 else 1e-4) * np.abs(adv[valid]).mean() * 3
    # the loss's own gradient moves with the log-prob error: |dg| <= 2 |g| dlogp, 2 x 4e-3 rms for bf16
    tol = 1.8e-2 if bf16 else 1e-4
    for k, got in out["grads"].items():
        assert rel_fro(to_np64(got), grads_ref[k]) <= tol, (k, rel_fro(to_np64(got), grads_ref[k]))
    assert rel_fro(to_np64(out["grad_r0"]), gr0_ref) <= tol
    assert bool((out["grad_r0"][dev_mask == 0] == 0).all())

    # a second pass that accumulates, then a captured one: bit-identical gradients
    first = {k: t.clone() for k, t in out["grads"].items()}
    gr0 = out["grad_r0"].clone()
    tail(r0, params, batch, rng)
    assert all(torch.equal(first[k], t) for k, t in tail.grads.items()) and torch.equal(gr0, tail.grad_r0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tail(r0, params, batch, rng)
    for t in tail.grads.values():
        t.fill_(7.0)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(first[k], t) for k, t in tail.grads.items()) and torch.equal(gr0, tail.grad_r0)
    rng[1] += 1                                            # the replay draws another mask
    graph.replay()
    torch.cuda.synchronize()
    assert not torch.equal(gr0, tail.grad_r0)

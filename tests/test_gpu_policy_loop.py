"""The operators as a trainer uses them: tokens are drawn from the policy's tail, the same rows go through the loss with the
log-probs that the draw left, and the weights are updated with the gradients; against the fp64 definitions chained the same way.

Tolerances: log-probs as in the path (2e-3 for bf16 inputs whose hidden rows come out of a chain of bf16 operators: 2e-2 as in
the forward chain's own check; 1e-4 for fp32).  The draw and the pass compute the same rows with the same kernels, so that
their log-probs differ by the LM head's fp32 sums alone: 2^-24 K times the largest |hidden| |w| sum, below 1e-3.
Updates: one AdamW step moves a weight by at most lr (1 + decay |w|) / (1 - b1) ..., so the check is on the step's own arithmetic
with the gradients that the pass left (they are checked against the definitions elsewhere)."""
import numpy as np
import pytest
import torch

import paper_2512_06547_b200 as a3po
from oracle import a3po_oracle as orc
from oracle import operators_oracle as ops
from paper_2512_06547_b200.policy_tail import PolicySampler, PolicyTail
from tests.helpers import to_np64

pytestmark = pytest.mark.gpu
DEV = "cuda"


def make(n, h, f, v, td, layer, seed=3):
    gen = np.random.default_rng(seed)
    new = lambda *s, k=1.0, c=0.0: torch.from_numpy((gen.standard_normal(s) * k + c).astype(np.float32)).to(td).to(DEV)
    params = {"gamma_in": new(h, k=0.1, c=1.0), "w_gate_up": new(2 * f, h, k=h ** -0.5), "w_down": new(h, f, k=f ** -0.5),
              "gamma_out": new(h, k=0.1, c=1.0), "w": new(v, h, k=2.0 * h ** -0.5)}
    if layer:
        params.update(beta_in=new(h, k=0.1), beta_out=new(h, k=0.1))
    mask = (gen.random(n) < 0.8).astype(np.uint8)
    mask[0] = 1
    r0 = new(n, h, k=1.5)
    r0[torch.from_numpy(mask == 0).to(DEV)] = float("nan")
    return params, r0, mask, gen


@pytest.mark.parametrize("td,n,h,f,v,layer", [(torch.float32, 50, 64, 192, 1000, True), (torch.bfloat16, 13, 512, 1024, 4136, False),
                                              (torch.bfloat16, 150, 256, 520, 2056, False), (torch.bfloat16, 1, 1536, 4608, 20008, False)])
@pytest.mark.parametrize("bits", [32, 8])
def test_rollout_loss_and_update(td, n, h, f, v, layer, bits):
    params, r0, mask, gen = make(n, h, f, v, td, layer)
    kind = a3po.A3PO_NORM_LAYER if layer else a3po.A3PO_NORM_RMS
    dev = lambda x, t: torch.from_numpy(np.ascontiguousarray(x)).to(t).to(DEV)
    m = dev(mask, torch.uint8)
    sampler, tail = PolicySampler(n, h, f, v, td, kind=kind), PolicyTail(n, h, f, v, td, kind=kind)
    opt = tail.optimizer(params, lr=1e-2, betas=(0.9, 0.95), max_grad_norm=0.5, state_bits=bits)
    u = gen.random(n).astype(np.float32)
    p, top_k = np.full(n, 0.95, np.float32), np.full(n, 30, np.int32)
    before = None
    for step in range(3):
        got = sampler(r0, params, dev(u, torch.float32), top_k=dev(top_k, torch.int32), top_p=dev(p, torch.float32), row_mask=m)
        token, behav = got["token"].clone(), got["logp"].clone()
        torch.cuda.synchronize()
        assert int(got["status"].item()) == 0
        on = mask != 0
        assert (to_np64(token)[~on] == -1).all() and (to_np64(behav)[~on] == 0).all()
        # the draw against the definition on the logits that it was made from
        logits = to_np64(got["logits"])
        for i in np.flatnonzero(on)[:20]:
            ref = ops.sample_row(logits[i], float(u[i]), top_k=30, top_p=0.95)
            assert int(token[i]) == ref["token"] and abs(float(behav[i]) - ref["logp"]) <= 1e-6 * max(1.0, abs(ref["logp"]))
        # and the logits against the chained definitions
        sel = lambda x: np.where(on[:, None], x, 0.0)
        pn = {k: to_np64(x) for k, x in params.items()}
        a, _, _ = ops.norm_fwd(sel(np.nan_to_num(to_np64(r0))), pn["gamma_in"], pn.get("beta_in"), layer, 1e-6, mask)
        r1 = sel(np.nan_to_num(to_np64(r0))) + ops.gated_ffn_fwd(a, pn["w_gate_up"], pn["w_down"], mask=mask)
        hidden, _, _ = ops.norm_fwd(r1, pn["gamma_out"], pn.get("beta_out"), layer, 1e-6, mask)
        tok = np.where(on, to_np64(token), 0)
        logp_ref, _ = orc.token_logprobs_fwd(hidden, pn["w"], tok, row_mask=mask)
        assert np.abs(to_np64(behav) - logp_ref)[on].max() <= (1e-4 if td == torch.float32 else 4e-2)
        # the pass on the drawn tokens: the policy is the one that drew them
        batch = dict(targets=dev(tok, torch.int32), behav_logp=behav, versions=torch.full((n,), 5, dtype=torch.int32, device=DEV),
                     current_version=5 + step, adv=dev(gen.standard_normal(n).astype(np.float32), torch.float32), mask=m, clip_eps=0.2)
        out = tail(r0, params, batch)
        torch.cuda.synchronize()
        assert float((out["logp"] - behav).abs()[m != 0].max()) <= 1e-3
        # the update
        if before is None:
            before = {k: to_np64(x) for k, x in params.items()}
            state = {k: (np.zeros(x.size), np.zeros(x.size)) for k, x in before.items()}
        tail.update(opt)
        torch.cuda.synchronize()
        grads = [to_np64(g).ravel() for g in out["grads"].values()]
        norm, scale = ops.clip_scale(grads, 0.5)
        assert norm > 0 and abs(float(opt.grad_norm.item()) - norm) <= 1e-6 * norm
        if step == 0:
            for (k, g), w in zip(out["grads"].items(), grads):
                ref, _, _ = ops.adamw(before[k].ravel(), w, *state[k], 1, 1e-2, 0.9, 0.95, 1e-8, 0.01 if g.dim() > 1 else 0.0, scale)
                # a bf16 weight is a rounding of its master; the step itself is at most 1.0 lr here, good to 2^-18 of it
                bound = 1e-2 * 2.0 ** -18 + (2.0 ** -8 if td == torch.bfloat16 else 2.0 ** -22) * np.abs(ref) + 1e-7
                assert (np.abs(to_np64(params[k]).ravel() - ref) <= bound).all(), k
    assert int(opt.steps.item()) == 3


def test_rollout_pass_captured():
    n, h, f, v = 9, 256, 512, 3000
    params, r0, mask, gen = make(n, h, f, v, torch.bfloat16, False)
    r0 = torch.nan_to_num(r0)
    u = torch.rand(n, device=DEV)
    sampler = PolicySampler(n, h, f, v)
    k = torch.full((n,), 40, dtype=torch.int32, device=DEV)
    first = {x: t.clone() for x, t in sampler(r0, params, u, top_k=k).items()}
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = sampler(r0, params, u, top_k=k)
    for t in out.values():
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(out[x], first[x]) for x in out)
    u.copy_(1 - u)
    graph.replay()
    torch.cuda.synchronize()
    moved = {x: t.clone() for x, t in out.items()}
    again = sampler(r0, params, u, top_k=k)
    torch.cuda.synchronize()
    assert all(torch.equal(moved[x], again[x]) for x in again) and not torch.equal(moved["token"], first["token"])

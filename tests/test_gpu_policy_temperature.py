"""Tokens drawn at a temperature and trained at it: the pass's log-probs are those that the draw left.

Both compute the same rows with the same kernels up to the LM head, so that their log-probs differ by its fp32 sums alone, as at
temperature 1 (2^-24 K times the largest |hidden| |w| sum, below 1e-3), times the 1 / t that logits are multiplied with."""
import pytest
import torch

import paper_2512_06547_b200 as a3po
from paper_2512_06547_b200.policy_tail import PolicySampler, PolicyTail
from tests.test_gpu_policy_loop import make

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("td,n,h,f,v", [(torch.float32, 50, 64, 192, 1000), (torch.bfloat16, 150, 256, 520, 2056)])
@pytest.mark.parametrize("t", [0.7, 1.0, 1.6])
def test_rollout_and_loss_at_a_temperature(td, n, h, f, v, t):
    params, r0, mask, gen = make(n, h, f, v, td, False)
    m = torch.from_numpy(mask).to(DEV)
    new = lambda x, ty=torch.float32: torch.full((n,), x, dtype=ty, device=DEV)
    sampler, tail = PolicySampler(n, h, f, v, td), PolicyTail(n, h, f, v, td)
    got = sampler(r0, params, torch.from_numpy(gen.random(n).astype("float32")).to(DEV), temperature=new(t), row_mask=m)
    token, behav = got["token"].clamp_min(0), got["logp"].clone()
    batch = dict(targets=token, behav_logp=behav, versions=new(5, torch.int32), current_version=5, adv=new(1.0), mask=m,
                 clip_eps=0.2)
    out = tail(r0, params, batch, inv_temperature=1 / t)
    torch.cuda.synchronize()
    assert float((out["logp"] - behav).abs()[m != 0].max()) <= 1e-3 / min(t, 1.0)
    # the gradients are the step's at that temperature
    logp, lse, grad_logp, loss = (torch.empty(n, device=DEV) for _ in range(4))
    grad_hidden, grad_w = torch.empty_like(tail.hidden), torch.empty_like(tail.grads["w"])
    a3po.a3po_train_step(tail.hidden, params["w"], token, behav, batch["versions"], 5, batch["adv"], m, 0.2, logp, lse, grad_logp,
                         loss[:1], grad_hidden, grad_w, tail.ws, inv_temperature=1 / t)
    torch.cuda.synchronize()
    assert torch.equal(out["logp"], logp) and torch.equal(out["loss"], loss[:1])
    assert torch.equal(tail.grad_hidden, grad_hidden) and torch.equal(out["grads"]["w"], grad_w)


def test_a_temperature_moves_the_log_probs():
    n, h, f, v = 20, 64, 192, 1000
    params, r0, mask, gen = make(n, h, f, v, torch.float32, False)
    m = torch.from_numpy(mask).to(DEV)
    new = lambda x, ty=torch.float32: torch.full((n,), x, dtype=ty, device=DEV)
    tail = PolicyTail(n, h, f, v, torch.float32)
    batch = dict(targets=new(3, torch.int32), behav_logp=new(-1.0), versions=new(5, torch.int32), current_version=5, adv=new(1.0),
                 mask=m, clip_eps=0.2)
    logp = [tail(r0, params, batch, **kw)["logp"].clone() for kw in ({}, dict(inv_temperature=1.0), dict(inv_temperature=2.0))]
    torch.cuda.synchronize()
    assert torch.equal(logp[0], logp[1]) and not torch.allclose(logp[0], logp[2])

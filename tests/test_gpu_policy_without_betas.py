"""A tail of layer norms whose params hold no beta, or one of the two: the pass computes gradients of both, and the update is of the
parameters that there are."""
import pytest
import torch

import paper_2512_06547_b200 as a3po
from paper_2512_06547_b200.optimizer import AdamW
from paper_2512_06547_b200.policy_tail import PolicyTail
from tests.test_gpu_policy_loop import make

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("betas", [(), ("beta_out",), ("beta_in", "beta_out")])
@pytest.mark.parametrize("given", ["left out", "None"])
def test_update(betas, given):
    n, h, f, v = 20, 64, 192, 1000
    params, r0, mask, gen = make(n, h, f, v, torch.float32, True)
    for name in ("beta_in", "beta_out"):
        if name not in betas:
            if given == "None":
                params[name] = None
            else:
                del params[name]
    new = lambda x, ty=torch.float32: torch.full((n,), x, dtype=ty, device=DEV)
    m = torch.from_numpy(mask).to(DEV)
    tail = PolicyTail(n, h, f, v, torch.float32, kind=a3po.A3PO_NORM_LAYER)
    opt = tail.optimizer(params, lr=1e-2, max_grad_norm=1.0)
    batch = dict(targets=new(3, torch.int32), behav_logp=new(-3.0), versions=new(5, torch.int32), current_version=5, adv=new(1.0),
                 mask=m, clip_eps=0.2)
    before = {k: p.clone() for k, p in params.items() if p is not None}
    out = tail(r0, params, batch)
    tail.update(opt)
    torch.cuda.synchronize()
    assert len(opt.weights) == len(before)
    for k, p in before.items():
        moved = (params[k] - p).abs()
        assert 0 < float(moved.max()) <= 0.011, k               # a first step moves a weight by lr (1 + decay |w|) at most
    squares = sum(float(out["grads"][k].double().square().sum()) for k in before)
    assert abs(float(opt.grad_norm.item()) - squares ** 0.5) <= 1e-6 * squares ** 0.5    # of what is updated


def test_update_by_an_optimizer_of_the_callers_own():
    n, h, f, v = 20, 64, 192, 1000
    params, r0, mask, gen = make(n, h, f, v, torch.float32, False)
    new = lambda x, ty=torch.float32: torch.full((n,), x, dtype=ty, device=DEV)
    tail = PolicyTail(n, h, f, v, torch.float32)
    opt = AdamW([params[k] for k in tail.grads], lr=1e-2)
    before = {k: params[k].clone() for k in tail.grads}
    tail(r0, params, dict(targets=new(3, torch.int32), behav_logp=new(-3.0), versions=new(5, torch.int32), current_version=5,
                          adv=new(1.0), mask=torch.from_numpy(mask).to(DEV), clip_eps=0.2))
    tail.update(opt)
    torch.cuda.synchronize()
    assert int(opt.steps.item()) == 1 and all(not torch.equal(params[k], before[k]) for k in before)

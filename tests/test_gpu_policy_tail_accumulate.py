"""PolicyTail with accumulate_grads: a pass adds its gradients to what the buffers hold."""
import numpy as np
import pytest
import torch

from paper_2512_06547_b200 import workloads
from paper_2512_06547_b200.policy_tail import PolicyTail
import paper_2512_06547_b200 as a3po

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("name,kw,f,layer", [
    ("tiny", {}, 192, True), ("tiny", {}, 192, False),
    ("1p5b", dict(V=4096 + 40, n_prompts=1, group=2, row_len=192, len_lo=60, len_hi=192), 1024 + 72, True),
    ("1p5b", dict(V=2048 + 8, n_prompts=1, group=2, row_len=11, len_lo=5, len_hi=9), 520, False)])
def test_accumulation(name, kw, f, layer):
    wl = workloads.make_workload(name, DEV, **kw)
    n, h, v = wl.N, wl.H, wl.V
    td = torch.bfloat16 if wl.dtype == "bf16" else torch.float32
    gen = torch.Generator(device=DEV).manual_seed(4)
    new = lambda *s, k=1.0, c=0.0: (torch.randn(*s, generator=gen, device=DEV) * k + c).to(td)
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(DEV)
    mask = dev(wl.mask)
    params = {"gamma_in": new(h, k=0.1, c=1.0), "w_gate_up": new(2 * f, h, k=h ** -0.5), "w_down": new(h, f, k=f ** -0.5),
              "gamma_out": new(h, k=0.1, c=1.0), "w": wl.w}
    if layer:
        params.update(beta_in=new(h, k=0.1), beta_out=new(h, k=0.1))
    def rows():
        r = new(n, h, k=1.5)
        r[mask == 0] = float("nan")
        return r
    batch = dict(targets=dev(wl.targets), behav_logp=torch.full((n,), -3.0, device=DEV), versions=dev(wl.versions),
                 current_version=wl.current_version, adv=dev(wl.adv), mask=mask, clip_eps=wl.clip_eps)
    tail = PolicyTail(n, h, f, v, td, kind=a3po.A3PO_NORM_LAYER if layer else a3po.A3PO_NORM_RMS, dropout_p=0.125)
    rng = torch.tensor([5, 6], dtype=torch.int64, device=DEV)
    one, two = rows(), rows()
    def grads(r, accumulate=False):
        out = tail(r, params, batch, rng, accumulate_grads=accumulate)
        return {k: t.clone() for k, t in out["grads"].items()}
    g1, g2 = grads(one), grads(two)
    both = grads(one, True)                                # on top of g2: every call computes its sum first and adds it once
    for k in g1:
        assert bool((g1[k] != 0).any()) and torch.equal(both[k], g2[k] + g1[k]), k
    assert int(tail.status.item()) == 0
    # the rows' gradients do not accumulate
    tail(one, params, batch, rng)
    first = tail.grad_r0.clone()
    tail(one, params, batch, rng, accumulate_grads=True)
    assert torch.equal(first, tail.grad_r0)

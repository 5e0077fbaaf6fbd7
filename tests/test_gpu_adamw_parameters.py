"""Weights that autograd knows: masters made of them are tensors of their own, which can be copied and loaded."""
import copy

import pytest
import torch

from paper_2512_06547_b200.optimizer import AdamW

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_masters_of_parameters():
    w = torch.nn.Parameter(torch.ones(300, device=DEV, dtype=torch.bfloat16))
    opt = AdamW([w], lr=0.1, masters=True)
    (w.float() ** 2).sum().backward()
    opt.step([w.grad])
    held = copy.deepcopy(opt.masters)
    opt.step([w.grad])
    opt.masters[0].copy_(held[0])
    torch.cuda.synchronize()
    assert not opt.masters[0].requires_grad and opt.masters[0].grad_fn is None
    assert torch.equal(opt.masters[0], held[0]) and float(w.detach().max()) < 1

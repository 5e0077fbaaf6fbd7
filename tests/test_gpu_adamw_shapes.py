"""Gradients whose number of elements is right and whose shape is another's."""
import pytest
import torch

from paper_2512_06547_b200.optimizer import AdamW

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_shapes():
    w = torch.zeros(6, 4, device=DEV)
    opt = AdamW([w], lr=0.1, weight_decay=0.0)
    g = torch.arange(1.0, 25.0, device=DEV)
    for bad in (g.view(4, 6), g.view(6, 2, 2), g.view(1, 24), g.view(24, 1)):
        with pytest.raises(ValueError):
            opt.step([bad])
    assert int(opt.steps.item()) == 0
    opt.step([g.view(6, 4)])
    opt.step([g])                    # a piece of a flat buffer of gradients
    torch.cuda.synchronize()
    assert int(opt.steps.item()) == 2 and bool((w < 0).all())
    scalar = torch.zeros((), device=DEV)
    one = AdamW([scalar], lr=0.1)
    one.step([torch.ones((), device=DEV)])
    one.step([torch.ones(1, device=DEV)])
    torch.cuda.synchronize()
    assert int(one.steps.item()) == 2 and float(scalar) < 0

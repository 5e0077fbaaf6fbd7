"""Draws from batches whose rows have all finished, by the two launches of rows without a filter, with the writes of the mask and the
logits and the next draw right behind them: the next draw is what it is alone."""
import pytest
import torch

import paper_2512_06547_b200 as a3po

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("td", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,v", [(1, 151936), (5, 4099), (600, 20011)])
def test_all_rows_masked(td, n, v):
    gen = torch.Generator(device=DEV).manual_seed(5)
    held = (torch.randn(n, v, generator=gen, device=DEV) * 2).to(td)
    u = torch.rand(n, generator=gen, device=DEV)
    ws = a3po.new_workspace(a3po.a3po_sample_workspace_bytes(n, v), DEV)
    new = lambda dtype: torch.full((n,), 9, dtype=dtype, device=DEV)
    outs = [(new(torch.int32), new(torch.float32), new(torch.int32)) for _ in range(3)]
    draw = lambda x, mask, out: a3po.a3po_sample(x, u, out[0], ws, row_mask=mask, logp=out[1], n_kept=out[2])
    draw(held, None, outs[0])
    torch.cuda.synchronize()
    logits, mask = torch.full_like(held, float("nan")), torch.zeros(n, dtype=torch.uint8, device=DEV)
    for _ in range(20):
        mask.zero_()
        logits.fill_(float("nan"))
        draw(logits, mask, outs[1])
        mask.fill_(1)
        logits.copy_(held)
        draw(logits, mask, outs[2])
    torch.cuda.synchronize()
    assert (outs[1][0] == -1).all() and not outs[1][1].any() and not outs[1][2].any()
    for a, b in zip(outs[0], outs[2]):
        assert torch.equal(a, b)


@pytest.mark.parametrize("filters", [False, True])
def test_masked_rows_between_others(filters):
    n, v = 64, 8191
    gen = torch.Generator(device=DEV).manual_seed(6)
    logits = torch.randn(n, v, generator=gen, device=DEV) * 2
    u = torch.rand(n, generator=gen, device=DEV)
    ws = a3po.new_workspace(a3po.a3po_sample_workspace_bytes(n, v), DEV)
    more = dict(top_k=torch.full((n,), 30, dtype=torch.int32, device=DEV)) if filters else {}
    whole, some = (torch.empty(n, dtype=torch.int32, device=DEV) for _ in range(2))
    a3po.a3po_sample(logits, u, whole, ws, **more)
    for keep in (0, 1, 31):
        mask = torch.zeros(n, dtype=torch.uint8, device=DEV)
        mask[:keep] = 1
        a3po.a3po_sample(torch.where(mask[:, None] != 0, logits, float("nan")), u, some, ws, row_mask=mask, **more)
        torch.cuda.synchronize()
        assert torch.equal(some[:keep], whole[:keep]) and (some[keep:] == -1).all()

"""fp32 outputs of long sums: weight gradients over many rows, and fp32 logits of wide rows, to a few roundings (2-norm)."""
import pytest
import torch

import paper_2512_06547_b200 as a3po

pytestmark = pytest.mark.gpu
DEV = "cuda"


def rel(a, b):
    return float((a.double() - b).norm() / b.norm())


@pytest.mark.parametrize("n,k,m", [(16384, 512, 512), (16384, 64, 40), (50000, 136, 264), (4100, 1536, 1536)])
@pytest.mark.parametrize("masked", [False, True])
def test_weight_gradient(n, k, m, masked):
    """Sums of 512 products are cut off at each of 32 additions in the tensor cores (each at most 2^-23 of the sum), then added with
    rounding: 32 2^-23 + n / 512 2^-24 < 1e-5 for these n, and in the 2-norm well below."""
    gen = torch.Generator(device=DEV).manual_seed(n + m)
    x = torch.randn(n, k, device=DEV, generator=gen).bfloat16()
    gy = torch.randn(n, m, device=DEV, generator=gen).bfloat16()
    w = torch.randn(m, k, device=DEV, generator=gen).bfloat16()
    mask = (torch.rand(n, device=DEV, generator=gen) < 0.6).to(torch.uint8) if masked else None
    gw = torch.empty(m, k, device=DEV)
    gb = torch.empty(m, device=DEV)
    ws = a3po.new_workspace(a3po.a3po_linear_workspace_bytes(n, k, m, a3po.A3PO_BF16, has_row_mask=masked, is_bwd=True), DEV)
    a3po.a3po_linear_bwd(x, w, gy, None, gw, ws, grad_bias=gb, row_mask=mask)
    torch.cuda.synchronize()
    g = gy.double() if mask is None else gy.double() * mask.unsqueeze(1)
    assert rel(gw, g.t() @ x.double()) <= 1e-5
    assert rel(gb, g.sum(dim=0)) <= 1e-5


@pytest.mark.parametrize("n,k,m", [(40, 4096, 1024), (40, 10240, 256), (130, 4096, 20000), (600, 2056, 4104), (20, 8200, 2568)])
def test_fp32_output(n, k, m):
    gen = torch.Generator(device=DEV).manual_seed(k)
    x = torch.randn(n, k, device=DEV, generator=gen).bfloat16()
    w = torch.randn(m, k, device=DEV, generator=gen).bfloat16()
    y = torch.empty(n, m, device=DEV)
    ws = a3po.new_workspace(a3po.a3po_linear_workspace_bytes(n, k, m, a3po.A3PO_BF16), DEV)
    a3po.a3po_linear_fwd(x, w, y, ws)
    torch.cuda.synchronize()
    assert rel(y, x.double() @ w.double().t()) <= 1e-5

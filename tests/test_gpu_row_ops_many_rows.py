"""The row operators where a block works through many rows: its ring of rows wraps, masks and statistics are read ahead, masked
rows are skipped in between, and the weight gradients collect many rows per block.  Every row is different; references are
fp64 on the GPU.  Tolerances are those of tests/test_gpu_row_ops.py (u = 2^-24, e half a step of the storage type), except
the weight gradients, which are exact here: the rows' statistics are inputs of the backward, so that with small integers for x,
grad_y and mean and powers of two for rstd every product and every partial sum is a multiple of 1/2 below 2^23."""
import pytest
import torch

import paper_2512_06547_b200 as a3po
from tests.philox_torch import dropout_factors

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
TD = {"f32": torch.float32, "bf16": torch.bfloat16}
SEED, OFFSET = 0x123456789ABCDEF, (5 << 32) + 3
P = 0.3

# (n, h): rows over blocks that fit 148 SMs
SHAPES = [
    (80000, 520, "bf16"),      # a block a row, 16-byte rows: up to 68 rows per block, dealt out in groups of 8
    (40001, 520, "f32"),
    (20003, 1003, "bf16"),     # rows that start at any element
    (20003, 1003, "f32"),
    (700001, 40, "bf16"),      # 32 rows at a time per block
    (300000, 33, "f32"),
    (60000, 512, "bf16"),      # 8 rows at a time, 2 chunks per thread
    (30000, 4096, "bf16"),     # forward: a block per 16 rows; backward: 46 rows per block
    (6000, 6001, "bf16"),      # long rows, element-wise
    (6000, 8192, "f32"),
    (3000, 16384, "bf16"),
    (2000, 12001, "f32"),
]


def half_step(dt):
    return torch.finfo(TD[dt]).eps / 2


def make_mask(n, kind, gen):
    if kind == "none":
        return None
    if kind == "random":
        m = torch.rand(n, generator=gen, device=DEV) > 0.35
    else:                       # right padding: runs of valid and of masked rows
        t = torch.arange(n, device=DEV)
        m = (t % 257) < 40 + (t // 257 * 37) % 217
    return m.to(torch.uint8)


def poison(mask, *ts):
    for t in ts:
        if mask is not None:
            t[mask == 0] = float("nan")


def wide(t, mask):
    t = t.double()
    return t if mask is None else t.masked_fill_((mask == 0).unsqueeze(1) if t.dim() == 2 else mask == 0, 0.0)


def close(got, ref, bound, what):
    bad = ~((got.double() - ref).abs() <= bound + 1e-37)
    assert not bool(bad.any()), (what, int(bad.sum()), bad.nonzero()[:3].tolist())


def check_forward(x, mask, gamma, beta, layer, y, mean, rstd, dt, eps):
    xs = wide(x, mask)
    mabs = xs.abs().mean(dim=1, keepdim=True)
    mu = xs.mean(dim=1, keepdim=True) if layer else torch.zeros_like(mabs)
    keep = torch.ones_like(mabs) if mask is None else (mask != 0).double().unsqueeze(1)
    rs = 1 / ((xs - mu).square().mean(dim=1, keepdim=True) + eps).sqrt()
    g, b = gamma.double(), beta.double() if beta is not None else torch.zeros_like(gamma, dtype=torch.double)
    ref = ((xs - mu) * rs * g + b) * keep
    spread = rs * g.abs()
    close(y, ref, 64 * U * ((xs - mu).abs() * spread + b.abs() + spread * mabs) + half_step(dt) * ref.abs(), "y")
    k, rs, mabs = keep[:, 0], rs[:, 0], mabs[:, 0]
    if layer:
        close(mean, mu[:, 0] * k, 40 * U * mabs, "mean")
        close(rstd, rs * k, rs * (24 * U + 40 * U * mabs * rs), "rstd")
    else:
        close(rstd, rs * k, 24 * U * rs, "rstd")


@pytest.mark.parametrize("masked", ["none", "random", "padding"])
@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("n,h,dt", SHAPES)
def test_forward(n, h, dt, layer, masked):
    gen = torch.Generator(device=DEV).manual_seed(n + h)
    td = TD[dt]
    kind = a3po.A3PO_NORM_LAYER if layer else a3po.A3PO_NORM_RMS
    eps = float(torch.tensor(1e-5))
    row = torch.rand(n, 1, generator=gen, device=DEV) * 3 + 0.2        # every row of a size of its own
    x = ((torch.randn(n, h, generator=gen, device=DEV) + 0.5) * row).to(td)
    gamma = (torch.randn(h, generator=gen, device=DEV) * 0.2 + 1).to(td)
    beta = (torch.randn(h, generator=gen, device=DEV) * 0.3).to(td) if layer else None
    mask = make_mask(n, masked, gen)
    poison(mask, x)
    y, rstd = torch.full_like(x, 9.0), torch.full((n,), 9.0, device=DEV)
    mean = torch.full((n,), 9.0, device=DEV) if layer else None
    a3po.a3po_norm_fwd(x, gamma, y, rstd, kind=kind, beta=beta, mean=mean, eps=1e-5, row_mask=mask)
    check_forward(x, mask, gamma, beta, layer, y, mean, rstd, dt, eps)

    res = (torch.randn(n, h, generator=gen, device=DEV) * 2).to(td)
    poison(mask, res)
    rng = torch.tensor([SEED, OFFSET], dtype=torch.int64, device=DEV)
    r = torch.full_like(x, 9.0)
    a3po.a3po_dropout_norm_fwd(x, res, P, rng, gamma, r, y, rstd, kind=kind, beta=beta, mean=mean, eps=1e-5, row_mask=mask)
    factor = dropout_factors(n, h, P, SEED, OFFSET, DEV)
    xs, rs = wide(x, mask) * factor, wide(res, mask)
    ref = xs + rs
    close(r, ref, 3 * U * (xs.abs() + rs.abs()) + half_step(dt) * ref.abs() * (1 + 4 * U), "r")
    check_forward(r, mask, gamma, beta, layer, y, mean, rstd, dt, eps)
    del factor, xs, rs, ref
    r2 = torch.full_like(x, 9.0)
    a3po.a3po_dropout_fwd(x, P, rng, r2, residual=res, row_mask=mask)  # a block's many turns (odd H), or none
    assert torch.equal(r, r2)


@pytest.mark.parametrize("masked", ["none", "random", "padding"])
@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("n,h,dt", SHAPES)
def test_backward(n, h, dt, layer, masked):
    gen = torch.Generator(device=DEV).manual_seed(2 * n + h)
    td = TD[dt]
    kind = a3po.A3PO_NORM_LAYER if layer else a3po.A3PO_NORM_RMS
    ints = lambda lo, hi, *s: torch.randint(lo, hi + 1, s, generator=gen, device=DEV).float()
    # |gy xhat| <= 1 (4 + 1) 2 = 10 on at most 700,001 rows, in halves: below 2^23
    x, gy = ints(-4, 4, n, h).to(td), ints(-1, 1, n, h).to(td)
    gr = torch.randn(n, h, generator=gen, device=DEV).to(td)
    rstd = torch.tensor([0.5, 1.0, 2.0], device=DEV)[torch.randint(0, 3, (n,), generator=gen, device=DEV)]
    mean = ints(-1, 1, n) if layer else None
    gamma = (torch.randn(h, generator=gen, device=DEV) * 0.2 + 1).to(td)
    mask = make_mask(n, masked, gen)
    stats = [rstd.clone()] + ([mean.clone()] if layer else [])
    poison(mask, x, gy, gr, *stats)                       # statistics of masked rows may be anything
    gx, gg = torch.full_like(x, 9.0), torch.full((h,), 9.0, device=DEV)
    gb = torch.full((h,), 9.0, device=DEV)
    ws = torch.full((a3po.a3po_norm_bwd_workspace_bytes(n, h),), 0xFF, dtype=torch.uint8, device=DEV)
    a3po.a3po_norm_bwd(x, gamma, stats[0], gy, gx, gg, ws, kind=kind, mean=stats[1] if layer else None, grad_beta=gb,
                       row_mask=mask)
    xs, gys, rs = wide(x, mask), wide(gy, mask), wide(rstd, mask).unsqueeze(1)
    xhat = (xs - (wide(mean, mask).unsqueeze(1) if layer else 0.0)) * rs
    want_gamma, want_beta = (gys * xhat).sum(dim=0), gys.sum(dim=0)
    assert torch.equal(gg.double(), want_gamma) and torch.equal(gb.double(), want_beta)
    g = gys * gamma.double()
    inner = (g * xhat).mean(dim=1, keepdim=True)
    ref = (g - (g.mean(dim=1, keepdim=True) if layer else 0.0) - xhat * inner) * rs
    size = rs * (g.abs() + (g.abs().mean(dim=1, keepdim=True) if layer else 0.0)
                 + xhat.abs() * (g * xhat).abs().mean(dim=1, keepdim=True))
    close(gx, ref, 64 * U * size + half_step(dt) * ref.abs(), "grad_x")

    rng = torch.tensor([SEED, OFFSET], dtype=torch.int64, device=DEV)
    gres, gbr = torch.full_like(x, 9.0), torch.full_like(x, 9.0)
    gg.fill_(1.0), gb.fill_(2.0)
    a3po.a3po_dropout_norm_bwd(x, P, rng, gamma, stats[0], gy, gres, gbr, gg, ws, kind=kind, mean=stats[1] if layer else None,
                               grad_r=gr, grad_beta=gb, accumulate_grad_w=True, row_mask=mask)
    assert torch.equal(gg.double(), want_gamma + 1) and torch.equal(gb.double(), want_beta + 2)
    grs = wide(gr, mask)
    ref, size = ref + grs, size + grs.abs()
    close(gres, ref, 64 * U * size + half_step(dt) * ref.abs(), "grad_residual")
    factor = dropout_factors(n, h, P, SEED, OFFSET, DEV)
    # d(grad_residual before rounding): its error scaled, one more rounding of the product, and the store's
    ref = ref * factor
    close(gbr, ref, 64 * U * size * factor + 2 * U * ref.abs() + half_step(dt) * ref.abs() * (1 + 64 * U), "grad_x")


def test_rows_past_the_32_bit_element_count():
    """More than 2^31 elements, every row different: rows at the ends, around the 2^31st element and scattered."""
    h = 4096
    n = (1 << 31) // h + 4001
    gen = torch.Generator(device=DEV).manual_seed(3)
    x = torch.empty(n, h, dtype=torch.bfloat16, device=DEV)
    for lo in range(0, n, 65536):
        x[lo:lo + 65536] = torch.randn(min(65536, n - lo), h, generator=gen, device=DEV)
    gamma = torch.ones(h, dtype=torch.bfloat16, device=DEV)
    y, rstd, mean = torch.empty_like(x), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    a3po.a3po_norm_fwd(x, gamma, y, rstd, kind=a3po.A3PO_NORM_LAYER, mean=mean)
    mid = (1 << 31) // h
    rows = torch.tensor([0, 1, 2, mid - 1, mid, mid + 1, n - 3, n - 2, n - 1], device=DEV)
    rows = torch.cat([rows, torch.randint(0, n, (500,), generator=gen, device=DEV)])
    eps = float(torch.tensor(1e-6))
    check_forward(x[rows], None, gamma, None, True, y[rows], mean[rows], rstd[rows], "bf16", eps)
    gx, gg, gb = y, torch.empty(h, device=DEV), torch.empty(h, device=DEV)
    gy = x.roll(1, 0)                                   # another input of distinct rows
    ws = a3po.new_workspace(a3po.a3po_norm_bwd_workspace_bytes(n, h))
    a3po.a3po_norm_bwd(x, gamma, rstd, gy, gx, gg, ws, kind=a3po.A3PO_NORM_LAYER, mean=mean, grad_beta=gb)
    xs, g, rs = x[rows].double(), gy[rows].double(), rstd[rows].double().unsqueeze(1)
    xhat = (xs - mean[rows].double().unsqueeze(1)) * rs
    m0, m1 = g.mean(dim=1, keepdim=True), (g * xhat).mean(dim=1, keepdim=True)
    ref = (g - m0 - xhat * m1) * rs
    size = rs * (g.abs() + g.abs().mean(dim=1, keepdim=True) + xhat.abs() * (g * xhat).abs().mean(dim=1, keepdim=True))
    close(gx[rows], ref, 64 * U * size + 2.0 ** -8 * ref.abs(), "grad_x")

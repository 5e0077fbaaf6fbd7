"""Norm, dropout and their join against the fp64 definitions (oracle/operators_oracle.py).

Tolerances.  u = 2^-24 is half a step of fp32, e = eps(type) / 2 half a step of the stored type, relative to the value.
  forward   y = (x - mean) rstd gamma + beta: the row sums are trees of at most ~40 additions (16 or 32 per thread, 5
            shuffles, at most 32 warps), so mean is off by <= 40 u mean|x| and rstd by <= 24 u relative; with the four
            roundings of the expression |dy| <= 64 u (|y - beta| + |beta| + |gamma| rstd mean|x|) + e |y|
  backward  the same count for the two row sums: |dgx| <= 64 u rstd (|gx| + mean|gx| + |xhat| mean|gx xhat|) + e |gx|
  dgamma    a part adds ceil(N / parts) rows one after the other, then parts / 8 + 8 terms: at most N / 8 + N / parts + 16
            <= N + 16 roundings of partial sums, each at most u sum|gy xhat|
  dropout   x scale: scale is one fp32 rounding of the exact quotient, the product another, the add a third:
            |dy| <= 3 u (|x scale| + |residual|) + e |y|; which elements are dropped is exact
  join      r is a stored value that may land on the neighbour of a tie: compared by itself, and y with the norm of the r
            that was stored
Subnormal results may be flushed or rounded coarsely: 1e-37 is added to every bound."""
import numpy as np
import pytest
import torch

import paper_2512_06547_b200 as a3po
from oracle import operators_oracle as orc
from tests.helpers import to_np64
from tests.test_gpu_guard_bands import Guarded

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
TD = {"f32": torch.float32, "bf16": torch.bfloat16}
SEED, OFFSET = 0x9ABCDEF012345678 - (1 << 64), (7 << 32) + 11


def half_step(dt):
    return torch.finfo(TD[dt]).eps / 2


def rng_words(seed=SEED, offset=OFFSET):
    return torch.tensor([seed, offset], dtype=torch.int64, device=DEV)


class Case:
    def __init__(self, n, h, dt, seed, masked=0.0, scale=1.0, shift=0.0):
        gen = np.random.default_rng(seed)
        td = TD[dt]
        new = lambda *s, k=1.0, b=0.0: torch.from_numpy((gen.standard_normal(s) * k + b).astype(np.float32)).to(td).to(DEV)
        self.n, self.h, self.dt, self.td = n, h, dt, td
        self.x, self.res, self.gy, self.gr = new(n, h, k=scale, b=shift), new(n, h, k=2.0), new(n, h), new(n, h)
        self.gamma, self.beta = new(h, k=0.2, b=1.0), new(h, k=0.3)
        self.mask = None
        if masked:
            m = (gen.random(n) >= masked).astype(np.uint8)
            self.mask = torch.from_numpy(m).to(DEV)
            for t in (self.x, self.res, self.gy, self.gr):
                t[self.mask == 0] = float("nan")
        self.mask_np = None if self.mask is None else to_np64(self.mask)


def close(got, ref, bound, what):
    got = to_np64(got)
    assert got.shape == ref.shape
    bad = ~(np.abs(got - ref) <= bound + 1e-37)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:3].tolist(), got[bad][:3], ref[bad][:3], bound[bad][:3])


def sel(c, a):
    a = to_np64(a)
    return a if c.mask_np is None else np.where((c.mask_np != 0)[:, None], a, 0.0)


def check_norm_fwd(c, x, y, mean, rstd, beta, layer, eps):
    y_ref, mean_ref, rstd_ref = orc.norm_fwd(to_np64(x), to_np64(c.gamma), None if beta is None else to_np64(beta), layer,
                                             eps, c.mask_np)
    xs = sel(c, x)
    mabs = np.abs(xs).mean(axis=1, keepdims=True)
    b = 0.0 if beta is None else np.abs(to_np64(beta))
    g = np.abs(to_np64(c.gamma))
    spread = rstd_ref[:, None] * g
    bound = 64 * U * (np.abs(xs - mean_ref[:, None]) * spread + b + spread * mabs) + half_step(c.dt) * np.abs(y_ref)
    close(y, y_ref, bound, "y")
    if layer:
        close(mean, mean_ref, 40 * U * mabs[:, 0], "mean")
        # the centred row inherits the error of the mean: (x - mean)^2 moves by 2 |x - mean| dmean, which sums to
        # 2 dmean sum|x - mean| <= 2 dmean H std, so rstd moves by rstd^2 std dmean <= rstd dmean rstd
        close(rstd, rstd_ref, rstd_ref * (24 * U + 40 * U * mabs[:, 0] * rstd_ref), "rstd")
    else:
        close(rstd, rstd_ref, 24 * U * rstd_ref, "rstd")


def check_norm_bwd(c, x, mean, rstd, gy, gr, layer, gx, gg, gb, gamma_before=None):
    mn = None if mean is None else to_np64(mean)
    gx_ref, gg_ref, gb_ref = orc.norm_bwd(to_np64(x), to_np64(c.gamma), mn, to_np64(rstd), to_np64(gy), layer, c.mask_np)
    rs = to_np64(rstd)[:, None]
    xhat = (sel(c, x) - (mn[:, None] if layer else 0.0)) * rs
    g = sel(c, gy) * to_np64(c.gamma)
    size = rs * (np.abs(g) + (np.abs(g).mean(axis=1, keepdims=True) if layer else 0.0)
                 + np.abs(xhat) * np.abs(g * xhat).mean(axis=1, keepdims=True))
    if gr is not None:
        gx_ref = gx_ref + sel(c, gr)
        size = size + np.abs(sel(c, gr))
    close(gx, gx_ref, 64 * U * size + half_step(c.dt) * np.abs(gx_ref), "grad of the normalised rows")
    add = 0.0 if gamma_before is None else to_np64(gamma_before)
    k = (c.n + 16) * U
    close(gg, gg_ref + add, k * np.abs(sel(c, gy) * xhat).sum(axis=0) + U * np.abs(gg_ref + add), "grad_gamma")
    if gb is not None:
        close(gb, gb_ref, k * np.abs(sel(c, gy)).sum(axis=0), "grad_beta")
    return gx_ref


SHAPES = [(1, 1), (1, 8), (3, 5), (9, 64), (17, 96), (130, 256), (33, 1003), (129, 1536), (21, 2048), (64, 4096),
          (700, 40), (5, 8200), (4, 16384), (3, 16392), (2, 20001)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("n,h", SHAPES)
def test_norm(n, h, layer, dt):
    c = Case(n, h, dt, 10 * n + h, masked=0.25 if n > 2 else 0.0, scale=1.5, shift=0.5)
    kind = a3po.A3PO_NORM_LAYER if layer else a3po.A3PO_NORM_RMS
    G = Guarded()
    y = G.new("y", (n, h), c.td, 9.0)
    rstd = G.new("rstd", (n,), torch.float32, 9.0)
    mean = G.new("mean", (n,), torch.float32, 9.0) if layer else None
    beta = c.beta if layer else None
    a3po.a3po_norm_fwd(c.x, c.gamma, y, rstd, kind=kind, beta=beta, mean=mean, eps=1e-5, row_mask=c.mask)
    G.check("norm_fwd")
    check_norm_fwd(c, c.x, y, mean, rstd, beta, layer, float(np.float32(1e-5)))
    y2 = torch.full_like(y, 7.0)
    a3po.a3po_norm_fwd(c.x, c.gamma, y2, kind=kind, beta=beta, eps=1e-5, row_mask=c.mask)     # no statistics wanted
    assert torch.equal(y, y2)
    gx = G.new("grad_x", (n, h), c.td, 9.0)
    gg = G.new("grad_gamma", (h,), torch.float32, 9.0)
    gb = G.new("grad_beta", (h,), torch.float32, 9.0) if layer else None
    ws = G.new("ws", (a3po.a3po_norm_bwd_workspace_bytes(n, h),), torch.uint8)
    a3po.a3po_norm_bwd(c.x, c.gamma, rstd, c.gy, gx, gg, ws, kind=kind, mean=mean, grad_beta=gb, row_mask=c.mask)
    G.check("norm_bwd")
    check_norm_bwd(c, c.x, mean, rstd, c.gy, None, layer, gx, gg, gb)
    before = gg.clone()
    a3po.a3po_norm_bwd(c.x, c.gamma, rstd, c.gy, gx, gg, ws, kind=kind, mean=mean, accumulate_grad_w=True,
                       row_mask=c.mask)
    check_norm_bwd(c, c.x, mean, rstd, c.gy, None, layer, gx, gg, None, gamma_before=before)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,h", [(1, 1), (3, 13), (40, 64), (33, 1003), (65, 512), (2, 4096)])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.9999999, 1.0, 2.0 ** -17 * 1.5])
def test_dropout(n, h, p, dt):
    c = Case(n, h, dt, 3 * n + h, masked=0.2 if n > 2 else 0.0)
    keep = orc.dropout_factors(n, h, p, SEED, OFFSET)
    rng = rng_words()
    for res in (None, c.res):
        G = Guarded()
        y = G.new("y", (n, h), c.td, 9.0)
        a3po.a3po_dropout_fwd(c.x, p, rng if p else None, y, residual=res, row_mask=c.mask)
        G.check("dropout_fwd")
        ref = orc.dropout(to_np64(c.x), keep, None if res is None else to_np64(res), c.mask_np)
        size = np.abs(sel(c, c.x) * keep) + (0.0 if res is None else np.abs(sel(c, res)))
        close(y, ref, 3 * U * size + half_step(dt) * np.abs(ref), "y")
        if res is None:
            assert np.array_equal(to_np64(y) == 0, (ref == 0))         # exactly the elements that were dropped
    gx = torch.full_like(c.x, 9.0)
    a3po.a3po_dropout_bwd(c.gy, p, rng if p else None, gx, row_mask=c.mask)
    ref = orc.dropout(to_np64(c.gy), keep, None, c.mask_np)
    close(gx, ref, 3 * U * np.abs(ref) + half_step(dt) * np.abs(ref), "grad_x")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("p", [0.0, 0.3])
@pytest.mark.parametrize("n,h", [(1, 8), (9, 64), (33, 1003), (17, 1536), (6, 4096), (3, 16400)])
def test_join(n, h, p, layer, dt):
    c = Case(n, h, dt, 7 * n + h, masked=0.25 if n > 2 else 0.0)
    kind = a3po.A3PO_NORM_LAYER if layer else a3po.A3PO_NORM_RMS
    rng = rng_words() if p else None
    keep = orc.dropout_factors(n, h, p, SEED, OFFSET)
    G = Guarded()
    r, y = G.new("r", (n, h), c.td, 9.0), G.new("y", (n, h), c.td, 9.0)
    rstd = G.new("rstd", (n,), torch.float32, 9.0)
    mean = G.new("mean", (n,), torch.float32, 9.0) if layer else None
    beta = c.beta if layer else None
    a3po.a3po_dropout_norm_fwd(c.x, c.res, p, rng, c.gamma, r, y, rstd, kind=kind, beta=beta, mean=mean, eps=1e-6,
                               row_mask=c.mask)
    G.check("dropout_norm_fwd")
    r_ref = orc.dropout(to_np64(c.x), keep, to_np64(c.res), c.mask_np)
    size = np.abs(sel(c, c.x) * keep) + np.abs(sel(c, c.res))
    close(r, r_ref, 3 * U * size + half_step(dt) * np.abs(r_ref) * (1 + 4 * U), "r")
    check_norm_fwd(c, r, y, mean, rstd, beta, layer, float(np.float32(1e-6)))
    # the join is the two operators one after the other, bit for bit
    r2, y2, rstd2 = torch.empty_like(r), torch.empty_like(y), torch.empty_like(rstd)
    a3po.a3po_dropout_fwd(c.x, p, rng, r2, residual=c.res, row_mask=c.mask)
    assert torch.equal(r, r2)
    for gr in (None, c.gr):
        gres, gx = G.new("grad_residual", (n, h), c.td, 9.0), G.new("grad_x", (n, h), c.td, 9.0)
        gg = G.new("grad_gamma", (h,), torch.float32, 9.0)
        gb = G.new("grad_beta", (h,), torch.float32, 9.0) if layer else None
        ws = G.new("ws", (a3po.a3po_norm_bwd_workspace_bytes(n, h),), torch.uint8)
        a3po.a3po_dropout_norm_bwd(r, p, rng, c.gamma, rstd, c.gy, gres, gx, gg, ws, kind=kind, mean=mean, grad_r=gr,
                                   grad_beta=gb, row_mask=c.mask)
        G.check("dropout_norm_bwd")
        gres_ref = check_norm_bwd(c, r, mean, rstd, c.gy, gr, layer, gres, gg, gb)
        gres2, gg2 = torch.empty_like(gres), torch.empty_like(gg)      # without the branch's gradient: the rest as before
        a3po.a3po_dropout_norm_bwd(r, 0.0, None, c.gamma, rstd, c.gy, gres2, None, gg2, ws, kind=kind, mean=mean,
                                   grad_r=gr, row_mask=c.mask)
        assert torch.equal(gres, gres2) and torch.equal(gg, gg2)
        # grad_x = d(grad_residual before rounding): within the same bound, scaled
        ratio = to_np64(gx)
        ref = gres_ref * keep
        size = np.abs(gres_ref) + np.abs(to_np64(gres) - gres_ref) + 1e-30
        assert np.all(np.abs(ratio - ref) <= keep * (np.abs(to_np64(gres) - gres_ref) + 2 * half_step(dt) * np.abs(gres_ref)
                                                     + 70 * U * size.max(axis=1, keepdims=True) * 8) + 1e-37)
        assert np.all(ratio[keep == 0] == 0)


def test_gradient_by_differences():
    """The norm's kernel gradient against central differences of the kernel's own forward (fp32)."""
    n, h = 3, 24
    c = Case(n, h, "f32", 5, scale=1.0)
    for layer in (False, True):
        kind = a3po.A3PO_NORM_LAYER if layer else a3po.A3PO_NORM_RMS
        y, rstd = torch.empty_like(c.x), torch.empty(n, device=DEV)
        mean = torch.empty(n, device=DEV) if layer else None
        def value(x):
            a3po.a3po_norm_fwd(x, c.gamma, y, rstd, kind=kind, beta=c.beta, mean=mean)
            return float((y.double() * c.gy.double()).sum())
        value(c.x)
        gx, gg, ws = torch.empty_like(c.x), torch.empty(h, device=DEV), a3po.new_workspace(a3po.a3po_norm_bwd_workspace_bytes(n, h))
        a3po.a3po_norm_bwd(c.x, c.gamma, rstd, c.gy, gx, gg, ws, kind=kind, mean=mean)
        step = 2.0 ** -7                        # x +- step is exact to 2^-24 relative
        for i in range(0, n * h, 5):
            a, b = c.x.clone(), c.x.clone()
            a.view(-1)[i] += step
            b.view(-1)[i] -= step
            d = (value(a) - value(b)) / float(a.view(-1)[i] - b.view(-1)[i])
            # truncation step^2 / 6 times a third derivative of order |gy| |gamma| rstd^3 (~ 10), rounding of the sums of
            # 24 terms of order 1: 64 u * 24 / step
            assert abs(d - float(gx.view(-1)[i])) <= 10 * step ** 2 * 10 + 64 * U * 24 / step


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_unaligned_rows(dt):
    """Buffers that start one element past a 16-byte boundary take the element-wise path: its threads own other columns,
    so row sums add up in another order (the same bound against the definition holds); dropout is the same bit for bit."""
    n, h = 19, 264
    c = Case(n, h, dt, 77, masked=0.2)
    def shifted(t):
        raw = torch.empty(t.numel() + 1, dtype=t.dtype, device=DEV)
        raw[1:].copy_(t.reshape(-1))
        return raw[1:].view(t.shape)
    y, rstd, mean = torch.empty_like(c.x), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    a3po.a3po_norm_fwd(c.x, c.gamma, y, rstd, kind=a3po.A3PO_NORM_LAYER, beta=c.beta, mean=mean, row_mask=c.mask)
    y2, rstd2, mean2 = shifted(torch.zeros_like(c.x)), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    a3po.a3po_norm_fwd(shifted(c.x), shifted(c.gamma), y2, rstd2, kind=a3po.A3PO_NORM_LAYER, beta=shifted(c.beta),
                       mean=mean2, row_mask=c.mask)
    check_norm_fwd(c, c.x, y, mean, rstd, c.beta, True, float(np.float32(1e-6)))
    check_norm_fwd(c, c.x, y2, mean2, rstd2, c.beta, True, float(np.float32(1e-6)))
    d1, d2 = torch.empty_like(c.x), shifted(torch.zeros_like(c.x))
    a3po.a3po_dropout_fwd(c.x, 0.25, rng_words(), d1, residual=c.res, row_mask=c.mask)
    a3po.a3po_dropout_fwd(shifted(c.x), 0.25, rng_words(), d2, residual=shifted(c.res), row_mask=c.mask)
    assert torch.equal(d1, d2)


def test_empty_and_fully_masked():
    h = 48
    gamma = torch.ones(h, device=DEV)
    e = torch.empty(0, h, device=DEV)
    z = torch.empty(0, device=DEV)
    gg = torch.full((h,), 5.0, device=DEV)
    ws = a3po.new_workspace(a3po.a3po_norm_bwd_workspace_bytes(0, h))
    a3po.a3po_norm_fwd(e, gamma, e, z)
    a3po.a3po_dropout_fwd(e, 0.5, rng_words(), e)
    a3po.a3po_norm_bwd(e, gamma, z, e, e, gg, ws, accumulate_grad_w=True)
    assert bool((gg == 5.0).all())
    a3po.a3po_norm_bwd(e, gamma, z, e, e, gg, ws)
    assert bool((gg == 0.0).all())
    n = 37
    x = torch.full((n, h), float("nan"), device=DEV)
    mask = torch.zeros(n, dtype=torch.uint8, device=DEV)
    y, rstd, gx = torch.full_like(x, 3.0), torch.full((n,), 3.0, device=DEV), torch.full_like(x, 3.0)
    ws = a3po.new_workspace(a3po.a3po_norm_bwd_workspace_bytes(n, h))
    a3po.a3po_norm_fwd(x, gamma, y, rstd, row_mask=mask)
    a3po.a3po_norm_bwd(x, gamma, rstd, x, gx, gg, ws, row_mask=mask)
    for t in (y, rstd, gx, gg):
        assert bool((t == 0).all())
    a3po.a3po_dropout_fwd(x, 0.5, rng_words(), y, residual=x, row_mask=mask)
    assert bool((y == 0).all())


def test_special_values_stay_in_their_row_and_column():
    """An infinity or NaN in a valid row spoils that row (and its columns' weight gradients), nothing else; a dropped
    infinity is 0."""
    n, h = 6, 64
    c = Case(n, h, "bf16", 3)
    x = c.x.clone()
    x[2, 5], x[4, 7] = float("inf"), float("nan")
    y, y0 = torch.empty_like(x), torch.empty_like(x)
    a3po.a3po_norm_fwd(x, c.gamma, y)
    a3po.a3po_norm_fwd(c.x, c.gamma, y0)
    ok = [0, 1, 3, 5]
    assert torch.equal(y[ok], y0[ok]) and torch.isnan(y[4]).all() and torch.isnan(y[2, 5])
    d = torch.empty_like(x)
    a3po.a3po_dropout_fwd(torch.full_like(x, float("inf")), 0.5, rng_words(), d)
    keep = torch.from_numpy(orc.dropout_factors(n, h, 0.5, SEED, OFFSET) != 0).to(DEV)
    assert torch.isinf(d[keep]).all() and bool((d[~keep] == 0).all())


def test_streams_graph_and_repeatability():
    """The same call twice is bit-identical; on another stream too; captured, a replay follows changed inputs and a
    changed {seed, offset}."""
    n, h, p = 513, 1536, 0.2
    c = Case(n, h, "bf16", 12, masked=0.3)
    rng = rng_words()
    ws = a3po.new_workspace(a3po.a3po_norm_bwd_workspace_bytes(n, h))
    def buffers():
        return dict(r=torch.empty_like(c.x), y=torch.empty_like(c.x), rstd=torch.empty(n, device=DEV),
                    gres=torch.empty_like(c.x), gx=torch.empty_like(c.x), gg=torch.empty(h, device=DEV))
    def run(b):
        a3po.a3po_dropout_norm_fwd(c.x, c.res, p, rng, c.gamma, b["r"], b["y"], b["rstd"], row_mask=c.mask)
        a3po.a3po_dropout_norm_bwd(b["r"], p, rng, c.gamma, b["rstd"], c.gy, b["gres"], b["gx"], b["gg"], ws,
                                   row_mask=c.mask, grad_r=c.gr)
    same = lambda a, b: all(torch.equal(a[k], b[k]) for k in a)
    one, two = buffers(), buffers()
    run(one); run(two)
    assert same(one, two)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    three = buffers()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(three)
    torch.cuda.current_stream().wait_stream(side)
    assert same(one, three)
    g = torch.cuda.CUDAGraph()
    four = buffers()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        run(four)
    g.replay()
    torch.cuda.synchronize()
    assert same(one, four)
    rng[1] += 1
    c.x.mul_(2)
    run(one)
    g.replay()
    torch.cuda.synchronize()
    assert same(one, four)
    assert not torch.equal(one["gx"], three["gx"])


def test_many_rows():
    """More chunks than 32-bit indexes of elements can address: the last rows are right (2^31 + elements, bf16)."""
    h = 4096
    n = (1 << 31) // h + 5
    x = torch.ones(n, h, dtype=torch.bfloat16, device=DEV)
    x[-1] = 3.0
    y = torch.empty_like(x)
    a3po.a3po_dropout_fwd(x, 0.25, rng_words(), y)
    for row in (n - 1, n - 2, 7):
        seen = np.array([orc.philox4x32_10((g, row, OFFSET & 0xFFFFFFFF, OFFSET >> 32),
                                           ((SEED % (1 << 64)) & 0xFFFFFFFF, (SEED % (1 << 64)) >> 32)) for g in range(4)])
        u = np.stack([seen & 0xFFFF, seen >> 16], axis=2).reshape(-1)
        want = np.where(u >= 16384, 3.0 if row == n - 1 else 1.0, 0.0) * (65536 / (65536 - 16384))
        assert np.allclose(to_np64(y[row, :32]), want, rtol=2.0 ** -8)
    gamma = torch.ones(h, dtype=torch.bfloat16, device=DEV)
    a3po.a3po_norm_fwd(x, gamma, y, eps=0.0)
    assert bool((y[-2:] == 1.0).all()) and bool((y[:2] == 1.0).all())


def test_ties_round_as_with_the_exact_scale():
    """p = 1/4: the scale 4/3 is not an fp32 number, but x = 3 k and x * 4/3 + residual are exact, and half of these sums are
    ties in bf16: they go to the even neighbour."""
    n, h = 64, 512
    gen = np.random.default_rng(2)
    x = torch.from_numpy((3 * gen.integers(-40, 41, (n, h))).astype(np.float32)).bfloat16().to(DEV)
    res = torch.from_numpy((gen.integers(-128, 128, (n, h)) * 4 + 1025).astype(np.float32)).bfloat16().to(DEV)
    keep = torch.from_numpy(orc.dropout_factors(n, h, 0.25, SEED, OFFSET) != 0).to(DEV)
    want = torch.where(keep, x.double() * 4 / 3, torch.zeros((), device=DEV, dtype=torch.double)) + res.double()
    want = want.float().bfloat16()                       # exact sums of integers: one rounding, ties to even
    r, y = torch.empty_like(x), torch.empty_like(x)
    a3po.a3po_dropout_fwd(x, 0.25, rng_words(), y, residual=res)
    a3po.a3po_dropout_norm_fwd(x, res, 0.25, rng_words(), torch.ones(h, dtype=torch.bfloat16, device=DEV), r, torch.empty_like(x))
    assert torch.equal(y, want) and torch.equal(r, want)

"""The gated feed-forward block against its fp64 definition (oracle/operators_oracle.py).

Elementwise bounds, propagated from the formulas.  e: half a step of the storage type (bf16 2^-8, fp32 2^-24); c: error of
an accumulation of K fp32 products relative to sum |a b|, K 2^-24 for the FP32 pipes, and for the matrix instructions,
which may truncate where they align addends, K 2^-22.  With |act'| <= 1.13, |act''| <= 1 for both activations:
  Eg = c |x| |Wg|^T, Eu likewise;  Ea = 1.13 Eg + 2^-19 |a| (the approximate exponential and reciprocal)
  forward   Eh = Ea |u| + |a| Eu + e |h|;   Ey = (Eh + c |h|) |Wd|^T + e |y|
  backward  works on kept g, u, k = 2^-15 (24 of their bits, cut; fp32: e): Eg += k |g|, Eu += k |u|;  Es = Eg + 2^-19;
            Edh = c |dy| |Wd|
            Edg = Edh |u s| + |dh| (Eu |s| + |u| Es) + e |dg|,   Edu = Edh |a| + |dh| Ea + e |du|
            products of these with exact matrices add up as absolute values, plus c of the last sum and e of the store
Products of two errors are covered by a factor 1.05 (every relative error here is below 2 %).
Besides that the 2-norm: independent roundings of at most e have an rms of at most e / sqrt(3) each; y has two of them
(h, y), a gradient two (dg or du or h, the store) and, of kept g and u and the approximate functions, less than one more."""
import math

import numpy as np
import pytest
import torch

import paper_2512_06547_b200 as a3po
from oracle import operators_oracle as orc
from tests.helpers import rel_fro, to_np64
from tests.test_gpu_guard_bands import Guarded

pytestmark = pytest.mark.gpu
DEV = "cuda"
TD = {"f32": torch.float32, "bf16": torch.bfloat16}
ACT = {"silu": a3po.A3PO_ACT_SILU, "gelu_tanh": a3po.A3PO_ACT_GELU_TANH}


class Case:
    def __init__(self, n, h, f, dt, seed, masked=0.0, gate_scale=1.0):
        gen = np.random.default_rng(seed)
        new = lambda *s, k=1.0: torch.from_numpy((gen.standard_normal(s) * k).astype(np.float32)).to(TD[dt]).to(DEV)
        self.n, self.h, self.f, self.dt = n, h, f, dt
        self.x, self.gy = new(n, h), new(n, h)
        self.wgu, self.wd = new(2 * f, h, k=gate_scale * h ** -0.5), new(h, f, k=f ** -0.5)
        self.mask = None
        if masked:
            m = (gen.random(n) >= masked).astype(np.uint8)
            self.mask = torch.from_numpy(m).to(DEV)
            self.x[self.mask == 0] = float("nan")
            self.gy[self.mask == 0] = float("inf")
        self.code = a3po.A3PO_F32 if dt == "f32" else a3po.A3PO_BF16
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def ws(self, bwd, new=a3po.new_workspace):
        return new(a3po.a3po_gated_ffn_workspace_bytes(self.n, self.h, self.f, self.code, self.mask is not None, bwd))

    def kept(self, new=a3po.new_workspace):
        return new(a3po.a3po_gated_ffn_kept_bytes(self.n, self.f, self.code))

    def expect(self, act):
        """Values and elementwise bounds of y, grad_x, grad_w_gate_up, grad_w_down."""
        f = self.f
        m = None if self.mask is None else to_np64(self.mask)
        x, gy = orc._select(m, to_np64(self.x)), orc._select(m, to_np64(self.gy))
        wgu, wd = to_np64(self.wgu), to_np64(self.wd)
        y = orc.gated_ffn_fwd(x, wgu, wd, act)
        gx, ggu, gd = orc.gated_ffn_bwd(x, wgu, wd, gy, act)
        e = torch.finfo(TD[self.dt]).eps / 2
        unit = 2.0 ** -24 if self.dt == "f32" else 2.0 ** -22
        ab = np.abs
        g, u = x @ wgu[:f].T, x @ wgu[f:].T
        a, s = orc.activation(act, g)
        hid, dh = a * u, gy @ wd
        eg, eu = self.h * unit * (ab(x) @ ab(wgu[:f]).T), self.h * unit * (ab(x) @ ab(wgu[f:]).T)
        ea = 1.13 * eg + 2.0 ** -19 * ab(a)
        eh = ea * ab(u) + ab(a) * eu + e * ab(hid)
        ey = (eh + f * unit * ab(hid)) @ ab(wd).T + e * ab(y)
        k = min(e, 2.0 ** -15)
        eg, eu = eg + k * ab(g), eu + k * ab(u)
        ea, es = 1.13 * eg + 2.0 ** -19 * ab(a), eg + 2.0 ** -19
        edh = self.h * unit * (ab(gy) @ ab(wd))
        dg, du = dh * u * s, dh * a
        edg = edh * ab(u * s) + ab(dh) * (eu * ab(s) + ab(u) * es) + e * ab(dg)
        edu = edh * ab(a) + ab(dh) * ea + e * ab(du)
        eh = ea * ab(u) + ab(a) * eu + e * ab(hid)
        d, ed = np.concatenate([dg, du], axis=1), np.concatenate([edg, edu], axis=1)
        egx = (ed + 2 * f * unit * ab(d)) @ ab(wgu) + e * ab(gx)
        eggu = (ed + self.n * unit * ab(d)).T @ ab(x)
        egd = ab(gy).T @ (eh + self.n * unit * ab(hid))
        return {"y": (y, ey), "grad_x": (gx, egx), "grad_w_gate_up": (ggu, eggu), "grad_w_down": (gd, egd)}, e


def check(name, got, value, bound, e, roundings, store=0.0):
    got = to_np64(got)
    bad = ~(np.abs(got - value) <= 1.05 * (bound + store * np.abs(value)) + 1e-36)
    assert not bad.any(), (name, int(bad.sum()), np.argwhere(bad)[:3].tolist(), got[bad][:3], value[bad][:3])
    if value.size >= 256 and np.any(value):
        # fp32: the sums' own rounding shows beside the roundings of storage (random signs: sqrt of the length)
        limit = math.sqrt(roundings) * e / math.sqrt(3) if e > 1e-6 else 2e-6
        assert rel_fro(got, value) <= limit, (name, rel_fro(got, value), limit)


SHAPES = [  # few rows, then tile tails in every dimension, K split over few output tiles, many tiles
    (1, 8, 8, "bf16"), (1, 1536, 264, "bf16"), (5, 64, 24, "bf16"), (9, 72, 40, "bf16"), (16, 520, 136, "bf16"),
    (17, 256, 136, "bf16"), (32, 1536, 264, "bf16"),
    (5, 2056, 2056, "bf16"), (16, 2048, 2072, "bf16"), (27, 2064, 2200, "bf16"),   # pairs of blocks, odd last pair
    (20, 4104, 5000, "bf16"),                        # few rows but large weights: on tiles (h f > 20 million)
    (33, 64, 40, "bf16"), (40, 256, 2056, "bf16"), (129, 256, 776, "bf16"), (257, 72, 1000, "bf16"),
    (300, 1536, 520, "bf16"), (700, 512, 1304, "bf16"), (1000, 264, 2056, "bf16"), (2500, 512, 1024, "bf16"),
    (1, 1, 1, "bf16"), (37, 12, 50, "bf16"), (70, 33, 65, "bf16"), (130, 64, 100, "bf16"),
    (1, 1, 1, "f32"), (7, 8, 8, "f32"), (65, 40, 129, "f32"), (512, 64, 192, "f32")]


@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("masked", [0.0, 0.35])
@pytest.mark.parametrize("n,h,f,dt", SHAPES)
def test_forward_and_backward(n, h, f, dt, masked, act):
    c = Case(n, h, f, dt, n + h + f, masked=masked if n > 2 else 0.0, gate_scale=1.7)
    want, e = c.expect(act)
    G = Guarded()
    new = lambda nbytes: G.new("scratch", (nbytes,), torch.uint8, 0xFF)      # NaN patterns: scratch must not be read first
    y = G.new("y", (n, h), TD[dt], 9.0)
    kept = c.kept(new)
    a3po.a3po_gated_ffn_fwd(c.x, c.wgu, c.wd, y, c.ws(False, new), row_mask=c.mask, kept=kept, activation=ACT[act],
                            status=c.status)
    G.check("gated_ffn_fwd")
    check("y", y, *want["y"], e, 2)
    y2 = torch.full_like(y, 3.0)
    a3po.a3po_gated_ffn_fwd(c.x, c.wgu, c.wd, y2, c.ws(False), row_mask=c.mask, activation=ACT[act], status=c.status)
    assert torch.equal(y, y2)                                                # without keeping: the same result
    for gdt in {torch.float32, TD[dt]}:
        gx = G.new("grad_x", (n, h), TD[dt], 9.0)
        ggu, gd = G.new("grad_w_gate_up", (2 * f, h), gdt, 9.0), G.new("grad_w_down", (h, f), gdt, 9.0)
        a3po.a3po_gated_ffn_bwd(c.x, c.wgu, c.wd, kept, c.gy, gx, ggu, gd, c.ws(True, new), row_mask=c.mask,
                                activation=ACT[act], status=c.status)
        G.check("gated_ffn_bwd")
        store = torch.finfo(gdt).eps / 2
        check("grad_x", gx, *want["grad_x"], e, 3)
        check("grad_w_gate_up", ggu, *want["grad_w_gate_up"], e, 3, store)
        check("grad_w_down", gd, *want["grad_w_down"], e, 3, store)
        if gdt == torch.float32:
            before_gu, before_d = ggu.clone(), gd.clone()
            a3po.a3po_gated_ffn_bwd(c.x, c.wgu, c.wd, kept, c.gy, gx, ggu, gd, c.ws(True), row_mask=c.mask,
                                    activation=ACT[act], accumulate_grad_w=True, status=c.status)
            # adding a value to itself is exact
            assert torch.equal(ggu, 2 * before_gu) and torch.equal(gd, 2 * before_d)
    assert int(c.status.item()) == 0
    if c.mask is not None:
        off = c.mask == 0
        assert bool((y[off] == 0).all()) and bool((gx[off] == 0).all())


@pytest.mark.parametrize("n,h,f,dt", [(20, 64, 64, "bf16"), (150, 64, 64, "bf16"), (20, 33, 50, "f32")])
def test_everything_masked_and_no_rows(n, h, f, dt):
    c = Case(n, h, f, dt, 5, masked=1.0)
    assert int(c.mask.sum()) == 0
    y, gx = torch.full_like(c.x, 3.0), torch.full_like(c.x, 3.0)
    ggu, gd = torch.full((2 * f, h), 3.0, device=DEV), torch.full((h, f), 3.0, device=DEV)
    kept = c.kept()
    def run(accumulate):
        a3po.a3po_gated_ffn_fwd(c.x, c.wgu, c.wd, y, c.ws(False), row_mask=c.mask, kept=kept, status=c.status)
        a3po.a3po_gated_ffn_bwd(c.x, c.wgu, c.wd, kept, c.gy, gx, ggu, gd, c.ws(True), row_mask=c.mask,
                                accumulate_grad_w=accumulate, status=c.status)
    run(True)
    assert bool((y == 0).all()) and bool((gx == 0).all())
    assert bool((ggu == 3).all()) and bool((gd == 3).all())
    run(False)
    assert bool((ggu == 0).all()) and bool((gd == 0).all()) and int(c.status.item()) == 0
    ggu.fill_(3.0); gd.fill_(3.0)
    e = c.x[:0].contiguous()
    ws = a3po.new_workspace(a3po.a3po_gated_ffn_workspace_bytes(0, h, f, c.code, False, True))
    a3po.a3po_gated_ffn_fwd(e, c.wgu, c.wd, e, ws, kept=kept)
    a3po.a3po_gated_ffn_bwd(e, c.wgu, c.wd, kept, e, e, ggu, gd, ws, accumulate_grad_w=True)
    assert bool((ggu == 3).all()) and bool((gd == 3).all())
    a3po.a3po_gated_ffn_bwd(e, c.wgu, c.wd, kept, e, e, ggu, gd, ws)
    assert bool((ggu == 0).all()) and bool((gd == 0).all())


def test_large_gate_values():
    """Gates far outside the activation's knee: no overflow of the exponential, of the cube or of its derivative."""
    n, h, f = 64, 64, 64
    for dt in ("bf16", "f32"):
        c = Case(n, h, f, dt, 8)
        c.wgu[:f] *= 1e4
        for act in ("silu", "gelu_tanh"):
            want, e = c.expect(act)
            y, gx = torch.empty_like(c.x), torch.empty_like(c.x)
            ggu, gd, kept = torch.empty_like(c.wgu), torch.empty_like(c.wd), c.kept()
            a3po.a3po_gated_ffn_fwd(c.x, c.wgu, c.wd, y, c.ws(False), kept=kept, activation=ACT[act])
            a3po.a3po_gated_ffn_bwd(c.x, c.wgu, c.wd, kept, c.gy, gx, ggu, gd, c.ws(True), activation=ACT[act])
            for t in (y, gx, ggu, gd):
                assert torch.isfinite(t.float()).all()
            # (the slope's knee is narrower than the rounding of such gates: values are compared for y only)
            check("y", y, *want["y"], e, 1e9)


def test_gradient_by_differences():
    """grad_x and the weight gradients against central differences of the kernel's own forward (fp32)."""
    n, h, f = 4, 6, 10
    c = Case(n, h, f, "f32", 21)
    kept, y = c.kept(), torch.empty_like(c.x)
    for act in ("silu", "gelu_tanh"):
        def value():
            a3po.a3po_gated_ffn_fwd(c.x, c.wgu, c.wd, y, c.ws(False), kept=kept, activation=ACT[act])
            return float((y.double() * c.gy.double()).sum())
        value()
        gx, ggu, gd = torch.empty_like(c.x), torch.empty_like(c.wgu), torch.empty_like(c.wd)
        a3po.a3po_gated_ffn_bwd(c.x, c.wgu, c.wd, kept, c.gy, gx, ggu, gd, c.ws(True), activation=ACT[act])
        step = 2.0 ** -6
        for t, grad in ((c.x, gx), (c.wgu, ggu), (c.wd, gd)):
            for i in range(0, t.numel(), 7):
                old = float(t.view(-1)[i])
                t.view(-1)[i] = old + step
                hi, up = value(), float(t.view(-1)[i])
                t.view(-1)[i] = old - step
                lo, down = value(), float(t.view(-1)[i])
                t.view(-1)[i] = old
                # truncation: step^2 / 6 times third derivatives of order 10; rounding: 24 terms of order 1, 32 u each
                assert abs((hi - lo) / (up - down) - float(grad.view(-1)[i])) <= 2 * step ** 2 * 10 + 24 * 32 * 2 ** -24 / step


def test_rows_do_not_depend_on_the_batch():
    """The few-rows kernels and the tile kernels agree within the forward's bound on the same rows, and the kept values of
    one serve the backward whatever kernel wrote them (32 rows and 33 rows of one problem)."""
    c = Case(33, 512, 776, "bf16", 31)
    want, e = c.expect("silu")
    y33, y32 = torch.empty_like(c.x), torch.empty_like(c.x[:32])
    a3po.a3po_gated_ffn_fwd(c.x, c.wgu, c.wd, y33, c.ws(False))
    x32 = c.x[:32].contiguous()
    ws = a3po.new_workspace(a3po.a3po_gated_ffn_workspace_bytes(32, 512, 776, c.code, False, False))
    a3po.a3po_gated_ffn_fwd(x32, c.wgu, c.wd, y32, ws)
    check("33 rows", y33, *want["y"], e, 2)
    check("32 rows", y32, want["y"][0][:32], want["y"][1][:32], e, 2)


@pytest.mark.parametrize("n", [13, 600])
def test_streams_graph_and_repeatability(n):
    """Two calls, another stream and a captured replay are bit-identical; the replay follows changed inputs and mask."""
    c = Case(n, 512, 1304, "bf16", 41, masked=0.3)
    ws = a3po.new_workspace(max(c.ws(False).numel(), c.ws(True).numel()))
    kept = c.kept()
    def buffers():
        return [torch.empty_like(c.x), torch.empty_like(c.x), torch.empty(c.wgu.shape, device=DEV),
                torch.empty(c.wd.shape, device=DEV)]
    def run(b):
        a3po.a3po_gated_ffn_fwd(c.x, c.wgu, c.wd, b[0], ws, row_mask=c.mask, kept=kept, status=c.status)
        a3po.a3po_gated_ffn_bwd(c.x, c.wgu, c.wd, kept, c.gy, b[1], b[2], b[3], ws, row_mask=c.mask, status=c.status)
    same = lambda a, b: all(torch.equal(s, t) for s, t in zip(a, b))
    one, two, three, four = (buffers() for _ in range(4))
    run(one); run(two)
    assert same(one, two)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(three)
    torch.cuda.current_stream().wait_stream(side)
    assert same(one, three)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run(four)
    g.replay()
    torch.cuda.synchronize()
    assert same(one, four)
    c.mask.copy_(1 - c.mask)
    c.x.normal_(); c.gy.normal_()
    c.x[c.mask == 0] = float("nan")
    run(one)
    g.replay()
    torch.cuda.synchronize()
    assert same(one, four) and not same(one, three) and int(c.status.item()) == 0


def test_two_streams_at_once():
    a, b = Case(600, 512, 1304, "bf16", 51, masked=0.2), Case(300, 1536, 520, "bf16", 52)
    def run(c):
        out = [torch.empty_like(c.x), torch.empty_like(c.x), torch.empty(c.wgu.shape, device=DEV), torch.empty(c.wd.shape, device=DEV)]
        kept = c.kept()
        a3po.a3po_gated_ffn_fwd(c.x, c.wgu, c.wd, out[0], c.ws(False), row_mask=c.mask, kept=kept, status=c.status)
        a3po.a3po_gated_ffn_bwd(c.x, c.wgu, c.wd, kept, c.gy, *out[1:], c.ws(True), row_mask=c.mask, status=c.status)
        return out
    alone = [run(a), run(b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = []
        for c, s in zip((a, b), streams):
            with torch.cuda.stream(s):
                got.append(run(c))
        torch.cuda.synchronize()
        for x, y in zip(alone, got):
            assert all(torch.equal(s, t) for s, t in zip(x, y))
    assert int(a.status.item()) == 0 and int(b.status.item()) == 0

"""The linear operator against the fp64 definition (oracle/operators_oracle.py).

u = 2^-24 (fp32), h = 2^-8 (bf16; u for fp32 outputs): half a step, relative to the value.  A product of n terms is off by at most
n u sum|terms|, in whatever order fp32 sums are taken.
  z   |dz0| <= (K + 2) u A,  A = |x| |W|^T + |b|
  y   the activation's slope is at most 1.13 and its exponential and reciprocal are good to 2^-20 of it: |dy| <= 1.13 |dz0| +
      2^-20 |act| + u (|y| + |act|) + h |y|
  dz  |act''| <= 1: |ddz| <= |dy| (|dz0| + 2^-19 (1 + |z|)), and the operand of the products rounds by h |dz| more (bf16 with an
      activation)
  dx, dW, db: the sums of those over |W|, |x| and the rows, n u of the sum's terms, and h of the result."""
import numpy as np
import pytest
import torch

import paper_2512_06547_b200 as a3po
from oracle import operators_oracle as orc
from tests.helpers import to_np64

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
TD = {"f32": torch.float32, "bf16": torch.bfloat16}
CODE = {"f32": a3po.A3PO_F32, "bf16": a3po.A3PO_BF16}
ACT = {"none": a3po.A3PO_ACT_NONE, "silu": a3po.A3PO_ACT_SILU, "gelu_tanh": a3po.A3PO_ACT_GELU_TANH}


class Case:
    def __init__(self, n, k, m, dt, act, bias, residual, masked, seed=0, zscale=1.0):
        gen = np.random.default_rng(1000 * seed + n + 7 * k + 13 * m)
        td = TD[dt]
        new = lambda *s, c=1.0: torch.from_numpy((gen.standard_normal(s) * c).astype(np.float32)).to(td).to(DEV)
        self.n, self.k, self.m, self.dt, self.act = n, k, m, dt, act
        self.x, self.w = new(n, k), new(m, k, c=zscale * k ** -0.5)
        self.bias = new(m, c=0.5) if bias else None
        self.res = new(n, m, c=2.0) if residual else None
        self.gy = new(n, m)
        self.mask = None
        if masked:
            keep = (gen.random(n) >= masked).astype(np.uint8)
            self.mask = torch.from_numpy(keep).to(DEV)
            for t in (self.x, self.gy) + ((self.res,) if residual else ()):
                t[self.mask == 0] = float("nan")

    def buffers(self, bwd):
        ws = a3po.new_workspace(a3po.a3po_linear_workspace_bytes(self.n, self.k, self.m, CODE[self.dt], ACT[self.act],
                                                                 self.mask is not None, bwd), DEV)
        ws.fill_(255)      # NaN in every type
        return ws

    def forward(self, y_dt=None, keep=True, stream=None):
        y = torch.full((self.n, self.m), 77.0, dtype=TD[y_dt or self.dt], device=DEV)
        kept = None
        if keep and self.act != "none":
            kept = a3po.new_workspace(a3po.a3po_linear_kept_bytes(self.n, self.m, CODE[self.dt], ACT[self.act]), DEV)
            kept.fill_(255)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        a3po.a3po_linear_fwd(self.x, self.w, y, self.buffers(False), bias=self.bias, residual=self.res, row_mask=self.mask,
                             kept=kept, activation=ACT[self.act], status=status, stream=stream)
        return y, kept, status

    def backward(self, kept, grad_dt=None, want=("x", "w", "b"), start=None, stream=None):
        new = lambda *s, t: torch.full(s, 77.0 if start is None else start, dtype=t, device=DEV)
        gx = new(self.n, self.k, t=TD[self.dt]) if "x" in want else None
        gw = new(self.m, self.k, t=TD[grad_dt or self.dt]) if "w" in want else None
        gb = new(self.m, t=torch.float32) if "b" in want else None
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        a3po.a3po_linear_bwd(self.x, self.w, self.gy, gx, gw, self.buffers(True), kept=kept, grad_bias=gb, row_mask=self.mask,
                             activation=ACT[self.act], accumulate_grad_w=start is not None, status=status, stream=stream)
        return gx, gw, gb, status

    def host(self):
        f = lambda t: None if t is None else to_np64(t)
        return f(self.x), f(self.w), f(self.bias), f(self.res), f(self.gy), f(self.mask)


def within(got, ref, bound, what):
    got = to_np64(got)
    assert got.shape == ref.shape, what
    bad = ~(np.abs(got - ref) <= bound + 1e-37)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:3].tolist(), got[bad][:3], ref[bad][:3], bound[bad][:3])


def check(c, y_dt=None, grad_dt=None, keep=True):
    y, kept, status = c.forward(y_dt, keep)
    gx, gw, gb, status2 = c.backward(kept, grad_dt)
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and int(status2.item()) == 0
    x, w, b, r, gy, mask = c.host()
    ref_y, z = orc.linear_fwd(x, w, b, r, c.act, mask)
    ref_x, ref_w, ref_b, dz = orc.linear_bwd(x, w, z, gy, c.act, mask)
    sel = lambda a: orc._select(mask, a)
    half = lambda t: 2.0 ** -8 if t == torch.bfloat16 else U
    xs, ws = np.abs(sel(x)), np.abs(w)
    dz0 = (c.k + 2) * U * (xs @ ws.T + (0 if b is None else np.abs(b)))
    act = np.abs(sel(orc.linear_activation(c.act, z)[0]))
    more = 0 if c.act == "none" else 2.0 ** -20 * act
    within(y, ref_y, sel(1.13 * dz0 + more + U * (np.abs(ref_y) + act)) + half(y.dtype) * np.abs(ref_y), "y")
    ddz = np.zeros_like(dz)
    if c.act != "none":
        ddz = np.abs(sel(gy)) * (dz0 + 2.0 ** -19 * (1 + np.abs(sel(z))))
    op = ddz + (2.0 ** -8 * np.abs(dz) * 1.01 if c.act != "none" and c.dt == "bf16" else U * np.abs(dz))
    within(gx, ref_x, op @ ws + c.m * U * (np.abs(dz) @ ws) + half(gx.dtype) * (np.abs(ref_x) + op @ ws), "grad_x")
    ow = op.T @ xs
    within(gw, ref_w, ow + c.n * U * (np.abs(dz).T @ xs) + half(gw.dtype) * (np.abs(ref_w) + ow), "grad_w")
    within(gb, ref_b, ddz.sum(axis=0) + (c.n + 2) * U * np.abs(dz).sum(axis=0), "grad_bias")


# one token, few rows of both tile counts, K splits, ragged tiles, several tiles and waves; K below, at and past a k-block
BF16_SIZES = [(1, 8, 8), (1, 2048, 520), (5, 2056, 264), (8, 64, 96), (13, 1000, 40), (16, 4096, 8), (17, 512, 72), (32, 72, 1032),
              (33, 264, 136), (100, 1536, 256), (128, 64, 40), (129, 520, 600), (300, 2048, 256), (515, 136, 1288), (1000, 8, 8),
              (2051, 72, 2056)]


@pytest.mark.parametrize("n,k,m", BF16_SIZES)
@pytest.mark.parametrize("act,bias,residual", [("none", False, False), ("none", True, True), ("silu", True, False),
                                               ("gelu_tanh", True, True)])
@pytest.mark.parametrize("masked", [0.0, 0.4])
def test_bf16(n, k, m, act, bias, residual, masked):
    c = Case(n, k, m, "bf16", act, bias, residual, masked)
    check(c, y_dt="f32" if (n + m) % 3 == 0 else None, grad_dt="f32" if n % 2 else None)


@pytest.mark.parametrize("dt,n,k,m", [("f32", 1, 1, 1), ("f32", 3, 65, 17), ("f32", 70, 33, 129), ("f32", 257, 128, 200),
                                      ("f32", 1030, 64, 72), ("bf16", 3, 65, 17), ("bf16", 70, 33, 136), ("bf16", 300, 64, 67)])
@pytest.mark.parametrize("act,bias,residual,masked", [("none", False, False, 0.0), ("silu", True, True, 0.3),
                                                      ("gelu_tanh", False, True, 0.0), ("none", True, False, 0.5)])
def test_fp32_pipes(dt, n, k, m, act, bias, residual, masked):
    check(Case(n, k, m, dt, act, bias, residual, masked), y_dt="f32" if m % 2 else None, grad_dt="f32" if n % 2 else None)


@pytest.mark.parametrize("dt,n,k,m", [("bf16", 20, 64, 40), ("bf16", 100, 64, 136), ("bf16", 200, 264, 136), ("f32", 50, 31, 20), ("f32", 90, 31, 20)])
@pytest.mark.parametrize("act", ["none", "silu"])
def test_no_row_takes_part(dt, n, k, m, act):
    check(Case(n, k, m, dt, act, True, True, 1.1))


@pytest.mark.parametrize("dt,n,k,m", [("bf16", 20, 64, 40), ("bf16", 128, 64, 136), ("bf16", 129, 64, 136), ("bf16", 200, 264, 136), ("f32", 64, 31, 20), ("f32", 65, 31, 20)])
@pytest.mark.parametrize("masked", [0.0, 0.4])
def test_wanted_gradients_alone_and_accumulated(dt, n, k, m, masked):
    for act in ("none", "gelu_tanh"):
        c = Case(n, k, m, dt, act, True, False, masked)
        _, kept, _ = c.forward()
        full = c.backward(kept, "f32")
        for want in ("x", "w", "b", "xb", "wb", "xw"):
            got = c.backward(kept, "f32", want)
            torch.cuda.synchronize()
            for name, a, b in zip("xwb", got, full):
                assert a is None if name not in want else torch.equal(a, b), (act, want, name)
        more = c.backward(kept, "f32", start=1.0)
        torch.cuda.synchronize()
        assert torch.equal(more[0], full[0])
        for a, b in zip(more[1:3], full[1:3]):
            assert ((a - (b + 1.0)).abs() <= 2 * U * (1.0 + b.abs())).all()


@pytest.mark.parametrize("n,offset", [(1024, 0), (1025, 3), (5000, 0), (5000, 1), (262144, 0), (262144, 5), (262145, 0)])
def test_masks_of_many_rows(n, offset):
    """Rows of several blocks of the row index, whatever the mask's alignment and its nonzero bytes."""
    c = Case(n, 8, 16, "bf16", "silu", True, False, 0.4)
    gen = np.random.default_rng(n + offset)
    values = to_np64(c.mask).astype(np.uint8) * gen.choice(np.array([1, 2, 128, 255], np.uint8), n)
    room = torch.full((n + 16,), 1, dtype=torch.uint8, device=DEV)
    mask = room[offset:offset + n]
    mask.copy_(torch.from_numpy(values))
    c.mask = mask
    check(c)


@pytest.mark.parametrize("n,k,m", [(2048, 136, 72), (4100, 264, 136), (9000, 8, 8)])
@pytest.mark.parametrize("act,masked", [("none", 0.0), ("silu", 0.3), ("none", 0.995), ("silu", 0.995), ("gelu_tanh", 1.1), ("none", 1.1)])
@pytest.mark.parametrize("grad_dt", ["bf16", "f32"])
def test_weight_gradients_in_parts_of_the_rows(n, k, m, act, masked, grad_dt):
    """Few tiles, many rows; of 0.995 and more masked, parts of the split are left without a row."""
    c = Case(n, k, m, "bf16", act, True, False, masked)
    check(c, grad_dt=grad_dt)
    if grad_dt == "f32":
        _, kept, _ = c.forward()
        full, more = c.backward(kept, "f32"), c.backward(kept, "f32", start=1.0)
        torch.cuda.synchronize()
        for a, b in zip(more[1:3], full[1:3]):
            assert ((a - (b + 1.0)).abs() <= 2 * U * (1.0 + b.abs())).all()


def test_large_values_and_infinite_slopes():
    """Activations far out: z up to hundreds either way stays finite."""
    for dt, n, k, m in (("bf16", 40, 64, 64), ("f32", 40, 33, 20)):
        for act in ("silu", "gelu_tanh"):
            check(Case(n, k, m, dt, act, True, False, 0.0, zscale=100.0))


def test_gradients_against_differences():
    """Directional derivative of sum(y gy) by central differences in fp64 of the definition's own forward."""
    c = Case(60, 48, 40, "f32", "gelu_tanh", True, True, 0.3)
    _, kept, _ = c.forward()
    gx, gw, gb, _ = c.backward(kept)
    torch.cuda.synchronize()
    x, w, b, r, gy, mask = c.host()
    gen = np.random.default_rng(1)
    dx, dw, db = gen.standard_normal(x.shape), gen.standard_normal(w.shape), gen.standard_normal(b.shape)
    x = orc._select(mask, x)
    f = lambda e: (orc.linear_fwd(x + e * dx, w + e * dw, b + e * db, r, c.act, mask)[0] * orc._select(mask, gy)).sum()
    e = 1e-4
    slope = (f(e) - f(-e)) / (2 * e)
    mine = (to_np64(gx) * dx).sum() + (to_np64(gw) * dw).sum() + (to_np64(gb) * db).sum()
    scale = np.abs(to_np64(gx) * dx).sum() + np.abs(to_np64(gw) * dw).sum() + np.abs(to_np64(gb) * db).sum()
    assert abs(slope - mine) <= 1e-5 * scale     # fp32 products of at most 60 terms, and e^2 of the third derivative


@pytest.mark.parametrize("n,k,m,masked", [(9, 512, 264, 0.0), (400, 264, 520, 0.4)])
def test_captured_and_on_two_streams(n, k, m, masked):
    a, b = (Case(n, k, m, "bf16", "silu", True, True, masked, seed=s) for s in (1, 2))

    def both_ways(c, stream=None):
        y, kept, _ = c.forward(stream=stream)
        return (y,) + c.backward(kept, "f32", stream=stream)[:3]

    refs = [both_ways(c) for c in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(4):
        got = []
        for s, c in zip(streams, (a, b)):
            with torch.cuda.stream(s):
                got.append(both_ways(c))
        torch.cuda.synchronize()
        for g, ref in zip(got, refs):
            assert all(torch.equal(p, q) for p, q in zip(g, ref))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both_ways(a)
    a.x.copy_(b.x); a.w.copy_(b.w); a.bias.copy_(b.bias); a.res.copy_(b.res); a.gy.copy_(b.gy)
    if masked:
        a.mask.copy_(b.mask)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(out, refs[1]))


@pytest.mark.parametrize("n", [1, 30])
def test_logits_of_a_large_vocabulary(n):
    c = Case(n, 1536, 151936, "bf16", "none", False, False, 0.0)
    y, _, _ = c.forward("f32")
    torch.cuda.synchronize()
    ref = (c.x.double() @ c.w.double().t())
    bound = 1538 * U * (c.x.double().abs() @ c.w.double().abs().t()) + U * ref.abs()
    assert ((y.double() - ref).abs() <= bound).all()

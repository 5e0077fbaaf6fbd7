"""The feed-forward block where every pair of CTAs works through several output tiles of each of its products, over dozens of
k-blocks: accumulators and staging slabs are used again, kept values are prefetched from tile to tile, launches are paced,
and the backward's last three run beside one another.  Values and elementwise bounds are those of tests/test_gpu_gated_ffn.py
(derived there), evaluated in fp64 on the GPU."""
import math

import pytest
import torch

import paper_2512_06547_b200 as a3po

pytestmark = pytest.mark.gpu
DEV = "cuda"
ACT = {"silu": a3po.A3PO_ACT_SILU, "gelu_tanh": a3po.A3PO_ACT_GELU_TANH}
UNIT = 2.0 ** -22      # error of an addition in the matrix instructions
E = 2.0 ** -8          # half a step of bf16


def activation(act, g):
    if act == "silu":
        s = 1 / (1 + torch.exp(-g))
        return g * s, s + g * s * (1 - s)
    th = torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1 + th), 0.5 * (1 + th) + 0.5 * g * (1 - th * th) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * g ** 2)


class Case:
    def __init__(self, n, h, f, masked, seed):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        new = lambda *s, k=1.0: (torch.randn(*s, generator=gen, device=DEV) * k).bfloat16()
        self.n, self.h, self.f = n, h, f
        self.x, self.gy = new(n, h), new(n, h)
        self.wgu, self.wd = new(2 * f, h, k=1.7 * h ** -0.5), new(h, f, k=f ** -0.5)
        self.mask = None
        if masked:
            self.mask = (torch.rand(n, generator=gen, device=DEV) >= masked).to(torch.uint8)
            self.x[self.mask == 0] = float("nan")
            self.gy[self.mask == 0] = float("inf")
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def rows(self, t):
        return t.double() if self.mask is None else t.double().masked_fill_((self.mask == 0).unsqueeze(1), 0.0)

    def run(self, act, grad_dtype=torch.float32, into=None):
        has = self.mask is not None
        size = lambda bwd: a3po.a3po_gated_ffn_workspace_bytes(self.n, self.h, self.f, a3po.A3PO_BF16, has, bwd)
        ws = torch.full((max(size(False), size(True)),), 0xFF, dtype=torch.uint8, device=DEV)   # NaN patterns
        kept = torch.full((a3po.a3po_gated_ffn_kept_bytes(self.n, self.f, a3po.A3PO_BF16),), 0xFF, dtype=torch.uint8, device=DEV)
        if into is None:
            into = [torch.full_like(self.x, 9.0), torch.full_like(self.x, 9.0),
                    torch.full(self.wgu.shape, 9.0, dtype=grad_dtype, device=DEV),
                    torch.full(self.wd.shape, 9.0, dtype=grad_dtype, device=DEV)]
            add = False
        else:
            add = True
        a3po.a3po_gated_ffn_fwd(self.x, self.wgu, self.wd, into[0], ws, row_mask=self.mask, kept=kept, activation=ACT[act],
                                status=self.status)
        a3po.a3po_gated_ffn_bwd(self.x, self.wgu, self.wd, kept, self.gy, *into[1:], ws, row_mask=self.mask,
                                activation=ACT[act], accumulate_grad_w=add, status=self.status)
        return into


def check(name, got, value, bound, roundings, store=0.0):
    got = got.double()
    bad = ~((got - value).abs() <= 1.05 * (bound + store * value.abs()) + 1e-36)
    assert not bool(bad.any()), (name, int(bad.sum()), bad.nonzero()[:3].tolist())
    err, limit = float((got - value).norm() / value.norm()), math.sqrt(roundings) * E / math.sqrt(3)
    assert err <= limit, (name, err, limit)


def compare(c, act, out, store):
    """In the order of tests/test_gpu_gated_ffn.py Case.expect, each intermediate dropped when it has been used."""
    n, h, f = c.n, c.h, c.f
    x, gy, wgu, wd = c.rows(c.x), c.rows(c.gy), c.wgu.double(), c.wd.double()
    y, gx, ggu, gd = out
    g, u = x @ wgu[:f].t(), x @ wgu[f:].t()
    a, s = activation(act, g)
    hid = a * u
    eg, eu = h * UNIT * (x.abs() @ wgu[:f].abs().t()), h * UNIT * (x.abs() @ wgu[f:].abs().t())
    ea = 1.13 * eg + 2.0 ** -19 * a.abs()
    ref = hid @ wd.t()
    check("y", y, ref, (ea * u.abs() + a.abs() * eu + E * hid.abs() + f * UNIT * hid.abs()) @ wd.abs().t() + E * ref.abs(), 2)
    k = 2.0 ** -15
    eg, eu = eg + k * g.abs(), eu + k * u.abs()
    ea, es = 1.13 * eg + 2.0 ** -19 * a.abs(), eg + 2.0 ** -19
    eh = ea * u.abs() + a.abs() * eu + E * hid.abs()
    ref = gy.t() @ hid
    check("grad_w_down", gd, ref, gy.abs().t() @ (eh + n * UNIT * hid.abs()), 3, store)
    del eh, hid
    dh, edh = gy @ wd, h * UNIT * (gy.abs() @ wd.abs())
    d = torch.cat([dh * u * s, dh * a], dim=1)
    ed = torch.cat([edh * (u * s).abs() + dh.abs() * (eu * s.abs() + u.abs() * es), edh * a.abs() + dh.abs() * ea], dim=1) + E * d.abs()
    del g, u, a, s, eg, eu, ea, es, dh, edh
    ref = d @ wgu
    check("grad_x", gx, ref, (ed + 2 * f * UNIT * d.abs()) @ wgu.abs() + E * ref.abs(), 3)
    ref = d.t() @ x
    check("grad_w_gate_up", ggu, ref, (ed + n * UNIT * d.abs()).t() @ x.abs(), 3, store)
    if c.mask is not None:
        assert bool((y[c.mask == 0] == 0).all()) and bool((gx[c.mask == 0] == 0).all())


# 256 x 256 tiles (gate/up: 256 x 128 units) over 74 pairs.  9,000 x 4,104 x 9,224: 36 row, 17 and 37 column tiles, so 612 to
# 2,628 of them, more than 8 to a pair in every product (each launch is paced), K of 64 to 288 k-blocks; masked, the
# rows' K and M come from the device.  4,200 x 2,056 x 6,152: 153 to 833 tiles, some launches paced, others not.
@pytest.mark.parametrize("n,h,f,masked,act,grad_dtype", [
    (9000, 4104, 9224, 0.0, "silu", torch.float32), (9000, 4104, 9224, 0.3, "gelu_tanh", torch.bfloat16),
    (4200, 2056, 6152, 0.0, "gelu_tanh", torch.bfloat16), (4200, 2056, 6152, 0.4, "silu", torch.float32),
    (20000, 520, 1544, 0.35, "silu", torch.float32)])     # K of 9 k-blocks: epilogues one behind the other
def test_values(n, h, f, masked, act, grad_dtype):
    c = Case(n, h, f, masked, n + h)
    out = c.run(act, grad_dtype)
    compare(c, act, out, torch.finfo(grad_dtype).eps / 2)
    if grad_dtype == torch.float32:
        before = [t.clone() for t in out]
        c.run(act, into=out)                              # adding a value to itself is exact
        assert torch.equal(out[2], 2 * before[2]) and torch.equal(out[3], 2 * before[3])
        assert torch.equal(out[0], before[0]) and torch.equal(out[1], before[1])
    assert int(c.status.item()) == 0


def test_runs_streams_and_replays_agree():
    """Several waves of tiles: bit for bit the same again, beside another call on another stream, and captured."""
    a, b = Case(4200, 2056, 6152, 0.4, 1), Case(9000, 1032, 4104, 0.0, 2)
    same = lambda s, t: all(torch.equal(p, q) for p, q in zip(s, t))
    alone = [a.run("silu"), b.run("gelu_tanh")]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(4):
        got = []
        for c, act, s in ((a, "silu", streams[0]), (b, "gelu_tanh", streams[1])):
            with torch.cuda.stream(s):
                got.append(c.run(act))
        torch.cuda.synchronize()
        assert same(alone[0], got[0]) and same(alone[1], got[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        replayed = a.run("silu")
    for _ in range(2):
        for t in replayed:
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert same(alone[0], replayed)
    assert int(a.status.item()) == 0 and int(b.status.item()) == 0


def test_gradients_of_the_same_rows_from_either_family():
    """32 rows go through the few-rows kernels, the same rows as part of 33 through tiles; the backward takes what either of
    them kept, and the rows' results lie within the bounds of the same values."""
    h, f = 512, 776
    c33 = Case(33, h, f, 0.0, 31)
    c32 = Case(32, h, f, 0.0, 31)
    c32.x, c32.gy, c32.wgu, c32.wd = c33.x[:32].contiguous(), c33.gy[:32].contiguous(), c33.wgu, c33.wd
    for c in (c33, c32):
        compare(c, "silu", c.run("silu"), 2.0 ** -24)
    last = c33.gy.clone()
    last[:32] = 0                                          # the weight gradients of 33 rows are those of 32 and of the last
    both, first = c33.run("silu"), c32.run("silu")
    c33.gy = last
    rest = c33.run("silu")
    for i in (2, 3):
        whole, parts = both[i].double(), first[i].double() + rest[i].double()
        assert float((whole - parts).norm() / whole.norm()) <= 2 * E / math.sqrt(3)   # a rounding of dg, du, h on each side

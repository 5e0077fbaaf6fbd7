"""AdamW against the fp64 definition (oracle/operators_oracle.py).

u = 2^-24, half a step of fp32.  m' = b1 m + (1 - b1) s g: both factors are one rounding each of the 64-bit ones, s g another, the product
another, the sum the last: |dm'| <= 4 u (|b1 m| + |(1 - b1) s g|).  v' has two more (s g enters squared): 6 u v'.
w': the quotient of the corrected moments has the moments' errors (half of v's, from the root), the two corrections, their
products, the root, the sum with eps and a quotient of 2 steps: |dq| <= 20 u |q| + |dm'| / ((1 - b1^t) den); lr, decay and w
add 4 u (lr decay |w|) and two roundings of w.  A bf16 weight is one more rounding, 2^-8 of itself... half a step: eps / 2.
8 bits: codes and scales are the definition's bit for bit (they are computed in 64 bits: only values within about 2^-50 of
the middle between two codes could differ)."""
import numpy as np
import pytest
import torch

import paper_2512_06547_b200 as a3po
from oracle import operators_oracle as orc
from paper_2512_06547_b200.optimizer import AdamW, decode_state
from tests.helpers import to_np64

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
TD = {"f32": torch.float32, "bf16": torch.bfloat16}
B1, B2, EPS, LR = 0.9, 0.95, 1e-8, 3e-3


def tensors(sizes, td, seed, scale, offset=0):
    """Separate tensors, or (offset) neighbours in one buffer that start `offset` elements off its alignment."""
    gen = np.random.default_rng(seed)
    parts = [torch.from_numpy((gen.standard_normal(n) * scale).astype(np.float32)).to(td).to(DEV) for n in sizes]
    if not offset:
        return parts
    flat = torch.empty(sum(sizes) + offset, dtype=td, device=DEV)
    out, at = [], offset
    for p in parts:
        flat[at:at + p.numel()] = p
        out.append(flat[at:at + p.numel()])
        at += p.numel()
    return out


class Reference:
    """The definition on the host, state by state as the library stores it."""

    def __init__(self, opt, wdt):
        self.wdt, self.bits = wdt, opt.state_bits
        source = opt.masters if opt.masters is not None else opt.weights
        self.w = [to_np64(x) for x in source]
        self.m, self.v = [to_np64(x).copy() for x in opt.m], [to_np64(x).copy() for x in opt.v]
        if self.bits == 8:
            self.ms, self.vs = [to_np64(x) for x in opt.m_scales], [to_np64(x) for x in opt.v_scales]

    def check(self, opt, grads, t, lr, decay, max_norm):
        grads = [to_np64(g) for g in grads]
        norm, scale = orc.clip_scale(grads, max_norm)
        assert abs(float(opt.grad_norm.item()) - norm) <= U * norm * 1.01
        for i, g in enumerate(grads):
            m0 = orc.state_decode(self.m[i], self.ms[i], True) if self.bits == 8 else self.m[i]
            v0 = orc.state_decode(self.v[i], self.vs[i], False) if self.bits == 8 else self.v[i]
            w, m, v = orc.adamw(self.w[i], g, m0, v0, t, lr, B1, B2, EPS, decay[i], scale)
            dm = 4 * U * (np.abs(B1 * m0) + np.abs((1 - B1) * scale * g))
            if self.bits == 8:
                for got, got_scale, x, signed in ((opt.m[i], opt.m_scales[i], m, True), (opt.v[i], opt.v_scales[i], v, False)):
                    codes, scales = orc.state_encode(x, signed)
                    assert np.array_equal(to_np64(got_scale), scales), (i, signed)
                    assert np.array_equal(got.cpu().numpy(), codes), (i, signed, int((got.cpu().numpy() != codes).sum()))
                    values = torch.empty(x.size, device=DEV)
                    decode_state(got, got_scale, signed=signed, out=values)
                    assert np.array_equal(to_np64(values), orc.state_decode(codes, scales, signed).astype(np.float32)), (i, signed)
            else:
                assert (np.abs(to_np64(opt.m[i]) - m) <= dm + 1e-40).all(), i
                assert (np.abs(to_np64(opt.v[i]) - v) <= 6 * U * v + 1e-40).all(), i
            den = np.sqrt(v / (1 - B2 ** t)) + EPS
            q = m / (1 - B1 ** t) / den
            bound = lr * (20 * U * np.abs(q) + dm / ((1 - B1 ** t) * den) + 4 * U * decay[i] * np.abs(self.w[i])) \
                + 2 * U * np.abs(self.w[i]) + U * np.abs(w) + 1e-40
            if opt.masters is not None:
                assert (np.abs(to_np64(opt.masters[i]) - w) <= bound).all(), i
                assert torch.equal(opt.weights[i], opt.masters[i].to(TD[self.wdt])), i
                self.w[i] = to_np64(opt.masters[i])
            else:
                half = torch.finfo(TD[self.wdt]).eps / 2 if self.wdt == "bf16" else 0.0
                assert (np.abs(to_np64(opt.weights[i]) - w) <= bound + half * (np.abs(w) + bound)).all(), i
                self.w[i] = to_np64(opt.weights[i])
            self.m[i], self.v[i] = to_np64(opt.m[i]).copy(), to_np64(opt.v[i]).copy()
            if self.bits == 8:
                self.ms[i], self.vs[i] = to_np64(opt.m_scales[i]), to_np64(opt.v_scales[i])


SIZES = [1, 5, 255, 256, 257, 2048, 2049, 10007, 0, 3, 70001]


@pytest.mark.parametrize("offset", [0, 1, 3])
@pytest.mark.parametrize("wdt,masters", [("f32", None), ("bf16", True), ("bf16", None)])
@pytest.mark.parametrize("gdt", ["f32", "bf16"])
@pytest.mark.parametrize("bits", [32, 8])
def test_three_steps(bits, gdt, wdt, masters, offset):
    decay = [0.1 if i % 2 else 0.0 for i in range(len(SIZES))]
    w = tensors(SIZES, TD[wdt], 1, 0.5, offset)
    opt = AdamW(w, lr=LR, betas=(B1, B2), eps=EPS, weight_decay=decay, max_grad_norm=1.0, state_bits=bits, masters=masters)
    ref = Reference(opt, wdt)
    lr = float(opt.lr.item())
    for t in (1, 2, 3):
        grads = tensors(SIZES, TD[gdt], 10 + t, 10.0 ** -t, offset)
        before = [g.clone() for g in grads]
        opt.step(grads)
        torch.cuda.synchronize()
        assert int(opt.steps.item()) == t
        ref.check(opt, grads, t, lr, decay, 1.0)
        assert all(torch.equal(a, c) for a, c in zip(grads, before))


@pytest.mark.parametrize("bits", [32, 8])
def test_many_tensors(bits):
    """More tensors than one launch's table holds, without a clip."""
    sizes = [1 + (37 * i) % 700 for i in range(903)]
    opt = AdamW(tensors(sizes, torch.float32, 2, 1.0), lr=LR, betas=(B1, B2), eps=EPS, weight_decay=0.01, state_bits=bits)
    ref = Reference(opt, "f32")
    grads = tensors(sizes, torch.float32, 3, 0.1)
    opt.step(grads)
    torch.cuda.synchronize()
    ref.check(opt, grads, 1, float(opt.lr.item()), [0.01] * len(sizes), 0.0)


@pytest.mark.parametrize("bits", [32, 8])
def test_gradients_of_unlike_size_zeros_and_subnormals(bits):
    n = 256 * 6 + 17
    gen = np.random.default_rng(4)
    g = (gen.standard_normal(n) * 10.0 ** gen.uniform(-18, 2, n)).astype(np.float32)
    g[:256] = 0.0                     # a block of zeros: scales 0
    g[256:512] = 1e-42                # squares that are 0 in fp32
    g[512:768] = np.float32(2.0 ** -3)    # all equal: the largest code everywhere
    w = tensors([n], torch.float32, 5, 1.0)
    opt = AdamW(w, lr=LR, betas=(B1, B2), eps=EPS, weight_decay=0.0, state_bits=bits)
    ref = Reference(opt, "f32")
    if bits == 8:
        for t in (1, 2):
            opt.step([torch.from_numpy(g).to(DEV)])
            torch.cuda.synchronize()
            ref.check(opt, [torch.from_numpy(g)], t, float(opt.lr.item()), [0.0], 0.0)
            assert (opt.v[0][768:] > 0).all()      # no second moment above 0 is stored as 0
    else:
        g[256:512] = 0.0              # fp32 states flush what is below the type
        g[np.abs(g) < 1e-18] = 0.0
        opt.step([torch.from_numpy(g).to(DEV)])
        torch.cuda.synchronize()
        ref.check(opt, [torch.from_numpy(g)], 1, float(opt.lr.item()), [0.0], 0.0)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_that_is_not_finite_changes_nothing(bits, bad):
    sizes = [300, 5000]
    opt = AdamW(tensors(sizes, torch.bfloat16, 6, 1.0), lr=LR, state_bits=bits, masters=True, max_grad_norm=1.0)
    good = tensors(sizes, torch.float32, 7, 0.1)
    opt.step(good)
    held = lambda: [x.clone() for x in opt.weights + opt.masters + opt.m + opt.v + (opt.m_scales or []) + (opt.v_scales or [])]
    before = held()
    worse = [g.clone() for g in good]
    worse[1][4321] = bad
    opt.step(worse)
    torch.cuda.synchronize()
    assert int(opt.steps.item()) == 1 and not np.isfinite(opt.grad_norm.item())
    assert all(torch.equal(a, c) for a, c in zip(before, held()))
    opt.step(good)
    torch.cuda.synchronize()
    assert int(opt.steps.item()) == 2 and np.isfinite(opt.grad_norm.item())
    assert not torch.equal(before[0], opt.weights[0])


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_steps_follow_rate_and_count(bits):
    sizes = [700, 4097]
    make = lambda: AdamW(tensors(sizes, torch.bfloat16, 8, 1.0), lr=LR, state_bits=bits, masters=True, max_grad_norm=0.5)
    eager, captured = make(), make()
    grads = tensors(sizes, torch.float32, 9, 0.1)
    eager.step(grads)
    captured.step(grads)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.step(grads)
    for rate in (1e-3, 5e-4):
        for o in (eager, captured):
            o.lr.fill_(rate)
        eager.step(grads)
        graph.replay()
        torch.cuda.synchronize()
        for name in ("weights", "masters", "m", "v"):
            assert all(torch.equal(a, c) for a, c in zip(getattr(eager, name), getattr(captured, name))), name
        assert torch.equal(eager.steps, captured.steps) and torch.equal(eager.grad_norm, captured.grad_norm)


def test_two_optimizers_on_two_streams():
    sizes = [100003, 333]
    grads = tensors(sizes, torch.float32, 11, 0.1)
    make = lambda: AdamW(tensors(sizes, torch.float32, 12, 1.0), lr=LR, state_bits=8, max_grad_norm=0.5)
    alone = make()
    for _ in range(4):
        alone.step(grads)
    torch.cuda.synchronize()
    both, streams = [make(), make()], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(4):
        for o, s in zip(both, streams):
            o.step(grads, stream=s)
    torch.cuda.synchronize()
    for o in both:
        assert all(torch.equal(a, c) for a, c in zip(o.weights + o.m + o.v, alone.weights + alone.m + alone.v))


def test_minimises_a_quadratic_the_same_in_8_bits():
    """Both states walk the same way: the 8-bit path stays within a tenth of the distance that the 32-bit one has walked."""
    target = tensors([5000], torch.float32, 13, 1.0)[0]
    ends = []
    for bits in (32, 8):
        w = torch.zeros(5000, device=DEV)
        opt = AdamW([w], lr=1e-2, weight_decay=0.0, state_bits=bits)
        for _ in range(50):
            opt.step([w - target])
        ends.append(w.clone())
    assert float((ends[1] - ends[0]).norm()) <= 0.1 * float(ends[0].norm())


def test_tensors_are_looked_at_in_every_step():
    w, g = torch.zeros(600, device=DEV), torch.ones(600, device=DEV)
    opt = AdamW([w], lr=0.1)
    opt.step([g])
    g.resize_(300)                                  # a tensor that the last step took
    with pytest.raises(ValueError):
        opt.step([g])
    g = torch.ones(600, device=DEV)
    kept, w.data = w.data, torch.zeros(600, device=DEV)
    with pytest.raises(ValueError):
        opt.step([g])
    w.data = kept
    for name, bad in (("lr", torch.zeros(2, device=DEV)), ("lr", torch.zeros(1)), ("steps", torch.zeros(1, device=DEV)),
                      ("grad_norm", torch.zeros(1, dtype=torch.float64, device=DEV))):
        good = getattr(opt, name)
        setattr(opt, name, bad)
        with pytest.raises((TypeError, ValueError)):
            opt.step([g])
        setattr(opt, name, good)
    opt.step([g])
    torch.cuda.synchronize()
    assert int(opt.steps.item()) == 2 and torch.equal(w, w[:1].expand(600)) and float(w[0]) < 0.0

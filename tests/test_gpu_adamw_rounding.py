"""States of 8 bits over many steps: codes that are rounded at random (from the 33rd step on) against the definition
(oracle/operators_oracle.py), and averages that follow their 32-bit ones.

Codes and scales are the definition's bit for bit: they are computed in 64 bits, so that only a value within about 2^-46 of a step
of a border between two codes could differ, and the borders are multiples of 2^-17 of a step.
Averages: a code that is rounded up with the probability of its share f of the way is right on average, and the recursions are
linear, so that E m and E v are the 32-bit ones.  Such a rounding has the variance f (1 - f) (step between the codes)^2, of which a
step later b^2 is left: var' = b^2 var + f (1 - f) step^2, with the f of the very run.  The roundings of different elements
are independent: the sum over many is asked to be within 6 standard deviations, and the few roundings to the nearest code of the
first 32 steps, each at most 1/16 of a value, within what is left of them: b^(t - 32) / 16 / (1 - b) at most, and never more than
32 / 16 of the value then; gradients are alike until step 500, so that these errors have no common sign, and what is left of
them is taken as another variance of (v / 16)^2 a step."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as orc
from paper_2512_06547_b200.optimizer import AdamW, decode_state
from tests.helpers import to_np64

pytestmark = pytest.mark.gpu
DEV = "cuda"
B1, B2 = 0.9, 0.95


def place(parts, offset):
    """Separate tensors, or neighbours in one buffer that start `offset` elements off its alignment."""
    if not offset:
        return [torch.from_numpy(p).to(DEV) for p in parts]
    flat = torch.empty(sum(p.size for p in parts) + offset, device=DEV)
    out, at = [], offset
    for p in parts:
        flat[at:at + p.size] = torch.from_numpy(p).to(DEV)
        out.append(flat[at:at + p.size])
        at += p.size
    return out


def check_steps(sizes, offset, grads_of, first, count):
    gen = np.random.default_rng(1)
    w = place([gen.standard_normal(n).astype(np.float32) for n in sizes], offset)
    steps = torch.full((1,), first - 1, dtype=torch.int64, device=DEV)
    opt = AdamW(w, lr=1e-3, betas=(B1, B2), state_bits=8, max_grad_norm=1.0, step=steps)
    m, v = [np.zeros(n) for n in sizes], [np.zeros(n) for n in sizes]
    for t in range(first, first + count):
        grads = grads_of(t)
        opt.step(place(grads, offset))
        torch.cuda.synchronize()
        _, scale = orc.clip_scale(grads, 1.0)
        encode = (lambda x, signed, i: orc.state_encode(x, signed)) if t <= 32 else (
            lambda x, signed, i: orc.state_encode_at_random(x, signed, t, i))
        for i, g in enumerate(grads):
            _, m1, v1 = orc.adamw(np.zeros(g.size), g, m[i], v[i], t, 0.0, B1, B2, 1e-8, 0.0, scale)
            for got, got_scale, x, signed in ((opt.m[i], opt.m_scales[i], m1, True), (opt.v[i], opt.v_scales[i], v1, False)):
                codes, scales = encode(x, signed, i)
                assert np.array_equal(to_np64(got_scale), scales), (t, i, signed)
                differ = np.flatnonzero(got.cpu().numpy() != codes)
                assert differ.size == 0, (t, i, signed, differ[:5], got.cpu().numpy()[differ[:5]], codes[differ[:5]])
            m[i] = orc.state_decode(opt.m[i].cpu().numpy(), to_np64(opt.m_scales[i]), True)
            v[i] = orc.state_decode(opt.v[i].cpu().numpy(), to_np64(opt.v_scales[i]), False)


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("first", [31, 40, 1 << 33])
def test_codes_are_the_definitions(first, offset):
    sizes = [1, 5, 255, 256, 257, 2049, 0, 3, 10007]
    gen = np.random.default_rng(first % 1000)
    check_steps(sizes, offset, lambda t: [(gen.standard_normal(n) * 10.0 ** gen.uniform(-3, -1)).astype(np.float32) for n in sizes],
                first, 4)


def test_codes_of_many_tensors():
    sizes = [1 + (37 * i) % 300 for i in range(805)]
    gen = np.random.default_rng(2)
    check_steps(sizes, 0, lambda t: [gen.standard_normal(n).astype(np.float32) for n in sizes], 100, 2)


def test_codes_of_gradients_of_unlike_size():
    """Codes below 8, zeros, scales that are subnormal or 0."""
    n = 256 * 6 + 17
    gen = np.random.default_rng(4)

    def grads(t):
        g = (gen.standard_normal(n) * 10.0 ** gen.uniform(-18, 2, n)).astype(np.float32)
        g[:256] = 0.0
        g[256:512] = 1e-33
        g[512:768] = np.float32(2.0 ** -3)
        return [g]
    check_steps([n], 0, grads, 50, 4)


def averages(opt, i=0):
    if opt.state_bits == 32:
        return opt.m[i].double(), opt.v[i].double()
    n = opt.m[i].numel()
    new = lambda: torch.empty(n, device=DEV)
    return (decode_state(opt.m[i], opt.m_scales[i], signed=True, out=new()).double(),
            decode_state(opt.v[i], opt.v_scales[i], signed=False, out=new()).double())


def variance(x, scales):
    """Of the rounding of x at random."""
    unit = torch.repeat_interleave(scales.double(), 256)
    a = x.abs() / unit
    step = torch.exp2((torch.frexp(a)[1] - 4).clamp_min(0).double())
    f = a / step - torch.floor(a / step)
    return f * (1 - f) * (step * unit).square()


@pytest.mark.parametrize("later", [1.0, 0.1, 0.0])
@pytest.mark.parametrize("beta2", [0.95, 0.999])
def test_averages_follow_those_in_32_bits(beta2, later):
    """Gradients that stay, fall to a tenth, or stop, for every other element of a block."""
    n, falls_at, steps = 256 * 96, 500, 2500
    gen = torch.Generator(device=DEV).manual_seed(7)
    falls = torch.arange(n, device=DEV) % 2 == 0
    wide, narrow = [AdamW([torch.zeros(n, device=DEV)], lr=1e-3, betas=(B1, beta2), weight_decay=0.0, state_bits=bits)
                    for bits in (32, 8)]
    betas = (B1, beta2)
    var = [torch.zeros(n, dtype=torch.float64, device=DEV) for _ in betas]
    factor = torch.ones(n, device=DEV)
    held = averages(narrow)
    for t in range(1, steps + 1):
        if t == falls_at:
            factor[falls] = later
        g = (torch.randn(n, generator=gen, device=DEV) + 0.5) * factor
        wide.step([g])
        narrow.step([g])
        for k, (beta, add, scales) in enumerate(zip(betas, (g.double(), g.double().square()), (narrow.m_scales[0], narrow.v_scales[0]))):
            x = beta * held[k] + (1 - beta) * add
            var[k] = beta ** 2 * var[k] + (variance(x, scales) if t > 32 else (x / 16).square())
        held = averages(narrow)
    for part in (falls, ~falls):
        for k, (a, b, scales) in enumerate(zip(averages(narrow), averages(wide), (narrow.m_scales[0], narrow.v_scales[0]))):
            far, most = abs(float((a[part] - b[part]).sum())), 6 * float(var[k][part].sum().sqrt())
            # of fp32 sums and values, which stand still as subnormals: 0.9 times a few of the smallest is as many of them
            most += 2.0 ** -20 * float(b[part].abs().sum()) + 2.0 ** -126 * n
            if k and later == 0.0 and part is falls:
                most += float(torch.repeat_interleave(scales.double(), 256)[part].sum())   # v above 0 is not stored as 0
            assert far <= most, ("mv"[k], far, most, float(b[part].sum()))
    if later == 0.0:
        assert not bool(averages(narrow)[0][falls].any())            # m has long been 0


def test_runs_repeat_and_replay():
    gen = torch.Generator(device=DEV).manual_seed(8)
    w = torch.randn(5003, generator=gen, device=DEV)
    grads = torch.randn(5003, generator=gen, device=DEV)
    make = lambda: AdamW([w.clone()], lr=1e-2, state_bits=8)
    eager, again, replayed = make(), make(), make()
    replayed.step([grads])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        replayed.step([grads])
    for _ in range(49):
        graph.replay()
    for o in (eager, again):
        for _ in range(50):
            o.step([grads])
    torch.cuda.synchronize()
    for o in (again, replayed):
        assert int(o.steps.item()) == 50
        for a, b in zip((eager.weights, eager.m, eager.v, eager.m_scales, eager.v_scales), (o.weights, o.m, o.v, o.m_scales, o.v_scales)):
            assert torch.equal(a[0], b[0])

"""Sampling against the fp64 definition (oracle/operators_oracle.py).

Weights are off by at most 2^-32 of their value and sums by that share of the total (the 53-bit additions add less than 2^-40
for up to 2^18 terms), so a token may differ from the definition's only where u times the total lies within
SLACK = 2^-31 of the total of the token's own stretch: the stretch of the returned token, widened by that, has to hold u.
n_kept: the mass that top_p compares is a sum of multiples of 2^-43, each off by half of one, in units of the largest weight
(which is 1, so the total is at least 1): V 2^-44 < 2^-26 for V <= 2^18, of which borders are only asked to be free in these
inputs; where the definition's share lies that close to a border the next count is accepted too.
logp = z - log W: z is a quotient in 64 bits, log W is off by at most 2^-31; one rounding to fp32: |d| <= 2^-31 + 2^-24 |logp|."""
import numpy as np
import pytest
import torch

import paper_2512_06547_b200 as a3po
from oracle import operators_oracle as orc
from tests.helpers import to_np64

pytestmark = pytest.mark.gpu
DEV = "cuda"
TD = {"f32": torch.float32, "bf16": torch.bfloat16}
SLACK = 2.0 ** -31


def dev(x, dtype):
    return None if x is None else torch.tensor(np.asarray(x), dtype=dtype, device=DEV)


def run(logits, u, mask=None, temperature=None, top_k=None, top_p=None, min_p=None, stream=None):
    n, v = logits.shape
    out = dict(token=torch.full((n,), -7, dtype=torch.int32, device=DEV), logp=torch.full((n,), 9.0, device=DEV),
               kept_logp=torch.full((n,), 9.0, device=DEV), n_kept=torch.full((n,), -7, dtype=torch.int32, device=DEV))
    ws = a3po.new_workspace(a3po.a3po_sample_workspace_bytes(n, v), DEV)
    a3po.a3po_sample(logits, u, out["token"], ws, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p,
                     row_mask=mask, logp=out["logp"], kept_logp=out["kept_logp"], n_kept=out["n_kept"], stream=stream)
    return out


def check(logits, u, mask=None, temperature=None, top_k=None, top_p=None, min_p=None):
    """Every row of one call against the definition."""
    n, v = logits.shape
    got = run(logits, dev(u, torch.float32), dev(mask, torch.uint8), dev(temperature, torch.float32), dev(top_k, torch.int32),
              dev(top_p, torch.float32), dev(min_p, torch.float32))
    torch.cuda.synchronize()
    got = {k: to_np64(x) for k, x in got.items()}
    rows = to_np64(logits)
    pick = lambda a, i, off: off if a is None else np.float32(np.asarray(a)[i])
    for i in range(n):
        args = dict(temperature=float(pick(temperature, i, 1.0)), top_k=int(pick(top_k, i, 0)), min_p=float(pick(min_p, i, 0.0)))
        p = float(pick(top_p, i, 1.0))
        ref = None if mask is not None and not mask[i] else orc.sample_row(rows[i], float(np.float32(u[i])), top_p=p, **args)
        mine = {k: x[i] for k, x in got.items()}
        if ref is None:
            assert mine == dict(token=-1, logp=0.0, kept_logp=0.0, n_kept=0), (i, mine)
            continue
        counts = {ref["n_kept"]}
        if p < 1:
            for q in (p * (1 - 2.0 ** -26), p * (1 + 2.0 ** -26)):
                counts.add(_count_at(rows[i], q, args))
        assert mine["n_kept"] in counts, (i, v, mine, ref["n_kept"])
        token = int(mine["token"])
        if mine["n_kept"] == ref["n_kept"]:
            assert ref["kept"][token], (i, token)
            total = ref["sums"][-1]
            at = min(max(float(np.float32(u[i])), 0.0), 1.0) * total
            below = ref["sums"][token - 1] if token else 0.0
            assert below - SLACK * total <= at <= ref["sums"][token] + SLACK * total, (i, token, ref["token"])
            bound = SLACK + 2.0 ** -24 * abs(ref["kept_logp"] - ref["z"] + _z(rows[i], token, args))
            klp = _z(rows[i], token, args) - np.log(total)
            assert abs(mine["kept_logp"] - klp) <= bound, (i, mine["kept_logp"], klp)
        lp = _z(rows[i], token, args) - np.log(ref["w"].sum())
        assert abs(mine["logp"] - lp) <= SLACK + 2.0 ** -24 * abs(lp), (i, mine["logp"], lp)
    return got


def _z(row, token, args):
    row = np.where(np.isnan(row), -np.inf, row)
    t = args["temperature"] if args["temperature"] > 0 else 1.0
    return 0.0 if row[token] == row.max() else (row[token] - row.max()) / t


def _count_at(row, p, args):
    """n_kept with a share that is not an fp32 number."""
    full = orc.sample_row(row, 0.5, top_p=1.0, temperature=args["temperature"], top_k=args["top_k"])
    n = full["n_kept"]
    run_ = np.cumsum(full["w"][full["order"][:n]])
    count = 1 + int((run_[:-1] < p * run_[-1]).sum()) if args["temperature"] > 0 else 1
    if args["min_p"] > 0:
        count = max(1, int((full["w"][full["order"][:count]] >= args["min_p"]).sum()))
    return count


def make(n, v, dt, seed, sigma=2.0, banned=0.0):
    gen = np.random.default_rng(seed)
    x = gen.standard_normal((n, v)).astype(np.float32) * np.float32(sigma)
    x[np.arange(n), gen.integers(0, v, n)] += 4
    if banned:
        x[gen.random((n, v)) < banned] = -np.inf
    return torch.from_numpy(x).to(TD[dt]).to(DEV), gen


SIZES = [(3, 1), (2, 7), (5, 32), (4, 129), (3, 1000), (3, 1024), (2, 1025), (2, 8191), (3, 32003), (2, 50257), (3, 151936),
         (1, 262144)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,v", SIZES)
def test_temperature_alone(n, v, dt):
    x, gen = make(n, v, dt, 100 + v)
    check(x, gen.random(n), temperature=gen.choice([0.0, 0.3, 0.8, 1.0, 2.5], n))
    check(x, gen.random(n))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,v", SIZES)
def test_filters(n, v, dt):
    x, gen = make(n, v, dt, 200 + v, banned=0.1 if v > 100 else 0.0)
    u = gen.random(n)
    check(x, u, top_k=gen.choice([1, 2, 20, 50, 1000, v, 0], n))
    check(x, u, top_p=gen.choice([0.1, 0.5, 0.9, 0.95, 0.999, 1.0], n))
    check(x, u, min_p=gen.choice([0.0, 0.01, 0.1, 0.5, 1.0], n))
    check(x, u, temperature=gen.choice([0.0, 0.6, 1.0, 1.5], n), top_k=gen.choice([0, 5, 40, 300], n),
          top_p=gen.choice([0.3, 0.9, 1.0], n), min_p=gen.choice([0.0, 0.02], n))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_many_rows_with_a_mask(dt):
    n, v = 301, 4099
    x, gen = make(n, v, dt, 3)
    mask = (gen.random(n) < 0.7).astype(np.uint8)
    x[torch.from_numpy(mask == 0).to(DEV)] = float("nan")
    check(x, gen.random(n), mask=mask)
    check(x, gen.random(n), mask=mask, top_k=np.full(n, 30), top_p=np.full(n, 0.9))


@pytest.mark.parametrize("filters", [False, True])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_equal_logits(dt, filters):
    """Borders that are reached exactly: equal weights, shares that are whole numbers of tokens."""
    for v in (10, 1000, 32000, 151936):
        x = torch.full((4, v), 1.7, device=DEV).to(TD[dt])
        u = np.array([0.0, 0.25, 0.5, 0.75])
        more = dict(top_p=[0.5, 0.25, 0.5, 1.0], top_k=[0, 0, v // 2, 3]) if filters else {}
        got = check(x, u, **more)
        kept = [v // 2, max(1, v // 4 + (v % 4 > 0)), max(1, v // 4 + (v // 2 % 2 > 0)), 3] if filters else [v] * 4
        assert got["n_kept"].tolist() == kept
        want = [int(np.floor(a * k)) for a, k in zip(u, kept)]
        assert got["token"].tolist() == want


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_extreme_rows(dt):
    """Infinities, NaN, the type's lowest value, nothing at all, one token, -0 beside 0, large and subnormal logits."""
    v = 2100
    low = torch.finfo(TD[dt]).min
    gen = np.random.default_rng(5)
    x = torch.from_numpy(gen.standard_normal((16, v)).astype(np.float32)).to(TD[dt]).to(DEV)
    x[0] = float("-inf")
    x[1] = float("nan")
    x[2] = float("-inf"); x[2, 2099] = -3.0
    x[3, 5] = float("inf"); x[3, 1700] = float("inf")
    x[4] = low
    x[5, :2000] = low
    x[6, ::2] = float("nan")
    x[7, 1:] = float("-inf")
    x[8] = 0.0; x[8, ::2] = -0.0
    x[9] *= 1e30
    x[10] *= 1e-38
    x[11] += 1000.0
    x[12] -= 30000.0
    x[13, 77] = 200.0
    x[14, :] = -200.0; x[14, 3] = 0.0
    x[15, :1024] = float("-inf")
    u = gen.random(16)
    for uu in (u, np.zeros(16), np.full(16, 1 - 2.0 ** -24), np.full(16, 1.0), np.full(16, -1.0)):
        check(x, uu)
        check(x, uu, temperature=np.resize([1.0, 0.01, 30.0], 16))
        check(x, uu, top_k=np.full(16, 900))
        check(x, uu, top_p=np.full(16, 0.9))
        check(x, uu, min_p=np.full(16, 0.2), top_k=np.resize([0, 1, 2000], 16), top_p=np.resize([0.0, 0.7, 1.0], 16))


def test_temperatures_at_the_ends():
    x, gen = make(8, 700, "f32", 6)
    t = [1e-30, 1e-3, 1e3, 1e30, float("inf"), 1e-40, -1.0, 0.0]
    u = gen.random(8)
    for more in ({}, dict(top_k=np.full(8, 50)), dict(top_p=np.full(8, 0.8)), dict(min_p=np.full(8, 0.3))):
        check(x, u, temperature=t, **more)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("start", [0, 1, 3, 6])
def test_rows_apart_and_off_16_bytes(dt, start):
    n, v, ld = 5, 3001, 3307
    gen = np.random.default_rng(7)
    buf = torch.from_numpy(gen.standard_normal(n * ld + 16).astype(np.float32) * 2).to(TD[dt]).to(DEV)
    x = buf[start:start + n * ld].view(n, ld)[:, :v]
    buf.view(-1)[start + v:start + ld] = float("inf")        # between the rows: not to be read
    u = gen.random(n)
    check(x, u)
    check(x, u, top_k=np.full(n, 100), top_p=np.full(n, 0.9))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,v", [(320, 33), (320, 1024), (320, 1025), (320, 4096), (700, 2048), (300, 8192)])
def test_many_short_rows(n, v, dt):
    """Rows by small blocks and, one logit or row further, by large ones; ties in every third, more kept than a small block holds."""
    x, gen = make(n, v, dt, 300 + v, banned=0.05)
    x[::3] = x[::3].float().round().to(TD[dt])
    u = gen.random(n)
    check(x, u)
    check(x, u, top_k=gen.choice([1, 30, 600, v, 0], n))
    check(x, u, top_p=gen.choice([0.2, 0.9, 0.999], n))
    check(x, u, temperature=gen.choice([0.0, 0.3, 1.0, 5.0], n), top_k=gen.choice([0, 20, 700], n), top_p=gen.choice([0.5, 0.99], n),
          min_p=gen.choice([0.0, 0.01], n))


@pytest.mark.parametrize("dt,v,start", [("f32", 393216, 0), ("f32", 393216, 1), ("f32", 393215, 3), ("bf16", 786432, 0),
                                        ("bf16", 786432, 5), ("bf16", 786425, 7)])
def test_longest_rows_with_filters(dt, v, start):
    """Rows that fill eight SMs, one of them flat but for ties that no step of distance bounds."""
    gen = np.random.default_rng(v + start)
    buf = torch.from_numpy(gen.standard_normal(2 * v + 16).astype(np.float32) * 2).to(TD[dt]).to(DEV)
    x = buf[start:start + 2 * v].view(2, v)
    x[1] = 1.0
    x[1, v - 5000:] = 1.5
    u = gen.random(2)
    check(x, u, top_k=np.array([50, 4000]))
    check(x, u, top_p=np.array([0.9, 0.5]))
    check(x, u, top_k=np.array([100000, 300000]), top_p=np.array([0.999, 0.7]), min_p=np.array([1e-6, 0.0]))


@pytest.mark.parametrize("filters", [False, True])
def test_two_streams_capture_and_repeat(filters):
    n, v = 40, 20011
    x, gen = make(n, v, "bf16", 8)
    y, _ = make(n, v, "bf16", 9)
    u = dev(gen.random(n), torch.float32)
    more = dict(top_k=dev(np.full(n, 60), torch.int32), top_p=dev(np.full(n, 0.9), torch.float32)) if filters else {}
    first, second = run(x, u, **more), run(y, u, **more)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = []
        for s, l in zip(streams, (x, y)):
            with torch.cuda.stream(s):
                got.append(run(l, u, **more))
        torch.cuda.synchronize()
        for a, b in zip(got, (first, second)):
            for k in a:
                assert torch.equal(a[k], b[k])
    graph = torch.cuda.CUDAGraph()
    held = x.clone()
    with torch.cuda.graph(graph):
        out = run(held, u, **more)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(out[k], first[k]) for k in out)
    held.copy_(y)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(out[k], second[k]) for k in out)


def test_frequencies():
    """Tokens of many draws come as often as their probabilities say: 5 standard deviations of the count."""
    v, n = 50, 200000
    gen = np.random.default_rng(10)
    row = torch.from_numpy(gen.standard_normal((1, v)).astype(np.float32)).to(DEV)
    x = row.expand(n, v).contiguous()
    u = torch.rand(n, device=DEV, generator=torch.Generator(device=DEV).manual_seed(3))
    got = run(x, u)
    q = np.exp(to_np64(row)[0]); q /= q.sum()
    count = np.bincount(to_np64(got["token"]), minlength=v)
    assert (np.abs(count - n * q) <= 5 * np.sqrt(n * q * (1 - q)) + 1).all()

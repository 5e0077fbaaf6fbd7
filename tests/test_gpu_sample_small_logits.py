"""bf16 logits that are close to 0 beside the largest (or the largest beside them): the difference of the two is not an fp32 number, and
its rounding, at most 2^-24 of it, goes into the weight.

w = exp(d / t), d off by 2^-24 |d|: w is off by 2^-24 |d| / t of itself, so sums by the sum of that, besides the 2^-31 that every
weight carries (twice, in SLACK, for the rest of the arithmetic).  A token may be the neighbour of the definition's where u times the
total is within that of the border.  The error is largest where the largest logit and those next to it weigh about the same and differ by just under half a step of the
difference: 5.5 and 6.90625 over 2.2e-7, once in 250 and 1,000.  Random numbers lie around the borders in steps of 2^-24."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as orc
from tests.helpers import to_np64
from tests.test_gpu_sample import SLACK, dev, run

pytestmark = pytest.mark.gpu
DEV = "cuda"


def rows(v):
    """12 (first, in the middle, last) over 4.5e-7; 1e-6 over -9 and -9.0625; 5.5 and 6.90625 every so often over 2.2e-7."""
    x = np.full((6, v), 4.5e-7, np.float32)
    x[0, 0] = x[1, v // 2] = x[2, v - 1] = 12.0
    x[3] = np.where(np.arange(v) % 2 == 0, -9.0, -9.0625)
    x[3, v // 3] = 1e-6
    x[4:] = 2.2e-7
    x[4, ::250] = 5.5
    x[5, ::1000] = 6.90625
    return torch.from_numpy(x).bfloat16().to(DEV)


@pytest.mark.parametrize("filters", ["none", "top_p", "min_p"])
@pytest.mark.parametrize("t", [1.0, 0.75])
@pytest.mark.parametrize("v,copies", [(1000, 1), (1000, 100), (8000, 1), (32000, 1), (151936, 1)])
def test_borders(v, copies, t, filters):
    x = rows(v)
    kinds, host = x.shape[0], to_np64(x)
    x = x.repeat(copies, 1)           # many short rows without a filter take another kernel
    n = x.shape[0]
    args = {"none": {}, "top_p": dict(top_p=0.999), "min_p": dict(min_p=1e-12)}[filters]
    more = {k: dev(np.full(n, a), torch.float32) for k, a in args.items()}
    refs = [orc.sample_row(host[i], 0.5, temperature=t, **args) for i in range(kinds)]
    off = []
    for i, ref in enumerate(refs):
        w = np.where(ref["kept"], ref["w"], 0.0)
        off.append(SLACK + 2.0 ** -24 * float((w * np.abs(host[i] - host[i].max())).sum()) / t / ref["sums"][-1])
    best = host.argmax(axis=1)
    border = np.array([refs[i]["sums"][best[i]] / refs[i]["sums"][-1] for i in range(kinds)])
    before = np.array([(refs[i]["sums"][best[i] - 1] if best[i] else 0.0) / refs[i]["sums"][-1] for i in range(kinds)])
    for around in (border, before):
        for step in (-64, -8, -2, -1, 0, 1, 2, 8, 64):
            u = np.tile(np.clip(around + step * 2.0 ** -24, 0, 1 - 2.0 ** -24).astype(np.float32), copies)
            got = run(x, dev(u, torch.float32), temperature=dev(np.full(n, t), torch.float32), **more)
            torch.cuda.synchronize()
            for i, ref in enumerate(refs):
                token, total = int(got["token"][i]), ref["sums"][-1]
                assert int(got["n_kept"][i]) == ref["n_kept"] and ref["kept"][token]
                below = ref["sums"][token - 1] / total if token else 0.0
                assert below - off[i] <= float(u[i]) <= ref["sums"][token] / total + off[i], (i, step, token)
                z = (host[i, token] - host[i].max()) / t
                for name, all_of in (("logp", ref["w"].sum()), ("kept_logp", total)):
                    lp = z - np.log(all_of)
                    whole = SLACK + 2.0 ** -24 * float((ref["w"] * np.abs(host[i] - host[i].max())).sum()) / t / all_of
                    assert abs(float(got[name][i]) - lp) <= whole + 2.0 ** -24 * abs(lp), (i, name)

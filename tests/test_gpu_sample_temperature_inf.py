"""Infinite temperatures: they count as 1e30, at which every finite logit of ordinary size has the weight 1, an infinite one beside
finite ones has all of it, and min-p = 1 keeps the largest alone (a weight of less than 1 is less than 1 whatever 64 bits make of it)."""
import numpy as np
import pytest
import torch

from tests.helpers import to_np64
from tests.test_gpu_sample import TD, check, dev, make, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("v", [700, 5000])
def test_infinite_temperatures(v, dt):
    n = 6
    x, gen = make(n, v, dt, 20)
    x[1, 17] = float("inf")
    x[2, 3] = x[2, v - 5] = float("inf")
    x[3, ::3] = float("-inf")
    x[4] = torch.finfo(TD[dt]).min
    x[5, 1:] = float("-inf")
    top = to_np64(x).max(axis=1, keepdims=True)
    largest = to_np64(x) == top
    hot = dev(np.full(n, np.inf), torch.float32)
    for u in (gen.random(n), np.zeros(n), np.full(n, 1 - 2.0 ** -24)):
        for more in ({}, dict(top_k=np.full(n, 50)), dict(top_p=np.full(n, 0.8)), dict(min_p=np.full(n, 0.3)), dict(min_p=np.full(n, 2.0))):
            same = check(x, u, temperature=np.full(n, 1e30), **more)
            got = run(x, dev(u, torch.float32), temperature=hot, top_k=dev(more.get("top_k"), torch.int32),
                      top_p=dev(more.get("top_p"), torch.float32), min_p=dev(more.get("min_p"), torch.float32))
            torch.cuda.synchronize()
            for k in same:
                assert np.array_equal(to_np64(got[k]), same[k]), (k, more)
        got = run(x, dev(u, torch.float32), temperature=hot, min_p=dev(np.ones(n), torch.float32))
        torch.cuda.synchronize()
        assert to_np64(got["n_kept"]).tolist() == largest.sum(axis=1).tolist()
        assert largest[np.arange(n), to_np64(got["token"]).astype(int)].all()

"""Pins of the fp64 definitions the operator tests compare with: published random-number vectors, finite differences,
closed forms."""
import math

import numpy as np
import pytest

from oracle import operators_oracle as orc


def test_philox_known_answers():
    """The vectors published with the generator (zeros, ones, digits of pi)."""
    hexes = lambda c, k: ["%08x" % w for w in orc.philox4x32_10(c, k)]
    assert hexes([0] * 4, [0] * 2) == ["6627e8d5", "e169c58d", "bc57ac4c", "9b00dbd8"]
    assert hexes([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2) == ["408f276d", "41c83b0e", "a20bc7c6", "6d5451fd"]
    assert hexes([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0]) == [
        "d16cfe09", "94fdcceb", "5001e420", "24126ea1"]


def test_dropout_factors():
    assert np.all(orc.dropout_factors(3, 11, 0.0, 5, 6) == 1.0)
    assert np.all(orc.dropout_factors(3, 11, 1.0, 5, 6) == 0.0)
    f = orc.dropout_factors(64, 256, 0.25, 123, 1 << 40)
    assert set(np.unique(f)) == {0.0, 65536 / (65536 - 16384)}
    kept = float((f != 0).mean())
    assert abs(kept - 0.75) <= 5 * math.sqrt(0.25 * 0.75 / f.size)       # five standard deviations of the share
    assert np.any(f != orc.dropout_factors(64, 256, 0.25, 123, (1 << 40) + 1))
    # an element's mask depends on its place only, not on the matrix around it
    assert np.array_equal(f[:10, :100], orc.dropout_factors(10, 100, 0.25, 123, 1 << 40))


def _fd(fun, x, i, eps=1e-5):
    a, b = x.copy(), x.copy()
    a.flat[i] += eps
    b.flat[i] -= eps
    return (fun(a) - fun(b)) / (2 * eps)


@pytest.mark.parametrize("layer", [False, True])
def test_norm_gradients_by_differences(layer):
    rng = np.random.default_rng(1)
    n, h = 4, 7
    x, gy = rng.standard_normal((n, h)) + 0.3, rng.standard_normal((n, h))
    gamma, beta = rng.standard_normal(h), rng.standard_normal(h)
    mask = np.array([1, 0, 1, 1])
    x[1] = np.nan
    loss = lambda xx, gg, bb: float((orc.norm_fwd(xx, gg, bb, layer, 1e-3, mask)[0] * np.where(mask[:, None], gy, 0)).sum())
    y, mean, rstd = orc.norm_fwd(x, gamma, beta, layer, 1e-3, mask)
    assert np.all(y[1] == 0) and mean[1] == 0 and rstd[1] == 0
    dx, dg, db = orc.norm_bwd(x, gamma, mean, rstd, gy, layer, mask)
    assert np.all(dx[1] == 0)
    for i in range(n * h):
        if i // h != 1:
            assert dx.flat[i] == pytest.approx(_fd(lambda v: loss(v, gamma, beta), x, i), abs=1e-7)
    for i in range(h):
        assert dg[i] == pytest.approx(_fd(lambda v: loss(x, v, beta), gamma, i), abs=1e-7)
        assert db[i] == pytest.approx(_fd(lambda v: loss(x, gamma, v), beta, i), abs=1e-7)
    if layer:
        assert np.allclose(dx[[0, 2, 3]].sum(axis=1), 0, atol=1e-12)     # a shift of the row changes nothing


def test_norm_closed_forms():
    x = np.array([[3.0, 3.0, 3.0, 3.0]])
    y, mean, rstd = orc.norm_fwd(x, np.ones(4), None, True, 1e-6)
    assert np.all(y == 0) and mean[0] == 3.0 and rstd[0] == pytest.approx(1e3)
    y, _, rstd = orc.norm_fwd(x, np.ones(4), None, False, 0.0)
    assert np.allclose(y, 1.0) and rstd[0] == pytest.approx(1 / 3)


@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
def test_gated_ffn_gradients_by_differences(act):
    rng = np.random.default_rng(2)
    n, h, f = 4, 5, 6
    x, gy = rng.standard_normal((n, h)), rng.standard_normal((n, h))
    wgu, wd = rng.standard_normal((2 * f, h)), rng.standard_normal((h, f))
    mask = np.array([1, 1, 0, 1])
    x[2] = np.inf
    loss = lambda xx, a, b: float((orc.gated_ffn_fwd(xx, a, b, act, mask) * np.where(mask[:, None], gy, 0)).sum())
    assert np.all(orc.gated_ffn_fwd(x, wgu, wd, act, mask)[2] == 0)
    dx, dgu, dd = orc.gated_ffn_bwd(x, wgu, wd, gy, act, mask)
    for got, fun, at in ((dx, lambda v: loss(v, wgu, wd), x), (dgu, lambda v: loss(x, v, wd), wgu),
                         (dd, lambda v: loss(x, wgu, v), wd)):
        for i in range(0, at.size, 3):
            if np.isfinite(at.flat[i]):
                assert got.flat[i] == pytest.approx(_fd(fun, at, i), rel=1e-6, abs=1e-6)
    assert np.all(dx[2] == 0)


def test_activation_values():
    v, d = orc.activation("silu", np.array([0.0, 40.0, -40.0]))
    assert np.allclose(v, [0, 40, 0], atol=1e-12) and np.allclose(d, [0.5, 1, 0], atol=1e-12)
    v, d = orc.activation("gelu_tanh", np.array([0.0, 40.0, -40.0]))
    assert np.allclose(v, [0, 40, 0], atol=1e-12) and np.allclose(d, [0.5, 1, 0], atol=1e-12)
    # the tanh form stays within 5e-4 of g Phi(g)
    g = np.linspace(-4, 4, 41)
    phi = np.array([0.5 * (1 + math.erf(t / math.sqrt(2))) for t in g])
    assert np.max(np.abs(orc.activation("gelu_tanh", g)[0] - g * phi)) < 5e-4

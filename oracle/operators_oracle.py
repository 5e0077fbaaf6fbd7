"""Plain fp64 definitions (numpy) of the operators around the LM head: norm, dropout with a counter-based mask, their
join on the residual stream, and the gated feed-forward block.  Written from the formulas; shares nothing with csrc/.

Rows whose mask is 0 are selected away: whatever they hold, their outputs are 0 and they add nothing to a sum.
"""
from __future__ import annotations

import math

import numpy as np

U32 = (1 << 32) - 1


def _select(mask, a):
    a = np.asarray(a, dtype=np.float64)
    if mask is None:
        return a
    return np.where((np.asarray(mask) != 0)[:, None], a, 0.0)


# ------------------------------------------------------------------------------ random numbers
def philox4x32_10(counter, key):
    """One block of Philox4x32 with ten rounds (Salmon et al. 2011): four 32-bit words from plain integers."""
    c, k = [int(v) & U32 for v in counter], [int(v) & U32 for v in key]
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & U32, (a >> 32) ^ c[3] ^ k[1], a & U32]
        k = [(k[0] + 0x9E3779B9) & U32, (k[1] + 0xBB67AE85) & U32]
    return c


def dropout_factors(n, h, p, seed, offset):
    """[n, h]: 0 where the element is dropped, else 65536 / (65536 - T) with T = round(65536 p), p as fp32."""
    t = int(np.rint(65536.0 * np.float64(np.float32(p))))
    scale = 65536.0 / (65536 - t) if t < 65536 else 0.0
    out = np.zeros((n, h))
    seed, offset = int(seed) % (1 << 64), int(offset) % (1 << 64)
    for row in range(n):
        for g in range((h + 7) // 8):
            w = philox4x32_10((g, row, offset & U32, offset >> 32), (seed & U32, seed >> 32))
            u = [v for x in w for v in (x & 0xFFFF, x >> 16)]
            for j in range(min(8, h - 8 * g)):
                out[row, 8 * g + j] = scale if u[j] >= t else 0.0
    return out


def dropout(x, factors, residual=None, mask=None):
    x = _select(mask, x)
    y = np.where(factors != 0.0, x * factors, 0.0)      # dropped elements are selected away, not multiplied
    return y if residual is None else y + _select(mask, residual)


# ------------------------------------------------------------------------------ norm
def norm_fwd(x, gamma, beta=None, layer=False, eps=1e-6, mask=None):
    """Returns y, mean [n], rstd [n] (both 0 for rows masked out)."""
    n = x.shape[0]
    x = _select(mask, x)
    keep = np.ones(n, dtype=bool) if mask is None else np.asarray(mask) != 0
    mean = x.mean(axis=1) if layer else np.zeros(n)
    d = x - mean[:, None]
    with np.errstate(divide="ignore", invalid="ignore"):
        rstd = 1.0 / np.sqrt((d * d).mean(axis=1) + eps)
        y = d * rstd[:, None] * np.asarray(gamma, dtype=np.float64)
    if beta is not None:
        y = y + np.asarray(beta, dtype=np.float64)
    return np.where(keep[:, None], y, 0.0), np.where(keep, mean, 0.0), np.where(keep, rstd, 0.0)


def norm_bwd(x, gamma, mean, rstd, grad_y, layer=False, mask=None):
    """Returns grad_x, grad_gamma, grad_beta, given the forward's statistics (mean ignored unless layer)."""
    keep = np.ones(x.shape[0], dtype=bool) if mask is None else np.asarray(mask) != 0
    x, gy = _select(mask, x), _select(mask, grad_y)
    rstd = np.where(keep, np.asarray(rstd, dtype=np.float64), 0.0)
    mu = np.where(keep, np.asarray(mean, dtype=np.float64), 0.0) if layer else np.zeros(x.shape[0])
    xhat = (x - mu[:, None]) * rstd[:, None]
    gx = gy * np.asarray(gamma, dtype=np.float64)
    m1 = (gx * xhat).mean(axis=1, keepdims=True)
    m0 = gx.mean(axis=1, keepdims=True) if layer else 0.0
    return (gx - m0 - xhat * m1) * rstd[:, None], (gy * xhat).sum(axis=0), gy.sum(axis=0)


# ------------------------------------------------------------------------------ gated feed-forward block
def activation(name, g):
    """Value and derivative of the gate's activation."""
    g = np.asarray(g, dtype=np.float64)
    if name == "silu":
        s = 1.0 / (1.0 + np.exp(-g))
        return g * s, s + g * s * (1.0 - s)
    inner = math.sqrt(2.0 / math.pi) * (g + 0.044715 * g ** 3)
    th = np.tanh(inner)
    slope = math.sqrt(2.0 / math.pi) * (1.0 + 3 * 0.044715 * g ** 2)
    return 0.5 * g * (1.0 + th), 0.5 * (1.0 + th) + 0.5 * g * (1.0 - th * th) * slope


def gated_ffn_fwd(x, w_gate_up, w_down, act="silu", mask=None):
    f = w_gate_up.shape[0] // 2
    x = _select(mask, x)
    g, u = x @ np.asarray(w_gate_up[:f], dtype=np.float64).T, x @ np.asarray(w_gate_up[f:], dtype=np.float64).T
    return (activation(act, g)[0] * u) @ np.asarray(w_down, dtype=np.float64).T


def gated_ffn_bwd(x, w_gate_up, w_down, grad_y, act="silu", mask=None):
    """Returns grad_x, grad_w_gate_up, grad_w_down."""
    f = w_gate_up.shape[0] // 2
    x, gy = _select(mask, x), _select(mask, grad_y)
    wgu, wd = np.asarray(w_gate_up, dtype=np.float64), np.asarray(w_down, dtype=np.float64)
    g, u = x @ wgu[:f].T, x @ wgu[f:].T
    a, da = activation(act, g)
    dh = gy @ wd
    dgu = np.concatenate([dh * u * da, dh * a], axis=1)
    return dgu @ wgu, dgu.T @ x, gy.T @ (a * u)

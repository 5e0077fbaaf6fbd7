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


# ------------------------------------------------------------------------------ sampling
def sample_row(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row: token, logp, kept_logp, n_kept, and what they come from (w: all weights, kept: truth values by index).
    None where no logit is above -inf."""
    l = np.asarray(logits, dtype=np.float64)
    l = np.where(np.isnan(l), -np.inf, l)
    if not (l > -np.inf).any():
        return None
    top = l.max()
    t = float(temperature) if temperature > 0 else 1.0
    with np.errstate(invalid="ignore"):
        w = np.where(l == top, 1.0, np.exp((l - top) / t))
    order = np.lexsort((np.arange(l.size), -l))
    n = l.size if top_k <= 0 else min(int(top_k), l.size)
    if temperature <= 0:
        n = 1
    run = np.cumsum(w[order[:n]])
    if float(np.float32(top_p)) < 1 and temperature > 0:
        share = max(float(np.float32(top_p)), 0.0) * run[-1]
        n = 1 + int((run[:-1] < share).sum())
    if min_p > 0 and temperature > 0:
        n = max(1, int((w[order[:n]] >= float(np.float32(min_p))).sum()))
    kept = np.zeros(l.size, dtype=bool)
    kept[order[:n]] = True
    kept &= l > -np.inf
    sums = np.cumsum(np.where(kept, w, 0.0))
    over = np.flatnonzero(sums > max(float(u), 0.0) * sums[-1]) if u == u else np.flatnonzero(sums > 0)
    token = int(over[0]) if over.size else int(np.flatnonzero(kept & (w > 0))[-1])
    z = 0.0 if l[token] == top else (l[token] - top) / t
    return dict(token=token, logp=z - np.log(w.sum()), kept_logp=z - np.log(sums[-1]), n_kept=int(kept.sum()), w=w,
                kept=kept, sums=sums, order=order, z=z)


# ------------------------------------------------------------------------------ AdamW
STATE_BLOCK = 256


def state_table(codes):
    return np.array([c if c < 8 else (8 + c % 8) << (c // 8 - 1) for c in range(codes)], dtype=np.float64)


def state_decode(codes, scales, signed):
    """Values of an 8-bit state: codes [n], scales [ceil(n / 256)]."""
    codes = np.asarray(codes, dtype=np.int64)
    scale = np.repeat(np.asarray(scales, dtype=np.float64), STATE_BLOCK)[:codes.size]
    if not signed:
        return state_table(256)[codes] * scale
    return state_table(128)[codes % 128] * np.where(codes >= 128, -1.0, 1.0) * scale


def state_encode(x, signed):
    """codes (uint8), scales (fp32) of values x [n], by search among the table's values; halves go to the even code."""
    x = np.asarray(x, dtype=np.float64)
    table = state_table(128 if signed else 256)
    codes, scales = np.zeros(x.size, dtype=np.uint8), np.zeros(-(-x.size // STATE_BLOCK), dtype=np.float32)
    for i in range(scales.size):
        part = x[i * STATE_BLOCK:(i + 1) * STATE_BLOCK]
        scales[i] = np.float32(np.abs(part).max() / table[-1])
        a = np.abs(part) / np.float64(scales[i]) if scales[i] > 0 else np.zeros(part.size)
        mid = (table[1:] + table[:-1]) / 2
        c = np.searchsorted(mid, a, side="left")
        tie = (c < mid.size) & (a == mid[np.minimum(c, mid.size - 1)]) & (c % 2 == 1)
        c = c + tie
        if signed:
            c = np.where(part < 0, c + 128, c)
        elif scales[i] > 0:
            c = np.where(part > 0, np.maximum(c, 1), c)
        codes[i * STATE_BLOCK:(i + 1) * STATE_BLOCK] = c
    return codes, scales


def _philox4x32_10_of(counter, key):
    """philox4x32_10 for arrays: counter of four (uint64 arrays or numbers), key of two numbers; four uint64 arrays."""
    c, k = [np.asarray(x, dtype=np.uint64) for x in counter], [int(x) & U32 for x in key]
    low, half = np.uint64(U32), np.uint64(32)
    for _ in range(10):
        a, b = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(b >> half) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> half) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & U32, (k[1] + 0xBB67AE85) & U32]
    return c


def state_random(n, signed, step, tensor=0):
    """[n]: the shares in (0, 1) by which the states of a call's tensor are rounded in step number `step`.  Element e of a block
    of 256: word e % 4 of the Philox block with counter (32 tensor + e % 128 // 4, block, step, upper bits of the step xor 2^24 times
    the block's) and key 0; first moments take the upper half in the block's first 128 elements and the lower in the others, second
    moments the other."""
    e, block = np.arange(n) % STATE_BLOCK, np.arange(n) // STATE_BLOCK
    last = (step >> 32) ^ ((block >> 32) << 24)
    words = _philox4x32_10_of((32 * tensor + e % 128 // 4, block & U32, np.full(n, step & U32), last), (0, 0))
    word = np.choose(e % 4, words)
    half = np.where((e < 128) == signed, word >> np.uint64(16), word & np.uint64(0xFFFF))
    return (half.astype(np.float64) + 0.5) / 65536


def state_encode_at_random(x, signed, step, tensor=0):
    """As state_encode, but cut off after the random share of the step to the next code is added."""
    x = np.asarray(x, dtype=np.float64)
    table = state_table(128 if signed else 256)
    share = state_random(x.size, signed, step, tensor)
    codes, scales = np.zeros(x.size, dtype=np.uint8), np.zeros(-(-x.size // STATE_BLOCK), dtype=np.float32)
    for i in range(scales.size):
        at = slice(i * STATE_BLOCK, (i + 1) * STATE_BLOCK)
        part = x[at]
        scales[i] = np.float32(np.abs(part).max() / table[-1])
        a = np.abs(part) / np.float64(scales[i]) if scales[i] > 0 else np.zeros(part.size)
        c = np.searchsorted(table, a, side="right") - 1
        up = np.minimum(c + 1, table.size - 1)
        way = np.where(up > c, (a - table[c]) / np.maximum(table[up] - table[c], 1.0), 0.0)
        c = np.where(way + share[at] >= 1, up, c)
        if signed:
            c = np.where(part < 0, c + 128, c)
        elif scales[i] > 0:
            c = np.where(part > 0, np.maximum(c, 1), c)
        codes[at] = c
    return codes, scales


def adamw(w, g, m, v, t, lr, beta1, beta2, eps, decay, scale=1.0):
    """One step on one tensor (t: number of this step): w', m', v'."""
    g = np.asarray(g, dtype=np.float64) * scale
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    step = m / (1 - beta1 ** t) / (np.sqrt(v / (1 - beta2 ** t)) + eps)
    return w - lr * (decay * w + step), m, v


def clip_scale(grads, max_norm):
    """Global norm of a list of gradients, and the factor that clipping puts on them (an fp32 number)."""
    norm = math.sqrt(sum(float((np.asarray(g, dtype=np.float64) ** 2).sum()) for g in grads))
    return norm, float(np.float32(min(1.0, max_norm / (norm + 1e-6)))) if max_norm > 0 else 1.0


# ------------------------------------------------------------------------------ linear operator
def linear_activation(name, z):
    """act(z) and its slope; "none" is z itself."""
    return (z, np.ones_like(z)) if name == "none" else activation(name, z)


def linear_fwd(x, w, bias=None, residual=None, act="none", mask=None):
    z = _select(mask, x) @ np.asarray(w, dtype=np.float64).T
    if bias is not None:
        z = z + bias
    y = linear_activation(act, z)[0]
    if residual is not None:
        y = y + _select(mask, residual)
    return _select(mask, y), z


def linear_bwd(x, w, z, grad_y, act="none", mask=None):
    """grad_x, grad_w, grad_bias and dz."""
    dz = _select(mask, grad_y) * np.where(np.isfinite(z), linear_activation(act, z)[1], 0.0)
    return dz @ np.asarray(w, dtype=np.float64), dz.T @ _select(mask, x), dz.sum(axis=0), dz

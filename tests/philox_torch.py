"""Philox4x32-10 over whole matrices in torch int64 arithmetic, for tests with more elements than the scalar oracle can draw
(tests/test_philox_torch.py pins it to that oracle)."""
import torch

LOW = 0xFFFFFFFF


def _mul(a, m):
    """High and low word of a * m, in 16-bit limbs."""
    lo, hi = a & 0xFFFF, a >> 16
    p = lo * m
    mid = hi * m + (p >> 16)
    return mid >> 16, ((mid & 0xFFFF) << 16) | (p & 0xFFFF)


def dropout_factors(n, h, p, seed, offset, device="cpu", first_row=0):
    """[n, h] float64: 0 where the element is dropped, else 65536 / (65536 - T); rows first_row .. first_row + n."""
    t = int(round(65536.0 * float(torch.tensor(p, dtype=torch.float32))))
    groups = (h + 7) // 8
    seed, offset = int(seed) % (1 << 64), int(offset) % (1 << 64)
    c0 = torch.arange(groups, device=device).repeat(n, 1)
    c1 = torch.arange(first_row, first_row + n, device=device).unsqueeze(1).repeat(1, groups)
    c2, c3 = torch.full_like(c0, offset & LOW), torch.full_like(c0, offset >> 32)
    k0, k1 = seed & LOW, seed >> 32
    for _ in range(10):
        h0, l0 = _mul(c0, 0xD2511F53)
        h1, l1 = _mul(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & LOW, (k1 + 0xBB67AE85) & LOW
    u = torch.stack([half for c in (c0, c1, c2, c3) for half in (c & 0xFFFF, c >> 16)], dim=2).reshape(n, 8 * groups)[:, :h]
    scale = 65536.0 / (65536 - t) if t < 65536 else 0.0
    return (u >= t).double() * scale

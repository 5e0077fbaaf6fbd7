"""Sampling, the linear operator and AdamW write inside their buffers: outputs and workspaces of exactly the stated size between
guard bands (as in test_gpu_guard_bands.py), which the calls leave as they are."""
import numpy as np
import pytest
import torch

import paper_2512_06547_b200 as a3po
from paper_2512_06547_b200.optimizer import AdamW, decode_state
from tests.test_gpu_guard_bands import Guarded

pytestmark = pytest.mark.gpu
DEV = "cuda"
TD = {"f32": torch.float32, "bf16": torch.bfloat16}
CODE = {"f32": a3po.A3PO_F32, "bf16": a3po.A3PO_BF16}


def randn(gen, *shape, dt=torch.float32, k=1.0):
    return torch.from_numpy((gen.standard_normal(shape) * k).astype(np.float32)).to(dt).to(DEV)


# one row, a few rows, K splits, masked tiles, parts of the rows, the FP32 pipes
@pytest.mark.parametrize("dt,n,k,m", [("bf16", 1, 2048, 520), ("bf16", 13, 1000, 40), ("bf16", 100, 1536, 264), ("bf16", 515, 136, 1288),
                                      ("bf16", 4500, 264, 136), ("bf16", 70, 33, 137), ("f32", 131, 65, 193)])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("act", [a3po.A3PO_ACT_NONE, a3po.A3PO_ACT_SILU])
def test_linear(dt, n, k, m, masked, act):
    gen = np.random.default_rng(n + k)
    x, w, gy, res = (randn(gen, *s, dt=TD[dt]) for s in ((n, k), (m, k), (n, m), (n, m)))
    bias = randn(gen, m, dt=TD[dt])
    mask = torch.from_numpy((gen.random(n) < 0.6).astype(np.uint8)).to(DEV) if masked else None
    for y_dt, g_dt in (("f32", "f32"), (dt, dt)):
        G = Guarded()
        y, kept = G.new("y", (n, m), TD[y_dt]), None
        if act != a3po.A3PO_ACT_NONE:
            kept = G.new("kept", (a3po.a3po_linear_kept_bytes(n, m, CODE[dt], act),), torch.uint8)
        status = G.new("status", (1,), torch.int32, 0)
        ws = G.new("ws_fwd", (a3po.a3po_linear_workspace_bytes(n, k, m, CODE[dt], act, masked, False),), torch.uint8)
        a3po.a3po_linear_fwd(x, w, y, ws, bias=bias, residual=res, row_mask=mask, kept=kept, activation=act, status=status)
        G.check("linear_fwd")
        gx, gw, gb = G.new("grad_x", (n, k), TD[dt]), G.new("grad_w", (m, k), TD[g_dt]), G.new("grad_bias", (m,), torch.float32)
        ws_b = G.new("ws_bwd", (a3po.a3po_linear_workspace_bytes(n, k, m, CODE[dt], act, masked, True),), torch.uint8)
        a3po.a3po_linear_bwd(x, w, gy, gx, gw, ws_b, kept=kept, grad_bias=gb, row_mask=mask, activation=act, status=status)
        G.check("linear_bwd")
        assert int(status.item()) == 0
        for t in (y, gx, gw, gb):
            assert torch.isfinite(t.float()).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,v", [(1, 1), (3, 1023), (37, 32003), (5, 151936), (700, 129)])
@pytest.mark.parametrize("filters", [(), ("top_k",), ("top_p",), ("min_p",), ("top_k", "top_p", "min_p")])
def test_sample(dt, n, v, filters):
    gen = np.random.default_rng(n + v)
    logits, u = randn(gen, n, v, dt=TD[dt], k=2.5), torch.from_numpy(gen.random(n).astype(np.float32)).to(DEV)
    per_row = {"top_k": torch.full((n,), 40, dtype=torch.int32, device=DEV), "top_p": torch.full((n,), 0.9, device=DEV),
               "min_p": torch.full((n,), 0.02, device=DEV)}
    G = Guarded()
    token, n_kept = G.new("token", (n,), torch.int32), G.new("n_kept", (n,), torch.int32)
    logp, kept_logp = G.new("logp", (n,), torch.float32), G.new("kept_logp", (n,), torch.float32)
    ws = G.new("ws", (a3po.a3po_sample_workspace_bytes(n, v),), torch.uint8)
    a3po.a3po_sample(logits, u, token, ws, logp=logp, kept_logp=kept_logp, n_kept=n_kept, **{f: per_row[f] for f in filters})
    G.check("sample")
    assert ((token >= 0) & (token < v)).all() and (n_kept >= 1).all() and (logp <= kept_logp + 1e-6).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("wdt,gdt", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
def test_adamw(bits, wdt, gdt):
    gen = np.random.default_rng(bits)
    sizes = [1, 3, 255, 256, 257, 5000, 8192 + 7, 100003] + [33] * 30        # more than the smaller table holds
    G = Guarded()
    state = torch.float32 if bits == 32 else torch.uint8
    new = lambda name, dtype, ns: [G.new(f"{name}{i}", (n,), dtype, 0) for i, n in enumerate(ns)]
    weights, m, v = new("w", TD[wdt], sizes), new("m", state, sizes), new("v", state, sizes)
    for w in weights:
        w.copy_(randn(gen, w.numel()))
    kw = dict(masters=new("master", torch.float32, sizes)) if wdt == "bf16" else {}
    for master, w in zip(kw.get("masters", ()), weights):
        master.copy_(w)
    if bits == 8:
        blocks = [-(-n // 256) for n in sizes]
        kw.update(m_scales=new("ms", torch.float32, blocks), v_scales=new("vs", torch.float32, blocks))
    opt = AdamW(weights, lr=1e-2, max_grad_norm=1.0, state_bits=bits, m=m, v=v, **kw)
    room = G.new("ws", (opt._ws.numel(),), torch.uint8)
    opt._ws = room
    for _ in range(2):
        opt.step([randn(gen, n, dt=TD[gdt]) for n in sizes])
        G.check("adamw")
    if bits == 8:
        for i, n in enumerate(sizes[:8]):
            out = G.new(f"values{i}", (n,), torch.float32)
            decode_state(m[i], opt.m_scales[i], signed=True, out=out)
        G.check("state values")
    assert all(torch.isfinite(w.float()).all() for w in weights)

"""Measured cases of the operators around the LM head: the gated feed-forward block, dropout whose mask is never
stored, the norm before the LM head, and the residual join of the last two (dropout, add, norm in one pass).

Each operator has a plain form here (elementary torch operations in 32 bits, rounded once at the end) and, where
`own` is true, the calls of this package that a training or serving program makes in its place.

Shapes: H = 64, 1536 and 4096 and the row counts are those of the package's tiny, 1.5B-shaped and 8B-shaped batches;
the feed-forward width is a generic 3 H.  `keep` is the share of rows whose mask is set (padding is the rest); rows
that are masked out hold NaN in every input, because nothing of them may be read into a result.

The dropout mask of element (row, col) is a function of (seed, offset, row, col) alone: Philox4x32-10 (Salmon,
Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011) with key = seed and
counter = (col / 8, row, offset low, offset high) gives eight 16-bit numbers u, the (col mod 8)-th of which decides:
kept iff u >= T with T = round(65536 p), and what is kept is scaled by 65536 / (65536 - T).
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one token through a feed-forward block of the 8B-shaped width while serving: streams 302 MB of weights
        dict(name="ffn_one_token", op="ffn_fwd", N=1, H=4096, F=12288, dt="bf16", act="silu", keep=1.0),
        # a few tokens at the 1.5B-shaped width (a small serving batch), the other activation
        dict(name="ffn_13_tokens", op="ffn_fwd", N=13, H=1536, F=4608, dt="bf16", act="gelu_tanh", keep=1.0),
        # the 1.5B-shaped training batch (16 sequences of up to 1024 tokens, right padding masked), there and back
        dict(name="ffn_train_1p5b", op="ffn_train", N=16384, H=1536, F=4608, dt="bf16", act="silu", keep=0.625),
        # a slice of the 8B-shaped training batch without padding, there and back: the largest case
        dict(name="ffn_train_8b", op="ffn_train", N=16384, H=4096, F=12288, dt="bf16", act="silu", keep=1.0),
        # the tiny fp32 configuration that correctness runs use
        dict(name="ffn_train_tiny", op="ffn_train", N=512, H=64, F=192, dt="f32", act="gelu_tanh", keep=0.9),
        # residual stream + dropout over the whole 8B-shaped batch
        dict(name="dropout_8b", op="dropout_fwd", N=131072, H=4096, dt="bf16", p=0.1, residual=True, keep=1.0),
        # gradient through dropout of a ragged packed batch, odd row length, fp32
        dict(name="dropout_bwd_odd", op="dropout_bwd", N=777, H=1537, dt="f32", p=0.3, residual=False, keep=0.95),
        # the final norm of one token while serving
        dict(name="norm_one_token", op="norm_fwd", N=1, H=4096, dt="bf16", kind="rms", keep=1.0),
        # gradient of the final norm over the 8B-shaped batch, padding masked
        dict(name="norm_bwd_8b", op="norm_bwd", N=131072, H=4096, dt="bf16", kind="rms", keep=0.61),
        # gradient of a layer norm with odd row length (rows start at any 2-byte boundary)
        dict(name="norm_bwd_odd", op="norm_bwd", N=5001, H=1003, dt="bf16", kind="layer", keep=0.9),
        # block output + dropout joins the residual stream and is normalised, 1.5B-shaped batch
        dict(name="join_fwd_1p5b", op="join_fwd", N=16384, H=1536, dt="bf16", kind="layer", p=0.1, keep=0.625),
        # and its gradient over the 8B-shaped batch
        dict(name="join_bwd_8b", op="join_bwd", N=65536, H=4096, dt="bf16", kind="rms", p=0.1, keep=1.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["ffn_fwd", "ffn_train", "ffn_train", "dropout_fwd", "dropout_bwd", "norm_fwd", "norm_bwd",
                     "join_fwd", "join_bwd"])
    keep = rng.choice([1.0, rng.uniform(0.3, 1.0)])
    if op.startswith("ffn"):
        act = rng.choice(["silu", "gelu_tanh"])
        if rng.random() < 0.2:      # fp32: small shapes of correctness runs, any size
            return dict(op=op, N=_log_int(rng, 1, 2048), H=rng.randint(3, 256), F=rng.randint(5, 768), dt="f32",
                        act=act, keep=keep)
        n = _log_int(rng, 1, 64) if op == "ffn_fwd" and rng.random() < 0.7 else _log_int(rng, 1, 16384)
        return dict(op=op, N=n, H=8 * rng.randint(32, 512), F=8 * rng.randint(64, 1536), dt="bf16", act=act, keep=keep)
    dt = rng.choice(["bf16", "bf16", "f32"])
    h = rng.choice([_log_int(rng, 16, 8192), 8 * rng.randint(8, 1024)])
    n = max(1, min(_log_int(rng, 1, 131072), (1 << 28) // h))
    case = dict(op=op, N=n, H=h, dt=dt, keep=keep)
    if op.startswith(("dropout", "join")):
        case["p"] = rng.uniform(0.02, 0.6)
    if op.startswith("dropout"):
        case["residual"] = op == "dropout_fwd" and rng.random() < 0.5
    if op.startswith(("norm", "join")):
        case["kind"] = rng.choice(["rms", "layer"])
    return case


def _valid_rows(case):
    return max(1, int(round(case["keep"] * case["N"])))


def work(case):
    n, h, es = _valid_rows(case), case["H"], 4 if case["dt"] == "f32" else 2
    op = case["op"]
    if op == "ffn_fwd":
        f = case["F"]
        return {"bytes": es * (3 * f * h + 2 * n * h), "flops": 6 * n * f * h}
    if op == "ffn_train":   # forward 6, backward 12 n f h; x, grad_y in, y, grad_x out, weights in, their gradients out
        f = case["F"]
        return {"bytes": es * (2 * 3 * f * h + 4 * n * h), "flops": 18 * n * f * h}
    passes = {"dropout_fwd": 3 if case.get("residual") else 2, "dropout_bwd": 2, "norm_fwd": 2, "norm_bwd": 3,
              "join_fwd": 4, "join_bwd": 5}[op]
    return {"bytes": es * passes * n * h, "flops": 8 * n * h}


# ------------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    dev = "cuda" if torch.cuda.is_available() else "cpu"
    gen = torch.Generator(device=dev)
    gen.manual_seed(1000003 * int(seed) + 17)
    n, h, td = case["N"], case["H"], DTYPES[case["dt"]]

    def normal(*shape, scale=1.0):
        out = torch.empty(shape, dtype=td, device=dev)
        slab = max(1, (1 << 27) // max(1, shape[-1]))
        flat = out.view(-1, shape[-1])
        for lo in range(0, flat.shape[0], slab):
            part = flat[lo:lo + slab]
            part.copy_(torch.randn(part.shape, generator=gen, device=dev) * scale)
        return out

    s = {"case": dict(case), "mask": None}
    if _valid_rows(case) < n:
        order = torch.randperm(n, generator=gen, device=dev)
        s["mask"] = torch.zeros(n, dtype=torch.uint8, device=dev)
        s["mask"][order[:_valid_rows(case)]] = 1

    def rows(scale=1.0):
        t = normal(n, h, scale=scale)
        if s["mask"] is not None:
            t.masked_fill_((s["mask"] == 0).unsqueeze(1), float("nan"))
        return t

    op = case["op"]
    if op.startswith("ffn"):
        f = case["F"]
        s["x"] = rows()
        s["w_gate_up"] = normal(2 * f, h, scale=h ** -0.5)
        s["w_down"] = normal(h, f, scale=f ** -0.5)
        if op == "ffn_train":
            s["grad_y"] = rows()
        return s
    if op.startswith(("dropout", "join")):
        s["rng"] = torch.tensor([0x1234567 + 7919 * int(seed), 3 + (int(seed) << 33)], dtype=torch.int64, device=dev)
    if op == "dropout_fwd":
        s["x"] = rows()
        s["residual"] = rows() if case["residual"] else None
    elif op == "dropout_bwd":
        s["grad_y"] = rows()
    else:
        s["gamma"] = (normal(1, h, scale=0.1) + 1).view(h).to(td)
        s["beta"] = normal(1, h, scale=0.1).view(h) if case["kind"] == "layer" else None
        if op.endswith("fwd"):
            s["x"] = rows()
            s["residual"] = rows(2.0) if op == "join_fwd" else None
        else:
            s["x"] = rows(2.0)                       # what was normalised, and its statistics as the forward left them
            s["grad_y"] = rows()
            s["grad_r"] = rows() if op == "join_bwd" else None
            x = s["x"].float()
            s["mean"] = x.mean(dim=1) if case["kind"] == "layer" else None
            if case["kind"] == "layer":
                x = x - s["mean"].unsqueeze(1)
            s["rstd"] = torch.rsqrt(x.square().mean(dim=1) + EPS)
            if s["mask"] is not None:
                s["rstd"].masked_fill_(s["mask"] == 0, 0.0)
                if s["mean"] is not None:
                    s["mean"].masked_fill_(s["mask"] == 0, 0.0)
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _valid(s, t):
    """`t` in 32 bits with the rows that are masked out selected away."""
    t = t.float()
    return t if s["mask"] is None else torch.where((s["mask"] != 0).unsqueeze(1), t, torch.zeros((), device=t.device))


def _mulhilo(a, m):
    """High and low 32 bits of a * m for int64 tensors holding 32-bit values (16-bit limbs: nothing overflows)."""
    lo, hi = a & 0xFFFF, a >> 16
    p0, p1 = lo * m, hi * m                          # below 2^48
    mid = p1 + (p0 >> 16)
    return mid >> 16, ((mid & 0xFFFF) << 16) | (p0 & 0xFFFF)


def _kept_scale(s):
    """1 / (1 - p) where the element is kept, 0 where it is dropped: [N, H] in 32 bits."""
    case, rng = s["case"], s["rng"]
    n, h = case["N"], case["H"]
    threshold = int(round(65536 * float(np.float32(case["p"]))))
    groups = (h + 7) // 8
    dev = rng.device
    c0 = torch.arange(groups, device=dev).view(1, groups).expand(n, groups)
    c1 = torch.arange(n, device=dev).view(n, 1).expand(n, groups)
    c2 = (rng[1] & 0xFFFFFFFF).expand(n, groups)
    c3 = ((rng[1] >> 32) & 0xFFFFFFFF).expand(n, groups)
    k0, k1 = rng[0] & 0xFFFFFFFF, (rng[0] >> 32) & 0xFFFFFFFF
    for _ in range(10):
        h0, l0 = _mulhilo(c0, 0xD2511F53)
        h1, l1 = _mulhilo(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    u = torch.stack([c0 & 0xFFFF, c0 >> 16, c1 & 0xFFFF, c1 >> 16, c2 & 0xFFFF, c2 >> 16, c3 & 0xFFFF, c3 >> 16],
                    dim=2).view(n, groups * 8)[:, :h]
    scale = 65536.0 / (65536 - threshold) if threshold < 65536 else 0.0
    return (u >= threshold).float() * scale


def _act_and_slope(name, g):
    if name == "silu":
        sg = 1 / (1 + torch.exp(-g))
        return g * sg, sg * (1 + g * (1 - sg))
    c = 2 * math.sqrt(2 / math.pi)
    sg = 1 / (1 + torch.exp(-c * (g + 0.044715 * g * g * g)))
    return g * sg, sg + g * sg * (1 - sg) * c * (1 + 3 * 0.044715 * g * g)


def _plain_ffn(s):
    case = s["case"]
    f, td = case["F"], DTYPES[case["dt"]]
    x, wgu, wd = _valid(s, s["x"]), s["w_gate_up"].float(), s["w_down"].float()
    g, u = x @ wgu[:f].t(), x @ wgu[f:].t()
    a, slope = _act_and_slope(case["act"], g)
    hid = a * u
    out = {"y": (hid @ wd.t()).to(td)}
    if case["op"] == "ffn_train":
        gy = _valid(s, s["grad_y"])
        dh = gy @ wd
        out["grad_w_down"] = (gy.t() @ hid).to(td)
        dgu = torch.cat([dh * u * slope, dh * a], dim=1)
        out["grad_x"] = (dgu @ wgu).to(td)
        out["grad_w_gate_up"] = (dgu.t() @ x).to(td)
    return out


def _plain_norm_fwd(s, x):
    """y of the stored rows `x`, and the statistics."""
    case, out = s["case"], {}
    if case["kind"] == "layer":
        out["mean"] = x.mean(dim=1)
        x = x - out["mean"].unsqueeze(1)
    out["rstd"] = torch.rsqrt(x.square().mean(dim=1) + EPS)
    y = x * out["rstd"].unsqueeze(1) * s["gamma"].float()
    if s["beta"] is not None:
        y = y + s["beta"].float()
    if s["mask"] is not None:
        keep = s["mask"] != 0
        y = y * keep.unsqueeze(1)
        out["rstd"] = out["rstd"] * keep
    out["y"] = y.to(DTYPES[case["dt"]])
    return out


def _plain_norm_bwd(s):
    """Gradient of the normalised rows in 32 bits, and those of gamma and beta."""
    layer = s["case"]["kind"] == "layer"
    x, gy, rstd = _valid(s, s["x"]), _valid(s, s["grad_y"]), s["rstd"].unsqueeze(1)
    xhat = (x - s["mean"].unsqueeze(1)) * rstd if layer else x * rstd
    out = {"grad_gamma": (gy * xhat).sum(dim=0)}
    if layer:
        out["grad_beta"] = gy.sum(dim=0)
    gx = gy * s["gamma"].float()
    inner = (gx * xhat).mean(dim=1, keepdim=True)
    if layer:
        gx = gx - gx.mean(dim=1, keepdim=True)
    return (gx - xhat * inner) * rstd, out


def _plain(s):
    case = s["case"]
    op, td = case["op"], DTYPES[case["dt"]]
    if op.startswith("ffn"):
        return _plain_ffn(s)
    if op == "dropout_fwd":
        y = _valid(s, s["x"]) * _kept_scale(s)
        if s["residual"] is not None:
            y = y + _valid(s, s["residual"])
        return {"y": y.to(td)}
    if op == "dropout_bwd":
        return {"grad_x": (_valid(s, s["grad_y"]) * _kept_scale(s)).to(td)}
    if op == "norm_fwd":
        return _plain_norm_fwd(s, _valid(s, s["x"]))
    if op == "join_fwd":
        r = (_valid(s, s["x"]) * _kept_scale(s) + _valid(s, s["residual"])).to(td)
        return {"r": r, **_plain_norm_fwd(s, r.float())}
    gx, out = _plain_norm_bwd(s)
    if op == "join_bwd":
        gr = gx + _valid(s, s["grad_r"])
        return {"grad_residual": gr.to(td), "grad_x": (gr * _kept_scale(s)).to(td), **out}
    return {"grad_x": gx.to(td), **out}


# ------------------------------------------------------------------------------------------------ the package's calls
def _own(s):
    import paper_2512_06547_b200 as a3po
    case = s["case"]
    op, n, h = case["op"], case["N"], case["H"]
    if "calls" not in s:          # a program's own buffers, made once for its shapes: outputs, kept values, scratch
        dt = a3po.A3PO_F32 if case["dt"] == "f32" else a3po.A3PO_BF16
        masked = s["mask"] is not None
        out, dev, td = {}, s["mask" if masked else "x" if "x" in s else "grad_y"].device, DTYPES[case["dt"]]
        new = lambda *shape, dtype=td: torch.empty(shape, dtype=dtype, device=dev)  # noqa: E731
        ws = kept = None
        if op.startswith("ffn"):
            f, train = case["F"], op == "ffn_train"
            act = a3po.A3PO_ACT_SILU if case["act"] == "silu" else a3po.A3PO_ACT_GELU_TANH
            ws = a3po.new_workspace(max(a3po.a3po_gated_ffn_workspace_bytes(n, h, f, dt, masked, bwd)
                                        for bwd in ((False, True) if train else (False,))), dev)
            out["y"] = new(n, h)
            if train:
                kept = a3po.new_workspace(a3po.a3po_gated_ffn_kept_bytes(n, f, dt), dev)
                out.update(grad_x=new(n, h), grad_w_gate_up=new(2 * f, h), grad_w_down=new(h, f))
            s["act"] = act
        elif op.startswith("dropout"):
            out["y" if op == "dropout_fwd" else "grad_x"] = new(n, h)
        else:
            s["kind"] = a3po.A3PO_NORM_LAYER if case["kind"] == "layer" else a3po.A3PO_NORM_RMS
            layer = case["kind"] == "layer"
            if op.endswith("fwd"):
                out["y"] = new(n, h)
                out["rstd"] = new(n, dtype=torch.float32)
                if layer:
                    out["mean"] = new(n, dtype=torch.float32)
                if op == "join_fwd":
                    out["r"] = new(n, h)
            else:
                ws = a3po.new_workspace(a3po.a3po_norm_bwd_workspace_bytes(n, h), dev)
                out["grad_x"] = new(n, h)
                out["grad_gamma"] = new(h, dtype=torch.float32)
                if layer:
                    out["grad_beta"] = new(h, dtype=torch.float32)
                if op == "join_bwd":
                    out["grad_residual"] = new(n, h)
        s["calls"] = (out, ws, kept)
    out, ws, kept = s["calls"]
    mask = s["mask"]
    if op.startswith("ffn"):
        a3po.a3po_gated_ffn_fwd(s["x"], s["w_gate_up"], s["w_down"], out["y"], ws, row_mask=mask, kept=kept,
                                activation=s["act"])
        if op == "ffn_train":
            a3po.a3po_gated_ffn_bwd(s["x"], s["w_gate_up"], s["w_down"], kept, s["grad_y"], out["grad_x"],
                                    out["grad_w_gate_up"], out["grad_w_down"], ws, row_mask=mask, activation=s["act"])
    elif op == "dropout_fwd":
        a3po.a3po_dropout_fwd(s["x"], case["p"], s["rng"], out["y"], residual=s["residual"], row_mask=mask)
    elif op == "dropout_bwd":
        a3po.a3po_dropout_bwd(s["grad_y"], case["p"], s["rng"], out["grad_x"], row_mask=mask)
    elif op == "norm_fwd":
        a3po.a3po_norm_fwd(s["x"], s["gamma"], out["y"], out["rstd"], kind=s["kind"], beta=s["beta"],
                           mean=out.get("mean"), eps=EPS, row_mask=mask)
    elif op == "norm_bwd":
        a3po.a3po_norm_bwd(s["x"], s["gamma"], s["rstd"], s["grad_y"], out["grad_x"], out["grad_gamma"], ws,
                           kind=s["kind"], mean=s["mean"], grad_beta=out.get("grad_beta"), row_mask=mask)
    elif op == "join_fwd":
        a3po.a3po_dropout_norm_fwd(s["x"], s["residual"], case["p"], s["rng"], s["gamma"], out["r"], out["y"],
                                   out["rstd"], kind=s["kind"], beta=s["beta"], mean=out.get("mean"), eps=EPS,
                                   row_mask=mask)
    else:
        a3po.a3po_dropout_norm_bwd(s["x"], case["p"], s["rng"], s["gamma"], s["rstd"], s["grad_y"],
                                   out["grad_residual"], out["grad_x"], out["grad_gamma"], ws, kind=s["kind"],
                                   mean=s["mean"], grad_r=s["grad_r"], grad_beta=out.get("grad_beta"), row_mask=mask)
    return out


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------ in 64 bits
def _exact_kept(case, rng):
    """The dropout factors from 64-bit unsigned products, [N, H] float64."""
    n, h = case["N"], case["H"]
    seed, offset = (int(v) % (1 << 64) for v in rng.tolist())
    low = np.uint64(0xFFFFFFFF)
    groups = -(-h // 8)
    ctr = [np.broadcast_to(np.arange(groups, dtype=np.uint64), (n, groups)),
           np.broadcast_to(np.arange(n, dtype=np.uint64)[:, None], (n, groups)),
           np.full((n, groups), offset & 0xFFFFFFFF, dtype=np.uint64), np.full((n, groups), offset >> 32, dtype=np.uint64)]
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        a, b = ctr[0] * np.uint64(0xD2511F53), ctr[2] * np.uint64(0xCD9E8D57)
        ctr = [(b >> np.uint64(32)) ^ ctr[1] ^ np.uint64(key[0]), b & low,
               (a >> np.uint64(32)) ^ ctr[3] ^ np.uint64(key[1]), a & low]
        key = [(key[0] + 0x9E3779B9) % (1 << 32), (key[1] + 0xBB67AE85) % (1 << 32)]
    words = np.stack(ctr, axis=2).astype("<u4")                       # [N, groups, 4]
    halves = words.view("<u2").reshape(n, groups * 8)[:, :h]          # low half first
    threshold = int(np.rint(65536 * np.float64(np.float32(case["p"]))))
    factor = 65536.0 / (65536 - threshold) if threshold < 65536 else 0.0
    return np.where(halves >= threshold, factor, 0.0)


def exact(case, seed):
    """The same outputs by differentiating the definition in 64 bits; None where the mask's 64-bit arithmetic on the
    host would take too long."""
    op, n, h = case["op"], case["N"], case["H"]
    if op.startswith(("dropout", "join")) and n * h > (1 << 25):
        return None
    s = prepare(case, seed)
    keep = torch.ones(n, 1, dtype=torch.bool, device=(s.get("x") if "x" in s else s["grad_y"]).device)
    if s["mask"] is not None:
        keep = (s["mask"] != 0).unsqueeze(1)

    def wide(t):
        return t.double().masked_fill_(~keep, 0.0) if t.dim() == 2 and t.shape[0] == n and t.shape[1] == h else t.double()

    def leaf(t):
        return wide(t).requires_grad_(True)

    if op.startswith("ffn"):
        f = case["F"]
        train = op == "ffn_train"
        x = torch.where(keep, s["x"], torch.zeros_like(s["x"])).double().requires_grad_(train)
        wgu, wd = s["w_gate_up"].double().requires_grad_(train), s["w_down"].double().requires_grad_(train)
        gu = torch.nn.functional.linear(x, wgu)
        g, u = gu.split(f, dim=1)
        a = (torch.nn.functional.silu(g) if case["act"] == "silu"
             else torch.nn.functional.gelu(g, approximate="tanh"))
        y = torch.nn.functional.linear(a * u, wd)
        out = {"y": y.detach()}
        if train:
            gy = torch.where(keep, s["grad_y"], torch.zeros_like(s["grad_y"])).double()
            out["grad_x"], out["grad_w_gate_up"], out["grad_w_down"] = torch.autograd.grad(y, (x, wgu, wd), gy)
        return out
    factor = torch.from_numpy(_exact_kept(case, s["rng"])).to(keep.device) if "rng" in s else None
    if op == "dropout_fwd":
        y = wide(s["x"]) * factor
        return {"y": y if s["residual"] is None else y + wide(s["residual"])}
    if op == "dropout_bwd":
        return {"grad_x": wide(s["grad_y"]) * factor}

    def norm(v, gamma, beta):
        mean = v.mean(dim=1, keepdim=True) if case["kind"] == "layer" else torch.zeros_like(v[:, :1])
        rstd = 1 / ((v - mean).pow(2).mean(dim=1, keepdim=True) + EPS).sqrt()
        y = (v - mean) * rstd * gamma
        return torch.where(keep, y if beta is None else y + beta, torch.zeros_like(y)), mean, rstd * keep

    gamma = s["gamma"].double()
    beta = s["beta"].double() if s["beta"] is not None else None
    if op.endswith("fwd"):
        out = {}
        v = wide(s["x"])
        if op == "join_fwd":          # the norm is that of the stored rows
            out["r"] = v * factor + wide(s["residual"])
            v = out["r"].float().to(DTYPES[case["dt"]]).double()
        y, mean, rstd = norm(v, gamma, beta)
        out.update(y=y, rstd=rstd.squeeze(1))
        if case["kind"] == "layer":
            out["mean"] = mean.squeeze(1)
        return out
    x = leaf(s["x"])
    gamma.requires_grad_(True)
    wanted = [x, gamma]
    if beta is not None:
        beta.requires_grad_(True)
        wanted.append(beta)
    y, _, _ = norm(x, gamma, beta)
    grads = torch.autograd.grad(y, wanted, wide(s["grad_y"]))
    out = {"grad_gamma": grads[1]}
    if beta is not None:
        out["grad_beta"] = grads[2]
    if op == "join_bwd":
        out["grad_residual"] = grads[0] + wide(s["grad_r"])
        out["grad_x"] = out["grad_residual"] * factor
    else:
        out["grad_x"] = grads[0]
    return out

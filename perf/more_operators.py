"""Measured cases of the operators that close the loop around the policy's tail: the matrix product with bias,
activation and residual (logits of the next token, projections onto the residual stream), the sampling of a token from
logits with the log-probabilities that the loss takes as behaviour policy, and the AdamW step with its gradient norm.

Each operator has a plain form here (elementary torch operations, in 32 bits and in 64 where the outcome hangs on a border:
sums that a random number or a share of the mass is compared with, values that are rounded to 8 bits) and, where `own`
is true, the calls of this package that a training or serving program makes in its place.

Shapes: H = 64, 1536 and 4096, V = 151936 and the row counts are those of the package's tiny, 1.5B-shaped and 8B-shaped
batches; the inner width is a generic 3 H.  `keep` is the share of rows whose mask is set; rows that are masked out hold NaN,
because nothing of them may be read into a result.

Sampling of a row, with l its logits (NaN counts as -inf) and t its temperature (t <= 0: greedy, and t = 1 below):
    w_i = exp((l_i - max l) / t);  tokens are ranked by l, ties by the lower index first
    top-k   keeps the k first (k <= 0: all);
    top-p   keeps of those the shortest run of ranks whose weight is at least top_p times their total (top_p >= 1: all);
    min-p   keeps of those the ones with w_i >= min_p (min_p <= 0: all);   the first rank is always kept, greedy keeps it alone
    token = the first kept i in index order at which the running sum of kept weights exceeds u times their total
    logp = log(w_token / sum of all w), kept_logp = log(w_token / sum of kept w), n_kept = kept tokens with l > -inf
A row that is masked out or has no logit above -inf gives token -1, and 0 for the rest.

AdamW: s = min(1, max_norm / (norm + 1e-6)) with the norm over all gradients, g = s grad,
    m' = b1 m + (1 - b1) g,  v' = b2 v + (1 - b2) g^2,  w' = w - lr (decay w + (m' / (1 - b1^t)) / (sqrt(v' / (1 - b2^t)) + eps))
States of 8 bits hold blocks of 256 elements: q(code) * scale with q(c) = c below 8, else (8 + c mod 8) 2^(c div 8 - 1); the
first moment has a sign and codes up to 127, scale = max|m'| / q(127); the second codes up to 255, scale = max v' / q(255),
and a value above 0 is not rounded to 0.  Rounding is to the nearest q, halves to the even code.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BLOCK = 256
BETA1, BETA2, ADAM_EPS = 0.9, 0.95, 1e-8


# ------------------------------------------------------------------------------------------------ cases
def listed():
    tail_1p5b = "%d,%d,%d,1536,1536" % (151936 * 1536, 2 * 4608 * 1536, 1536 * 4608)
    return [
        # logits of one token while serving, 8B-shaped head, kept in fp32 for the sampler: streams 1.2 GB of weights
        dict(name="logits_one_token", op="linear_fwd", N=1, K=4096, M=151936, dt="bf16", out="f32", act="none", bias=False,
             residual=False, keep=1.0),
        # a small serving batch through a projection back onto the residual stream, 1.5B-shaped
        dict(name="linear_13_tokens", op="linear_fwd", N=13, K=4608, M=1536, dt="bf16", out="bf16", act="gelu_tanh",
             bias=True, residual=True, keep=1.0),
        # the 1.5B-shaped training batch (right padding masked) through a biased projection with an activation, there and back
        dict(name="linear_train_1p5b", op="linear_train", N=16384, K=1536, M=4608, dt="bf16", grads="bf16", act="silu",
             bias=True, residual=False, keep=0.625),
        # a slice of the 8B-shaped batch through an output projection onto the residual stream, fp32 weight gradients
        dict(name="linear_train_8b", op="linear_train", N=16384, K=4096, M=4096, dt="bf16", grads="f32", act="none",
             bias=False, residual=True, keep=1.0),
        # the fp32 correctness configuration at odd sizes
        dict(name="linear_train_odd", op="linear_train", N=509, K=65, M=193, dt="f32", grads="f32", act="gelu_tanh",
             bias=True, residual=True, keep=0.9),
        # one token from fp32 logits: the smallest call of a serving loop
        dict(name="sample_one", op="sample", N=1, V=151936, dt="f32", filters="none", sigma=2.5, keep=1.0),
        # a serving batch in which every request has its own settings, some greedy
        dict(name="sample_serve", op="sample", N=64, V=151936, dt="bf16", filters="mixed", sigma=2.5, keep=1.0),
        # rollouts of a training step: the policy as it is, temperature alone
        dict(name="sample_rollout", op="sample", N=2048, V=151936, dt="bf16", filters="none", sigma=1.5, keep=1.0),
        # an odd vocabulary in fp32, every filter on, finished rows masked, banned tokens at -inf
        dict(name="sample_odd", op="sample", N=37, V=32003, dt="f32", filters="all", sigma=3.0, keep=0.8),
        # weights of the 1.5B-shaped tail: fp32 masters, bf16 copies, fp32 gradients, states in 32 bits
        dict(name="adamw_1p5b", op="adamw", sizes=tail_1p5b, wdt="bf16", gdt="f32", bits=32, clip=1.0),
        # the same with states in 8 bits
        dict(name="adamw_1p5b_8bit", op="adamw", sizes=tail_1p5b, wdt="bf16", gdt="f32", bits=8, clip=1.0),
        # the tiny fp32 tail
        dict(name="adamw_tiny", op="adamw", sizes="64000,24576,12288,64,64", wdt="f32", gdt="f32", bits=32, clip=1.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear_fwd", "linear_train", "linear_train", "sample", "sample", "adamw"])
    keep = rng.choice([1.0, rng.uniform(0.3, 1.0)])
    if op.startswith("linear"):
        case = dict(op=op, act=rng.choice(["none", "silu", "gelu_tanh"]), bias=rng.random() < 0.5,
                    residual=rng.random() < 0.5, keep=keep)
        if rng.random() < 0.2:      # fp32: small shapes of correctness runs, any size
            case.update(N=_log_int(rng, 1, 2048), K=rng.randint(3, 512), M=rng.randint(5, 768), dt="f32")
        else:
            k, m = 8 * rng.randint(16, 512), 8 * _log_int(rng, 16, 1536)
            few = op == "linear_fwd" and rng.random() < 0.7
            n = _log_int(rng, 1, 64) if few else _log_int(rng, 1, 16384)
            case.update(N=min(n, (1 << 38) // (k * m)), K=k, M=m, dt="bf16")
        if op == "linear_fwd":
            case["out"] = "f32" if case["dt"] == "f32" or rng.random() < 0.3 else "bf16"
        else:   # bf16: the gradient that goes through an activation is itself an operand in 16 bits
            case["grads"] = "f32" if case["dt"] == "f32" or case["act"] == "none" and rng.random() < 0.5 else "bf16"
        return case
    if op == "sample":
        v = _log_int(rng, 32, 200000)
        n = max(1, min(_log_int(rng, 1, 2048), (1 << 27) // v))
        return dict(op=op, N=n, V=v, dt=rng.choice(["bf16", "f32"]), sigma=rng.uniform(1.0, 4.0), keep=keep,
                    filters=rng.choice(["none", "top_k", "top_p", "min_p", "mixed", "all"]))
    sizes = ",".join(str(_log_int(rng, 3, 1 << 22)) for _ in range(rng.randint(1, 40)))
    return dict(op=op, sizes=sizes, wdt=rng.choice(["bf16", "f32"]), gdt=rng.choice(["bf16", "f32"]),
                bits=rng.choice([8, 32]), clip=rng.choice([0.0, 1.0]))


def _valid_rows(case):
    return max(1, int(round(case["keep"] * case["N"])))


def work(case):
    if case["op"] == "adamw":   # weights (and bf16 copies), gradients, states with a scale each per 256 elements
        n = sum(int(s) for s in case["sizes"].split(","))
        per = 8 + (2 if case["wdt"] == "bf16" else 0) + (4 if case["gdt"] == "f32" else 2)
        per += 16 if case["bits"] == 32 else 4 + 16 / BLOCK
        return {"bytes": int(n * per), "flops": 16 * n}
    n, es = _valid_rows(case), 4 if case["dt"] == "f32" else 2
    if case["op"] == "sample":
        return {"bytes": es * n * case["V"], "flops": 4 * n * case["V"]}
    k, m = case["K"], case["M"]
    side = es * (m * case["bias"] + n * m * case["residual"])
    if case["op"] == "linear_fwd":
        return {"bytes": es * (k * m + n * k) + side + (4 if case["out"] == "f32" else 2) * n * m, "flops": 2 * n * k * m}
    gs = 4 if case["grads"] == "f32" else 2   # x, y, grad_y, grad_x, the weights and their gradients
    return {"bytes": es * (2 * n * k + 2 * n * m + k * m) + side + gs * k * m, "flops": 6 * n * k * m}


# ------------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    dev = "cuda" if torch.cuda.is_available() else "cpu"
    gen = torch.Generator(device=dev)
    gen.manual_seed(1000003 * int(seed) + 29)
    s = {"case": dict(case), "mask": None}

    def normal(shape, td, scale=1.0):
        out = torch.empty(shape, dtype=td, device=dev)
        flat = out.view(-1)
        for lo in range(0, flat.numel(), 1 << 27):
            part = flat[lo:lo + (1 << 27)]
            part.copy_(torch.randn(part.shape, generator=gen, device=dev) * scale)
        return out

    if case["op"] == "adamw":
        sizes = [int(x) for x in case["sizes"].split(",")]
        blocks = [-(-n // BLOCK) for n in sizes]       # a trainer's flat buffers: every tensor starts on a block
        nb = sum(blocks)
        real = torch.zeros(nb, BLOCK, device=dev)      # 1 where a tensor has an element
        starts = [sum(blocks[:i]) for i in range(len(sizes))]
        for at, n in zip(starts, sizes):
            real.view(-1)[at * BLOCK:at * BLOCK + n] = 1
        td, f32 = DTYPES[case["wdt"]], torch.float32
        s["sizes"], s["starts"], s["real"] = sizes, starts, real
        s["decays"] = [0.1 if n > 4096 else 0.0 for n in sizes]   # norms and biases do not decay
        s["master"] = normal((nb, BLOCK), f32, 0.02).mul_(real)
        s["weight"] = s["master"].to(td) if td != f32 else s["master"]
        s["grad"] = normal((nb, BLOCK), DTYPES[case["gdt"]], 1e-3).mul_(real)
        s["grad"].mul_(torch.exp(torch.randn(nb, 1, generator=gen, device=dev)).to(s["grad"].dtype))   # rows of unlike size
        s["lr"] = torch.full((1,), 3e-4, device=dev)
        s["step"] = torch.full((1,), 20, dtype=torch.int64, device=dev)
        # states as some steps before left them
        s["m"] = normal((nb, BLOCK), f32, 4e-4).mul_(real)
        s["v"] = normal((nb, BLOCK), f32, 1e-3).square_().mul_(real)
        if case["bits"] == 8:
            s["m"], s["m_scale"] = _to_8bit(s["m"].double(), True)
            s["v"], s["v_scale"] = _to_8bit(s["v"].double(), False)
        return s

    n = case["N"]
    if _valid_rows(case) < n:
        order = torch.randperm(n, generator=gen, device=dev)
        s["mask"] = torch.zeros(n, dtype=torch.uint8, device=dev)
        s["mask"][order[:_valid_rows(case)]] = 1
    hole = None if s["mask"] is None else (s["mask"] == 0).unsqueeze(1)

    def rows(width, td, scale=1.0):
        t = normal((n, width), td, scale)
        return t if hole is None else t.masked_fill_(hole, float("nan"))

    td = DTYPES[case["dt"]]
    if case["op"].startswith("linear"):
        k, m = case["K"], case["M"]
        s["x"], s["w"] = rows(k, td), normal((m, k), td, k ** -0.5)
        s["bias"] = normal((m,), td, 0.3) if case["bias"] else None
        s["residual"] = rows(m, td, 2.0) if case["residual"] else None
        s["grad_y"] = rows(m, td) if case["op"] == "linear_train" else None
        return s

    v, how = case["V"], case["filters"]
    s["logits"] = rows(v, td, case["sigma"])
    # some tokens of each row stand out, as after training
    at = torch.randint(0, v, (n, 4), generator=gen, device=dev)
    lift = torch.rand(n, 4, generator=gen, device=dev) * 8 + 2
    s["logits"].scatter_add_(1, at, lift.to(td))
    if how == "all":                                   # banned tokens
        for lo in range(0, n, 64):
            ban = torch.rand(s["logits"][lo:lo + 64].shape, generator=gen, device=dev) < 0.2
            s["logits"][lo:lo + 64].masked_fill_(ban, float("-inf"))
    s["u"] = torch.rand(n, generator=gen, device=dev)

    def pick(values, dtype):
        return torch.tensor(values, dtype=dtype, device=dev)[torch.randint(0, len(values), (n,), generator=gen, device=dev)]

    mixed = how == "mixed"
    s["temperature"] = s["top_k"] = s["top_p"] = s["min_p"] = None
    if how != "none":
        s["temperature"] = pick([0.0, 0.6, 0.8, 1.0] if mixed else [0.6, 0.7, 1.0], torch.float32)
    if how in ("top_k", "all", "mixed"):
        s["top_k"] = pick([0, 20, 50] if mixed else [1, 20, 50, 1000], torch.int32)
    if how in ("top_p", "all", "mixed"):
        s["top_p"] = pick([0.9, 0.95, 1.0], torch.float32)
    if how in ("min_p", "all", "mixed"):
        s["min_p"] = pick([0.0, 0.05] if mixed else [0.02, 0.05, 0.1], torch.float32)
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _plain_act(name, z):
    """The activation and its slope."""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "silu":
        sg = 1 / (1 + torch.exp(-z))
        return z * sg, sg * (1 + z * (1 - sg))
    c = 2 * math.sqrt(2 / math.pi)
    sg = 1 / (1 + torch.exp(-c * (z + 0.044715 * z * z * z)))
    return z * sg, sg + z * sg * (1 - sg) * c * (1 + 3 * 0.044715 * z * z)


def _plain_linear(s):
    case, td = s["case"], DTYPES[s["case"]["dt"]]

    def valid(t):
        t = t.float()
        return t if s["mask"] is None else torch.where((s["mask"] != 0).unsqueeze(1), t, torch.zeros((), device=t.device))

    x, w = valid(s["x"]), s["w"].float()
    z = x @ w.t()
    if s["bias"] is not None:
        z = z + s["bias"].float()
    y, slope = _plain_act(case["act"], z)
    if s["residual"] is not None:
        y = y + valid(s["residual"])
    if s["mask"] is not None:
        y = y * (s["mask"] != 0).unsqueeze(1)
    if case["op"] == "linear_fwd":
        return {"y": y.to(DTYPES[case["out"]])}
    gd = DTYPES[case["grads"]]
    dz = valid(s["grad_y"]) * slope
    out = {"y": y.to(td), "grad_x": (dz @ w).to(td), "grad_w": (dz.t() @ x).to(gd)}
    if s["bias"] is not None:
        out["grad_bias"] = dz.sum(dim=0)
    return out


def _plain_sample(s):
    logits = s["logits"]
    n, v = logits.shape
    dev = logits.device
    low = torch.full((), float("-inf"), dtype=torch.float64, device=dev)
    l = torch.where(torch.isnan(logits), low, logits.double())
    if s["mask"] is not None:
        l = torch.where((s["mask"] != 0).unsqueeze(1), l, low)
    temp = torch.ones(n, device=dev) if s["temperature"] is None else s["temperature"]
    greedy = (temp <= 0).unsqueeze(1)
    t = torch.where(temp > 0, temp, torch.ones_like(temp)).double().unsqueeze(1)
    top = l.max(dim=1, keepdim=True).values
    live = top > low
    w = torch.where(l == top, torch.ones_like(l), torch.exp((l - top) / t))
    w = torch.where(live & (l > low), w, torch.zeros_like(w))
    if s["temperature"] is None and s["top_k"] is None and s["top_p"] is None and s["min_p"] is None:
        kept = w                                        # weights of kept tokens
        n_kept = ((l > low) & live).sum(dim=1)
    else:
        _, order = torch.sort(l, dim=1, descending=True, stable=True)
        ranked, rank = w.gather(1, order), torch.arange(v, device=dev).unsqueeze(0)
        on = torch.where(greedy, rank == 0, l.gather(1, order) > low)
        if s["top_k"] is not None:
            k = s["top_k"].unsqueeze(1)
            on = on & ((rank < k) | (k <= 0))
        if s["top_p"] is not None:
            p = s["top_p"].double().unsqueeze(1)
            run = torch.cumsum(ranked * on, dim=1)
            before = torch.cat([torch.zeros(n, 1, dtype=run.dtype, device=dev), run[:, :-1]], dim=1)
            on = on & ((before < p * run[:, -1:]) | (p >= 1) | (rank == 0))
        if s["min_p"] is not None:
            on = on & ((ranked >= s["min_p"].double().unsqueeze(1)) | (rank == 0))
        on = on & live
        n_kept = on.sum(dim=1)
        kept = torch.zeros_like(w).scatter_(1, order, ranked * on)
    run = torch.cumsum(kept, dim=1)
    total = run[:, -1:].contiguous()
    token = torch.searchsorted(run, s["u"].double().unsqueeze(1) * total, right=True).clamp_(max=v - 1)
    live = live.squeeze(1)

    def out(x, dead):
        return torch.where(live, x, torch.full_like(x, dead))

    mine = torch.where(l.gather(1, token) == top, torch.zeros_like(top), (l.gather(1, token) - top) / t)
    return {"token": out(token.squeeze(1), -1).to(torch.int32),
            "logp": out((mine - w.sum(dim=1, keepdim=True).log()).squeeze(1), 0).float(),
            "kept_logp": out((mine - total.log()).squeeze(1), 0).float(), "n_kept": out(n_kept, 0).to(torch.int32)}


def _q(code):
    """What a code of 8 bits (0 .. 255) stands for, before the scale."""
    return torch.where(code < 8, code, torch.bitwise_left_shift(8 + code % 8, (code // 8 - 1).clamp_min(0)))


def _to_8bit(x, signed):
    """Codes (uint8; bit 7 is the sign where there is one) and fp32 scales of rows of 256 values in 64 bits."""
    top = 15.0 * 2 ** (14 if signed else 30)
    scale = (x.abs().amax(dim=1, keepdim=True) / top).float()
    inv = torch.where(scale > 0, 1 / scale.double(), torch.zeros_like(x[:, :1]))
    a = x.abs() * inv
    e = (torch.frexp(a)[1] - 4).clamp_min(0)            # 8 2^e <= a < 16 2^e, or e = 0
    c = torch.round(a / torch.bitwise_left_shift(torch.ones_like(e), e)) + 8 * e    # 8 .. 16 in steps of one: 16 is the next power's first
    if not signed:
        c = torch.where((x > 0) & (inv > 0), c.clamp_min(1), c)
    c = c.clamp_max(127 if signed else 255).to(torch.uint8)
    return (torch.where(x < 0, c + 128, c) if signed else c), scale.squeeze(1)


def _from_8bit(code, scale, signed):
    c = code.to(torch.int64)
    q = _q(c % 128) * torch.where(c >= 128, -1, 1) if signed else _q(c)
    return q.double() * scale.double().unsqueeze(1)


def _plain_adamw(s):
    case = s["case"]
    eight = case["bits"] == 8
    g = s["grad"].double()
    norm = g.square().sum().sqrt()
    out = {"grad_norm": norm.float().reshape(1)}
    coef = torch.clamp(case["clip"] / (norm + 1e-6), max=1.0).float() if case["clip"] > 0 else torch.ones((), device=g.device)
    s["step"] += 1
    t = s["step"].double()
    bc1, bc2 = 1 - torch.pow(torch.full_like(t, BETA1), t), 1 - torch.pow(torch.full_like(t, BETA2), t)
    g = g * coef.double() if eight else s["grad"].float() * coef
    blocks = torch.tensor([-(-n // BLOCK) for n in s["sizes"]], device=g.device)
    decay = torch.repeat_interleave(torch.tensor(s["decays"], device=g.device), blocks).unsqueeze(1)
    m = _from_8bit(s["m"], s["m_scale"], True) if eight else s["m"]
    v = _from_8bit(s["v"], s["v_scale"], False) if eight else s["v"]
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g * g
    if eight:
        code, scale = _to_8bit(m, True)
        s["m"].copy_(code)
        s["m_scale"].copy_(scale)
        code, scale = _to_8bit(v, False)
        s["v"].copy_(code)
        s["v_scale"].copy_(scale)
        out["m"] = _from_8bit(s["m"], s["m_scale"], True).float()
        out["v"] = _from_8bit(s["v"], s["v_scale"], False).float()
        m, v = m.float(), v.float()
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
        out["m"], out["v"] = s["m"], s["v"]
    update = (m / bc1.float()) / (torch.sqrt(v / bc2.float()) + ADAM_EPS)
    s["master"].sub_(s["lr"] * (decay * s["master"] + update))
    if s["weight"] is not s["master"]:
        s["weight"].copy_(s["master"])
    return {"master": s["master"], "weight": s["weight"], **out}


# ------------------------------------------------------------------------------------------------ the package's calls
def _own_linear(s):
    import paper_2512_06547_b200 as a3po
    case, td = s["case"], DTYPES[s["case"]["dt"]]
    n, k, m, train = case["N"], case["K"], case["M"], case["op"] == "linear_train"
    if "calls" not in s:          # a program's own buffers, made once for its shapes: outputs, kept values, scratch
        dev, masked = s["x"].device, s["mask"] is not None
        dt = a3po.A3PO_F32 if case["dt"] == "f32" else a3po.A3PO_BF16
        act = {"none": a3po.A3PO_ACT_NONE, "silu": a3po.A3PO_ACT_SILU, "gelu_tanh": a3po.A3PO_ACT_GELU_TANH}[case["act"]]
        new = lambda *shape, dtype=td: torch.empty(shape, dtype=dtype, device=dev)  # noqa: E731
        ws = a3po.new_workspace(max(a3po.a3po_linear_workspace_bytes(n, k, m, dt, act, masked, bwd)
                                    for bwd in ((False, True) if train else (False,))), dev)
        out, kept = {"y": new(n, m, dtype=td if train else DTYPES[case["out"]])}, None
        if train:
            out.update(grad_x=new(n, k), grad_w=new(m, k, dtype=DTYPES[case["grads"]]))
            if s["bias"] is not None:
                out["grad_bias"] = new(m, dtype=torch.float32)
            if case["act"] != "none":
                kept = a3po.new_workspace(a3po.a3po_linear_kept_bytes(n, m, dt, act), dev)
        s["calls"] = (out, ws, kept, act)
    out, ws, kept, act = s["calls"]
    a3po.a3po_linear_fwd(s["x"], s["w"], out["y"], ws, bias=s["bias"], residual=s["residual"], row_mask=s["mask"],
                         kept=kept, activation=act)
    if train:
        a3po.a3po_linear_bwd(s["x"], s["w"], s["grad_y"], out["grad_x"], out["grad_w"], ws, kept=kept,
                             grad_bias=out.get("grad_bias"), row_mask=s["mask"], activation=act)
    return out


def _own_sample(s):
    import paper_2512_06547_b200 as a3po
    n, v = s["logits"].shape
    if "calls" not in s:
        dev = s["logits"].device
        out = {"token": torch.empty(n, dtype=torch.int32, device=dev), "logp": torch.empty(n, device=dev),
               "kept_logp": torch.empty(n, device=dev), "n_kept": torch.empty(n, dtype=torch.int32, device=dev)}
        s["calls"] = (out, a3po.new_workspace(a3po.a3po_sample_workspace_bytes(n, v), dev))
    out, ws = s["calls"]
    a3po.a3po_sample(s["logits"], s["u"], out["token"], ws, temperature=s["temperature"], top_k=s["top_k"],
                     top_p=s["top_p"], min_p=s["min_p"], row_mask=s["mask"], logp=out["logp"], kept_logp=out["kept_logp"],
                     n_kept=out["n_kept"])
    return out


def _own_adamw(s):
    from paper_2512_06547_b200.optimizer import AdamW, decode_state
    case = s["case"]
    if "optimizer" not in s:
        def parts(flat):
            return [flat.view(-1)[at * BLOCK:at * BLOCK + n] for at, n in zip(s["starts"], s["sizes"])]

        def scales(flat):
            return [flat[at:at - (-n // BLOCK)] for at, n in zip(s["starts"], s["sizes"])]

        eight, mixed = case["bits"] == 8, s["weight"] is not s["master"]
        s["grads"] = parts(s["grad"])
        s["optimizer"] = AdamW(parts(s["weight"]), lr=s["lr"], betas=(BETA1, BETA2), eps=ADAM_EPS, weight_decay=s["decays"],
                               max_grad_norm=case["clip"], state_bits=case["bits"], masters=parts(s["master"]) if mixed else None,
                               m=parts(s["m"]), v=parts(s["v"]), m_scales=scales(s["m_scale"]) if eight else None,
                               v_scales=scales(s["v_scale"]) if eight else None, step=s["step"])
    opt = s["optimizer"]
    opt.step(s["grads"])
    out = {"master": s["master"], "weight": s["weight"], "grad_norm": opt.grad_norm, "m": s["m"], "v": s["v"]}
    if case["bits"] == 8:   # what the codes stand for
        out["m"] = decode_state(s["m"].view(-1), s["m_scale"], signed=True).view(s["m"].shape)
        out["v"] = decode_state(s["v"].view(-1), s["v_scale"], signed=False).view(s["v"].shape)
    return out


def run(state):
    op = state["case"]["op"]
    if op == "sample":
        return _own_sample(state) if own else _plain_sample(state)
    if op == "adamw":
        return _own_adamw(state) if own else _plain_adamw(state)
    return _own_linear(state) if own else _plain_linear(state)


# ------------------------------------------------------------------------------------------------ in 64 bits
def _exact_linear(case, s):
    keep = torch.ones(case["N"], 1, dtype=torch.bool, device=s["w"].device)
    if s["mask"] is not None:
        keep = (s["mask"] != 0).unsqueeze(1)

    def wide(t):
        return torch.where(keep, t, torch.zeros_like(t)).double()

    train = case["op"] == "linear_train"
    x, w = wide(s["x"]).requires_grad_(train), s["w"].double().requires_grad_(train)
    b = s["bias"].double().requires_grad_(train) if s["bias"] is not None else None
    y = torch.nn.functional.linear(x, w, b)
    if case["act"] != "none":
        y = torch.nn.functional.silu(y) if case["act"] == "silu" else torch.nn.functional.gelu(y, approximate="tanh")
    if s["residual"] is not None:
        y = y + wide(s["residual"])
    y = torch.where(keep, y, torch.zeros_like(y))
    if not train:
        return {"y": y}
    grads = torch.autograd.grad(y, (x, w) if b is None else (x, w, b), wide(s["grad_y"]))
    out = {"y": y.detach(), "grad_x": grads[0], "grad_w": grads[1]}
    if b is not None:
        out["grad_bias"] = grads[2]
    return out


def _exact_sample(case, s):
    """Row by row, from probabilities."""
    names = ("token", "logp", "kept_logp", "n_kept")
    out = {name: [] for name in names}
    n = case["N"]

    given = {name: None if s[name] is None else s[name].tolist() for name in ("temperature", "top_k", "top_p", "min_p")}

    def setting(name, i, off):
        return off if given[name] is None else given[name][i]

    for i in range(n):
        row = s["logits"][i].double()
        row = row.masked_fill(row.isnan(), float("-inf"))
        if (s["mask"] is not None and not bool(s["mask"][i])) or not bool((row > float("-inf")).any()):
            got = (-1, 0.0, 0.0, 0)
        else:
            t = setting("temperature", i, 1.0)
            logq = torch.log_softmax(row / (t if t > 0 else 1.0), dim=0)
            q = logq.exp()
            allowed = row > float("-inf")
            k, p, lowest = setting("top_k", i, 0), setting("top_p", i, 1.0), setting("min_p", i, 0.0)
            if t <= 0:
                k = 1
            if 0 < k < row.numel():
                value = torch.topk(row, int(k)).values[-1]
                ties = torch.nonzero(row == value).squeeze(1)[:int(k) - int((row > value).sum())]
                allowed = allowed & (row > value)
                allowed[ties] = row[ties] > float("-inf")
            if p < 1:
                ids = torch.nonzero(allowed).squeeze(1)
                ids = ids[torch.argsort(row[ids], descending=True, stable=True)]
                share = torch.cumsum(q[ids], dim=0)
                count = 1 + int((share[:-1] < p * share[-1]).sum())
                allowed = torch.zeros_like(allowed)
                allowed[ids[:count]] = True
            best = torch.argmax(torch.where(allowed, row, torch.full_like(row, float("-inf"))))
            if lowest > 0:
                allowed = allowed & (q >= lowest * q[best])
                allowed[best] = True
            mass = torch.where(allowed, q, torch.zeros_like(q))
            share = torch.cumsum(mass, dim=0)
            token = int((share <= float(s["u"][i]) * share[-1]).sum())
            among = torch.log_softmax(torch.where(allowed, row, torch.full_like(row, float("-inf"))) / (t if t > 0 else 1.0), dim=0)
            got = (token, float(logq[token]), float(among[token]), int(allowed.sum()))
        for name, x in zip(names, got):
            out[name].append(x)
    return {name: torch.tensor(x, dtype=torch.int32 if name in ("token", "n_kept") else torch.float64) for name, x in out.items()}


def _exact_adamw(case, s):
    dev = s["grad"].device

    def table(codes):
        return torch.tensor([c if c < 8 else (8 + c % 8) << (c // 8 - 1) for c in range(codes)], dtype=torch.float64, device=dev)

    def decoded(code, scale, signed):
        t = table(128 if signed else 256)
        t = torch.cat([t, -t]) if signed else t
        return t[code.long()] * scale.double().view(-1, 1)

    def stored(x, signed):
        """What x becomes in 8 bits: the nearest of the table's values times the block's scale."""
        t = table(128 if signed else 256)
        scale = (x.abs().max(dim=1, keepdim=True).values / t[-1]).float().double()
        a = torch.where(scale > 0, x.abs() / scale, torch.zeros_like(x))
        code = torch.bucketize(a, (t[1:] + t[:-1]) / 2)
        if not signed:
            code = torch.where(x > 0, code.clamp_min(1), code)
        return torch.sign(x) * t[code] * scale

    g = s["grad"].double()
    norm = torch.linalg.vector_norm(g)
    factor = min(1.0, case["clip"] / (float(norm) + 1e-6)) if case["clip"] > 0 else 1.0
    if case["bits"] == 8:     # the factor is an fp32 number of the operator
        factor = float(torch.tensor(factor, dtype=torch.float32))
    g = g * factor
    t = int(s["step"]) + 1
    eight = case["bits"] == 8
    m = decoded(s["m"], s["m_scale"], True) if eight else s["m"].double()
    v = decoded(s["v"], s["v_scale"], False) if eight else s["v"].double()
    m, v = torch.lerp(g, m, BETA1), torch.lerp(g.square(), v, BETA2)
    w = s["master"].double()
    per_tensor = zip(s["decays"], s["sizes"])
    decay = torch.cat([torch.full((-(-n // BLOCK), 1), d, dtype=torch.float64, device=dev) for d, n in per_tensor])
    lr = float(s["lr"])
    w = w * (1 - lr * decay) - lr / (1 - BETA1 ** t) * m / ((v / (1 - BETA2 ** t)).sqrt() + ADAM_EPS)
    return {"master": w, "weight": w, "grad_norm": norm.reshape(1), "m": stored(m, True) if eight else m,
            "v": stored(v, False) if eight else v}


def exact(case, seed):
    """The same outputs in 64 bits; None where sampling row by row would take too long."""
    if case["op"] == "sample" and case["N"] > 512:
        return None
    s = prepare(case, seed)
    return {"sample": _exact_sample, "adamw": _exact_adamw}.get(case["op"], _exact_linear)(case, s)

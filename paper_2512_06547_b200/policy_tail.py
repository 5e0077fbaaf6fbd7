"""The last feed-forward block of the policy, the final norm, the LM head and the A-3PO loss as one training pass, the same
layers with the sampling of the next token as one rollout pass, and the update of their weights.

For trainers that own the tail of the network: everything from the residual stream `r0` [N, H] that enters the last
block's feed-forward half to the loss, and back to grad_r0, through the library's calls:

    a            = norm(r0) gamma_in (+ beta_in)                     a3po_norm_fwd
    y            = (act(a Wg^T) * (a Wu^T)) Wd^T                     a3po_gated_ffn_fwd
    r1, hidden   = r0 + dropout(y), norm(r1) gamma_out (+ beta_out)  a3po_dropout_norm_fwd
    loss, ...    = LM head, log-softmax, A-3PO loss and back         a3po_train_step
    and the backward of the first three, in reverse order

Rows with mask 0 (padding) take no part in any of them and get zero gradients.  All buffers are made once for the
largest batch and reused by every pass; a pass launches on the current stream, never synchronises and can be captured
into a CUDA graph (after one uncaptured pass).  The random numbers of dropout come from the device words
rng = {seed, offset}: a trainer advances the offset between passes (in place, so a captured graph follows).

PolicySampler runs the forward half on the rows whose next token is wanted, and draws it:

    logits       = hidden W^T                                        a3po_linear_fwd (fp32)
    token, logp  = temperature, top-k, top-p, min-p; random numbers  a3po_sample

where logp is what the loss takes as behav_logp.  It is a log-prob at the row's temperature t (1 for a greedy row), so a pass over
rows that were drawn at another one than 1 takes inv_temperature = 1 / t: both sides of the importance weight are then the same
policy's.  Rows of unlike temperatures need passes of their own, whose losses are means over their rows.

PolicyTail.optimizer makes an AdamW over the pass's parameters, and PolicyTail.update takes its step with the gradients that the
last pass left.
"""
from __future__ import annotations

import torch

from . import binding as b
from .optimizer import AdamW


class PolicyTail:
    """Buffers and calls for batches of exactly n rows.

    params: dict with gamma_in [H], w_gate_up [2 F, H], w_down [H, F], gamma_out [H], w [V, H], and optionally beta_in,
    beta_out [H]; all of `dtype`.  beta: gradients of beta_in and beta_out are wanted (default: of layer norms); without
    them a pass refuses params that hold a beta."""

    def __init__(self, n, h, f, v, dtype=torch.bfloat16, *, kind=b.A3PO_NORM_RMS, activation=b.A3PO_ACT_SILU, dropout_p=0.0,
                 eps=1e-6, beta=None, device="cuda"):
        self.n, self.h, self.f, self.v, self.dtype = n, h, f, v, dtype
        self.kind, self.activation, self.p, self.eps = kind, activation, float(dropout_p), eps
        layer = kind == b.A3PO_NORM_LAYER
        dt = b.A3PO_F32 if dtype == torch.float32 else b.A3PO_BF16
        rows = lambda: torch.empty((n, h), dtype=dtype, device=device)
        f32 = lambda *s: torch.empty(s, dtype=torch.float32, device=device)
        self.a, self.y, self.r1, self.hidden = rows(), rows(), rows(), rows()
        self.rstd_in, self.rstd_out = f32(n), f32(n)
        self.mean_in, self.mean_out = (f32(n), f32(n)) if layer else (None, None)
        self.logp, self.lse, self.grad_logp, self.loss = f32(n), f32(n), f32(n), f32(1)
        self.grad_hidden, self.grad_r1, self.grad_y, self.grad_a, self.grad_r0 = rows(), rows(), rows(), rows(), rows()
        self.grads = {"gamma_in": f32(h), "gamma_out": f32(h), "w_gate_up": f32(2 * f, h), "w_down": f32(h, f), "w": f32(v, h)}
        self.beta = layer if beta is None else bool(beta)
        if self.beta:
            self.grads.update(beta_in=f32(h), beta_out=f32(h))
        self.stats = b.new_stats(device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self.kept = b.new_workspace(b.a3po_gated_ffn_kept_bytes(n, f, dt), device)
        self.ws = b.new_workspace(max(b.a3po_train_step_workspace_bytes(n, h, v, dt),
                                      b.a3po_norm_bwd_workspace_bytes(n, h),
                                      b.a3po_gated_ffn_workspace_bytes(n, h, f, dt, True, False),
                                      b.a3po_gated_ffn_workspace_bytes(n, h, f, dt, True, True)), device)

    def __call__(self, r0, params, batch, rng=None, *, inv_temperature=1.0, accumulate_grads=False):
        """One pass.  batch: targets, behav_logp, versions, current_version, adv, mask, clip_eps as a3po_train_step takes
        them; inv_temperature: of the policy that is trained, the one that behav_logp was drawn at.  Returns a dict of this
        object's own buffers: loss, stats, logp, status, grad_r0 and grads (by parameter, fp32; added to what they hold
        with accumulate_grads)."""
        if not self.beta and (params.get("beta_in") is not None or params.get("beta_out") is not None):
            raise ValueError("params hold a beta, but this PolicyTail was made without gradients for it (beta=True)")
        mask, g = batch["mask"], self.grads
        norm = dict(kind=self.kind, row_mask=mask)
        b.a3po_norm_fwd(r0, params["gamma_in"], self.a, self.rstd_in, beta=params.get("beta_in"), mean=self.mean_in,
                        eps=self.eps, **norm)
        b.a3po_gated_ffn_fwd(self.a, params["w_gate_up"], params["w_down"], self.y, self.ws, row_mask=mask,
                             kept=self.kept, activation=self.activation, status=self.status)
        b.a3po_dropout_norm_fwd(self.y, r0, self.p, rng, params["gamma_out"], self.r1, self.hidden, self.rstd_out,
                                beta=params.get("beta_out"), mean=self.mean_out, eps=self.eps, **norm)
        b.a3po_train_step(self.hidden, params["w"], batch["targets"], batch["behav_logp"], batch["versions"],
                          batch["current_version"], batch["adv"], mask, batch["clip_eps"], self.logp, self.lse,
                          self.grad_logp, self.loss, self.grad_hidden, g["w"], self.ws, stats=self.stats,
                          accumulate_grad_w=accumulate_grads, inv_temperature=inv_temperature, status=self.status)
        b.a3po_dropout_norm_bwd(self.r1, self.p, rng, params["gamma_out"], self.rstd_out, self.grad_hidden,
                                self.grad_r1, self.grad_y, g["gamma_out"], self.ws, mean=self.mean_out,
                                grad_beta=g.get("beta_out"), accumulate_grad_w=accumulate_grads, **norm)
        b.a3po_gated_ffn_bwd(self.a, params["w_gate_up"], params["w_down"], self.kept, self.grad_y, self.grad_a,
                             g["w_gate_up"], g["w_down"], self.ws, row_mask=mask, activation=self.activation,
                             accumulate_grad_w=accumulate_grads, status=self.status)
        # r0 feeds the norm and the residual stream: both gradients in one pass, nothing went through dropout here
        b.a3po_dropout_norm_bwd(r0, 0.0, None, params["gamma_in"], self.rstd_in, self.grad_a, self.grad_r0, None,
                                g["gamma_in"], self.ws, mean=self.mean_in, grad_r=self.grad_r1,
                                grad_beta=g.get("beta_in"), accumulate_grad_w=accumulate_grads, **norm)
        return {"loss": self.loss, "stats": self.stats, "logp": self.logp, "status": self.status,
                "grad_r0": self.grad_r0, "grads": g}

    def optimizer(self, params, *, weight_decay=0.01, **kw):
        """AdamW over `params` (in the order of self.grads, without a beta that they do not hold), with fp32 masters of bf16 weights;
        norms do not decay.  kw as for AdamW."""
        names = [k for k in self.grads if params.get(k) is not None or k not in ("beta_in", "beta_out")]
        weights = [params[k] for k in names]
        if self.dtype != torch.float32:
            kw.setdefault("masters", True)
        made = AdamW(weights, weight_decay=[float(weight_decay) if w.dim() > 1 else 0.0 for w in weights], **kw)
        made.names = names
        return made

    def update(self, optimizer):
        """The optimizer's step with the gradients that the last pass left (fp32), on the current stream: of the parameters that
        self.optimizer made it for, else of all in the order of self.grads."""
        optimizer.step([self.grads[k] for k in getattr(optimizer, "names", self.grads)])


class PolicySampler:
    """Buffers and calls for drawing the next token of n rows of the residual stream at once (single tokens while serving,
    batches of rollouts).  params as PolicyTail takes them.  A pass launches on the current stream, never synchronises and can
    be captured into a CUDA graph (after one uncaptured pass)."""

    def __init__(self, n, h, f, v, dtype=torch.bfloat16, *, kind=b.A3PO_NORM_RMS, activation=b.A3PO_ACT_SILU, eps=1e-6,
                 device="cuda"):
        self.kind, self.activation, self.eps = kind, activation, eps
        dt = b.A3PO_F32 if dtype == torch.float32 else b.A3PO_BF16
        rows = lambda: torch.empty((n, h), dtype=dtype, device=device)
        per_row = lambda dtype: torch.empty(n, dtype=dtype, device=device)
        self.a, self.y, self.r1, self.hidden = rows(), rows(), rows(), rows()
        self.logits = torch.empty((n, v), dtype=torch.float32, device=device)
        self.token, self.n_kept = per_row(torch.int32), per_row(torch.int32)
        self.logp, self.kept_logp = per_row(torch.float32), per_row(torch.float32)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self.ws = b.new_workspace(max(b.a3po_gated_ffn_workspace_bytes(n, h, f, dt, True, False),
                                      b.a3po_linear_workspace_bytes(n, h, v, dt, has_row_mask=True),
                                      b.a3po_sample_workspace_bytes(n, v)), device)

    def __call__(self, r0, params, u, *, temperature=None, top_k=None, top_p=None, min_p=None, row_mask=None):
        """r0 [n, H], u fp32 [n] in [0, 1); the rest as a3po_sample takes it (rows with row_mask 0 have finished: token -1).
        Returns a dict of this object's own buffers: token, logp (of the whole softmax at the row's temperature), kept_logp
        (among the tokens that the filters kept), n_kept, logits, hidden and status."""
        norm = dict(kind=self.kind, eps=self.eps, row_mask=row_mask)
        b.a3po_norm_fwd(r0, params["gamma_in"], self.a, beta=params.get("beta_in"), **norm)
        b.a3po_gated_ffn_fwd(self.a, params["w_gate_up"], params["w_down"], self.y, self.ws, row_mask=row_mask,
                             activation=self.activation, status=self.status)
        b.a3po_dropout_norm_fwd(self.y, r0, 0.0, None, params["gamma_out"], self.r1, self.hidden, beta=params.get("beta_out"),
                                **norm)
        b.a3po_linear_fwd(self.hidden, params["w"], self.logits, self.ws, row_mask=row_mask, status=self.status)
        b.a3po_sample(self.logits, u, self.token, self.ws, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p,
                      row_mask=row_mask, logp=self.logp, kept_logp=self.kept_logp, n_kept=self.n_kept)
        return {"token": self.token, "logp": self.logp, "kept_logp": self.kept_logp, "n_kept": self.n_kept,
                "logits": self.logits, "hidden": self.hidden, "status": self.status}

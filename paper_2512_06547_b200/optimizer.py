"""AdamW over a list of tensors through a3po_adamw_step: one call for the gradient norm, its clip and the update of every
tensor, with states in 32 or 8 bits and fp32 masters of bf16 weights.  The count of steps and the learning rate are device words,
so a step can be captured into a CUDA graph (after one uncaptured step) and replayed with another rate."""
from __future__ import annotations

import ctypes

import torch

from . import binding as b

STATE_BLOCK = 256   # elements of an 8-bit state that share a scale


def decode_state(codes, scales, *, signed, out=None):
    """fp32 values of an 8-bit state: codes uint8 [n], scales fp32 [ceil(n / 256)]; signed: a first moment."""
    out = torch.empty(codes.shape, dtype=torch.float32, device=codes.device) if out is None else out
    b.a3po_adamw_state_values(codes, scales, out, signed=signed)
    return out


def _like(given, weights, dtype, name, sizes=None):
    sizes = [w.numel() for w in weights] if sizes is None else sizes
    if given is None:
        return [torch.zeros(n, dtype=dtype, device=w.device) for n, w in zip(sizes, weights)]
    given = list(given)
    if len(given) != len(weights):
        raise ValueError(f"{name}: expected one tensor per weight")
    for t, n in zip(given, sizes):
        b._want(t, dtype, name)
        if t.numel() != n:
            raise ValueError(f"{name}: expected {n} elements, got {t.numel()}")
    b._here(*given)
    return given


class AdamW:
    """weights: contiguous tensors of one type (fp32 or bf16), updated in place by step(grads).

    lr: a number, or an fp32 device scalar that the caller changes between steps.  weight_decay: a number, or one per weight.
    max_grad_norm: 0 for no clipping; grad_norm holds the norm of the last step's gradients before clipping either way.  The norm is
    over this object's gradients: weights of another type, in an object of their own, are clipped by themselves.  A step whose
    norm is not finite changes nothing.  state_bits: 32 or 8; from step 33 on, states of 8 bits are rounded at random (by numbers
    that the step, the place of the weight and the element give), so that they follow their averages whatever the betas.
    masters: True (bf16 weights) keeps an fp32 copy of each weight, which is what is updated; a list gives the copies.
    m, v, m_scales, v_scales, step: states to go on from (kept and updated in place), as this object's attributes of these names
    hold them.  The weights and states that an object was made with stay its own: new contents are copied into them (lr, steps and
    grad_norm may be replaced)."""

    def __init__(self, weights, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, *, max_grad_norm=0.0, state_bits=32,
                 masters=None, m=None, v=None, m_scales=None, v_scales=None, step=None):
        self.weights = list(weights)
        if state_bits not in (8, 32):
            raise ValueError("state_bits: 8 or 32")
        dtype = self.weights[0].dtype if self.weights else torch.float32
        self._weight_dt = b._dtype_code(self.weights[0]) if self.weights else b.A3PO_F32
        for w in self.weights:
            b._want(w, dtype, "weights")
        b._here(*self.weights)
        if len({w.data_ptr() for w in self.weights if w.numel()}) < sum(w.numel() > 0 for w in self.weights):
            raise ValueError("weights: the same tensor twice")
        device = self.weights[0].device if self.weights else torch.device("cuda", torch.cuda.current_device())
        count = len(self.weights)
        decay = [float(weight_decay)] * count if isinstance(weight_decay, (int, float)) else [float(d) for d in weight_decay]
        if len(decay) != count:
            raise ValueError("weight_decay: expected a number or one per weight")
        if masters is True:
            masters = [w.detach().float() for w in self.weights]
        if masters is not None and masters is not False:
            if dtype == torch.float32:
                raise ValueError("masters: fp32 weights are their own")
            self.masters = _like(masters, self.weights, torch.float32, "masters")
        else:
            self.masters = None
        state = torch.uint8 if state_bits == 8 else torch.float32
        self.m, self.v = _like(m, self.weights, state, "m"), _like(v, self.weights, state, "v")
        self.m_scales = self.v_scales = None
        if state_bits == 8:
            blocks = [-(-w.numel() // STATE_BLOCK) for w in self.weights]
            self.m_scales = _like(m_scales, self.weights, torch.float32, "m_scales", blocks)
            self.v_scales = _like(v_scales, self.weights, torch.float32, "v_scales", blocks)
        elif m_scales is not None or v_scales is not None:
            raise ValueError("m_scales, v_scales: of states of 8 bits only")
        self.lr = lr if isinstance(lr, torch.Tensor) else torch.full((1,), float(lr), device=device)
        self.steps = torch.zeros(1, dtype=torch.int64, device=device) if step is None else step
        self.grad_norm = torch.zeros(1, device=device)
        self.state_bits, self.eps, self.max_grad_norm = state_bits, float(eps), float(max_grad_norm)
        self.beta1, self.beta2 = float(betas[0]), float(betas[1])
        self._ws = b.new_workspace(b.a3po_adamw_workspace_bytes(count), device)
        self._table = (b.A3poAdamWTensor * count)()
        self._device = device.index
        at = lambda tensors, i: None if tensors is None else tensors[i].data_ptr()
        for i, w in enumerate(self.weights):
            self._table[i] = b.A3poAdamWTensor(w.data_ptr(), at(self.masters, i), None, at(self.m, i), at(self.v, i),
                                               at(self.m_scales, i), at(self.v_scales, i), w.numel(), decay[i])
        self._rows = [(self._table[i], w, w.data_ptr(), w.numel(), w.shape) for i, w in enumerate(self.weights)]

    def step(self, grads, *, stream=None):
        """grads: one tensor per weight, of its shape or flat, all fp32 or all bf16."""
        if len(grads) != len(self.weights):
            raise ValueError("grads: expected one tensor per weight")
        device, here = self._device, torch.cuda.current_device()
        dtype = grads[0].dtype if grads else torch.float32
        fine = device == here
        for g, (row, w, at, n, shape) in zip(grads, self._rows):
            fine &= (g.dtype is dtype and (g.shape == shape or g.shape == (n,)) and g.get_device() == device and g.is_contiguous()
                     and w.data_ptr() == at)
            row.grad = g.data_ptr()
        for t, ty in ((self.lr, torch.float32), (self.steps, torch.int64), (self.grad_norm, torch.float32)):
            fine &= t.dtype is ty and t.numel() == 1 and t.get_device() == device
        if not fine:   # say what is wrong
            self._refuse(grads, dtype, here)
        grad_dt = b._dtype_code(grads[0]) if grads else b.A3PO_F32
        rc = b.load_library().a3po_adamw_step(
            ctypes.addressof(self._table), len(self._table), self._weight_dt, grad_dt, self.state_bits, self.beta1, self.beta2,
            self.eps, self.max_grad_norm, self.lr.data_ptr(), self.steps.data_ptr(), self.grad_norm.data_ptr(),
            self._ws.data_ptr(), self._ws.numel(), b._stream(stream))
        b._check("a3po_adamw_step", rc)

    def _refuse(self, grads, dtype, here):
        if self._device != here:
            raise ValueError(f"expected the current device cuda:{self._device}, got cuda:{here}")
        for g, (_, w, at, n, shape) in zip(grads, self._rows):
            if g.dtype is not dtype:
                raise TypeError("grads: expected tensors of one type")
            b._want(g, dtype, "grads")
            b._here(g)
            if g.shape != shape and g.shape != (n,):
                raise ValueError(f"grads: expected the weight's shape {tuple(shape)}, or its elements in a row, got {tuple(g.shape)}")
            if w.data_ptr() != at:
                raise ValueError("weights: a weight's storage is another than when the object was made")
        for t, ty, name in ((self.lr, torch.float32, "lr"), (self.steps, torch.int64, "steps"),
                            (self.grad_norm, torch.float32, "grad_norm")):
            b._want(t, ty, name)
            b._here(t)
            if t.numel() != 1:
                raise ValueError(f"{name}: expected one element")
        raise ValueError("expected tensors on the current device")

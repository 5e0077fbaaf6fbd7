"""ctypes binding of liba3po.so: same names as the C ABI, argument marshalling only.

Tensors are torch tensors used as typed device (or, for the host entry, pinned host) buffers;
torch does none of the arithmetic.  Every function raises if the compiled library is missing or
a call returns an error code: there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import c_char_p, c_double, c_float, c_int, c_int32, c_int64, c_size_t, c_void_p

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "lib", "liba3po.so")

A3PO_F32 = 0
A3PO_BF16 = 1
A3PO_ACT_SILU = 0
A3PO_ACT_GELU_TANH = 1
A3PO_ACT_NONE = 2
A3PO_NORM_RMS = 0
A3PO_NORM_LAYER = 1
STATUS_TARGET_OUT_OF_RANGE = 1
STATUS_WAIT_TIMEOUT = 2
STATUS_KEPT_RANGE = 4


class A3poStats(ctypes.Structure):
    _fields_ = [("n_valid", c_int64), ("n_clipped", c_int64), ("iw_max", c_float), ("iw_min", c_float)]


class A3poAdamWTensor(ctypes.Structure):
    """One entry of a3po_adamw_step's table (device addresses)."""
    _fields_ = [("weight", c_void_p), ("master", c_void_p), ("grad", c_void_p), ("m", c_void_p), ("v", c_void_p),
                ("m_scale", c_void_p), ("v_scale", c_void_p), ("n", c_int64), ("weight_decay", c_float)]


class A3poError(RuntimeError):
    def __init__(self, fn, code, text):
        super().__init__(f"{fn} failed: {text} (code {code})")
        self.code = code


_SIGNATURES = {
    "a3po_status_string": (c_char_p, [c_int]),
    "a3po_version": (c_int, []),
    "a3po_kernel_launch_count": (c_int64, []),
    "a3po_kernel_name": (c_char_p, [c_int]),
    "a3po_profile_enable": (c_int, [c_int]),
    "a3po_profile_read": (c_int, [c_int, c_void_p, c_void_p, c_void_p]),
    "a3po_token_logprobs_workspace_bytes": (c_size_t, [c_int64, c_int, c_int, c_int, c_int]),
    "a3po_token_logprobs_min_workspace_bytes": (c_size_t, [c_int64, c_int, c_int, c_int, c_int]),
    "a3po_loss_workspace_bytes": (c_size_t, [c_int64]),
    "a3po_train_step_stage_bytes": (c_size_t, [c_int64, c_int, c_int]),
    "a3po_host_to_device_bytes": (c_int64, []),
    "a3po_train_step_workspace_bytes": (c_size_t, [c_int64, c_int, c_int, c_int]),
    "a3po_token_logprobs_fwd": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_int, c_int, c_int, c_float,
                                        c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p, c_void_p]),
    "a3po_token_logprobs_bwd": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_int, c_int, c_int,
                                        c_float, c_void_p, c_void_p, c_int, c_void_p, c_size_t, c_void_p, c_void_p]),
    "a3po_loss_fwd": (c_int, [c_void_p, c_void_p, c_void_p, c_int, c_void_p, c_int, c_int32, c_void_p, c_void_p,
                              c_int64, c_float, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "a3po_loss_fwd_static": (c_int, [c_void_p, c_void_p, c_void_p, c_int, c_void_p, c_int, c_int32, c_void_p, c_void_p,
                                     c_int64, c_float, c_void_p, c_void_p, c_void_p]),
    "a3po_loss_bwd": (c_int, [c_void_p, c_void_p, c_void_p, c_int, c_void_p, c_int, c_int32, c_void_p, c_void_p,
                              c_int64, c_float, c_int, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "a3po_loss_fwd_bwd": (c_int, [c_void_p, c_void_p, c_void_p, c_int, c_void_p, c_int, c_int32, c_void_p, c_void_p,
                                  c_int64, c_float, c_int, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t,
                                  c_void_p]),
    "a3po_decoupled_loss_fwd_bwd": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_float, c_void_p,
                                            c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "a3po_grpo_workspace_bytes": (c_size_t, [c_int]),
    "a3po_grpo_advantages": (c_int, [c_void_p, c_int, c_int, c_void_p, c_int64, c_float, c_void_p, c_void_p, c_size_t,
                                     c_void_p]),
    "a3po_selftest_wait_timeout": (c_int, [c_void_p, ctypes.c_uint, c_void_p]),
    "a3po_kept_bytes": (c_size_t, [c_int64, c_int]),
    "a3po_token_logprobs_fwd_keep_workspace_bytes": (c_size_t, [c_int64, c_int, c_int]),
    "a3po_token_logprobs_bwd_kept_workspace_bytes": (c_size_t, [c_int64, c_int, c_int]),
    "a3po_token_logprobs_fwd_keep": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_int, c_int, c_float,
                                             c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p, c_size_t,
                                             c_void_p, c_void_p]),
    "a3po_token_logprobs_bwd_kept": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t,
                                             c_int64, c_int, c_int, c_float, c_void_p, c_void_p, c_int, c_void_p,
                                             c_size_t, c_void_p, c_void_p]),
    "a3po_train_step_min_workspace_bytes": (c_size_t, [c_int64, c_int, c_int, c_int]),
    "a3po_train_step": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_int, c_int, c_int,
                                c_int32, c_float, c_float, c_void_p, c_void_p, c_int, c_void_p, c_void_p, c_void_p,
                                c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p,
                                c_void_p]),
    "a3po_mask_count_workspace_bytes": (c_size_t, []),
    "a3po_mask_count": (c_int, [c_void_p, c_int64, c_void_p, c_void_p, c_size_t, c_void_p]),
    "a3po_dp_loss_scale": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]),
    "a3po_train_step_host": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_int, c_int,
                                     c_int, c_int32, c_float, c_float, c_void_p, c_void_p, c_int, c_void_p, c_void_p,
                                     c_size_t, c_void_p, c_size_t, c_void_p, c_void_p, c_void_p, c_void_p]),
    "a3po_norm_fwd": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_int, c_int, c_int, c_float, c_void_p,
                              c_void_p, c_void_p, c_void_p]),
    "a3po_norm_bwd_workspace_bytes": (c_size_t, [c_int64, c_int]),
    "a3po_norm_bwd": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_int, c_int, c_int,
                              c_void_p, c_void_p, c_void_p, c_int, c_void_p, c_size_t, c_void_p]),
    "a3po_dropout_fwd": (c_int, [c_void_p, c_void_p, c_void_p, c_int64, c_int, c_int, c_float, c_void_p, c_void_p,
                                 c_void_p]),
    "a3po_dropout_bwd": (c_int, [c_void_p, c_void_p, c_int64, c_int, c_int, c_float, c_void_p, c_void_p, c_void_p]),
    "a3po_dropout_norm_fwd": (c_int, [c_void_p, c_void_p, c_float, c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_int,
                                      c_int, c_int, c_float, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]),
    "a3po_dropout_norm_bwd": (c_int, [c_void_p, c_float, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                      c_void_p, c_int64, c_int, c_int, c_int, c_void_p, c_void_p, c_void_p, c_void_p,
                                      c_int, c_void_p, c_size_t, c_void_p]),
    "a3po_gated_ffn_kept_bytes": (c_size_t, [c_int64, c_int, c_int]),
    "a3po_gated_ffn_workspace_bytes": (c_size_t, [c_int64, c_int, c_int, c_int, c_int, c_int]),
    "a3po_gated_ffn_fwd": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_int, c_int, c_int, c_int, c_void_p,
                                   c_void_p, c_size_t, c_void_p, c_size_t, c_void_p, c_void_p]),
    "a3po_gated_ffn_bwd": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p, c_int64, c_int,
                                   c_int, c_int, c_int, c_void_p, c_void_p, c_void_p, c_int, c_int, c_void_p, c_size_t,
                                   c_void_p, c_void_p]),
    "a3po_sample_workspace_bytes": (c_size_t, [c_int64, c_int]),
    "a3po_sample": (c_int, [c_void_p, c_int64, c_void_p, c_int64, c_int, c_int, c_void_p, c_void_p, c_void_p, c_void_p,
                            c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "a3po_adamw_workspace_bytes": (c_size_t, [c_int]),
    "a3po_adamw_step": (c_int, [c_void_p, c_int, c_int, c_int, c_int, c_double, c_double, c_float, c_float, c_void_p, c_void_p,
                                c_void_p, c_void_p, c_size_t, c_void_p]),
    "a3po_adamw_state_values": (c_int, [c_void_p, c_void_p, c_int64, c_int, c_void_p, c_void_p]),
    "a3po_linear_kept_bytes": (c_size_t, [c_int64, c_int, c_int, c_int]),
    "a3po_linear_workspace_bytes": (c_size_t, [c_int64, c_int, c_int, c_int, c_int, c_int, c_int]),
    "a3po_linear_fwd": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_int, c_int, c_int, c_int, c_void_p,
                                c_int, c_void_p, c_size_t, c_void_p, c_size_t, c_void_p, c_void_p]),
    "a3po_linear_bwd": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p, c_int64, c_int, c_int, c_int, c_int,
                                c_void_p, c_void_p, c_int, c_void_p, c_int, c_void_p, c_size_t, c_void_p, c_void_p]),
}

_lib = None


def exported_symbols():
    """Names every build of the library must export (those declared in include/a3po.h)."""
    return sorted(_SIGNATURES)


def load_library(path: str | None = None):
    """Load liba3po.so once and attach argument types.  Raises if it has not been built."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise RuntimeError(
            f"{p} not found: build it with `python -m paper_2512_06547_b200.build` "
            "(there is no fallback implementation)")
    lib = ctypes.CDLL(p)
    for name, (res, args) in _SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    if path is None:
        _lib = lib
    return lib


def _check(fn, code):
    if code != 0:
        raise A3poError(fn, code, load_library().a3po_status_string(code).decode())


def _ptr(t):
    return None if t is None else t.data_ptr()


# Handle of the current stream without building a torch.cuda.Stream object (3.4 us of a small call's time).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream=None):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return A3PO_F32
    if t.dtype == torch.bfloat16:
        return A3PO_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _want(t, dtype, name, device_type="cuda"):
    if t is None:
        return
    if t.dtype is not dtype or not t.is_contiguous() or (not t.is_cuda if device_type == "cuda"
                                                         else t.device.type != device_type):
        raise TypeError(f"{name}: expected contiguous {dtype} tensor on {device_type}, got {t.dtype} on {t.device}")


# ------------------------------------------------------------------------------ sizes
def a3po_version() -> int:
    return load_library().a3po_version()


def a3po_kernel_launch_count() -> int:
    return load_library().a3po_kernel_launch_count()


def a3po_profile_enable(on: bool) -> None:
    _check("a3po_profile_enable", load_library().a3po_profile_enable(int(bool(on))))


def a3po_profile_read(max_entries: int = 1 << 16):
    """Returns [(kernel name, milliseconds), ...] for the launches recorded since the last read."""
    lib = load_library()
    ids = (c_int * max_entries)()
    ms = (c_float * max_entries)()
    count = c_int(0)
    _check("a3po_profile_read", lib.a3po_profile_read(max_entries, ids, ms, ctypes.byref(count)))
    return [(lib.a3po_kernel_name(ids[i]).decode(), float(ms[i])) for i in range(count.value)]


def a3po_token_logprobs_workspace_bytes(N, H, V, dt, is_bwd) -> int:
    return load_library().a3po_token_logprobs_workspace_bytes(N, H, V, dt, int(is_bwd))


def a3po_token_logprobs_min_workspace_bytes(N, H, V, dt, is_bwd) -> int:
    return load_library().a3po_token_logprobs_min_workspace_bytes(N, H, V, dt, int(is_bwd))


def a3po_loss_workspace_bytes(N) -> int:
    return load_library().a3po_loss_workspace_bytes(N)


def a3po_train_step_stage_bytes(N, H, dt) -> int:
    return load_library().a3po_train_step_stage_bytes(N, H, dt)


def a3po_host_to_device_bytes() -> int:
    return int(load_library().a3po_host_to_device_bytes())


def a3po_train_step_workspace_bytes(N, H, V, dt) -> int:
    return load_library().a3po_train_step_workspace_bytes(N, H, V, dt)


def new_workspace(nbytes: int, device="cuda") -> torch.Tensor:
    """A byte buffer usable as `ws` (torch's CUDA allocations are at least 256-byte aligned)."""
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


# ------------------------------------------------------------------------------ LM head
def a3po_token_logprobs_fwd(hidden, w, targets, logp, lse, ws, *, row_mask=None, entropy=None,
                            inv_temperature=1.0, status=None, stream=None):
    dt = _dtype_code(hidden)
    _want(hidden, hidden.dtype, "hidden"); _want(w, hidden.dtype, "w")
    _want(targets, torch.int32, "targets"); _want(row_mask, torch.uint8, "row_mask")
    _want(logp, torch.float32, "logp"); _want(lse, torch.float32, "lse"); _want(entropy, torch.float32, "entropy")
    _want(status, torch.int32, "status"); _want(ws, torch.uint8, "ws")
    n, h = hidden.shape
    v = w.shape[0]
    if w.shape[1] != h or targets.numel() != n or logp.numel() != n or lse.numel() != n:
        raise ValueError("shape mismatch")
    rc = load_library().a3po_token_logprobs_fwd(_ptr(hidden), _ptr(w), _ptr(targets), _ptr(row_mask), n, h, v, dt,
                                                float(inv_temperature), _ptr(logp), _ptr(lse), _ptr(entropy),
                                                _ptr(ws), ws.numel(), _ptr(status), _stream(stream))
    _check("a3po_token_logprobs_fwd", rc)


def a3po_token_logprobs_bwd(hidden, w, targets, lse, grad_logp, grad_hidden, grad_w, ws, *, accumulate_grad_w=False,
                            inv_temperature=1.0, status=None, stream=None):
    dt = _dtype_code(hidden)
    _want(hidden, hidden.dtype, "hidden"); _want(w, hidden.dtype, "w"); _want(grad_hidden, hidden.dtype, "grad_hidden")
    _want(targets, torch.int32, "targets"); _want(lse, torch.float32, "lse"); _want(grad_logp, torch.float32, "grad_logp")
    _want(grad_w, torch.float32, "grad_w"); _want(status, torch.int32, "status"); _want(ws, torch.uint8, "ws")
    n, h = hidden.shape
    v = w.shape[0]
    if w.shape[1] != h or grad_hidden.shape != hidden.shape or grad_w.shape != w.shape or grad_logp.numel() != n:
        raise ValueError("shape mismatch")
    rc = load_library().a3po_token_logprobs_bwd(_ptr(hidden), _ptr(w), _ptr(targets), _ptr(lse), _ptr(grad_logp), n, h,
                                                v, dt, float(inv_temperature), _ptr(grad_hidden), _ptr(grad_w),
                                                int(bool(accumulate_grad_w)), _ptr(ws), ws.numel(), _ptr(status),
                                                _stream(stream))
    _check("a3po_token_logprobs_bwd", rc)


def a3po_kept_bytes(N, V) -> int:
    return load_library().a3po_kept_bytes(N, V)


def a3po_token_logprobs_fwd_keep_workspace_bytes(N, H, V) -> int:
    return load_library().a3po_token_logprobs_fwd_keep_workspace_bytes(N, H, V)


def a3po_token_logprobs_bwd_kept_workspace_bytes(N, H, V) -> int:
    return load_library().a3po_token_logprobs_bwd_kept_workspace_bytes(N, H, V)


def a3po_token_logprobs_fwd_keep(hidden, w, targets, logp, lse, kept, ws, *, row_mask=None, entropy=None,
                                 inv_temperature=1.0, status=None, stream=None):
    """Forward that also fills `kept` (uint8 buffer of a3po_kept_bytes) for a3po_token_logprobs_bwd_kept."""
    _want(hidden, torch.bfloat16, "hidden"); _want(w, torch.bfloat16, "w")
    _want(targets, torch.int32, "targets"); _want(row_mask, torch.uint8, "row_mask")
    _want(logp, torch.float32, "logp"); _want(lse, torch.float32, "lse"); _want(entropy, torch.float32, "entropy")
    _want(kept, torch.uint8, "kept"); _want(ws, torch.uint8, "ws"); _want(status, torch.int32, "status")
    n, h = hidden.shape
    v = w.shape[0]
    if w.shape[1] != h or targets.numel() != n or logp.numel() != n or lse.numel() != n:
        raise ValueError("shape mismatch")
    rc = load_library().a3po_token_logprobs_fwd_keep(_ptr(hidden), _ptr(w), _ptr(targets), _ptr(row_mask), n, h, v,
                                                     float(inv_temperature), _ptr(logp), _ptr(lse), _ptr(entropy),
                                                     _ptr(kept), kept.numel(), _ptr(ws), ws.numel(), _ptr(status),
                                                     _stream(stream))
    _check("a3po_token_logprobs_fwd_keep", rc)


def a3po_token_logprobs_bwd_kept(hidden, w, targets, lse, grad_logp, kept, grad_hidden, grad_w, ws, *,
                                 accumulate_grad_w=False, inv_temperature=1.0, status=None, stream=None):
    """Backward from what a3po_token_logprobs_fwd_keep kept (no recomputation of the LM head)."""
    _want(hidden, torch.bfloat16, "hidden"); _want(w, torch.bfloat16, "w")
    _want(grad_hidden, torch.bfloat16, "grad_hidden"); _want(targets, torch.int32, "targets")
    _want(lse, torch.float32, "lse"); _want(grad_logp, torch.float32, "grad_logp")
    _want(grad_w, torch.float32, "grad_w"); _want(kept, torch.uint8, "kept"); _want(ws, torch.uint8, "ws")
    _want(status, torch.int32, "status")
    n, h = hidden.shape
    v = w.shape[0]
    if w.shape[1] != h or grad_hidden.shape != hidden.shape or grad_w.shape != w.shape or grad_logp.numel() != n:
        raise ValueError("shape mismatch")
    rc = load_library().a3po_token_logprobs_bwd_kept(_ptr(hidden), _ptr(w), _ptr(targets), _ptr(lse), _ptr(grad_logp),
                                                     _ptr(kept), kept.numel(), n, h, v, float(inv_temperature),
                                                     _ptr(grad_hidden), _ptr(grad_w), int(bool(accumulate_grad_w)),
                                                     _ptr(ws), ws.numel(), _ptr(status), _stream(stream))
    _check("a3po_token_logprobs_bwd_kept", rc)


# ------------------------------------------------------------------------------ loss
def _loss_common(logp, behav_logp, versions, adv, mask, cu_seqlens):
    _want(logp, torch.float32, "logp"); _want(behav_logp, torch.float32, "behav_logp")
    _want(versions, torch.int32, "versions"); _want(adv, torch.float32, "adv"); _want(mask, torch.uint8, "mask")
    _want(cu_seqlens, torch.int32, "cu_seqlens")
    n = logp.numel()
    if behav_logp.numel() != n or adv.numel() != n or mask.numel() != n:
        raise ValueError("shape mismatch")
    per_seq = cu_seqlens is not None
    b = cu_seqlens.numel() - 1 if per_seq else 0
    if per_seq and versions.numel() != b:
        raise ValueError("versions must have one entry per sequence when cu_seqlens is given")
    if not per_seq and versions.numel() != n:
        raise ValueError("versions must have one entry per token")
    return n, int(per_seq), b


def new_stats(device="cuda") -> torch.Tensor:
    """Device storage for one a3po_stats struct (24 bytes)."""
    return torch.zeros(ctypes.sizeof(A3poStats), dtype=torch.uint8, device=device)


def read_stats(stats: torch.Tensor) -> dict:
    raw = bytes(stats.cpu().numpy().tobytes())
    s = A3poStats.from_buffer_copy(raw)
    return dict(n_valid=s.n_valid, n_clipped=s.n_clipped, iw_max=s.iw_max, iw_min=s.iw_min)


def a3po_loss_fwd(logp, behav_logp, versions, current_version, adv, mask, clip_eps, loss, ws, *, stats=None,
                  cu_seqlens=None, stream=None):
    n, per_seq, b = _loss_common(logp, behav_logp, versions, adv, mask, cu_seqlens)
    _want(loss, torch.float32, "loss"); _want(stats, torch.uint8, "stats"); _want(ws, torch.uint8, "ws")
    rc = load_library().a3po_loss_fwd(_ptr(logp), _ptr(behav_logp), _ptr(versions), per_seq, _ptr(cu_seqlens), b,
                                      int(current_version), _ptr(adv), _ptr(mask), n, float(clip_eps), _ptr(loss),
                                      _ptr(stats), _ptr(ws), ws.numel(), _stream(stream))
    _check("a3po_loss_fwd", rc)


LOSS_FWD_STATIC_MAX_TOKENS = 1 << 20


def a3po_loss_fwd_static(logp, behav_logp, versions, current_version, adv, mask, clip_eps, loss, *, stats=None,
                         cu_seqlens=None, stream=None):
    """a3po_loss_fwd for callers that cannot supply a workspace: the scratch is a fixed array inside the
    library (at most LOSS_FWD_STATIC_MAX_TOKENS tokens; calls on one device must not overlap)."""
    n, per_seq, b = _loss_common(logp, behav_logp, versions, adv, mask, cu_seqlens)
    _want(loss, torch.float32, "loss"); _want(stats, torch.uint8, "stats")
    rc = load_library().a3po_loss_fwd_static(_ptr(logp), _ptr(behav_logp), _ptr(versions), per_seq, _ptr(cu_seqlens),
                                             b, int(current_version), _ptr(adv), _ptr(mask), n, float(clip_eps),
                                             _ptr(loss), _ptr(stats), _stream(stream))
    _check("a3po_loss_fwd_static", rc)


def a3po_loss_bwd(logp, behav_logp, versions, current_version, adv, mask, clip_eps, grad_logp, ws, *,
                  detach_prox=True, grad_loss=None, fwd_stats=None, cu_seqlens=None, stream=None):
    n, per_seq, b = _loss_common(logp, behav_logp, versions, adv, mask, cu_seqlens)
    _want(grad_logp, torch.float32, "grad_logp"); _want(grad_loss, torch.float32, "grad_loss")
    _want(fwd_stats, torch.uint8, "fwd_stats"); _want(ws, torch.uint8, "ws")
    rc = load_library().a3po_loss_bwd(_ptr(logp), _ptr(behav_logp), _ptr(versions), per_seq, _ptr(cu_seqlens), b,
                                      int(current_version), _ptr(adv), _ptr(mask), n, float(clip_eps),
                                      int(bool(detach_prox)), _ptr(grad_loss), _ptr(fwd_stats), _ptr(grad_logp),
                                      _ptr(ws), ws.numel(), _stream(stream))
    _check("a3po_loss_bwd", rc)


def a3po_loss_fwd_bwd(logp, behav_logp, versions, current_version, adv, mask, clip_eps, loss, grad_logp, ws, *,
                      detach_prox=True, stats=None, cu_seqlens=None, stream=None):
    n, per_seq, b = _loss_common(logp, behav_logp, versions, adv, mask, cu_seqlens)
    _want(loss, torch.float32, "loss"); _want(grad_logp, torch.float32, "grad_logp")
    _want(stats, torch.uint8, "stats"); _want(ws, torch.uint8, "ws")
    rc = load_library().a3po_loss_fwd_bwd(_ptr(logp), _ptr(behav_logp), _ptr(versions), per_seq, _ptr(cu_seqlens), b,
                                          int(current_version), _ptr(adv), _ptr(mask), n, float(clip_eps),
                                          int(bool(detach_prox)), _ptr(loss), _ptr(stats), _ptr(grad_logp), _ptr(ws),
                                          ws.numel(), _stream(stream))
    _check("a3po_loss_fwd_bwd", rc)


def a3po_decoupled_loss_fwd_bwd(logp, behav_logp, prox_logp, adv, mask, clip_eps, loss, ws, *, grad_logp=None,
                                stats=None, stream=None):
    """Eq. 2 with an explicit proximal log-prob array (the "recompute" baseline; prox = behav gives Eq. 1)."""
    for t, nm in ((logp, "logp"), (behav_logp, "behav_logp"), (prox_logp, "prox_logp"), (adv, "adv"),
                  (loss, "loss"), (grad_logp, "grad_logp")):
        _want(t, torch.float32, nm)
    _want(mask, torch.uint8, "mask"); _want(stats, torch.uint8, "stats"); _want(ws, torch.uint8, "ws")
    n = logp.numel()
    if not (behav_logp.numel() == prox_logp.numel() == adv.numel() == mask.numel() == n):
        raise ValueError("shape mismatch")
    rc = load_library().a3po_decoupled_loss_fwd_bwd(_ptr(logp), _ptr(behav_logp), _ptr(prox_logp), _ptr(adv),
                                                    _ptr(mask), n, float(clip_eps), _ptr(loss), _ptr(stats),
                                                    _ptr(grad_logp), _ptr(ws), ws.numel(), _stream(stream))
    _check("a3po_decoupled_loss_fwd_bwd", rc)


def a3po_grpo_workspace_bytes(B) -> int:
    return load_library().a3po_grpo_workspace_bytes(B)


def a3po_grpo_advantages(rewards, group_size, cu_seqlens, adv, ws, *, norm_eps=1e-6, stream=None):
    """adv[t] = group-normalised reward of the sequence that owns row t."""
    _want(rewards, torch.float32, "rewards"); _want(cu_seqlens, torch.int32, "cu_seqlens")
    _want(adv, torch.float32, "adv"); _want(ws, torch.uint8, "ws")
    b = rewards.numel()
    if cu_seqlens.numel() != b + 1:
        raise ValueError("cu_seqlens must have B + 1 entries")
    rc = load_library().a3po_grpo_advantages(_ptr(rewards), b, int(group_size), _ptr(cu_seqlens), adv.numel(),
                                             float(norm_eps), _ptr(adv), _ptr(ws), ws.numel(), _stream(stream))
    _check("a3po_grpo_advantages", rc)


def a3po_selftest_wait_timeout(status, timeout_ms=50, stream=None):
    """Runs the bounded-wait self-test kernel; afterwards `status` must hold STATUS_WAIT_TIMEOUT."""
    _want(status, torch.int32, "status")
    _check("a3po_selftest_wait_timeout",
           load_library().a3po_selftest_wait_timeout(_ptr(status), int(timeout_ms), _stream(stream)))


# ------------------------------------------------------------------------------ whole step, device inputs
def a3po_train_step_min_workspace_bytes(N, H, V, dt) -> int:
    return load_library().a3po_train_step_min_workspace_bytes(N, H, V, dt)


def a3po_train_step(hidden, w, targets, behav_logp, versions, current_version, adv, mask, clip_eps, logp, lse,
                    grad_logp, loss, grad_hidden, grad_w, ws, *, stats=None, entropy=None, loss_scale=None,
                    accumulate_grad_w=False, inv_temperature=1.0, status=None, stream=None):
    """token_logprobs_fwd -> loss_fwd_bwd -> token_logprobs_bwd in one call; with the recommended workspace the
    backward reuses the softmax kept by the forward instead of recomputing the logits."""
    dt = _dtype_code(hidden)
    _want(hidden, hidden.dtype, "hidden"); _want(w, hidden.dtype, "w"); _want(grad_hidden, hidden.dtype, "grad_hidden")
    _want(targets, torch.int32, "targets"); _want(versions, torch.int32, "versions"); _want(mask, torch.uint8, "mask")
    for t, nm in ((behav_logp, "behav_logp"), (adv, "adv"), (logp, "logp"), (lse, "lse"), (grad_logp, "grad_logp"),
                  (loss, "loss"), (grad_w, "grad_w")):
        _want(t, torch.float32, nm)
    _want(stats, torch.uint8, "stats"); _want(status, torch.int32, "status"); _want(ws, torch.uint8, "ws")
    _want(entropy, torch.float32, "entropy"); _want(loss_scale, torch.float32, "loss_scale")
    n, h = hidden.shape
    v = w.shape[0]
    if w.shape[1] != h or grad_w.shape != w.shape or grad_hidden.shape != hidden.shape:
        raise ValueError("shape mismatch")
    for t in (targets, behav_logp, versions, adv, mask, logp, lse, grad_logp) + ((entropy,) if entropy is not None
                                                                                  else ()):
        if t.numel() != n:
            raise ValueError("per-token arrays must have N entries")
    rc = load_library().a3po_train_step(
        _ptr(hidden), _ptr(targets), _ptr(behav_logp), _ptr(versions), _ptr(adv), _ptr(mask), n, h, v, dt,
        int(current_version), float(clip_eps), float(inv_temperature), _ptr(w), _ptr(grad_w),
        int(bool(accumulate_grad_w)), _ptr(grad_hidden), _ptr(logp), _ptr(lse), _ptr(entropy), _ptr(grad_logp),
        _ptr(loss), _ptr(stats), _ptr(loss_scale), _ptr(ws), ws.numel(), _ptr(status), _stream(stream))
    _check("a3po_train_step", rc)


# ------------------------------------------------------------------------------ data-parallel helpers
def a3po_mask_count_workspace_bytes() -> int:
    return load_library().a3po_mask_count_workspace_bytes()


def a3po_mask_count(mask, count, ws, *, stream=None):
    """count (int64 device tensor, 1 element) = number of non-zero mask bytes."""
    _want(mask, torch.uint8, "mask"); _want(count, torch.int64, "count"); _want(ws, torch.uint8, "ws")
    _check("a3po_mask_count", load_library().a3po_mask_count(_ptr(mask), mask.numel(), _ptr(count), _ptr(ws),
                                                             ws.numel(), _stream(stream)))


def a3po_dp_loss_scale(m_local, m_global, scale, *, loss_local=None, weighted_loss=None, stream=None):
    """scale = M_local / M_global; with loss_local also weighted_loss = scale * loss_local (device scalars)."""
    _want(m_local, torch.int64, "m_local"); _want(m_global, torch.int64, "m_global")
    _want(scale, torch.float32, "scale"); _want(loss_local, torch.float32, "loss_local")
    _want(weighted_loss, torch.float32, "weighted_loss")
    _check("a3po_dp_loss_scale", load_library().a3po_dp_loss_scale(_ptr(m_local), _ptr(m_global), _ptr(loss_local),
                                                                   _ptr(scale), _ptr(weighted_loss), _stream(stream)))


# ------------------------------------------------------------------------------ whole step, host inputs
def a3po_train_step_host(h_hidden, h_targets, h_behav_logp, h_versions, h_adv, h_mask, current_version, clip_eps,
                         d_w, d_grad_w, d_grad_hidden, d_stage, d_ws, h_loss, *, h_stats=None, accumulate_grad_w=False,
                         inv_temperature=1.0, d_status=None, stream=None):
    dt = _dtype_code(h_hidden)
    for t, ty, nm in ((h_hidden, h_hidden.dtype, "h_hidden"), (h_targets, torch.int32, "h_targets"),
                      (h_behav_logp, torch.float32, "h_behav_logp"), (h_versions, torch.int32, "h_versions"),
                      (h_adv, torch.float32, "h_adv"), (h_mask, torch.uint8, "h_mask"),
                      (h_loss, torch.float32, "h_loss"), (h_stats, torch.uint8, "h_stats")):
        _want(t, ty, nm, device_type="cpu")
    _want(d_w, h_hidden.dtype, "d_w"); _want(d_grad_w, torch.float32, "d_grad_w")
    _want(d_grad_hidden, h_hidden.dtype, "d_grad_hidden"); _want(d_stage, torch.uint8, "d_stage")
    _want(d_ws, torch.uint8, "d_ws"); _want(d_status, torch.int32, "d_status")
    n, h = h_hidden.shape
    v = d_w.shape[0]
    rc = load_library().a3po_train_step_host(
        _ptr(h_hidden), _ptr(h_targets), _ptr(h_behav_logp), _ptr(h_versions), _ptr(h_adv), _ptr(h_mask), n, h, v, dt,
        int(current_version), float(clip_eps), float(inv_temperature), _ptr(d_w), _ptr(d_grad_w),
        int(bool(accumulate_grad_w)), _ptr(d_grad_hidden), _ptr(d_stage), d_stage.numel(), _ptr(d_ws), d_ws.numel(),
        _ptr(h_loss), _ptr(h_stats), _ptr(d_status), _stream(stream))
    _check("a3po_train_step_host", rc)


# ------------------------------------------------------------------------------ rows in front of the LM head
def _here(*tensors):
    """Every tensor is on the current CUDA device, whose stream the kernels are launched on."""
    device = None
    for t in tensors:
        if t is not None:
            if not t.is_cuda:
                raise TypeError(f"expected a tensor on a CUDA device, got {t.device}")
            if device is None:
                device = torch.cuda.current_device()
            if t.get_device() != device:
                raise ValueError(f"expected tensors on the current device cuda:{device}, got {t.device}")


def _rows(x, mats, vecs=(), per_row=(), row_mask=None):
    """dtype code, N and H of the row operators' matrices [N, H], parameters [H] and per-row scalars [N], after checking
    that they belong together and that the kernels will run where the tensors are.  (Small calls are bound by the host:
    the checks look at each tensor once and say what is wrong only when something is.)"""
    dtype, shape, device = x.dtype, x.shape, x.get_device()
    n, h = shape
    fine = device >= 0 and device == torch.cuda.current_device() and x.is_contiguous()
    for t in mats:
        if t is not None:
            fine &= t.dtype is dtype and t.get_device() == device and t.shape == shape and t.is_contiguous()
    for t in vecs:
        if t is not None:
            fine &= t.get_device() == device and t.numel() == h
    for t in per_row:
        if t is not None:
            fine &= t.dtype is torch.float32 and t.get_device() == device and t.numel() == n and t.is_contiguous()
    if row_mask is not None:
        fine &= (row_mask.dtype is torch.uint8 and row_mask.get_device() == device and row_mask.numel() == n
                 and row_mask.is_contiguous())
    if not fine:
        _here(x, *mats, *vecs, *per_row, row_mask)
        for t in (x, *mats):
            _want(t, dtype, "matrix")
        for t in per_row:
            _want(t, torch.float32, "per-row scalar")
        _want(row_mask, torch.uint8, "row_mask")
        raise ValueError("shape mismatch")
    return _dtype_code(x), n, h


def _rng_words(rng, p):
    """{seed, offset}: an int64 device tensor of two words (their bits are taken as uint64)."""
    if rng is None:
        if p > 0:
            raise ValueError("rng: {seed, offset} needed for p > 0")
        return
    _here(rng)
    _want(rng, torch.int64, "rng")
    if rng.numel() != 2:
        raise ValueError("rng: expected the two words {seed, offset}")


def a3po_norm_bwd_workspace_bytes(N, H) -> int:
    return load_library().a3po_norm_bwd_workspace_bytes(N, H)


def a3po_norm_fwd(x, gamma, y, rstd=None, *, kind=A3PO_NORM_RMS, beta=None, mean=None, eps=1e-6, row_mask=None,
                  stream=None):
    """y = norm(x) gamma + beta; mean / rstd (fp32 [N]) are left for the backward when given."""
    dt, n, h = _rows(x, (y,), (gamma, beta), (mean, rstd), row_mask)
    _want(gamma, x.dtype, "gamma"); _want(beta, x.dtype, "beta")
    rc = load_library().a3po_norm_fwd(_ptr(x), _ptr(gamma), _ptr(beta), _ptr(row_mask), n, h, dt, kind, float(eps), _ptr(y),
                                      _ptr(mean), _ptr(rstd), _stream(stream))
    _check("a3po_norm_fwd", rc)


def a3po_norm_bwd(x, gamma, rstd, grad_y, grad_x, grad_gamma, ws, *, kind=A3PO_NORM_RMS, mean=None, grad_beta=None,
                  accumulate_grad_w=False, row_mask=None, stream=None):
    dt, n, h = _rows(x, (grad_y, grad_x), (gamma, grad_gamma, grad_beta), (mean, rstd), row_mask)
    _want(gamma, x.dtype, "gamma"); _want(grad_gamma, torch.float32, "grad_gamma")
    _want(grad_beta, torch.float32, "grad_beta"); _want(ws, torch.uint8, "ws"); _here(ws)
    rc = load_library().a3po_norm_bwd(_ptr(x), _ptr(gamma), _ptr(mean), _ptr(rstd), _ptr(row_mask), _ptr(grad_y), n, h,
                                      dt, kind, _ptr(grad_x), _ptr(grad_gamma), _ptr(grad_beta),
                                      int(bool(accumulate_grad_w)), _ptr(ws), ws.numel(), _stream(stream))
    _check("a3po_norm_bwd", rc)


def a3po_dropout_fwd(x, p, rng, y, *, residual=None, row_mask=None, stream=None):
    """y = residual + dropout(x); the mask is a function of rng = {seed, offset} and the element's place."""
    dt, n, h = _rows(x, (residual, y), row_mask=row_mask)
    _rng_words(rng, p)
    rc = load_library().a3po_dropout_fwd(_ptr(x), _ptr(residual), _ptr(row_mask), n, h, dt, float(p), _ptr(rng), _ptr(y),
                                         _stream(stream))
    _check("a3po_dropout_fwd", rc)


def a3po_dropout_bwd(grad_y, p, rng, grad_x, *, row_mask=None, stream=None):
    dt, n, h = _rows(grad_y, (grad_x,), row_mask=row_mask)
    _rng_words(rng, p)
    rc = load_library().a3po_dropout_bwd(_ptr(grad_y), _ptr(row_mask), n, h, dt, float(p), _ptr(rng), _ptr(grad_x),
                                         _stream(stream))
    _check("a3po_dropout_bwd", rc)


def a3po_dropout_norm_fwd(x, residual, p, rng, gamma, r, y, rstd=None, *, kind=A3PO_NORM_RMS, beta=None, mean=None,
                          eps=1e-6, row_mask=None, stream=None):
    """r = residual + dropout(x), y = norm(r) gamma + beta, in one pass."""
    dt, n, h = _rows(x, (residual, r, y), (gamma, beta), (mean, rstd), row_mask)
    _want(gamma, x.dtype, "gamma"); _want(beta, x.dtype, "beta"); _rng_words(rng, p)
    rc = load_library().a3po_dropout_norm_fwd(_ptr(x), _ptr(residual), float(p), _ptr(rng), _ptr(gamma), _ptr(beta),
                                              _ptr(row_mask), n, h, dt, kind, float(eps), _ptr(r), _ptr(y), _ptr(mean),
                                              _ptr(rstd), _stream(stream))
    _check("a3po_dropout_norm_fwd", rc)


def a3po_dropout_norm_bwd(r, p, rng, gamma, rstd, grad_y, grad_residual, grad_x, grad_gamma, ws, *,
                          kind=A3PO_NORM_RMS, mean=None, grad_r=None, grad_beta=None, accumulate_grad_w=False,
                          row_mask=None, stream=None):
    """Gradients of the join from its stored sum r; grad_x = None: the branch's gradient is not wanted."""
    dt, n, h = _rows(r, (grad_y, grad_r, grad_residual, grad_x), (gamma, grad_gamma, grad_beta), (mean, rstd), row_mask)
    _want(gamma, r.dtype, "gamma"); _want(grad_gamma, torch.float32, "grad_gamma")
    _want(grad_beta, torch.float32, "grad_beta"); _want(ws, torch.uint8, "ws"); _here(ws); _rng_words(rng, p)
    rc = load_library().a3po_dropout_norm_bwd(_ptr(r), float(p), _ptr(rng), _ptr(gamma), _ptr(mean), _ptr(rstd),
                                              _ptr(row_mask), _ptr(grad_y), _ptr(grad_r), n, h, dt, kind,
                                              _ptr(grad_residual), _ptr(grad_x), _ptr(grad_gamma), _ptr(grad_beta),
                                              int(bool(accumulate_grad_w)), _ptr(ws), ws.numel(), _stream(stream))
    _check("a3po_dropout_norm_bwd", rc)


# ------------------------------------------------------------------------------ gated feed-forward block
def a3po_gated_ffn_kept_bytes(N, F, dt) -> int:
    return load_library().a3po_gated_ffn_kept_bytes(N, F, dt)


def a3po_gated_ffn_workspace_bytes(N, H, F, dt, has_row_mask, is_bwd) -> int:
    return load_library().a3po_gated_ffn_workspace_bytes(N, H, F, dt, int(bool(has_row_mask)), int(bool(is_bwd)))


def _ffn_weights(x, w_gate_up, w_down, h):
    _want(w_gate_up, x.dtype, "w_gate_up"); _want(w_down, x.dtype, "w_down")
    f = w_down.shape[1]
    if tuple(w_gate_up.shape) != (2 * f, h) or w_down.shape[0] != h:
        raise ValueError("shape mismatch")
    return f


def a3po_gated_ffn_fwd(x, w_gate_up, w_down, y, ws, *, row_mask=None, kept=None, activation=A3PO_ACT_SILU, status=None,
                       stream=None):
    """y = (act(x Wg^T) * (x Wu^T)) Wd^T; w_gate_up stacks Wg and Wu.  `kept` (uint8 buffer of
    a3po_gated_ffn_kept_bytes) is filled for a3po_gated_ffn_bwd when given."""
    dt, n, h = _rows(x, (y,), row_mask=row_mask)
    f = _ffn_weights(x, w_gate_up, w_down, h)
    _here(w_gate_up, w_down, kept, ws, status)
    _want(kept, torch.uint8, "kept"); _want(ws, torch.uint8, "ws"); _want(status, torch.int32, "status")
    rc = load_library().a3po_gated_ffn_fwd(_ptr(x), _ptr(w_gate_up), _ptr(w_down), _ptr(row_mask), n, h, f, dt, activation,
                                           _ptr(y), _ptr(kept), 0 if kept is None else kept.numel(), _ptr(ws), ws.numel(),
                                           _ptr(status), _stream(stream))
    _check("a3po_gated_ffn_fwd", rc)


def a3po_gated_ffn_bwd(x, w_gate_up, w_down, kept, grad_y, grad_x, grad_w_gate_up, grad_w_down, ws, *, row_mask=None,
                       activation=A3PO_ACT_SILU, accumulate_grad_w=False, status=None, stream=None):
    """Gradients of a3po_gated_ffn_fwd from what it kept; the weight gradients are fp32 or of the weights' type."""
    dt, n, h = _rows(x, (grad_y, grad_x), row_mask=row_mask)
    f = _ffn_weights(x, w_gate_up, w_down, h)
    _here(w_gate_up, w_down, kept, grad_w_gate_up, grad_w_down, ws, status)
    gdt = _dtype_code(grad_w_down)
    _want(grad_w_gate_up, grad_w_down.dtype, "grad_w_gate_up"); _want(grad_w_down, grad_w_down.dtype, "grad_w_down")
    _want(kept, torch.uint8, "kept"); _want(ws, torch.uint8, "ws"); _want(status, torch.int32, "status")
    if grad_w_gate_up.shape != w_gate_up.shape or grad_w_down.shape != w_down.shape:
        raise ValueError("shape mismatch")
    rc = load_library().a3po_gated_ffn_bwd(_ptr(x), _ptr(w_gate_up), _ptr(w_down), _ptr(row_mask), _ptr(kept),
                                           kept.numel(), _ptr(grad_y), n, h, f, dt, activation, _ptr(grad_x),
                                           _ptr(grad_w_gate_up), _ptr(grad_w_down), gdt, int(bool(accumulate_grad_w)),
                                           _ptr(ws), ws.numel(), _ptr(status), _stream(stream))
    _check("a3po_gated_ffn_bwd", rc)


# ------------------------------------------------------------------------------ linear operator
def a3po_linear_kept_bytes(N, M, dt, activation=A3PO_ACT_NONE) -> int:
    return load_library().a3po_linear_kept_bytes(N, M, dt, activation)


def a3po_linear_workspace_bytes(N, K, M, dt, activation=A3PO_ACT_NONE, has_row_mask=False, is_bwd=False) -> int:
    return load_library().a3po_linear_workspace_bytes(N, K, M, dt, activation, int(bool(has_row_mask)), int(bool(is_bwd)))


def _linear_shapes(x, w, same, f32, others, row_mask):
    """dtype code, N, K and M after checking x [N, K], w [M, K] and, as (tensor, shape, elements): `same` of x's type, `f32` of
    fp32 (`others`: a tensor's own type), all contiguous on the current device."""
    dt = _dtype_code(x)
    if x.dim() != 2 or w.dim() != 2 or w.shape[1] != x.shape[1]:
        raise ValueError("shape mismatch")
    (n, k), m = x.shape, w.shape[0]
    device, dtype = x.get_device(), x.dtype
    fine = (device >= 0 and device == torch.cuda.current_device() and x.is_contiguous() and w.dtype is dtype
            and w.get_device() == device and w.is_contiguous())
    sizes = {"nk": (n, k), "nm": (n, m), "mk": (m, k), "m": (m,)}
    for tensors, ty in ((same, dtype), (f32, torch.float32), (others, None)):
        for t, size in tensors:
            if t is not None:
                fine &= ((ty is None or t.dtype is ty) and t.get_device() == device and t.is_contiguous()
                         and (size == "" or (t.numel() == m if size == "m" else t.shape == sizes[size])))
    if row_mask is not None:
        fine &= (row_mask.dtype is torch.uint8 and row_mask.get_device() == device and row_mask.numel() == n
                 and row_mask.is_contiguous())
    if not fine:   # say what is wrong
        every = [t for t, _ in same + f32 + others]
        _here(x, w, *every, row_mask)
        _want(x, dtype, "x"); _want(w, dtype, "w"); _want(row_mask, torch.uint8, "row_mask")
        for tensors, ty in ((same, dtype), (f32, torch.float32)):
            for t, _ in tensors:
                _want(t, ty, "matrix or vector")
        for t, _ in others:
            if t is not None:
                _want(t, t.dtype, "matrix or buffer")
        raise ValueError("shape mismatch")
    return dt, n, k, m


def a3po_linear_fwd(x, w, y, ws, *, bias=None, residual=None, row_mask=None, kept=None, activation=A3PO_ACT_NONE,
                    status=None, stream=None):
    """y = act(x w^T + bias) + residual; y has x's type or is fp32.  `kept` (uint8 buffer of a3po_linear_kept_bytes) is filled for
    a3po_linear_bwd when given; without an activation there is nothing to keep."""
    own = ((residual, "nm"), (bias, "m"))
    f32, same = (((y, "nm"),), own) if y.dtype is torch.float32 else ((), own + ((y, "nm"),))
    dt, n, k, m = _linear_shapes(x, w, same, f32, ((kept, ""), (ws, ""), (status, "")), row_mask)
    if (kept is not None and kept.dtype is not torch.uint8) or ws.dtype is not torch.uint8 or (
            status is not None and status.dtype is not torch.int32):
        raise TypeError("kept and ws: expected uint8 buffers; status: int32")
    rc = load_library().a3po_linear_fwd(_ptr(x), _ptr(w), _ptr(bias), _ptr(residual), _ptr(row_mask), n, k, m, dt, activation,
                                        _ptr(y), _dtype_code(y), _ptr(kept), 0 if kept is None else kept.numel(), _ptr(ws),
                                        ws.numel(), _ptr(status), _stream(stream))
    _check("a3po_linear_fwd", rc)


def a3po_linear_bwd(x, w, grad_y, grad_x, grad_w, ws, *, kept=None, grad_bias=None, row_mask=None,
                    activation=A3PO_ACT_NONE, accumulate_grad_w=False, status=None, stream=None):
    """Gradients of a3po_linear_fwd; grad_x, grad_w or both may be None.  grad_w is fp32 or of the weights' type, grad_bias fp32;
    the residual's gradient is grad_y itself."""
    gdt = A3PO_F32 if grad_w is None else _dtype_code(grad_w)
    dt, n, k, m = _linear_shapes(x, w, ((grad_y, "nm"), (grad_x, "nk")), ((grad_bias, "m"),),
                                 ((grad_w, "mk"), (kept, ""), (ws, ""), (status, "")), row_mask)
    if (kept is not None and kept.dtype is not torch.uint8) or ws.dtype is not torch.uint8 or (
            status is not None and status.dtype is not torch.int32):
        raise TypeError("kept and ws: expected uint8 buffers; status: int32")
    rc = load_library().a3po_linear_bwd(_ptr(x), _ptr(w), _ptr(row_mask), _ptr(kept), 0 if kept is None else kept.numel(),
                                        _ptr(grad_y), n, k, m, dt, activation, _ptr(grad_x), _ptr(grad_w), gdt,
                                        _ptr(grad_bias), int(bool(accumulate_grad_w)), _ptr(ws), ws.numel(), _ptr(status),
                                        _stream(stream))
    _check("a3po_linear_bwd", rc)


# ------------------------------------------------------------------------------ sampling
def a3po_sample_workspace_bytes(N, V) -> int:
    return load_library().a3po_sample_workspace_bytes(N, V)


def a3po_sample(logits, u, token, ws, *, temperature=None, top_k=None, top_p=None, min_p=None, row_mask=None, logp=None,
                kept_logp=None, n_kept=None, stream=None):
    """One token per row of logits [N, V] (rows may lie apart) from given random numbers u in [0, 1); token -1: nothing to
    sample.  logp: of the whole softmax (the behaviour log-prob of the loss), kept_logp: among the tokens that the filters
    kept, n_kept of them.  temperature, top_p, min_p (fp32) and top_k (int32): one value per row, or None."""
    if logits.dim() != 2:
        raise ValueError("logits: expected [N, V]")
    n, v = logits.shape
    ld, step = logits.stride()
    device = logits.get_device()
    fine = (device >= 0 and device == torch.cuda.current_device() and (step == 1 or v == 1) and (ld >= v or n <= 1)
            and ws.dtype is torch.uint8 and ws.get_device() == device and ws.is_contiguous())
    for t in (u, temperature, top_p, min_p, logp, kept_logp):
        if t is not None:
            fine &= t.dtype is torch.float32 and t.get_device() == device and t.numel() == n and t.is_contiguous()
    for t in (token, top_k, n_kept):
        if t is not None:
            fine &= t.dtype is torch.int32 and t.get_device() == device and t.numel() == n and t.is_contiguous()
    if row_mask is not None:
        fine &= (row_mask.dtype is torch.uint8 and row_mask.get_device() == device and row_mask.numel() == n
                 and row_mask.is_contiguous())
    dt = _dtype_code(logits)
    if not fine:   # say what is wrong
        if not logits.is_cuda or (v > 1 and step != 1) or (n > 1 and ld < v):
            raise TypeError("logits: expected rows of neighbouring elements on cuda")
        _here(logits, u, token, ws, temperature, top_k, top_p, min_p, row_mask, logp, kept_logp, n_kept)
        for t, ty, nm in ((u, torch.float32, "u"), (token, torch.int32, "token"), (temperature, torch.float32, "temperature"),
                          (top_k, torch.int32, "top_k"), (top_p, torch.float32, "top_p"), (min_p, torch.float32, "min_p"),
                          (row_mask, torch.uint8, "row_mask"), (logp, torch.float32, "logp"),
                          (kept_logp, torch.float32, "kept_logp"), (n_kept, torch.int32, "n_kept")):
            _want(t, ty, nm)
        _want(ws, torch.uint8, "ws")
        raise ValueError("expected one value per row")
    rc = load_library().a3po_sample(_ptr(logits), ld if n > 1 else v, _ptr(row_mask), n, v, dt,
                                    _ptr(temperature), _ptr(top_k), _ptr(top_p), _ptr(min_p), _ptr(u), _ptr(token),
                                    _ptr(logp), _ptr(kept_logp), _ptr(n_kept), _ptr(ws), ws.numel(), _stream(stream))
    _check("a3po_sample", rc)


# ------------------------------------------------------------------------------ AdamW
def a3po_adamw_workspace_bytes(count) -> int:
    return load_library().a3po_adamw_workspace_bytes(count)


def a3po_adamw_step(table, weight_dt, grad_dt, state_bits, lr, step, ws, *, beta1=0.9, beta2=0.999, eps=1e-8,
                    max_grad_norm=0.0, grad_norm=None, stream=None):
    """One AdamW step over the tensors of `table`, a ctypes array of A3poAdamWTensor (optimizer.AdamW builds it from
    tensors, which it checks)."""
    _here(lr, step, ws, grad_norm)
    _want(lr, torch.float32, "lr"); _want(step, torch.int64, "step"); _want(ws, torch.uint8, "ws")
    _want(grad_norm, torch.float32, "grad_norm")
    if lr.numel() != 1 or step.numel() != 1 or (grad_norm is not None and grad_norm.numel() != 1):
        raise ValueError("lr, step and grad_norm: expected one element")
    rc = load_library().a3po_adamw_step(ctypes.addressof(table), len(table), weight_dt, grad_dt, state_bits, beta1, beta2,
                                        eps, max_grad_norm, _ptr(lr), _ptr(step), _ptr(grad_norm), _ptr(ws), ws.numel(),
                                        _stream(stream))
    _check("a3po_adamw_step", rc)


def a3po_adamw_state_values(codes, scales, values, *, signed, stream=None):
    """values (fp32) = what the bytes of an 8-bit optimizer state stand for."""
    _here(codes, scales, values)
    _want(codes, torch.uint8, "codes"); _want(scales, torch.float32, "scales"); _want(values, torch.float32, "values")
    n = codes.numel()
    if values.numel() != n or scales.numel() != -(-n // 256):
        raise ValueError("shape mismatch")
    _check("a3po_adamw_state_values",
           load_library().a3po_adamw_state_values(_ptr(codes), _ptr(scales), n, int(bool(signed)), _ptr(values),
                                                  _stream(stream)))

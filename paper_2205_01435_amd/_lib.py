"""ctypes binding of libwm.so: argument marshalling only.

Every step of the hot path runs in the HIP library; this module turns torch
device tensors into pointers, allocates caller-owned buffers with torch, and
raises ``WmError`` on a non-OK status.  There is no fallback: if libwm.so is
missing or fails to load, every entry point raises.
"""

from __future__ import annotations

import ctypes
import math
import os
from dataclasses import dataclass

import torch
from torch._C._dynamo.guards import TensorGuards

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libwm.so")

WM_OK, WM_ERR_INVALID_ARG, WM_ERR_UNSUPPORTED, WM_ERR_WORKSPACE, WM_ERR_HIP = 0, -1, -2, -3, -4
WM_FP32, WM_BF16 = 0, 1
WM_FLAG_DONE, WM_FLAG_TRACE, WM_FLAG_CHECK, WM_FLAG_STEP_MASK, WM_FLAG_SIGMA_TAU = 1, 2, 4, 8, 16
WM_FLAG_TEST_ABORT = 0x80000000
WS_ROLLOUT, WS_NLL, WS_CONTROLLER, WS_NLL_GRAD = 0, 1, 2, 3
_DTYPES = {"fp32": WM_FP32, "bf16": WM_BF16}

# Every symbol the C header declares.
EXPORTS = ("wm_packed_weights_bytes", "wm_pack_weights", "wm_workspace_bytes", "wm_controller_step",
           "wm_rollout", "wm_rollout_noalloc", "wm_nll", "wm_nll_grad", "wm_returns", "wm_adam_step", "wm_poly_lr",
           "wm_embed", "wm_embed_grad_workspace_bytes", "wm_embed_grad", "wm_layer_norm",
           "wm_layer_norm_grad_workspace_bytes", "wm_layer_norm_grad", "wm_linrec_states_bytes",
           "wm_linrec_workspace_bytes", "wm_linrec", "wm_linrec_grad", "wm_clip_grads_workspace_bytes",
           "wm_clip_grads", "wm_rotary_table", "wm_qk_norm", "wm_qk_norm_grad_workspace_bytes", "wm_qk_norm_grad",
           "wm_linattn_states_bytes", "wm_linattn_workspace_bytes", "wm_linattn", "wm_linattn_grad", "wm_glu_saved_bytes",
           "wm_glu",
           "wm_glu_grad_workspace_bytes", "wm_glu_grad",
           "wm_profile_enable", "wm_profile_read", "wm_profile_reset", "wm_profile_phases",
           "wm_profile_phases_read", "wm_workspace_status",
           "wm_last_error", "wm_version")


class WmError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"libwm status {status}: {msg}")
        self.status = status


class CDims(ctypes.Structure):
    _fields_ = [("Z", ctypes.c_int32), ("H", ctypes.c_int32), ("A", ctypes.c_int32),
                ("K", ctypes.c_int32), ("dtype", ctypes.c_int32), ("N", ctypes.c_int32),
                ("L", ctypes.c_int32)]


class CWeights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("W_g", "b_g", "W_m", "b_m", "w_r", "b_r", "w_d", "b_d", "W_c", "b_c")]


class CGradTensor(ctypes.Structure):
    _fields_ = [("grad", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n", ctypes.c_int64),
                ("dtype", ctypes.c_int32)]


_lib = None


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libwm.so (once) and declare the C signatures."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise WmError(WM_ERR_UNSUPPORTED,
                      f"{path} is missing: build it with `python -m paper_2205_01435_amd.build`")
    lib = ctypes.CDLL(path)
    P, I32, U32, U64, F32, SZ = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint32,
                                 ctypes.c_uint64, ctypes.c_float, ctypes.c_size_t)
    pd = ctypes.POINTER(CDims)
    lib.wm_packed_weights_bytes.argtypes = [pd]
    lib.wm_packed_weights_bytes.restype = SZ
    lib.wm_pack_weights.argtypes = [pd, ctypes.POINTER(CWeights), P, SZ, P]
    lib.wm_pack_weights.restype = I32
    lib.wm_workspace_bytes.argtypes = [pd, I32, I32, I32]
    lib.wm_workspace_bytes.restype = SZ
    lib.wm_controller_step.argtypes = [pd, P, I32, U32, P, P, P, U64, U32, P, P, P]
    lib.wm_controller_step.restype = I32
    lib.wm_rollout.argtypes = [pd, P, I32, I32, U32, U32, P, P, P, P, P, P, U64, F32, U32,
                               P, P, P, P, P, P, P, P, P, SZ, P]
    lib.wm_rollout.restype = I32
    lib.wm_rollout_noalloc.argtypes = [pd, P, I32, I32, U32, U32, P, P, P, P, P, P, U64, F32, U32,
                                       P, P, P, P, P, P, P, P, P]
    lib.wm_rollout_noalloc.restype = I32
    lib.wm_nll.argtypes = [pd, P, I32, I32, P, P, P, P, P, U32, P, P, P, P, P, SZ, P]
    lib.wm_nll.restype = I32
    lib.wm_nll_grad.argtypes = [pd, P, I32, I32, P, P, P, P, P, U32, P, P, P, P, P, P, P, P, P, P, SZ, P]
    lib.wm_nll_grad.restype = I32
    lib.wm_returns.argtypes = [I32, I32, P, P, P, F32, F32, P, P, P]
    lib.wm_returns.restype = I32
    lib.wm_adam_step.argtypes = [ctypes.c_int64, P, P, P, P, I32, F32, F32, F32, F32, P]
    lib.wm_adam_step.restype = I32
    lib.wm_poly_lr.argtypes = [I32, F32, F32, I32]
    lib.wm_poly_lr.restype = F32
    I64, pg = ctypes.c_int64, ctypes.POINTER(CGradTensor)
    lib.wm_embed.argtypes = [I32, I64, I32, I32, P, P, F32, P, I64, P]
    lib.wm_embed.restype = I32
    lib.wm_embed_grad_workspace_bytes.argtypes = [I64, I32, I32]
    lib.wm_embed_grad_workspace_bytes.restype = SZ
    lib.wm_embed_grad.argtypes = [I32, I64, I32, I32, P, P, I64, F32, P, P, SZ, P]
    lib.wm_embed_grad.restype = I32
    lib.wm_layer_norm.argtypes = [I32, I64, I32, P, I64, P, P, F32, P, I64, P, P, P]
    lib.wm_layer_norm.restype = I32
    lib.wm_layer_norm_grad_workspace_bytes.argtypes = [I64, I32]
    lib.wm_layer_norm_grad_workspace_bytes.restype = SZ
    lib.wm_layer_norm_grad.argtypes = [I32, I64, I32, P, I64, P, I64, P, P, P, P, I64, P, P, P, SZ, P]
    lib.wm_layer_norm_grad.restype = I32
    for f in (lib.wm_linrec_states_bytes, lib.wm_linrec_workspace_bytes):
        f.argtypes, f.restype = [I32, I32, I32], SZ
    lib.wm_linrec.argtypes = [I32, I32, I32, I32, P, I64, I64, P, I64, I64, P, P, P, P, P, P, SZ, P, SZ, P]
    lib.wm_linrec.restype = I32
    lib.wm_linrec_grad.argtypes = [I32, I32, I32, I32, P, I64, I64, P, I64, I64, P, P, P, I64, I64, P, P, SZ,
                                   P, I64, I64, P, I64, I64, P, P, SZ, P]
    lib.wm_linrec_grad.restype = I32
    lib.wm_clip_grads_workspace_bytes.argtypes = [I32, pg]
    lib.wm_clip_grads_workspace_bytes.restype = SZ
    lib.wm_clip_grads.argtypes = [I32, pg, F32, P, P, SZ, P]
    lib.wm_clip_grads.restype = I32
    lib.wm_rotary_table.argtypes = [I32, ctypes.c_double, P]
    lib.wm_rotary_table.restype = I32
    lib.wm_qk_norm.argtypes = [I32, I64, I32, I32, I32, I32, I32, P, I64, P, I64, P, P, F32, P, P, P, I64, P, I64, P]
    lib.wm_qk_norm.restype = I32
    lib.wm_qk_norm_grad_workspace_bytes.argtypes = [I64, I32, I32, I32]
    lib.wm_qk_norm_grad_workspace_bytes.restype = SZ
    lib.wm_qk_norm_grad.argtypes = [I32, I64, I32, I32, I32, I32, I32, P, I64, P, I64, P, P, F32, P, P, P, I64, P, I64,
                                    P, I64, P, I64, P, P, P, SZ, P]
    lib.wm_qk_norm_grad.restype = I32
    for f in (lib.wm_linattn_states_bytes, lib.wm_linattn_workspace_bytes):
        f.argtypes, f.restype = [I32, I32, I32, I32, I32], SZ
    lib.wm_linattn.argtypes = [I32, I32, I32, I32, I32, I32, P, I64, I64, P, I64, I64, P, I64, I64, P, F32, P, P, P, P, P,
                               P, SZ, P, SZ, P]
    lib.wm_linattn.restype = I32
    lib.wm_linattn_grad.argtypes = [I32, I32, I32, I32, I32, I32, P, I64, I64, P, I64, I64, P, I64, I64, P, F32, P, P, P,
                                    P, I64, I64, P, P, SZ, P, I64, I64, P, I64, I64, P, I64, I64, P, P, SZ, P]
    lib.wm_linattn_grad.restype = I32
    lib.wm_glu_saved_bytes.argtypes = [I32, I64, I32, I32]
    lib.wm_glu_saved_bytes.restype = SZ
    lib.wm_glu.argtypes = [I32, I64, I32, I32, I32, P, I64, P, P, I64, P, SZ, P]
    lib.wm_glu.restype = I32
    lib.wm_glu_grad_workspace_bytes.argtypes = [I32, I64, I32, I32]
    lib.wm_glu_grad_workspace_bytes.restype = SZ
    lib.wm_glu_grad.argtypes = [I32, I64, I32, I32, I32, P, I64, P, P, SZ, P, I64, P, I64, P, P, SZ, P]
    lib.wm_glu_grad.restype = I32
    lib.wm_profile_enable.argtypes = [ctypes.c_char_p]
    lib.wm_profile_enable.restype = I32
    lib.wm_profile_read.argtypes = [ctypes.c_char_p, ctypes.POINTER(ctypes.c_double),
                                    ctypes.POINTER(ctypes.c_int64)]
    lib.wm_profile_read.restype = I32
    lib.wm_profile_reset.argtypes = []
    lib.wm_profile_reset.restype = I32
    lib.wm_profile_phases.argtypes = [I32]
    lib.wm_profile_phases.restype = I32
    lib.wm_profile_phases_read.argtypes = [ctypes.POINTER(ctypes.c_double), I32]
    lib.wm_profile_phases_read.restype = I32
    lib.wm_workspace_status.argtypes = [P, P]
    lib.wm_workspace_status.restype = I32
    lib.wm_last_error.argtypes = []
    lib.wm_last_error.restype = ctypes.c_char_p
    lib.wm_version.argtypes = []
    lib.wm_version.restype = ctypes.c_char_p
    _lib = lib
    return lib


def _check(status: int):
    if status != WM_OK:
        raise WmError(status, load().wm_last_error().decode())


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream():
    # the current device's current stream, without building a Stream object
    # (2.7 us of an 11 us call)
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _dev_f32(x, device):
    return torch.as_tensor(x, dtype=torch.float32).to(device).contiguous()


def _need(name, t, dtype, shape, device=None, optional=False):
    """Checks a tensor argument before its pointer crosses the C ABI."""
    if t is None:
        if optional:
            return
        raise ValueError(f"{name} is required")
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, the model on {device}")


def _mask_dtype(t):
    return t.dtype if t is not None and t.dtype in (torch.uint8, torch.bool) else torch.uint8


def status(bufs) -> None:
    """Wait for the current stream and raise WmError if the last call that
    used ``bufs.workspace`` failed on the device (a timed-out barrier wait of
    the persistent kernels, or WM_FLAG_CHECK violations).  A recurrence that
    needs no workspace has nothing that could; the buffers of the other
    sequence-core and attending-core operators hold no status and are
    refused."""
    if isinstance(bufs, (EmbedGradBuffers, LayerNormBuffers, ClipPlan, QkNormBuffers, LinattnBuffers, GluBuffers)):
        raise ValueError(f"{type(bufs).__name__} holds no status")
    if isinstance(bufs, LinrecBuffers) and bufs.ws_bytes == 0:
        torch.cuda.current_stream().synchronize()
        return
    _check(load().wm_workspace_status(_ptr(bufs.workspace), _stream()))


@dataclass
class Model:
    """Packed weights on a device plus their dims."""

    dims: CDims
    packed: torch.Tensor
    Z: int
    H: int
    A: int
    K: int
    dtype: str


def make_dims(Z, H, A, K, dtype="fp32", N=0, L=0) -> CDims:
    """N, L > 0: the two-level controller (N xfers + NO-OP, L locations, A = N L)."""
    return CDims(Z, H, A, K, _DTYPES[dtype], N, L)


def packed_bytes(dims: CDims) -> int:
    return load().wm_packed_weights_bytes(ctypes.byref(dims))


def workspace_bytes(dims: CDims, B: int, T: int, which: int) -> int:
    return load().wm_workspace_bytes(ctypes.byref(dims), B, T, which)


def pack(weights: dict, Z: int, H: int, A: int, K: int, dtype: str = "fp32",
         device="cuda", N: int = 0, L: int = 0) -> Model:
    """Copy canonical float32 weights to the device and pack them (N, L > 0:
    the two-level controller, W_c [N+1+L, Z+H])."""
    lib = load()
    dims = make_dims(Z, H, A, K, dtype, N, L)
    n = lib.wm_packed_weights_bytes(ctypes.byref(dims))
    if n == 0:
        raise WmError(WM_ERR_UNSUPPORTED, lib.wm_last_error().decode())
    canon = {k: _dev_f32(np_or_t, device).reshape(-1) for k, np_or_t in weights.items()}
    packed = torch.empty(n, dtype=torch.uint8, device=device)
    cw = CWeights(*[ctypes.c_void_p(canon[k].data_ptr()) for k in
                    ("W_g", "b_g", "W_m", "b_m", "w_r", "b_r", "w_d", "b_d", "W_c", "b_c")])
    _check(lib.wm_pack_weights(ctypes.byref(dims), ctypes.byref(cw), _ptr(packed), n, _stream()))
    torch.cuda.current_stream().synchronize()  # canon tensors may be freed after return
    return Model(dims, packed, Z, H, A, K, dtype)


def repack(m: Model, canon: dict):
    """Re-pack canonical float32 device tensors (every weight, the
    controller's included) into m.packed on the current stream (after an
    optimiser step); nothing is allocated and nothing waits."""
    lib = load()
    for k in ("W_g", "b_g", "W_m", "b_m", "w_r", "b_r", "w_d", "b_d", "W_c", "b_c"):
        t = canon[k]
        assert t.is_cuda and t.dtype == torch.float32 and t.is_contiguous(), k
    cw = CWeights(*[ctypes.c_void_p(canon[k].data_ptr()) for k in
                    ("W_g", "b_g", "W_m", "b_m", "w_r", "b_r", "w_d", "b_d", "W_c", "b_c")])
    _check(lib.wm_pack_weights(ctypes.byref(m.dims), ctypes.byref(cw), _ptr(m.packed), m.packed.numel(),
                               _stream()))


def two_level_mask(m: Model, xm, lm):
    """The one buffer the library reads for the two-level controller: the
    xfer masks [B, N+1], then the location masks [B, N, L] (uint8)."""
    return _two_level_mask(m, (xm, lm), xm.shape[0])


def _two_level_mask(m: Model, mask, B: int):
    """(xfer mask [B, N+1], location mask [B, N, L]) as the one buffer the
    library reads, xfer masks first; a flat buffer of that layout is taken
    as it is."""
    N, L = m.dims.N, m.dims.L
    dev = m.packed.device
    if isinstance(mask, torch.Tensor):
        _need("two-level mask", mask, _mask_dtype(mask), (B * (N + 1) + B * N * L,), dev)
        return mask
    xm, lm = mask
    _need("xfer mask", xm, _mask_dtype(xm), (B, N + 1), dev)
    _need("location mask", lm, _mask_dtype(lm), (B, N, L), dev)
    return torch.cat([xm.reshape(-1), lm.reshape(-1)]).contiguous()


def controller_step(m: Model, z, h, mask, seed: int, step: int, traj0: int = 0,
                    want_probs: bool = True):
    """Returns (probs or None, action [B] int32).  One-level: probs [B, A].
    Two-level (N > 0): ``mask`` is (xfer mask [B, N+1], location mask
    [B, N, L]) and probs [B, N+1+L] (always returned)."""
    lib = load()
    B = z.shape[0]
    dev = m.packed.device
    _need("z", z, torch.float32, (B, m.Z), dev)
    _need("h", h, torch.float32, (B, m.H), dev)
    if m.dims.N > 0:
        mask = _two_level_mask(m, mask, B)
        probs = torch.empty((B, m.dims.N + 1 + m.dims.L), dtype=torch.float32, device=dev)
    else:
        _need("mask", mask, _mask_dtype(mask), (B, m.A), dev)
        probs = torch.empty((B, m.A), dtype=torch.float32, device=dev) if want_probs else None
    action = torch.empty(B, dtype=torch.int32, device=dev)
    _check(lib.wm_controller_step(ctypes.byref(m.dims), _ptr(m.packed), B, traj0, _ptr(z),
                                  _ptr(h), _ptr(mask), seed, step, _ptr(probs), _ptr(action),
                                  _stream()))
    return probs, action


class RolloutBuffers:
    """Caller-owned device buffers of one rollout shape (reusable across calls)."""

    def __init__(self, m: Model, B: int, T: int, trace: bool = False, final_state: bool = True,
                 workspace: bool = True):
        dev = m.packed.device
        self.B, self.T, self.Z, self.H = B, T, m.Z, m.H
        self.z_out = torch.empty((T + 1, B, m.Z), dtype=torch.float32, device=dev)
        self.actions = torch.empty((T, B), dtype=torch.int32, device=dev)
        self.rewards = torch.empty((T, B), dtype=torch.float32, device=dev)
        self.dones = torch.empty((T, B), dtype=torch.uint8, device=dev)
        self.h_T = torch.empty((B, m.H), dtype=torch.float32, device=dev) if final_state else None
        self.c_T = torch.empty((B, m.H), dtype=torch.float32, device=dev) if final_state else None
        self.h_trace = (torch.empty((T + 1, B, m.H), dtype=torch.float32, device=dev)
                        if trace else None)
        self.c_trace = (torch.empty((T + 1, B, m.H), dtype=torch.float32, device=dev)
                        if trace else None)
        nws = workspace_bytes(m.dims, B, T, WS_ROLLOUT) if workspace else 0
        self.workspace = torch.empty(max(nws, 1), dtype=torch.uint8, device=dev) if workspace else None
        self.ws_bytes = nws


def rollout(m: Model, z0, mask, *, T: int, seed: int, tau: float = 1.0, done: bool = True,
            traj0: int = 0, step0: int = 0, h0=None, c0=None, done_io=None, lengths=None,
            trace: bool = False,
            bufs: RolloutBuffers | None = None, sigma_tau: bool = False, check: bool = False,
            extra_flags: int = 0, noalloc: bool = False) -> RolloutBuffers:
    """Launch wm_rollout on the current stream; returns the filled buffers
    (``lengths`` [B] int32: per-trajectory horizons, later steps padded;
    ``sigma_tau`` sets WM_FLAG_SIGMA_TAU; a [T, B, A] mask sets
    WM_FLAG_STEP_MASK; ``check`` sets WM_FLAG_CHECK, which waits for the
    stream; ``noalloc`` calls wm_rollout_noalloc, whose workspace is the
    library's static device scratch)."""
    lib = load()
    B = z0.shape[0]
    dev = m.packed.device
    _need("z0", z0, torch.float32, (B, m.Z), dev)
    _need("h0", h0, torch.float32, (B, m.H), dev, optional=True)
    _need("c0", c0, torch.float32, (B, m.H), dev, optional=True)
    _need("done_io", done_io, _mask_dtype(done_io), (B,), dev, optional=True)
    _need("lengths", lengths, torch.int32, (B,), dev, optional=True)
    if m.dims.N > 0:
        mask = _two_level_mask(m, mask, B)
        step_mask = False
    else:
        step_mask = mask is not None and mask.dim() == 3
        want = (T, B, m.dims.A) if step_mask else (B, m.dims.A)
        _need("mask", mask, _mask_dtype(mask), want, dev)
    if bufs is None:
        bufs = RolloutBuffers(m, B, T, trace=trace, workspace=not noalloc)
    if T > 0 and ((bufs.B, bufs.T) != (B, T) or bufs.Z != m.Z or bufs.H != m.H):
        raise ValueError(f"buffers for B={bufs.B} T={bufs.T} Z={bufs.Z} H={bufs.H}; the call has "
                         f"B={B} T={T} Z={m.Z} H={m.H}")
    if trace and bufs.h_trace is None:
        raise ValueError("trace=True needs buffers made with trace=True")
    flags = (WM_FLAG_DONE if done else 0) | (WM_FLAG_TRACE if trace else 0) | \
        (WM_FLAG_SIGMA_TAU if sigma_tau else 0) | (WM_FLAG_STEP_MASK if step_mask else 0) | \
        (WM_FLAG_CHECK if check else 0) | extra_flags
    common = (ctypes.byref(m.dims), _ptr(m.packed), B, T, traj0, step0, _ptr(z0), _ptr(h0), _ptr(c0),
              _ptr(done_io), _ptr(lengths), _ptr(mask), seed, tau, flags, _ptr(bufs.z_out), _ptr(bufs.actions),
              _ptr(bufs.rewards), _ptr(bufs.dones), _ptr(bufs.h_T), _ptr(bufs.c_T),
              _ptr(bufs.h_trace if trace else None), _ptr(bufs.c_trace if trace else None))
    if noalloc:
        _check(lib.wm_rollout_noalloc(*common, _stream()))
    else:
        if bufs.workspace is None:
            raise ValueError("these buffers have no workspace (made for wm_rollout_noalloc)")
        _check(lib.wm_rollout(*common, _ptr(bufs.workspace), bufs.ws_bytes, _stream()))
    return bufs


class NllBuffers:
    def __init__(self, m: Model, B: int, T: int):
        dev = m.packed.device
        self.B, self.T = B, T
        self.loglik = torch.empty((T, B), dtype=torch.float32, device=dev)
        self.reward_se = torch.empty((T, B), dtype=torch.float32, device=dev)
        self.done_bce = torch.empty((T, B), dtype=torch.float32, device=dev)
        self.means = torch.empty(3, dtype=torch.float32, device=dev)
        nws = workspace_bytes(m.dims, B, T, WS_NLL)
        self.workspace = torch.empty(max(nws, 1), dtype=torch.uint8, device=dev)
        self.ws_bytes = nws


def _nll_inputs(m: Model, z, actions, rewards, dones, lengths):
    T, B = actions.shape
    dev = m.packed.device
    _need("actions", actions, torch.int32, (T, B), dev)
    _need("z", z, torch.float32, (T + 1, B, m.Z), dev)
    _need("rewards", rewards, torch.float32, (T, B), dev)
    _need("dones", dones, _mask_dtype(dones), (T, B), dev)
    _need("lengths", lengths, torch.int32, (B,), dev, optional=True)
    return T, B


def nll(m: Model, z, actions, rewards, dones, lengths=None,
        bufs: NllBuffers | None = None, check: bool = False, extra_flags: int = 0) -> NllBuffers:
    """Launch wm_nll on the current stream; returns the filled buffers
    (``check`` sets WM_FLAG_CHECK, which waits for the stream)."""
    lib = load()
    T, B = _nll_inputs(m, z, actions, rewards, dones, lengths)
    if bufs is None:
        bufs = NllBuffers(m, B, T)
    if (bufs.B, bufs.T) != (B, T):
        raise ValueError(f"buffers for B={bufs.B} T={bufs.T}; the call has B={B} T={T}")
    flags = (WM_FLAG_CHECK if check else 0) | extra_flags
    _check(lib.wm_nll(ctypes.byref(m.dims), _ptr(m.packed), B, T, _ptr(z), _ptr(actions),
                      _ptr(rewards), _ptr(dones), _ptr(lengths), flags, _ptr(bufs.loglik),
                      _ptr(bufs.reward_se), _ptr(bufs.done_bce), _ptr(bufs.means),
                      _ptr(bufs.workspace), bufs.ws_bytes, _stream()))
    return bufs


GRAD_SHAPES = {  # canonical gradient shapes, as the weights
    "W_g": lambda Z, H, A, K: (4 * H, Z + A + H), "b_g": lambda Z, H, A, K: (4 * H,),
    "W_m": lambda Z, H, A, K: (3 * Z * K, H), "b_m": lambda Z, H, A, K: (3 * Z * K,),
    "w_r": lambda Z, H, A, K: (H,), "b_r": lambda Z, H, A, K: (1,),
    "w_d": lambda Z, H, A, K: (H,), "b_d": lambda Z, H, A, K: (1,),
}


def flat_views(flat, Z: int, H: int, A: int, K: int) -> dict:
    """Views of a flat float32 tensor as the world-model weights, in the
    order of GRAD_SHAPES (the layout of GradBuffers.flat)."""
    out, o = {}, 0
    for k, f in GRAD_SHAPES.items():
        shp = f(Z, H, A, K)
        n = math.prod(shp)
        out[k] = flat[o:o + n].view(shp)
        o += n
    return out


class GradBuffers:
    """Loss, gradients (views of one flat buffer, GRAD_SHAPES order) and the
    workspace of one wm_nll_grad shape."""

    def __init__(self, m: Model, B: int, T: int):
        dev = m.packed.device
        self.B, self.T = B, T
        self.loss = torch.empty(1, dtype=torch.float32, device=dev)
        n = sum(math.prod(f(m.Z, m.H, m.A, m.K)) for f in GRAD_SHAPES.values())
        self.flat = torch.empty(n, dtype=torch.float32, device=dev)
        self.grads = flat_views(self.flat, m.Z, m.H, m.A, m.K)
        nws = workspace_bytes(m.dims, B, T, WS_NLL_GRAD)
        self.workspace = torch.empty(max(nws, 1), dtype=torch.uint8, device=dev)
        self.ws_bytes = nws


def nll_grad(m: Model, z, actions, rewards, dones, lengths=None,
             bufs: GradBuffers | None = None, check: bool = False, extra_flags: int = 0) -> GradBuffers:
    """Launch wm_nll_grad on the current stream: the training loss (summed
    NLL means) and its gradient in the canonical weight layout."""
    lib = load()
    T, B = _nll_inputs(m, z, actions, rewards, dones, lengths)
    if bufs is None:
        bufs = GradBuffers(m, B, T)
    if (bufs.B, bufs.T) != (B, T):
        raise ValueError(f"buffers for B={bufs.B} T={bufs.T}; the call has B={B} T={T}")
    g = bufs.grads
    flags = (WM_FLAG_CHECK if check else 0) | extra_flags
    _check(lib.wm_nll_grad(ctypes.byref(m.dims), _ptr(m.packed), B, T, _ptr(z), _ptr(actions),
                           _ptr(rewards), _ptr(dones), _ptr(lengths), flags, _ptr(bufs.loss),
                           _ptr(g["W_g"]), _ptr(g["b_g"]), _ptr(g["W_m"]), _ptr(g["b_m"]),
                           _ptr(g["w_r"]), _ptr(g["b_r"]), _ptr(g["w_d"]), _ptr(g["b_d"]),
                           _ptr(bufs.workspace), bufs.ws_bytes, _stream()))
    return bufs


def returns(rewards, dones, gamma: float, values=None, lam: float = 1.0, out=None, adv=None):
    """Launch wm_returns on the current stream over device tensors
    rewards [T, B] float32 and dones [T, B] uint8 (values [T+1, B] float32 or
    None).  Returns (returns [T, B], advantages [T, B] or None)."""
    lib = load()
    T, B = rewards.shape
    if out is None:
        out = torch.empty((T, B), dtype=torch.float32, device=rewards.device)
    if values is not None and adv is None:
        adv = torch.empty((T, B), dtype=torch.float32, device=rewards.device)
    _check(lib.wm_returns(B, T, _ptr(rewards), _ptr(dones), _ptr(values), gamma, lam, _ptr(out),
                          _ptr(adv if values is not None else None), _stream()))
    return out, (adv if values is not None else None)


def adam_step(params, grads, m, v, step: int, lr: float, beta1: float = 0.9, beta2: float = 0.999,
              eps: float = 1e-8):
    """Launch wm_adam_step on the current stream over flat float32 device
    tensors of one size (updated in place)."""
    n = params.numel()
    assert grads.numel() == n and m.numel() == n and v.numel() == n
    _check(load().wm_adam_step(n, _ptr(params), _ptr(grads), _ptr(m), _ptr(v), step, lr, beta1, beta2,
                               eps, _stream()))


def poly_lr(epoch: int, lr0: float, lr_end: float, epochs: int = 5000) -> float:
    return float(load().wm_poly_lr(epoch, lr0, lr_end, epochs))


# ---------------------------------------------------------------------------
# sequence-core operators (activations in float32 or bfloat16)
# ---------------------------------------------------------------------------

_ACT = {torch.float32: WM_FP32, torch.bfloat16: WM_BF16}


def _act(name, t, dtype=None):
    """The wm_dtype of an activation tensor; ``dtype`` (a torch type) must match."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype not in _ACT or (dtype is not None and t.dtype != dtype):
        raise ValueError(f"{name} has dtype {t.dtype}, expected {dtype or 'float32 or bfloat16'}")
    return _ACT[t.dtype]


def _arr(name, t, dtype, shape, device, optional=False):
    """The address of a contiguous array argument (None if it is optional and
    absent): _need's checks, spelled out only where one fails."""
    if t is None and optional:
        return None
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.is_contiguous()
            and t.device == device):
        _need(name, t, dtype, shape, device)
    return t.data_ptr()


def _rows(name, t, H, dtype, device):
    """(rows, distance between rows) of a [..., H] tensor with unit stride
    along H whose leading dimensions step evenly."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.device != device:
        _act(name, t, dtype)
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    shape = t.shape
    if not shape or shape[-1] != H:
        raise ValueError(f"{name} has shape {tuple(shape)}, expected [..., {H}]")
    if t.is_contiguous():
        return t.numel() // H if H else 0, H
    if len(shape) != 2:
        try:
            t = t.view(-1, H)
        except RuntimeError:
            raise ValueError(f"{name}'s rows are not evenly spaced (strides {t.stride()})") from None
    n, (ld, unit) = t.shape[0], t.stride()
    if H > 1 and unit != 1:
        raise ValueError(f"{name} must have unit stride along its last dimension")
    if n <= 1:
        return n, H
    if ld < H:
        raise ValueError(f"{name}'s rows overlap (stride {ld}, width {H})")
    return n, ld


def embed(table, tokens, scale: float = 1.0, out=None):
    """Launch wm_embed on the current stream: rows of ``table`` [V, H] for
    int32 ``tokens`` of any shape, times ``scale`` (zero rows for tokens
    outside [0, V)).  Returns ``out``, tokens.shape + (H,) in the table's type."""
    dt = _act("table", table)
    dev, dtype = table.device, table.dtype
    if table.dim() != 2:
        raise ValueError(f"table has shape {tuple(table.shape)}, expected [V, H]")
    V, H = table.shape
    pt = _arr("table", table, dtype, table.shape, dev)
    pk = _arr("tokens", tokens, torch.int32, getattr(tokens, "shape", ()), dev)
    n = tokens.numel()
    if out is None:
        out = torch.empty((*tokens.shape, H), dtype=dtype, device=dev)
    rows, ld = _rows("out", out, H, dtype, dev)
    if rows != n:
        raise ValueError(f"out has {rows} rows for {n} tokens")
    _check(load().wm_embed(dt, n, V, H, pk, pt, scale, out.data_ptr(), ld, _stream()))
    return out


class EmbedGradBuffers:
    """The table's gradient [V, H] float32 and the workspace of wm_embed_grad
    for up to n tokens."""

    def __init__(self, n: int, V: int, H: int, device="cuda"):
        self.n, self.V, self.H = n, V, H
        self.grad = torch.empty((V, H), dtype=torch.float32, device=device)
        self.ws_bytes = load().wm_embed_grad_workspace_bytes(n, V, H)
        self.workspace = torch.empty(max(self.ws_bytes, 1), dtype=torch.uint8, device=device)


def embed_grad(tokens, dout, V: int, scale: float = 1.0, bufs: EmbedGradBuffers | None = None) -> EmbedGradBuffers:
    """Launch wm_embed_grad on the current stream: the gradient of embed with
    respect to its table, from ``dout`` (tokens.shape + (H,))."""
    dt = _act("dout", dout)
    dev, H = dout.device, dout.shape[-1]
    pk = _arr("tokens", tokens, torch.int32, getattr(tokens, "shape", ()), dev)
    n = tokens.numel()
    rows, ld = _rows("dout", dout, H, dout.dtype, dev)
    if rows != n:
        raise ValueError(f"dout has {rows} rows for {n} tokens")
    if bufs is None:
        bufs = EmbedGradBuffers(n, V, H, dev)
    if (bufs.V, bufs.H) != (V, H) or bufs.grad.device != dev:
        raise ValueError(f"buffers for V={bufs.V} H={bufs.H} on {bufs.grad.device}; the call has V={V} H={H} on {dev}")
    _check(load().wm_embed_grad(dt, n, V, H, pk, dout.data_ptr(), ld, scale, bufs.grad.data_ptr(),
                                bufs.workspace.data_ptr(), bufs.ws_bytes, _stream()))
    return bufs


class LayerNormBuffers:
    """Output and statistics of layer norm over ``rows`` rows of width H, and
    with ``grad`` its gradients and workspace."""

    def __init__(self, rows: int, H: int, dtype=torch.float32, device="cuda", grad: bool = True):
        self.rows, self.H, self.dtype = rows, H, dtype
        self.y = torch.empty((rows, H), dtype=dtype, device=device)
        self.mean = torch.empty(rows, dtype=torch.float32, device=device) if grad else None
        self.rstd = torch.empty(rows, dtype=torch.float32, device=device) if grad else None
        self.dx = torch.empty((rows, H), dtype=dtype, device=device) if grad else None
        self.dgamma = torch.empty(H, dtype=torch.float32, device=device) if grad else None
        self.dbeta = torch.empty(H, dtype=torch.float32, device=device) if grad else None
        self.ws_bytes = load().wm_layer_norm_grad_workspace_bytes(rows, H) if grad else 0
        self.workspace = torch.empty(max(self.ws_bytes, 1), dtype=torch.uint8, device=device) if grad else None


def _norm_bufs(x, bufs, rows, H):
    if (bufs.rows, bufs.H, bufs.dtype) != (rows, H, x.dtype) or bufs.y.device != x.device:
        raise ValueError(f"buffers for rows={bufs.rows} H={bufs.H} {bufs.dtype} on {bufs.y.device}; the call has "
                         f"rows={rows} H={H} {x.dtype} on {x.device}")


def layer_norm(x, gamma=None, beta=None, eps: float = 1e-5, bufs: LayerNormBuffers | None = None) -> LayerNormBuffers:
    """Launch wm_layer_norm on the current stream over the rows of ``x``
    [..., H] (gamma, beta [H] float32 or None); returns the filled buffers."""
    dt = _act("x", x)
    dev, H = x.device, x.shape[-1]
    rows, ld = _rows("x", x, H, x.dtype, dev)
    pg = _arr("gamma", gamma, torch.float32, (H,), dev, optional=True)
    pb = _arr("beta", beta, torch.float32, (H,), dev, optional=True)
    if bufs is None:
        bufs = LayerNormBuffers(rows, H, x.dtype, dev)
    _norm_bufs(x, bufs, rows, H)
    _check(load().wm_layer_norm(dt, rows, H, x.data_ptr(), ld, pg, pb, eps, bufs.y.data_ptr(), H,
                                _ptr(bufs.mean), _ptr(bufs.rstd), _stream()))
    return bufs


def layer_norm_grad(x, dy, gamma=None, bufs: LayerNormBuffers | None = None) -> LayerNormBuffers:
    """Launch wm_layer_norm_grad on the current stream: dx, dgamma and dbeta
    from the forward call's input and the statistics in its ``bufs``."""
    dt = _act("x", x)
    dev, H = x.device, x.shape[-1]
    rows, ld = _rows("x", x, H, x.dtype, dev)
    nd, dld = _rows("dy", dy, H, x.dtype, dev)
    pg = _arr("gamma", gamma, torch.float32, (H,), dev, optional=True)
    if bufs is None or bufs.dx is None:
        raise ValueError("layer_norm_grad needs the forward call's buffers, made with grad=True")
    _norm_bufs(x, bufs, rows, H)
    if nd != rows:
        raise ValueError(f"dy has {nd} rows, x has {rows}")
    _check(load().wm_layer_norm_grad(dt, rows, H, x.data_ptr(), ld, dy.data_ptr(), dld, pg,
                                     bufs.mean.data_ptr(), bufs.rstd.data_ptr(), bufs.dx.data_ptr(), H,
                                     bufs.dgamma.data_ptr(), bufs.dbeta.data_ptr(), bufs.workspace.data_ptr(),
                                     bufs.ws_bytes, _stream()))
    return bufs


class LinrecBuffers:
    """Output, final state and workspace of the gated linear recurrence over
    [T, B, H]; with ``grad`` the saved states and the gradients (dx and dgate
    are the halves of one [T, B, 2H] tensor, ``dxg``)."""

    def __init__(self, T: int, B: int, H: int, dtype=torch.float32, device="cuda", grad: bool = True):
        self.T, self.B, self.H, self.dtype = T, B, H, dtype
        lib = load()
        self.y = torch.empty((T, B, H), dtype=dtype, device=device)
        self.h_T = torch.empty((B, H), dtype=torch.float32, device=device)
        self.ws_bytes = lib.wm_linrec_workspace_bytes(T, B, H)
        self.workspace = torch.empty(max(self.ws_bytes, 1), dtype=torch.uint8, device=device)
        self.states_bytes = lib.wm_linrec_states_bytes(T, B, H) if grad else 0
        self.states = torch.empty(max(self.states_bytes, 1), dtype=torch.uint8, device=device) if grad else None
        self.dxg = torch.empty((T, B, 2 * H), dtype=dtype, device=device) if grad else None
        self.dx = self.dxg[..., :H] if grad else None
        self.dgate = self.dxg[..., H:] if grad else None
        self.dh0 = torch.empty((B, H), dtype=torch.float32, device=device) if grad else None


def _seq(name, t, shape, dtype, device):
    """Checks a [T, B, H] tensor with unit stride along H; its strides."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.shape != shape or t.device != device:
        _act(name, t, dtype)
        raise ValueError(f"{name} is {tuple(t.shape)} on {t.device}, expected {tuple(shape)} on {device}")
    st = t.stride()
    if st[2] != 1 and shape[2] > 1:
        raise ValueError(f"{name} must have unit stride along its last dimension")
    return st


def _linrec_args(x, gate, resets, lengths, bufs):
    dt = _act("x", x)
    if x.dim() != 3:
        raise ValueError(f"x has shape {tuple(x.shape)}, expected [T, B, H]")
    dev, shape = x.device, x.shape
    sx, sg = _seq("x", x, shape, x.dtype, dev), _seq("gate", gate, shape, x.dtype, dev)
    pr = _arr("resets", resets, _mask_dtype(resets), shape[:2], dev, optional=True)
    pl = _arr("lengths", lengths, torch.int32, shape[1:2], dev, optional=True)
    if bufs is not None and ((bufs.T, bufs.B, bufs.H) != shape or bufs.dtype is not x.dtype or bufs.y.device != dev):
        raise ValueError(f"buffers for T={bufs.T} B={bufs.B} H={bufs.H} {bufs.dtype} on {bufs.y.device}; the call has "
                         f"{tuple(shape)} {x.dtype} on {dev}")
    return dt, dev, shape, sx, sg, pr, pl


def linrec(x, gate, h0=None, resets=None, lengths=None, bufs: LinrecBuffers | None = None) -> LinrecBuffers:
    """Launch wm_linrec on the current stream: h_t = a_t h_{t-1} + (1 - a_t)
    x_t with a = sigmoid(gate) over ``x``, ``gate`` [T, B, H] (resets [T, B]
    uint8: the step starts a new trajectory; lengths [B] int32); returns the
    filled buffers (y, h_T, and the states that linrec_grad reads)."""
    dt, dev, (T, B, H), sx, sg, pr, pl = _linrec_args(x, gate, resets, lengths, bufs)
    ph = _arr("h0", h0, torch.float32, (B, H), dev, optional=True)
    if bufs is None:
        bufs = LinrecBuffers(T, B, H, x.dtype, dev)
    _check(load().wm_linrec(dt, T, B, H, x.data_ptr(), sx[0], sx[1], gate.data_ptr(), sg[0], sg[1], ph, pr, pl,
                            bufs.y.data_ptr(), bufs.h_T.data_ptr(), _ptr(bufs.states), bufs.states_bytes,
                            bufs.workspace.data_ptr(), bufs.ws_bytes, _stream()))
    return bufs


def linrec_grad(x, gate, dy, dh_T=None, resets=None, lengths=None, bufs: LinrecBuffers | None = None) -> LinrecBuffers:
    """Launch wm_linrec_grad on the current stream: dx, dgate and dh0 from
    the forward call's inputs and the states in its ``bufs``."""
    dt, dev, (T, B, H), sx, sg, pr, pl = _linrec_args(x, gate, resets, lengths, bufs)
    if bufs is None or bufs.states is None:
        raise ValueError("linrec_grad needs the forward call's buffers, made with grad=True")
    sd = _seq("dy", dy, x.shape, x.dtype, dev)
    ph = _arr("dh_T", dh_T, torch.float32, (B, H), dev, optional=True)
    ox, og = bufs.dx.stride(), bufs.dgate.stride()
    _check(load().wm_linrec_grad(dt, T, B, H, x.data_ptr(), sx[0], sx[1], gate.data_ptr(), sg[0], sg[1], pr, pl,
                                 dy.data_ptr(), sd[0], sd[1], ph, bufs.states.data_ptr(), bufs.states_bytes,
                                 bufs.dx.data_ptr(), ox[0], ox[1], bufs.dgate.data_ptr(), og[0], og[1],
                                 bufs.dh0.data_ptr(), bufs.workspace.data_ptr(), bufs.ws_bytes, _stream()))
    return bufs


_address = torch.Tensor.data_ptr


class ClipPlan:
    """The gradient tensors of a training program (contiguous, float32 or
    bfloat16), where their clipped values go (``outs``; None = in place), the
    norm and the workspace of wm_clip_grads.  The tensors may be given other
    memory, sizes or types later, up to what the workspace serves."""

    def __init__(self, grads, outs=None):
        self.grads = list(grads)
        self.outs = self.grads if outs is None else list(outs)
        self.norm = None
        self._fill()
        dev = self.grads[0].device
        self.norm = torch.empty(1, dtype=torch.float32, device=dev)
        self.ws_bytes = load().wm_clip_grads_workspace_bytes(len(self.grads), self.table)
        self.workspace = torch.empty(max(self.ws_bytes, 1), dtype=torch.uint8, device=dev)

    def _fill(self):
        """The table of the tensors as they are, whole or not at all."""
        if not self.grads:
            raise ValueError("no gradient tensors")
        if len(self.outs) != len(self.grads):
            raise ValueError(f"{len(self.outs)} outputs for {len(self.grads)} tensors")
        dev = self.grads[0].device if self.norm is None else self.norm.device
        table = (CGradTensor * len(self.grads))()
        for i, (g, o) in enumerate(zip(self.grads, self.outs)):
            dt = _act(f"grads[{i}]", g)
            _need(f"grads[{i}]", g, g.dtype, g.shape, dev)
            _need(f"outs[{i}]", o, g.dtype, g.shape, dev)
            table[i] = CGradTensor(g.data_ptr(), o.data_ptr(), g.numel(), dt)
        all_ = self.grads if self.outs is self.grads else [*self.grads, *self.outs]
        self.table, self.ptrs = table, list(map(_address, all_))
        self.same = TensorGuards(*all_, dynamic_dims_sizes=None, dynamic_dims_strides=None).check


def clip_grads(plan: ClipPlan, max_norm: float):
    """Launch wm_clip_grads on the current stream over the plan's tensors:
    plan.norm becomes their global norm, plan.outs their values scaled to
    max_norm where the norm is above it.  Returns plan.norm (a device tensor:
    nothing waits)."""
    # The table is that of the tensors while their number, types, devices, sizes
    # and strides (in one call for all of them: 15 tensors and 15 outputs 2.2 us,
    # one by one 8) and addresses (1.8 us) are what they were.
    grads, outs = plan.grads, plan.outs
    all_ = grads if outs is grads else [*grads, *outs]
    if not (len(grads) == len(plan.table) and len(all_) == len(plan.ptrs) and plan.same(*all_)
            and list(map(_address, all_)) == plan.ptrs):
        plan._fill()
    _check(load().wm_clip_grads(len(plan.table), plan.table, max_norm, plan.norm.data_ptr(), plan.workspace.data_ptr(),
                                plan.ws_bytes, _stream()))
    return plan.norm


# ---------------------------------------------------------------------------
# attending-core operators (activations in float32 or bfloat16)
# ---------------------------------------------------------------------------

def _here(device):
    """Launches go to the current device: refuses tensors of another one."""
    if device.index != torch.cuda.current_device():
        raise ValueError(f"tensors on {device}, but the current device is {torch.cuda.current_device()}")


class Rotary:
    """The rotation's angles for the first R values of a head: pair i turns by
    base^(-2 i / R) a step; pairs are (i, i + R / 2), or with ``neighbours``
    (2 i, 2 i + 1)."""

    def __init__(self, R: int, base: float = 10000.0, neighbours: bool = False, device="cuda"):
        self.R, self.base, self.neighbours = R, base, bool(neighbours)
        host = (ctypes.c_uint64 * max(R // 2, 1))()
        _check(load().wm_rotary_table(R, base, host))
        # 64-bit words, held in a signed type
        self.table = torch.tensor([v - (v >> 63 << 64) for v in host], dtype=torch.int64).to(device)


class QkNormBuffers:
    """Normed and rotated queries [rows, Hq, D] and keys [rows, Hk, D], and with
    ``grad`` the gradients and the workspace of wm_qk_norm_grad."""

    def __init__(self, rows: int, Hq: int, Hk: int, D: int, dtype=torch.float32, device="cuda", grad: bool = True):
        self.rows, self.Hq, self.Hk, self.D, self.dtype = rows, Hq, Hk, D, dtype
        new = lambda h: torch.empty((rows, h, D), dtype=dtype, device=device)  # noqa: E731
        self.q, self.k = new(Hq), new(Hk)
        self.dq, self.dk = (new(Hq), new(Hk)) if grad else (None, None)
        self.dgamma_q, self.dgamma_k = ((torch.empty(D, dtype=torch.float32, device=device) for _ in range(2)) if grad
                                        else (None, None))
        self.ws_bytes = load().wm_qk_norm_grad_workspace_bytes(rows, Hq, Hk, D) if grad else 0
        self.workspace = torch.empty(max(self.ws_bytes, 1), dtype=torch.uint8, device=device) if grad else None


def _heads(name, t, H, D, dtype, device):
    """(rows, distance between rows) of a [..., H, D] tensor whose heads lie one
    after the other and whose leading dimensions step evenly."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.device != device:
        _act(name, t, dtype)
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    shape = t.shape
    if len(shape) < 2 or shape[-2] != H or shape[-1] != D:
        raise ValueError(f"{name} has shape {tuple(shape)}, expected [..., {H}, {D}]")
    n = shape[0] if len(shape) == 3 else math.prod(shape[:-2])
    if t.is_contiguous():
        return n, H * D
    st = t.stride()
    if n and H and ((D > 1 and st[-1] != 1) or (H > 1 and st[-2] != D)):
        raise ValueError(f"{name}'s heads must lie one after the other (strides {st})")
    if n <= 1:
        return n, H * D
    lead = [(s, d) for s, d in zip(shape[:-2], st[:-2]) if s > 1]
    for (_, a), (s, b) in zip(lead, lead[1:]):
        if a != s * b:
            raise ValueError(f"{name}'s rows are not evenly spaced (strides {st})")
    if lead[-1][1] < H * D:
        raise ValueError(f"{name}'s rows overlap (stride {lead[-1][1]}, width {H * D})")
    return n, lead[-1][1]


def _qk_args(q, k, positions, rotary, gamma_q, gamma_k, bufs, grad):
    dt = _act("q", q)
    dev, dtype, shape = q.device, q.dtype, q.shape
    _here(dev)
    if len(shape) < 2:
        raise ValueError(f"q has shape {tuple(shape)}, expected [..., Hq, D]")
    Hq, D = shape[-2], shape[-1]
    rows, ldq = _heads("q", q, Hq, D, dtype, dev)
    Hk, ldk, pk = 0, 0, None
    if k is not None:
        Hk = k.shape[-2] if isinstance(k, torch.Tensor) and k.dim() >= 2 else 1
        nk, ldk = _heads("k", k, Hk, D, dtype, dev)
        if nk != rows:
            raise ValueError(f"k has {nk} rows, q has {rows}")
        pk = k.data_ptr()
    pp = _arr("positions", positions, torch.int32, getattr(positions, "shape", ()), dev)
    if positions.numel() != rows:
        raise ValueError(f"{positions.numel()} positions for {rows} rows")
    R, nb, pt = 0, 0, None
    if rotary is not None:
        table = rotary.table
        if table.device != dev:
            raise ValueError(f"the rotation's table is on {table.device}, expected {dev}")
        if table.dtype is not torch.int64 or table.numel() < rotary.R // 2 or not table.is_contiguous():
            raise ValueError(f"the rotation's table must hold {rotary.R // 2} int64 words")
        R, nb, pt = rotary.R, rotary.neighbours, table.data_ptr()
    pgq = _arr("gamma_q", gamma_q, torch.float32, (D,), dev, optional=True)
    pgk = _arr("gamma_k", gamma_k, torch.float32, (D,), dev, optional=True)
    if bufs is None:
        bufs = QkNormBuffers(rows, Hq, Hk, D, dtype, dev, grad=grad)
    if (bufs.rows, bufs.Hq, bufs.Hk, bufs.D) != (rows, Hq, Hk, D) or bufs.dtype is not dtype or bufs.q.device != dev:
        raise ValueError(f"buffers for rows={bufs.rows} Hq={bufs.Hq} Hk={bufs.Hk} D={bufs.D} {bufs.dtype} on "
                         f"{bufs.q.device}; the call has rows={rows} Hq={Hq} Hk={Hk} D={D} {dtype} on {dev}")
    return (dt, rows, Hq, Hk, D, R, nb, q.data_ptr(), ldq, pk, ldk, pgq, pgk), (pp, pt), bufs


def _head_out(name, t, rows, H, D, like):
    """Checks an output of ``rows`` x H heads, which may lie inside wider rows; the
    distance between its rows."""
    n, ld = _heads(name, t, H, D, like.dtype, like.device)
    if n != rows:
        raise ValueError(f"{name} has {n} rows, the call {rows}")
    return ld


def qk_norm(q, k, positions, rotary: Rotary | None, gamma_q=None, gamma_k=None, eps: float = 1e-6,
            bufs: QkNormBuffers | None = None) -> QkNormBuffers:
    """Launch wm_qk_norm on the current stream: every head of ``q`` [..., Hq, D]
    and ``k`` [..., Hk, D] (None: queries alone) divided by its root mean
    square, times gamma_q and gamma_k ([D] float32 or None), and rotated by its
    row's int32 position.  Returns the filled buffers (q, k; the buffers' own may be
    set to q and k themselves: in place)."""
    head, (pp, pt), bufs = _qk_args(q, k, positions, rotary, gamma_q, gamma_k, bufs, False)
    lq = _head_out("bufs.q", bufs.q, bufs.rows, bufs.Hq, bufs.D, q)
    lk = _head_out("bufs.k", bufs.k, bufs.rows, bufs.Hk, bufs.D, q) if bufs.Hk else 0
    _check(load().wm_qk_norm(*head, eps, pp, pt, bufs.q.data_ptr(), lq, bufs.k.data_ptr(), lk, _stream()))
    return bufs


def qk_norm_grad(q, k, dq_out, dk_out, positions, rotary: Rotary | None, gamma_q=None, gamma_k=None, eps: float = 1e-6,
                 bufs: QkNormBuffers | None = None) -> QkNormBuffers:
    """Launch wm_qk_norm_grad on the current stream: dq, dk, dgamma_q and
    dgamma_k from the forward call's inputs and the gradients of its outputs."""
    head, (pp, pt), bufs = _qk_args(q, k, positions, rotary, gamma_q, gamma_k, bufs, True)
    if bufs.dq is None:
        raise ValueError("qk_norm_grad needs buffers made with grad=True")
    n, ldq = _heads("dq_out", dq_out, bufs.Hq, bufs.D, q.dtype, q.device)
    m, ldk = (n, 0) if k is None else _heads("dk_out", dk_out, bufs.Hk, bufs.D, q.dtype, q.device)
    if n != bufs.rows or m != bufs.rows:
        raise ValueError(f"dq_out has {n} rows, dk_out {m}, q has {bufs.rows}")
    pgq = _arr("bufs.dgamma_q", bufs.dgamma_q, torch.float32, (bufs.D,), q.device)
    pgk = _arr("bufs.dgamma_k", bufs.dgamma_k, torch.float32, (bufs.D,), q.device)
    lq = _head_out("bufs.dq", bufs.dq, bufs.rows, bufs.Hq, bufs.D, q)
    lk = _head_out("bufs.dk", bufs.dk, bufs.rows, bufs.Hk, bufs.D, q) if bufs.Hk else 0
    _check(load().wm_qk_norm_grad(*head, eps, pp, pt, dq_out.data_ptr(), ldq, None if k is None else dk_out.data_ptr(), ldk,
                                  bufs.dq.data_ptr(), lq, bufs.dk.data_ptr(), lk,
                                  pgq, pgk, bufs.workspace.data_ptr(),
                                  bufs.ws_bytes, _stream()))
    return bufs


class LinattnBuffers:
    """Output [T, B, N, V], final state [B, N, K, V] and workspace of linear
    attention; with ``grad`` the saved states and the gradients (dq, dk and dv
    contiguous)."""

    def __init__(self, T: int, B: int, N: int, K: int, V: int, dtype=torch.float32, device="cuda", grad: bool = True):
        self.T, self.B, self.N, self.K, self.V, self.dtype = T, B, N, K, V, dtype
        lib = load()
        seq = lambda w: torch.empty((T, B, N, w), dtype=dtype, device=device)  # noqa: E731
        state = lambda: torch.empty((B, N, K, V), dtype=torch.float32, device=device)  # noqa: E731
        self.y, self.h_T = seq(V), state()
        self.dq, self.dk, self.dv, self.dh0 = (seq(K), seq(K), seq(V), state()) if grad else (None,) * 4
        self.ws_bytes = lib.wm_linattn_workspace_bytes(T, B, N, K, V)
        self.workspace = torch.empty(max(self.ws_bytes, 1), dtype=torch.uint8, device=device)
        self.states_bytes = lib.wm_linattn_states_bytes(T, B, N, K, V) if grad else 0
        self.states = torch.empty(max(self.states_bytes, 1), dtype=torch.uint8, device=device) if grad else None


def _steps(name, t, shape, dtype, device):
    """Checks a [T, B, N, W] tensor whose heads lie one after the other; its
    strides of steps and rows."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.shape != shape or t.device != device:
        _act(name, t, dtype)
        raise ValueError(f"{name} is {tuple(t.shape)} on {t.device}, expected {tuple(shape)} on {device}")
    st = t.stride()
    if (shape[3] > 1 and st[3] != 1) or (shape[2] > 1 and st[2] != shape[3]):
        raise ValueError(f"{name}'s heads must lie one after the other (strides {st})")
    return st[0], st[1]


def _linattn_args(q, k, v, decay, h0, resets, lengths, bufs):
    dt = _act("q", q)
    dev, dtype = q.device, q.dtype
    _here(dev)
    if q.dim() != 4 or not isinstance(v, torch.Tensor) or v.dim() != 4:
        raise ValueError("q, k and v must be [T, B, N, K] and [T, B, N, V]")
    T, B, N, K = q.shape
    V = v.shape[3]
    qt, qb = _steps("q", q, (T, B, N, K), dtype, dev)
    kt, kb = _steps("k", k, (T, B, N, K), dtype, dev)
    vt, vb = _steps("v", v, (T, B, N, V), dtype, dev)
    pd = _arr("decay", decay, torch.float32, (N,), dev)
    ph = _arr("h0", h0, torch.float32, (B, N, K, V), dev, optional=True)
    pr = _arr("resets", resets, _mask_dtype(resets), (T, B), dev, optional=True)
    pl = _arr("lengths", lengths, torch.int32, (B,), dev, optional=True)
    if bufs is None:
        bufs = LinattnBuffers(T, B, N, K, V, dtype, dev)
    if (bufs.T, bufs.B, bufs.N, bufs.K, bufs.V, bufs.dtype) != (T, B, N, K, V, dtype) or bufs.y.device != dev:
        raise ValueError(f"buffers for T={bufs.T} B={bufs.B} N={bufs.N} K={bufs.K} V={bufs.V} {bufs.dtype} on "
                         f"{bufs.y.device}; the call has T={T} B={B} N={N} K={K} V={V} {dtype} on {dev}")
    head = (dt, T, B, N, K, V, q.data_ptr(), qt, qb, k.data_ptr(), kt, kb, v.data_ptr(), vt, vb, pd)
    return head, (ph, pr, pl), bufs


def linattn(q, k, v, decay, scale: float = 1.0, h0=None, resets=None, lengths=None,
            bufs: LinattnBuffers | None = None) -> LinattnBuffers:
    """Launch wm_linattn on the current stream: S_t = decay S_{t-1} + k_t v_t^T,
    y_t = scale S_t^T q_t for every head over ``q``, ``k`` [T, B, N, K] and
    ``v`` [T, B, N, V] (decay [N] float32; resets [T, B] uint8: the step starts
    a new trajectory; lengths [B] int32).  Returns the filled buffers (y, h_T, and
    the states that linattn_grad reads; buffers made with grad=False hold the outputs
    alone)."""
    head, masks, bufs = _linattn_args(q, k, v, decay, h0, resets, lengths, bufs)
    py = _arr("bufs.y", bufs.y, q.dtype, v.shape, q.device)
    ph = _arr("bufs.h_T", bufs.h_T, torch.float32, (bufs.B, bufs.N, bufs.K, bufs.V), q.device)
    _check(load().wm_linattn(*head, scale, *masks, py, ph, _ptr(bufs.states),
                             bufs.states_bytes, bufs.workspace.data_ptr(), bufs.ws_bytes, _stream()))
    return bufs


def linattn_grad(q, k, v, decay, dy, scale: float = 1.0, h0=None, dh_T=None, resets=None, lengths=None,
                 bufs: LinattnBuffers | None = None) -> LinattnBuffers:
    """Launch wm_linattn_grad on the current stream: dq, dk, dv and dh0 from the
    forward call's inputs, the gradients of its outputs and the states in its
    ``bufs``."""
    if bufs is None or bufs.states is None:
        raise ValueError("linattn_grad needs the forward call's buffers, made with grad=True")
    head, masks, bufs = _linattn_args(q, k, v, decay, h0, resets, lengths, bufs)
    T, B, N, K, V = bufs.T, bufs.B, bufs.N, bufs.K, bufs.V
    yt, yb = _steps("dy", dy, (T, B, N, V), q.dtype, q.device)
    ph = _arr("dh_T", dh_T, torch.float32, (B, N, K, V), q.device, optional=True)
    p0 = _arr("bufs.dh0", bufs.dh0, torch.float32, (B, N, K, V), q.device)
    out = []  # (they may lie inside wider rows: parts of a projection's gradient)
    for name, t, w in (("bufs.dq", bufs.dq, K), ("bufs.dk", bufs.dk, K), ("bufs.dv", bufs.dv, V)):
        out += (t.data_ptr(), *_steps(name, t, (T, B, N, w), q.dtype, q.device))
    _check(load().wm_linattn_grad(*head, scale, *masks, dy.data_ptr(), yt, yb, ph, bufs.states.data_ptr(),
                                  bufs.states_bytes, *out, p0, bufs.workspace.data_ptr(), bufs.ws_bytes,
                                  _stream()))
    return bufs


_GLU_ACTS = {"silu": 0, "gelu": 1}


class GluBuffers:
    """Output [rows, F] of the gated projection, and with ``grad`` what it saves for
    the gradient, the gradients and the workspace."""

    def __init__(self, rows: int, D: int, F: int, dtype=torch.float32, device="cuda", grad: bool = True):
        self.rows, self.D, self.F, self.dtype = rows, D, F, dtype
        lib = load()
        new = lambda *s: torch.empty(s, dtype=dtype, device=device)  # noqa: E731
        raw = lambda n: torch.empty(max(n, 1), dtype=torch.uint8, device=device) if grad else None  # noqa: E731
        self.h = new(rows, F)
        self.dx, self.dW = (new(rows, D), new(2 * F, D)) if grad else (None, None)
        self.saved_bytes = lib.wm_glu_saved_bytes(_ACT[dtype], rows, D, F) if grad else 0
        self.ws_bytes = lib.wm_glu_grad_workspace_bytes(_ACT[dtype], rows, D, F) if grad else 0
        self.saved, self.workspace = raw(self.saved_bytes), raw(self.ws_bytes)


def _glu_args(x, W, act, bufs):
    dt = _act("x", x)
    dev, dtype = x.device, x.dtype
    _here(dev)
    if act not in _GLU_ACTS:
        raise ValueError(f"act is {act!r}, expected one of {sorted(_GLU_ACTS)}")
    if not isinstance(W, torch.Tensor) or W.dim() != 2 or W.shape[0] % 2 or W.shape[0] == 0:
        raise ValueError("W must be [2F, D]")
    F, D = W.shape[0] // 2, W.shape[1]
    pw = _arr("W", W, dtype, (2 * F, D), dev)
    rows, ld = _rows("x", x, D, dtype, dev)
    if bufs is not None and ((bufs.rows, bufs.D, bufs.F, bufs.dtype) != (rows, D, F, dtype) or bufs.h.device != dev):
        raise ValueError(f"buffers for rows={bufs.rows} D={bufs.D} F={bufs.F} {bufs.dtype} on {bufs.h.device}; the call has "
                         f"rows={rows} D={D} F={F} {dtype} on {dev}")
    return (dt, rows, D, F, _GLU_ACTS[act], x.data_ptr(), ld, pw)


def glu(x, W, act: str = "silu", bufs: GluBuffers | None = None) -> GluBuffers:
    """Launch wm_glu on the current stream: act(x W[:F]^T) * (x W[F:]^T) for the
    rows of ``x`` [..., D] and ``W`` [2F, D]; returns the filled buffers (h, and
    what glu_grad reads, 2F values a row; buffers made with grad=False hold h alone)."""
    head = _glu_args(x, W, act, bufs)
    if bufs is None:
        bufs = GluBuffers(head[1], head[2], head[3], x.dtype, x.device)
    n, lh = _rows("bufs.h", bufs.h, bufs.F, x.dtype, x.device)
    if n != bufs.rows:
        raise ValueError(f"bufs.h has {n} rows, x has {bufs.rows}")
    _check(load().wm_glu(*head, bufs.h.data_ptr(), lh, _ptr(bufs.saved), bufs.saved_bytes, _stream()))
    return bufs


def glu_grad(x, W, dh, act: str = "silu", bufs: GluBuffers | None = None) -> GluBuffers:
    """Launch wm_glu_grad on the current stream: dx and dW (in the weights' type)
    from the forward call's inputs and what it saved in its ``bufs``."""
    head = _glu_args(x, W, act, bufs)
    if bufs is None or bufs.saved is None:
        raise ValueError("glu_grad needs the forward call's buffers, made with grad=True")
    n, ld = _rows("dh", dh, bufs.F, x.dtype, x.device)
    if n != bufs.rows:
        raise ValueError(f"dh has {n} rows, x has {bufs.rows}")
    n, lx = _rows("bufs.dx", bufs.dx, bufs.D, x.dtype, x.device)
    if n != bufs.rows:
        raise ValueError(f"bufs.dx has {n} rows, x has {bufs.rows}")
    pw = _arr("bufs.dW", bufs.dW, x.dtype, (2 * bufs.F, bufs.D), x.device)
    _check(load().wm_glu_grad(*head, bufs.saved.data_ptr(), bufs.saved_bytes, dh.data_ptr(), ld, bufs.dx.data_ptr(),
                              lx, pw, bufs.workspace.data_ptr(), bufs.ws_bytes, _stream()))
    return bufs


def profile_enable(prefix: str | None):
    """Bracket launches of kernels whose name starts with ``prefix`` with HIP
    events (None turns it off)."""
    _check(load().wm_profile_enable(None if prefix is None else prefix.encode()))


def profile_read(prefix: str | None = None) -> tuple[float, int]:
    """(summed milliseconds, launch count) of the recorded launches."""
    ms, n = ctypes.c_double(), ctypes.c_int64()
    _check(load().wm_profile_read(None if prefix is None else prefix.encode(), ctypes.byref(ms),
                                  ctypes.byref(n)))
    return ms.value, n.value


def profile_reset():
    _check(load().wm_profile_reset())


PHASE_SLOTS = ("T", "step", "ctrl", "ctrl_barrier", "gates", "gates_barrier", "mdn", "mdn_barrier",
               "ctrl_mean", "gates_mean", "mdn_mean", "setup", "tail")


def profile_phases(on: bool):
    """Stamp the phase boundaries of later persistent-kernel launches."""
    _check(load().wm_profile_phases(1 if on else 0))


def profile_phases_read() -> dict:
    """Per-step phase durations (us) of the last stamped launch, by slot."""
    out = (ctypes.c_double * len(PHASE_SLOTS))()
    _check(load().wm_profile_phases_read(out, len(PHASE_SLOTS)))
    return dict(zip(PHASE_SLOTS, list(out)))


def version() -> str:
    return load().wm_version().decode()

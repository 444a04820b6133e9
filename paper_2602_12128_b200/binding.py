"""ctypes binding of libhla.so: the same entry points as include/hla.h, taking
torch tensors (device memory and streams only - every step of the operator
runs in the library's kernels).  There is no fallback: if the library cannot be
loaded, importing callers get an exception."""
from __future__ import annotations

import ctypes
import os
from ctypes import POINTER, byref, c_char_p, c_double, c_float, c_int32, c_int64, c_size_t, c_uint64, c_void_p

import torch

from . import build as _build

HLA_OK, HLA_ERR_INVALID_ARG, HLA_ERR_UNSUPPORTED, HLA_ERR_WORKSPACE, HLA_ERR_CUDA, HLA_ERR_DEVICE_TIMEOUT, HLA_ERR_NO_MEMORY = range(7)
HLA_BF16, HLA_F32 = 0, 1
HLA_PHI_MLP, HLA_PHI_NONE = 0, 1

EXPORTS = [
    "hla_create", "hla_set_phi", "hla_workspace_bytes", "hla_workspace_layout", "hla_forward", "hla_backward", "hla_forward_keys", "hla_forward_queries", "hla_backward_queries", "hla_backward_keys", "hla_backward_weights", "hla_set_phi_v", "hla_set_carry", "hla_value_mod_forward", "hla_value_mod_backward", "hla_forward_static",
    "hla_last_device_status", "hla_selftest_bounded_wait", "hla_last_launch_count", "hla_timing_enable", "hla_timing_collect", "hla_timing_get",
    "hla_destroy", "hla_status_string",
    "hla_heads_create", "hla_heads_workspace_bytes", "hla_heads_forward", "hla_heads_backward", "hla_heads_destroy",
    "hla_adamw_create", "hla_adamw_set_grads", "hla_adamw_workspace_bytes", "hla_adamw_step", "hla_adamw_destroy",
    "hla_scan_create", "hla_scan_workspace_bytes", "hla_scan_forward", "hla_scan_backward",
    "hla_scan_last_device_status", "hla_scan_selftest_bounded_wait", "hla_scan_destroy",
]


class HlaConfig(ctypes.Structure):
    _fields_ = [("B", c_int32), ("H", c_int32), ("N", c_int32), ("d", c_int32), ("F", c_int32), ("d_phi", c_int32),
                ("phi", c_int32), ("dtype", c_int32), ("eps", c_float), ("n_splits", c_int32), ("causal", c_int32), ("value_mod", c_int32)]


class HlaMlp(ctypes.Structure):
    _fields_ = [("W1", c_void_p), ("b1", c_void_p), ("W2", c_void_p), ("b2", c_void_p)]


class HlaVmlp(ctypes.Structure):
    _fields_ = [("ln_g", c_void_p), ("ln_b", c_void_p), ("W1", c_void_p), ("b1", c_void_p), ("W2", c_void_p), ("b2", c_void_p)]


class HlaMlpGrad(ctypes.Structure):
    _fields_ = [("dW1", c_void_p), ("db1", c_void_p), ("dW2", c_void_p), ("db2", c_void_p)]


class HlaWsLayout(ctypes.Structure):
    _fields_ = [("status", c_size_t), ("qf", c_size_t), ("kf", c_size_t), ("state", c_size_t), ("eta", c_size_t),
                ("dstate", c_size_t), ("dqf", c_size_t), ("dkf", c_size_t), ("state_ld", c_int32), ("state_rows", c_int32), ("n_splits", c_int32),
                ("tensor_core", c_int32)]


HLA_PAIR_ADJACENT, HLA_PAIR_HALVES = 0, 1
HLA_STATE_F32, HLA_STATE_Q8 = 0, 1
HLA_GATE_LOG, HLA_GATE_SIGMOID = 0, 1
HLA_SCAN_STATUS_BYTES = 256


class HlaHeadsConfig(ctypes.Structure):
    _fields_ = [("B", c_int32), ("H", c_int32), ("N", c_int32), ("d", c_int32), ("dtype", c_int32), ("pairing", c_int32), ("norm", c_int32),
                ("n_axes", c_int32), ("axis_width", c_int32 * 3), ("grid", c_int32 * 3), ("start", c_int32 * 3), ("eps", c_float), ("q_scale", c_float),
                ("theta", c_double), ("inv_freq", POINTER(c_double))]


class HlaRows(ctypes.Structure):
    _fields_ = [("data", c_void_p), ("batch_stride", c_int64), ("token_stride", c_int64)]


class HlaAdamwTensor(ctypes.Structure):
    _fields_ = [("param", c_void_p), ("copy", c_void_p), ("grad", c_void_p), ("m", c_void_p), ("v", c_void_p), ("m_scale", c_void_p), ("v_scale", c_void_p),
                ("n", c_int64), ("lr_mul", c_float), ("weight_decay", c_float), ("param_dtype", c_int32), ("grad_dtype", c_int32)]


class HlaAdamwConfig(ctypes.Structure):
    _fields_ = [("beta1", c_double), ("beta2", c_double), ("eps", c_double), ("state", c_int32), ("seed", c_uint64)]


class HlaAdamwStepArgs(ctypes.Structure):
    _fields_ = [("lr", c_double), ("step", c_int64), ("lr_device", c_void_p), ("step_device", c_void_p), ("max_norm", c_float), ("grad_scale", c_float),
                ("norm", c_void_p)]


class HlaScanConfig(ctypes.Structure):
    _fields_ = [("B", c_int32), ("N", c_int32), ("C", c_int32), ("dtype", c_int32), ("gate", c_int32), ("convex", c_int32),
                ("x_batch_stride", c_int64), ("x_token_stride", c_int64), ("g_batch_stride", c_int64), ("g_token_stride", c_int64)]


class HlaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (hla_status {status})")


_lib = None


def library_path() -> str:
    return _build.LIB


def load_library(rebuild: bool = False) -> ctypes.CDLL:
    """Loads libhla.so (building it with nvcc first if it is missing or stale)."""
    global _lib
    if _lib is not None and not rebuild:
        return _lib
    path = _build.build(force=rebuild)
    if not os.path.exists(path):
        raise RuntimeError(f"HLA CUDA library missing: {path}")
    lib = ctypes.CDLL(path)
    lib.hla_create.argtypes = [POINTER(HlaConfig), POINTER(c_void_p)]
    lib.hla_create.restype = c_int32
    lib.hla_set_phi.argtypes = [c_void_p, POINTER(HlaMlp), POINTER(HlaMlp)]
    lib.hla_set_phi.restype = c_int32
    lib.hla_workspace_bytes.argtypes = [c_void_p]
    lib.hla_workspace_bytes.restype = c_size_t
    lib.hla_workspace_layout.argtypes = [c_void_p, POINTER(HlaWsLayout)]
    lib.hla_workspace_layout.restype = c_int32
    lib.hla_forward.argtypes = [c_void_p] + [c_void_p] * 4 + [c_void_p, c_size_t, c_void_p]
    lib.hla_forward.restype = c_int32
    lib.hla_backward.argtypes = [c_void_p] + [c_void_p] * 8 + [c_void_p, c_size_t, c_void_p]
    lib.hla_backward.restype = c_int32
    lib.hla_forward_keys.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.hla_forward_keys.restype = c_int32
    lib.hla_forward_queries.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.hla_forward_queries.restype = c_int32
    for name in ("hla_backward_queries", "hla_backward_keys"):
        getattr(lib, name).argtypes = [c_void_p] + [c_void_p] * 8 + [c_void_p, c_size_t, c_void_p]
        getattr(lib, name).restype = c_int32
    lib.hla_backward_weights.argtypes = [c_void_p, c_void_p, c_void_p, POINTER(HlaMlpGrad), POINTER(HlaMlpGrad), c_void_p, c_size_t, c_void_p]
    lib.hla_backward_weights.restype = c_int32
    lib.hla_set_carry.argtypes = [c_void_p, c_int32]
    lib.hla_set_carry.restype = c_int32
    lib.hla_set_phi_v.argtypes = [c_void_p, POINTER(HlaVmlp), POINTER(HlaVmlp)]
    lib.hla_set_phi_v.restype = c_int32
    lib.hla_value_mod_forward.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.hla_value_mod_forward.restype = c_int32
    lib.hla_value_mod_backward.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int32, c_void_p, c_size_t, c_void_p]
    lib.hla_value_mod_backward.restype = c_int32
    lib.hla_forward_static.argtypes = [c_void_p] + [c_void_p] * 4 + [c_void_p, POINTER(c_void_p)]
    lib.hla_forward_static.restype = c_int32
    lib.hla_last_device_status.argtypes = [c_void_p, c_void_p, c_void_p]
    lib.hla_last_device_status.restype = c_int32
    lib.hla_selftest_bounded_wait.argtypes = [c_void_p, c_void_p, c_size_t, c_void_p]
    lib.hla_selftest_bounded_wait.restype = c_int32
    lib.hla_last_launch_count.argtypes = [c_void_p]
    lib.hla_last_launch_count.restype = c_int32
    lib.hla_timing_enable.argtypes = [c_void_p, c_int32]
    lib.hla_timing_enable.restype = c_int32
    lib.hla_timing_collect.argtypes = [c_void_p]
    lib.hla_timing_collect.restype = c_int32
    lib.hla_timing_get.argtypes = [c_void_p, c_int32, POINTER(c_char_p), POINTER(ctypes.c_double), POINTER(ctypes.c_int64)]
    lib.hla_timing_get.restype = c_int32
    lib.hla_destroy.argtypes = [c_void_p]
    lib.hla_destroy.restype = c_int32
    for name, args in {
        "hla_heads_create": [POINTER(HlaHeadsConfig), POINTER(c_void_p)],
        "hla_heads_forward": [c_void_p] * 7 + [c_int64] + [c_void_p] * 4,
        "hla_heads_backward": [c_void_p] * 9 + [c_int64] + [c_void_p] * 6 + [c_size_t, c_void_p],
        "hla_heads_destroy": [c_void_p],
        "hla_adamw_create": [POINTER(HlaAdamwConfig), POINTER(HlaAdamwTensor), c_int32, POINTER(c_void_p)],
        "hla_adamw_set_grads": [c_void_p, POINTER(c_void_p), c_int32],
        "hla_adamw_step": [c_void_p, c_void_p, c_void_p, c_size_t, c_void_p],
        "hla_adamw_destroy": [c_void_p],
        "hla_scan_create": [POINTER(HlaScanConfig), POINTER(c_void_p)],
        "hla_scan_forward": [c_void_p] * 7 + [c_size_t, c_void_p],
        "hla_scan_backward": [c_void_p] * 11 + [c_size_t, c_void_p],
        "hla_scan_last_device_status": [c_void_p, c_void_p, c_void_p],
        "hla_scan_selftest_bounded_wait": [c_void_p, c_void_p, c_size_t, c_void_p],
        "hla_scan_destroy": [c_void_p],
    }.items():
        getattr(lib, name).argtypes = args
        getattr(lib, name).restype = c_int32
    for name in ("hla_heads_workspace_bytes", "hla_adamw_workspace_bytes", "hla_scan_workspace_bytes"):
        getattr(lib, name).argtypes = [c_void_p]
        getattr(lib, name).restype = c_size_t
    lib.hla_status_string.argtypes = [c_int32]
    lib.hla_status_string.restype = c_char_p
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load_library().hla_status_string(int(status)).decode()


def _ptr(t) -> int:
    if t is None:
        return 0
    if isinstance(t, int):
        return t
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return t.data_ptr()


# The handle of PyTorch's current stream without building a Stream object for it (3 of the 4 us that this took of every call; a
# feature-level step of 12 heads x 4999 tokens, 38 us of device time, was bound by the host).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is not None and torch.cuda.is_initialized():
            return _raw_stream(torch.cuda.current_device())
        return torch.cuda.current_stream().cuda_stream if torch.cuda.is_available() else 0
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


# ---- the C entry points, one to one ------------------------------------------
def hla_create(cfg: HlaConfig) -> int:
    out = c_void_p()
    st = load_library().hla_create(byref(cfg), byref(out))
    if st != HLA_OK:
        raise HlaError(st, "hla_create")
    return out.value


def hla_set_phi(ctx: int, phi_q, phi_k) -> None:
    """phi_q = (W1, b1, W2, b2) device tensors; phi_k = list of F such tuples."""
    q = HlaMlp(*[_ptr(t) for t in phi_q])
    ks = (HlaMlp * len(phi_k))(*[HlaMlp(*[_ptr(t) for t in w]) for w in phi_k])
    st = load_library().hla_set_phi(ctx, byref(q), ks)
    if st != HLA_OK:
        raise HlaError(st, "hla_set_phi")


def hla_workspace_bytes(ctx: int) -> int:
    return int(load_library().hla_workspace_bytes(ctx))


def hla_workspace_layout(ctx: int) -> HlaWsLayout:
    out = HlaWsLayout()
    st = load_library().hla_workspace_layout(ctx, byref(out))
    if st != HLA_OK:
        raise HlaError(st, "hla_workspace_layout")
    return out


def hla_forward(ctx: int, Q, K, V, O, workspace, stream=None, workspace_bytes=None) -> None:
    nbytes = workspace.numel() * workspace.element_size() if workspace_bytes is None else workspace_bytes
    st = load_library().hla_forward(ctx, _ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(workspace), nbytes, _stream(stream))
    if st != HLA_OK:
        raise HlaError(st, "hla_forward")


def hla_backward(ctx: int, Q, K, V, O, dO, dQ, dK, dV, workspace, stream=None, workspace_bytes=None) -> None:
    nbytes = workspace.numel() * workspace.element_size() if workspace_bytes is None else workspace_bytes
    st = load_library().hla_backward(ctx, _ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(dO), _ptr(dQ), _ptr(dK), _ptr(dV),
                                     _ptr(workspace), nbytes, _stream(stream))
    if st != HLA_OK:
        raise HlaError(st, "hla_backward")


def hla_forward_keys(ctx: int, K, V, workspace, stream=None) -> None:
    st = load_library().hla_forward_keys(ctx, _ptr(K), _ptr(V), _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream))
    if st != HLA_OK:
        raise HlaError(st, "hla_forward_keys")


def hla_forward_queries(ctx: int, Q, O, workspace, stream=None) -> None:
    st = load_library().hla_forward_queries(ctx, _ptr(Q), _ptr(O), _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream))
    if st != HLA_OK:
        raise HlaError(st, "hla_forward_queries")


def _backward_half(name, ctx, Q, K, V, O, dO, dQ, dK, dV, workspace, stream):
    st = getattr(load_library(), name)(ctx, _ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(dO), _ptr(dQ), _ptr(dK), _ptr(dV), _ptr(workspace),
                                       workspace.numel() * workspace.element_size(), _stream(stream))
    if st != HLA_OK:
        raise HlaError(st, name)


def hla_backward_queries(ctx: int, Q, K, V, O, dO, dQ, dK, dV, workspace, stream=None) -> None:
    _backward_half("hla_backward_queries", ctx, Q, K, V, O, dO, dQ, dK, dV, workspace, stream)


def hla_backward_keys(ctx: int, Q, K, V, O, dO, dQ, dK, dV, workspace, stream=None) -> None:
    _backward_half("hla_backward_keys", ctx, Q, K, V, O, dO, dQ, dK, dV, workspace, stream)


def hla_backward_weights(ctx: int, Q, K, dphi_q, dphi_k, workspace, stream=None, workspace_bytes=None) -> None:
    """dphi_q = (dW1, db1, dW2, db2) fp32 device tensors or None; dphi_k = list of F such tuples or None."""
    nbytes = workspace.numel() * workspace.element_size() if workspace_bytes is None else workspace_bytes
    q = byref(HlaMlpGrad(*[_ptr(t) for t in dphi_q])) if dphi_q is not None else None
    ks = (HlaMlpGrad * len(dphi_k))(*[HlaMlpGrad(*[_ptr(t) for t in w]) for w in dphi_k]) if dphi_k is not None else None
    st = load_library().hla_backward_weights(ctx, _ptr(Q), _ptr(K), q, ks, _ptr(workspace), nbytes, _stream(stream))
    if st != HLA_OK:
        raise HlaError(st, "hla_backward_weights")


def hla_set_carry(ctx: int, carry: bool) -> None:
    st = load_library().hla_set_carry(ctx, 1 if carry else 0)
    if st != HLA_OK:
        raise HlaError(st, "hla_set_carry")


def hla_set_phi_v(ctx: int, v1, v2) -> None:
    """v1, v2 = (ln_g, ln_b, W1, b1, W2, b2) device tensors of the two value-modulation maps."""
    a, b = HlaVmlp(*[_ptr(t) for t in v1]), HlaVmlp(*[_ptr(t) for t in v2])
    st = load_library().hla_set_phi_v(ctx, byref(a), byref(b))
    if st != HLA_OK:
        raise HlaError(st, "hla_set_phi_v")


def hla_value_mod_forward(ctx: int, T, V, Out, workspace, stream=None) -> None:
    st = load_library().hla_value_mod_forward(ctx, _ptr(T), _ptr(V), _ptr(Out), _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream))
    if st != HLA_OK:
        raise HlaError(st, "hla_value_mod_forward")


def hla_value_mod_backward(ctx: int, T, V, dOut, dT, dV, accumulate_dV, workspace, stream=None) -> None:
    st = load_library().hla_value_mod_backward(ctx, _ptr(T), _ptr(V), _ptr(dOut), _ptr(dT), _ptr(dV), 1 if accumulate_dV else 0, _ptr(workspace),
                                               workspace.numel() * workspace.element_size(), _stream(stream))
    if st != HLA_OK:
        raise HlaError(st, "hla_value_mod_backward")


HLA_STATIC_WS_BYTES = 16 * 1024 * 1024


def hla_forward_static(ctx: int, Q, K, V, O, stream=None) -> int:
    """hla_forward on the scratch array the library itself carries (no workspace tensor, nothing allocated).
    Returns that array's device address (an int), usable as `workspace` for hla_last_device_status."""
    scratch = c_void_p()
    st = load_library().hla_forward_static(ctx, _ptr(Q), _ptr(K), _ptr(V), _ptr(O), _stream(stream), byref(scratch))
    if st != HLA_OK:
        raise HlaError(st, "hla_forward_static")
    return scratch.value


def hla_last_device_status(ctx: int, workspace, stream=None) -> int:
    return int(load_library().hla_last_device_status(ctx, _ptr(workspace), _stream(stream)))


def hla_selftest_bounded_wait(ctx: int, workspace, stream=None) -> None:
    nbytes = workspace.numel() * workspace.element_size()
    st = load_library().hla_selftest_bounded_wait(ctx, _ptr(workspace), nbytes, _stream(stream))
    if st != HLA_OK:
        raise HlaError(st, "hla_selftest_bounded_wait")


def hla_last_launch_count(ctx: int) -> int:
    return int(load_library().hla_last_launch_count(ctx))


def hla_timing_enable(ctx: int, on: bool) -> None:
    st = load_library().hla_timing_enable(ctx, 1 if on else 0)
    if st != HLA_OK:
        raise HlaError(st, "hla_timing_enable")


def hla_timing_collect(ctx: int) -> dict:
    """After a stream synchronise: {kernel name: (total_ms, launches)} of the launches recorded since the last collect."""
    lib = load_library()
    n = lib.hla_timing_collect(ctx)
    out = {}
    for i in range(n):
        name = c_char_p()
        ms = ctypes.c_double()
        cnt = ctypes.c_int64()
        st = lib.hla_timing_get(ctx, i, byref(name), byref(ms), byref(cnt))
        if st != HLA_OK:
            raise HlaError(st, "hla_timing_get")
        out[name.value.decode()] = (ms.value, cnt.value)
    return out


def hla_destroy(ctx: int) -> None:
    st = load_library().hla_destroy(ctx)
    if st != HLA_OK:
        raise HlaError(st, "hla_destroy")


# ---- a small convenience holder (context + workspace) -------------------------
class Hla:
    """Owns a context and its workspace tensor.  All compute happens in hla_forward / hla_backward."""

    def __init__(self, B, H, N, d, dtype="bf16", phi="mlp", F=0, d_phi=0, eps=0.0, n_splits=0, device="cuda", value_mod=False, causal=False):
        self.cfg = HlaConfig(B, H, N, d, F, d_phi, HLA_PHI_MLP if phi == "mlp" else HLA_PHI_NONE,
                             HLA_BF16 if dtype == "bf16" else HLA_F32, eps, n_splits, 1 if causal else 0, 1 if value_mod else 0)
        self.torch_dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.ctx = hla_create(self.cfg)
        self.layout = hla_workspace_layout(self.ctx)
        self.device = device
        self.workspace = torch.empty(hla_workspace_bytes(self.ctx), dtype=torch.uint8, device=device) if device else None
        self._weights = None

    def set_phi(self, phi_q, phi_k):
        self._weights = (phi_q, phi_k)      # keep the tensors alive: the library only borrows pointers
        hla_set_phi(self.ctx, phi_q, phi_k)

    def forward(self, Q, K, V, O=None, stream=None):
        if O is None:
            O = torch.empty_like(V)
        hla_forward(self.ctx, Q, K, V, O, self.workspace, stream)
        return O

    def backward(self, Q, K, V, O, dO, dQ=None, dK=None, dV=None, stream=None):
        dQ = torch.empty_like(Q) if dQ is None else dQ
        dK = torch.empty_like(K) if dK is None else dK
        dV = torch.empty_like(V) if dV is None else dV
        hla_backward(self.ctx, Q, K, V, O, dO, dQ, dK, dV, self.workspace, stream)
        return dQ, dK, dV

    def state_region(self, gradient=False):
        """The fp32 state (or gradient state) of the last pass as a flat view of the workspace: what shards of a sequence add."""
        n = self.cfg.B * self.cfg.H * self.layout.state_rows * self.layout.state_ld
        return self.region("dstate" if gradient else "state")[:n]

    def set_carry(self, carry: bool):
        hla_set_carry(self.ctx, carry)

    def set_phi_v(self, v1, v2):
        self._vweights = (v1, v2)           # keep the tensors alive: the library only borrows pointers
        hla_set_phi_v(self.ctx, v1, v2)

    def value_mod_forward(self, T, V, Out=None, stream=None):
        Out = torch.empty_like(T) if Out is None else Out
        hla_value_mod_forward(self.ctx, T, V, Out, self.workspace, stream)
        return Out

    def value_mod_backward(self, T, V, dOut, dT=None, dV=None, accumulate_dV=False, stream=None):
        dT = torch.empty_like(T) if dT is None else dT
        dV = torch.empty_like(V) if dV is None else dV
        hla_value_mod_backward(self.ctx, T, V, dOut, dT, dV, accumulate_dV, self.workspace, stream)
        return dT, dV

    def backward_weights(self, Q, K, stream=None):
        """Weight gradients of phi_q and phi_k1..F (fp32, shapes of the weights), after backward()."""
        F = self.cfg.F or 3
        d, dphi = self.cfg.d, self.cfg.d_phi or (6 if F == 3 else 12)
        mk = lambda: tuple(torch.empty(s, dtype=torch.float32, device=self.device) for s in ((d, d), (d,), (d, dphi), (dphi,)))
        gq, gk = mk(), [mk() for _ in range(F)]
        hla_backward_weights(self.ctx, Q, K, gq, gk, self.workspace, stream)
        return gq, gk

    def region(self, name, dtype=torch.float32):
        """View of a persistent workspace region (see hla_ws_layout) as a flat tensor from its offset to the end."""
        off = getattr(self.layout, name)
        if off == ctypes.c_size_t(-1).value:
            raise KeyError(name)
        return self.workspace[off:].view(dtype)

    def device_status(self, stream=None) -> int:
        return hla_last_device_status(self.ctx, self.workspace, stream)

    def launches(self) -> int:
        return hla_last_launch_count(self.ctx)

    def close(self):
        if self.ctx:
            hla_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---- operators beside the attention ------------------------------------------
_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_CODES = {torch.bfloat16: HLA_BF16, torch.float32: HLA_F32}


def _dtype(name):
    if name not in _DTYPES:
        raise ValueError(f"dtype {name!r}: 'bf16' or 'f32' is wanted")
    return _DTYPES[name]


def _f32(x) -> float:
    """What an fp32 field of the library's structures makes of a number: 0 stands for a default in some of them."""
    return c_float(x).value


_current_device = getattr(torch._C, "_cuda_getDevice", None)


def _device() -> int:
    """The current device: work is enqueued on its current stream."""
    return _current_device() if _current_device is not None and torch.cuda.is_initialized() else torch.cuda.current_device() if torch.cuda.is_available() else 0


def _here(t, what, dtype, shape=None, device=None):
    """A tensor on the current device of the given type and shape."""
    device = _device() if device is None else device
    if t.dtype is dtype and (shape is None or t.shape == shape) and t.get_device() == device:
        return t
    if t.dtype is not dtype:
        raise ValueError(f"{what}: {dtype} is wanted, not {t.dtype}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{what}: shape {tuple(shape)} is wanted, not {tuple(t.shape)}")
    if not t.is_cuda:
        raise ValueError(f"{what}: a CUDA tensor is wanted")
    raise ValueError(f"{what}: on {t.device}, but the current device is cuda:{device}")


def _dense(t, what, dtype, shape=None, device=None):
    if t is None:
        return 0
    _here(t, what, dtype, shape, device)
    if not t.is_contiguous():
        raise ValueError(f"{what}: must be contiguous")
    return t.data_ptr()


def _scalar(t, what, dtype):
    if t.numel() != 1:
        raise ValueError(f"{what}: one element is wanted, not {t.numel()}")
    return _dense(t, what, dtype)


class _Maker:
    """Makes uninitialised tensors of one shape and type.  torch.empty with size, type and device takes 3.1 us of the host, torch.empty_like of a
    tensor that has the shape but no memory 1.4 us; a call for one token is bound by the host.  (Large ones, to whom a microsecond is nothing and
    whose pattern would for a moment need their memory, are made like one element, expanded: 2.3 us.)"""

    def __init__(self, shape, dtype, device):
        self.shape, self.dtype, self.device = shape, dtype, -1
        if device is not None and torch.device(device).type == "cuda":
            if shape.numel() <= 1 << 22:
                self.like = torch.empty(shape, dtype=dtype, device=device)
                self.like.untyped_storage().resize_(0)
            else:
                self.like = torch.empty((), dtype=dtype, device=device).expand(shape)
            self.device = self.like.get_device()

    def __call__(self, device: int):
        if device != self.device:
            return torch.empty(self.shape, dtype=self.dtype, device=f"cuda:{device}")
        return torch.empty_like(self.like)


class _Owner:
    """Holds a context of the library until it is closed or collected."""
    ctx, _destroy = None, ""
    workspace, _scratch, _need, _on = None, 0, 0, -1

    def _make_workspace(self, name, device):
        self._need = int(getattr(load_library(), name)(self.ctx))
        if device is not None and self._need:      # (0 is a device)
            self.workspace = torch.empty(self._need, dtype=torch.uint8, device=device)
            self._scratch, self._on = self.workspace.data_ptr(), self.workspace.get_device()

    def _workspace_here(self, device):
        if self._on not in (-1, device):
            raise ValueError(f"the workspace is on {self.workspace.device}, but the current device is cuda:{device}")

    def close(self):
        if self.ctx:
            getattr(load_library(), self._destroy)(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _create(name, *args) -> int:
    out = c_void_p()
    st = getattr(load_library(), name)(*args, byref(out))
    if st != HLA_OK:
        raise HlaError(st, name)
    return out.value


class _Slot:
    """One strided argument of Heads: what it is called, the library's description of it and the strides that this has."""

    def __init__(self, what):
        self.what, self.rows, self.strides = what, HlaRows(), None
        self.at = byref(self.rows)


class Heads(_Owner):
    """Head preparation around a projection (hla_heads_*): RMS norm of the rows of q and k, rotation by up to three axes, scale of q, and
    the move from [B,N,H,d] (any token stride: parts of one projection) to the [B,H,N,d] that Hla takes; and its backward.

    axes: channels that turn with each axis.  grid: tokens along each axis (None: every call is given `positions`, int32 [N, axes] or
    [B, N, axes]).  inv_freq: one value per pair (None: theta ** (-j / n) for pair j of an axis of n pairs).

    Here and in the classes below, work is enqueued on `stream` (None: the current one), tensors that a call makes belong to the current stream, and
    the calls of one object share its workspace: they have to follow one another, in a captured graph too."""
    _destroy = "hla_heads_destroy"

    def __init__(self, B, H, N, d, dtype="bf16", axes=(), grid=None, start=(0, 0, 0), theta=10000.0, inv_freq=None, pairing="interleaved", norm=False,
                 eps=1e-6, q_scale=1.0, device="cuda"):
        if pairing not in ("interleaved", "half"):
            raise ValueError(f"pairing {pairing!r}: 'interleaved' or 'half' is wanted")
        if len(axes) > 3 or (grid is not None and len(grid) != len(axes)):
            raise ValueError("up to three axes, and a grid of as many")
        if inv_freq is not None and len(inv_freq) != sum(axes) // 2:
            raise ValueError(f"inv_freq: {sum(axes) // 2} values are wanted, not {len(inv_freq)}")
        if _f32(q_scale) == 0.0 or not theta > 0.0:
            raise ValueError("q_scale must not be 0 (as fp32), and theta must be positive")
        if norm and _f32(eps) == 0.0:
            raise ValueError("eps must not be 0 (as fp32) with norm: the library takes that for 1e-6")
        for what, v in (("axes", axes), ("grid", grid or ()), ("start", start)):
            if any(not -(1 << 31) <= int(x) < 1 << 31 for x in v):      # (ctypes would wrap it round)
                raise ValueError(f"{what}: 32-bit integers are wanted, not {tuple(v)}")
        three = lambda v: (c_int32 * 3)(*[int(x) for x in v])  # noqa: E731
        freq = (c_double * len(inv_freq))(*[float(f) for f in inv_freq]) if inv_freq is not None else None
        self.torch_dtype = _dtype(dtype)
        self.cfg = HlaHeadsConfig(B, H, N, d, _CODES[self.torch_dtype], HLA_PAIR_HALVES if pairing == "half" else HLA_PAIR_ADJACENT, 1 if norm else 0,
                                  len(axes), three(axes), three(grid or ()), three(start), eps, q_scale, theta, freq)
        self.ctx = _create("hla_heads_create", byref(self.cfg))
        self.cfg.inv_freq = None            # (copied by the library)
        self.device = device
        self._rows, self._out, self._weight = torch.Size((B, N, H, d)), torch.Size((B, H, N, d)), torch.Size((d,))
        self._places = {2: (torch.Size((N, len(axes))), 0), 3: (torch.Size((B, N, len(axes))), N * len(axes))}
        self._new, self._new_dw = _Maker(self._out, self.torch_dtype, device), _Maker(self._weight, torch.float32, device)
        self._make_workspace("hla_heads_workspace_bytes", device)
        self._slots = [_Slot(what) for what in ("q", "k", "v", "dq", "dk", "dv")]
        self._forward, self._backward = load_library().hla_heads_forward, load_library().hla_heads_backward

    def _strided(self, t, slot, device):
        """The tensor's place and strides for the library, in a slot of its own (reused: a context serves one call at a time)."""
        row = self._slots[slot]
        if t.dtype is not self.torch_dtype or t.shape != self._rows or t.get_device() != device:
            _here(t, row.what, self.torch_dtype, self._rows, device)
        strides = t.stride()
        if strides != row.strides:
            sb, sn, sh, sd = strides
            H, d = self.cfg.H, self.cfg.d
            if (sd != 1 and d > 1) or (sh != d and H > 1):
                raise ValueError(f"{row.what}: the {H} x {d} channels of a token must be contiguous")
            row.rows.batch_stride, row.rows.token_stride = sb, sn
            row.strides = strides
        row.rows.data = t.data_ptr()
        return row.at

    def _positions(self, p, device):
        if p is None:
            return 0, 0
        shape, batch_stride = self._places.get(p.dim(), self._places[3])
        return _dense(p, "positions", torch.int32, shape, device), batch_stride

    def forward(self, q=None, k=None, v=None, wq=None, wk=None, positions=None, Q=None, K=None, V=None, stream=None):
        """q, k, v [B,N,H,d] (None: left out) -> Q, K, V [B,H,N,d].  wq, wk: norm weights [d] (None: ones)."""
        dt, dev, shape = self.torch_dtype, _device(), self._out
        rows, outs, at = [None] * 3, [Q, K, V], [0] * 3
        for i, t in enumerate((q, k, v)):
            if t is not None:
                rows[i] = self._strided(t, i, dev)
                if outs[i] is None:
                    outs[i] = self._new(dev)
                    at[i] = outs[i].data_ptr()
                    continue
            if outs[i] is not None:
                at[i] = _dense(outs[i], "output", dt, shape, dev)
        pos, pos_batch = self._positions(positions, dev) if positions is not None else (0, 0)
        st = self._forward(self.ctx, rows[0], rows[1], rows[2], _dense(wq, "wq", dt, self._weight, dev) if wq is not None else 0,
                           _dense(wk, "wk", dt, self._weight, dev) if wk is not None else 0, pos, pos_batch, at[0], at[1], at[2], _stream(stream))
        if st != HLA_OK:
            raise HlaError(st, "hla_heads_forward")
        return outs

    def backward(self, dQ=None, dK=None, dV=None, q=None, k=None, v=None, dq=None, dk=None, dv=None, wq=None, wk=None, positions=None, dwq=None, dwk=None,
                 stream=None):
        """Writes the gradients of q, k, v into dq, dk, dv (views [B,N,H,d]; only where dQ, dK, dV are given) and returns those of the norm
        weights (fp32 [d]; None without norm).  v is accepted next to q and k and not read."""
        dt, dev, f32 = self.torch_dtype, _device(), torch.float32
        self._workspace_here(dev)
        norm = self.cfg.norm == 1
        x = [self._strided(t, i, dev) if norm and t is not None else None for i, t in enumerate((q, k))]
        out = [self._strided(t, 3 + i, dev) if t is not None else None for i, t in enumerate((dq, dk, dv))]
        if norm and dQ is not None and dwq is None:
            dwq = self._new_dw(dev)
        if norm and dK is not None and dwk is None:
            dwk = self._new_dw(dev)
        pos, pos_batch = self._positions(positions, dev)
        shape, w = self._out, self._weight
        st = self._backward(self.ctx, _dense(dQ, "dQ", dt, shape, dev), _dense(dK, "dK", dt, shape, dev), _dense(dV, "dV", dt, shape, dev), x[0], x[1],
                            _dense(wq, "wq", dt, w, dev), _dense(wk, "wk", dt, w, dev), pos, pos_batch, out[0], out[1], out[2], _dense(dwq, "dwq", f32, w, dev),
                            _dense(dwk, "dwk", f32, w, dev), self._scratch, self._need, _stream(stream))
        if st != HLA_OK:
            raise HlaError(st, "hla_heads_backward")
        return dwq, dwk


class AdamW(_Owner):
    """One AdamW step over a list of tensors (hla_adamw_*).  params: fp32 or bf16; grads: fp32 or bf16, read where they are at every step
    (set_grads names others); copies: bf16 copies of fp32 params that a step rewrites.  state: "f32", or "q8" for moments of one byte with a scale
    per 128 elements.  ms, vs (and m_scales, v_scales) are made with zeros where they are not given.  weight_decay, lr_mul: a number, or one for each tensor.
    norm: fp32 scalar that receives the norm of the gradients in steps with max_norm > 0 (made where not given)."""
    _destroy = "hla_adamw_destroy"

    def __init__(self, params, grads, ms=None, vs=None, m_scales=None, v_scales=None, copies=None, state=None, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0,
                 lr_mul=1.0, seed=0, norm=None, device="cuda"):
        n = len(params)
        state = state or ("q8" if ms and ms[0].dtype is torch.uint8 else "f32")
        if state not in ("f32", "q8"):
            raise ValueError(f"state {state!r}: 'f32' or 'q8' is wanted")
        q8 = state == "q8"
        kind, groups = torch.uint8 if q8 else torch.float32, lambda p: (p.numel() + 127) // 128
        make = lambda size, dt: [torch.zeros(size(p), dtype=dt, device=p.device) for p in params]  # noqa: E731
        ms = make(torch.Tensor.numel, kind) if ms is None else ms
        vs = make(torch.Tensor.numel, kind) if vs is None else vs
        if q8:
            m_scales = make(groups, torch.float32) if m_scales is None else m_scales
            v_scales = make(groups, torch.float32) if v_scales is None else v_scales
        each = lambda v: [float(x) for x in v] if hasattr(v, "__len__") else [float(v)] * n  # noqa: E731
        decay, mul = each(weight_decay), each(lr_mul)
        for what, v in (("grads", grads), ("ms", ms), ("vs", vs), ("m_scales", m_scales), ("v_scales", v_scales), ("copies", copies), ("weight_decay", decay), ("lr_mul", mul)):
            if v is not None and len(v) != n:
                raise ValueError(f"{what}: one for each of the {n} params is wanted, not {len(v)}")
        if any(_f32(x) == 0.0 for x in mul):
            raise ValueError("lr_mul must not be 0 (as fp32): leave out tensors that are not trained")
        rows = (HlaAdamwTensor * n)()
        for i, p in enumerate(params):
            if p.dtype not in _CODES or grads[i].dtype not in _CODES:
                raise ValueError(f"params[{i}], grads[{i}]: torch.float32 or torch.bfloat16 is wanted")
            size, rows_of = p.numel(), groups(p)
            count = lambda t, what, dt, k: 0 if t is None else _dense(t, f"{what}[{i}]", dt) if t.numel() == k else self._wrong(what, i, k, t)  # noqa: E731
            rows[i] = HlaAdamwTensor(_dense(p, f"params[{i}]", p.dtype), count(copies[i] if copies else None, "copies", torch.bfloat16, size),
                                     count(grads[i], "grads", grads[i].dtype, size), count(ms[i], "ms", kind, size), count(vs[i], "vs", kind, size),
                                     count(m_scales[i], "m_scales", torch.float32, rows_of) if q8 else 0, count(v_scales[i], "v_scales", torch.float32, rows_of) if q8 else 0,
                                     size, mul[i], decay[i], _CODES[p.dtype], _CODES[grads[i].dtype])
        self.norm = torch.zeros((), dtype=torch.float32, device=device) if norm is None else norm
        _scalar(self.norm, "norm", torch.float32)
        cfg = HlaAdamwConfig(betas[0], betas[1], eps, HLA_STATE_Q8 if q8 else HLA_STATE_F32, seed)
        self.ctx = _create("hla_adamw_create", byref(cfg), rows, n)
        # the library only borrows pointers
        keep = lambda v: None if v is None else list(v)  # noqa: E731
        self.params, self.grads, self.ms, self.vs, self.m_scales, self.v_scales, self.copies = map(keep, (params, grads, ms, vs, m_scales, v_scales, copies))
        self.steps = 0
        self._make_workspace("hla_adamw_workspace_bytes", self.norm.device)
        self._on, self._norm = self.norm.get_device(), self.norm.data_ptr()
        self._step = load_library().hla_adamw_step

    @staticmethod
    def _wrong(what, i, k, t):
        raise ValueError(f"{what}[{i}]: {k} elements are wanted, not {t.numel()}")

    def set_grads(self, grads):
        if len(grads) != len(self.grads):
            raise ValueError(f"grads: {len(self.grads)} are wanted, not {len(grads)}")
        for i, (new, old) in enumerate(zip(grads, self.grads)):
            _dense(new, f"grads[{i}]", old.dtype)
            if new.numel() != old.numel():
                self._wrong("grads", i, old.numel(), new)
        st = load_library().hla_adamw_set_grads(self.ctx, (c_void_p * len(grads))(*[g.data_ptr() for g in grads]), len(grads))
        if st != HLA_OK:
            raise HlaError(st, "hla_adamw_set_grads")
        self.grads = list(grads)

    def step(self, lr, step=None, max_norm=0.0, grad_scale=1.0, stream=None):
        """lr: a number, or an fp32 CUDA scalar that the step reads.  step: its number from 1 on (None: counted here), or an int64 CUDA scalar: with
        both on the device a captured step can be replayed with new values."""
        a = HlaAdamwStepArgs(0.0, 1, 0, 0, max_norm, grad_scale, self._norm)
        if a.grad_scale == 0.0:
            raise ValueError("grad_scale must not be 0 (as fp32)")
        if a.max_norm == 0.0 and max_norm != 0.0:
            raise ValueError(f"max_norm: {max_norm} is 0 as fp32, which stands for no norm")
        if isinstance(lr, torch.Tensor):
            a.lr_device = _scalar(lr, "lr", torch.float32)
        else:
            a.lr = lr
        if isinstance(step, torch.Tensor):
            a.step_device = _scalar(step, "step", torch.int64)
        else:
            a.step = self.steps + 1 if step is None else step
        if self._on != _device():
            raise ValueError(f"the tensors are on cuda:{self._on}, but the current device is cuda:{_device()}")
        st = self._step(self.ctx, byref(a), self._scratch, self._need, _stream(stream))
        if st != HLA_OK:
            raise HlaError(st, "hla_adamw_step")
        if not isinstance(step, torch.Tensor):
            self.steps = a.step


class Scan(_Owner):
    """Gated linear recurrence h_t = a_t h_{t-1} + u_t over tokens (hla_scan_*), a = exp(g) (gate "log") or sigmoid(g) (gate "sigmoid"), u = x or, with
    convex, (1 - a) x; and its backward.  x, g [B,N,C], channels contiguous; states are fp32 [B,C]."""
    _destroy = "hla_scan_destroy"

    def __init__(self, B, N, C, dtype="bf16", gate="log", convex=False, device="cuda"):
        if gate not in ("log", "sigmoid"):
            raise ValueError(f"gate {gate!r}: 'log' or 'sigmoid' is wanted")
        self.torch_dtype = _dtype(dtype)
        self.cfg = HlaScanConfig(B, N, C, _CODES[self.torch_dtype], HLA_GATE_SIGMOID if gate == "sigmoid" else HLA_GATE_LOG, 1 if convex else 0, 0, 0, 0, 0)
        self._make()
        self._made_for = self._seen = None
        self.device = device
        self._shape, self._state = torch.Size((B, N, C)), torch.Size((B, C))
        self._new, self._new_state = _Maker(self._shape, self.torch_dtype, device), _Maker(self._state, torch.float32, device)
        self._make_workspace("hla_scan_workspace_bytes", device)
        if self.workspace is not None:
            self.workspace[:HLA_SCAN_STATUS_BYTES].zero_()
        self._forward, self._backward = load_library().hla_scan_forward, load_library().hla_scan_backward

    def _make(self):
        new = _create("hla_scan_create", byref(self.cfg))
        self.close()
        self.ctx = new

    def _strides(self, x, g, device):
        """Follows the strides of x and g (a context has those it was made for)."""
        dt, shape = self.torch_dtype, self._shape
        if x.dtype is not dt or x.shape != shape or x.get_device() != device or g.dtype is not dt or g.shape != shape or g.get_device() != device:
            _here(x, "x", dt, shape, device)
            _here(g, "g", dt, shape, device)
        strides = x.stride(), g.stride()
        if self._need > HLA_SCAN_STATUS_BYTES:
            self._workspace_here(device)
        if strides == self._seen:
            return
        B, N, C = self._shape
        want = []
        for (sb, sn, sc), what in zip(strides, ("x", "g")):
            if sc != 1 and C > 1:
                raise ValueError(f"{what}: the channels of a token must be contiguous")
            if (N > 1 and sn < C) or (B > 1 and sb < C):
                raise ValueError(f"{what}: tokens must not share memory")
            sn = sn if N > 1 else C
            want += [sb if B > 1 else N * sn, sn]
        if want != self._made_for:
            c = self.cfg
            c.x_batch_stride, c.x_token_stride, c.g_batch_stride, c.g_token_stride = want
            self._make()
            self._made_for = want
        self._seen = strides

    def _scratch_on(self, device):
        """The workspace, but on another device than its own (where it is not needed) none."""
        return (self._scratch, self._need) if device == self._on else (0, 0)

    def device_status(self, stream=None) -> int:
        """Synchronises the stream: HLA_OK, or HLA_ERR_DEVICE_TIMEOUT where a wait between blocks has run out since this was last asked."""
        return int(load_library().hla_scan_last_device_status(self.ctx, self._scratch, _stream(stream)))

    def forward(self, x, g, h0=None, h=None, h_last=None, stream=None):
        """h [B,N,C] and the state behind the last token.  h_last may be the tensor h0."""
        dev, f32 = _device(), torch.float32
        self._strides(x, g, dev)
        h = self._new(dev) if h is None else h
        h_last = self._new_state(dev) if h_last is None else h_last
        st = self._forward(self.ctx, x.data_ptr(), g.data_ptr(), _dense(h0, "h0", f32, self._state, dev), _dense(h, "h", self.torch_dtype, self._shape, dev),
                           _dense(h_last, "h_last", f32, self._state, dev), *self._scratch_on(dev), _stream(stream))
        if st != HLA_OK:
            raise HlaError(st, "hla_scan_forward")
        return h, h_last

    def backward(self, x, g, h, dh, h0=None, dlast=None, dx=None, dg=None, stream=None):
        """dx, dg [B,N,C] and, where h0 is given, its gradient (else None).  h: what forward returned; dlast: gradient of the state behind the last token."""
        dev, f32, dt, shape = _device(), torch.float32, self.torch_dtype, self._shape
        self._strides(x, g, dev)
        dx = self._new(dev) if dx is None else dx
        dg = self._new(dev) if dg is None else dg
        dh0 = self._new_state(dev) if h0 is not None else None
        st = self._backward(self.ctx, x.data_ptr(), g.data_ptr(), _dense(h0, "h0", f32, self._state, dev), _dense(h, "h", dt, shape, dev),
                            _dense(dh, "dh", dt, shape, dev), _dense(dlast, "dlast", f32, self._state, dev), _dense(dx, "dx", dt, shape, dev),
                            _dense(dg, "dg", dt, shape, dev), 0 if dh0 is None else dh0.data_ptr(), *self._scratch_on(dev), _stream(stream))
        if st != HLA_OK:
            raise HlaError(st, "hla_scan_backward")
        return dx, dg, dh0

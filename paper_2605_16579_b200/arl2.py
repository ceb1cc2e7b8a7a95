"""ctypes binding of ``libarl2.so`` (the C ABI in ``include/arl2.h``), same names.

Argument marshalling only: every step of the layer runs in the library's CUDA kernels.
PyTorch appears here as the owner of device memory and streams -- tensors are passed as
``data_ptr()`` and the current CUDA stream as a ``void*``.  There is no fallback: if the
library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libarl2.so")

ARL2_BF16, ARL2_FP32 = 0, 1
ARL2_FLAG_FORCE_SIMT = 1
ARL2_FLAG_TOKEN_GATES = 2
ARL2_FLAG_GATE_SCALAR = 4
ARL2_FLAG_GATE_ELEMENTWISE = 8
ARL2_FLAG_DELTA_DECAYED_PREDICTION = 32
ARL2_CACHE_CAUSAL = 1
ARL2_NORM_NONE, ARL2_NORM_LAYER, ARL2_NORM_RMS, ARL2_NORM_TOKEN, ARL2_NORM_HEAD, ARL2_NORM_LENGTH = range(6)
ARL2_MODULATION_FP32_RESIDUAL = 1


def ARL2_FLAG_DEBUG_WAIT_LIMIT(polls: int) -> int:
    return (polls + 1) << 16

EXPORTS = (
    "arl2_workspace_bytes", "arl2_create", "arl2_set_params", "arl2_denoise_step", "arl2_commit",
    "arl2_reset", "arl2_get_state", "arl2_set_state", "arl2_sync_status", "arl2_launch_count",
    "arl2_set_profile_events", "arl2_commit_static_scratch", "arl2_commit_delta", "arl2_commit_tokens", "arl2_teacher_step", "arl2_commit_decay_tokens",
    "arl2_step_kernel_name", "arl2_destroy", "arl2_last_error", "arl2_version", "arl2_debug_set_wait_limit", "arl2_debug_set_walk_wait_limit", "arl2_clean_pass", "arl2_denoise_step_token_level",
    "arl2_projection_workspace_bytes", "arl2_set_projections", "arl2_project_in", "arl2_project_out",
    "arl2_cache_page_bytes", "arl2_cache_workspace_bytes", "arl2_cache_least_workspace_bytes", "arl2_cache_create", "arl2_cache_set_workspace",
    "arl2_cache_append", "arl2_cache_attend", "arl2_cache_destroy",
    "arl2_modulate", "arl2_modulate_backward", "arl2_modulation_workspace_bytes", "arl2_rotate", "arl2_rotate_backward", "arl2_rotation_workspace_bytes",
    "arl2_recurrence_workspace_bytes", "arl2_recur", "arl2_recur_backward",
)


class Arl2Error(RuntimeError):
    pass


class arl2_config(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("B", ctypes.c_int32), ("H", ctypes.c_int32), ("L", ctypes.c_int32), ("D", ctypes.c_int32),
        ("io_dtype", ctypes.c_int32),
        ("softmax_scale", ctypes.c_float), ("l2_eps", ctypes.c_float),
        ("commit_rule", ctypes.c_int32), ("flags", ctypes.c_uint32),
    ]


class arl2_cache_config(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("kv_heads", ctypes.c_int32), ("page_tokens", ctypes.c_int32), ("num_pages", ctypes.c_int32),
        ("max_pages", ctypes.c_int32), ("rope_rows", ctypes.c_int32),
    ]


class arl2_rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch_stride", ctypes.c_int64), ("row_stride", ctypes.c_int64)]


class arl2_modulation_config(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32), ("frame_tokens", ctypes.c_int32), ("norm", ctypes.c_int32), ("post_norm", ctypes.c_int32),
        ("eps", ctypes.c_float), ("flags", ctypes.c_uint32),
    ]


class arl2_rotation_config(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32), ("kv_heads", ctypes.c_int32), ("rope_rows", ctypes.c_int32), ("axis_pairs", ctypes.c_int32 * 3),
        ("grid_rows", ctypes.c_int32), ("grid_columns", ctypes.c_int32), ("norm", ctypes.c_int32), ("eps", ctypes.c_float),
    ]


class arl2_recurrence_config(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("block_tokens", ctypes.c_int32)]


_lib = None


def load(build_if_missing: bool = False) -> ctypes.CDLL:
    """Load the library (once).  Raises Arl2Error when it is absent: there is no CPU path."""
    global _lib
    if _lib is not None:
        return _lib
    if build_if_missing:
        from . import build as _build

        _build.build_library()
    if not os.path.exists(LIB_PATH):
        raise Arl2Error(
            f"{LIB_PATH} is missing: build it with `python -m paper_2605_16579_b200.build` "
            "(nvcc, sm_100a).  The layer has no CPU or PyTorch fallback."
        )
    lib = ctypes.CDLL(LIB_PATH)
    vp, cp = ctypes.c_void_p, ctypes.POINTER(arl2_config)
    lib.arl2_workspace_bytes.restype = ctypes.c_size_t
    lib.arl2_workspace_bytes.argtypes = [cp]
    lib.arl2_create.restype = ctypes.c_int
    lib.arl2_create.argtypes = [cp, vp, vp, ctypes.c_size_t, vp, ctypes.POINTER(vp)]
    lib.arl2_set_params.restype = ctypes.c_int
    lib.arl2_set_params.argtypes = [vp] * 7
    lib.arl2_denoise_step.restype = ctypes.c_int
    lib.arl2_denoise_step.argtypes = [vp] * 7
    lib.arl2_commit.restype = ctypes.c_int
    lib.arl2_commit.argtypes = [vp] * 5
    lib.arl2_clean_pass.restype = ctypes.c_int
    lib.arl2_clean_pass.argtypes = [vp] * 8
    lib.arl2_denoise_step_token_level.restype = ctypes.c_int
    lib.arl2_denoise_step_token_level.argtypes = [vp] * 8
    lib.arl2_projection_workspace_bytes.restype = ctypes.c_size_t
    lib.arl2_projection_workspace_bytes.argtypes = [cp]
    lib.arl2_set_projections.restype = ctypes.c_int
    lib.arl2_set_projections.argtypes = [vp] * 7 + [ctypes.c_size_t, vp]
    lib.arl2_project_in.restype = ctypes.c_int
    lib.arl2_project_in.argtypes = [vp] * 7
    lib.arl2_project_out.restype = ctypes.c_int
    lib.arl2_project_out.argtypes = [vp] * 4
    lib.arl2_teacher_step.restype = ctypes.c_int
    lib.arl2_teacher_step.argtypes = [vp, vp, vp, vp, ctypes.c_int32, vp, vp]
    lib.arl2_commit_delta.restype = ctypes.c_int
    lib.arl2_commit_delta.argtypes = [vp] * 6
    lib.arl2_commit_decay_tokens.restype = ctypes.c_int
    lib.arl2_commit_decay_tokens.argtypes = [vp] * 5
    lib.arl2_commit_tokens.restype = ctypes.c_int
    lib.arl2_commit_tokens.argtypes = [vp] * 6
    lib.arl2_reset.restype = ctypes.c_int
    lib.arl2_reset.argtypes = [vp, ctypes.c_int32, vp]
    lib.arl2_get_state.restype = ctypes.c_int
    lib.arl2_get_state.argtypes = [vp, vp, vp]
    lib.arl2_set_state.restype = ctypes.c_int
    lib.arl2_set_state.argtypes = [vp, vp, vp]
    lib.arl2_sync_status.restype = ctypes.c_int
    lib.arl2_sync_status.argtypes = [vp, vp]
    lib.arl2_debug_set_wait_limit.restype = ctypes.c_int
    lib.arl2_debug_set_wait_limit.argtypes = [vp, ctypes.c_int32]
    lib.arl2_debug_set_walk_wait_limit.restype = ctypes.c_int
    lib.arl2_debug_set_walk_wait_limit.argtypes = [vp, ctypes.c_int32]
    lib.arl2_set_profile_events.restype = ctypes.c_int
    lib.arl2_set_profile_events.argtypes = [vp, vp, vp]
    lib.arl2_commit_static_scratch.restype = ctypes.c_int
    lib.arl2_commit_static_scratch.argtypes = [cp] + [vp] * 9
    ccp, i32, i64, u32 = ctypes.POINTER(arl2_cache_config), ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32
    lib.arl2_cache_page_bytes.restype = ctypes.c_size_t
    lib.arl2_cache_page_bytes.argtypes = [cp, ccp]
    lib.arl2_cache_workspace_bytes.restype = ctypes.c_size_t
    lib.arl2_cache_workspace_bytes.argtypes = [cp, ccp]
    lib.arl2_cache_least_workspace_bytes.restype = ctypes.c_size_t
    lib.arl2_cache_least_workspace_bytes.argtypes = [cp, ccp]
    lib.arl2_cache_set_workspace.restype = ctypes.c_int
    lib.arl2_cache_set_workspace.argtypes = [vp, vp, ctypes.c_size_t, vp]
    lib.arl2_cache_create.restype = ctypes.c_int
    lib.arl2_cache_create.argtypes = [vp, ccp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp, ctypes.POINTER(vp)]
    lib.arl2_cache_append.restype = ctypes.c_int
    lib.arl2_cache_append.argtypes = [vp, vp, i64, i64, vp, i64, i64, i32, vp, vp, vp, vp]
    lib.arl2_cache_attend.restype = ctypes.c_int
    lib.arl2_cache_attend.argtypes = [vp, vp, i64, i64, i32, vp, vp, u32, vp, vp]
    lib.arl2_cache_destroy.restype = None
    lib.arl2_cache_destroy.argtypes = [vp]
    rp, mp, tp = ctypes.POINTER(arl2_rows), ctypes.POINTER(arl2_modulation_config), ctypes.POINTER(arl2_rotation_config)
    lib.arl2_modulation_workspace_bytes.restype = ctypes.c_size_t
    lib.arl2_modulation_workspace_bytes.argtypes = [cp, mp, i32]
    lib.arl2_modulate.restype = ctypes.c_int
    lib.arl2_modulate.argtypes = [vp, mp, i32, vp, vp, rp, rp, rp, vp, vp, vp, vp, vp]
    lib.arl2_modulate_backward.restype = ctypes.c_int
    lib.arl2_modulate_backward.argtypes = [vp, mp, i32, vp, vp, vp, vp, rp, rp] + [vp] * 10 + [ctypes.c_size_t, vp]
    lib.arl2_rotation_workspace_bytes.restype = ctypes.c_size_t
    lib.arl2_rotation_workspace_bytes.argtypes = [cp, tp, i32]
    lib.arl2_rotate.restype = ctypes.c_int
    lib.arl2_rotate.argtypes = [vp, tp, vp, vp, i32, rp, rp, vp, vp, vp, vp, vp, vp, vp]
    lib.arl2_rotate_backward.restype = ctypes.c_int
    lib.arl2_rotate_backward.argtypes = [vp, tp, vp, vp, i32, vp, vp, rp, rp] + [vp] * 9 + [ctypes.c_size_t, vp]
    ep = ctypes.POINTER(arl2_recurrence_config)
    lib.arl2_recurrence_workspace_bytes.restype = ctypes.c_size_t
    lib.arl2_recurrence_workspace_bytes.argtypes = [cp, ep, i32, i32]
    lib.arl2_recur.restype = ctypes.c_int
    lib.arl2_recur.argtypes = [vp, ep, i32, rp, rp, rp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.arl2_recur_backward.restype = ctypes.c_int
    lib.arl2_recur_backward.argtypes = [vp, ep, i32, vp, rp, rp, rp] + [vp] * 9 + [ctypes.c_size_t, vp]
    lib.arl2_launch_count.restype = ctypes.c_uint64
    lib.arl2_launch_count.argtypes = [vp]
    lib.arl2_step_kernel_name.restype = ctypes.c_char_p
    lib.arl2_step_kernel_name.argtypes = [vp]
    lib.arl2_destroy.restype = None
    lib.arl2_destroy.argtypes = [vp]
    lib.arl2_last_error.restype = ctypes.c_char_p
    lib.arl2_version.restype = ctypes.c_char_p
    _lib = lib
    return lib


def _check(status: int, what: str):
    if status != 0:
        msg = load().arl2_last_error().decode()
        raise Arl2Error(f"{what} failed with status {status}: {msg}")


def _ptr(t):
    return None if t is None else t.data_ptr()


# The handle of a device's current stream; a torch without the short cut makes a Stream object of it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def make_config(B, H, L, D, dtype, softmax_scale=0.0, l2_eps=0.0, commit_rule=0, flags=0):
    io = {"bf16": ARL2_BF16, "fp32": ARL2_FP32, torch.bfloat16: ARL2_BF16,
          torch.float32: ARL2_FP32}[dtype]
    return arl2_config(ctypes.sizeof(arl2_config), B, H, L, D, io, softmax_scale, l2_eps,
                       commit_rule, flags)


def arl2_workspace_bytes(cfg: arl2_config) -> int:
    n = load().arl2_workspace_bytes(ctypes.byref(cfg))
    if n == 0:
        raise Arl2Error("arl2_workspace_bytes: " + load().arl2_last_error().decode())
    return n


class Layer:
    """One context: owns (through torch) the state and workspace buffers it hands to the library.

    Methods mirror the C entry points one to one; tensors must be contiguous CUDA tensors of
    the configured dtype.
    """

    def __init__(self, B, H, L, D, dtype="bf16", device="cuda:0", softmax_scale=0.0, l2_eps=0.0,
                 flags=0, state=None, workspace=None):
        """``state`` ([B, H, D, D] fp32) and ``workspace`` (uint8, >= arl2_workspace_bytes, 256-byte
        aligned) may be handed in by a caller that manages its own device memory; by default torch
        allocates them here."""
        lib = load()
        self.cfg = make_config(B, H, L, D, dtype, softmax_scale, l2_eps, 0, flags)
        self.B, self.H, self.L, self.D = B, H, L, D
        self.flags = flags
        self.device = torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self._index = self.device.index
        self.dtype = torch.bfloat16 if self.cfg.io_dtype == ARL2_BF16 else torch.float32
        self._lib = lib
        self.workspace_bytes = arl2_workspace_bytes(self.cfg)
        with torch.cuda.device(self.device):
            if state is None:
                state = torch.empty(B, H, D, D, dtype=torch.float32, device=self.device)
            if workspace is None:
                workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=self.device)
            self._want(state, (B, H, D, D), torch.float32, "state")
            if not (workspace.get_device() == self._index and workspace.dtype == torch.uint8 and workspace.is_contiguous()
                    and workspace.numel() >= self.workspace_bytes):
                raise Arl2Error(f"workspace: expected >= {self.workspace_bytes} contiguous bytes on {self.device}")
            self.state, self.workspace = state, workspace
            ctx = ctypes.c_void_p()
            _check(lib.arl2_create(ctypes.byref(self.cfg), _ptr(self.state), _ptr(self.workspace),
                                   self.workspace.numel(), _stream(), ctypes.byref(ctx)),
                   "arl2_create")
        self._ctx = ctx
        self._params = None  # keeps the parameter tensors alive
        self.reset()

    # -- the C entry points ------------------------------------------------------------
    def set_params(self, wq=None, wk=None, wv=None, rope_cos=None, rope_sin=None):
        for w in (wq, wk, wv):
            if w is not None:
                self._want(w, (self.H, self.D, self.D), self.dtype, "feature map")
        for t in (rope_cos, rope_sin):
            if t is not None:
                self._want(t, (self.L, self.D // 2), torch.float32, "rope table")
        self._params = (wq, wk, wv, rope_cos, rope_sin)
        self._run("arl2_set_params", _ptr(wq), _ptr(wk), _ptr(wv), _ptr(rope_cos), _ptr(rope_sin))

    def denoise_step(self, q, k, v, gate_logits, out=None):
        shape = (self.B, self.L, self.H, self.D)
        for t in (q, k, v):
            self._want(t, shape, self.dtype, "q/k/v")
        gshape = ((self.B, self.L) if self.flags & ARL2_FLAG_GATE_SCALAR else
                  (self.B, self.L, self.H, self.D) if self.flags & ARL2_FLAG_GATE_ELEMENTWISE else
                  (self.B, self.L, self.H))
        self._want(gate_logits, gshape, torch.float32, "gate_logits")
        if out is None:
            out = torch.empty(shape, dtype=self.dtype, device=self.device)
        else:
            self._want(out, shape, self.dtype, "out")
        self._run("arl2_denoise_step", _ptr(q), _ptr(k), _ptr(v), _ptr(gate_logits), _ptr(out))
        return out

    def clean_pass(self, q, k_clean, v_clean, gate_logits, decay_logits, out=None):
        """The clean pass in one call: the output against the pre-update state, then the commit."""
        shape = (self.B, self.L, self.H, self.D)
        for t in (q, k_clean, v_clean):
            self._want(t, shape, self.dtype, "q/k_clean/v_clean")
        gshape = ((self.B, self.L) if self.flags & ARL2_FLAG_GATE_SCALAR else
                  (self.B, self.L, self.H, self.D) if self.flags & ARL2_FLAG_GATE_ELEMENTWISE else
                  (self.B, self.L, self.H))
        self._want(gate_logits, gshape, torch.float32, "gate_logits")
        self._want(decay_logits, (self.B, self.H), torch.float32, "decay_logits")
        if out is None:
            out = torch.empty(shape, dtype=self.dtype, device=self.device)
        else:
            self._want(out, shape, self.dtype, "out")
        self._run("arl2_clean_pass", _ptr(q), _ptr(k_clean), _ptr(v_clean), _ptr(gate_logits), _ptr(decay_logits), _ptr(out))
        return out

    def denoise_step_token_level(self, q, k, v, gate_logits, alpha_logits=None, out=None):
        """Comparison mode: token i reads the state advanced by the block's tokens before it."""
        shape = (self.B, self.L, self.H, self.D)
        for t in (q, k, v):
            self._want(t, shape, self.dtype, "q/k/v")
        self._want(gate_logits, (self.B, self.L, self.H), torch.float32, "gate_logits")
        if alpha_logits is not None:
            self._want(alpha_logits, (self.B, self.L, self.H), torch.float32, "alpha_logits")
        if out is None:
            out = torch.empty(shape, dtype=self.dtype, device=self.device)
        else:
            self._want(out, shape, self.dtype, "out")
        self._run("arl2_denoise_step_token_level", _ptr(q), _ptr(k), _ptr(v), _ptr(gate_logits), _ptr(alpha_logits), _ptr(out))
        return out

    def set_projections(self, w_q, w_k, w_v, w_g, w_o):
        """W_q, W_k, W_v, W_o [d, d] and W_g [d, H], bf16, (in, out): the module around the core."""
        d = self.H * self.D
        for w in (w_q, w_k, w_v, w_o):
            self._want(w, (d, d), torch.bfloat16, "projection weight")
        self._want(w_g, (d, self.H), torch.bfloat16, "gate weight")
        n = load().arl2_projection_workspace_bytes(ctypes.byref(self.cfg))
        with torch.cuda.device(self.device):
            self._pack = torch.empty(n, dtype=torch.uint8, device=self.device)
            self._proj = (w_q, w_k, w_v, w_g, w_o)
            _check(load().arl2_set_projections(self._ctx, _ptr(w_q), _ptr(w_k), _ptr(w_v), _ptr(w_g), _ptr(w_o),
                                               _ptr(self._pack), n, _stream()), "arl2_set_projections")

    def project_in(self, x, q=None, k=None, v=None, gate_logits=None):
        """x [B, L, d] bf16 -> q, k, v [B, L, H, D] bf16 and gate logits [B, L, H] fp32."""
        d = self.H * self.D
        self._want(x, (self.B, self.L, d), torch.bfloat16, "x")
        shape = (self.B, self.L, self.H, self.D)
        q, k, v = (torch.empty(shape, dtype=torch.bfloat16, device=self.device) if t is None else t for t in (q, k, v))
        if gate_logits is None:
            gate_logits = torch.empty(self.B, self.L, self.H, dtype=torch.float32, device=self.device)
        for t in (q, k, v):
            self._want(t, shape, torch.bfloat16, "q/k/v")
        self._want(gate_logits, (self.B, self.L, self.H), torch.float32, "gate_logits")
        self._run("arl2_project_in", _ptr(x), _ptr(q), _ptr(k), _ptr(v), _ptr(gate_logits))
        return q, k, v, gate_logits

    def project_out(self, o, y=None):
        """o [B, L, H, D] bf16 -> y [B, L, d] bf16 = o W_o."""
        d = self.H * self.D
        self._want(o, (self.B, self.L, self.H, self.D), torch.bfloat16, "o")
        if y is None:
            y = torch.empty(self.B, self.L, d, dtype=torch.bfloat16, device=self.device)
        self._want(y, (self.B, self.L, d), torch.bfloat16, "y")
        self._run("arl2_project_out", _ptr(o), _ptr(y))
        return y

    def teacher_step(self, q, k_cache, v_cache, out=None):
        """Eq. 1: softmax attention of q [B, L, H, D] over a cache [B, Lk, H, D] (no rotation, no state)."""
        shape = (self.B, self.L, self.H, self.D)
        self._want(q, shape, self.dtype, "q")
        lk = int(k_cache.shape[1])
        self._want(k_cache, (self.B, lk, self.H, self.D), self.dtype, "k_cache")
        self._want(v_cache, (self.B, lk, self.H, self.D), self.dtype, "v_cache")
        if out is None:
            out = torch.empty(shape, dtype=self.dtype, device=self.device)
        else:
            self._want(out, shape, self.dtype, "out")
        self._run("arl2_teacher_step", _ptr(q), _ptr(k_cache), _ptr(v_cache), lk, _ptr(out))
        return out

    def commit(self, k_clean, v_clean, decay_logits):
        shape = (self.B, self.L, self.H, self.D)
        self._want(k_clean, shape, self.dtype, "k_clean")
        self._want(v_clean, shape, self.dtype, "v_clean")
        self._want(decay_logits, (self.B, self.H), torch.float32, "decay_logits")
        self._run("arl2_commit", _ptr(k_clean), _ptr(v_clean), _ptr(decay_logits))

    def commit_delta(self, k_clean, v_clean, decay_logits, beta_logits=None):
        """Eq. 4 as printed, at block level: S <- sigmoid(a) S + K'^T diag(beta) (V' - K' S_old)."""
        shape = (self.B, self.L, self.H, self.D)
        self._want(k_clean, shape, self.dtype, "k_clean")
        self._want(v_clean, shape, self.dtype, "v_clean")
        self._want(decay_logits, (self.B, self.H), torch.float32, "decay_logits")
        if beta_logits is not None:
            self._want(beta_logits, (self.B, self.L, self.H), torch.float32, "beta_logits")
        self._run("arl2_commit_delta", _ptr(k_clean), _ptr(v_clean), _ptr(decay_logits), _ptr(beta_logits))

    def commit_decay_tokens(self, k_clean, v_clean, alpha_logits):
        """Gated-linear commit with one forget gate per token: S <- alpha_l S + K'_l^T V'_l in order."""
        shape = (self.B, self.L, self.H, self.D)
        self._want(k_clean, shape, self.dtype, "k_clean")
        self._want(v_clean, shape, self.dtype, "v_clean")
        self._want(alpha_logits, (self.B, self.L, self.H), torch.float32, "alpha_logits")
        self._run("arl2_commit_decay_tokens", _ptr(k_clean), _ptr(v_clean), _ptr(alpha_logits))

    def commit_tokens(self, k_clean, v_clean, alpha_logits=None, beta_logits=None):
        """Eq. 4 token by token with per-token gates [B, L, H] (None = gate 1); the layer must have
        been created with flags=ARL2_FLAG_TOKEN_GATES."""
        shape = (self.B, self.L, self.H, self.D)
        self._want(k_clean, shape, self.dtype, "k_clean")
        self._want(v_clean, shape, self.dtype, "v_clean")
        for name, g in (("alpha_logits", alpha_logits), ("beta_logits", beta_logits)):
            if g is not None:
                self._want(g, (self.B, self.L, self.H), torch.float32, name)
        self._run("arl2_commit_tokens", _ptr(k_clean), _ptr(v_clean), _ptr(alpha_logits), _ptr(beta_logits))

    def reset(self, stream_index: int = -1):
        self._run("arl2_reset", stream_index)

    def get_state(self) -> torch.Tensor:
        """Copy of S as a CPU fp32 tensor [B, H, D, D] (synchronises the stream)."""
        dst = torch.empty(self.B, self.H, self.D, self.D, dtype=torch.float32)
        with torch.cuda.device(self.device):
            self._run("arl2_get_state", _ptr(dst))
            torch.cuda.current_stream().synchronize()
        return dst

    def set_state(self, src: torch.Tensor):
        src = src.to(torch.float32).contiguous()
        assert tuple(src.shape) == (self.B, self.H, self.D, self.D)
        with torch.cuda.device(self.device):
            self._run("arl2_set_state", _ptr(src))
            torch.cuda.current_stream().synchronize()

    def sync_status(self):
        self._run("arl2_sync_status")

    def debug_set_wait_limit(self, polls: int):
        """Test hook: bounded waits in the tensor-core kernels give up after ``polls`` polls (< 0: default)."""
        _check(load().arl2_debug_set_wait_limit(self._ctx, polls), "arl2_debug_set_wait_limit")

    def debug_set_walk_wait_limit(self, polls: int):
        """Test hook: the same for the first wait of the last thread block of ``commit_tokens``' walk alone."""
        _check(load().arl2_debug_set_walk_wait_limit(self._ctx, polls), "arl2_debug_set_walk_wait_limit")

    def set_profile_events(self, before: "torch.cuda.Event", after: "torch.cuda.Event"):
        """The next denoise_step records these events around its dominant kernel."""
        for ev in (before, after):
            if not ev.cuda_event:   # torch creates the CUDA event lazily, at its first record
                ev.record()
        _check(load().arl2_set_profile_events(self._ctx, ctypes.c_void_p(before.cuda_event),
                                              ctypes.c_void_p(after.cuda_event)),
               "arl2_set_profile_events")

    @property
    def launch_count(self) -> int:
        return int(load().arl2_launch_count(self._ctx))

    @property
    def step_kernel(self) -> str:
        return load().arl2_step_kernel_name(self._ctx).decode()

    def close(self):
        if self._ctx is not None:
            load().arl2_destroy(self._ctx)
            self._ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- helpers -----------------------------------------------------------------------
    def _run(self, name, *args):
        """One call of the library on the layer's device and its current stream.

        The device is switched only where another one is current, and the stream's handle is taken as it is: with a
        device context and a Stream object per call the host needed 13.0 us for a commit, now 7.6; 20.8 for a step, now 13.5."""
        current = torch.cuda.current_device()
        index = self.device.index
        if index is None or index == current:
            status = getattr(self._lib, name)(self._ctx, *args, _raw_stream(current))
        else:
            with torch.cuda.device(index):
                status = getattr(self._lib, name)(self._ctx, *args, _raw_stream(index))
        if status != 0:
            _check(status, name)

    def _want(self, t, shape, dtype, what):
        # (get_device: the GPU's number, -1 on the host; a kernel on one GPU is not to be given another's memory)
        if t.shape == shape and t.dtype is dtype and t.get_device() == self._index and t.is_contiguous() and isinstance(t, torch.Tensor):
            return
        if not (isinstance(t, torch.Tensor) and t.get_device() == self._index and t.is_contiguous()
                and tuple(t.shape) == tuple(shape) and t.dtype == dtype):
            raise Arl2Error(f"{what}: expected a contiguous tensor {tuple(shape)} {dtype} on {self.device}, got "
                            f"{tuple(t.shape)} {t.dtype} on {t.device}")


class Cache:
    """A paged key/value cache held in 4 bits (the arl2_cache_* entry points), of a layer's B, H, D and dtype.

    ``page_table`` ([B, max_pages] int32) says which pages of the pool hold a stream's tokens, in order; the caller hands them
    out.  ``pages`` (uint8 [num_pages, page_bytes], uncleared) and ``page_table`` (filled with -1) are made here unless they
    are handed in.  Rotary tables: [positions, D/2] fp32, both or neither.  Calls on one cache are for one stream at a time.

    ``workspace``: scratch (uint8, at least ``workspace_range(...)[0]`` bytes) that this cache uses beside others whose calls do not
    overlap with its own, as in a stack whose layers run one after the other: ``Cache(..., workspace=first.workspace)``.  By default
    ``workspace_range(...)[1]`` bytes of its own, with which no call waits for room.
    """

    def __init__(self, layer, num_pages, max_pages, kv_heads=None, page_tokens=64, rope_cos=None, rope_sin=None, pages=None, page_table=None,
                 workspace=None):
        lib = load()
        self._lib, self._cache = lib, None
        self._append, self._attend = lib.arl2_cache_append, lib.arl2_cache_attend
        self.layer, self.device, self.dtype, self._index = layer, layer.device, layer.dtype, layer._index
        self._B, self._H, self._D = layer.B, layer.H, layer.D
        self.kv_heads = layer.H if kv_heads is None else kv_heads
        rows = 0 if rope_cos is None else int(rope_cos.shape[0])
        self.cfg = arl2_cache_config(ctypes.sizeof(arl2_cache_config), self.kv_heads, page_tokens, num_pages, max_pages, rows)
        self.page_bytes = lib.arl2_cache_page_bytes(ctypes.byref(layer.cfg), ctypes.byref(self.cfg))
        if self.page_bytes == 0:
            raise Arl2Error("arl2_cache_page_bytes: " + lib.arl2_last_error().decode())
        for t in (rope_cos, rope_sin):
            if t is not None:
                layer._want(t, (rows, layer.D // 2), torch.float32, "rope table")
        with torch.cuda.device(self.device):
            if pages is None:
                pages = torch.empty(num_pages, self.page_bytes, dtype=torch.uint8, device=self.device)
            if page_table is None:
                page_table = torch.full((layer.B, max_pages), -1, dtype=torch.int32, device=self.device)
            layer._want(pages, (num_pages, self.page_bytes), torch.uint8, "pages")
            layer._want(page_table, (layer.B, max_pages), torch.int32, "page_table")
            self.pages, self.page_table, self._rope = pages, page_table, (rope_cos, rope_sin)
            handle = ctypes.c_void_p()
            _check(lib.arl2_cache_create(layer._ctx, ctypes.byref(self.cfg), _ptr(pages), _ptr(page_table), _ptr(rope_cos), _ptr(rope_sin),
                                         None, 0, _stream(), ctypes.byref(handle)), "arl2_cache_create")
            self._cache = handle
            if workspace is None:
                n = lib.arl2_cache_workspace_bytes(ctypes.byref(layer.cfg), ctypes.byref(self.cfg))
                workspace = torch.empty(n, dtype=torch.uint8, device=self.device)
        self.set_workspace(workspace)

    @staticmethod
    def workspace_range(layer, num_pages, max_pages, kv_heads=None, page_tokens=64):
        """Bytes of scratch of such a cache: the least that it works with, and those with which every call is as fast as it can be."""
        lib = load()
        cfg = arl2_cache_config(ctypes.sizeof(arl2_cache_config), layer.H if kv_heads is None else kv_heads, page_tokens, num_pages, max_pages, 0)
        sizes = tuple(f(ctypes.byref(layer.cfg), ctypes.byref(cfg)) for f in (lib.arl2_cache_least_workspace_bytes, lib.arl2_cache_workspace_bytes))
        if 0 in sizes:
            raise Arl2Error("arl2_cache_workspace_bytes: " + lib.arl2_last_error().decode())
        return sizes

    @property
    def workspace(self):
        return self._workspace

    def set_workspace(self, workspace):
        """Scratch of later calls (arl2_cache_set_workspace); what was captured before keeps the scratch that it was captured with."""
        if not (isinstance(workspace, torch.Tensor) and workspace.get_device() == self._index and workspace.dtype == torch.uint8
                and workspace.is_contiguous()):
            raise Arl2Error(f"workspace: expected contiguous uint8 on {self.device}")
        self._run(self._lib.arl2_cache_set_workspace, workspace.data_ptr(), workspace.numel())
        self._workspace = workspace

    def append(self, k, v, start, held=False):
        """Rows k, v [B, T, kv_heads, D] of tokens start[b] .. start[b] + T - 1 (start: int32 [B], negative: idle stream), keys
        rotated to their positions.  ``held=True`` returns (k, v) as the cache now holds them, which may also be given as a pair
        of tensors to write to."""
        tokens = k.shape[1]
        shape = (self._B, tokens, self.kv_heads, self._D)
        k_batch, k_token = self._rows(k, shape, "k")
        v_batch, v_token = self._rows(v, shape, "v")
        self.layer._want(start, (self._B,), torch.int32, "start")
        kh = vh = None
        if held is True:
            kh, vh = self._empty(k, shape), self._empty(v, shape)
        elif held is not False:
            kh, vh = held
            self.layer._want(kh, shape, self.dtype, "held keys")
            self.layer._want(vh, shape, self.dtype, "held values")
        self._run(self._append, k.data_ptr(), k_batch, k_token, v.data_ptr(), v_batch, v_token, tokens, start.data_ptr(), _ptr(kh), _ptr(vh))
        return None if kh is None else (kh, vh)

    def attend(self, q, lengths, q_start=None, causal=False, out=None):
        """Attention of q [B, T, H, D] over the first lengths[b] tokens held (int32 [B]); q is rotated to its positions
        q_start[b] + i, by default those of the last T tokens.  ``causal``: query i sees the tokens up to its own position."""
        queries = q.shape[1]
        shape = (self._B, queries, self._H, self._D)
        q_batch, q_token = self._rows(q, shape, "q")
        want = self.layer._want
        want(lengths, (self._B,), torch.int32, "lengths")
        if q_start is not None:
            want(q_start, (self._B,), torch.int32, "q_start")
        if out is None:
            out = self._empty(q, shape)
        else:
            want(out, shape, self.dtype, "out")
        self._run(self._attend, q.data_ptr(), q_batch, q_token, queries, lengths.data_ptr(), _ptr(q_start), ARL2_CACHE_CAUSAL if causal else 0, out.data_ptr())
        return out

    def close(self):
        if self._cache is not None:
            self._lib.arl2_cache_destroy(self._cache)
            self._cache = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- helpers -----------------------------------------------------------------------
    def _rows(self, t, shape, what):
        """The batch and token strides of a tensor whose heads and channels are contiguous."""
        if isinstance(t, torch.Tensor) and t.get_device() == self._index and t.dtype is self.dtype and t.shape == shape:
            token = shape[2] * shape[3]
            if t.is_contiguous():
                return shape[1] * token, token
            st = t.stride()
            if st[3] == 1 and (st[2] == shape[3] or shape[2] == 1):
                # (a dimension of one element may have any stride)
                return st[0] if shape[0] > 1 else 0, st[1] if shape[1] > 1 else token
        raise Arl2Error(f"{what}: expected a tensor {tuple(shape)} {self.dtype} on {self.device} with contiguous heads and channels, got "
                        f"{tuple(t.shape)} {t.dtype} with strides {tuple(t.stride())} on {t.device}")

    def _empty(self, like, shape):
        # (empty_like costs the host less than empty, and gives the same for a contiguous tensor)
        return torch.empty_like(like) if like.is_contiguous() else torch.empty(shape, dtype=self.dtype, device=self.device)

    def _run(self, call, *args):
        if self.layer._ctx is None:
            raise Arl2Error(f"{call.__name__}: the cache's layer has been closed")
        current = torch.cuda.current_device()
        index = self.device.index
        if index is None or index == current:
            status = call(self._cache, *args, _raw_stream(current))
        else:
            with torch.cuda.device(index):
                status = call(self._cache, *args, _raw_stream(index))
        if status != 0:
            _check(status, call.__name__)



class _BlockOp:
    """What stands around a layer's core shares its context: B, H, D, dtype, device.

    The calls record nothing for autograd, whatever requires a gradient: ``backward`` is called with what ``forward`` was given, by hand or from an
    autograd function (examples/train_memory.py has three)."""

    def __init__(self, layer):
        self.layer = layer
        self.device, self.dtype = layer.device, layer.dtype
        self._lib, self._index = layer._lib, layer.device.index
        self._B, self._H, self._D = layer.B, layer.H, layer.D
        self._width = layer.H * layer.D
        self._sizes = {}
        self._byte = torch.empty(1, dtype=torch.uint8, device=self.device) if self.device.type == "cuda" and self._lib is not None else None

    def _run(self, call, *args):
        ctx = self.layer._ctx
        if ctx is None:
            raise Arl2Error(f"{call.__name__}: the layer has been closed")
        current, index = torch.cuda.current_device(), self._index
        if index is None or index == current:
            status = call(ctx, *args, _raw_stream(current))
        else:
            with torch.cuda.device(index):
                status = call(ctx, *args, _raw_stream(index))
        if status != 0:
            _check(status, call.__name__)

    def _strided(self, t, shape, dtype, what, inner):
        """arl2_rows of a tensor [B, rows, ...] whose dimensions from `inner` on are contiguous."""
        if isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.get_device() == self._index:
            st, row = t.stride(), 1
            for i in range(len(shape) - 1, inner - 1, -1):
                if shape[i] != 1 and st[i] != row:
                    break
                row *= shape[i]
            else:
                # (a dimension of one element may have any stride)
                return arl2_rows(t.data_ptr(), st[0] if shape[0] > 1 else 0, st[1] if shape[1] > 1 else row)
        raise Arl2Error(f"{what}: expected a tensor {tuple(shape)} {dtype} on {self.device} with contiguous rows, got "
                        + (f"{tuple(t.shape)} {t.dtype} with strides {tuple(t.stride())} on {t.device}" if isinstance(t, torch.Tensor) else f"{t!r}"))

    def _heads(self, t, shape, what):
        """The same of [B, T, heads, D] of the layer's type, whose heads and channels are contiguous."""
        if isinstance(t, torch.Tensor) and t.dtype is self.dtype and t.shape == shape and t.get_device() == self._index:
            batch, token, head, channel = t.stride()
            if channel == 1 and (head == shape[3] or shape[2] == 1):
                return arl2_rows(t.data_ptr(), batch if shape[0] > 1 else 0, token if shape[1] > 1 else shape[2] * shape[3])
        return self._strided(t, shape, self.dtype, what, 2)

    def _fp32(self, like):
        """A contiguous fp32 tensor of another's shape, or None."""
        return None if like is None else torch.empty_like(like, memory_format=torch.contiguous_format)

    def _bytes(self, call, *key):
        """What a size query of the library says: a function of the configurations and the tokens alone, asked once."""
        n = self._sizes.get(key)
        if n is None:
            n = call(ctypes.byref(self.layer.cfg), self._cfg, *key)
            if n == 0:
                raise Arl2Error(f"{call.__name__}: " + self._lib.arl2_last_error().decode())
            if len(self._sizes) < 256:
                self._sizes[key] = n
        return n

    def _tokens(self, t, what, dims):
        shape = t.shape if isinstance(t, torch.Tensor) else ()
        if len(shape) != dims:
            raise Arl2Error(f"{what}: expected a tensor of {dims} dimensions")
        return shape[1]

    def _scratch(self, n, given):
        """Scratch of one call: the caller's, or memory that torch hands out for the current stream (or the graph being captured)."""
        if given is None:
            return self._byte.new_empty(n)      # (costs the host less than torch.empty)
        if not (isinstance(given, torch.Tensor) and given.get_device() == self._index and given.dtype == torch.uint8 and given.is_contiguous()):
            raise Arl2Error(f"workspace: expected contiguous uint8 on {self.device}")
        return given


class Modulation(_BlockOp):
    """The end of one block part and the beginning of the next (arl2_modulate): r = x + gate P(y), n = N(r) weight (1 + scale) + shift.

    ``frame_tokens`` tokens share a row of gate, scale and shift.  ``norm`` (N) is "layer" or "rms", ``post`` (P) one of them or None.
    ``residual``: the type of x and r, the layer's or torch.float32.
    """

    def __init__(self, layer, frame_tokens, norm="layer", post=None, eps=0.0, residual=None):
        super().__init__(layer)
        self.frame_tokens = frame_tokens
        self.residual = self.dtype if residual is None else residual
        if self.residual not in (self.dtype, torch.float32):
            raise Arl2Error(f"residual: expected {self.dtype} or {torch.float32}, got {residual}")
        names = {None: ARL2_NORM_NONE, "layer": ARL2_NORM_LAYER, "rms": ARL2_NORM_RMS}
        if norm not in names or post not in names:
            raise Arl2Error(f"norm, post: expected one of {list(names)}, got {norm!r} and {post!r}")
        flags = ARL2_MODULATION_FP32_RESIDUAL if self.residual is not self.dtype else 0
        self.cfg = arl2_modulation_config(ctypes.sizeof(arl2_modulation_config), frame_tokens, names[norm], names[post], eps, flags)
        self._cfg = ctypes.byref(self.cfg)
        self._modulate = self._lib.arl2_modulate
        self.workspace_bytes(1)     # (what the library refuses is refused here)

    def workspace_bytes(self, tokens):
        return self._bytes(self._lib.arl2_modulation_workspace_bytes, tokens)

    def _modulation(self, t, shape, what):
        if t is None:
            return None
        if isinstance(t, torch.Tensor) and t.dtype is torch.float32 and t.get_device() == self._index and t.shape == shape:
            batch, frame, channel = t.stride()
            if channel == 1:
                return arl2_rows(t.data_ptr(), batch if shape[0] > 1 else 0, frame if shape[1] > 1 else 0)
        return self._strided(t, shape, torch.float32, what, 2)

    def _weight(self, t, what):
        if t is not None:
            self.layer._want(t, (self._width,), torch.float32, what)
        return _ptr(t)

    def forward(self, x, y=None, gate=None, scale=None, shift=None, weight=None, post_weight=None, normed=True, r=None, n=None):
        """x, y [B, T, H * D]; gate, scale, shift fp32 [B, ceil(T / frame_tokens), H * D] with contiguous rows (others may be strided or
        expanded); weights fp32 [H * D].  Returns (r, n): r is x itself where there is no y, n is None with ``normed=False``.  ``r`` may
        be given as x, and ``n`` as y: in place."""
        tokens = self._tokens(x, "x", 3)
        shape, want = (self._B, tokens, self._width), self.layer._want
        want(x, shape, self.residual, "x")
        if y is None:
            if r is not None:
                raise Arl2Error("r: nothing is written without y")
        else:
            want(y, shape, self.dtype, "y")
            if r is None:
                r = torch.empty_like(x)
            else:
                want(r, shape, self.residual, "r")
        if not normed:
            if n is not None:
                raise Arl2Error("n: nothing is written with normed=False")
        elif n is None:
            n = torch.empty_like(y) if y is not None else torch.empty(shape, dtype=self.dtype, device=self.device)
        else:
            want(n, shape, self.dtype, "n")
        rows = (shape[0], -(-tokens // self.frame_tokens), shape[2])
        self._run(self._modulate, self._cfg, tokens, x.data_ptr(), _ptr(y), self._modulation(gate, rows, "gate"), self._modulation(scale, rows, "scale"),
                  self._modulation(shift, rows, "shift"), None if weight is None else self._weight(weight, "weight"),
                  None if post_weight is None else self._weight(post_weight, "post_weight"), _ptr(r), _ptr(n))
        return (x if r is None else r), n

    def backward(self, r, dn=None, dr=None, y=None, gate=None, scale=None, shift=None, weight=None, post_weight=None, workspace=None):
        """Gradients (dx, dy, dgate, dscale, dshift, dweight, dpost_weight) from dn and dr, those of n and r (either may be None); None for
        what forward was called without.  ``r`` is what forward returned; ``shift`` is not read."""
        tokens = self._tokens(dn if dr is None else dr, "dn or dr", 3)
        shape, want = (self._B, tokens, self._width), self.layer._want
        if r is not None or dn is not None:
            want(r, shape, self.residual, "r") if isinstance(r, torch.Tensor) else self._tokens(r, "r", 3)
        for t, kind, what in ((dn, self.dtype, "dn"), (dr, self.residual, "dr"), (y, self.dtype, "y")):
            if t is not None:
                want(t, shape, kind, what)
        rows = (shape[0], -(-tokens // self.frame_tokens), shape[2])
        gate_rows, scale_rows = self._modulation(gate, rows, "gate"), self._modulation(scale, rows, "scale")
        self._modulation(shift, rows, "shift")
        w, pw = self._weight(weight, "weight"), self._weight(post_weight, "post_weight")
        dx = torch.empty_like(r if r is not None else dr)
        dy = None if y is None else torch.empty_like(y)
        normed = dn is not None
        dgate, dscale, dshift = self._fp32(gate), self._fp32(scale) if normed else None, self._fp32(shift) if normed else None
        dweight, dpost = self._fp32(weight) if normed else None, self._fp32(post_weight)
        ws = self._scratch(self.workspace_bytes(tokens), workspace)
        self._run(self._lib.arl2_modulate_backward, self._cfg, tokens, _ptr(r), _ptr(dn), _ptr(dr), _ptr(y), gate_rows, scale_rows, w, pw,
                  dx.data_ptr(), _ptr(dy), _ptr(dgate), _ptr(dscale), _ptr(dshift), _ptr(dweight), _ptr(dpost), ws.data_ptr(), ws.numel())
        return dx, dy, dgate, dscale, dshift, dweight, dpost


class Rotation(_BlockOp):
    """Queries and keys on their way to the attention (arl2_rotate): a norm, then the rotation of adjacent channels by positions along up
    to three axes.

    ``rope_cos``, ``rope_sin`` fp32 [positions, D / 2]; ``axes``: pairs that turn with the first, second and third position (the rest do not turn).
    Positions of token l: (start + l // (rows * columns), l // columns % rows, l % columns) for ``grid`` = (rows, columns).
    ``norm``: None, "token" (RMS over all heads), "head" (RMS over one) or "l2" (rows of length one, the layer's L2Norm).
    """

    def __init__(self, layer, rope_cos, rope_sin, axes, grid=(1, 1), norm=None, kv_heads=None, eps=0.0):
        super().__init__(layer)
        self.kv_heads = layer.H if kv_heads is None else kv_heads
        names = {None: ARL2_NORM_NONE, "token": ARL2_NORM_TOKEN, "head": ARL2_NORM_HEAD, "l2": ARL2_NORM_LENGTH}
        if norm not in names:
            raise Arl2Error(f"norm: expected one of {list(names)}, got {norm!r}")
        self.norm = norm
        self._tokens(rope_cos, "rope table", 2)
        rows = rope_cos.shape[0]
        for t in (rope_cos, rope_sin):
            layer._want(t, (rows, self._D // 2), torch.float32, "rope table")
        axes = tuple(axes) + (0,) * (3 - len(axes))
        if len(axes) != 3:
            raise Arl2Error(f"axes: expected at most three, got {axes}")
        self._rope = (rope_cos, rope_sin)
        self._tables = (rope_cos.data_ptr(), rope_sin.data_ptr())
        self.cfg = arl2_rotation_config(ctypes.sizeof(arl2_rotation_config), self.kv_heads, rows, axes, grid[0], grid[1], names[norm], eps)
        self._cfg = ctypes.byref(self.cfg)
        self.workspace_bytes(1)

    def workspace_bytes(self, tokens):
        return self._bytes(self._lib.arl2_rotation_workspace_bytes, tokens)

    def _where(self, start, positions, tokens):
        if start is not None:
            self.layer._want(start, (self._B,), torch.int32, "start")
        if positions is not None:
            self.layer._want(positions, (self._B, tokens, 3), torch.int32, "positions")
        return _ptr(start), _ptr(positions)

    def _weight(self, t, heads, what):
        if t is not None:
            self.layer._want(t, (heads * self._D if self.norm == "token" else self._D,), torch.float32, what)
        return _ptr(t)

    def forward(self, q, k=None, start=None, positions=None, q_weight=None, k_weight=None, q_out=None, k_out=None):
        """q [B, T, H, D], k [B, T, kv_heads, D] (heads and channels contiguous) -> the same, rotated, contiguous; (q, None) without k.
        ``start`` int32 [B] (first position along the first axis), or ``positions`` int32 [B, T, 3].  An output given as its own
        contiguous input is written in place."""
        tokens = self._tokens(q, "q", 4)
        q_shape, k_shape = (self._B, tokens, self._H, self._D), (self._B, tokens, self.kv_heads, self._D)
        q_rows = self._heads(q, q_shape, "q")
        k_rows = None if k is None else self._heads(k, k_shape, "k")
        if q_out is None:
            q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
        else:
            self.layer._want(q_out, q_shape, self.dtype, "q_out")
        if k_out is not None:
            self.layer._want(k_out, k_shape, self.dtype, "k_out")
        elif k is not None:
            k_out = torch.empty_like(k, memory_format=torch.contiguous_format)
        self._run(self._lib.arl2_rotate, self._cfg, *self._tables, tokens, q_rows, k_rows, *self._where(start, positions, tokens),
                  self._weight(q_weight, self._H, "q_weight"), self._weight(k_weight, self.kv_heads, "k_weight"), q_out.data_ptr(), _ptr(k_out))
        return q_out, k_out

    def backward(self, dq_out, dk_out=None, q=None, k=None, start=None, positions=None, q_weight=None, k_weight=None, workspace=None):
        """Gradients (dq, dk, dq_weight, dk_weight) from those of the outputs; q and k are the inputs (needed only with a norm).
        None for what forward was called without."""
        tokens = self._tokens(dq_out, "dq_out", 4)
        q_shape, k_shape = (self._B, tokens, self._H, self._D), (self._B, tokens, self.kv_heads, self._D)
        self.layer._want(dq_out, q_shape, self.dtype, "dq_out")
        if dk_out is not None:
            self.layer._want(dk_out, k_shape, self.dtype, "dk_out")
        q_rows = None if q is None else self._heads(q, q_shape, "q")
        k_rows = None if k is None else self._heads(k, k_shape, "k")
        dq, dk = torch.empty_like(dq_out), None if dk_out is None else torch.empty_like(dk_out)
        q_w, k_w = self._weight(q_weight, self._H, "q_weight"), self._weight(k_weight, self.kv_heads, "k_weight")
        dq_weight = None if q_weight is None else torch.empty_like(q_weight)
        dk_weight = None if k_weight is None or dk_out is None else torch.empty_like(k_weight)
        ws = None
        if dq_weight is not None or dk_weight is not None or workspace is not None:
            ws = self._scratch(self.workspace_bytes(tokens), workspace)
        self._run(self._lib.arl2_rotate_backward, self._cfg, *self._tables, tokens, dq_out.data_ptr(), _ptr(dk_out), q_rows, k_rows,
                  *self._where(start, positions, tokens), q_w, k_w, dq.data_ptr(), _ptr(dk), _ptr(dq_weight), _ptr(dk_weight), _ptr(ws),
                  0 if ws is None else ws.numel())
        return dq, dk, dq_weight, dk_weight

class Recurrence(_BlockOp):
    """The state over the blocks of a whole sequence (arl2_recur): out_i = q_i S_n for the tokens i of block n of ``block_tokens`` tokens,
    S_{n+1} = sigmoid(a_n) S_n + K_n^T V_n.  Reads and sets no state of the layer."""

    def __init__(self, layer, block_tokens):
        super().__init__(layer)
        self.block_tokens = block_tokens
        self._states = (layer.B, layer.H, layer.D, layer.D)
        self.cfg = arl2_recurrence_config(ctypes.sizeof(arl2_recurrence_config), block_tokens)
        self._cfg = ctypes.byref(self.cfg)
        self.workspace_bytes(1)

    def workspace_bytes(self, tokens, backward=False):
        return self._bytes(self._lib.arl2_recurrence_workspace_bytes, tokens, int(backward))

    def _inputs(self, q, k, v, decay_logits, state):
        tokens = self._tokens(q, "q", 4)
        shape, heads = (self._B, tokens, self._H, self._D), self._heads
        rows = heads(q, shape, "q"), heads(k, shape, "k"), heads(v, shape, "v")
        self.layer._want(decay_logits, (self._B, -(-tokens // self.block_tokens), self._H), torch.float32, "decay_logits")
        if state is not None:
            self._state(state, "state")
        return tokens, shape, rows

    def _state(self, t, what):
        self.layer._want(t, self._states, torch.float32, what)

    def _new_state(self, like):
        return torch.empty(self._states, dtype=torch.float32, device=self.device) if like is None else torch.empty_like(like)

    def forward(self, q, k, v, decay_logits, state=None, final=True, out=None, workspace=None):
        """q, k, v [B, T, H, D] (heads and channels contiguous), decay_logits fp32 [B, ceil(T / block_tokens), H], state fp32 [B, H, D, D] or None
        (zeros) -> (out [B, T, H, D], the state behind the last block, or None with ``final=False``)."""
        tokens, shape, rows = self._inputs(q, k, v, decay_logits, state)
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
        else:
            self.layer._want(out, shape, self.dtype, "out")
        last = self._new_state(state) if final else None
        ws = self._scratch(self.workspace_bytes(tokens), workspace)
        self._run(self._lib.arl2_recur, self._cfg, tokens, *rows, decay_logits.data_ptr(), _ptr(state), out.data_ptr(), _ptr(last), ws.data_ptr(), ws.numel())
        return out, last

    def backward(self, dout, q, k, v, decay_logits, state=None, dstate=None, initial=True, workspace=None):
        """Gradients (dq, dk, dv, ddecay_logits, the gradient of ``state``) from dout [B, T, H, D] and dstate, that of the state behind the last
        block (None: zeros); the last is None with ``initial=False``."""
        tokens, shape, rows = self._inputs(q, k, v, decay_logits, state)
        self.layer._want(dout, shape, self.dtype, "dout")
        if dstate is not None:
            self._state(dstate, "dstate")
        dq, dk, dv = torch.empty_like(dout), torch.empty_like(dout), torch.empty_like(dout)
        ddecay = torch.empty_like(decay_logits)
        first = self._new_state(dstate if state is None else state) if initial else None
        ws = self._scratch(self.workspace_bytes(tokens, True), workspace)
        self._run(self._lib.arl2_recur_backward, self._cfg, tokens, dout.data_ptr(), *rows, decay_logits.data_ptr(), _ptr(state), _ptr(dstate),
                  dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), ddecay.data_ptr(), _ptr(first), ws.data_ptr(), ws.numel())
        return dq, dk, dv, ddecay, first



STATIC_SCRATCH_BYTES = 8 << 20


def commit_static_scratch(cfg: arl2_config, state, k_clean, v_clean, decay_logits, wk=None, wv=None,
                          rope_cos=None, rope_sin=None):
    """arl2_commit_static_scratch: the commit for callers that may not allocate device memory.

    Updates ``state`` ([B, H, D, D] fp32, CUDA) in place; no context, no workspace.  The partial
    sums of the reduction live in an array built into the library (8 MiB per GPU), so shapes
    with B*H*ceil(L/512)*D*D*4 bytes above that are refused, and calls that overlap on the GPU
    must be ordered by the caller.
    """
    with torch.cuda.device(state.device):
        _check(load().arl2_commit_static_scratch(ctypes.byref(cfg), _ptr(state), _ptr(k_clean),
                                                 _ptr(v_clean), _ptr(decay_logits), _ptr(wk), _ptr(wv),
                                                 _ptr(rope_cos), _ptr(rope_sin), _stream()),
               "arl2_commit_static_scratch")

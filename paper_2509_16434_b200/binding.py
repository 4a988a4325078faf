"""Thin ctypes binding of libppo_b200.so: same names as the C ABI, argument marshalling only.

torch is used for device memory and streams; every computation happens inside the library.
The library must exist (build with `python -m paper_2509_16434_b200.build` or
`__graft_entry__.build()`); there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import math
import os
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libppo_b200.so")

PPO_OK = 0
STATUS_NAMES = {0: "OK", 1: "INVALID_ARG", 2: "SHAPE", 3: "ALIGN", 4: "STATE", 5: "CUDA", 6: "TIMEOUT", 7: "UNSUPPORTED"}
(FIELD_DEPTH, FIELD_PROPRIO, FIELD_ACTION, FIELD_LOGP, FIELD_VALUE, FIELD_REWARD, FIELD_DONE, FIELD_ADV, FIELD_RET,
 FIELD_SCRATCH, NUM_FIELDS) = range(11)

EXPORTS = [
    "ppo_status_string", "ppo_buffer_field_bytes", "ppo_buffer_bytes", "ppo_buffer_alloc", "ppo_buffer_free",
    "ppo_buffer_field_ptr", "ppo_buffer_write_step", "ppo_compute_gae", "ppo_shuffle_gather_minibatch",
    "ppo_model_create", "ppo_model_destroy", "ppo_model_param_count", "ppo_model_arena_elems",
    "ppo_model_num_tensors", "ppo_model_tensor_info", "ppo_model_workspace_bytes", "ppo_model_bind",
    "ppo_model_sync_shadow", "ppo_encoder_fwd", "ppo_loss_fwd_bwd", "ppo_encoder_bwd", "ppo_model_zero_grad",
    "ppo_adam_step", "ppo_policy_sample", "ppo_poll_status", "ppo_model_activation_ptr", "ppo_gae_static",
    "ppo_model_sync_masks", "ppo_buffer_write_obs", "ppo_buffer_write_outcome", "ppo_policy_act", "ppo_launch_count",
    "ppo_selftest_wait_timeout", "ppo_buffer_render_depth", "ppo_model_set_sequence", "ppo_shuffle_gather_sequences",
    "ppo_model_read_state", "ppo_state_reset", "ppo_policy_step", "ppo_selftest_first_gradient",
    "ppo_decay_attention_workspace_bytes", "ppo_decay_attention_fwd", "ppo_decay_attention_bwd", "ppo_decay_attention_step",
    "ppo_group_norm_workspace_bytes", "ppo_group_norm_fwd", "ppo_group_norm_bwd", "ppo_token_logp",
    "ppo_token_loss_workspace_bytes", "ppo_token_loss_fwd_bwd",
    "ppo_causal_conv_workspace_bytes", "ppo_causal_conv_fwd", "ppo_causal_conv_bwd", "ppo_causal_conv_step",
    "ppo_selective_scan_workspace_bytes", "ppo_selective_scan_fwd", "ppo_selective_scan_bwd", "ppo_selective_scan_step",
    "ppo_qk_norm_rotate_workspace_bytes", "ppo_qk_norm_rotate_fwd", "ppo_qk_norm_rotate_bwd",
]


class PpoError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)} ({status})")


class BufferDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("N", "T", "H", "W", "P", "A")]


class ModelDesc(C.Structure):
    _fields_ = [("H", C.c_int32), ("W", C.c_int32), ("n_conv", C.c_int32), ("conv_c", C.c_int32 * 8),
                ("conv_k", C.c_int32 * 8), ("n_fc", C.c_int32), ("fc", C.c_int32 * 4), ("P", C.c_int32),
                ("A", C.c_int32), ("norm", C.c_int32), ("embed", C.c_int32), ("n_lstm", C.c_int32),
                ("lstm_h", C.c_int32)]


class Minibatch(C.Structure):
    _fields_ = [("depth_f16", C.c_void_p), ("proprio", C.c_void_p), ("action", C.c_void_p),
                ("logp_old", C.c_void_p), ("value_old", C.c_void_p), ("adv", C.c_void_p), ("ret", C.c_void_p),
                ("index", C.c_void_p), ("B", C.c_int32)]


class DecayAttentionDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("T", "Be", "heads", "kv_heads", "dk", "dv", "dtype")] + \
               [(n, C.c_int64) for n in ("ldq", "ldk", "ldv", "ldo")] + [("scale", C.c_float)]


class GroupNormDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("B", "HW", "C", "groups", "act", "dtype")] + [("ldx", C.c_int64), ("ldy", C.c_int64)]


class TokenDesc(C.Structure):
    _fields_ = [("rows", C.c_int32), ("vocab", C.c_int32), ("dtype", C.c_int32), ("ld", C.c_int64), ("scale", C.c_float)]


class TokenLossCoef(C.Structure):
    _fields_ = [(n, C.c_float) for n in ("clip_low", "clip_high", "kl_coef", "ent_coef", "grad_scale")] + [("B_total", C.c_int32)]


class CausalConvDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("T", "Be", "C", "width", "act", "dtype")] + [("ldx", C.c_int64), ("ldy", C.c_int64)]


class SelectiveScanDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("T", "Be", "channels", "N", "groups", "dtype", "softplus")] + \
               [(n, C.c_int64) for n in ("ldx", "lddt", "ldb", "ldc", "ldz", "ldy")]


class QkNormDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("rows", "heads", "kv_heads", "d", "pairs", "interleaved", "dtype")] + \
               [(n, C.c_int64) for n in ("ldq", "ldk", "ldqo", "ldko")]


_lib = None


def lib():
    """Loads the CUDA library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it first (python -m paper_2509_16434_b200.build)")
        L = C.CDLL(LIB_PATH)
        L.ppo_status_string.restype = C.c_char_p
        L.ppo_buffer_bytes.restype = C.c_size_t
        L.ppo_buffer_field_bytes.restype = C.c_size_t
        L.ppo_buffer_field_bytes.argtypes = [C.POINTER(BufferDesc), C.c_int, C.c_int]
        L.ppo_buffer_field_ptr.restype = C.c_void_p
        L.ppo_buffer_field_ptr.argtypes = [C.c_void_p, C.c_int]
        L.ppo_buffer_alloc.argtypes = [C.POINTER(BufferDesc), C.c_void_p, C.c_size_t, C.POINTER(C.c_void_p)]
        L.ppo_buffer_free.argtypes = [C.c_void_p]
        L.ppo_buffer_write_step.argtypes = [C.c_void_p, C.c_int] + [C.c_void_p] * 8
        L.ppo_compute_gae.argtypes = [C.c_void_p, C.c_void_p, C.c_float, C.c_float, C.c_int, C.c_void_p, C.c_void_p]
        L.ppo_shuffle_gather_minibatch.argtypes = [C.c_void_p, C.c_uint64, C.c_uint32, C.c_int, C.c_int,
                                                   C.POINTER(Minibatch), C.c_void_p]
        L.ppo_model_create.argtypes = [C.POINTER(ModelDesc), C.POINTER(C.c_void_p)]
        L.ppo_model_destroy.argtypes = [C.c_void_p]
        L.ppo_model_param_count.restype = C.c_size_t
        L.ppo_model_param_count.argtypes = [C.c_void_p]
        L.ppo_model_arena_elems.restype = C.c_size_t
        L.ppo_model_arena_elems.argtypes = [C.c_void_p]
        L.ppo_model_num_tensors.argtypes = [C.c_void_p]
        L.ppo_model_tensor_info.argtypes = [C.c_void_p, C.c_int, C.POINTER(C.c_int64), C.POINTER(C.c_int64)]
        L.ppo_model_workspace_bytes.restype = C.c_size_t
        L.ppo_model_workspace_bytes.argtypes = [C.c_void_p, C.c_int]
        L.ppo_model_bind.argtypes = [C.c_void_p] * 7 + [C.c_size_t, C.c_int]
        L.ppo_model_sync_shadow.argtypes = [C.c_void_p, C.c_void_p]
        L.ppo_model_zero_grad.argtypes = [C.c_void_p, C.c_void_p]
        L.ppo_model_sync_masks.argtypes = [C.c_void_p, C.c_int, C.c_void_p]
        L.ppo_encoder_fwd.argtypes = [C.c_void_p, C.POINTER(Minibatch), C.c_int, C.c_int, C.c_void_p, C.c_void_p,
                                      C.c_void_p]
        L.ppo_loss_fwd_bwd.argtypes = [C.c_void_p, C.POINTER(Minibatch), C.c_int, C.c_int, C.c_int, C.c_void_p,
                                       C.c_void_p, C.c_float, C.c_float, C.c_float, C.c_void_p, C.c_void_p,
                                       C.c_void_p, C.c_void_p]
        L.ppo_encoder_bwd.argtypes = [C.c_void_p, C.POINTER(Minibatch), C.c_int, C.c_int, C.c_void_p, C.c_void_p,
                                      C.c_int, C.c_void_p]
        L.ppo_adam_step.argtypes = [C.c_void_p, C.c_float, C.c_float, C.c_float, C.c_float, C.c_int64, C.c_void_p]
        L.ppo_policy_sample.argtypes = [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                        C.c_void_p]
        L.ppo_policy_step.argtypes = [C.c_void_p, C.POINTER(Minibatch), C.c_int] + [C.c_void_p] * 9
        L.ppo_poll_status.argtypes = [C.c_void_p]
        L.ppo_buffer_write_obs.argtypes = [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]
        L.ppo_buffer_write_outcome.argtypes = [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]
        L.ppo_policy_act.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p]
        L.ppo_buffer_render_depth.argtypes = [C.c_void_p, C.c_int, C.c_float, C.c_float, C.c_float, C.c_void_p, C.c_int,
                                              C.c_void_p, C.c_void_p]
        L.ppo_model_set_sequence.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]
        L.ppo_shuffle_gather_sequences.argtypes = [C.c_void_p, C.c_uint64, C.c_uint32, C.c_int, C.c_int,
                                                   C.POINTER(Minibatch), C.c_void_p, C.c_void_p]
        L.ppo_model_read_state.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.ppo_state_reset.argtypes = [C.c_void_p] * 3 + [C.c_int] * 3 + [C.c_void_p]
        L.ppo_launch_count.restype = C.c_uint64
        L.ppo_launch_count.argtypes = []
        L.ppo_selftest_wait_timeout.argtypes = [C.c_longlong, C.c_void_p, C.c_void_p]
        L.ppo_selftest_first_gradient.argtypes = [C.c_void_p, C.POINTER(Minibatch), C.c_int, C.c_int, C.c_int, C.c_void_p]
        L.ppo_gae_static.argtypes = [C.c_void_p] * 4 + [C.c_int, C.c_int, C.c_float, C.c_float, C.c_int] + [C.c_void_p] * 4
        L.ppo_model_activation_ptr.argtypes = [C.c_void_p, C.c_int, C.c_int, C.POINTER(C.c_void_p),
                                               C.POINTER(C.c_size_t)]
        L.ppo_decay_attention_workspace_bytes.restype = C.c_size_t
        L.ppo_decay_attention_workspace_bytes.argtypes = [C.POINTER(DecayAttentionDesc), C.c_int]
        L.ppo_decay_attention_fwd.argtypes = [C.POINTER(DecayAttentionDesc)] + [C.c_void_p] * 9 + [C.c_size_t, C.c_void_p]
        L.ppo_decay_attention_bwd.argtypes = [C.POINTER(DecayAttentionDesc)] + [C.c_void_p] * 13 + [C.c_size_t, C.c_void_p]
        L.ppo_decay_attention_step.argtypes = [C.POINTER(DecayAttentionDesc)] + [C.c_void_p] * 8
        L.ppo_group_norm_workspace_bytes.restype = C.c_size_t
        L.ppo_group_norm_workspace_bytes.argtypes = [C.POINTER(GroupNormDesc), C.c_int]
        L.ppo_group_norm_fwd.argtypes = [C.POINTER(GroupNormDesc), C.c_float] + [C.c_void_p] * 7 + [C.c_size_t, C.c_void_p]
        L.ppo_group_norm_bwd.argtypes = [C.POINTER(GroupNormDesc)] + [C.c_void_p] * 9 + [C.c_int, C.c_void_p, C.c_size_t, C.c_void_p]
        L.ppo_token_logp.argtypes = [C.POINTER(TokenDesc)] + [C.c_void_p] * 5
        L.ppo_token_loss_workspace_bytes.restype = C.c_size_t
        L.ppo_token_loss_workspace_bytes.argtypes = [C.POINTER(TokenDesc)]
        L.ppo_token_loss_fwd_bwd.argtypes = [C.POINTER(TokenDesc), C.POINTER(TokenLossCoef)] + [C.c_void_p] * 7 + \
                                            [C.c_int64, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_size_t, C.c_void_p]
        L.ppo_causal_conv_workspace_bytes.restype = C.c_size_t
        L.ppo_causal_conv_workspace_bytes.argtypes = [C.POINTER(CausalConvDesc)]
        L.ppo_causal_conv_fwd.argtypes = [C.POINTER(CausalConvDesc)] + [C.c_void_p] * 8
        L.ppo_causal_conv_bwd.argtypes = [C.POINTER(CausalConvDesc)] + [C.c_void_p] * 11 + [C.c_int, C.c_void_p, C.c_size_t, C.c_void_p]
        L.ppo_causal_conv_step.argtypes = [C.POINTER(CausalConvDesc)] + [C.c_void_p] * 7
        L.ppo_selective_scan_workspace_bytes.restype = C.c_size_t
        L.ppo_selective_scan_workspace_bytes.argtypes = [C.POINTER(SelectiveScanDesc), C.c_int]
        L.ppo_selective_scan_fwd.argtypes = [C.POINTER(SelectiveScanDesc)] + [C.c_void_p] * 13 + [C.c_size_t, C.c_void_p]
        L.ppo_selective_scan_bwd.argtypes = [C.POINTER(SelectiveScanDesc)] + [C.c_void_p] * 21 + [C.c_int, C.c_void_p, C.c_size_t, C.c_void_p]
        L.ppo_selective_scan_step.argtypes = [C.POINTER(SelectiveScanDesc)] + [C.c_void_p] * 12
        L.ppo_qk_norm_rotate_workspace_bytes.restype = C.c_size_t
        L.ppo_qk_norm_rotate_workspace_bytes.argtypes = [C.POINTER(QkNormDesc)]
        L.ppo_qk_norm_rotate_fwd.argtypes = [C.POINTER(QkNormDesc), C.c_float] + [C.c_void_p] * 9
        L.ppo_qk_norm_rotate_bwd.argtypes = [C.POINTER(QkNormDesc), C.c_float] + [C.c_void_p] * 12 + [C.c_int, C.c_void_p, C.c_size_t, C.c_void_p]
        _lib = L
    return _lib


def _check(status: int, where: str):
    if status != PPO_OK:
        raise PpoError(status, where)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _mbref(mb):
    return C.byref(mb.c if hasattr(mb, "c") else mb)


def _stream(stream=None):
    # the raw handle without a torch.cuda.Stream object around it: every call of the library asks for it
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream


def ppo_status_string(status: int) -> str:
    return lib().ppo_status_string(status).decode()


def ppo_poll_status(stream=None) -> int:
    return lib().ppo_poll_status(_stream(stream))


def buffer_desc(N, T, H, W, P=32, A=12) -> BufferDesc:
    return BufferDesc(N, T, H, W, P, A)


def ppo_buffer_bytes(desc: BufferDesc) -> int:
    return lib().ppo_buffer_bytes(C.byref(desc))


def ppo_buffer_field_bytes(desc: BufferDesc, field: int, depth_elem_bytes: int = 2) -> int:
    return lib().ppo_buffer_field_bytes(C.byref(desc), field, depth_elem_bytes)


class Buffer:
    """Handle of the on-device rollout buffer; owns the torch storage the library carves up."""

    _DT = {FIELD_DEPTH: torch.float16, FIELD_DONE: torch.uint8}

    def __init__(self, desc: BufferDesc, device="cuda"):
        self.desc = desc
        nbytes = ppo_buffer_bytes(desc)
        if nbytes == 0:
            raise PpoError(1, "ppo_buffer_bytes")
        self.storage = torch.empty(nbytes, dtype=torch.uint8, device=device)
        h = C.c_void_p()
        _check(lib().ppo_buffer_alloc(C.byref(desc), _ptr(self.storage), nbytes, C.byref(h)), "ppo_buffer_alloc")
        self.handle = h
        self._slabs = self._views()  # the slabs stay where they are for the life of the handle

    def _views(self):
        d = self.desc
        shapes = {FIELD_DEPTH: (d.T, d.N, d.H, d.W), FIELD_PROPRIO: (d.T, d.N, d.P), FIELD_ACTION: (d.T, d.N, d.A),
                  FIELD_SCRATCH: (ppo_buffer_field_bytes(d, FIELD_SCRATCH) // 4,)}
        typed = {dt: self.storage.view(dt) for dt in (torch.float32, torch.float16, torch.uint8)}
        ptr, start = lib().ppo_buffer_field_ptr, self.storage.data_ptr()
        views = {}
        for f in range(NUM_FIELDS):
            dt, shape = self._DT.get(f, torch.float32), shapes.get(f, (d.T, d.N))
            stride = tuple(math.prod(shape[i + 1:]) for i in range(len(shape)))
            views[f] = typed[dt].as_strided(shape, stride, (ptr(self.handle, f) - start) // dt.itemsize)
        return views

    def close(self):
        if self.handle:
            lib().ppo_buffer_free(self.handle)
            self.handle = None
            self._slabs = {}

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def field(self, f: int) -> torch.Tensor:
        """A torch view of one slab (no copy)."""
        # A new tensor on a view made with the handle, not by the first call, whose mode (inference, a transform) would stay with
        # it.  Asking the library for the address and slicing, casting and shaping the storage each time took 8 us, a rollout step
        # of 16 envs that looks at seven slabs 83 us of host time instead of 29.
        v = self._slabs.get(f)
        if v is None:
            raise TypeError(f"no slab {f!r}" if self.handle else "the buffer is closed")
        return v.detach()


def ppo_buffer_write_step(buf: Buffer, t: int, depth, proprio, action, logp, value, reward, done, stream=None):
    _check(lib().ppo_buffer_write_step(buf.handle, t, _ptr(depth), _ptr(proprio), _ptr(action), _ptr(logp),
                                       _ptr(value), _ptr(reward), _ptr(done), _stream(stream)),
           "ppo_buffer_write_step")


def ppo_buffer_write_obs(buf: Buffer, t: int, depth, proprio, stream=None):
    _check(lib().ppo_buffer_write_obs(buf.handle, t, _ptr(depth), _ptr(proprio), _stream(stream)),
           "ppo_buffer_write_obs")


def ppo_buffer_write_outcome(buf: Buffer, t: int, reward, done, stream=None):
    _check(lib().ppo_buffer_write_outcome(buf.handle, t, _ptr(reward), _ptr(done), _stream(stream)),
           "ppo_buffer_write_outcome")


def ppo_buffer_render_depth(buf: Buffer, t: int, hfov: float, near: float, far: float, plane, prims, stream=None):
    """plane [N,4] fp32, prims [N,K,8] fp32 device tensors: renders the scenes into slab row t of the depth field."""
    _check(lib().ppo_buffer_render_depth(buf.handle, t, hfov, near, far, _ptr(plane), prims.shape[1], _ptr(prims),
                                         _stream(stream)), "ppo_buffer_render_depth")


def ppo_launch_count() -> int:
    return int(lib().ppo_launch_count())


def ppo_selftest_wait_timeout(limit_cycles: int, gave_up, stream=None):
    _check(lib().ppo_selftest_wait_timeout(limit_cycles, _ptr(gave_up), _stream(stream)),
           "ppo_selftest_wait_timeout")


def ppo_selftest_first_gradient(m: Model, mb: MinibatchArrays, row0: int, rows: int, one_launch: bool, stream=None):
    _check(lib().ppo_selftest_first_gradient(m.handle, _mbref(mb), row0, rows, int(one_launch), _stream(stream)),
           "ppo_selftest_first_gradient")


def ppo_compute_gae(buf: Buffer, last_value, gamma: float, lam: float, normalize=True, stats_out=None,
                    stream=None):
    """normalize: False / True (two launches) / 2 (one cooperative launch)."""
    _check(lib().ppo_compute_gae(buf.handle, _ptr(last_value), gamma, lam, int(normalize), _ptr(stats_out),
                                 _stream(stream)), "ppo_compute_gae")


def ppo_gae_static(reward, value, done, last_value, gamma: float, lam: float, normalize: bool, adv, ret,
                   stats_out=None, stream=None):
    """GAE (+ advantage normalisation) on bare [T, N] device tensors without any device allocation by the
    library: for callers that may not call cudaMalloc (fixed arenas, fixed memory budgets).  At most 524288 envs;
    calls that could overlap on the GPU must be serialised (they share one scratch array inside the library)."""
    T, N = reward.shape
    _check(lib().ppo_gae_static(_ptr(reward), _ptr(value), _ptr(done), _ptr(last_value), T, N, gamma, lam,
                                int(normalize), _ptr(adv), _ptr(ret), _ptr(stats_out), _stream(stream)),
           "ppo_gae_static")


class MinibatchArrays:
    """Caller-owned device arrays of one gathered minibatch."""

    def __init__(self, desc: BufferDesc, B: int, device="cuda", with_index: bool = True):
        self.B = B
        self.depth = torch.empty((B, desc.H, desc.W), dtype=torch.float16, device=device)
        self.proprio = torch.empty((B, desc.P), dtype=torch.float32, device=device)
        self.action = torch.empty((B, desc.A), dtype=torch.float32, device=device)
        self.logp_old = torch.empty(B, dtype=torch.float32, device=device)
        self.value_old = torch.empty(B, dtype=torch.float32, device=device)
        self.adv = torch.empty(B, dtype=torch.float32, device=device)
        self.ret = torch.empty(B, dtype=torch.float32, device=device)
        self.index = torch.empty(B, dtype=torch.int32, device=device) if with_index else None
        self.c = Minibatch(self.depth.data_ptr(), self.proprio.data_ptr(), self.action.data_ptr(),
                           self.logp_old.data_ptr(), self.value_old.data_ptr(), self.adv.data_ptr(),
                           self.ret.data_ptr(), self.index.data_ptr() if with_index else None, B)

    def bytes(self) -> int:
        ts = [self.depth, self.proprio, self.action, self.logp_old, self.value_old, self.adv, self.ret]
        return sum(t.numel() * t.element_size() for t in ts)


def ppo_shuffle_gather_minibatch(buf: Buffer, seed: int, epoch: int, mb_index: int, num_minibatches: int,
                                 out: MinibatchArrays, stream=None):
    _check(lib().ppo_shuffle_gather_minibatch(buf.handle, seed, epoch, mb_index, num_minibatches, C.byref(out.c),
                                              _stream(stream)), "ppo_shuffle_gather_minibatch")


def model_desc(H, W, conv_c: Sequence[int], conv_k: Sequence[int], fc: Sequence[int], P=32, A=12, norm=False,
               embed=0, n_lstm=0, lstm_h=0) -> ModelDesc:
    d = ModelDesc()
    d.H, d.W, d.n_conv, d.n_fc, d.P, d.A = H, W, len(conv_c), len(fc), P, A
    d.norm, d.embed, d.n_lstm, d.lstm_h = int(norm), int(embed), int(n_lstm), int(lstm_h)
    for i, v in enumerate(conv_c):
        d.conv_c[i] = v
    for i, v in enumerate(conv_k):
        d.conv_k[i] = v
    for i, v in enumerate(fc):
        d.fc[i] = v
    return d


class Model:
    """Handle of the policy/value network with its torch-owned parameter arena and workspace."""

    def __init__(self, desc: ModelDesc, microbatch: int, device="cuda"):
        self.desc = desc
        h = C.c_void_p()
        _check(lib().ppo_model_create(C.byref(desc), C.byref(h)), "ppo_model_create")
        self.handle = h
        self.microbatch = microbatch
        n = lib().ppo_model_arena_elems(h)
        self.arena = n
        self.master = torch.zeros(n, dtype=torch.float32, device=device)
        self.shadow = torch.zeros(n, dtype=torch.bfloat16, device=device)
        self.grad = torch.zeros(n, dtype=torch.float32, device=device)
        self.adam_m = torch.zeros(n, dtype=torch.float32, device=device)
        self.adam_v = torch.zeros(n, dtype=torch.float32, device=device)
        ws = lib().ppo_model_workspace_bytes(h, microbatch)
        self.workspace = torch.empty(ws, dtype=torch.uint8, device=device)
        _check(lib().ppo_model_bind(h, _ptr(self.master), _ptr(self.shadow), _ptr(self.grad), _ptr(self.adam_m),
                                    _ptr(self.adam_v), _ptr(self.workspace), ws, microbatch), "ppo_model_bind")

    def close(self):
        if self.handle:
            lib().ppo_model_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def param_count(self) -> int:
        return lib().ppo_model_param_count(self.handle)

    def tensors(self):
        out = []
        for i in range(lib().ppo_model_num_tensors(self.handle)):
            off, sz = C.c_int64(), C.c_int64()
            _check(lib().ppo_model_tensor_info(self.handle, i, C.byref(off), C.byref(sz)), "ppo_model_tensor_info")
            out.append((off.value, sz.value))
        return out

    def activation(self, kind: int, index: int) -> torch.Tensor:
        """A flat bf16 torch view of a saved activation inside the workspace (see ppo_model_activation_ptr)."""
        p, n = C.c_void_p(), C.c_size_t()
        _check(lib().ppo_model_activation_ptr(self.handle, kind, index, C.byref(p), C.byref(n)),
               "ppo_model_activation_ptr")
        off = p.value - self.workspace.data_ptr()
        if kind == 2:
            return self.workspace[off:off + 4 * n.value].view(torch.int32)
        if kind in (4, 6, 7):
            return self.workspace[off:off + 4 * n.value].view(torch.float32)
        return self.workspace[off:off + 2 * n.value].view(torch.bfloat16)

    def load(self, theta, stream=None):
        """Copies an fp32 parameter vector (numpy or torch, arena layout) into master and refreshes the shadow."""
        t = torch.as_tensor(theta, dtype=torch.float32)
        self.master.copy_(t.to(self.master.device))
        ppo_model_sync_shadow(self, stream)


def ppo_model_set_sequence(m: Model, T: int, Be: int, done, h_init, c_init):
    """done uint8 [T,Be], h_init / c_init fp32 [n_lstm,Be,lstm_h]: the tensors must stay alive until the backward pass."""
    _check(lib().ppo_model_set_sequence(m.handle, T, Be, _ptr(done), _ptr(h_init), _ptr(c_init)), "ppo_model_set_sequence")


def ppo_model_read_state(m: Model, h_out, c_out, stream=None):
    """fp32 [n_lstm,Be,lstm_h] each: the state after the last step of the latest forward, zero where that step was done."""
    _check(lib().ppo_model_read_state(m.handle, _ptr(h_out), _ptr(c_out), _stream(stream)), "ppo_model_read_state")


def ppo_state_reset(h, c, done, stream=None):
    """h, c fp32 [layers,n,H], done uint8 [n]: zeroes the state rows of the envs whose flag is set."""
    _check(lib().ppo_state_reset(_ptr(h), _ptr(c), _ptr(done), h.shape[0], h.shape[1], h.shape[2], _stream(stream)),
           "ppo_state_reset")


def ppo_shuffle_gather_sequences(buf: Buffer, seed: int, epoch: int, mb_index: int, num_minibatches: int,
                                 out: "MinibatchArrays", done_out, stream=None):
    _check(lib().ppo_shuffle_gather_sequences(buf.handle, seed, epoch, mb_index, num_minibatches, C.byref(out.c),
                                              _ptr(done_out), _stream(stream)), "ppo_shuffle_gather_sequences")


def ppo_model_sync_shadow(m: Model, stream=None):
    _check(lib().ppo_model_sync_shadow(m.handle, _stream(stream)), "ppo_model_sync_shadow")


def ppo_model_sync_masks(m: Model, rows: int, stream=None):
    _check(lib().ppo_model_sync_masks(m.handle, rows, _stream(stream)), "ppo_model_sync_masks")


def ppo_model_zero_grad(m: Model, stream=None):
    _check(lib().ppo_model_zero_grad(m.handle, _stream(stream)), "ppo_model_zero_grad")


def ppo_encoder_fwd(m: Model, mb: MinibatchArrays, row0: int, rows: int, mean, value, stream=None):
    _check(lib().ppo_encoder_fwd(m.handle, _mbref(mb), row0, rows, _ptr(mean), _ptr(value), _stream(stream)),
           "ppo_encoder_fwd")


def ppo_loss_fwd_bwd(m: Model, mb: MinibatchArrays, row0: int, rows: int, B_total: int, mean, value, clip: float,
                     vf_coef: float, ent_coef: float, loss_out, dmean, dvalue, stream=None):
    _check(lib().ppo_loss_fwd_bwd(m.handle, _mbref(mb), row0, rows, B_total, _ptr(mean), _ptr(value), clip,
                                  vf_coef, ent_coef, _ptr(loss_out), _ptr(dmean), _ptr(dvalue), _stream(stream)),
           "ppo_loss_fwd_bwd")


def ppo_encoder_bwd(m: Model, mb: MinibatchArrays, row0: int, rows: int, dmean, dvalue, accumulate: bool,
                    stream=None):
    _check(lib().ppo_encoder_bwd(m.handle, _mbref(mb), row0, rows, _ptr(dmean), _ptr(dvalue), int(accumulate),
                                 _stream(stream)), "ppo_encoder_bwd")


def ppo_adam_step(m: Model, lr: float, beta1: float, beta2: float, eps: float, step: int, stream=None):
    _check(lib().ppo_adam_step(m.handle, lr, beta1, beta2, eps, step, _stream(stream)), "ppo_adam_step")


def ppo_policy_step(m: Model, obs: Minibatch, rows: int, done, h, c, eps, mean, value, action, logp, stream=None):
    """One decision: forward pass, sampling and, for a recurrent model (else done, h, c are None), the state in place."""
    _check(lib().ppo_policy_step(m.handle, _mbref(obs), rows, _ptr(done), _ptr(h), _ptr(c), _ptr(eps), _ptr(mean), _ptr(value),
                                 _ptr(action), _ptr(logp), _stream(stream)), "ppo_policy_step")


def ppo_policy_act(m: Model, buf: Buffer, t: int, eps, stream=None):
    _check(lib().ppo_policy_act(m.handle, buf.handle, t, _ptr(eps), _stream(stream)), "ppo_policy_act")


def ppo_policy_sample(m: Model, rows: int, mean, eps, action, logp, stream=None):
    _check(lib().ppo_policy_sample(m.handle, rows, _ptr(mean), _ptr(eps), _ptr(action), _ptr(logp),
                                   _stream(stream)), "ppo_policy_sample")


# ------------------------------------------------------------------- operators for policies in tokens --

_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_ACTS = {"none": 0, "relu": 1, "silu": 2}


# Checks of tensors, in few steps each: a decision of a few envs takes the GPU less than 5 us.


def _dense(where: str, dev: int, t, dtype, shape):
    """The address of a dense tensor of that type and shape on device `dev` (-1: host), None of None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != dev:
        raise PpoError(1, where)
    if t.shape != shape or not t.is_contiguous():
        raise PpoError(2, where)
    return t.data_ptr()


def _operand(where: str, dev: int, t, dtype, shape, lead: int):
    """The address of a tensor, and the elements from one row to the next: its last dimensions make up a row, dense, and its first
    `lead` ones number the rows in order."""
    if t.dtype is not dtype or t.get_device() != dev:
        raise PpoError(1, where)
    if t.shape != shape:
        raise PpoError(2, where)
    row = 1
    for n in shape[lead:]:
        row *= n
    if t.is_contiguous():
        return t.data_ptr(), row
    stride, inner = t.stride(), 1
    for i in range(len(shape) - 1, lead - 1, -1):
        if shape[i] != 1 and stride[i] != inner:
            raise PpoError(2, where)
        inner *= shape[i]
    ld, count = None, 1
    for i in range(lead - 1, -1, -1):
        if shape[i] != 1:
            ld = stride[i] // count if ld is None else ld
            if stride[i] != ld * count:
                raise PpoError(2, where)
        count *= shape[i]
    return t.data_ptr(), row if ld is None else ld


def _device_of(where: str, t, types) -> int:
    """The device of the operands, which has to be the one the call runs on."""
    dev = t.get_device()
    if t.dtype not in types or (dev >= 0 and dev != torch._C._cuda_getDevice()):
        raise PpoError(1, where)
    return dev


def _stream_on(where: str, dev: int, stream):
    """The stream; looked up last, when everything else is known to fit: tensors of the host go no further."""
    if dev < 0:
        raise PpoError(1, where)
    return _stream(stream)


def _space(where: str, dev: int, t):
    """Address and bytes of a workspace."""
    if t is None:
        return None, 0
    if t.get_device() != dev or not t.is_contiguous():
        raise PpoError(1, where)
    return t.data_ptr(), t.numel() * t.element_size()


_F32, _U8, _I32 = torch.float32, torch.uint8, torch.int32


def ppo_decay_attention_workspace_bytes(q, k, v, backward: bool) -> int:
    """Bytes the calls with these q [T,Be,heads,dk], k [T,Be,kv_heads,dk], v [T,Be,kv_heads,dv] need (0: none)."""
    T, Be, heads, dk = q.shape
    kv, dv = v.shape[2:]
    d = DecayAttentionDesc(T, Be, heads, kv, dk, dv, _DTYPES[q.dtype], heads * dk, kv * dk, kv * dv, heads * dv, 1.0)
    return lib().ppo_decay_attention_workspace_bytes(C.byref(d), int(backward))


def _attention(where: str, q, k, v, o, scale: float, lead: int):
    """Descriptor, device, and the addresses of q, k, v, o."""
    dev, dtype = _device_of(where, q, _DTYPES), q.dtype
    shape = tuple(q.shape)
    if len(shape) != lead + 2 or k.dim() != lead + 2 or v.dim() != lead + 2:
        raise PpoError(2, where)
    rows, (heads, dk), kv, dv = shape[:lead], shape[lead:], k.shape[lead], v.shape[lead + 1]
    pq, ldq = _operand(where, dev, q, dtype, shape, lead)
    pk, ldk = _operand(where, dev, k, dtype, rows + (kv, dk), lead)
    pv, ldv = _operand(where, dev, v, dtype, rows + (kv, dv), lead)
    po, ldo = _operand(where, dev, o, dtype, rows + (heads, dv), lead)
    T, Be = rows if lead == 2 else (1, rows[0])
    return DecayAttentionDesc(T, Be, heads, kv, dk, dv, _DTYPES[dtype], ldq, ldk, ldv, ldo, scale), dev, pq, pk, pv, po


def ppo_decay_attention_fwd(q, k, v, decay, o, done=None, state_in=None, state_out=None, scale: float = 1.0, workspace=None, stream=None):
    """q [T,Be,heads,dk], k [T,Be,kv_heads,dk], v [T,Be,kv_heads,dv] -> o [T,Be,heads,dv] (fp32 or bf16; rows may be parts of wider
    ones); decay fp32 [heads]; done uint8 [T,Be]; states fp32 [Be,heads,dk,dv]."""
    f = "ppo_decay_attention_fwd"
    d, dev, pq, pk, pv, po = _attention(f, q, k, v, o, scale, 2)
    T, Be, heads, dk = q.shape
    state = (Be, heads, dk, v.shape[3])
    ws, n = _space(f, dev, workspace)
    _check(lib().ppo_decay_attention_fwd(C.byref(d), pq, pk, pv, _dense(f, dev, decay, _F32, (heads,)), _dense(f, dev, done, _U8, (T, Be)),
                                         _dense(f, dev, state_in, _F32, state), po, _dense(f, dev, state_out, _F32, state), ws, n, _stream_on(f, dev, stream)), f)


def ppo_decay_attention_bwd(q, k, v, decay, do, dq, dk, dv, done=None, state_in=None, dstate_out=None, dstate_in=None, scale: float = 1.0,
                            workspace=None, stream=None):
    """Gradients dq, dk, dv (shaped and strided as q, k, v) and dstate_in from do [T,Be,heads,dv] and dstate_out."""
    f = "ppo_decay_attention_bwd"
    d, dev, pq, pk, pv, po = _attention(f, q, k, v, do, scale, 2)
    out = []
    for t, like, ld in ((dq, q, d.ldq), (dk, k, d.ldk), (dv, v, d.ldv)):
        p, ldt = _operand(f, dev, t, q.dtype, tuple(like.shape), 2)
        if ldt != ld:
            raise PpoError(2, f)
        out.append(p)
    T, Be, heads, n = q.shape
    state = (Be, heads, n, v.shape[3])
    ws, n = _space(f, dev, workspace)
    _check(lib().ppo_decay_attention_bwd(C.byref(d), pq, pk, pv, _dense(f, dev, decay, _F32, (heads,)), _dense(f, dev, done, _U8, (T, Be)),
                                         _dense(f, dev, state_in, _F32, state), po, _dense(f, dev, dstate_out, _F32, state), *out,
                                         _dense(f, dev, dstate_in, _F32, state), ws, n, _stream_on(f, dev, stream)), f)


def ppo_decay_attention_step(q, k, v, decay, state, o, start=None, scale: float = 1.0, stream=None):
    """One decision: q [Be,heads,dk], k [Be,kv_heads,dk], v [Be,kv_heads,dv] -> o [Be,heads,dv], state fp32 [Be,heads,dk,dv] in place;
    start uint8 [Be]: envs that start from a zero state."""
    f = "ppo_decay_attention_step"
    d, dev, pq, pk, pv, po = _attention(f, q, k, v, o, scale, 1)
    Be, heads, dk = q.shape
    _check(lib().ppo_decay_attention_step(C.byref(d), pq, pk, pv, _dense(f, dev, decay, _F32, (heads,)), _dense(f, dev, start, _U8, (Be,)),
                                          _dense(f, dev, state, _F32, (Be, heads, dk, v.shape[2])), po, _stream_on(f, dev, stream)), f)


def ppo_group_norm_workspace_bytes(x, groups: int, backward: bool) -> int:
    """Bytes the calls with this x [B,HW,C] need (0: none)."""
    B, HW, n = x.shape
    d = GroupNormDesc(B, HW, n, groups, 0, _DTYPES[x.dtype], n, n)
    return lib().ppo_group_norm_workspace_bytes(C.byref(d), int(backward))


def _norm(where: str, x, groups: int, y, act: str):
    """Descriptor, device, and the addresses of x and y."""
    dev = _device_of(where, x, _DTYPES)
    if act not in _ACTS:
        raise PpoError(1, where)
    shape = tuple(x.shape)
    if len(shape) != 3:
        raise PpoError(2, where)
    px, ldx = _operand(where, dev, x, x.dtype, shape, 2)
    py, ldy = _operand(where, dev, y, x.dtype, shape, 2)
    return GroupNormDesc(*shape, groups, _ACTS[act], _DTYPES[x.dtype], ldx, ldy), dev, shape, px, py


def ppo_group_norm_fwd(x, groups: int, gamma, beta, y, mean, rstd, act: str = "none", eps: float = 1e-5, workspace=None, stream=None):
    """x, y [B,HW,C] (fp32, bf16 or fp16; pixels may be parts of wider rows); gamma, beta fp32 [C] or None; mean, rstd fp32
    [B,groups] are written; act: none, relu or silu."""
    f = "ppo_group_norm_fwd"
    d, dev, (B, _, n), px, py = _norm(f, x, groups, y, act)
    ws, size = _space(f, dev, workspace)
    _check(lib().ppo_group_norm_fwd(C.byref(d), eps, px, _dense(f, dev, gamma, _F32, (n,)), _dense(f, dev, beta, _F32, (n,)), py,
                                    _dense(f, dev, mean, _F32, (B, groups)), _dense(f, dev, rstd, _F32, (B, groups)), ws, size, _stream_on(f, dev, stream)), f)


def ppo_group_norm_bwd(x, groups: int, gamma, beta, mean, rstd, dy, dx, dgamma=None, dbeta=None, act: str = "none", accumulate: bool = False,
                       workspace=None, stream=None):
    """dx (strided as x) and, unless they are None, dgamma and dbeta fp32 [C] (added to where accumulate) from dy."""
    f = "ppo_group_norm_bwd"
    d, dev, shape, px, py = _norm(f, x, groups, dy, act)
    B, _, n = shape
    pd, ldd = _operand(f, dev, dx, x.dtype, shape, 2)
    if ldd != d.ldx:
        raise PpoError(2, f)
    ws, size = _space(f, dev, workspace)
    _check(lib().ppo_group_norm_bwd(C.byref(d), px, _dense(f, dev, gamma, _F32, (n,)), _dense(f, dev, beta, _F32, (n,)),
                                    _dense(f, dev, mean, _F32, (B, groups)), _dense(f, dev, rstd, _F32, (B, groups)), py, pd,
                                    _dense(f, dev, dgamma, _F32, (n,)), _dense(f, dev, dbeta, _F32, (n,)), int(accumulate), ws, size, _stream_on(f, dev, stream)), f)


def _token(where: str, logits, scale: float):
    """Descriptor, device, the shape of a row's scalar, and the address of the logits."""
    dev, shape = _device_of(where, logits, _DTYPES), tuple(logits.shape)
    if len(shape) != 2:
        raise PpoError(2, where)
    p, ld = _operand(where, dev, logits, logits.dtype, shape, 1)
    return TokenDesc(*shape, _DTYPES[logits.dtype], ld, scale), dev, shape[:1], p


def ppo_token_logp(logits, tokens, logp, entropy=None, scale: float = 1.0, stream=None):
    """logits [rows,vocab] (fp32, bf16 or fp16; rows may be parts of wider ones), tokens int32 [rows] -> logp, entropy fp32 [rows] of
    the distributions of scale * logits."""
    f = "ppo_token_logp"
    d, dev, row, p = _token(f, logits, scale)
    _check(lib().ppo_token_logp(C.byref(d), p, _dense(f, dev, tokens, _I32, row), _dense(f, dev, logp, _F32, row), _dense(f, dev, entropy, _F32, row),
                                _stream_on(f, dev, stream)), f)


def ppo_token_loss_workspace_bytes(logits) -> int:
    rows, vocab = logits.shape
    d = TokenDesc(rows, vocab, _DTYPES[logits.dtype], vocab, 1.0)
    return lib().ppo_token_loss_workspace_bytes(C.byref(d))


def ppo_token_loss_fwd_bwd(logits, tokens, logp_old, adv, B_total: int, dlogits, loss_out, logp_ref=None, weight=None, clip_low: float = 0.2,
                           clip_high: float = 0.2, kl_coef: float = 0.0, ent_coef: float = 0.0, scale: float = 1.0, grad_scale: float = 1.0,
                           logp_out=None, accumulate: bool = False, workspace=None, stream=None):
    """Clipped policy loss over logits [rows,vocab] with its gradient in dlogits (may be logits); logp_old, adv, logp_ref, weight,
    logp_out fp32 [rows]; loss_out fp32 [5] = L_pi, KL, H, mean(old - logp), clip fraction (added to where accumulate)."""
    f = "ppo_token_loss_fwd_bwd"
    d, dev, row, p = _token(f, logits, scale)
    pg, ldg = _operand(f, dev, dlogits, logits.dtype, tuple(logits.shape), 1)
    c = TokenLossCoef(clip_low, clip_high, kl_coef, ent_coef, grad_scale, B_total)
    ws, size = _space(f, dev, workspace)
    _check(lib().ppo_token_loss_fwd_bwd(C.byref(d), C.byref(c), p, _dense(f, dev, tokens, _I32, row), _dense(f, dev, logp_old, _F32, row),
                                        _dense(f, dev, logp_ref, _F32, row), _dense(f, dev, adv, _F32, row), _dense(f, dev, weight, _F32, row), pg, ldg,
                                        _dense(f, dev, logp_out, _F32, row), _dense(f, dev, loss_out, _F32, (5,)), int(accumulate), ws, size,
                                        _stream_on(f, dev, stream)), f)


def ppo_causal_conv_workspace_bytes(x, width: int) -> int:
    """Bytes the gradients of this x [T,Be,C] need (0: none)."""
    T, Be, n = x.shape
    d = CausalConvDesc(T, Be, n, width, 0, _DTYPES[x.dtype], n, n)
    return lib().ppo_causal_conv_workspace_bytes(C.byref(d))


def _conv(where: str, x, weight, y, act: str, lead: int):
    """Descriptor, device, and the addresses of x, weight, y."""
    dev, shape = _device_of(where, x, _DTYPES), tuple(x.shape)
    if act not in _ACTS:
        raise PpoError(1, where)
    if len(shape) != lead + 1 or weight.dim() != 2:
        raise PpoError(2, where)
    px, ldx = _operand(where, dev, x, x.dtype, shape, lead)
    py, ldy = _operand(where, dev, y, x.dtype, shape, lead)
    T, Be = shape[:2] if lead == 2 else (1, shape[0])
    n, width = shape[lead], weight.shape[1]
    return CausalConvDesc(T, Be, n, width, _ACTS[act], _DTYPES[x.dtype], ldx, ldy), dev, px, _dense(where, dev, weight, _F32, (n, width)), py


def ppo_causal_conv_fwd(x, weight, bias, y, done=None, state_in=None, state_out=None, act: str = "none", stream=None):
    """x, y [T,Be,C] (fp32, bf16 or fp16; rows may be parts of wider ones), weight fp32 [C,width], bias fp32 [C] or None; done uint8 [T,Be];
    states [Be,width-1,C] of the type of x; act: none, relu or silu."""
    f = "ppo_causal_conv_fwd"
    d, dev, px, pw, py = _conv(f, x, weight, y, act, 2)
    state = (d.Be, d.width - 1, d.C)
    _check(lib().ppo_causal_conv_fwd(C.byref(d), px, pw, _dense(f, dev, bias, _F32, (d.C,)), _dense(f, dev, done, _U8, (d.T, d.Be)),
                                     _dense(f, dev, state_in, x.dtype, state), py, _dense(f, dev, state_out, x.dtype, state), _stream_on(f, dev, stream)), f)


def ppo_causal_conv_bwd(x, weight, bias, dy, dx, dweight=None, dbias=None, done=None, state_in=None, dstate_out=None, dstate_in=None, act: str = "none",
                        accumulate: bool = False, workspace=None, stream=None):
    """dx (strided as x) and dstate_in from dy and dstate_out; dweight fp32 [C,width], dbias fp32 [C] (added to where accumulate)."""
    f = "ppo_causal_conv_bwd"
    d, dev, px, pw, py = _conv(f, x, weight, dy, act, 2)
    pd, ldd = _operand(f, dev, dx, x.dtype, tuple(x.shape), 2)
    if ldd != d.ldx:
        raise PpoError(2, f)
    state = (d.Be, d.width - 1, d.C)
    ws, size = _space(f, dev, workspace)
    _check(lib().ppo_causal_conv_bwd(C.byref(d), px, pw, _dense(f, dev, bias, _F32, (d.C,)), _dense(f, dev, done, _U8, (d.T, d.Be)),
                                     _dense(f, dev, state_in, x.dtype, state), py, _dense(f, dev, dstate_out, x.dtype, state), pd,
                                     _dense(f, dev, dstate_in, x.dtype, state), _dense(f, dev, dweight, _F32, (d.C, d.width)),
                                     _dense(f, dev, dbias, _F32, (d.C,)), int(accumulate), ws, size, _stream_on(f, dev, stream)), f)


def ppo_causal_conv_step(x, weight, bias, state, y, start=None, act: str = "none", stream=None):
    """One decision: x, y [Be,C], state [Be,width-1,C] in place; start uint8 [Be]: envs that start from a zero state."""
    f = "ppo_causal_conv_step"
    d, dev, px, pw, py = _conv(f, x, weight, y, act, 1)
    _check(lib().ppo_causal_conv_step(C.byref(d), px, pw, _dense(f, dev, bias, _F32, (d.C,)), _dense(f, dev, start, _U8, (d.Be,)),
                                      _dense(f, dev, state, x.dtype, (d.Be, d.width - 1, d.C)), py, _stream_on(f, dev, stream)), f)


def ppo_selective_scan_workspace_bytes(x, B, backward: bool) -> int:
    """Bytes the calls with these x [T,Be,C], B [T,Be,groups,N] need (0: none)."""
    (T, Be, n), (groups, N) = x.shape, B.shape[2:]
    d = SelectiveScanDesc(T, Be, n, N, groups, _DTYPES[x.dtype], 0, n, n, groups * N, groups * N, n, n)
    return lib().ppo_selective_scan_workspace_bytes(C.byref(d), int(backward))


def _scan(where: str, x, dt, A, B, Cm, D, z, dt_bias, y, softplus: bool, lead: int):
    """Descriptor, device, and the addresses of x, dt, A, B, C, D, z, dt_bias; and that of y."""
    dev, dtype, shape = _device_of(where, x, _DTYPES), x.dtype, tuple(x.shape)
    if len(shape) != lead + 1 or B.dim() != lead + 2:
        raise PpoError(2, where)
    n, few = shape[lead], shape[:lead] + tuple(B.shape[lead:])
    px, ldx = _operand(where, dev, x, dtype, shape, lead)
    pt, ldt = _operand(where, dev, dt, dtype, shape, lead)
    pb, ldb = _operand(where, dev, B, dtype, few, lead)
    pc, ldc = _operand(where, dev, Cm, dtype, few, lead)
    pz, ldz = (None, n) if z is None else _operand(where, dev, z, dtype, shape, lead)
    py, ldy = _operand(where, dev, y, dtype, shape, lead)
    T, Be = shape[:2] if lead == 2 else (1, shape[0])
    groups, N = few[lead:]
    d = SelectiveScanDesc(T, Be, n, N, groups, _DTYPES[dtype], int(softplus), ldx, ldt, ldb, ldc, ldz, ldy)
    return d, dev, (px, pt, _dense(where, dev, A, _F32, (n, N)), pb, pc, _dense(where, dev, D, _F32, (n,)), pz, _dense(where, dev, dt_bias, _F32, (n,))), py


def ppo_selective_scan_fwd(x, dt, A, B, C_, y, D=None, z=None, dt_bias=None, softplus: bool = True, done=None, state_in=None, state_out=None,
                           workspace=None, stream=None):
    """x, dt, z, y [T,Be,channels], B, C_ [T,Be,groups,N] (fp32, bf16 or fp16; rows may be parts of wider ones); A fp32 [channels,N]; D, dt_bias
    fp32 [channels]; done uint8 [T,Be]; states fp32 [Be,channels,N]."""
    f = "ppo_selective_scan_fwd"
    d, dev, ins, py = _scan(f, x, dt, A, B, C_, D, z, dt_bias, y, softplus, 2)
    state = (d.Be, d.channels, d.N)
    ws, size = _space(f, dev, workspace)
    _check(lib().ppo_selective_scan_fwd(C.byref(d), *ins, _dense(f, dev, done, _U8, (d.T, d.Be)), _dense(f, dev, state_in, _F32, state), py,
                                        _dense(f, dev, state_out, _F32, state), ws, size, _stream_on(f, dev, stream)), f)


def ppo_selective_scan_bwd(x, dt, A, B, C_, dy, dx, ddt, dA, dB, dC, D=None, z=None, dt_bias=None, softplus: bool = True, done=None, state_in=None,
                           dstate_out=None, dD=None, dz=None, ddt_bias=None, dstate_in=None, accumulate: bool = False, workspace=None, stream=None):
    """dx, ddt, dB, dC, dz (strided as x, dt, B, C_, z) and dstate_in from dy and dstate_out; dA, dD, ddt_bias fp32 (None: not wanted; added
    to where accumulate)."""
    f = "ppo_selective_scan_bwd"
    d, dev, ins, py = _scan(f, x, dt, A, B, C_, D, z, dt_bias, dy, softplus, 2)
    if (z is None) != (dz is None):
        raise PpoError(1, f)
    out = []
    for t, like, ld in ((dx, x, d.ldx), (ddt, dt, d.lddt), (dB, B, d.ldb), (dC, C_, d.ldc), (dz, z, d.ldz)):
        if t is None and like is None:
            out.append(None)
            continue
        p, ldt = _operand(f, dev, t, x.dtype, tuple(like.shape), 2)
        if ldt != ld:
            raise PpoError(2, f)
        out.append(p)
    state, n = (d.Be, d.channels, d.N), (d.channels,)
    ws, size = _space(f, dev, workspace)
    _check(lib().ppo_selective_scan_bwd(C.byref(d), *ins, _dense(f, dev, done, _U8, (d.T, d.Be)), _dense(f, dev, state_in, _F32, state), py,
                                        _dense(f, dev, dstate_out, _F32, state), out[0], out[1], _dense(f, dev, dA, _F32, n + (d.N,)), out[2], out[3],
                                        _dense(f, dev, dD, _F32, n), out[4], _dense(f, dev, ddt_bias, _F32, n), _dense(f, dev, dstate_in, _F32, state),
                                        int(accumulate), ws, size, _stream_on(f, dev, stream)), f)


def ppo_selective_scan_step(x, dt, A, B, C_, state, y, D=None, z=None, dt_bias=None, softplus: bool = True, start=None, stream=None):
    """One decision: x, dt, z, y [Be,channels], B, C_ [Be,groups,N], state fp32 [Be,channels,N] in place; start uint8 [Be]: envs that start
    from a zero state."""
    f = "ppo_selective_scan_step"
    d, dev, ins, py = _scan(f, x, dt, A, B, C_, D, z, dt_bias, y, softplus, 1)
    _check(lib().ppo_selective_scan_step(C.byref(d), *ins, _dense(f, dev, start, _U8, (d.Be,)), _dense(f, dev, state, _F32, (d.Be, d.channels, d.N)), py,
                                         _stream_on(f, dev, stream)), f)


def ppo_qk_norm_rotate_workspace_bytes(q, k) -> int:
    """Bytes the gradients of gamma need with these q [rows,heads,d], k [rows,kv_heads,d]."""
    (rows, heads, n), kv = q.shape, k.shape[1]
    d = QkNormDesc(rows, heads, kv, n, 0, 0, _DTYPES[q.dtype], heads * n, kv * n, heads * n, kv * n)
    return lib().ppo_qk_norm_rotate_workspace_bytes(C.byref(d))


def _qk(where: str, q, k, gamma_q, gamma_k, pos, freq, q_out, k_out, interleaved: bool):
    """Descriptor, device, the addresses of q, k, gamma_q, gamma_k, pos, freq, and those of q_out, k_out."""
    dev, shape = _device_of(where, q, _DTYPES), tuple(q.shape)
    if len(shape) != 3 or k.dim() != 3:
        raise PpoError(2, where)
    (rows, heads, n), kv = shape, k.shape[1]
    few = (rows, kv, n)
    pq, ldq = _operand(where, dev, q, q.dtype, shape, 1)
    pk, ldk = _operand(where, dev, k, q.dtype, few, 1)
    po, ldqo = _operand(where, dev, q_out, q.dtype, shape, 1)
    pp, ldko = _operand(where, dev, k_out, q.dtype, few, 1)
    pairs = 0 if freq is None else freq.numel()
    d = QkNormDesc(rows, heads, kv, n, pairs, int(interleaved), _DTYPES[q.dtype], ldq, ldk, ldqo, ldko)
    ins = (pq, pk, _dense(where, dev, gamma_q, _F32, (n,)), _dense(where, dev, gamma_k, _F32, (n,)), _dense(where, dev, pos, _I32, (rows,)),
           _dense(where, dev, freq, torch.float64, (pairs,)))
    return d, dev, ins, (po, pp)


def ppo_qk_norm_rotate_fwd(q, k, gamma_q, gamma_k, pos, freq, q_out, k_out, eps: float = 1e-6, interleaved: bool = False, stream=None):
    """q, q_out [rows,heads,d], k, k_out [rows,kv_heads,d] (fp32, bf16 or fp16; rows may be parts of wider ones; an output may be its input); gamma
    fp32 [d] or None; pos int32 [rows]; freq fp64 [pairs], radians a position (None: no rotation)."""
    f = "ppo_qk_norm_rotate_fwd"
    d, dev, ins, outs = _qk(f, q, k, gamma_q, gamma_k, pos, freq, q_out, k_out, interleaved)
    _check(lib().ppo_qk_norm_rotate_fwd(C.byref(d), eps, *ins, *outs, _stream_on(f, dev, stream)), f)


def ppo_qk_norm_rotate_bwd(q, k, gamma_q, gamma_k, pos, freq, dq_out, dk_out, dq, dk, dgamma_q=None, dgamma_k=None, eps: float = 1e-6,
                           interleaved: bool = False, accumulate: bool = False, workspace=None, stream=None):
    """dq, dk (strided as q, k) from dq_out, dk_out; dgamma_q, dgamma_k fp32 [d] (None: not wanted; added to where accumulate)."""
    f = "ppo_qk_norm_rotate_bwd"
    d, dev, ins, outs = _qk(f, q, k, gamma_q, gamma_k, pos, freq, dq_out, dk_out, interleaved)
    pq, ldq = _operand(f, dev, dq, q.dtype, tuple(q.shape), 1)
    pk, ldk = _operand(f, dev, dk, q.dtype, tuple(k.shape), 1)
    if ldq != d.ldq or ldk != d.ldk:
        raise PpoError(2, f)
    ws, size = _space(f, dev, workspace)
    _check(lib().ppo_qk_norm_rotate_bwd(C.byref(d), eps, *ins, *outs, pq, pk, _dense(f, dev, dgamma_q, _F32, (d.d,)), _dense(f, dev, dgamma_k, _F32, (d.d,)),
                                        int(accumulate), ws, size, _stream_on(f, dev, stream)), f)

"""Thin ctypes binding of the C ABI in include/tli.h.

Argument marshalling only: every step of the verification runs in the CUDA
library.  torch is used for device memory and streams.  There is no CPU
fallback: if ``libtli.so`` is missing or cannot be loaded, importing a function
from here raises.
"""
from __future__ import annotations

import ctypes
import os
import struct
import threading
import warnings
from typing import Dict, Optional

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtli.so")

TLI_F32 = 0
TLI_BF16 = 1
TLI_OK = 0
TLI_ERR_ARG = -1
TLI_ERR_BAD_MAP = -2
TLI_ERR_CUDA = -3
TLI_ERR_WORKSPACE = -4
TLI_ERR_UNSUPPORTED = -5
TLI_ERR_STATIC_SCRATCH = -6
TLI_ROW_DRAFT_RANGE = 1
TLI_ROW_DRAFT_UNMAPPED = 2
TLI_ROW_NONFINITE = 4
TLI_ROW_FALLBACK = 8
TLI_ROW_TIMEOUT = 16
TLI_ROW_BAD_TEMPERATURE = 32
TLI_ROW_BAD_FILTER = 64
TLI_ROW_LEFT_OUT = 128
TLI_SIDE_TARGET = 0
TLI_SIDE_DRAFTER = 1
TLI_SUPPORT_ALL = 0
TLI_SUPPORT_SHARED = 1
TLI_MAX_B = 65535
TLI_MAX_K = 64
TLI_MAX_V = 1048576
TLI_MAX_SHARDS = 64
TLI_MAX_TOKENS = 4194304
TLI_MAX_H = 65536
TLI_MAX_TARGETS = 256
TLI_MAX_HEAD_TOKENS = 262144
TLI_STATIC_SCRATCH_BYTES = 4194304

EXPORTS = ("tli_create", "tli_destroy", "tli_workspace_bytes", "tli_verify", "tli_verify_static", "tli_verify_profile", "tli_set_tiled", "tli_set_max_cluster", "tli_reset", "tli_selftest_bounded_wait",
           "tli_draft_workspace_bytes", "tli_draft_sample", "tli_slem_workspace_bytes", "tli_slem_verify",
           "tli_verify_host_buffer_bytes", "tli_verify_host", "tli_rates_workspace_bytes", "tli_acceptance_rates",
           "tli_sample_workspace_bytes", "tli_sample", "tli_filter_workspace_bytes", "tli_filter",
           "tli_embed", "tli_embed_grad_workspace_bytes", "tli_embed_grad",
           "tli_loss", "tli_loss_grad",
           "tli_head_loss_workspace_bytes", "tli_head_loss", "tli_head_loss_grad_workspace_bytes", "tli_head_loss_grad",
           "tli_ctx_info",
           "tli_shard_create", "tli_shard_info", "tli_shard_workspace_bytes", "tli_shard_record_bytes", "tli_shard_rows_bytes",
           "tli_shard_stats", "tli_shard_decide", "tli_shard_weights", "tli_shard_select",
           "tli_verify_plan", "tli_launch_probe",
           "tli_status_string", "tli_last_cuda_error")


class tli_verify_args(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("K", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("target_logits", ctypes.c_void_p), ("t_stride_b", ctypes.c_int64), ("t_stride_k", ctypes.c_int64),
        ("drafter_logits", ctypes.c_void_p), ("d_stride_b", ctypes.c_int64), ("d_stride_k", ctypes.c_int64),
        ("draft_ids", ctypes.c_void_p), ("temperature", ctypes.c_void_p), ("uniforms", ctypes.c_void_p),
        ("accepted", ctypes.c_void_p), ("next_token", ctypes.c_void_p), ("row_status", ctypes.c_void_p),
        ("p_draft", ctypes.c_void_p), ("q_draft", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
        ("draft_lengths", ctypes.c_void_p),
    ]


class tli_verify_host_args(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("K", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("target_logits", ctypes.c_void_p), ("drafter_logits", ctypes.c_void_p), ("draft_ids", ctypes.c_void_p),
        ("temperature", ctypes.c_void_p), ("uniforms", ctypes.c_void_p),
        ("accepted", ctypes.c_void_p), ("next_token", ctypes.c_void_p), ("row_status", ctypes.c_void_p),
        ("device_buffer", ctypes.c_void_p), ("device_buffer_bytes", ctypes.c_size_t),
    ]


class tli_rates_args(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("K", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("target_logits", ctypes.c_void_p), ("t_stride_b", ctypes.c_int64), ("t_stride_k", ctypes.c_int64),
        ("drafter_logits", ctypes.c_void_p), ("d_stride_b", ctypes.c_int64), ("d_stride_k", ctypes.c_int64),
        ("temperature", ctypes.c_void_p),
        ("mass", ctypes.c_void_p), ("alpha_union", ctypes.c_void_p), ("alpha_tli", ctypes.c_void_p),
        ("position_status", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
    ]


class tli_draft_args(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("R", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("drafter_logits", ctypes.c_void_p), ("d_stride_b", ctypes.c_int64), ("d_stride_r", ctypes.c_int64),
        ("temperature", ctypes.c_void_p), ("uniforms", ctypes.c_void_p),
        ("draft_ids", ctypes.c_void_p), ("q_draft", ctypes.c_void_p), ("draft_status", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
    ]


class tli_slem_args(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("M", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("target_logits", ctypes.c_void_p), ("t_stride_b", ctypes.c_int64), ("t_stride_k", ctypes.c_int64),
        ("candidates", ctypes.c_void_p), ("lengths", ctypes.c_void_p),
        ("temperature", ctypes.c_void_p), ("uniforms", ctypes.c_void_p),
        ("accepted", ctypes.c_void_p), ("next_token", ctypes.c_void_p), ("sampled", ctypes.c_void_p),
        ("row_status", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
    ]


class tli_sample_args(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("R", ctypes.c_int32), ("dtype", ctypes.c_int32), ("side", ctypes.c_int32),
        ("logits", ctypes.c_void_p), ("stride_b", ctypes.c_int64), ("stride_r", ctypes.c_int64),
        ("temperature", ctypes.c_void_p), ("top_k", ctypes.c_void_p), ("top_p", ctypes.c_void_p),
        ("min_p", ctypes.c_void_p), ("uniforms", ctypes.c_void_p),
        ("tokens", ctypes.c_void_p), ("prob", ctypes.c_void_p), ("status", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
    ]


class tli_filter_args(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("R", ctypes.c_int32), ("dtype", ctypes.c_int32), ("side", ctypes.c_int32),
        ("logits", ctypes.c_void_p), ("stride_b", ctypes.c_int64), ("stride_r", ctypes.c_int64),
        ("temperature", ctypes.c_void_p), ("top_k", ctypes.c_void_p), ("top_p", ctypes.c_void_p),
        ("min_p", ctypes.c_void_p),
        ("out", ctypes.c_void_p), ("out_stride_b", ctypes.c_int64), ("out_stride_r", ctypes.c_int64),
        ("status", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
    ]


class tli_embed_args(ctypes.Structure):
    _fields_ = [
        ("N", ctypes.c_int32), ("H", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("ids_side", ctypes.c_int32), ("table_side", ctypes.c_int32),
        ("ids", ctypes.c_void_p), ("table", ctypes.c_void_p), ("table_stride", ctypes.c_int64),
        ("scale", ctypes.c_float),
        ("out", ctypes.c_void_p), ("out_stride", ctypes.c_int64), ("table_ids", ctypes.c_void_p),
    ]


class tli_embed_grad_args(ctypes.Structure):
    _fields_ = [
        ("N", ctypes.c_int32), ("H", ctypes.c_int32), ("grad_dtype", ctypes.c_int32), ("out_dtype", ctypes.c_int32),
        ("ids_side", ctypes.c_int32), ("table_side", ctypes.c_int32),
        ("ids", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("grad_stride", ctypes.c_int64),
        ("scale", ctypes.c_float),
        ("out", ctypes.c_void_p), ("out_stride", ctypes.c_int64),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
    ]


class tli_loss_args(ctypes.Structure):
    _fields_ = [
        ("N", ctypes.c_int32), ("k", ctypes.c_int32), ("dtype", ctypes.c_int32), ("side", ctypes.c_int32),
        ("ids_side", ctypes.c_int32), ("support", ctypes.c_int32), ("teacher_dtype", ctypes.c_int32),
        ("logits", ctypes.c_void_p), ("stride", ctypes.c_int64), ("ids", ctypes.c_void_p), ("teacher", ctypes.c_void_p),
        ("temperature", ctypes.c_void_p), ("loss", ctypes.c_void_p), ("stats", ctypes.c_void_p), ("status", ctypes.c_void_p),
    ]


class tli_loss_grad_args(ctypes.Structure):
    _fields_ = [
        ("N", ctypes.c_int32), ("k", ctypes.c_int32), ("dtype", ctypes.c_int32), ("side", ctypes.c_int32),
        ("ids_side", ctypes.c_int32), ("support", ctypes.c_int32), ("teacher_dtype", ctypes.c_int32),
        ("logits", ctypes.c_void_p), ("stride", ctypes.c_int64), ("ids", ctypes.c_void_p), ("teacher", ctypes.c_void_p),
        ("temperature", ctypes.c_void_p), ("stats", ctypes.c_void_p), ("grad_loss", ctypes.c_void_p),
        ("grad", ctypes.c_void_p), ("grad_stride", ctypes.c_int64),
    ]


class tli_head_loss_args(ctypes.Structure):
    _fields_ = [
        ("N", ctypes.c_int32), ("H", ctypes.c_int32), ("k", ctypes.c_int32), ("side", ctypes.c_int32),
        ("ids_side", ctypes.c_int32), ("support", ctypes.c_int32), ("teacher_dtype", ctypes.c_int32),
        ("hidden", ctypes.c_void_p), ("hidden_stride", ctypes.c_int64), ("weight", ctypes.c_void_p), ("weight_stride", ctypes.c_int64),
        ("ids", ctypes.c_void_p), ("teacher", ctypes.c_void_p), ("temperature", ctypes.c_void_p),
        ("loss", ctypes.c_void_p), ("stats", ctypes.c_void_p), ("target_logits", ctypes.c_void_p), ("status", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
    ]


class tli_head_loss_grad_args(ctypes.Structure):
    _fields_ = [
        ("N", ctypes.c_int32), ("H", ctypes.c_int32), ("k", ctypes.c_int32), ("side", ctypes.c_int32),
        ("ids_side", ctypes.c_int32), ("support", ctypes.c_int32), ("teacher_dtype", ctypes.c_int32),
        ("hidden", ctypes.c_void_p), ("hidden_stride", ctypes.c_int64), ("weight", ctypes.c_void_p), ("weight_stride", ctypes.c_int64),
        ("ids", ctypes.c_void_p), ("teacher", ctypes.c_void_p), ("temperature", ctypes.c_void_p),
        ("stats", ctypes.c_void_p), ("target_logits", ctypes.c_void_p), ("grad_loss", ctypes.c_void_p),
        ("grad_hidden", ctypes.c_void_p), ("grad_hidden_stride", ctypes.c_int64),
        ("grad_weight", ctypes.c_void_p), ("grad_weight_stride", ctypes.c_int64), ("status", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
    ]


class TLIError(RuntimeError):
    def __init__(self, code: int, where: str):
        lib = load()
        msg = lib.tli_status_string(code).decode()
        detail = lib.tli_last_cuda_error().decode() if code == TLI_ERR_CUDA else ""
        super().__init__("%s failed: %s (%d)%s" % (where, msg, code, (": " + detail) if detail else ""))
        self.code = code


_lib = None


def load() -> ctypes.CDLL:
    """Load libtli.so (built by ``python -m paper_2502_05202_b200.build``); raises if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("CUDA library %s is missing; run `python -m paper_2502_05202_b200.build`" % LIB_PATH)
        lib = ctypes.CDLL(LIB_PATH)
        lib.tli_create.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.c_int, ctypes.c_int32, ctypes.c_int32,
                                   ctypes.c_void_p]
        lib.tli_create.restype = ctypes.c_int
        lib.tli_destroy.argtypes = [ctypes.c_void_p]
        lib.tli_destroy.restype = ctypes.c_int
        lib.tli_workspace_bytes.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]
        lib.tli_workspace_bytes.restype = ctypes.c_size_t
        lib.tli_verify.argtypes = [ctypes.c_void_p, ctypes.POINTER(tli_verify_args), ctypes.c_void_p]
        lib.tli_verify.restype = ctypes.c_int
        lib.tli_verify_static.argtypes = [ctypes.c_void_p, ctypes.POINTER(tli_verify_args), ctypes.c_void_p]
        lib.tli_verify_static.restype = ctypes.c_int
        lib.tli_verify_profile.argtypes = [ctypes.c_void_p, ctypes.POINTER(tli_verify_args), ctypes.c_void_p,
                                           ctypes.POINTER(ctypes.c_float)]
        lib.tli_verify_profile.restype = ctypes.c_int
        lib.tli_draft_workspace_bytes.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]
        lib.tli_draft_workspace_bytes.restype = ctypes.c_size_t
        lib.tli_draft_sample.argtypes = [ctypes.c_void_p, ctypes.POINTER(tli_draft_args), ctypes.c_void_p]
        lib.tli_draft_sample.restype = ctypes.c_int
        lib.tli_slem_workspace_bytes.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]
        lib.tli_slem_workspace_bytes.restype = ctypes.c_size_t
        lib.tli_slem_verify.argtypes = [ctypes.c_void_p, ctypes.POINTER(tli_slem_args), ctypes.c_void_p]
        lib.tli_slem_verify.restype = ctypes.c_int
        lib.tli_verify_host_buffer_bytes.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]
        lib.tli_verify_host_buffer_bytes.restype = ctypes.c_size_t
        lib.tli_verify_host.argtypes = [ctypes.c_void_p, ctypes.POINTER(tli_verify_host_args), ctypes.c_void_p]
        lib.tli_verify_host.restype = ctypes.c_int
        lib.tli_rates_workspace_bytes.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]
        lib.tli_rates_workspace_bytes.restype = ctypes.c_size_t
        lib.tli_acceptance_rates.argtypes = [ctypes.c_void_p, ctypes.POINTER(tli_rates_args), ctypes.c_void_p]
        lib.tli_acceptance_rates.restype = ctypes.c_int
        for name, args in (("tli_sample", tli_sample_args), ("tli_filter", tli_filter_args), ("tli_embed", tli_embed_args),
                           ("tli_embed_grad", tli_embed_grad_args), ("tli_loss", tli_loss_args), ("tli_loss_grad", tli_loss_grad_args),
                           ("tli_head_loss", tli_head_loss_args), ("tli_head_loss_grad", tli_head_loss_grad_args)):
            getattr(lib, name).argtypes = [ctypes.c_void_p, ctypes.POINTER(args), ctypes.c_void_p]
            getattr(lib, name).restype = ctypes.c_int
        for name in ("tli_sample_workspace_bytes", "tli_filter_workspace_bytes"):
            getattr(lib, name).argtypes = [ctypes.c_void_p] + [ctypes.c_int32] * 4
            getattr(lib, name).restype = ctypes.c_size_t
        for name in ("tli_head_loss_workspace_bytes", "tli_head_loss_grad_workspace_bytes"):
            getattr(lib, name).argtypes = [ctypes.c_void_p] + [ctypes.c_int32] * 4
            getattr(lib, name).restype = ctypes.c_size_t
        lib.tli_embed_grad_workspace_bytes.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32]
        lib.tli_embed_grad_workspace_bytes.restype = ctypes.c_size_t
        lib.tli_shard_create.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.c_int, ctypes.c_int32, ctypes.c_int32,
                                         ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32]
        lib.tli_shard_create.restype = ctypes.c_int
        lib.tli_shard_info.argtypes = [ctypes.c_void_p] + [ctypes.POINTER(ctypes.c_int32)] * 6
        lib.tli_shard_info.restype = ctypes.c_int
        lib.tli_shard_workspace_bytes.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]
        lib.tli_shard_workspace_bytes.restype = ctypes.c_size_t
        lib.tli_shard_record_bytes.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32]
        lib.tli_shard_record_bytes.restype = ctypes.c_size_t
        lib.tli_shard_rows_bytes.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32]
        lib.tli_shard_rows_bytes.restype = ctypes.c_size_t
        lib.tli_shard_stats.argtypes = [ctypes.c_void_p, ctypes.POINTER(tli_verify_args), ctypes.c_void_p, ctypes.c_void_p]
        lib.tli_shard_stats.restype = ctypes.c_int
        lib.tli_shard_decide.argtypes = [ctypes.c_void_p, ctypes.POINTER(tli_verify_args), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
        lib.tli_shard_decide.restype = ctypes.c_int
        lib.tli_shard_weights.argtypes = [ctypes.c_void_p, ctypes.POINTER(tli_verify_args), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
        lib.tli_shard_weights.restype = ctypes.c_int
        lib.tli_shard_select.argtypes = [ctypes.c_void_p, ctypes.POINTER(tli_verify_args), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
        lib.tli_shard_select.restype = ctypes.c_int
        lib.tli_verify_plan.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(ctypes.c_int32)]
        lib.tli_verify_plan.restype = ctypes.c_int
        lib.tli_launch_probe.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p]
        lib.tli_launch_probe.restype = ctypes.c_int
        lib.tli_reset.argtypes = [ctypes.c_void_p, ctypes.c_void_p]
        lib.tli_reset.restype = ctypes.c_int
        lib.tli_set_tiled.argtypes = [ctypes.c_void_p, ctypes.c_int]
        lib.tli_set_tiled.restype = ctypes.c_int
        lib.tli_set_max_cluster.argtypes = [ctypes.c_void_p, ctypes.c_int]
        lib.tli_set_max_cluster.restype = ctypes.c_int
        lib.tli_selftest_bounded_wait.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_uint, ctypes.POINTER(ctypes.c_int)]
        lib.tli_selftest_bounded_wait.restype = ctypes.c_int
        lib.tli_ctx_info.argtypes = [ctypes.c_void_p] + [ctypes.POINTER(ctypes.c_int32)] * 3
        lib.tli_ctx_info.restype = ctypes.c_int
        lib.tli_status_string.argtypes = [ctypes.c_int]
        lib.tli_status_string.restype = ctypes.c_char_p
        lib.tli_last_cuda_error.argtypes = []
        lib.tli_last_cuda_error.restype = ctypes.c_char_p
        _lib = lib
    return _lib


def tli_create(device: int, V_t: int, V_d: int, id_map) -> int:
    """tli_create(): returns the context handle; ``id_map`` is a host int32 array [V_d]."""
    m = np.ascontiguousarray(id_map, dtype=np.int32)
    if m.shape != (V_d,):
        raise ValueError("id_map must have V_d entries")
    h = ctypes.c_void_p()
    rc = load().tli_create(ctypes.byref(h), int(device), int(V_t), int(V_d), m.ctypes.data)
    if rc != TLI_OK:
        raise TLIError(rc, "tli_create")
    return h.value


def tli_destroy(ctx: int) -> None:
    rc = load().tli_destroy(ctx)
    if rc != TLI_OK:
        raise TLIError(rc, "tli_destroy")


def tli_workspace_bytes(ctx: int, B: int, K: int, dtype: int) -> int:
    return int(load().tli_workspace_bytes(ctx, B, K, dtype))


def _logit_dtype(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return TLI_F32
    if t.dtype == torch.bfloat16:
        return TLI_BF16
    raise TypeError("logits must be float32 or bfloat16")


def make_args(target_logits: torch.Tensor, drafter_logits: torch.Tensor, draft_ids: torch.Tensor,
              temperature: torch.Tensor, uniforms: torch.Tensor, accepted: torch.Tensor,
              next_token: torch.Tensor, workspace: torch.Tensor, row_status: Optional[torch.Tensor] = None,
              p_draft: Optional[torch.Tensor] = None, q_draft: Optional[torch.Tensor] = None,
              draft_lengths: Optional[torch.Tensor] = None) -> tli_verify_args:
    """Fill a tli_verify_args from device tensors (no copies; the tensors must outlive the call)."""
    B, K1, _ = target_logits.shape
    K = K1 - 1
    dt = _logit_dtype(target_logits)
    if _logit_dtype(drafter_logits) != dt:
        raise TypeError("both logit tensors must have the same dtype")
    if target_logits.stride(2) != 1 or drafter_logits.stride(2) != 1:
        raise ValueError("the vocabulary axis must be contiguous")
    if drafter_logits.shape[0] != B or drafter_logits.shape[1] != K:
        raise ValueError("drafter logits must be [B, K, V_d]")
    for name, t, dtype, shape in (("draft_ids", draft_ids, torch.int32, (B, K)),
                                  ("temperature", temperature, torch.float32, (B,)),
                                  ("uniforms", uniforms, torch.float32, (B, K + 1)),
                                  ("accepted", accepted, torch.int32, (B,)),
                                  ("next_token", next_token, torch.int32, (B,))):
        if t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous():
            raise ValueError("%s must be a contiguous %s tensor of shape %s" % (name, dtype, shape))
    opt = lambda t: None if t is None else t.data_ptr()
    return tli_verify_args(
        B, K, dt,
        target_logits.data_ptr(), target_logits.stride(0), target_logits.stride(1),
        drafter_logits.data_ptr(), drafter_logits.stride(0), drafter_logits.stride(1),
        draft_ids.data_ptr(), temperature.data_ptr(), uniforms.data_ptr(),
        accepted.data_ptr(), next_token.data_ptr(), opt(row_status), opt(p_draft), opt(q_draft),
        workspace.data_ptr(), workspace.numel() * workspace.element_size(), opt(draft_lengths))


def tli_verify(ctx: int, args: tli_verify_args, stream: Optional[int] = None) -> None:
    """tli_verify() on ``stream`` (a cudaStream_t as int; default: torch's current stream)."""
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    rc = load().tli_verify(ctx, ctypes.byref(args), ctypes.c_void_p(stream))
    if rc != TLI_OK:
        raise TLIError(rc, "tli_verify")


def tli_verify_static(ctx: int, args: tli_verify_args, stream: Optional[int] = None) -> None:
    """tli_verify_static(): like tli_verify() but on the library's built-in 4 MiB scratch.

    For callers that cannot allocate device memory when they need to verify (all HBM already
    committed, or an allocation would stall the device).  ``args.workspace`` is ignored.  Calls
    that overlap on the GPU share the scratch and must be ordered by the caller."""
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    rc = load().tli_verify_static(ctx, ctypes.byref(args), ctypes.c_void_p(stream))
    if rc != TLI_OK:
        raise TLIError(rc, "tli_verify_static")


def tli_verify_host_buffer_bytes(ctx: int, B: int, K: int, dtype: int) -> int:
    return int(load().tli_verify_host_buffer_bytes(ctx, B, K, dtype))


def make_host_args(target_logits: torch.Tensor, drafter_logits: torch.Tensor, draft_ids: torch.Tensor,
                   temperature: torch.Tensor, uniforms: torch.Tensor, accepted: torch.Tensor, next_token: torch.Tensor,
                   device_buffer: torch.Tensor, row_status: Optional[torch.Tensor] = None) -> tli_verify_host_args:
    """Fill a tli_verify_host_args: contiguous CPU tensors (pinned for an asynchronous call) and a device buffer."""
    B, K1, _ = target_logits.shape
    for t in (target_logits, drafter_logits, draft_ids, temperature, uniforms, accepted, next_token):
        if t.is_cuda or not t.is_contiguous():
            raise ValueError("host tensors must be contiguous CPU tensors")
    return tli_verify_host_args(B, K1 - 1, _logit_dtype(target_logits), target_logits.data_ptr(), drafter_logits.data_ptr(),
                                draft_ids.data_ptr(), temperature.data_ptr(), uniforms.data_ptr(),
                                accepted.data_ptr(), next_token.data_ptr(),
                                None if row_status is None else row_status.data_ptr(),
                                device_buffer.data_ptr(), device_buffer.numel() * device_buffer.element_size())


def tli_verify_host(ctx: int, args: tli_verify_host_args, stream: Optional[int] = None) -> None:
    """tli_verify_host() on ``stream``; the outputs are valid after the stream has been synchronised."""
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    rc = load().tli_verify_host(ctx, ctypes.byref(args), ctypes.c_void_p(stream))
    if rc != TLI_OK:
        raise TLIError(rc, "tli_verify_host")


def tli_rates_workspace_bytes(ctx: int, B: int, K: int, dtype: int) -> int:
    return int(load().tli_rates_workspace_bytes(ctx, B, K, dtype))


def make_rates_args(target_logits: torch.Tensor, drafter_logits: torch.Tensor, temperature: torch.Tensor,
                    mass: torch.Tensor, alpha_union: torch.Tensor, alpha_tli: torch.Tensor, workspace: torch.Tensor,
                    position_status: Optional[torch.Tensor] = None) -> tli_rates_args:
    """Fill a tli_rates_args from device tensors (no copies; the tensors must outlive the call)."""
    B, K, _ = drafter_logits.shape
    dt = _logit_dtype(target_logits)
    if _logit_dtype(drafter_logits) != dt:
        raise TypeError("both logit tensors must have the same dtype")
    if target_logits.stride(2) != 1 or drafter_logits.stride(2) != 1:
        raise ValueError("the vocabulary axis must be contiguous")
    if target_logits.shape[0] != B or target_logits.shape[1] < K:
        raise ValueError("target logits must be [B, >=K, V_t]")
    for name, t in (("mass", mass), ("alpha_union", alpha_union), ("alpha_tli", alpha_tli)):
        if t.dtype != torch.float32 or tuple(t.shape) != (B, K) or not t.is_contiguous():
            raise ValueError("%s must be a contiguous float32 tensor of shape %s" % (name, (B, K)))
    return tli_rates_args(B, K, dt, target_logits.data_ptr(), target_logits.stride(0), target_logits.stride(1),
                          drafter_logits.data_ptr(), drafter_logits.stride(0), drafter_logits.stride(1),
                          temperature.data_ptr(), mass.data_ptr(), alpha_union.data_ptr(), alpha_tli.data_ptr(),
                          None if position_status is None else position_status.data_ptr(),
                          workspace.data_ptr(), workspace.numel() * workspace.element_size())


def tli_acceptance_rates(ctx: int, args: tli_rates_args, stream: Optional[int] = None) -> None:
    """tli_acceptance_rates() on ``stream`` (a cudaStream_t as int; default: torch's current stream)."""
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    rc = load().tli_acceptance_rates(ctx, ctypes.byref(args), ctypes.c_void_p(stream))
    if rc != TLI_OK:
        raise TLIError(rc, "tli_acceptance_rates")


def tli_draft_workspace_bytes(ctx: int, B: int, R: int, dtype: int) -> int:
    return int(load().tli_draft_workspace_bytes(ctx, B, R, dtype))


def make_draft_args(drafter_logits: torch.Tensor, temperature: torch.Tensor, uniforms: torch.Tensor,
                    draft_ids: torch.Tensor, workspace: torch.Tensor, q_draft: Optional[torch.Tensor] = None,
                    draft_status: Optional[torch.Tensor] = None) -> tli_draft_args:
    """Fill a tli_draft_args from device tensors (no copies; the tensors must outlive the call)."""
    B, R, _ = drafter_logits.shape
    dt = _logit_dtype(drafter_logits)
    if drafter_logits.stride(2) != 1:
        raise ValueError("the vocabulary axis must be contiguous")
    for name, t, dtype, shape in (("temperature", temperature, torch.float32, (B,)),
                                  ("uniforms", uniforms, torch.float32, (B, R)),
                                  ("draft_ids", draft_ids, torch.int32, (B, R))):
        if t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous():
            raise ValueError("%s must be a contiguous %s tensor of shape %s" % (name, dtype, shape))
    opt = lambda t: None if t is None else t.data_ptr()
    return tli_draft_args(B, R, dt, drafter_logits.data_ptr(), drafter_logits.stride(0), drafter_logits.stride(1),
                          temperature.data_ptr(), uniforms.data_ptr(), draft_ids.data_ptr(), opt(q_draft),
                          opt(draft_status), workspace.data_ptr(), workspace.numel() * workspace.element_size())


def tli_draft_sample(ctx: int, args: tli_draft_args, stream: Optional[int] = None) -> None:
    """tli_draft_sample() on ``stream`` (a cudaStream_t as int; default: torch's current stream)."""
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    rc = load().tli_draft_sample(ctx, ctypes.byref(args), ctypes.c_void_p(stream))
    if rc != TLI_OK:
        raise TLIError(rc, "tli_draft_sample")


def tli_slem_workspace_bytes(ctx: int, B: int, M: int, dtype: int) -> int:
    return int(load().tli_slem_workspace_bytes(ctx, B, M, dtype))


def make_slem_args(target_logits: torch.Tensor, candidates: torch.Tensor, temperature: torch.Tensor,
                   uniforms: torch.Tensor, accepted: torch.Tensor, next_token: torch.Tensor, workspace: torch.Tensor,
                   lengths: Optional[torch.Tensor] = None, sampled: Optional[torch.Tensor] = None,
                   row_status: Optional[torch.Tensor] = None) -> tli_slem_args:
    """Fill a tli_slem_args from device tensors (no copies; the tensors must outlive the call)."""
    B, M1, _ = target_logits.shape
    M = M1 - 1
    dt = _logit_dtype(target_logits)
    if target_logits.stride(2) != 1:
        raise ValueError("the vocabulary axis must be contiguous")
    for name, t, dtype, shape in (("candidates", candidates, torch.int32, (B, M)),
                                  ("temperature", temperature, torch.float32, (B,)),
                                  ("uniforms", uniforms, torch.float32, (B, M + 1)),
                                  ("accepted", accepted, torch.int32, (B,)),
                                  ("next_token", next_token, torch.int32, (B,))):
        if t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous():
            raise ValueError("%s must be a contiguous %s tensor of shape %s" % (name, dtype, shape))
    opt = lambda t: None if t is None else t.data_ptr()
    return tli_slem_args(B, M, dt, target_logits.data_ptr(), target_logits.stride(0), target_logits.stride(1),
                         candidates.data_ptr(), opt(lengths), temperature.data_ptr(), uniforms.data_ptr(),
                         accepted.data_ptr(), next_token.data_ptr(), opt(sampled), opt(row_status),
                         workspace.data_ptr(), workspace.numel() * workspace.element_size())


def tli_slem_verify(ctx: int, args: tli_slem_args, stream: Optional[int] = None) -> None:
    """tli_slem_verify() on ``stream`` (a cudaStream_t as int; default: torch's current stream)."""
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    rc = load().tli_slem_verify(ctx, ctypes.byref(args), ctypes.c_void_p(stream))
    if rc != TLI_OK:
        raise TLIError(rc, "tli_slem_verify")


def tli_sample_workspace_bytes(ctx: int, B: int, R: int, dtype: int, side: int) -> int:
    return int(load().tli_sample_workspace_bytes(ctx, B, R, dtype, side))


def tli_filter_workspace_bytes(ctx: int, B: int, R: int, dtype: int, side: int) -> int:
    return int(load().tli_filter_workspace_bytes(ctx, B, R, dtype, side))


def _check_rows(ctx: int, logits: torch.Tensor, side: int, tensors) -> None:
    if logits.dim() != 3:
        raise ValueError("logits must be [B, R, V]")
    if side not in (TLI_SIDE_TARGET, TLI_SIDE_DRAFTER):
        raise ValueError("side must be TLI_SIDE_TARGET or TLI_SIDE_DRAFTER")
    V_t, V_d = ctypes.c_int32(), ctypes.c_int32()
    rc = load().tli_ctx_info(ctx, ctypes.byref(V_t), ctypes.byref(V_d), None)
    if rc != TLI_OK:
        raise TLIError(rc, "tli_ctx_info")
    V = V_t.value if side == TLI_SIDE_TARGET else V_d.value
    if logits.shape[2] != V:
        raise ValueError("rows of this side have %d logits, not %d" % (V, logits.shape[2]))
    if V > 1 and logits.stride(2) != 1:
        raise ValueError("the vocabulary axis must be contiguous")
    for name, t, dtype, shape in tensors:
        if t is not None and (t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous()):
            raise ValueError("%s must be a contiguous %s tensor of shape %s" % (name, dtype, shape))
        if t is not None and t.device != logits.device:
            raise ValueError("%s must be on %s" % (name, logits.device))


def make_sample_args(ctx: int, logits: torch.Tensor, temperature: torch.Tensor, uniforms: torch.Tensor, tokens: torch.Tensor,
                     workspace: torch.Tensor, side: int = TLI_SIDE_TARGET, top_k: Optional[torch.Tensor] = None,
                     top_p: Optional[torch.Tensor] = None, min_p: Optional[torch.Tensor] = None,
                     prob: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None) -> tli_sample_args:
    """Fill a tli_sample_args from device tensors (no copies; the tensors must outlive the call)."""
    dt = _logit_dtype(logits)
    B, R = logits.shape[0], logits.shape[1] if logits.dim() == 3 else 0
    _check_rows(ctx, logits, side, (("temperature", temperature, torch.float32, (B,)), ("top_k", top_k, torch.int32, (B,)),
                                    ("top_p", top_p, torch.float32, (B,)), ("min_p", min_p, torch.float32, (B,)),
                                    ("uniforms", uniforms, torch.float32, (B, R)), ("tokens", tokens, torch.int32, (B, R)),
                                    ("prob", prob, torch.float32, (B, R)), ("status", status, torch.int32, (B, R))))
    opt = lambda t: None if t is None else t.data_ptr()
    return tli_sample_args(B, R, dt, side, logits.data_ptr(), logits.stride(0), logits.stride(1),
                           temperature.data_ptr(), opt(top_k), opt(top_p), opt(min_p), uniforms.data_ptr(),
                           tokens.data_ptr(), opt(prob), opt(status),
                           workspace.data_ptr(), workspace.numel() * workspace.element_size())


def tli_sample(ctx: int, args: tli_sample_args, stream: Optional[int] = None) -> None:
    """tli_sample() on ``stream`` (a cudaStream_t as int; default: torch's current stream)."""
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    rc = load().tli_sample(ctx, ctypes.byref(args), ctypes.c_void_p(stream))
    if rc != TLI_OK:
        raise TLIError(rc, "tli_sample")


def make_filter_args(ctx: int, logits: torch.Tensor, temperature: torch.Tensor, out: torch.Tensor, workspace: torch.Tensor,
                     side: int = TLI_SIDE_TARGET, top_k: Optional[torch.Tensor] = None, top_p: Optional[torch.Tensor] = None,
                     min_p: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None) -> tli_filter_args:
    """Fill a tli_filter_args from device tensors (no copies; the tensors must outlive the call)."""
    dt = _logit_dtype(logits)
    B, R = logits.shape[0], logits.shape[1] if logits.dim() == 3 else 0
    _check_rows(ctx, logits, side, (("temperature", temperature, torch.float32, (B,)), ("top_k", top_k, torch.int32, (B,)),
                                    ("top_p", top_p, torch.float32, (B,)), ("min_p", min_p, torch.float32, (B,)),
                                    ("status", status, torch.int32, (B, R))))
    if out.dtype != logits.dtype or out.shape != logits.shape or out.device != logits.device or (out.shape[2] > 1 and out.stride(2) != 1):
        raise ValueError("out must have the logits' type, shape and device, and a contiguous vocabulary axis")
    opt = lambda t: None if t is None else t.data_ptr()
    return tli_filter_args(B, R, dt, side, logits.data_ptr(), logits.stride(0), logits.stride(1),
                           temperature.data_ptr(), opt(top_k), opt(top_p), opt(min_p),
                           out.data_ptr(), out.stride(0), out.stride(1), opt(status),
                           workspace.data_ptr(), workspace.numel() * workspace.element_size())


def tli_filter(ctx: int, args: tli_filter_args, stream: Optional[int] = None) -> None:
    """tli_filter() on ``stream`` (a cudaStream_t as int; default: torch's current stream)."""
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    rc = load().tli_filter(ctx, ctypes.byref(args), ctypes.c_void_p(stream))
    if rc != TLI_OK:
        raise TLIError(rc, "tli_filter")


def _matrix(name: str, t: torch.Tensor) -> int:
    """Row stride of a [rows, H] tensor with contiguous rows."""
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError("%s must be a matrix with contiguous rows" % name)
    return t.stride(0)


def _check_ids(ids: torch.Tensor, N: int) -> None:
    if ids.dtype != torch.int32 or ids.numel() != N or not ids.is_contiguous():
        raise ValueError("ids must be a contiguous %s tensor of %d entries" % (torch.int32, N))


def make_embed_args(ids: torch.Tensor, table: torch.Tensor, out: torch.Tensor, scale: float = 1.0,
                    ids_side: int = TLI_SIDE_TARGET, table_side: int = TLI_SIDE_TARGET,
                    table_ids: Optional[torch.Tensor] = None) -> tli_embed_args:
    """Fill a tli_embed_args from device tensors (no copies; the tensors must outlive the call)."""
    N = ids.numel()
    _check_ids(ids, N)
    H = table.shape[-1]
    if tuple(out.shape) != (N, H) or out.dtype != table.dtype:
        raise ValueError("out must be [%d, %d] in the table's type" % (N, H))
    if table_ids is not None:
        _check_ids(table_ids, N)
    return tli_embed_args(N, H, _logit_dtype(table), ids_side, table_side, ids.data_ptr(), table.data_ptr(), _matrix("table", table),
                          float(scale), out.data_ptr(), _matrix("out", out), None if table_ids is None else table_ids.data_ptr())


def tli_embed(ctx: int, args: tli_embed_args, stream: Optional[int] = None) -> None:
    """tli_embed() on ``stream`` (a cudaStream_t as int; default: torch's current stream)."""
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    rc = load().tli_embed(ctx, ctypes.byref(args), ctypes.c_void_p(stream))
    if rc != TLI_OK:
        raise TLIError(rc, "tli_embed")


def tli_embed_grad_workspace_bytes(ctx: int, N: int, H: int) -> int:
    return int(load().tli_embed_grad_workspace_bytes(ctx, N, H))


def tli_head_loss_workspace_bytes(ctx: int, N: int, H: int, k: int, side: int) -> int:
    return int(load().tli_head_loss_workspace_bytes(ctx, N, H, k, side))


def tli_head_loss_grad_workspace_bytes(ctx: int, N: int, H: int, k: int, side: int) -> int:
    return int(load().tli_head_loss_grad_workspace_bytes(ctx, N, H, k, side))


def make_embed_grad_args(ids: torch.Tensor, grad: torch.Tensor, out: torch.Tensor, workspace: torch.Tensor, scale: float = 1.0,
                         ids_side: int = TLI_SIDE_TARGET, table_side: int = TLI_SIDE_TARGET) -> tli_embed_grad_args:
    """Fill a tli_embed_grad_args from device tensors (no copies; the tensors must outlive the call)."""
    N = ids.numel()
    _check_ids(ids, N)
    H = grad.shape[-1]
    if tuple(grad.shape) != (N, H) or out.dim() != 2 or out.shape[1] != H:
        raise ValueError("grad must be [%d, H] and out [V, H]" % N)
    return tli_embed_grad_args(N, H, _logit_dtype(grad), _logit_dtype(out), ids_side, table_side, ids.data_ptr(),
                               grad.data_ptr(), _matrix("grad", grad), float(scale), out.data_ptr(), _matrix("out", out),
                               workspace.data_ptr(), workspace.numel() * workspace.element_size())


def tli_embed_grad(ctx: int, args: tli_embed_grad_args, stream: Optional[int] = None) -> None:
    """tli_embed_grad() on ``stream`` (a cudaStream_t as int; default: torch's current stream)."""
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    rc = load().tli_embed_grad(ctx, ctypes.byref(args), ctypes.c_void_p(stream))
    if rc != TLI_OK:
        raise TLIError(rc, "tli_embed_grad")


def tli_verify_profile(ctx: int, args: tli_verify_args, stream: Optional[int] = None):
    """tli_verify_profile(): blocks; returns ms of (statistics kernel, decision kernel or 0, sampling kernel)."""
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    ms = (ctypes.c_float * 3)()
    rc = load().tli_verify_profile(ctx, ctypes.byref(args), ctypes.c_void_p(stream), ms)
    if rc != TLI_OK:
        raise TLIError(rc, "tli_verify_profile")
    return ms[0], ms[1], ms[2]


def tli_set_max_cluster(ctx: int, ctas: int) -> None:
    """tli_set_max_cluster(): widest cluster of the cluster kernel, 8 (portable) or 16 (where the device places it)."""
    rc = load().tli_set_max_cluster(ctx, int(ctas))
    if rc != TLI_OK:
        raise TLIError(rc, "tli_set_max_cluster")


def tli_set_tiled(ctx: int, enabled: bool) -> None:
    """tli_set_tiled(): the extra token by size (default) or always by the tile kernels."""
    rc = load().tli_set_tiled(ctx, 1 if enabled else 0)
    if rc != TLI_OK:
        raise TLIError(rc, "tli_set_tiled")


def tli_shard_create(device: int, V_t: int, V_d: int, id_map, n_shards: int, shard: int) -> int:
    """tli_shard_create(): the context of shard ``shard`` of ``n_shards``; returns the handle (an int)."""
    m = np.ascontiguousarray(id_map, dtype=np.int32)
    if m.shape != (V_d,):
        raise ValueError("id_map must have V_d entries")
    ctx = ctypes.c_void_p()
    rc = load().tli_shard_create(ctypes.byref(ctx), device, V_t, V_d, m.ctypes.data_as(ctypes.c_void_p), n_shards, shard)
    if rc != TLI_OK:
        raise TLIError(rc, "tli_shard_create")
    return ctx.value


def tli_shard_info(ctx: int) -> Dict[str, int]:
    """tli_shard_info(): the id ranges of a shard's context."""
    v = [ctypes.c_int32() for _ in range(6)]
    rc = load().tli_shard_info(ctx, *[ctypes.byref(x) for x in v])
    if rc != TLI_OK:
        raise TLIError(rc, "tli_shard_info")
    return dict(zip(("t_begin", "t_count", "d_begin", "d_count", "t_width", "d_width"), (x.value for x in v)))


def _shard_call(name: str, ctx: int, args: tli_verify_args, *buffers: torch.Tensor, stream: Optional[int] = None) -> None:
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    rc = getattr(load(), name)(ctx, ctypes.byref(args), *[ctypes.c_void_p(b.data_ptr()) for b in buffers], ctypes.c_void_p(stream))
    if rc != TLI_OK:
        raise TLIError(rc, name)


def tli_shard_stats(ctx: int, args: tli_verify_args, record: torch.Tensor, stream: Optional[int] = None) -> None:
    """tli_shard_stats(): this shard's statistics record."""
    _shard_call("tli_shard_stats", ctx, args, record, stream=stream)


def tli_shard_decide(ctx: int, args: tli_verify_args, records_all: torch.Tensor, rows: torch.Tensor,
                     stream: Optional[int] = None) -> None:
    """tli_shard_decide(): the decisions from all shards' records; packs this shard's slices of drafter row n."""
    _shard_call("tli_shard_decide", ctx, args, records_all, rows, stream=stream)


def tli_shard_weights(ctx: int, args: tli_verify_args, rows_all: torch.Tensor, mass: torch.Tensor,
                      stream: Optional[int] = None) -> None:
    """tli_shard_weights(): tile sums and totals of the extra token's weights over this shard's target ids."""
    _shard_call("tli_shard_weights", ctx, args, rows_all, mass, stream=stream)


def tli_shard_select(ctx: int, args: tli_verify_args, rows_all: torch.Tensor, masses_all: torch.Tensor,
                     stream: Optional[int] = None) -> None:
    """tli_shard_select(): the extra token on the shard that holds it, -1 elsewhere."""
    _shard_call("tli_shard_select", ctx, args, rows_all, masses_all, stream=stream)


def tli_verify_plan(ctx: int, B: int, K: int, dtype: int) -> Dict[str, int]:
    """tli_verify_plan(): how a batch of this shape will be run."""
    plan = (ctypes.c_int32 * 8)()
    rc = load().tli_verify_plan(ctx, B, K, dtype, plan)
    if rc != TLI_OK:
        raise TLIError(rc, "tli_verify_plan")
    return dict(zip(("launches", "cluster", "stats_ctas", "stage_bytes", "segment_bytes", "segments_per_target_row",
                     "segments_per_drafter_row", "cluster_smem_bytes"), plan))


def tli_launch_probe(ctx: int, B: int, K: int, dtype: int, stream: Optional[int] = None) -> None:
    """tli_launch_probe(): the launches of one call with kernels that do nothing."""
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    rc = load().tli_launch_probe(ctx, B, K, dtype, ctypes.c_void_p(stream))
    if rc != TLI_OK:
        raise TLIError(rc, "tli_launch_probe")


def tli_reset(ctx: int, stream: Optional[int] = None) -> None:
    """tli_reset(): the context's counters and its sticky time-out word back to zero, in stream order."""
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    rc = load().tli_reset(ctx, ctypes.c_void_p(stream))
    if rc != TLI_OK:
        raise TLIError(rc, "tli_reset")


def tli_selftest_bounded_wait(ctx: int, polls: int = 2000, stream: Optional[int] = None) -> bool:
    """tli_selftest_bounded_wait(): True if a wait on a barrier nothing completes gave up after `polls` polls."""
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    out = ctypes.c_int(0)
    rc = load().tli_selftest_bounded_wait(ctx, ctypes.c_void_p(stream), polls, ctypes.byref(out))
    if rc != TLI_OK:
        raise TLIError(rc, "tli_selftest_bounded_wait")
    return out.value == 1


# The argument structs of the calls below as bytes: packing them is a third of the cost of filling a ctypes.Structure, which counts where
# a call takes ten microseconds.  Native alignment ("@") lays them out as C does; "0P" pads the end.
_PACK_SAMPLE = struct.Struct("@iiiiPqqPPPPPPPPPN").pack
_PACK_FILTER = struct.Struct("@iiiiPqqPPPPPqqPPN").pack
_PACK_EMBED = struct.Struct("@iiiiiPPqfPqP").pack
_PACK_EMBED_GRAD = struct.Struct("@iiiiiiPPqfPqPN").pack
_PACK_LOSS = struct.Struct("@iiiiiiiPqPPPPPP").pack
_PACK_LOSS_GRAD = struct.Struct("@iiiiiiiPqPPPPPPq").pack
_PACK_HEAD_LOSS = struct.Struct("@iiiiiiiPqPqPPPPPPPPN").pack
_PACK_HEAD_LOSS_GRAD = struct.Struct("@iiiiiiiPqPqPPPPPPPqPqPPN").pack


_KEPT_BYTES = 64 << 20                                             # of scratch, per thread and stream of a Verifier


def _packed_entries():
    """The entry points of the calls below as functions of (ctx, packed struct, stream)."""
    load()
    lib = ctypes.CDLL(LIB_PATH)                                    # function objects of its own, the library is loaded once
    entries = [lib.tli_sample, lib.tli_filter, lib.tli_embed, lib.tli_embed_grad, lib.tli_loss, lib.tli_loss_grad,
               lib.tli_head_loss, lib.tli_head_loss_grad]
    for fn in entries:
        fn.argtypes, fn.restype = [ctypes.c_void_p, ctypes.c_char_p, ctypes.c_void_p], ctypes.c_int
    return entries


def _current_device() -> int:
    return torch._C._cuda_getDevice()


def _raw_stream(index: int) -> int:
    """The current stream of a device as an int, without an object for it."""
    return torch._C._cuda_getCurrentRawStream(index)


class Verifier:
    """Convenience owner of one context plus its scratch and output tensors."""

    def __init__(self, V_t: int, V_d: int, id_map, device: int = 0, tiled: bool = False):
        self.device = torch.device("cuda", device)
        self.V_t, self.V_d = int(V_t), int(V_d)
        self.ctx = tli_create(device, V_t, V_d, id_map)
        if tiled:
            tli_set_tiled(self.ctx, True)
        self._ws: Optional[torch.Tensor] = None
        self._index, self._plans = int(device), {}
        (self._fn_sample, self._fn_filter, self._fn_embed, self._fn_embed_grad, self._fn_loss,
         self._fn_loss_grad, self._fn_head_loss, self._fn_head_loss_grad) = _packed_entries()
        self._kept = threading.local()

    def close(self) -> None:
        if self.ctx:
            tli_destroy(self.ctx)
            self.ctx = 0
        self._ws, self._kept = None, threading.local()             # scratch of every thread and stream

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def workspace(self, B: int, K: int, dtype: int) -> torch.Tensor:
        need = tli_workspace_bytes(self.ctx, B, K, dtype)
        if need == 0:
            raise TLIError(TLI_ERR_UNSUPPORTED, "tli_workspace_bytes")
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(need, dtype=torch.uint8, device=self.device)
        return self._ws

    def draft(self, drafter_logits, temperature, uniforms) -> Dict[str, torch.Tensor]:
        """Draw one drafter id per row of ``drafter_logits`` [B,R,V_d] from q'; returns device tensors."""
        B, R, _ = drafter_logits.shape
        dev = self.device
        out = {"draft_ids": torch.empty(B, R, dtype=torch.int32, device=dev),
               "q_draft": torch.empty(B, R, dtype=torch.float32, device=dev),
               "draft_status": torch.empty(B, R, dtype=torch.int32, device=dev)}
        need = tli_draft_workspace_bytes(self.ctx, B, R, _logit_dtype(drafter_logits))
        if need == 0:
            raise TLIError(TLI_ERR_UNSUPPORTED, "tli_draft_workspace_bytes")
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(need, dtype=torch.uint8, device=dev)
        args = make_draft_args(drafter_logits, temperature, uniforms, out["draft_ids"], self._ws,
                               out["q_draft"], out["draft_status"])
        tli_draft_sample(self.ctx, args)
        return out

    # The calls below may overlap others on this context.  Scratch is kept per thread and stream (on one stream calls use it one
    # after the other; two threads could interleave the kernels of theirs), a captured call has its own, and what is more than
    # _KEPT_BYTES (a training batch's head gradients, hundreds of MB) goes back to torch's allocator behind the call, which takes
    # so long that asking for it again is nothing.  What depends on shapes alone is worked out once per shape.

    def _scratch(self, need: int) -> torch.Tensor:
        if need > _KEPT_BYTES or torch._C._cuda_isCurrentStreamCapturing() or _current_device() != self._index:
            return torch.empty(need, dtype=torch.uint8, device=self.device)
        kept = self._kept.__dict__
        stream = _raw_stream(self._index)
        ws = kept.get(stream)
        if ws is None or ws.numel() < need:
            ws = kept[stream] = torch.empty(need, dtype=torch.uint8, device=self.device)
        return ws

    def _plan(self, key, plan):
        if len(self._plans) > 1000:
            self._plans.clear()
        self._plans[key] = plan
        return plan

    def _call(self, fn, args: bytes) -> None:
        """One of the entry points below on the current stream; ``args``: its argument struct, packed."""
        if _current_device() == self._index:
            rc = fn(self.ctx, args, _raw_stream(self._index))
        else:
            with torch.cuda.device(self._index):
                rc = fn(self.ctx, args, _raw_stream(self._index))
        if rc != TLI_OK:
            raise TLIError(rc, fn.__name__)

    def _row_plan(self, logits, side):
        """(shape of a per-sequence tensor, shape of a per-row one, scratch bytes, dtype, strides)."""
        B, R, _ = logits.shape
        dt = _logit_dtype(logits)
        _check_rows(self.ctx, logits, side, ())
        need = tli_sample_workspace_bytes(self.ctx, B, R, dt, side)
        if need == 0 or tli_filter_workspace_bytes(self.ctx, B, R, dt, side) != need:
            raise TLIError(TLI_ERR_UNSUPPORTED, "tli_sample_workspace_bytes")
        sb, sr, _ = logits.stride()
        return (B,), (B, R), need, (B, R, dt, side), sb, sr

    def _rows(self, logits, side, temperature, top_k, top_p, min_p):
        if logits.dim() != 3:
            raise ValueError("logits must be [B, R, V]")
        key = (logits.shape, logits.stride(), logits.dtype, side)
        plan = self._plans.get(key)
        if plan is None:
            plan = self._plan(key, self._row_plan(logits, side))
        on, shape = self._index, plan[0]
        if logits.get_device() != on:
            raise ValueError("logits must be on %s" % self.device)
        for t, dtype in ((temperature, torch.float32), (top_k, torch.int32), (top_p, torch.float32), (min_p, torch.float32)):
            if t is not None and (t.dtype is not dtype or t.shape != shape or t.get_device() != on or not t.is_contiguous()):
                raise ValueError("temperature, top_k, top_p and min_p must be contiguous float32, int32, float32 and float32 "
                                 "tensors of shape %s on %s" % (shape, self.device))
        return plan

    def sample(self, logits, temperature, uniforms, side: int = TLI_SIDE_TARGET, top_k=None, top_p=None,
               min_p=None) -> Dict[str, torch.Tensor]:
        """Draw one id per row of ``logits`` [B,R,V] under temperature, top-k, top-p and min-p (per sequence,
        ``None`` = off); on the drafter side from the ids inside the intersection.  Returns device tensors."""
        _, shape, need, head, sb, sr = self._rows(logits, side, temperature, top_k, top_p, min_p)
        if uniforms.dtype is not torch.float32 or uniforms.shape != shape or uniforms.get_device() != self._index or not uniforms.is_contiguous():
            raise ValueError("uniforms must be a contiguous float32 tensor of shape %s on %s" % (shape, self.device))
        prob = torch.empty_like(uniforms)                          # (cheaper than torch.empty with a shape and a device)
        tokens = torch.empty_like(uniforms, dtype=torch.int32)
        status = torch.empty_like(tokens)
        ws = self._scratch(need)
        self._call(self._fn_sample, _PACK_SAMPLE(
            *head, logits.data_ptr(), sb, sr, temperature.data_ptr(), 0 if top_k is None else top_k.data_ptr(),
            0 if top_p is None else top_p.data_ptr(), 0 if min_p is None else min_p.data_ptr(), uniforms.data_ptr(),
            tokens.data_ptr(), prob.data_ptr(), status.data_ptr(), ws.data_ptr(), need))
        return {"tokens": tokens, "prob": prob, "status": status}

    def filter(self, logits, temperature, side: int = TLI_SIDE_TARGET, top_k=None, top_p=None, min_p=None,
               out=None) -> Dict[str, torch.Tensor]:
        """The rows of ``logits`` [B,R,V] with -inf outside the kept set (``out=logits``: in place)."""
        _, shape, need, head, sb, sr = self._rows(logits, side, temperature, top_k, top_p, min_p)
        if out is None:
            out = torch.empty_like(logits)
        elif out.dtype is not logits.dtype or out.shape != logits.shape or out.get_device() != self._index or (out.shape[2] > 1 and out.stride(2) != 1):
            raise ValueError("out must have the logits' type, shape and device, and a contiguous vocabulary axis")
        status = torch.empty(shape, dtype=torch.int32, device=self.device)
        ws = self._scratch(need)
        ob, orr, _ = out.stride()
        self._call(self._fn_filter, _PACK_FILTER(
            *head, logits.data_ptr(), sb, sr, temperature.data_ptr(), 0 if top_k is None else top_k.data_ptr(),
            0 if top_p is None else top_p.data_ptr(), 0 if min_p is None else min_p.data_ptr(),
            out.data_ptr(), ob, orr, status.data_ptr(), ws.data_ptr(), need))
        return {"logits": out, "status": status}

    def _table_rows(self, side: int) -> int:
        if side not in (TLI_SIDE_TARGET, TLI_SIDE_DRAFTER):
            raise ValueError("a side must be TLI_SIDE_TARGET or TLI_SIDE_DRAFTER")
        return self.V_t if side == TLI_SIDE_TARGET else self.V_d

    def _ids(self, ids) -> None:
        if ids.dtype is not torch.int32 or ids.get_device() != self._index or not ids.is_contiguous():
            raise ValueError("ids must be a contiguous int32 tensor on %s" % self.device)

    def embed(self, ids, table, scale: float = 1.0, ids_side: int = TLI_SIDE_TARGET,
              table_side: int = TLI_SIDE_TARGET) -> Dict[str, torch.Tensor]:
        """Rows of ``table`` [V,H] for ``ids`` (any shape) of either vocabulary, times ``scale``, and the ids in
        the table's vocabulary (-1, with a zero row, where there is none).  The rows are no part of an autograd graph:
        the table's gradient is :meth:`embed_grad`'s (a table that waits for one by other means gets a warning)."""
        if table.requires_grad and torch.is_grad_enabled():
            warnings.warn("embed() records no autograd graph: the table gets its gradient from embed_grad(), or detach it", stacklevel=2)
        self._ids(ids)
        V, dev = self._table_rows(table_side), self.device
        if table.dim() != 2 or table.shape[0] != V or table.get_device() != self._index:
            raise ValueError("table must be [%d, H] on %s" % (V, dev))
        stride, H = _matrix("table", table), table.shape[1]        # (H 1: any stride will do)
        rows = table.new_empty((*ids.shape, H))
        table_ids = torch.empty_like(ids)
        self._call(self._fn_embed, _PACK_EMBED(ids.numel(), H, _logit_dtype(table), ids_side, table_side, ids.data_ptr(), table.data_ptr(), stride,
                                               scale, rows.data_ptr(), H, table_ids.data_ptr()))
        return {"rows": rows, "table_ids": table_ids}

    def embed_grad(self, ids, grad, scale: float = 1.0, ids_side: int = TLI_SIDE_TARGET, table_side: int = TLI_SIDE_TARGET,
                   dtype: Optional[torch.dtype] = None) -> Dict[str, torch.Tensor]:
        """Gradient of :meth:`embed` with respect to the table, [V,H] in ``dtype`` (default: the type of ``grad``)."""
        self._ids(ids)
        N, V, dev = ids.numel(), self._table_rows(table_side), self.device
        H = grad.shape[-1]
        if grad.shape != (*ids.shape, H) or grad.get_device() != self._index:
            raise ValueError("grad must have the shape of ids, and H, on %s" % dev)
        if grad.dim() != 2:
            grad = grad.reshape(N, H)
        stride = _matrix("grad", grad)
        out = torch.empty((V, H), dtype=dtype or grad.dtype, device=dev)
        need = self._plans.get((N, H))
        if need is None:
            need = self._plan((N, H), tli_embed_grad_workspace_bytes(self.ctx, N, H))
        if need == 0:
            raise TLIError(TLI_ERR_UNSUPPORTED, "tli_embed_grad_workspace_bytes")
        ws = self._scratch(need)
        self._call(self._fn_embed_grad, _PACK_EMBED_GRAD(N, H, _logit_dtype(grad), _logit_dtype(out), ids_side, table_side, ids.data_ptr(),
                                                         grad.data_ptr(), stride, scale, out.data_ptr(), H, ws.data_ptr(), need))
        return {"grad": out}

    # The losses.  `ids` [N] are labels; `ids` [N, k] with `teacher` [N, k] a teacher's logits of k ids.  `stats` and `target_logits` are
    # the forward call's.  Like the other calls they record no autograd graph.

    def _loss_plan(self, N: int, ids, teacher, side: int, ids_side: int, shared: bool):
        """What a loss call needs of its targets, from shapes and types alone: the part of its argument struct behind its sizes."""
        if teacher is None:
            k, t_dtype = 1, 0
            if ids.shape != (N,) and ids.shape != (N, 1):
                raise ValueError("labels must be [%d]" % N)
        else:
            if ids.dim() != 2 or ids.shape[0] != N or teacher.shape != ids.shape:
                raise ValueError("ids and teacher must be [%d, k]" % N)
            k, t_dtype = ids.shape[1], _logit_dtype(teacher)
        self._table_rows(side), self._table_rows(ids_side)
        return k, (side, ids_side, TLI_SUPPORT_SHARED if shared else TLI_SUPPORT_ALL, t_dtype)

    def _per_row(self, name: str, t, shape) -> None:
        if t.dtype is not torch.float32 or t.shape != shape or t.get_device() != self._index or not t.is_contiguous():
            raise ValueError("%s must be a contiguous float32 tensor of shape %s on %s" % (name, tuple(shape), self.device))

    def _loss_args(self, kind: str, x, ids, teacher, temperature, side: int, ids_side: int, shared: bool, more=()):
        """The plan of a loss call with rows ``x`` (worked out once per shape), the teacher's and the temperature's pointers."""
        on = self._index
        if x.get_device() != on:
            raise ValueError("%s must be on %s" % ("hidden" if more else "logits", self.device))
        self._ids(ids)
        key = (kind, x.shape, x.stride(), x.dtype, ids.shape, None if teacher is None else (teacher.shape, teacher.dtype), side, ids_side, shared, *more)
        plan = self._plans.get(key)
        if plan is None:
            plan = self._plan(key, getattr(self, kind)(x, ids, teacher, side, ids_side, shared, *more))
        t_ptr = tau_ptr = 0
        if teacher is not None:
            if teacher.get_device() != on or not teacher.is_contiguous():
                raise ValueError("teacher must be contiguous, on %s" % self.device)
            t_ptr = teacher.data_ptr()
        if temperature is not None:
            self._per_row("temperature", temperature, plan[0])
            tau_ptr = temperature.data_ptr()
        return plan, t_ptr, tau_ptr

    def _row_losses(self, logits, ids, teacher, side, ids_side, shared):
        if logits.dim() != 2 or logits.shape[1] != self._table_rows(side):
            raise ValueError("logits must be [N, %d] on %s" % (self._table_rows(side), self.device))
        N = logits.shape[0]
        k, rest = self._loss_plan(N, ids, teacher, side, ids_side, shared)
        return (N,), (N, 2), (N, k, _logit_dtype(logits), *rest), _matrix("logits", logits)

    def loss(self, logits, ids, teacher=None, temperature=None, side: int = TLI_SIDE_TARGET, ids_side: int = TLI_SIDE_TARGET,
             shared: bool = False) -> Dict[str, torch.Tensor]:
        """Loss of every row of ``logits`` [N,V] against labels ``ids`` [N], or a teacher's logits ``teacher`` [N,k] of ``ids`` [N,k];
        ids of either vocabulary.  ``shared``: the softmax runs over the ids inside the intersection (drafter rows).  Returns ``loss`` [N],
        ``stats`` [N,2] (for :meth:`loss_grad`) and ``status`` [N]; no autograd graph is recorded."""
        if logits.requires_grad and torch.is_grad_enabled():
            warnings.warn("loss() records no autograd graph: the logits get their gradient from loss_grad(), or detach them", stacklevel=2)
        (one, two, head, stride), t_ptr, tau_ptr = self._loss_args("_row_losses", logits, ids, teacher, temperature, side, ids_side, shared)
        stats = logits.new_empty(two, dtype=torch.float32)
        loss = stats.new_empty(one)
        status = torch.empty_like(loss, dtype=torch.int32)
        self._call(self._fn_loss, _PACK_LOSS(*head, logits.data_ptr(), stride, ids.data_ptr(), t_ptr, tau_ptr, loss.data_ptr(), stats.data_ptr(),
                                             status.data_ptr()))
        return {"loss": loss, "stats": stats, "status": status}

    def loss_grad(self, logits, ids, stats, grad_loss=None, teacher=None, temperature=None, side: int = TLI_SIDE_TARGET,
                  ids_side: int = TLI_SIDE_TARGET, shared: bool = False, out=None) -> Dict[str, torch.Tensor]:
        """Gradient of sum(grad_loss * loss) with respect to the logits, in their type (``out=logits``: in place)."""
        (one, two, head, stride), t_ptr, tau_ptr = self._loss_args("_row_losses", logits, ids, teacher, temperature, side, ids_side, shared)
        self._per_row("stats", stats, two)
        if grad_loss is not None:
            self._per_row("grad_loss", grad_loss, one)
        if out is None:
            out = logits.new_empty(logits.shape)
        elif out is not logits and (out.dtype is not logits.dtype or out.shape != logits.shape or out.get_device() != self._index):
            raise ValueError("out must have the logits' type, shape and device")
        self._call(self._fn_loss_grad, _PACK_LOSS_GRAD(*head, logits.data_ptr(), stride, ids.data_ptr(), t_ptr, tau_ptr, stats.data_ptr(),
                                                       0 if grad_loss is None else grad_loss.data_ptr(), out.data_ptr(), _matrix("out", out)))
        return {"grad": out}

    def _head_losses(self, hidden, ids, teacher, side, ids_side, shared, grad, w_shape, w_stride, w_dtype):
        if hidden.dim() != 2 or hidden.dtype is not torch.bfloat16:
            raise ValueError("hidden must be a bfloat16 [N, H] tensor on %s" % self.device)
        N, H = hidden.shape
        V = self._table_rows(side)
        if w_dtype is not torch.bfloat16 or w_shape != (V, H) or (H > 1 and w_stride[1] != 1):
            raise ValueError("weight must be a bfloat16 [%d, %d] tensor with contiguous rows on %s" % (V, H, self.device))
        k, rest = self._loss_plan(N, ids, teacher, side, ids_side, shared)
        need = (tli_head_loss_grad_workspace_bytes if grad else tli_head_loss_workspace_bytes)(self.ctx, N, H, k, side)
        if need == 0:
            raise TLIError(TLI_ERR_UNSUPPORTED, "tli_head_loss_workspace_bytes (H a multiple of 8 up to %d, N up to %d, k up to %d)"
                           % (TLI_MAX_H, TLI_MAX_HEAD_TOKENS, TLI_MAX_TARGETS))
        return (N,), (N, 2), (N, H, k, *rest), _matrix("hidden", hidden), w_stride[0], need

    def head_loss(self, hidden, weight, ids, teacher=None, temperature=None, side: int = TLI_SIDE_TARGET,
                  ids_side: int = TLI_SIDE_TARGET, shared: bool = False) -> Dict[str, torch.Tensor]:
        """:meth:`loss` of the logits ``hidden`` [N,H] x ``weight`` [V,H]^T (bfloat16, summed in fp32), which are not written."""
        if (hidden.requires_grad or weight.requires_grad) and torch.is_grad_enabled():
            warnings.warn("head_loss() records no autograd graph: gradients come from head_loss_grad(), or detach its inputs", stacklevel=2)
        if weight.get_device() != self._index:
            raise ValueError("weight must be on %s" % self.device)
        (one, two, head, hs, wst, need), t_ptr, tau_ptr = self._loss_args(
            "_head_losses", hidden, ids, teacher, temperature, side, ids_side, shared, (False, weight.shape, weight.stride(), weight.dtype))
        stats = hidden.new_empty(two, dtype=torch.float32)
        loss = stats.new_empty(one)
        status = torch.empty_like(loss, dtype=torch.int32)
        at = torch.empty_like(ids, dtype=torch.float32)
        ws = self._scratch(need)
        self._call(self._fn_head_loss, _PACK_HEAD_LOSS(
            *head, hidden.data_ptr(), hs, weight.data_ptr(), wst, ids.data_ptr(), t_ptr, tau_ptr, loss.data_ptr(), stats.data_ptr(),
            at.data_ptr(), status.data_ptr(), ws.data_ptr(), need))
        return {"loss": loss, "stats": stats, "target_logits": at, "status": status}

    def head_loss_grad(self, hidden, weight, ids, stats, target_logits, grad_loss=None, teacher=None, temperature=None,
                       side: int = TLI_SIDE_TARGET, ids_side: int = TLI_SIDE_TARGET, shared: bool = False,
                       hidden_grad: bool = True, weight_grad: bool = True) -> Dict[str, Optional[torch.Tensor]]:
        """Gradients of sum(grad_loss * loss) with respect to ``hidden`` and ``weight``, in bfloat16 (``None`` where not asked for)."""
        if weight.get_device() != self._index:
            raise ValueError("weight must be on %s" % self.device)
        (one, two, head, hs, wst, need), t_ptr, tau_ptr = self._loss_args(
            "_head_losses", hidden, ids, teacher, temperature, side, ids_side, shared, (True, weight.shape, weight.stride(), weight.dtype))
        self._per_row("stats", stats, two)
        self._per_row("target_logits", target_logits, ids.shape)
        if grad_loss is not None:
            self._per_row("grad_loss", grad_loss, one)
        H = head[1]
        dh = hidden.new_empty(hidden.shape) if hidden_grad else None
        dw = weight.new_empty(weight.shape) if weight_grad else None
        status = stats.new_empty(one, dtype=torch.int32)
        ws = self._scratch(need)
        self._call(self._fn_head_loss_grad, _PACK_HEAD_LOSS_GRAD(
            *head, hidden.data_ptr(), hs, weight.data_ptr(), wst, ids.data_ptr(), t_ptr, tau_ptr, stats.data_ptr(), target_logits.data_ptr(),
            0 if grad_loss is None else grad_loss.data_ptr(), 0 if dh is None else dh.data_ptr(), H, 0 if dw is None else dw.data_ptr(), H,
            status.data_ptr(), ws.data_ptr(), need))
        return {"grad_hidden": dh, "grad_weight": dw, "status": status}

    def rates(self, target_logits, drafter_logits, temperature) -> Dict[str, torch.Tensor]:
        """Expected acceptance rates per draft position (mass, alpha_union, alpha_tli); device tensors."""
        B, K, _ = drafter_logits.shape
        dev = self.device
        out = {k: torch.empty(B, K, dtype=torch.float32, device=dev) for k in ("mass", "alpha_union", "alpha_tli")}
        out["position_status"] = torch.empty(B, K, dtype=torch.int32, device=dev)
        need = tli_rates_workspace_bytes(self.ctx, B, K, _logit_dtype(target_logits))
        if need == 0:
            raise TLIError(TLI_ERR_UNSUPPORTED, "tli_rates_workspace_bytes")
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(need, dtype=torch.uint8, device=dev)
        args = make_rates_args(target_logits, drafter_logits, temperature, out["mass"], out["alpha_union"],
                               out["alpha_tli"], self._ws, out["position_status"])
        tli_acceptance_rates(self.ctx, args)
        return out

    def slem(self, target_logits, candidates, temperature, uniforms, lengths=None) -> Dict[str, torch.Tensor]:
        """Exact-match verification of re-tokenised drafts ``candidates`` [B,M] against tokens sampled
        from ``target_logits`` [B,M+1,V_t]; returns device tensors."""
        B, M1, _ = target_logits.shape
        dev = self.device
        out = {"accepted": torch.empty(B, dtype=torch.int32, device=dev),
               "next_token": torch.empty(B, dtype=torch.int32, device=dev),
               "sampled": torch.empty(B, M1, dtype=torch.int32, device=dev),
               "row_status": torch.empty(B, dtype=torch.int32, device=dev)}
        need = tli_slem_workspace_bytes(self.ctx, B, M1 - 1, _logit_dtype(target_logits))
        if need == 0:
            raise TLIError(TLI_ERR_UNSUPPORTED, "tli_slem_workspace_bytes")
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(need, dtype=torch.uint8, device=dev)
        args = make_slem_args(target_logits, candidates, temperature, uniforms, out["accepted"], out["next_token"],
                              self._ws, lengths, out["sampled"], out["row_status"])
        tli_slem_verify(self.ctx, args)
        return out

    def verify(self, target_logits, drafter_logits, draft_ids, temperature, uniforms,
               diagnostics: bool = True, draft_lengths=None) -> Dict[str, torch.Tensor]:
        """One call on torch's current stream; returns device tensors (no synchronisation)."""
        B, K1, _ = target_logits.shape
        K = K1 - 1
        dev = self.device
        out = {"accepted": torch.empty(B, dtype=torch.int32, device=dev),
               "next_token": torch.empty(B, dtype=torch.int32, device=dev),
               "row_status": torch.empty(B, dtype=torch.int32, device=dev)}
        if diagnostics:
            out["p_draft"] = torch.empty(B, K, dtype=torch.float32, device=dev)
            out["q_draft"] = torch.empty(B, K, dtype=torch.float32, device=dev)
        ws = self.workspace(B, K, _logit_dtype(target_logits))
        args = make_args(target_logits, drafter_logits, draft_ids, temperature, uniforms,
                         out["accepted"], out["next_token"], ws, out["row_status"],
                         out.get("p_draft"), out.get("q_draft"), draft_lengths)
        tli_verify(self.ctx, args)
        return out

"""Thin ctypes binding of the C ABI in include/twist.h (argument marshalling only).

Every function has the name of its C entry point.  Tensors are torch CUDA tensors
(torch is used for device memory and streams only); the binding passes their
data pointers and the current CUDA stream.  A non-zero status raises TwistError.
The shared library must exist: there is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtwist.so")

OK = 0
ERR_NULL, ERR_SHAPE, ERR_INFEASIBLE, ERR_BAD_INDEX, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_CUDA, ERR_DEVICE_TIMEOUT = \
    -1, -2, -3, -4, -5, -6, -7, -8
FP32, BF16 = 0, 1
FFN_RELU, FFN_GELU, FFN_SWIGLU = 0, 1, 2
MODE_COVER, MODE_IID = 0, 1
KIND_FFN, KIND_HEAD = 0, 1
PROJ_QKV, PROJ_O = 0, 1
ROPE_HALF, ROPE_PAIRS = 0, 1
CACHE_BF16, CACHE_E4M3 = 0, 1
MAX_SEGMENTS = 8

EXPORTS = [
    "twist_abi_version", "twist_strerror", "twist_last_cuda_error", "twist_device_status", "twist_sample_masks",
    "twist_kv_groups", "twist_gather_subnets", "twist_aggregate", "twist_subnet_ffn_fwd", "twist_subnet_ffn_bwd",
    "twist_subnet_attn_proj_fwd", "twist_subnet_attn_proj_bwd", "twist_mse_workspace_bytes", "twist_mse_fwd_bwd",
    "twist_mse_fwd_bwd_noalloc", "twist_fused_loss_workspace_bytes", "twist_attn_core_fwd", "twist_attn_core_bwd",
    "twist_hidden_mask", "twist_selftest_wait", "twist_layernorm_workspace_bytes", "twist_layernorm_fwd",
    "twist_layernorm_bwd", "twist_qkv_col_mask", "twist_apply_col_mask", "twist_plan_create", "twist_plan_destroy",
    "twist_plan_stats", "twist_workspace_bytes", "twist_aggregate_partial", "twist_aggregate_finish",
    "twist_rope_fwd", "twist_rope_bwd", "twist_kv_append", "twist_attn_decode", "twist_attn_decode_workspace_bytes",
    "twist_kv_append_q8", "twist_attn_decode_q8", "twist_attn_weights", "twist_attn_core_weights", "twist_kv_evict",
    "twist_kv_evict_workspace_bytes", "twist_selftest_decode_quit",
]


class TwistError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str = ""):
        self.status = status
        super().__init__(f"{where}: status {status} ({detail})")


class GatherSegment(C.Structure):
    _fields_ = [("src", C.c_void_p), ("dst", C.c_void_p), ("dst_master", C.c_void_p), ("idx", C.c_void_p),
                ("count", C.c_void_p), ("idx_stride", C.c_int32), ("n_keep", C.c_int32), ("block_rows", C.c_int32),
                ("n_blocks", C.c_int32), ("src_row_offset", C.c_int64), ("dst_subnet_stride", C.c_int64),
                ("dst_row_offset", C.c_int64)]


class AggregateSegment(C.Structure):
    _fields_ = [("dst", C.c_void_p), ("dst_f32", C.c_void_p), ("sub", C.c_void_p), ("cover", C.c_void_p),
                ("pos", C.c_void_p), ("n_full", C.c_int32), ("block_rows", C.c_int32), ("dst_row_offset", C.c_int64),
                ("sub_subnet_stride", C.c_int64), ("sub_row_offset", C.c_int64), ("central", C.c_void_p),
                ("central_subnet", C.c_int32), ("n_keep", C.c_int32)]


class Optimizer(C.Structure):
    _fields_ = [("kind", C.c_int32), ("step", C.c_int32), ("beta1", C.c_float), ("beta2", C.c_float), ("eps", C.c_float)]


OPT_SGD, OPT_ADAM = 0, 1


def adam(step: int, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8) -> Optimizer:
    return Optimizer(OPT_ADAM, step, beta1, beta2, eps)


class FfnArgs(C.Structure):
    _fields_ = [("ffn_kind", C.c_int32), ("dtype", C.c_int32), ("n_subnets", C.c_int32), ("tokens", C.c_int32),
                ("d_model", C.c_int32), ("f_sub", C.c_int32), ("out_scale", C.c_float), ("lr", C.c_float),
                ("x", C.c_void_p), ("w_gu", C.c_void_p), ("w_down", C.c_void_p), ("w_gu_master", C.c_void_p),
                ("w_down_master", C.c_void_p), ("pre", C.c_void_p), ("hh", C.c_void_p), ("y", C.c_void_p),
                ("dy", C.c_void_p), ("dpre", C.c_void_p), ("dx", C.c_void_p), ("dw_gu", C.c_void_p),
                ("dw_down", C.c_void_p), ("tgt", C.c_void_p), ("loss", C.c_void_p), ("loss_ws", C.c_void_p),
                ("loss_ws_bytes", C.c_size_t), ("y_residual", C.c_void_p), ("dx_residual", C.c_void_p),
                ("opt", Optimizer), ("m_gu", C.c_void_p), ("v_gu", C.c_void_p), ("m_down", C.c_void_p),
                ("v_down", C.c_void_p), ("hidden_mask", C.c_void_p), ("plan", C.c_void_p),
                ("master_from_slice", C.c_int32)]


class ProjArgs(C.Structure):
    _fields_ = [("which", C.c_int32), ("dtype", C.c_int32), ("n_subnets", C.c_int32), ("tokens", C.c_int32),
                ("d_model", C.c_int32), ("n", C.c_int32), ("out_scale", C.c_float), ("lr", C.c_float),
                ("in_", C.c_void_p), ("w", C.c_void_p), ("w_master", C.c_void_p), ("out", C.c_void_p),
                ("d_out", C.c_void_p), ("d_in", C.c_void_p), ("dw", C.c_void_p), ("tgt", C.c_void_p),
                ("loss", C.c_void_p), ("loss_ws", C.c_void_p), ("loss_ws_bytes", C.c_size_t),
                ("valid_cols", C.c_void_p), ("seg_begin", C.c_int32), ("seg_width", C.c_int32),
                ("out_residual", C.c_void_p), ("d_in_residual", C.c_void_p), ("opt", Optimizer), ("m", C.c_void_p),
                ("v", C.c_void_p), ("col_mask", C.c_void_p), ("plan", C.c_void_p),
                ("master_from_slice", C.c_int32)]


class AttnCoreArgs(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("n_subnets", C.c_int32), ("n_seqs", C.c_int32), ("seq_len", C.c_int32),
                ("head_keep", C.c_int32), ("kv_max", C.c_int32), ("d_head", C.c_int32), ("n_heads", C.c_int32),
                ("n_kv_heads", C.c_int32), ("qkv", C.c_void_p), ("out", C.c_void_p), ("lse", C.c_void_p),
                ("d_out", C.c_void_p), ("d_qkv", C.c_void_p), ("delta", C.c_void_p), ("head_idx", C.c_void_p),
                ("kv_pos", C.c_void_p), ("kv_count", C.c_void_p), ("plan", C.c_void_p)]


class Config(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_heads", C.c_int32),
                ("n_kv_heads", C.c_int32), ("d_head", C.c_int32), ("d_ff", C.c_int32), ("ffn_kind", C.c_int32),
                ("n_subnets", C.c_int32), ("ffn_block", C.c_int32), ("ffn_keep", C.c_int32), ("head_keep", C.c_int32),
                ("sample_mode", C.c_int32), ("dtype", C.c_int32), ("tokens", C.c_int32), ("reserved", C.c_int32),
                ("seed", C.c_uint64)]


class Plan:
    """Owner of a twist_plan handle (the shapes of a workload and its cache of encoded tensor maps)."""

    def __init__(self, w):
        cfg = Config(C.sizeof(Config), w.n_layers, w.d_model, w.n_heads, w.n_kv_heads, w.d_head, w.d_ff, w.ffn_kind,
                     w.n_subnets, w.ffn_block, w.ffn_keep, w.head_keep, w.sample_mode, w.dtype, w.tokens, 0, w.seed_mask)
        self.handle = C.c_void_p()
        _check(lib().twist_plan_create(C.byref(cfg), C.byref(self.handle)), "twist_plan_create")

    @property
    def ptr(self) -> int:
        return self.handle.value

    def workspace_bytes(self) -> int:
        n = C.c_size_t(0)
        _check(lib().twist_workspace_bytes(self.handle, C.byref(n)), "twist_workspace_bytes")
        return n.value

    def stats(self):
        """(maps cached, cache hits, cache misses)"""
        a, b, c = C.c_uint64(0), C.c_uint64(0), C.c_uint64(0)
        _check(lib().twist_plan_stats(self.handle, C.byref(a), C.byref(b), C.byref(c)), "twist_plan_stats")
        return a.value, b.value, c.value

    def close(self):
        if self.handle and self.handle.value:
            lib().twist_plan_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class LayerNormArgs(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("n_subnets", C.c_int32), ("tokens", C.c_int32), ("d_model", C.c_int32),
                ("eps", C.c_float), ("lr", C.c_float), ("x", C.c_void_p), ("y", C.c_void_p), ("mean", C.c_void_p),
                ("rstd", C.c_void_p), ("gamma", C.c_void_p), ("beta", C.c_void_p), ("dy", C.c_void_p),
                ("dx", C.c_void_p), ("dx_residual", C.c_void_p), ("dgamma", C.c_void_p), ("dbeta", C.c_void_p),
                ("ws", C.c_void_p), ("ws_bytes", C.c_size_t), ("opt", Optimizer), ("m_gamma", C.c_void_p),
                ("v_gamma", C.c_void_p), ("m_beta", C.c_void_p), ("v_beta", C.c_void_p)]


class RopeArgs(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("n_subnets", C.c_int32), ("tokens", C.c_int32), ("head_keep", C.c_int32),
                ("kv_max", C.c_int32), ("d_head", C.c_int32), ("rot_dims", C.c_int32), ("layout", C.c_int32),
                ("seq_len", C.c_int32), ("in_", C.c_void_p), ("out", C.c_void_p), ("inv_freq", C.c_void_p),
                ("pos", C.c_void_p)]


class KvAppendArgs(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("n_subnets", C.c_int32), ("n_seqs", C.c_int32), ("tokens", C.c_int32),
                ("head_keep", C.c_int32), ("kv_max", C.c_int32), ("d_head", C.c_int32), ("page_size", C.c_int32),
                ("n_pages", C.c_int32), ("max_pages", C.c_int32), ("rot_dims", C.c_int32), ("layout", C.c_int32),
                ("page_stride", C.c_int64), ("q_stride", C.c_int64), ("qkv", C.c_void_p), ("q_out", C.c_void_p),
                ("k_cache", C.c_void_p), ("v_cache", C.c_void_p), ("page_table", C.c_void_p), ("kv_len", C.c_void_p),
                ("new_begin", C.c_void_p), ("new_len", C.c_void_p), ("kv_count", C.c_void_p), ("inv_freq", C.c_void_p)]


class AttnDecodeArgs(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("n_subnets", C.c_int32), ("n_seqs", C.c_int32), ("head_keep", C.c_int32),
                ("kv_max", C.c_int32), ("d_head", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("page_size", C.c_int32), ("n_pages", C.c_int32), ("max_pages", C.c_int32), ("max_len", C.c_int32),
                ("page_stride", C.c_int64), ("q_stride", C.c_int64), ("q", C.c_void_p), ("k_cache", C.c_void_p),
                ("v_cache", C.c_void_p), ("page_table", C.c_void_p), ("kv_len", C.c_void_p), ("head_idx", C.c_void_p),
                ("kv_pos", C.c_void_p), ("out", C.c_void_p), ("lse", C.c_void_p), ("ws", C.c_void_p),
                ("ws_bytes", C.c_size_t)]


class KvAppendQ8Args(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("n_subnets", C.c_int32), ("n_seqs", C.c_int32), ("tokens", C.c_int32),
                ("head_keep", C.c_int32), ("kv_max", C.c_int32), ("d_head", C.c_int32), ("page_size", C.c_int32),
                ("n_pages", C.c_int32), ("max_pages", C.c_int32), ("rot_dims", C.c_int32), ("layout", C.c_int32),
                ("page_stride", C.c_int64), ("q_stride", C.c_int64), ("qkv", C.c_void_p), ("q_out", C.c_void_p),
                ("k_cache", C.c_void_p), ("v_cache", C.c_void_p), ("scales", C.c_void_p), ("page_table", C.c_void_p),
                ("kv_len", C.c_void_p), ("seen", C.c_void_p), ("new_begin", C.c_void_p), ("new_len", C.c_void_p),
                ("kv_count", C.c_void_p), ("inv_freq", C.c_void_p)]


class AttnDecodeQ8Args(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("n_subnets", C.c_int32), ("n_seqs", C.c_int32), ("head_keep", C.c_int32),
                ("kv_max", C.c_int32), ("d_head", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("page_size", C.c_int32), ("n_pages", C.c_int32), ("max_pages", C.c_int32), ("max_len", C.c_int32),
                ("page_stride", C.c_int64), ("q_stride", C.c_int64), ("q", C.c_void_p), ("k_cache", C.c_void_p),
                ("v_cache", C.c_void_p), ("scales", C.c_void_p), ("page_table", C.c_void_p), ("kv_len", C.c_void_p),
                ("head_idx", C.c_void_p), ("kv_pos", C.c_void_p), ("out", C.c_void_p), ("lse", C.c_void_p),
                ("ws", C.c_void_p), ("ws_bytes", C.c_size_t)]


class AttnWeightsArgs(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("n_subnets", C.c_int32), ("n_seqs", C.c_int32), ("head_keep", C.c_int32),
                ("kv_max", C.c_int32), ("d_head", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("page_size", C.c_int32), ("n_pages", C.c_int32), ("max_pages", C.c_int32), ("max_len", C.c_int32),
                ("cache", C.c_int32), ("reserved", C.c_int32), ("page_stride", C.c_int64), ("q_stride", C.c_int64),
                ("q", C.c_void_p), ("lse", C.c_void_p), ("k_cache", C.c_void_p), ("scales", C.c_void_p),
                ("page_table", C.c_void_p), ("kv_len", C.c_void_p), ("new_len", C.c_void_p), ("seen", C.c_void_p),
                ("head_idx", C.c_void_p), ("kv_pos", C.c_void_p), ("prior", C.c_void_p), ("weights", C.c_void_p),
                ("slot_pos", C.c_void_p)]


class AttnCoreWeightsArgs(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("n_subnets", C.c_int32), ("n_seqs", C.c_int32), ("seq_len", C.c_int32),
                ("head_keep", C.c_int32), ("kv_max", C.c_int32), ("d_head", C.c_int32), ("n_heads", C.c_int32),
                ("n_kv_heads", C.c_int32), ("page_size", C.c_int32), ("n_pages", C.c_int32), ("max_pages", C.c_int32),
                ("last_queries", C.c_int32), ("reserved", C.c_int32), ("qkv", C.c_void_p), ("lse", C.c_void_p),
                ("page_table", C.c_void_p), ("new_len", C.c_void_p), ("head_idx", C.c_void_p), ("kv_pos", C.c_void_p),
                ("weights", C.c_void_p), ("slot_pos", C.c_void_p), ("plan", C.c_void_p)]


class KvEvictArgs(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("n_subnets", C.c_int32), ("n_seqs", C.c_int32), ("kv_max", C.c_int32),
                ("d_head", C.c_int32), ("page_size", C.c_int32), ("n_pages", C.c_int32), ("max_pages", C.c_int32),
                ("max_len", C.c_int32), ("recent", C.c_int32), ("cache", C.c_int32), ("reserved", C.c_int32),
                ("page_stride", C.c_int64), ("k_cache", C.c_void_p), ("v_cache", C.c_void_p), ("scales", C.c_void_p),
                ("page_table", C.c_void_p), ("kv_len", C.c_void_p), ("keep", C.c_void_p), ("seen", C.c_void_p),
                ("kv_count", C.c_void_p), ("weights", C.c_void_p), ("slot_pos", C.c_void_p), ("weights_out", C.c_void_p),
                ("slot_pos_out", C.c_void_p), ("ws", C.c_void_p), ("ws_bytes", C.c_size_t)]


_lib_handle = None


def lib() -> C.CDLL:
    """Loads libtwist.so (once).  Fails loudly when it has not been built."""
    global _lib_handle
    if _lib_handle is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2511_03983_b200.build` (there is no fallback)")
        h = C.CDLL(LIB_PATH)
        h.twist_abi_version.restype = C.c_uint32
        h.twist_strerror.restype = C.c_char_p
        h.twist_strerror.argtypes = [C.c_int32]
        h.twist_last_cuda_error.restype = C.c_char_p
        h.twist_device_status.argtypes = [C.POINTER(C.c_int32)]
        h.twist_selftest_wait.argtypes = [C.c_uint64, C.c_void_p]
        h.twist_sample_masks.argtypes = [C.c_uint64, C.c_uint64, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                         C.c_int32, C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p,
                                         C.c_void_p, C.c_void_p]
        h.twist_kv_groups.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                      C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        h.twist_hidden_mask.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]
        h.twist_qkv_col_mask.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                         C.c_void_p, C.c_void_p, C.c_void_p]
        h.twist_plan_create.argtypes = [C.c_void_p, C.c_void_p]
        h.twist_plan_destroy.argtypes = [C.c_void_p]
        h.twist_plan_stats.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        h.twist_workspace_bytes.argtypes = [C.c_void_p, C.c_void_p]
        h.twist_apply_col_mask.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p]
        h.twist_gather_subnets.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p]
        h.twist_aggregate.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_uint32, C.c_void_p]
        h.twist_aggregate_partial.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_uint32,
                                              C.c_void_p]
        h.twist_aggregate_finish.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_uint32, C.c_void_p]
        h.twist_layernorm_workspace_bytes.restype = C.c_size_t
        h.twist_layernorm_workspace_bytes.argtypes = [C.c_int32, C.c_int32, C.c_int32]
        for name in ("twist_subnet_ffn_fwd", "twist_subnet_ffn_bwd", "twist_subnet_attn_proj_fwd",
                     "twist_subnet_attn_proj_bwd", "twist_attn_core_fwd", "twist_attn_core_bwd",
                     "twist_layernorm_fwd", "twist_layernorm_bwd", "twist_rope_fwd", "twist_rope_bwd", "twist_kv_append",
                     "twist_attn_decode", "twist_kv_append_q8", "twist_attn_decode_q8", "twist_attn_weights",
                     "twist_attn_core_weights", "twist_kv_evict"):
            getattr(h, name).argtypes = [C.c_void_p, C.c_void_p]
        h.twist_selftest_decode_quit.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p]
        h.twist_attn_decode_workspace_bytes.restype = C.c_size_t
        h.twist_attn_decode_workspace_bytes.argtypes = [C.c_int32]
        h.twist_kv_evict_workspace_bytes.restype = C.c_size_t
        h.twist_kv_evict_workspace_bytes.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_int64]
        h.twist_mse_workspace_bytes.restype = C.c_size_t
        h.twist_mse_workspace_bytes.argtypes = [C.c_int32]
        h.twist_fused_loss_workspace_bytes.restype = C.c_size_t
        h.twist_fused_loss_workspace_bytes.argtypes = [C.c_int32, C.c_int32, C.c_int32]
        h.twist_mse_fwd_bwd.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32,
                                        C.c_int32, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_size_t,
                                        C.c_void_p]
        h.twist_mse_fwd_bwd_noalloc.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32,
                                                C.c_int32, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p]
        for name in EXPORTS:
            f = getattr(h, name)
            if name not in ("twist_abi_version", "twist_strerror", "twist_last_cuda_error",
                            "twist_mse_workspace_bytes", "twist_fused_loss_workspace_bytes",
                            "twist_layernorm_workspace_bytes", "twist_attn_decode_workspace_bytes",
                            "twist_kv_evict_workspace_bytes"):
                f.restype = C.c_int32
        _lib_handle = h
    return _lib_handle


def _check(status: int, where: str):
    if status != OK:
        h = lib()
        detail = h.twist_strerror(status).decode()
        if status == ERR_CUDA:
            detail += ": " + h.twist_last_cuda_error().decode()
        raise TwistError(status, where, detail)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device tensors must be contiguous CUDA tensors"
    return t.data_ptr()


# The raw handle of the current stream: torch.cuda.current_stream() builds a Stream object first (3.2 us against 0.2 us
# a call, a third of the host time of a small launch).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream() -> int:
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_device())


def _device() -> int:
    """Number of the current device."""
    if _raw_device is None or not torch.cuda.is_initialized():
        return torch.cuda.current_device()
    return _raw_device()


def twist_abi_version() -> int:
    return lib().twist_abi_version()


def twist_device_status() -> int:
    code = C.c_int32(0)
    _check(lib().twist_device_status(C.byref(code)), "twist_device_status")
    return code.value


def twist_selftest_wait(limit_ns: int):
    """Runs the library's bounded waits on barriers nobody arrives at (test / bring-up only); afterwards
    twist_device_status() reports ERR_DEVICE_TIMEOUT once."""
    _check(lib().twist_selftest_wait(limit_ns, _stream()), "twist_selftest_wait")


def twist_sample_masks(seed, rnd, layer_begin, n_layers, kind, n_full, n_subnets, n_sub, common: Sequence[int],
                       sample_mode, idx, cover, pos):
    arr = (C.c_int32 * max(1, len(common)))(*common)
    _check(lib().twist_sample_masks(seed, rnd, layer_begin, n_layers, kind, n_full, n_subnets, n_sub,
                                    C.cast(arr, C.c_void_p) if len(common) else None, len(common), sample_mode,
                                    _ptr(idx), _ptr(cover), _ptr(pos), _stream()), "twist_sample_masks")


def twist_kv_groups(head_idx, n_layers, n_subnets, head_keep, n_heads, n_kv_heads, d_head, kv_idx, kv_count, kv_cols,
                    kv_cover, kv_pos):
    _check(lib().twist_kv_groups(_ptr(head_idx), n_layers, n_subnets, head_keep, n_heads, n_kv_heads, d_head,
                                 _ptr(kv_idx), _ptr(kv_count), _ptr(kv_cols), _ptr(kv_cover), _ptr(kv_pos), _stream()),
           "twist_kv_groups")


def gather_segment(src, dst, dst_master, idx, count, idx_stride, n_keep, block_rows, src_row_offset,
                   dst_subnet_stride, dst_row_offset, n_blocks) -> GatherSegment:
    """Marshals one twist_gather_segment.  src/dst/... may be tensors or raw device addresses (ints).
    n_blocks: blocks in the partitioned range of src (the range idx entries are checked against)."""
    a = lambda v: v if (v is None or isinstance(v, int)) else _ptr(v)
    return GatherSegment(a(src), a(dst), a(dst_master), a(idx), a(count), idx_stride, n_keep, block_rows, n_blocks,
                         src_row_offset, dst_subnet_stride, dst_row_offset)


def twist_gather_subnets(segs: Sequence[GatherSegment], n_subnets, d, dtype):
    arr = (GatherSegment * len(segs))(*segs)
    _check(lib().twist_gather_subnets(C.cast(arr, C.c_void_p), len(segs), n_subnets, d, dtype, _stream()),
           "twist_gather_subnets")


def aggregate_segment(dst, dst_f32, sub, cover, pos, n_full, block_rows, dst_row_offset, sub_subnet_stride,
                      sub_row_offset, n_keep, central=None, central_subnet=0) -> AggregateSegment:
    """Marshals one twist_aggregate_segment.  n_keep: blocks of the segment in a subnet's slice (the range the
    ranks in pos are checked against)."""
    a = lambda v: v if (v is None or isinstance(v, int)) else _ptr(v)
    return AggregateSegment(a(dst), a(dst_f32), a(sub), a(cover), a(pos), n_full, block_rows, dst_row_offset,
                            sub_subnet_stride, sub_row_offset, a(central), central_subnet, n_keep)


def twist_hidden_mask(cover, n_full, block_rows, subnet_begin, n_subnets, mask):
    _check(lib().twist_hidden_mask(_ptr(cover), n_full, block_rows, subnet_begin, n_subnets, _ptr(mask), _stream()),
           "twist_hidden_mask")


def twist_qkv_col_mask(head_cover, kv_cover, n_heads, n_kv_heads, d_head, subnet_begin, n_subnets, mask, count):
    _check(lib().twist_qkv_col_mask(_ptr(head_cover), _ptr(kv_cover), n_heads, n_kv_heads, d_head, subnet_begin,
                                    n_subnets, _ptr(mask), _ptr(count), _stream()), "twist_qkv_col_mask")


def twist_apply_col_mask(in_, mask, out, n_subnets, tokens, width):
    _check(lib().twist_apply_col_mask(_ptr(in_), _ptr(mask), _ptr(out), n_subnets, tokens, width, _stream()),
           "twist_apply_col_mask")


def twist_aggregate(segs: Sequence[AggregateSegment], n_subnets, d, dtype, live_subnets=0xFFFFFFFF):
    arr = (AggregateSegment * len(segs))(*segs)
    _check(lib().twist_aggregate(C.cast(arr, C.c_void_p), len(segs), n_subnets, d, dtype, live_subnets, _stream()),
           "twist_aggregate")


def twist_aggregate_partial(segs: Sequence[AggregateSegment], n_subnets, subnet_begin, d, dtype, live_subnets=0xFFFFFFFF):
    arr = (AggregateSegment * len(segs))(*segs)
    _check(lib().twist_aggregate_partial(C.cast(arr, C.c_void_p), len(segs), n_subnets, subnet_begin, d, dtype,
                                         live_subnets, _stream()), "twist_aggregate_partial")


def twist_aggregate_finish(segs: Sequence[AggregateSegment], n_subnets, d, dtype, live_subnets=0xFFFFFFFF):
    arr = (AggregateSegment * len(segs))(*segs)
    _check(lib().twist_aggregate_finish(C.cast(arr, C.c_void_p), len(segs), n_subnets, d, dtype, live_subnets, _stream()),
           "twist_aggregate_finish")


def _ws_bytes(ws) -> int:
    return 0 if ws is None else ws.numel() * ws.element_size()


def _plan_ptr(plan) -> Optional[int]:
    return None if plan is None else plan.ptr


def ffn_args(ffn_kind, dtype, n_subnets, tokens, d_model, f_sub, out_scale, lr=0.0, opt: Optional[Optimizer] = None,
             plan: Optional["Plan"] = None, master_from_slice: bool = False, **t) -> FfnArgs:
    """Marshals twist_ffn_args.  tgt / loss / loss_ws request the fused loss of the forward call; hidden_mask
    (uint8 [S][f_sub]) the activation mask of Masked TwIST."""
    names = ["x", "w_gu", "w_down", "w_gu_master", "w_down_master", "pre", "hh", "y", "dy", "dpre", "dx", "dw_gu",
             "dw_down", "tgt", "loss", "loss_ws"]
    moments = ["m_gu", "v_gu", "m_down", "v_down"]
    unknown = set(t) - set(names) - {"y_residual", "dx_residual", "hidden_mask"} - set(moments)
    assert not unknown, unknown
    a = FfnArgs(ffn_kind, dtype, n_subnets, tokens, d_model, f_sub, out_scale, lr, *[_ptr(t.get(n)) for n in names],
                _ws_bytes(t.get("loss_ws")), _ptr(t.get("y_residual")), _ptr(t.get("dx_residual")),
                opt if opt is not None else Optimizer(), *[_ptr(t.get(n)) for n in moments],
                _ptr(t.get("hidden_mask")), _plan_ptr(plan), int(master_from_slice))
    a._keepalive = list(t.values()) + [plan]      # the struct holds raw addresses: keep their owners alive with it
    return a


def twist_subnet_ffn_fwd(a: FfnArgs):
    _check(lib().twist_subnet_ffn_fwd(C.byref(a), _stream()), "twist_subnet_ffn_fwd")


def twist_subnet_ffn_bwd(a: FfnArgs):
    _check(lib().twist_subnet_ffn_bwd(C.byref(a), _stream()), "twist_subnet_ffn_bwd")


def proj_args(which, dtype, n_subnets, tokens, d_model, n, out_scale, lr=0.0, seg_begin=0, seg_width=0,
              opt: Optional[Optimizer] = None, plan: Optional["Plan"] = None, master_from_slice: bool = False,
              **t) -> ProjArgs:
    """Marshals twist_proj_args.  tgt / loss / loss_ws (and the optional column mask valid_cols,
    seg_begin, seg_width) request the fused loss of the forward call."""
    names = ["in_", "w", "w_master", "out", "d_out", "d_in", "dw", "tgt", "loss", "loss_ws"]
    unknown = set(t) - set(names) - {"valid_cols", "out_residual", "d_in_residual", "m", "v", "col_mask"}
    assert not unknown, unknown
    a = ProjArgs(which, dtype, n_subnets, tokens, d_model, n, out_scale, lr, *[_ptr(t.get(n)) for n in names],
                 _ws_bytes(t.get("loss_ws")), _ptr(t.get("valid_cols")), seg_begin, seg_width,
                 _ptr(t.get("out_residual")), _ptr(t.get("d_in_residual")), opt if opt is not None else Optimizer(),
                 _ptr(t.get("m")), _ptr(t.get("v")), _ptr(t.get("col_mask")), _plan_ptr(plan), int(master_from_slice))
    a._keepalive = list(t.values()) + [plan]
    return a


def twist_subnet_attn_proj_fwd(a: ProjArgs):
    _check(lib().twist_subnet_attn_proj_fwd(C.byref(a), _stream()), "twist_subnet_attn_proj_fwd")


def twist_subnet_attn_proj_bwd(a: ProjArgs):
    _check(lib().twist_subnet_attn_proj_bwd(C.byref(a), _stream()), "twist_subnet_attn_proj_bwd")


def attn_core_args(dtype, n_subnets, n_seqs, seq_len, head_keep, kv_max, d_head, n_heads=0, n_kv_heads=0,
                   plan: Optional["Plan"] = None, **t) -> AttnCoreArgs:
    names = ["qkv", "out", "lse", "d_out", "d_qkv", "delta", "head_idx", "kv_pos", "kv_count"]
    unknown = set(t) - set(names)
    assert not unknown, unknown
    a = AttnCoreArgs(dtype, n_subnets, n_seqs, seq_len, head_keep, kv_max, d_head, n_heads, n_kv_heads,
                     *[_ptr(t.get(n)) for n in names], _plan_ptr(plan))
    a._keepalive = list(t.values()) + [plan]
    return a


def twist_attn_core_fwd(a: AttnCoreArgs):
    _check(lib().twist_attn_core_fwd(C.byref(a), _stream()), "twist_attn_core_fwd")


def twist_attn_core_bwd(a: AttnCoreArgs):
    _check(lib().twist_attn_core_bwd(C.byref(a), _stream()), "twist_attn_core_bwd")


def _tensor(name: str, t: torch.Tensor, dtype: torch.dtype, numel: int, dev: int) -> int:
    """Address of a dense tensor of the given type and size on the current device (the call runs on its current stream)."""
    if t.dtype is not dtype or t.numel() != numel or not t.is_contiguous():
        raise ValueError("%s: expected %d contiguous elements of %s, got %s of %s" % (name, numel, dtype, tuple(t.shape), t.dtype))
    if t.get_device() != dev:
        _elsewhere(name, t, dev)
    return t.data_ptr()


def _addresses(dev: int, *specs):
    """Addresses (0 for None) of tensors given as (name, tensor, dtype, numel), all dense and on the current device."""
    out = []
    for name, t, dtype, numel in specs:
        if t is None:
            out.append(0)
        elif t.dtype is dtype and t.numel() == numel and t.get_device() == dev and t.is_contiguous():
            out.append(t.data_ptr())
        else:
            out.append(_tensor(name, t, dtype, numel, dev))
    return out


def _elsewhere(name: str, t: torch.Tensor, dev: int):
    raise ValueError("%s: tensor on %s, current device is cuda:%d" % (name, t.device, dev))


def _rows(name: str, t: torch.Tensor, n_subnets: int, rows: int, width: int) -> int:
    """Distance of the rows of a [S][rows][width] view whose rows lie evenly spaced (columns of a wider buffer)."""
    if t.dtype is not torch.bfloat16 or t.shape != (n_subnets, rows, width):
        raise ValueError("%s: expected bf16 [%d][%d][%d], got %s of %s" % (name, n_subnets, rows, width, tuple(t.shape), t.dtype))
    s0, s1, s2 = t.stride()
    stride = s1 if rows > 1 else (s0 if n_subnets > 1 else width)
    if s2 != 1 or (n_subnets > 1 and s0 != rows * stride):
        raise ValueError("%s: rows are not evenly spaced (strides %s)" % (name, (s0, s1, s2)))
    return stride


def _cache(k: torch.Tensor, v: torch.Tensor, kv_max: int, d_head: int, dtype: torch.dtype = torch.bfloat16):
    """(page_size, n_pages, page_stride) of a paged cache [n_pages][kv_max][page_size][d_head]; pages may be spaced."""
    shape = k.shape
    if shape != v.shape or len(shape) != 4 or shape[1] != kv_max or shape[3] != d_head or k.dtype is not dtype or v.dtype is not dtype:
        raise ValueError("k_cache / v_cache: expected %s [pages][%d][page_size][%d], got %s and %s of %s and %s" % (
            dtype, kv_max, d_head, tuple(shape), tuple(v.shape), k.dtype, v.dtype))
    n, _, page, _ = shape
    strides = k.stride()
    if strides != v.stride() or strides[1:] != (page * d_head, d_head, 1):
        raise ValueError("k_cache / v_cache: a page must be dense and both spaced alike (strides %s and %s)" % (strides, v.stride()))
    return page, n, strides[0] if n > 1 else max(strides[0], kv_max * page * d_head)


def _cache_kind(k: torch.Tensor, scales: Optional[torch.Tensor]) -> int:
    """CACHE_BF16 or CACHE_E4M3, by the cache's type; an 8-bit cache has scales, a bf16 cache none."""
    kind = CACHE_E4M3 if k.dtype is torch.float8_e4m3fn else CACHE_BF16
    if (kind == CACHE_E4M3) != (scales is not None):
        raise ValueError("scales: an e4m3 cache has them, a bf16 cache has none (cache of %s)" % k.dtype)
    return kind


# The argument structs of the per-token calls are packed in one go (field by field costs 1 us a call more), and their
# tensors are checked in one expression; _tensor names the one that is wrong when it fails.
_ROPE_PACK = struct.Struct("9i4x4Q")
_APPEND_PACK = struct.Struct("12i2q10Q")
_DECODE_PACK = struct.Struct("12i2q11Q")
_Q8_PACK = struct.Struct("12i2q12Q")
_WEIGHTS_PACK = struct.Struct("14i2q13Q")
_EVICT_PACK = struct.Struct("12iq14Q")
_CORE_WEIGHTS_PACK = struct.Struct("14i9Q")
assert (_ROPE_PACK.size, _APPEND_PACK.size, _DECODE_PACK.size) == (C.sizeof(RopeArgs), C.sizeof(KvAppendArgs), C.sizeof(AttnDecodeArgs))
assert (_Q8_PACK.size, _Q8_PACK.size, _WEIGHTS_PACK.size, _EVICT_PACK.size, _CORE_WEIGHTS_PACK.size) == (
    C.sizeof(KvAppendQ8Args), C.sizeof(AttnDecodeQ8Args), C.sizeof(AttnWeightsArgs), C.sizeof(KvEvictArgs), C.sizeof(AttnCoreWeightsArgs))


def rope_args(dtype, n_subnets, tokens, head_keep, kv_max, d_head, rot_dims, seq_len=0, layout=ROPE_HALF, *, in_, out,
              inv_freq, pos=None) -> RopeArgs:
    """Marshals twist_rope_args.  in_, out: bf16 [S][T][(head_keep + 2 kv_max) d_head] (out may be in_); inv_freq: fp64
    [rot_dims / 2]; pos: int32 [S][T], or None for position t % seq_len."""
    dev = _device()
    n, bf = n_subnets * tokens * (head_keep + 2 * kv_max) * d_head, torch.bfloat16
    if not (in_.dtype is bf and in_.numel() == n and in_.is_contiguous() and in_.get_device() == dev
            and out.dtype is bf and out.numel() == n and out.is_contiguous() and out.get_device() == dev
            and inv_freq.dtype is torch.float64 and inv_freq.numel() == rot_dims // 2 and inv_freq.is_contiguous()
            and inv_freq.get_device() == dev):
        _tensor("in_", in_, bf, n, dev)
        _tensor("out", out, bf, n, dev)
        _tensor("inv_freq", inv_freq, torch.float64, rot_dims // 2, dev)
    a = RopeArgs.from_buffer_copy(_ROPE_PACK.pack(
        dtype, n_subnets, tokens, head_keep, kv_max, d_head, rot_dims, layout, seq_len, in_.data_ptr(), out.data_ptr(),
        inv_freq.data_ptr(), 0 if pos is None else _tensor("pos", pos, torch.int32, n_subnets * tokens, dev)))
    a._keepalive = (in_, out, inv_freq, pos)
    return a


def twist_rope_fwd(a: RopeArgs):
    _check(lib().twist_rope_fwd(C.byref(a), _stream()), "twist_rope_fwd")


def twist_rope_bwd(a: RopeArgs):
    _check(lib().twist_rope_bwd(C.byref(a), _stream()), "twist_rope_bwd")


def kv_append_args(dtype, n_subnets, n_seqs, tokens, head_keep, kv_max, d_head, rot_dims=0, layout=ROPE_HALF, *, qkv,
                   k_cache, v_cache, page_table, kv_len, q_out=None, new_begin=None, new_len=None, kv_count=None,
                   inv_freq=None) -> KvAppendArgs:
    """Marshals twist_kv_append_args.  qkv: bf16 [S][T][(head_keep + 2 kv_max) d_head]; k_cache, v_cache: bf16
    [n_pages][kv_max][page_size][d_head], pages evenly spaced (one buffer may hold both); page_table: int32
    [S][n_seqs][max_pages]; kv_len: int32 [S][n_seqs], the new tokens included; q_out: bf16 [S][T][head_keep d_head], rows
    evenly spaced (qkv[..., :head_keep * d_head] rotates Q in place)."""
    dev = _device()
    i32, bf = torch.int32, torch.bfloat16
    page, n_pages, stride = _cache(k_cache, v_cache, kv_max, d_head)
    if k_cache.get_device() != dev or v_cache.get_device() != dev or (q_out is not None and q_out.get_device() != dev):
        _elsewhere("k_cache / v_cache / q_out", k_cache, dev)
    seqs, n = n_subnets * n_seqs, n_subnets * tokens * (head_keep + 2 * kv_max) * d_head
    max_pages = page_table.shape[-1]
    if not (qkv.dtype is bf and qkv.numel() == n and qkv.is_contiguous() and qkv.get_device() == dev
            and page_table.dtype is i32 and page_table.numel() == seqs * max_pages and page_table.is_contiguous()
            and page_table.get_device() == dev
            and kv_len.dtype is i32 and kv_len.numel() == seqs and kv_len.is_contiguous() and kv_len.get_device() == dev):
        _tensor("qkv", qkv, bf, n, dev)
        _tensor("page_table", page_table, i32, seqs * max_pages, dev)
        _tensor("kv_len", kv_len, i32, seqs, dev)
    a = KvAppendArgs.from_buffer_copy(_APPEND_PACK.pack(
        dtype, n_subnets, n_seqs, tokens, head_keep, kv_max, d_head, page, n_pages, max_pages, rot_dims, layout, stride,
        0 if q_out is None else _rows("q_out", q_out, n_subnets, tokens, head_keep * d_head), qkv.data_ptr(),
        0 if q_out is None else q_out.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), page_table.data_ptr(), kv_len.data_ptr(),
        0 if new_begin is None else _tensor("new_begin", new_begin, i32, n_subnets * (n_seqs + 1), dev),
        0 if new_len is None else _tensor("new_len", new_len, i32, seqs, dev),
        0 if kv_count is None else _tensor("kv_count", kv_count, i32, n_subnets, dev),
        0 if inv_freq is None else _tensor("inv_freq", inv_freq, torch.float64, rot_dims // 2, dev)))
    a._keepalive = (qkv, q_out, k_cache, v_cache, page_table, kv_len, new_begin, new_len, kv_count, inv_freq)
    return a


def twist_kv_append(a: KvAppendArgs):
    _check(lib().twist_kv_append(C.byref(a), _stream()), "twist_kv_append")


def attn_decode_args(dtype, n_subnets, n_seqs, head_keep, kv_max, d_head, n_heads=0, n_kv_heads=0, max_len=0, *, q, k_cache,
                     v_cache, page_table, kv_len, out, ws, head_idx=None, kv_pos=None, lse=None) -> AttnDecodeArgs:
    """Marshals twist_attn_decode_args.  q: bf16 [S][n_seqs][head_keep d_head], rows evenly spaced; the cache as in
    kv_append_args; head_idx int32 [S][head_keep] and kv_pos int32 [S][n_kv_heads] for grouped-query sharing; out bf16
    [S][n_seqs][head_keep d_head]; lse fp32 [S][head_keep][n_seqs]; ws: scratch of at least
    twist_attn_decode_workspace_bytes(d_head) bytes."""
    dev = _device()
    i32, bf = torch.int32, torch.bfloat16
    page, n_pages, stride = _cache(k_cache, v_cache, kv_max, d_head)
    if k_cache.get_device() != dev or v_cache.get_device() != dev or q.get_device() != dev or ws.get_device() != dev:
        _elsewhere("k_cache / v_cache / q / ws", k_cache, dev)
    seqs, width = n_subnets * n_seqs, head_keep * d_head
    max_pages = page_table.shape[-1]
    if not (page_table.dtype is i32 and page_table.numel() == seqs * max_pages and page_table.is_contiguous()
            and page_table.get_device() == dev
            and kv_len.dtype is i32 and kv_len.numel() == seqs and kv_len.is_contiguous() and kv_len.get_device() == dev
            and out.dtype is bf and out.numel() == seqs * width and out.is_contiguous() and out.get_device() == dev
            and (lse is None or (lse.dtype is torch.float32 and lse.numel() == seqs * head_keep and lse.is_contiguous()
                                 and lse.get_device() == dev))
            and (head_idx is None or (head_idx.dtype is i32 and head_idx.numel() == n_subnets * head_keep
                                      and head_idx.is_contiguous() and head_idx.get_device() == dev))
            and (kv_pos is None or (kv_pos.dtype is i32 and kv_pos.numel() == n_subnets * n_kv_heads
                                    and kv_pos.is_contiguous() and kv_pos.get_device() == dev))):
        _tensor("page_table", page_table, i32, seqs * max_pages, dev)
        _tensor("kv_len", kv_len, i32, seqs, dev)
        _tensor("out", out, bf, seqs * width, dev)
        for name, t, dtype_, n in (("lse", lse, torch.float32, seqs * head_keep), ("head_idx", head_idx, i32, n_subnets * head_keep),
                                   ("kv_pos", kv_pos, i32, n_subnets * n_kv_heads)):
            if t is not None:
                _tensor(name, t, dtype_, n, dev)
    a = AttnDecodeArgs.from_buffer_copy(_DECODE_PACK.pack(
        dtype, n_subnets, n_seqs, head_keep, kv_max, d_head, n_heads, n_kv_heads, page, n_pages, max_pages, max_len, stride,
        _rows("q", q, n_subnets, n_seqs, width), q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), page_table.data_ptr(),
        kv_len.data_ptr(), 0 if head_idx is None else head_idx.data_ptr(), 0 if kv_pos is None else kv_pos.data_ptr(),
        out.data_ptr(), 0 if lse is None else lse.data_ptr(), ws.data_ptr(),
        ws.numel() * ws.element_size()))
    a._keepalive = (q, k_cache, v_cache, page_table, kv_len, out, ws, head_idx, kv_pos, lse)
    return a


def twist_attn_decode_workspace_bytes(d_head: int) -> int:
    return lib().twist_attn_decode_workspace_bytes(d_head)


def twist_attn_decode(a: AttnDecodeArgs):
    _check(lib().twist_attn_decode(C.byref(a), _stream()), "twist_attn_decode")


def kv_append_q8_args(dtype, n_subnets, n_seqs, tokens, head_keep, kv_max, d_head, rot_dims=0, layout=ROPE_HALF, *, qkv,
                      k_cache, v_cache, scales, page_table, kv_len, seen=None, q_out=None, new_begin=None, new_len=None,
                      kv_count=None, inv_freq=None) -> KvAppendQ8Args:
    """Marshals twist_kv_append_q8_args.  As kv_append_args, but k_cache, v_cache: torch.float8_e4m3fn, scales: fp32
    [n_pages][kv_max][page_size / 16][2]; seen: int32 [S][n_seqs], tokens of the sequence so far (None: kv_len)."""
    dev = _device()
    i32, bf = torch.int32, torch.bfloat16
    page, n_pages, stride = _cache(k_cache, v_cache, kv_max, d_head, torch.float8_e4m3fn)
    if k_cache.get_device() != dev or v_cache.get_device() != dev or (q_out is not None and q_out.get_device() != dev):
        _elsewhere("k_cache / v_cache / q_out", k_cache, dev)
    seqs, max_pages, f32 = n_subnets * n_seqs, page_table.shape[-1], torch.float32
    at_qkv, at_scales, at_table, at_len, at_seen, at_begin, at_new, at_count, at_freq = _addresses(
        dev, ("qkv", qkv, bf, n_subnets * tokens * (head_keep + 2 * kv_max) * d_head), ("scales", scales, f32, n_pages * kv_max * (page // 16) * 2),
        ("page_table", page_table, i32, seqs * max_pages), ("kv_len", kv_len, i32, seqs), ("seen", seen, i32, seqs),
        ("new_begin", new_begin, i32, n_subnets * (n_seqs + 1)), ("new_len", new_len, i32, seqs), ("kv_count", kv_count, i32, n_subnets),
        ("inv_freq", inv_freq, torch.float64, rot_dims // 2))
    a = KvAppendQ8Args.from_buffer_copy(_Q8_PACK.pack(
        dtype, n_subnets, n_seqs, tokens, head_keep, kv_max, d_head, page, n_pages, max_pages, rot_dims, layout, stride,
        0 if q_out is None else _rows("q_out", q_out, n_subnets, tokens, head_keep * d_head), at_qkv,
        0 if q_out is None else q_out.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), at_scales, at_table, at_len, at_seen, at_begin,
        at_new, at_count, at_freq))
    a._keepalive = (qkv, q_out, k_cache, v_cache, scales, page_table, kv_len, seen, new_begin, new_len, kv_count, inv_freq)
    return a


def twist_kv_append_q8(a: KvAppendQ8Args):
    _check(lib().twist_kv_append_q8(C.byref(a), _stream()), "twist_kv_append_q8")


def attn_decode_q8_args(dtype, n_subnets, n_seqs, head_keep, kv_max, d_head, n_heads=0, n_kv_heads=0, max_len=0, *, q, k_cache,
                        v_cache, scales, page_table, kv_len, out, ws, head_idx=None, kv_pos=None, lse=None) -> AttnDecodeQ8Args:
    """Marshals twist_attn_decode_q8_args.  As attn_decode_args, but k_cache, v_cache: torch.float8_e4m3fn, scales: fp32
    [n_pages][kv_max][page_size / 16][2]."""
    dev = _device()
    i32, bf = torch.int32, torch.bfloat16
    page, n_pages, stride = _cache(k_cache, v_cache, kv_max, d_head, torch.float8_e4m3fn)
    if k_cache.get_device() != dev or v_cache.get_device() != dev or q.get_device() != dev or ws.get_device() != dev:
        _elsewhere("k_cache / v_cache / q / ws", k_cache, dev)
    seqs, width, max_pages, f32 = n_subnets * n_seqs, head_keep * d_head, page_table.shape[-1], torch.float32
    at_scales, at_table, at_len, at_heads, at_pos, at_out, at_lse = _addresses(
        dev, ("scales", scales, f32, n_pages * kv_max * (page // 16) * 2), ("page_table", page_table, i32, seqs * max_pages),
        ("kv_len", kv_len, i32, seqs), ("head_idx", head_idx, i32, n_subnets * head_keep), ("kv_pos", kv_pos, i32, n_subnets * n_kv_heads),
        ("out", out, bf, seqs * width), ("lse", lse, f32, seqs * head_keep))
    a = AttnDecodeQ8Args.from_buffer_copy(_Q8_PACK.pack(
        dtype, n_subnets, n_seqs, head_keep, kv_max, d_head, n_heads, n_kv_heads, page, n_pages, max_pages, max_len, stride,
        _rows("q", q, n_subnets, n_seqs, width), q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), at_scales, at_table, at_len, at_heads,
        at_pos, at_out, at_lse, ws.data_ptr(), ws.numel() * ws.element_size()))
    a._keepalive = (q, k_cache, v_cache, scales, page_table, kv_len, out, ws, head_idx, kv_pos, lse)
    return a


def twist_attn_decode_q8(a: AttnDecodeQ8Args):
    _check(lib().twist_attn_decode_q8(C.byref(a), _stream()), "twist_attn_decode_q8")


def twist_selftest_decode_quit(a: AttnDecodeQ8Args, every: int, tile: int):
    """The decode call in which every `every`-th warp gives up before tile `tile` of an item (for tests)."""
    _check(lib().twist_selftest_decode_quit(C.byref(a), every, tile, _stream()), "twist_selftest_decode_quit")


def attn_weights_args(dtype, n_subnets, n_seqs, head_keep, kv_max, d_head, n_heads=0, n_kv_heads=0, max_len=0, *, q, lse, k_cache,
                      page_table, kv_len, weights, scales=None, prior=None, slot_pos=None, new_len=None, seen=None, head_idx=None,
                      kv_pos=None) -> AttnWeightsArgs:
    """Marshals twist_attn_weights_args.  q, lse, k_cache, page_table, kv_len, head_idx, kv_pos as given to the decode call
    (k_cache bf16, or float8_e4m3fn with its scales); prior, weights: fp32 [n_pages][kv_max][page_size] (prior may be
    weights, None: zeros); slot_pos: int32, the same shape; new_len, seen: int32 [S][n_seqs] (None: 1 each, kv_len)."""
    dev = _device()
    i32, f32 = torch.int32, torch.float32
    kind = _cache_kind(k_cache, scales)
    page, n_pages, stride = _cache(k_cache, k_cache, kv_max, d_head, k_cache.dtype if kind == CACHE_E4M3 else torch.bfloat16)
    if k_cache.get_device() != dev or q.get_device() != dev:
        _elsewhere("k_cache / q", k_cache, dev)
    seqs, max_pages, slots = n_subnets * n_seqs, page_table.shape[-1], n_pages * kv_max * page
    at = _addresses(
        dev, ("lse", lse, f32, seqs * head_keep), ("scales", scales, f32, n_pages * kv_max * (page // 16) * 2),
        ("page_table", page_table, i32, seqs * max_pages), ("kv_len", kv_len, i32, seqs), ("new_len", new_len, i32, seqs), ("seen", seen, i32, seqs),
        ("head_idx", head_idx, i32, n_subnets * head_keep), ("kv_pos", kv_pos, i32, n_subnets * n_kv_heads), ("prior", prior, f32, slots),
        ("weights", weights, f32, slots), ("slot_pos", slot_pos, i32, slots))
    a = AttnWeightsArgs.from_buffer_copy(_WEIGHTS_PACK.pack(
        dtype, n_subnets, n_seqs, head_keep, kv_max, d_head, n_heads, n_kv_heads, page, n_pages, max_pages, max_len, kind, 0, stride,
        _rows("q", q, n_subnets, n_seqs, head_keep * d_head), q.data_ptr(), at[0], k_cache.data_ptr(), *at[1:]))
    a._keepalive = (q, lse, k_cache, scales, page_table, kv_len, new_len, seen, head_idx, kv_pos, prior, weights, slot_pos)
    return a


def twist_attn_weights(a: AttnWeightsArgs):
    _check(lib().twist_attn_weights(C.byref(a), _stream()), "twist_attn_weights")


def attn_core_weights_args(dtype, n_subnets, n_seqs, seq_len, head_keep, kv_max, d_head, n_heads=0, n_kv_heads=0, last_queries=0, *,
                           qkv, lse, page_table, weights, slot_pos=None, new_len=None, head_idx=None, kv_pos=None,
                           plan: Optional["Plan"] = None) -> AttnCoreWeightsArgs:
    """Marshals twist_attn_core_weights_args.  qkv, lse, head_idx, kv_pos as given to the attention core; weights fp32 and
    slot_pos int32 [n_pages][kv_max][page_size]; page_table: int32 [S][n_seqs][max_pages]; new_len: int32 [S][n_seqs]."""
    dev = _device()
    i32, f32 = torch.int32, torch.float32
    if weights.dim() != 3 or weights.shape[1] != kv_max:
        raise ValueError("weights: expected fp32 [pages][%d][page_size], got %s" % (kv_max, tuple(weights.shape)))
    n_pages, _, page = weights.shape
    seqs, max_pages, tokens = n_subnets * n_seqs, page_table.shape[-1], n_subnets * n_seqs * seq_len
    at = _addresses(
        dev, ("qkv", qkv, torch.bfloat16, tokens * (head_keep + 2 * kv_max) * d_head), ("lse", lse, f32, tokens * head_keep),
        ("page_table", page_table, i32, seqs * max_pages), ("new_len", new_len, i32, seqs), ("head_idx", head_idx, i32, n_subnets * head_keep),
        ("kv_pos", kv_pos, i32, n_subnets * n_kv_heads), ("weights", weights, f32, n_pages * kv_max * page),
        ("slot_pos", slot_pos, i32, n_pages * kv_max * page))
    a = AttnCoreWeightsArgs.from_buffer_copy(_CORE_WEIGHTS_PACK.pack(
        dtype, n_subnets, n_seqs, seq_len, head_keep, kv_max, d_head, n_heads, n_kv_heads, page, n_pages, max_pages, last_queries, 0, *at,
        _plan_ptr(plan) or 0))
    a._keepalive = (qkv, lse, page_table, new_len, head_idx, kv_pos, weights, slot_pos, plan)
    return a


def twist_attn_core_weights(a: AttnCoreWeightsArgs):
    _check(lib().twist_attn_core_weights(C.byref(a), _stream()), "twist_attn_core_weights")


def kv_evict_args(dtype, n_subnets, n_seqs, kv_max, d_head, recent, max_len=0, *, k_cache, v_cache, page_table, kv_len, keep, weights,
                  slot_pos, ws, scales=None, seen=None, kv_count=None, weights_out=None, slot_pos_out=None) -> KvEvictArgs:
    """Marshals twist_kv_evict_args.  k_cache, v_cache: bf16, or float8_e4m3fn with their scales; kv_len, keep, seen: int32
    [S][n_seqs]; weights fp32 and slot_pos int32 [n_pages][kv_max][page_size], written in place or to weights_out,
    slot_pos_out; ws: scratch of at least twist_kv_evict_workspace_bytes(S, n_seqs, kv_max, max_len) bytes (max_len 0: the
    table's room)."""
    dev = _device()
    i32, f32 = torch.int32, torch.float32
    kind = _cache_kind(k_cache, scales)
    page, n_pages, stride = _cache(k_cache, v_cache, kv_max, d_head, torch.float8_e4m3fn if kind == CACHE_E4M3 else torch.bfloat16)
    if k_cache.get_device() != dev or v_cache.get_device() != dev or ws.get_device() != dev:
        _elsewhere("k_cache / v_cache / ws", k_cache, dev)
    seqs, max_pages, slots = n_subnets * n_seqs, page_table.shape[-1], n_pages * kv_max * page
    weights_out = weights if weights_out is None else weights_out
    slot_pos_out = slot_pos if slot_pos_out is None else slot_pos_out
    at = _addresses(
        dev, ("scales", scales, f32, n_pages * kv_max * (page // 16) * 2), ("page_table", page_table, i32, seqs * max_pages),
        ("kv_len", kv_len, i32, seqs), ("keep", keep, i32, seqs), ("seen", seen, i32, seqs), ("kv_count", kv_count, i32, n_subnets),
        ("weights", weights, f32, slots), ("slot_pos", slot_pos, i32, slots), ("weights_out", weights_out, f32, slots),
        ("slot_pos_out", slot_pos_out, i32, slots))
    a = KvEvictArgs.from_buffer_copy(_EVICT_PACK.pack(
        dtype, n_subnets, n_seqs, kv_max, d_head, page, n_pages, max_pages, max_len, recent, kind, 0, stride, k_cache.data_ptr(),
        v_cache.data_ptr(), *at, ws.data_ptr(), ws.numel() * ws.element_size()))
    a._keepalive = (k_cache, v_cache, scales, page_table, kv_len, keep, seen, kv_count, weights, slot_pos, weights_out, slot_pos_out, ws)
    return a


def twist_kv_evict_workspace_bytes(n_subnets: int, n_seqs: int, kv_max: int, max_len: int) -> int:
    return lib().twist_kv_evict_workspace_bytes(n_subnets, n_seqs, kv_max, max_len)


def twist_kv_evict(a: KvEvictArgs):
    _check(lib().twist_kv_evict(C.byref(a), _stream()), "twist_kv_evict")


def layernorm_args(dtype, n_subnets, tokens, d_model, eps, lr=0.0, opt: Optional[Optimizer] = None, **t) -> LayerNormArgs:
    """Marshals twist_layernorm_args (tensors by keyword: x, y, mean, rstd, gamma, beta, dy, dx, dx_residual,
    dgamma, dbeta, ws, m_gamma, v_gamma, m_beta, v_beta)."""
    names = ["x", "y", "mean", "rstd", "gamma", "beta", "dy", "dx", "dx_residual", "dgamma", "dbeta", "ws"]
    moments = ["m_gamma", "v_gamma", "m_beta", "v_beta"]
    unknown = set(t) - set(names) - set(moments)
    assert not unknown, unknown
    a = LayerNormArgs(dtype, n_subnets, tokens, d_model, eps, lr, *[_ptr(t.get(n)) for n in names],
                      _ws_bytes(t.get("ws")), opt if opt is not None else Optimizer(), *[_ptr(t.get(n)) for n in moments])
    a._keepalive = list(t.values())
    return a


def twist_layernorm_workspace_bytes(n_subnets: int, tokens: int, d_model: int) -> int:
    return lib().twist_layernorm_workspace_bytes(n_subnets, tokens, d_model)


def twist_layernorm_fwd(a: LayerNormArgs):
    _check(lib().twist_layernorm_fwd(C.byref(a), _stream()), "twist_layernorm_fwd")


def twist_layernorm_bwd(a: LayerNormArgs):
    _check(lib().twist_layernorm_bwd(C.byref(a), _stream()), "twist_layernorm_bwd")


def twist_mse_workspace_bytes(n_subnets: int) -> int:
    return lib().twist_mse_workspace_bytes(n_subnets)


def twist_fused_loss_workspace_bytes(n_subnets: int, tokens: int, width: int) -> int:
    return lib().twist_fused_loss_workspace_bytes(n_subnets, tokens, width)


def twist_mse_fwd_bwd(y, tgt, dy, loss, n_subnets, tokens, width, valid_cols, seg_begin, seg_width, dtype, ws):
    _check(lib().twist_mse_fwd_bwd(_ptr(y), _ptr(tgt), _ptr(dy), _ptr(loss), n_subnets, tokens, width,
                                   _ptr(valid_cols), seg_begin, seg_width, dtype, _ptr(ws),
                                   ws.numel() * ws.element_size(), _stream()),
           "twist_mse_fwd_bwd")


def twist_mse_fwd_bwd_noalloc(y, tgt, dy, loss, n_subnets, tokens, width, valid_cols, seg_begin, seg_width, dtype):
    """Loss and gradient like twist_mse_fwd_bwd, but with the library's built-in scratch: for callers
    that must not (or cannot) allocate device memory.  At most 32 subnets; calls must not overlap on
    the GPU; make the first call on a device outside stream capture."""
    _check(lib().twist_mse_fwd_bwd_noalloc(_ptr(y), _ptr(tgt), _ptr(dy), _ptr(loss), n_subnets, tokens, width,
                                           _ptr(valid_cols), seg_begin, seg_width, dtype, _stream()),
           "twist_mse_fwd_bwd_noalloc")

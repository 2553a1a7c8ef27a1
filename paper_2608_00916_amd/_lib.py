"""ctypes binding of libmoe.so (the C ABI of include/moe.h).

Argument marshalling only: every step of the block runs in the library's HIP
kernels.  Loading fails loudly if the library has not been built; there is no
fallback implementation.
"""
from __future__ import annotations

import ctypes
import os

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libmoe.so")

MOE_OK = 0
MOE_ERR_ARG = -1
MOE_ERR_SHAPE = -2
MOE_ERR_ALIGN = -3
MOE_ERR_WORKSPACE = -4
MOE_ERR_HIP = -5
MOE_MAX_EXPERTS = 256
MOE_MAX_TOPK = 32
MOE_F_MASK = 1
MOE_F_DW_FP32 = 2
MOE_F_RECOMPUTE = 4
MOE_F_OUT_FP32 = 8
MOE_F_CAUSAL = 16
MOE_F_LOGITS_FP32 = 32
MOE_I8_MAX_K = 131072
MOE_NORM_MAX_H = 32768
MOE_DECODE_MAX_T = 64
MOE_SAMPLE_MAX_V = 1 << 20
MOE_NOALLOC_SCRATCH_BYTES = 64 << 20

EXPORTS = (
    "moe_saved_bytes", "moe_fwd_workspace_bytes", "moe_bwd_workspace_bytes",
    "moe_saved_views", "moe_fwd", "moe_fwd_noalloc", "moe_bwd", "moe_infer_workspace_bytes", "moe_infer",
    "moe_lora_saved_bytes", "moe_lora_workspace_bytes", "moe_lora_fwd", "moe_lora_bwd",
    "moe_experts_saved_bytes", "moe_experts_workspace_bytes",
    "moe_experts_saved_views", "moe_experts_fwd", "moe_experts_bwd",
    "moe_i8_quant_rows", "moe_i8_quant_weight", "moe_i8_matmul", "moe_i8_linear_workspace_bytes", "moe_i8_linear",
    "moe_experts_i8_workspace_bytes", "moe_experts_i8", "moe_infer_i8_workspace_bytes", "moe_infer_i8",
    "moe_kv_plan", "moe_kv_append", "moe_kv_read", "moe_kv_attention_workspace_bytes", "moe_kv_attention",
    "moe_norm_fwd", "moe_norm_bwd_workspace_bytes", "moe_norm_bwd", "moe_decode_workspace_bytes", "moe_decode",
    "moe_decode_i8_workspace_bytes", "moe_decode_i8", "moe_sample_workspace_bytes", "moe_sample",
    "moe_trace_enable", "moe_trace_read", "moe_trace_name",
    "moe_last_error", "moe_version",
)


class MoeDims(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("H", ctypes.c_int32), ("E", ctypes.c_int32),
                ("F", ctypes.c_int32), ("top_k", ctypes.c_int32), ("flags", ctypes.c_uint32),
                ("aux_loss_coef", ctypes.c_float), ("z_loss_coef", ctypes.c_float)]


class MoeSavedView(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in (
        "logits", "topk_idx", "gates", "counts", "offsets", "row_token", "row_of",
        "xp", "g", "u", "a", "o", "router_loss")]


class MoeLora(ctypes.Structure):
    _fields_ = [("rank", ctypes.c_int32), ("scale", ctypes.c_float),
                ("a1", ctypes.c_void_p), ("b1_gate", ctypes.c_void_p), ("b1_up", ctypes.c_void_p),
                ("a2", ctypes.c_void_p), ("b2", ctypes.c_void_p)]


class MoeExpertsDims(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("H", ctypes.c_int32), ("E", ctypes.c_int32),
                ("F", ctypes.c_int32), ("flags", ctypes.c_uint32)]


class MoeExpertsSavedView(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("offsets", "g", "u", "a")]


class MoeI8Dims(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int32), ("N", ctypes.c_int32), ("K", ctypes.c_int32), ("flags", ctypes.c_uint32)]


class MoeI8Experts(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("w_gate", "w_up", "w_down", "s_gate", "s_up", "s_down")]


class MoeKvCache(ctypes.Structure):
    _fields_ = [("n_blocks", ctypes.c_int32), ("block_tokens", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p)]


class MoeKvBatch(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("T", ctypes.c_int32), ("W", ctypes.c_int32),
                ("row_start", ctypes.c_void_p), ("kv_len", ctypes.c_void_p), ("block_table", ctypes.c_void_p)]


class MoeKvPlanDims(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "T", "W", "n_blocks", "block_tokens", "free_cap")]


class MoeKvAttn(ctypes.Structure):
    _fields_ = [("heads", ctypes.c_int32), ("max_q", ctypes.c_int32), ("max_kv", ctypes.c_int32),
                ("scale", ctypes.c_float), ("flags", ctypes.c_uint32)]


class MoeNormDims(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("H", ctypes.c_int32), ("flags", ctypes.c_uint32), ("eps", ctypes.c_float)]


class MoeSampleDims(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("V", ctypes.c_int32), ("flags", ctypes.c_uint32)]


class MoeError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"{msg} (code {code})")
        self.code = code


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2608_00916_amd.build` "
            "(there is no fallback implementation)")
    L = ctypes.CDLL(LIB_PATH)
    P = ctypes.c_void_p
    S = ctypes.c_size_t
    D = ctypes.POINTER(MoeDims)
    ED = ctypes.POINTER(MoeExpertsDims)
    I, I64 = ctypes.c_int32, ctypes.c_int64
    QD, QW = ctypes.POINTER(MoeI8Dims), ctypes.POINTER(MoeI8Experts)
    KC, KB, KA = ctypes.POINTER(MoeKvCache), ctypes.POINTER(MoeKvBatch), ctypes.POINTER(MoeKvAttn)
    ND, SD = ctypes.POINTER(MoeNormDims), ctypes.POINTER(MoeSampleDims)
    sig = {
        "moe_saved_bytes": (S, [D]),
        "moe_fwd_workspace_bytes": (S, [D]),
        "moe_bwd_workspace_bytes": (S, [D]),
        "moe_saved_views": (ctypes.c_int, [D, P, ctypes.POINTER(MoeSavedView)]),
        "moe_fwd": (ctypes.c_int, [D, P, P, P, P, P, P, P, P, P, S, P]),
        "moe_fwd_noalloc": (ctypes.c_int, [D, P, P, P, P, P, P, P, P, P]),
        "moe_bwd": (ctypes.c_int, [D, P, P, P, P, P, P, P, P, P, P, P, P, P, S, P]),
        "moe_infer_workspace_bytes": (S, [D]),
        "moe_lora_saved_bytes": (S, [D, ctypes.c_int32]),
        "moe_lora_workspace_bytes": (S, [D, ctypes.c_int32]),
        "moe_lora_fwd": (ctypes.c_int, [D, P, P, P, P, P, ctypes.POINTER(MoeLora), P, P, P, P, S, P]),
        "moe_lora_bwd": (ctypes.c_int, [D, P, P, P, P, P, ctypes.POINTER(MoeLora), P, P, P, P, P, P, P, P, P, S,
                                        P]),
        "moe_infer": (ctypes.c_int, [D, P, P, P, P, P, P, P, P, S, P]),
        "moe_experts_saved_bytes": (S, [ED]),
        "moe_experts_workspace_bytes": (S, [ED]),
        "moe_experts_saved_views": (ctypes.c_int, [ED, P, ctypes.POINTER(MoeExpertsSavedView)]),
        "moe_experts_fwd": (ctypes.c_int, [ED, P, P, P, P, P, P, P, P, S, P]),
        "moe_experts_bwd": (ctypes.c_int, [ED, P, P, P, P, P, P, P, P, P, P, P, S, P]),
        "moe_i8_quant_rows": (ctypes.c_int, [I, I, P, I64, P, P, P]),
        "moe_i8_quant_weight": (ctypes.c_int, [I, I, I, P, P, P, P]),
        "moe_i8_matmul": (ctypes.c_int, [QD, P, P, P, P, P, I64, P]),
        "moe_i8_linear_workspace_bytes": (S, [QD]),
        "moe_i8_linear": (ctypes.c_int, [QD, P, I64, P, P, P, I64, P, S, P]),
        "moe_experts_i8_workspace_bytes": (S, [ED]),
        "moe_experts_i8": (ctypes.c_int, [ED, P, P, QW, P, P, S, P]),
        "moe_infer_i8_workspace_bytes": (S, [D]),
        "moe_infer_i8": (ctypes.c_int, [D, P, P, QW, P, P, P, S, P]),
        "moe_kv_plan": (ctypes.c_int, [ctypes.POINTER(MoeKvPlanDims)] + [P] * 12),
        "moe_kv_append": (ctypes.c_int, [KC, KB, P, P, I64, P]),
        "moe_kv_read": (ctypes.c_int, [KC, I, I, P, P, I, P, P, P]),
        "moe_kv_attention_workspace_bytes": (S, [KC, KB, KA]),
        "moe_kv_attention": (ctypes.c_int, [KC, KB, KA, P, I64, P, I64, P, S, P]),
        "moe_norm_fwd": (ctypes.c_int, [ND, P, I64, P, I64, P, P, P, P, P, P]),
        "moe_norm_bwd_workspace_bytes": (S, [ND]),
        "moe_norm_bwd": (ctypes.c_int, [ND, P, I64, P, P, I64, P, I64, P, P, P, S, P]),
        "moe_decode_workspace_bytes": (S, [D]),
        "moe_decode": (ctypes.c_int, [D, P, P, P, P, P, P, P, P, S, P]),
        "moe_decode_i8_workspace_bytes": (S, [D]),
        "moe_decode_i8": (ctypes.c_int, [D, P, P, QW, P, P, P, S, P]),
        "moe_sample_workspace_bytes": (S, [SD]),
        "moe_sample": (ctypes.c_int, [SD, P, I64, P, P, P, P, P, P, P, P, S, P]),
        "moe_trace_enable": (ctypes.c_int, [ctypes.c_int]),
        "moe_trace_read": (ctypes.c_int, [ctypes.POINTER(ctypes.c_double),
                                          ctypes.POINTER(ctypes.c_int32), ctypes.c_int]),
        "moe_trace_name": (ctypes.c_char_p, [ctypes.c_int]),
        "moe_last_error": (ctypes.c_char_p, []),
        "moe_version": (ctypes.c_int, []),
    }
    for name, (res, args) in sig.items():
        f = getattr(L, name)
        f.restype = res
        f.argtypes = args
    _lib = L
    return L


def check(rc: int) -> None:
    if rc != MOE_OK:
        raise MoeError(rc, lib().moe_last_error().decode())

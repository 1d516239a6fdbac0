"""ctypes declarations of the C ABI in include/ftcnn.h (argument marshalling only)."""
from __future__ import annotations

import ctypes as C
import os

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libftcnn.so")

F32, BF16 = 0, 1

CO1, CO2, CO3, CO4, CO5, CO6, CO7 = (1 << i for i in range(7))

SCHEME_NONE, SCHEME_COC, SCHEME_RC, SCHEME_CLC, SCHEME_FC, SCHEME_CKSUM, SCHEME_UNRESOLVED = range(7)
STATUS_CLEAN, STATUS_CORRECTED, STATUS_NEEDS_RECOMPUTE, STATUS_RECOMPUTED, STATUS_FAILED = range(5)
REPAIR_CHECKSUM, REPAIR_RECOMPUTE = 0, 1


class ConvDesc(C.Structure):
    _fields_ = [("n", C.c_int32), ("ch", C.c_int32), ("h", C.c_int32), ("w", C.c_int32),
                ("m", C.c_int32), ("r", C.c_int32), ("s", C.c_int32),
                ("stride", C.c_int32), ("pad", C.c_int32), ("groups", C.c_int32),
                ("dtype", C.c_int32), ("wbase", C.c_int32)]


_dp = C.c_void_p


class Checksums(C.Structure):
    _fields_ = [(name, _dp) for name in
                ("cd1", "cd2", "cw1", "cw2", "co5", "co6", "co7", "so5", "so6", "so7", "q5",
                 "co1", "co3", "co2", "co4", "bias", "cb")]


class Fix(C.Structure):
    _fields_ = [("n", C.c_int32), ("m", C.c_int32), ("x", C.c_int32), ("y", C.c_int32),
                ("scheme", C.c_int32)]


class ReportHeader(C.Structure):
    _fields_ = [("detected", C.c_int32), ("n_flagged", C.c_int32), ("status", C.c_int32),
                ("resolved_by", C.c_int32 * 7), ("n_fixes", C.c_int32), ("cap_fixes", C.c_int32),
                ("reserved", C.c_int32 * 2)]


class Policy(C.Structure):
    _fields_ = [("rc_on", C.c_int32), ("clc_on", C.c_int32), ("repair", C.c_int32),
                ("reserved", C.c_int32), ("kappa", C.c_double), ("eta", C.c_double)]


class Fault(C.Structure):
    _fields_ = [("n", C.c_int32), ("m", C.c_int32), ("x", C.c_int32), ("y", C.c_int32),
                ("kind", C.c_int32), ("bit", C.c_int32), ("value", C.c_double)]


class RopeScaling(C.Structure):
    _fields_ = [("max_pos", C.c_int32), ("rot", C.c_int32), ("scaling", C.c_int32), ("original", C.c_int32),
                ("base", C.c_double), ("factor", C.c_double), ("low", C.c_double), ("high", C.c_double),
                ("amplitude", C.c_double)]


class RopeDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("dtype", "tokens", "heads", "kv_heads", "dim", "rot", "layout", "max_pos",
                                         "weight_dtype")] + [("eps", C.c_float)] + [
        (n, C.c_int64 * 2) for n in ("q_stride", "k_stride", "q_out_stride", "k_out_stride")]


class AppendDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("dtype", "tokens", "kv_heads", "dim", "rot", "layout", "max_pos",
                                         "weight_dtype", "pages", "page")] + [
        ("eps", C.c_float), ("reserved", C.c_int32), ("k_stride", C.c_int64 * 2), ("v_stride", C.c_int64 * 2),
        ("k_cache_stride", C.c_int64 * 3), ("v_cache_stride", C.c_int64 * 3)]


class AttentionDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("dtype", "batch", "tokens", "heads", "kv_heads", "dim", "pages", "page",
                                         "list_len", "causal", "window", "max_q", "max_kv")] + [
        ("scale", C.c_float), ("q_stride", C.c_int64 * 2), ("out_stride", C.c_int64 * 2),
        ("k_cache_stride", C.c_int64 * 3), ("v_cache_stride", C.c_int64 * 3), ("list_stride", C.c_int64)]


EXPORTS = ("ftcnn_out_shape", "ftcnn_workspace_bytes", "ftcnn_report_bytes", "ftcnn_last_error",
           "ftcnn_encode", "ftcnn_conv_fwd", "ftcnn_checksum_conv", "ftcnn_verify", "ftcnn_correct",
           "ftcnn_verify_correct", "ftcnn_conv_fwd_ws", "ftcnn_conv_fwd_sums", "ftcnn_verify_correct_sums", "ftcnn_protected_conv",
           "ftcnn_inject", "ftcnn_set_kernel_events", "ftcnn_conv_fwd_bias", "ftcnn_check_weights",
           "ftcnn_relu_pool", "ftcnn_relu_pool_encode", "ftcnn_conv_fwd_sums_given", "ftcnn_conv_tile",
           "ftcnn_protected_conv_noalloc", "ftcnn_conv_stream_k", "ftcnn_rope_table", "ftcnn_qk_norm_rope",
           "ftcnn_kv_append", "ftcnn_paged_attention", "ftcnn_paged_attention_workspace_bytes")

_lib = None


def load(path: str = LIB_PATH):
    """Load the HIP library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with paper_2003_12203_amd/build.py "
                           "(hipcc, gfx950); there is no fallback implementation")
    L = C.CDLL(path)
    P = C.POINTER
    L.ftcnn_out_shape.argtypes = [P(ConvDesc), P(C.c_int32), P(C.c_int32)]
    L.ftcnn_out_shape.restype = C.c_int
    L.ftcnn_workspace_bytes.argtypes = [P(ConvDesc)]
    L.ftcnn_workspace_bytes.restype = C.c_size_t
    L.ftcnn_report_bytes.argtypes = [C.c_int32]
    L.ftcnn_report_bytes.restype = C.c_size_t
    L.ftcnn_conv_tile.argtypes = [P(ConvDesc), C.c_int32, P(C.c_int32)]
    L.ftcnn_conv_tile.restype = C.c_int
    L.ftcnn_conv_stream_k.argtypes = [P(ConvDesc), P(C.c_int32)]
    L.ftcnn_conv_stream_k.restype = C.c_int
    L.ftcnn_last_error.argtypes = []
    L.ftcnn_last_error.restype = C.c_char_p
    L.ftcnn_encode.argtypes = [P(ConvDesc), C.c_int32, _dp, _dp, _dp, _dp, _dp]
    L.ftcnn_encode.restype = C.c_int
    L.ftcnn_conv_fwd.argtypes = [P(ConvDesc), _dp, _dp, _dp, _dp]
    L.ftcnn_conv_fwd.restype = C.c_int
    L.ftcnn_checksum_conv.argtypes = [P(ConvDesc), C.c_uint32, _dp, _dp, P(Checksums), _dp]
    L.ftcnn_checksum_conv.restype = C.c_int
    L.ftcnn_verify.argtypes = [P(ConvDesc), _dp, P(Checksums), P(Policy), _dp, C.c_int32, _dp, _dp]
    L.ftcnn_verify.restype = C.c_int
    L.ftcnn_correct.argtypes = [P(ConvDesc), _dp, _dp, _dp, P(Checksums), P(Policy), _dp, _dp, _dp]
    L.ftcnn_correct.restype = C.c_int
    L.ftcnn_verify_correct.argtypes = [P(ConvDesc), _dp, _dp, _dp, P(Checksums), P(Policy), _dp, C.c_int32,
                                       _dp, _dp]
    L.ftcnn_verify_correct.restype = C.c_int
    L.ftcnn_check_weights.argtypes = [P(ConvDesc), _dp, _dp, _dp, _dp, _dp]
    L.ftcnn_check_weights.restype = C.c_int
    L.ftcnn_relu_pool.argtypes = [C.c_int32] * 7 + [_dp, _dp, _dp]
    L.ftcnn_relu_pool.restype = C.c_int
    L.ftcnn_relu_pool_encode.argtypes = [C.c_int32] * 8 + [_dp, _dp, _dp, _dp, _dp]
    L.ftcnn_relu_pool_encode.restype = C.c_int
    L.ftcnn_conv_fwd_bias.argtypes = [P(ConvDesc), _dp, _dp, _dp, _dp, _dp, _dp]
    L.ftcnn_conv_fwd_bias.restype = C.c_int
    L.ftcnn_conv_fwd_ws.argtypes = [P(ConvDesc), _dp, _dp, _dp, _dp, _dp]
    L.ftcnn_conv_fwd_ws.restype = C.c_int
    L.ftcnn_conv_fwd_sums.argtypes = [P(ConvDesc), _dp, _dp, _dp, P(Checksums), _dp, C.c_int32, P(Fault),
                                      C.c_int32, _dp, _dp]
    L.ftcnn_conv_fwd_sums.restype = C.c_int
    L.ftcnn_conv_fwd_sums_given.argtypes = L.ftcnn_conv_fwd_sums.argtypes
    L.ftcnn_conv_fwd_sums_given.restype = C.c_int
    L.ftcnn_verify_correct_sums.argtypes = [P(ConvDesc), _dp, _dp, _dp, P(Checksums), P(Policy), _dp,
                                            C.c_uint32, _dp, _dp]
    L.ftcnn_verify_correct_sums.restype = C.c_int
    L.ftcnn_protected_conv.argtypes = [P(ConvDesc), _dp, _dp, _dp, P(Checksums), P(Policy), _dp,
                                       C.c_int32, _dp, _dp]
    L.ftcnn_protected_conv.restype = C.c_int
    L.ftcnn_protected_conv_noalloc.argtypes = [P(ConvDesc), _dp, _dp, _dp, P(Checksums), P(Policy), _dp,
                                               C.c_int32, _dp]
    L.ftcnn_protected_conv_noalloc.restype = C.c_int
    L.ftcnn_inject.argtypes = [P(ConvDesc), _dp, P(Fault), C.c_int32, _dp]
    L.ftcnn_inject.restype = C.c_int
    L.ftcnn_set_kernel_events.argtypes = [_dp, _dp]
    L.ftcnn_set_kernel_events.restype = C.c_int
    L.ftcnn_rope_table.argtypes = [P(RopeScaling), _dp, _dp]
    L.ftcnn_rope_table.restype = C.c_int
    # descriptors of the serving operators come packed, as bytes in the layout of their structures
    L.ftcnn_qk_norm_rope.argtypes = [C.c_char_p] + [_dp] * 9
    L.ftcnn_qk_norm_rope.restype = C.c_int
    L.ftcnn_kv_append.argtypes = [C.c_char_p] + [_dp] * 9
    L.ftcnn_kv_append.restype = C.c_int
    L.ftcnn_paged_attention.argtypes = [C.c_char_p] + [_dp] * 10
    L.ftcnn_paged_attention.restype = C.c_int
    L.ftcnn_paged_attention_workspace_bytes.argtypes = [C.c_char_p]
    L.ftcnn_paged_attention_workspace_bytes.restype = C.c_size_t
    _lib = L
    return L

"""Python binding of libiseg.so (ctypes).

The `iseg_*` functions here carry the C ABI's names and arguments one to one:
they only turn torch tensors into device pointers, pass the current HIP
stream, and raise on a non-zero status.  Every computation runs in the HIP
kernels; there is no fallback.  The helpers below them (conv_fwd, bn_fwd, ...)
allocate outputs and workspaces with torch and call those entry points.

A quantized tensor is a pair (codes, exp): integer codes and a 1-element int32
device tensor holding the power-of-two exponent (value = code * 2^exp).
"""
import ctypes as C
import functools
import math
import os
import threading
from typing import NamedTuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "lib", "libiseg.so")

ISEG_OK, ISEG_ERR_ARG, ISEG_ERR_SHAPE, ISEG_ERR_UNSUPPORTED, ISEG_ERR_WORKSPACE, ISEG_ERR_DEVICE = range(6)
ISEG_DEV_RANGE, ISEG_DEV_NONFINITE, ISEG_DEV_DESC = 1, 4, 8
ISEG_I8, ISEG_I16, ISEG_I32, ISEG_I64, ISEG_F32, ISEG_F16, ISEG_BF16 = range(7)
ISEG_SCALE_MAX, ISEG_SCALE_POW2 = 0, 1
ISEG_Q_UQ, ISEG_Q_SQ = 0, 1
ISEG_OUT_Q8, ISEG_OUT_RAW = 0, 1
ISEG_G_KEEP, ISEG_G_DROP, ISEG_G_RAW = 0, 1, 2
(ISEG_KID_NONE, ISEG_KID_CONV_FWD, ISEG_KID_CONV_BWD_DATA, ISEG_KID_CONV_WGRAD, ISEG_KID_REQUANT,
 ISEG_KID_BN_FWD_APPLY, ISEG_KID_BN_BWD_APPLY, ISEG_KID_BN_FWD_STATS1, ISEG_KID_BN_FWD_STATS2,
 ISEG_KID_BN_BWD_STATS, ISEG_KID_MAXPOOL_BWD) = range(11)

_ERRS = {1: "ISEG_ERR_ARG", 2: "ISEG_ERR_SHAPE", 3: "ISEG_ERR_UNSUPPORTED",
         4: "ISEG_ERR_WORKSPACE", 5: "ISEG_ERR_DEVICE"}


class IsegError(RuntimeError):
    pass


class ConvGeom(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("N", "H", "W", "C", "K", "R", "S")] + \
               [(n, C.c_int32) for n in ("stride_h", "stride_w", "pad_h", "pad_w", "dil_h", "dil_w")]


class UpdateDesc(C.Structure):
    _fields_ = [("master", C.c_void_p), ("w_q", C.c_void_p), ("g", C.c_void_p), ("g_exp", C.c_void_p),
                ("g_q", C.c_void_p), ("g_q_exp", C.c_void_p), ("n", C.c_int64), ("kind", C.c_int32),
                ("master_exp", C.c_int32), ("tensor_id", C.c_uint32), ("k_w", C.c_int32)]


ISEG_UPD_CODES, ISEG_UPD_RAW = 0, 1


class WtDesc(C.Structure):
    _fields_ = [("w", C.c_void_p), ("wt", C.c_void_p), ("K", C.c_int32), ("RS", C.c_int32), ("C", C.c_int32),
                ("kind", C.c_int32), ("tile_begin", C.c_int64)]


ISEG_WT_NONE, ISEG_WT_CRSK, ISEG_WT_CRSK_FLIP = 0, 1, 2


class BnCfg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("k_mu", "k_sigma", "k_xhat", "k_gamma", "k_beta",
                                         "k_A", "k_E1", "k_E2", "eps_code", "relu")]


BN_DEFAULT = dict(k_mu=16, k_sigma=16, k_xhat=16, k_gamma=8, k_beta=8, k_A=8, k_E1=8, k_E2=16,
                  eps_code=0, relu=1)

class LayernormGeom(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("M", "C", "x_ld", "y_ld", "dx_ld")] + \
               [("x_dtype", C.c_int32), ("p_dtype", C.c_int32), ("eps", C.c_float), ("reserved", C.c_int32)]


class MatmulGeom(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("M", "N", "K", "lda", "ldb", "ldc")] + \
               [("out_dtype", C.c_int32), ("unaligned", C.c_int32)]


class LinearGeom(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("M", "N", "K", "x_ld", "w_ld", "codes_ld", "y_ld")] + \
               [(n, C.c_int32) for n in ("x_dtype", "y_dtype", "bits", "scale_mode", "unaligned", "reserved")]


class LinearBwdGeom(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("M", "N", "K", "dy_ld", "a_ld", "w_ld", "wt_ld", "dx_ld", "dw_ld")] + \
               [(n, C.c_int32) for n in ("dy_dtype", "out_dtype", "bits", "scale_mode", "unaligned", "reserved")]


class LogprobGeom(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("M", "V", "ld", "out_ld")] + \
               [(n, C.c_int32) for n in ("dtype", "token_dtype", "top_k", "reserved")]


class PageMapGeom(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("B", "T", "max_pages", "table_ld", "F", "n_pages")] + \
               [("page", C.c_int32), ("reserved", C.c_int32)]


class QkNormRopeGeom(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("T", "Hq", "Hk", "D", "q_ld", "q_hs", "k_ld", "k_hs", "yq_ld", "yq_hs",
                                         "yk_ld", "yk_hs", "dq_ld", "dq_hs", "dk_ld", "dk_hs")] + \
               [(n, C.c_int32) for n in ("dtype", "p_dtype", "pos_dtype", "rope_dim", "pairs", "norm")] + \
               [("eps", C.c_float), ("mscale", C.c_float)]


class Kv4Geom(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("T", "H", "D", "k_ld", "k_hs", "v_ld", "v_hs", "n_pages")] + \
               [(n, C.c_int32) for n in ("page", "dtype", "slot_dtype", "scale_mode")]


class Kv4AttentionGeom(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("T", "B", "Hq", "H", "D", "q_ld", "q_hs", "o_ld", "o_hs", "n_pages",
                                         "max_pages", "table_ld", "max_q", "max_kv", "window")] + \
               [("page", C.c_int32), ("dtype", C.c_int32), ("causal", C.c_int32), ("scale", C.c_float)]


class VerifyGeom(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("B", "S", "V", "t_bs", "t_ld", "d_bs", "d_ld")] + \
               [("dtype", C.c_int32), ("token_dtype", C.c_int32)]


_lib = None
_P, _I64, _I32, _U64, _U32, _SZ = C.c_void_p, C.c_int64, C.c_int32, C.c_uint64, C.c_uint32, C.c_size_t

_SIGS = {
    "iseg_quantize_ws": ([_I64], _SZ),
    "iseg_quantize": ([_P, _I64, _I32, _I32, _I32, _P, _P, _P, _SZ, _P, _P], C.c_int),
    "iseg_requant_ws": ([_I64], _SZ),
    "iseg_requant": ([_P, _I32, _I64, _P, _I32, _I32, _I32, _U64, _U32, _U32, _I32, _P, _P, _P, _SZ,
                      _P, _P], C.c_int),
    "iseg_conv_fwd_ws": ([_P, _I32], _SZ),
    "iseg_conv_fwd": ([_P, _P, _P, _P, _P, _I32, _P, _P, _P, _SZ, _P, _P], C.c_int),
    "iseg_conv_bwd_data_ws": ([_P, _I32], _SZ),
    "iseg_conv_bwd_data": ([_P, _P, _P, _P, _P, _I32, _P, _P, _P, _SZ, _P, _P], C.c_int),
    "iseg_conv_bwd_data_t": ([_P, _P, _P, _P, _P, _I32, _P, _I32, _P, _P, _P, _SZ, _P, _P], C.c_int),
    "iseg_conv_bwd_data_wt_kind": ([_P], C.c_int32),
    "iseg_weight_transpose_multi": ([_P, _I32, _I64, _P], C.c_int),
    "iseg_conv_bwd_weight_ws": ([_P, _I32], _SZ),
    "iseg_conv_bwd_weight": ([_P, _P, _P, _P, _P, _I32, _I32, _U64, _U32, _U32, _P, _P, _P, _SZ,
                              _P, _P], C.c_int),
    "iseg_bn_saved_bytes": ([_I64], _SZ),
    "iseg_bn_fwd_ws": ([_I64, _I64], _SZ),
    "iseg_bn_fwd": ([_P, _P, _I64, _I64, _P, _P, _P, _P, _P, _P, _P, _SZ, _P, _P], C.c_int),
    "iseg_bn_fwd_noalloc_max_bytes": ([], _SZ),
    "iseg_bn_fwd_noalloc": ([_P, _P, _I64, _I64, _P, _P, _P, _P, _P, _P, _P, _P], C.c_int),
    "iseg_bn_bwd_ws": ([_I64, _I64], _SZ),
    "iseg_bn_infer": ([_P, _P, _I64, _I64, _P, _P, _P, _P, _P], C.c_int),
    "iseg_conv_bn_infer_ws": ([_P], _SZ),
    "iseg_conv_bn_infer": ([_P, _P, _P, _P, _P, _P, _P, _P, _P, _SZ, _P, _P], C.c_int),
    "iseg_bn_i32_saved_bytes": ([_I64], _SZ),
    "iseg_bn_fwd_i32_ws": ([_I64, _I64], _SZ),
    "iseg_bn_fwd_i32": ([_P, _P, _I64, _I64, _P, _P, _P, _P, _P, _P, _P, _SZ, _P, _P], C.c_int),
    "iseg_bn_bwd_i32_ws": ([_I64, _I64], _SZ),
    "iseg_bn_bwd_i32": ([_P, _P, _P, _I64, _I64, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _SZ, _P, _P],
                        C.c_int),
    "iseg_bn_bwd": ([_P, _P, _P, _I64, _I64, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _SZ, _P, _P],
                    C.c_int),
    "iseg_weight_update": ([_P, _I64, _P, _P, _I32, _I32, _I32, _I32, _P, _P, _P], C.c_int),
    "iseg_weight_quant": ([_P, _I64, _I32, _I32, _P, _P], C.c_int),
    "iseg_maxpool_fwd": ([_P, _P, _I64, _I64, _I64, _I64, _I32, _I32, _I32, _P, _P, _P], C.c_int),
    "iseg_maxpool_bwd_ws": ([_I64, _I64, _I64, _I64], _SZ),
    "iseg_maxpool_bwd": ([_P, _P, _P, _I64, _I64, _I64, _I64, _I32, _I32, _I32, _I32, _P, _P, _P,
                          _SZ, _P, _P], C.c_int),
    "iseg_bn_param_update": ([_P, _P, _P, _P, _I64, _I32, _U64, _U32, _U32, _U32, _I32, _I32, _I32,
                              _I32, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P], C.c_int),
    "iseg_sum_requant_ws": ([_I64, _I64, _I64], _SZ),
    "iseg_sum_requant": ([_I32, _P, _P, _P, _P, _I64, _I64, _I64, _I32, _I32, _P, _P, _P, _SZ, _P, _P],
                         C.c_int),
    "iseg_relu_mask_bwd": ([_P, _I32, _P, _P, _P, _I64, _I64, _P, _P, _P], C.c_int),
    "iseg_sum_requant_relu_mask": ([_I32, _P, _P, _P, _I64, _I64, _I64, _I32, _I32, _P, _P, _P, _P, _P, _SZ,
                                    _P, _P], C.c_int),
    "iseg_concat_requant_ws": ([_I32], _SZ),
    "iseg_concat_requant": ([_I32, _P, _P, _P, _P, _I64, _I64, _I32, _P, _P, _P, _SZ, _P, _P], C.c_int),
    "iseg_concat_split": ([_P, _I64, _I32, _P, _P, _P], C.c_int),
    "iseg_spatial_sum_ws": ([_I64, _I64, _I64], _SZ),
    "iseg_spatial_sum": ([_P, _P, _I64, _I64, _I64, _I64, _I64, _I64, _I32, _P, _P, _P, _SZ, _P, _P],
                         C.c_int),
    "iseg_softmax_ce_ws": ([_I64, _I64, _I64, _I64, _I64, _I64], _SZ),
    "iseg_softmax_ce": ([_P, _P, _P, _I64, _I64, _I64, _I64, _I64, _I64, _I32, _P, _P, _P, _P, _P, _SZ,
                         _P, _P], C.c_int),
    "iseg_mse_onehot_ws": ([_I64], _SZ),
    "iseg_mse_onehot": ([_P, _P, _P, _I64, _I64, _I64, _I64, _I32, _P, _P, _P, _P, _SZ, _P, _P], C.c_int),
    "iseg_update_multi": ([_P, _I32, _I32, _U64, _U32, _I32, _I32, _I32, _P, _P], C.c_int),
    "iseg_layernorm_fwd": ([_P, _P, _P, _P, _P, _P, _P, _P, _P], C.c_int),
    "iseg_layernorm_bwd_ws": ([_P], _SZ),
    "iseg_layernorm_bwd": ([_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _SZ, _P], C.c_int),
    "iseg_quantize_rows": ([_P, _I32, _I64, _I64, _I64, _P, _I32, _I32, _P, _I64, _P, _P, _P], C.c_int),
    "iseg_quantize_cols_ws": ([_I64, _I64], _SZ),
    "iseg_quantize_cols": ([_P, _I32, _I64, _I64, _I64, _P, _I32, _I32, _P, _I64, _P, _P, _P, _SZ, _P, _P],
                           C.c_int),
    "iseg_transpose_i8": ([_P, _I64, _I64, _I64, _P, _I64, _P], C.c_int),
    "iseg_matmul_i8_ws": ([_P], _SZ),
    "iseg_matmul_i8": ([_P, _P, _P, _P, _P, _P, _P, _P, _SZ, _P], C.c_int),
    "iseg_linear_i8_fwd_ws": ([_P], _SZ),
    "iseg_linear_i8_fwd": ([_P, _P, _P, _P, _P, _P, _P, _P, _P, _SZ, _P, _P], C.c_int),
    "iseg_linear_i8_bwd_ws": ([_P], _SZ),
    "iseg_linear_i8_bwd": ([_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _SZ, _P, _P], C.c_int),
    "iseg_logprob_fwd_ws": ([_P], _SZ),
    "iseg_logprob_fwd": ([_P, _P, _P, _P, _P, _P, _P, _P, _P, _SZ, _P, _P], C.c_int),
    "iseg_logprob_bwd": ([_P, _P, _P, _P, _P, _P, _P, _P, _P, _P], C.c_int),
    "iseg_page_map_ws": ([_P], _SZ),
    "iseg_page_map": ([_P] * 14 + [_SZ, _P, _P], C.c_int),
    "iseg_qk_norm_rope_fwd": ([_P] * 11, C.c_int),
    "iseg_qk_norm_rope_bwd_ws": ([_P], _SZ),
    "iseg_qk_norm_rope_bwd": ([_P] * 14 + [_SZ, _P], C.c_int),
    "iseg_kv4_write": ([_P] * 10, C.c_int),
    "iseg_kv4_read": ([_P] * 10, C.c_int),
    "iseg_kv4_attention_ws": ([_P], _SZ),
    "iseg_kv4_attention": ([_P] * 12 + [_SZ, _P, _P], C.c_int),
    "iseg_verify_drafts_ws": ([_P], _SZ),
    "iseg_verify_drafts": ([_P] * 10 + [_SZ, _P, _P], C.c_int),
    "iseg_philox4x32_10": ([_P, _P, _P], None),
    "iseg_profile_arm": ([_I32, _P, _P], C.c_int),
    "iseg_conv_last_plan": ([], C.c_char_p),
    "iseg_status_read": ([_P, _P, _P], C.c_int),
    "iseg_status_clear": ([_P, _P], C.c_int),
    "iseg_check_codes": ([_P, _I64, _I32, _P, _P], C.c_int),
    "iseg_version": ([], C.c_char_p),
    "iseg_tape_create": ([], _P),
    "iseg_tape_destroy": ([_P], None),
    "iseg_tape_entry": ([C.c_char_p], C.c_int),
    "iseg_tape_entry_nargs": ([C.c_int], C.c_int),
    "iseg_tape_add_call": ([_P, C.c_int, _P, C.c_int, _P, _SZ, _P, C.c_int, _I32, _I64], C.c_int),
    "iseg_tape_add_record": ([_P, _I32, _P], C.c_int),
    "iseg_tape_add_wait": ([_P, _P, _I32], C.c_int),
    "iseg_tape_arm_count": ([_P], C.c_int),
    "iseg_tape_set_arm_events": ([_P, _P, _I32], C.c_int),
    "iseg_tape_run": ([_P, _U32, _P], C.c_int),
    "iseg_tape_size": ([_P], _I64),
}


def lib():
    """Load libiseg.so; raises if it has not been built (no fallback path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"libiseg.so not built at {LIB_PATH}; run __graft_entry__.build()")
        L = C.CDLL(LIB_PATH)
        for name, (args, res) in _SIGS.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = res
        _lib = L
    if _REC is not None:
        return _REC.lib
    return _lib


def _ptr(t):
    if t is None:
        return None
    if _REC is not None:
        _REC.keep.append(t)          # a recorded call's buffer stays allocated
        return C.c_void_p(t.data_ptr())
    return t.data_ptr()              # the declared argument types convert it


_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else None
_raw_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device


def _stream_handle(dev_index=None):
    """Raw handle of the current stream of a device (the current device by
    default): the launch path asks for it on every call, so it bypasses the
    Stream object construction of torch.cuda.current_stream()."""
    if dev_index is None:
        dev_index = _raw_device()
    if _raw_stream is not None:
        return _raw_stream(dev_index)
    return torch.cuda.current_stream(dev_index).cuda_stream


def _stream():
    return C.c_void_p(_stream_handle()) if _REC is not None else _stream_handle()


def _check(rc, name):
    if rc != ISEG_OK:
        raise IsegError(f"{name} returned {_ERRS.get(rc, rc)}")


def _ws_tuple(ws):
    return (_ptr(ws), ws.numel() if ws is not None else 0)


# --------------------------------------------------------------------------
# entry points, one to one with include/iseg.h
# --------------------------------------------------------------------------
def iseg_quantize(x, bits, mode, out_dtype, out, out_exp, ws, status=None):
    rc = lib().iseg_quantize(_ptr(x), x.numel(), bits, mode, out_dtype, _ptr(out), _ptr(out_exp),
                             *_ws_tuple(ws), _ptr(status), _stream())
    _check(rc, "iseg_quantize")


def iseg_requant(inp, in_dtype, in_exp, bits, stochastic, keep_scale, seed, tensor_id, step,
                 out_dtype, out, out_exp, ws, status=None):
    rc = lib().iseg_requant(_ptr(inp), in_dtype, inp.numel(), _ptr(in_exp), bits, stochastic,
                            keep_scale, seed, tensor_id, step, out_dtype, _ptr(out), _ptr(out_exp),
                            *_ws_tuple(ws), _ptr(status), _stream())
    _check(rc, "iseg_requant")


def iseg_conv_fwd(x, x_exp, w, w_exp, geom, out_mode, y, y_exp, ws, status=None):
    rc = lib().iseg_conv_fwd(_ptr(x), _ptr(x_exp), _ptr(w), _ptr(w_exp), C.byref(geom), out_mode,
                             _ptr(y), _ptr(y_exp), *_ws_tuple(ws), _ptr(status), _stream())
    _check(rc, "iseg_conv_fwd")


def iseg_conv_bwd_data(dy, dy_exp, w, w_exp, geom, out_mode, dx, dx_exp, ws, status=None):
    rc = lib().iseg_conv_bwd_data(_ptr(dy), _ptr(dy_exp), _ptr(w), _ptr(w_exp), C.byref(geom),
                                  out_mode, _ptr(dx), _ptr(dx_exp), *_ws_tuple(ws), _ptr(status),
                                  _stream())
    _check(rc, "iseg_conv_bwd_data")


def iseg_conv_bwd_data_t(dy, dy_exp, w, w_exp, wt, wt_kind, geom, out_mode, dx, dx_exp, ws, status=None):
    rc = lib().iseg_conv_bwd_data_t(_ptr(dy), _ptr(dy_exp), _ptr(w), _ptr(w_exp), _ptr(wt), wt_kind,
                                    C.byref(geom), out_mode, _ptr(dx), _ptr(dx_exp), *_ws_tuple(ws),
                                    _ptr(status), _stream())
    _check(rc, "iseg_conv_bwd_data_t")


def iseg_conv_bwd_data_wt_kind(geom):
    return int(lib().iseg_conv_bwd_data_wt_kind(C.byref(geom)))


def iseg_weight_transpose_multi(table, n, total_tiles):
    rc = lib().iseg_weight_transpose_multi(_ptr(table), n, total_tiles, _stream())
    _check(rc, "iseg_weight_transpose_multi")


def iseg_conv_bwd_weight(dy, dy_exp, x, x_exp, geom, g_mode, bits, seed, tensor_id, step, dw,
                         dw_exp, ws, status=None):
    rc = lib().iseg_conv_bwd_weight(_ptr(dy), _ptr(dy_exp), _ptr(x), _ptr(x_exp), C.byref(geom),
                                    g_mode, bits, seed, tensor_id, step, _ptr(dw), _ptr(dw_exp),
                                    *_ws_tuple(ws), _ptr(status), _stream())
    _check(rc, "iseg_conv_bwd_weight")


def iseg_bn_fwd(x, x_exp, M, Cc, gamma_q, beta_q, cfg, y, y_exp, saved, ws, status=None):
    rc = lib().iseg_bn_fwd(_ptr(x), _ptr(x_exp), M, Cc, _ptr(gamma_q), _ptr(beta_q), C.byref(cfg),
                           _ptr(y), _ptr(y_exp), _ptr(saved), *_ws_tuple(ws), _ptr(status),
                           _stream())
    _check(rc, "iseg_bn_fwd")


def iseg_bn_infer(z, z_exp, M, Cc, saved, a, a_exp, status=None):
    rc = lib().iseg_bn_infer(_ptr(z), _ptr(z_exp), M, Cc, _ptr(saved), _ptr(a), _ptr(a_exp), _ptr(status),
                             _stream())
    _check(rc, "iseg_bn_infer")


def iseg_conv_bn_infer(x, x_exp, w, w_exp, geom, saved, a, a_exp, ws, status=None):
    rc = lib().iseg_conv_bn_infer(_ptr(x), _ptr(x_exp), _ptr(w), _ptr(w_exp), C.byref(geom), _ptr(saved),
                                  _ptr(a), _ptr(a_exp), *_ws_tuple(ws), _ptr(status), _stream())
    _check(rc, "iseg_conv_bn_infer")


def bn_infer(z, z_exp, saved, status=None):
    """A codes of int8 codes z through a calibration forward's frozen state."""
    Cc = z.shape[-1]
    a = torch.empty_like(z)
    e = _out_exp(z.device)
    iseg_bn_infer(z, z_exp, z.numel() // Cc, Cc, saved, a, e, status)
    return a, e


def conv_bn_infer(x, x_exp, w, w_exp, saved, stride=1, pad=0, dil=1, status=None):
    """Conv + L1BN + ReLU? + Q_A of one layer with a calibration's frozen state."""
    N, H, W, Cc = x.shape
    K, R, S, _ = w.shape
    g = geom(N, H, W, Cc, K, R, S, stride, pad, dil)
    P, Q = conv_out_hw(g)
    a = torch.empty((N, P, Q, K), dtype=torch.int8, device=x.device)
    e = _out_exp(x.device)
    ws = workspace(x.device).get(lib().iseg_conv_bn_infer_ws(C.byref(g)))
    iseg_conv_bn_infer(x, x_exp, w, w_exp, g, saved, a, e, ws, status)
    return a, e


def iseg_bn_fwd_i32(x, x_exp, M, Cc, gamma_q, beta_q, cfg, y, y_exp, saved, ws, status=None):
    rc = lib().iseg_bn_fwd_i32(_ptr(x), _ptr(x_exp), M, Cc, _ptr(gamma_q), _ptr(beta_q), C.byref(cfg),
                               _ptr(y), _ptr(y_exp), _ptr(saved), *_ws_tuple(ws), _ptr(status), _stream())
    _check(rc, "iseg_bn_fwd_i32")


def iseg_bn_bwd_i32(dy, dy_exp, x, M, Cc, gamma_q, cfg, saved, dx, dx_exp, dgamma, dbeta, dgamma_exp,
                    dbeta_exp, ws, status=None):
    rc = lib().iseg_bn_bwd_i32(_ptr(dy), _ptr(dy_exp), _ptr(x), M, Cc, _ptr(gamma_q), C.byref(cfg),
                               _ptr(saved), _ptr(dx), _ptr(dx_exp), _ptr(dgamma), _ptr(dbeta),
                               _ptr(dgamma_exp), _ptr(dbeta_exp), *_ws_tuple(ws), _ptr(status), _stream())
    _check(rc, "iseg_bn_bwd_i32")


def iseg_bn_fwd_noalloc(x, x_exp, M, Cc, gamma_q, beta_q, cfg, y, y_exp, saved, status=None):
    rc = lib().iseg_bn_fwd_noalloc(_ptr(x), _ptr(x_exp), M, Cc, _ptr(gamma_q), _ptr(beta_q), C.byref(cfg),
                                   _ptr(y), _ptr(y_exp), _ptr(saved), _ptr(status), _stream())
    _check(rc, "iseg_bn_fwd_noalloc")


def iseg_bn_bwd(dy, dy_exp, x, M, Cc, gamma_q, cfg, saved, dx, dx_exp, dgamma, dbeta, dgamma_exp,
                dbeta_exp, ws, status=None):
    rc = lib().iseg_bn_bwd(_ptr(dy), _ptr(dy_exp), _ptr(x), M, Cc, _ptr(gamma_q), C.byref(cfg),
                           _ptr(saved), _ptr(dx), _ptr(dx_exp), _ptr(dgamma), _ptr(dbeta),
                           _ptr(dgamma_exp), _ptr(dbeta_exp), *_ws_tuple(ws), _ptr(status),
                           _stream())
    _check(rc, "iseg_bn_bwd")


def iseg_weight_update(master, g, g_exp, lr_shift, master_exp, k_U, k_W, w_q, status=None):
    rc = lib().iseg_weight_update(_ptr(master), master.numel(), _ptr(g), _ptr(g_exp), lr_shift,
                                  master_exp, k_U, k_W, _ptr(w_q), _ptr(status), _stream())
    _check(rc, "iseg_weight_update")


def iseg_bn_param_update(dgamma, dgamma_exp, dbeta, dbeta_exp, bits, seed, tid_gamma, tid_beta, step,
                         lr_shift, master_exp, k_U, k_W, gamma_m, beta_m, gamma_q, beta_q,
                         g_gamma=None, g_beta=None, g_gamma_exp=None, g_beta_exp=None, status=None):
    rc = lib().iseg_bn_param_update(_ptr(dgamma), _ptr(dgamma_exp), _ptr(dbeta), _ptr(dbeta_exp),
                                    dgamma.numel(), bits, seed, tid_gamma, tid_beta, step, lr_shift,
                                    master_exp, k_U, k_W, _ptr(gamma_m), _ptr(beta_m), _ptr(gamma_q),
                                    _ptr(beta_q), _ptr(g_gamma), _ptr(g_beta), _ptr(g_gamma_exp),
                                    _ptr(g_beta_exp), _ptr(status), _stream())
    _check(rc, "iseg_bn_param_update")


def iseg_update_multi(descs, n_desc, bits, seed, step, lr_shift, k_U, k_W, status=None):
    rc = lib().iseg_update_multi(_ptr(descs), n_desc, bits, seed, step, lr_shift, k_U, k_W, _ptr(status),
                                 _stream())
    _check(rc, "iseg_update_multi")


def iseg_weight_quant(master, k_U, k_W, w_q):
    rc = lib().iseg_weight_quant(_ptr(master), master.numel(), k_U, k_W, _ptr(w_q), _stream())
    _check(rc, "iseg_weight_quant")


def iseg_maxpool_fwd(x, x_exp, k, stride, pad, y, y_exp):
    N, H, W, Cc = x.shape
    rc = lib().iseg_maxpool_fwd(_ptr(x), _ptr(x_exp), N, H, W, Cc, k, stride, pad, _ptr(y),
                                _ptr(y_exp), _stream())
    _check(rc, "iseg_maxpool_fwd")


def iseg_maxpool_bwd(dy, dy_exp, x, k, stride, pad, bits, dx, dx_exp, ws, status=None):
    N, H, W, Cc = x.shape
    rc = lib().iseg_maxpool_bwd(_ptr(dy), _ptr(dy_exp), _ptr(x), N, H, W, Cc, k, stride, pad, bits,
                                _ptr(dx), _ptr(dx_exp), *_ws_tuple(ws), _ptr(status), _stream())
    _check(rc, "iseg_maxpool_bwd")


def _ptr_array(ts):
    if _REC is not None:
        _REC.keep.extend(t for t in ts if t is not None)
    return (C.c_void_p * len(ts))(*[None if t is None else t.data_ptr() for t in ts])


def _i32_array(v):
    return (C.c_int32 * len(v))(*[int(x) for x in v])


def _i64_array(v):
    return (C.c_int64 * len(v))(*[int(x) for x in v])


def iseg_sum_requant(ins, in_exps, exp_add, bcast, N, HW, Cc, relu, bits, out, out_exp, ws,
                     status=None):
    n = len(ins)
    rc = lib().iseg_sum_requant(n, _ptr_array(ins), _ptr_array(in_exps),
                                _i32_array(exp_add or [0] * n), _i32_array(bcast or [0] * n),
                                N, HW, Cc, relu, bits, _ptr(out), _ptr(out_exp), *_ws_tuple(ws),
                                _ptr(status), _stream())
    _check(rc, "iseg_sum_requant")


def iseg_sum_requant_relu_mask(ins, in_exps, exp_add, N, HW, Cc, bits, masks, mask_exps, out, out_exp, ws,
                               status=None):
    n = len(ins)
    rc = lib().iseg_sum_requant_relu_mask(n, _ptr_array(ins), _ptr_array(in_exps), _i32_array(exp_add or [0] * n),
                                          N, HW, Cc, bits, len(masks), _ptr_array(masks), _ptr_array(mask_exps),
                                          _ptr(out), _ptr(out_exp), *_ws_tuple(ws), _ptr(status), _stream())
    _check(rc, "iseg_sum_requant_relu_mask")


def iseg_relu_mask_bwd(dy, ins, in_exps, exp_add, Cc, dx, status=None):
    n = len(ins)
    rc = lib().iseg_relu_mask_bwd(_ptr(dy), n, _ptr_array(ins), _ptr_array(in_exps),
                                  _i32_array(exp_add or [0] * n), dy.numel(), Cc, _ptr(dx),
                                  _ptr(status), _stream())
    _check(rc, "iseg_relu_mask_bwd")


def iseg_concat_requant(ins, in_exps, widths, bcast, N, HW, bits, out, out_exp, ws, status=None):
    n = len(ins)
    rc = lib().iseg_concat_requant(n, _ptr_array(ins), _ptr_array(in_exps), _i64_array(widths),
                                   _i32_array(bcast or [0] * n), N, HW, bits, _ptr(out),
                                   _ptr(out_exp), *_ws_tuple(ws), _ptr(status), _stream())
    _check(rc, "iseg_concat_requant")


def iseg_concat_split(dy, rows, widths, outs):
    rc = lib().iseg_concat_split(_ptr(dy), rows, len(widths), _i64_array(widths), _ptr_array(outs),
                                 _stream())
    _check(rc, "iseg_concat_split")


def iseg_spatial_sum(x, x_exp, N, HW, ldc, c0, Cc, divisor, bits, out, out_exp, ws, status=None):
    rc = lib().iseg_spatial_sum(_ptr(x), _ptr(x_exp), N, HW, ldc, c0, Cc, divisor, bits, _ptr(out),
                                _ptr(out_exp), *_ws_tuple(ws), _ptr(status), _stream())
    _check(rc, "iseg_spatial_sum")


def iseg_softmax_ce(logits, logit_exp, labels, N, h, w, K, H, W, bits, loss, grad, err, err_exp,
                    ws, status=None):
    rc = lib().iseg_softmax_ce(_ptr(logits), _ptr(logit_exp), _ptr(labels), N, h, w, K, H, W, bits,
                               _ptr(loss), _ptr(grad), _ptr(err), _ptr(err_exp), *_ws_tuple(ws),
                               _ptr(status), _stream())
    _check(rc, "iseg_softmax_ce")


def iseg_mse_onehot(y, y_exp, labels, bits, loss, err, err_exp, ws, status=None):
    N, H, W, K = y.shape
    rc = lib().iseg_mse_onehot(_ptr(y), _ptr(y_exp), _ptr(labels), N, H, W, K, bits, _ptr(loss), _ptr(err),
                               _ptr(err_exp), *_ws_tuple(ws), _ptr(status), _stream())
    _check(rc, "iseg_mse_onehot")


def mse_onehot(y, y_exp, labels, bits=8, status=None):
    """(loss, E1 codes, exponent) of the MSE loss against one-hot labels."""
    loss = torch.empty(1, dtype=torch.float64, device=y.device)     # written whole by the kernel
    err = torch.empty_like(y)
    e = _out_exp(y.device)
    ws = workspace(y.device).get(lib().iseg_mse_onehot_ws(y.numel()))
    iseg_mse_onehot(y, y_exp, labels, bits, loss, err, e, ws, status)
    return loss, err, e


def iseg_layernorm_fwd(x, gamma, beta, geom, y, mean, rstd, status=None):
    rc = lib().iseg_layernorm_fwd(_ptr(x), _ptr(gamma), _ptr(beta), C.byref(geom), _ptr(y), _ptr(mean),
                                  _ptr(rstd), _ptr(status), _stream())
    _check(rc, "iseg_layernorm_fwd")


def iseg_layernorm_bwd(dy, x, gamma, mean, rstd, geom, dx, dgamma, dbeta, ws):
    rc = lib().iseg_layernorm_bwd(_ptr(dy), _ptr(x), _ptr(gamma), _ptr(mean), _ptr(rstd), C.byref(geom), _ptr(dx),
                                  _ptr(dgamma), _ptr(dbeta), *_ws_tuple(ws), _stream())
    _check(rc, "iseg_layernorm_bwd")


def iseg_quantize_rows(x, x_dtype, M, Cc, x_ld, mul, bits, scale_mode, codes, codes_ld, scale, status=None):
    rc = lib().iseg_quantize_rows(_ptr(x), x_dtype, M, Cc, x_ld, _ptr(mul), bits, scale_mode, _ptr(codes),
                                  codes_ld, _ptr(scale), _ptr(status), _stream())
    _check(rc, "iseg_quantize_rows")


def iseg_quantize_cols(x, x_dtype, M, Cc, x_ld, mul, bits, scale_mode, codes, codes_ld, scale, sums, ws,
                       status=None):
    rc = lib().iseg_quantize_cols(_ptr(x), x_dtype, M, Cc, x_ld, _ptr(mul), bits, scale_mode, _ptr(codes),
                                  codes_ld, _ptr(scale), _ptr(sums), *_ws_tuple(ws), _ptr(status), _stream())
    _check(rc, "iseg_quantize_cols")


def iseg_transpose_i8(inp, M, Cc, in_ld, out, out_ld):
    rc = lib().iseg_transpose_i8(_ptr(inp), M, Cc, in_ld, _ptr(out), out_ld, _stream())
    _check(rc, "iseg_transpose_i8")


def iseg_matmul_i8(a, a_scale, b, b_scale, bias, geom, out, ws):
    rc = lib().iseg_matmul_i8(_ptr(a), _ptr(a_scale), _ptr(b), _ptr(b_scale), _ptr(bias), C.byref(geom), _ptr(out),
                              *_ws_tuple(ws), _stream())
    _check(rc, "iseg_matmul_i8")


def iseg_linear_i8_fwd(x, w, w_scale, bias, geom, codes, scale, y, ws, status=None):
    rc = lib().iseg_linear_i8_fwd(_ptr(x), _ptr(w), _ptr(w_scale), _ptr(bias), C.byref(geom), _ptr(codes),
                                  _ptr(scale), _ptr(y), *_ws_tuple(ws), _ptr(status), _stream())
    _check(rc, "iseg_linear_i8_fwd")


def iseg_linear_i8_bwd(dy, a, a_scale, w, w_scale, w_t, geom, dx, dw, dbias, ws, status=None):
    rc = lib().iseg_linear_i8_bwd(_ptr(dy), _ptr(a), _ptr(a_scale), _ptr(w), _ptr(w_scale), _ptr(w_t), C.byref(geom),
                                  _ptr(dx), _ptr(dw), _ptr(dbias), *_ws_tuple(ws), _ptr(status), _stream())
    _check(rc, "iseg_linear_i8_bwd")


def iseg_logprob_fwd(logits, tokens, geom, logprob, lse, entropy, top_ids, top_logprob, ws, status=None):
    rc = lib().iseg_logprob_fwd(_ptr(logits), _ptr(tokens), C.byref(geom), _ptr(logprob), _ptr(lse), _ptr(entropy),
                                _ptr(top_ids), _ptr(top_logprob), *_ws_tuple(ws), _ptr(status), _stream())
    _check(rc, "iseg_logprob_fwd")


def iseg_logprob_bwd(logits, tokens, lse, entropy, g_logprob, g_entropy, geom, dlogits, status=None):
    rc = lib().iseg_logprob_bwd(_ptr(logits), _ptr(tokens), _ptr(lse), _ptr(entropy), _ptr(g_logprob),
                                _ptr(g_entropy), C.byref(geom), _ptr(dlogits), _ptr(status), _stream())
    _check(rc, "iseg_logprob_bwd")


def iseg_page_map(ctx, count, held, free_pages, n_free, geom, table, q_start, kv_len, positions, slots, held_out,
                  n_free_out, ws, status=None):
    rc = lib().iseg_page_map(_ptr(ctx), _ptr(count), _ptr(held), _ptr(free_pages), _ptr(n_free), C.byref(geom),
                             _ptr(table), _ptr(q_start), _ptr(kv_len), _ptr(positions), _ptr(slots), _ptr(held_out),
                             _ptr(n_free_out), *_ws_tuple(ws), _ptr(status), _stream())
    _check(rc, "iseg_page_map")


def iseg_qk_norm_rope_fwd(q, k, positions, inv_freq, gamma_q, gamma_k, geom, yq, yk, status=None):
    rc = lib().iseg_qk_norm_rope_fwd(_ptr(q), _ptr(k), _ptr(positions), _ptr(inv_freq), _ptr(gamma_q), _ptr(gamma_k),
                                     C.byref(geom), _ptr(yq), _ptr(yk), _ptr(status), _stream())
    _check(rc, "iseg_qk_norm_rope_fwd")


def iseg_qk_norm_rope_bwd(dyq, dyk, q, k, positions, inv_freq, gamma_q, gamma_k, geom, dq, dk, dgamma_q, dgamma_k,
                          ws):
    rc = lib().iseg_qk_norm_rope_bwd(_ptr(dyq), _ptr(dyk), _ptr(q), _ptr(k), _ptr(positions), _ptr(inv_freq),
                                     _ptr(gamma_q), _ptr(gamma_k), C.byref(geom), _ptr(dq), _ptr(dk), _ptr(dgamma_q),
                                     _ptr(dgamma_k), *_ws_tuple(ws), _stream())
    _check(rc, "iseg_qk_norm_rope_bwd")


def iseg_kv4_write(k, v, slots, geom, k_codes, k_scale, v_codes, v_scale, status=None):
    rc = lib().iseg_kv4_write(_ptr(k), _ptr(v), _ptr(slots), C.byref(geom), _ptr(k_codes), _ptr(k_scale),
                              _ptr(v_codes), _ptr(v_scale), _ptr(status), _stream())
    _check(rc, "iseg_kv4_write")


def iseg_kv4_read(k_codes, k_scale, v_codes, v_scale, slots, geom, k, v, status=None):
    rc = lib().iseg_kv4_read(_ptr(k_codes), _ptr(k_scale), _ptr(v_codes), _ptr(v_scale), _ptr(slots), C.byref(geom),
                             _ptr(k), _ptr(v), _ptr(status), _stream())
    _check(rc, "iseg_kv4_read")


def iseg_kv4_attention(q, k_codes, k_scale, v_codes, v_scale, table, q_start, kv_len, geom, out, lse, ws,
                       status=None):
    rc = lib().iseg_kv4_attention(_ptr(q), _ptr(k_codes), _ptr(k_scale), _ptr(v_codes), _ptr(v_scale), _ptr(table),
                                  _ptr(q_start), _ptr(kv_len), C.byref(geom), _ptr(out), _ptr(lse), *_ws_tuple(ws),
                                  _ptr(status), _stream())
    _check(rc, "iseg_kv4_attention")


def iseg_verify_drafts(target, draft, tokens, n_draft, u, u_sample, geom, out, accepted, ws, status=None):
    rc = lib().iseg_verify_drafts(_ptr(target), _ptr(draft), _ptr(tokens), _ptr(n_draft), _ptr(u), _ptr(u_sample),
                                  C.byref(geom), _ptr(out), _ptr(accepted), *_ws_tuple(ws), _ptr(status), _stream())
    _check(rc, "iseg_verify_drafts")


def iseg_philox4x32_10(ctr, key):
    c = (C.c_uint32 * 4)(*ctr)
    k = (C.c_uint32 * 2)(*key)
    o = (C.c_uint32 * 4)()
    lib().iseg_philox4x32_10(c, k, o)
    return list(o)


def iseg_conv_last_plan():
    return lib().iseg_conv_last_plan().decode()


def iseg_status_read(status):
    v = C.c_int32(0)
    _check(lib().iseg_status_read(_ptr(status), C.byref(v), _stream()), "iseg_status_read")
    return v.value


def iseg_status_clear(status):
    _check(lib().iseg_status_clear(_ptr(status), _stream()), "iseg_status_clear")


def iseg_check_codes(x, bits, status):
    _check(lib().iseg_check_codes(_ptr(x), x.numel(), bits, _ptr(status), _stream()), "iseg_check_codes")


def iseg_version():
    return lib().iseg_version().decode()


def iseg_profile_arm(kernel_id, start_event, stop_event):
    _check(lib().iseg_profile_arm(kernel_id, start_event, stop_event), "iseg_profile_arm")


# --------------------------------------------------------------------------
# in-place kernel timing (HIP events recorded around one kernel launch)
# --------------------------------------------------------------------------
_hip = None


def _hiprt():
    global _hip
    if _hip is None:
        h = C.CDLL("libamdhip64.so")
        h.hipEventCreate.argtypes = [C.POINTER(C.c_void_p)]
        h.hipEventElapsedTime.argtypes = [C.POINTER(C.c_float), C.c_void_p, C.c_void_p]
        h.hipEventSynchronize.argtypes = [C.c_void_p]
        h.hipEventDestroy.argtypes = [C.c_void_p]
        _hip = h
    return _hip


class KernelTimer:
    """Times every launch of one or more kernel families whose layer key
    matches, with a pair of HIP events that the library records around the
    launch on its own stream (iseg_profile_arm).  Families timed together
    must be separate entry-point calls (one arming is held at a time)."""

    def __init__(self, kernel_id, layer_match=None):
        self.kids = set(kernel_id) if isinstance(kernel_id, (tuple, list, set)) else {kernel_id}
        self.kid = next(iter(self.kids))
        self.match = tuple(layer_match) if layer_match is not None else None
        self.pairs = []                  # (start, stop, kernel id, layer key)
        self.free = []                   # created events not in use

    def wants(self, kid, key):
        return kid in self.kids and (self.match is None or tuple(key) == self.match)

    def _event(self):
        if self.free:
            return self.free.pop()
        e = C.c_void_p()
        if _hiprt().hipEventCreate(C.byref(e)):
            raise IsegError("hipEventCreate failed")
        return e

    def arm(self, kid=None, key=None):
        a, b = self._event(), self._event()
        kid = self.kid if kid is None else kid
        self.pairs.append((a, b, kid, tuple(key) if key is not None else None))
        iseg_profile_arm(kid, a, b)

    def reset(self):
        """Forget the timed launches and keep their events for the next ones
        (an untimed pass with the timer installed creates the events a timed
        region then reuses, keeping event creation out of it)."""
        h = _hiprt()
        for a, b, _, _ in self.pairs:
            h.hipEventSynchronize(b)
            self.free += [a, b]
        self.pairs = []

    def launches(self):
        """[(kernel id, layer key, ms)] of every timed launch."""
        h = _hiprt()
        out = []
        for a, b, kid, key in self.pairs:
            h.hipEventSynchronize(b)
            ms = C.c_float()
            if h.hipEventElapsedTime(C.byref(ms), a, b) == 0:
                out.append((kid, key, ms.value))
        return out

    def times_ms(self):
        return [t for _, _, t in self.launches()]

    def mean_ms(self):
        t = self.times_ms()
        return sum(t) / len(t) if t else None

    def count(self):
        return len(self.pairs)

    def close(self):
        h = _hiprt()
        for a, b, _, _ in self.pairs:
            h.hipEventDestroy(a)
            h.hipEventDestroy(b)
        for e in self.free:
            h.hipEventDestroy(e)
        self.pairs, self.free = [], []


_TIMER = None


def set_kernel_timer(timer):
    """Install (or remove, with None) the timer consulted by the helpers below."""
    global _TIMER
    if timer is None:
        iseg_profile_arm(ISEG_KID_NONE, None, None)
    _TIMER = timer


def _maybe_arm(kid, key):
    if _TIMER is not None and _TIMER.wants(kid, key):
        _TIMER.arm(kid, key)


# --------------------------------------------------------------------------
# workspace and helpers (allocation with torch; compute in the entry points)
# --------------------------------------------------------------------------
class Workspace:
    """A growable device scratch buffer shared by one thread's consecutive calls
    on one stream (stream order keeps the uses apart).  Each stream has its own,
    and each host thread: a call enqueues several kernels that hand data on
    through it, and the kernels of two threads' calls on one stream may
    alternate."""

    def __init__(self, device="cuda"):
        self.device = device
        self.buf = None
        self.views = {}              # recent sizes' views of buf (a slice costs 2 us of host time)

    def get(self, nbytes):
        nbytes = max(int(nbytes), 256)
        v = self.views.get(nbytes)
        if v is None:
            if self.buf is None or self.buf.numel() < nbytes:
                self.buf = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
                self.views = {}
            elif len(self.views) >= 64:
                self.views = {}
            v = self.views[nbytes] = self.buf[:nbytes]
        return v


class _ThreadWorkspaces(threading.local):
    def __init__(self):
        self.of = {}


_WS = _ThreadWorkspaces()


def workspace(device):
    """The calling thread's workspace of the current stream."""
    d = device if isinstance(device, torch.device) else torch.device(device)
    if d.type == "cuda":
        idx = d.index if d.index is not None else _raw_device()
        key = (idx, _stream_handle(idx))
    else:
        idx, key = None, (str(d), 0)
    mine = _WS.of
    ws = mine.get(key)
    if ws is None:
        ws = mine[key] = Workspace(torch.device("cuda", idx) if d.type == "cuda" else d)
    return ws


# --------------------------------------------------------------------------
# step tape: the calls of one step recorded, then replayed from native code
# --------------------------------------------------------------------------
_REC = None

# parameter index of the step counter (stochastic rounding, Eq. 5-6)
_STEP_ARG = {"iseg_conv_bwd_weight": 9, "iseg_update_multi": 4, "iseg_bn_param_update": 9, "iseg_requant": 9}
_U64_MASK = (1 << 64) - 1


def iseg_tape_create():
    return C.c_void_p(lib().iseg_tape_create())


def iseg_tape_destroy(h):
    lib().iseg_tape_destroy(h)


def iseg_tape_entry(name):
    return int(lib().iseg_tape_entry(name.encode()))


def iseg_tape_entry_nargs(entry):
    return int(lib().iseg_tape_entry_nargs(entry))


def iseg_tape_add_call(h, entry, words, blob, blob_words, step_word, step_base):
    w = (C.c_uint64 * max(len(words), 1))(*words)
    bw = (C.c_int32 * max(len(blob_words), 1))(*blob_words)
    b = (C.c_char * max(len(blob), 1)).from_buffer_copy(bytes(blob) or b"\0")
    _check(lib().iseg_tape_add_call(h, entry, w, len(words), b, len(blob), bw, len(blob_words), step_word,
                                    step_base), "iseg_tape_add_call")


def iseg_tape_add_record(h, slot, stream_handle):
    _check(lib().iseg_tape_add_record(h, slot, C.c_void_p(stream_handle)), "iseg_tape_add_record")


def iseg_tape_add_wait(h, stream_handle, slot):
    _check(lib().iseg_tape_add_wait(h, C.c_void_p(stream_handle), slot), "iseg_tape_add_wait")


def iseg_tape_arm_count(h):
    return int(lib().iseg_tape_arm_count(h))


def iseg_tape_set_arm_events(h, events, runs):
    """events: (start, stop) pairs of hipEvent_t handles, runs x armed calls of them."""
    flat = (C.c_void_p * max(len(events) * 2, 1))(*[e for pair in events for e in pair])
    _check(lib().iseg_tape_set_arm_events(h, flat, runs), "iseg_tape_set_arm_events")


def iseg_tape_run(h, step):
    failed = C.c_int64(-1)
    rc = lib().iseg_tape_run(h, int(step) & 0xFFFFFFFF, C.byref(failed))
    if rc != ISEG_OK:
        raise IsegError(f"iseg_tape_run: operation {failed.value} returned {_ERRS.get(rc, rc)}")


def iseg_tape_size(h):
    return int(lib().iseg_tape_size(h))


class _RecLib:
    """The library as seen while a tape records: each call of a tape entry
    point runs, then is appended to the tape."""

    def __init__(self, tape):
        self._tape = tape

    def __getattr__(self, name):
        f = getattr(_lib, name)
        if not name.startswith("iseg_") or name.startswith("iseg_tape_") or name not in self._tape.entries:
            return f
        tape = self._tape

        def call(*args):
            rc = f(*args)
            if rc == ISEG_OK:
                tape.add_call(name, args)
            return rc
        return call


class Tape:
    """One training step's library calls and stream orderings, recorded while
    the step runs inside `with tape:` (every call of a tape entry point made
    then is appended after it returns ISEG_OK), replayed from native code by
    run(step).  Keeps every buffer the recorded calls use allocated; the
    caller keeps the streams alive and replays with the same stream setup, in
    the order of the recording thread's own calls on these streams, whose
    workspaces the recorded calls share.  Calls of other threads are recorded
    too: only one thread calls while a tape records.""" 

    def __init__(self, step):
        L = lib()
        self.h = iseg_tape_create()
        if not self.h.value:
            raise IsegError("iseg_tape_create failed")
        self.step = int(step)
        self.keep = []
        self.slots = 0
        self.arms = []
        self.entries = {n: L.iseg_tape_entry(n.encode()) for n in _SIGS if n.startswith("iseg_")}
        self.entries = {n: e for n, e in self.entries.items() if e >= 0}
        self.lib = _RecLib(self)

    def __enter__(self):
        global _REC
        if _REC is not None:
            raise IsegError("a tape is already recording")
        _REC = self
        return self

    def __exit__(self, *exc):
        global _REC
        _REC = None
        return False

    def add_call(self, name, args):
        argtypes = getattr(_lib, name).argtypes
        words, blob, blob_words = [], bytearray(), []
        for i, a in enumerate(args):
            if a is None:
                words.append(0)
            elif isinstance(a, C.c_void_p):
                words.append(a.value or 0)
            elif type(a).__name__ == "CArgObject" or isinstance(a, C.Array):
                obj = a._obj if type(a).__name__ == "CArgObject" else a
                blob_words.append(i)
                words.append(len(blob))
                blob += C.string_at(C.addressof(obj), C.sizeof(obj))
                blob += bytes(-len(blob) % 8)
            elif isinstance(a, C._SimpleCData):
                words.append(int(a.value) & _U64_MASK)
            elif isinstance(a, int):
                words.append(a & _U64_MASK)
            else:
                raise IsegError(f"{name}: argument {i} of type {type(a).__name__} cannot be recorded")
            if argtypes[i] is not _P and isinstance(a, C.c_void_p):
                raise IsegError(f"{name}: argument {i} is a pointer where an integer is declared")
        sw = _STEP_ARG.get(name, -1)
        base = int(args[sw].value if isinstance(args[sw], C._SimpleCData) else args[sw]) - self.step if sw >= 0 else 0
        if name == "iseg_profile_arm":
            self.arms.append(int(args[0]))
        iseg_tape_add_call(self.h, self.entries[name], words, blob, blob_words, sw, base)

    def new_slot(self):
        self.slots += 1
        return self.slots - 1

    def add_record(self, slot, stream_handle):
        iseg_tape_add_record(self.h, slot, stream_handle)

    def add_wait(self, stream_handle, slot):
        iseg_tape_add_wait(self.h, stream_handle, slot)

    def set_arm_events(self, events, runs):
        """events: runs x (armed calls) (start, stop) pairs of hipEvent_t handles."""
        iseg_tape_set_arm_events(self.h, events, runs)

    def size(self):
        return iseg_tape_size(self.h)

    def run(self, step):
        iseg_tape_run(self.h, step)

    def close(self):
        if self.h is not None and self.h.value:
            iseg_tape_destroy(self.h)
        self.h = None
        self.keep = []

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _out_exp(device):
    """Exponent slot for a kernel to write (no initialization kernel)."""
    return torch.empty(1, dtype=torch.int32, device=device)


def new_exp(device="cuda", value=0):
    return torch.full((1,), int(value), dtype=torch.int32, device=device)


def geom(N, H, W, Cc, K, R, S, stride=1, pad=0, dil=1):
    st = stride if isinstance(stride, (tuple, list)) else (stride, stride)
    pd = pad if isinstance(pad, (tuple, list)) else (pad, pad)
    dl = dil if isinstance(dil, (tuple, list)) else (dil, dil)
    return ConvGeom(N, H, W, Cc, K, R, S, st[0], st[1], pd[0], pd[1], dl[0], dl[1])


def conv_out_hw(g):
    P = (g.H + 2 * g.pad_h - g.dil_h * (g.R - 1) - 1) // g.stride_h + 1
    Q = (g.W + 2 * g.pad_w - g.dil_w * (g.S - 1) - 1) // g.stride_w + 1
    return P, Q


def bn_cfg(**kw):
    d = dict(BN_DEFAULT)
    d.update(kw)
    return BnCfg(*[d[k] for k in ("k_mu", "k_sigma", "k_xhat", "k_gamma", "k_beta", "k_A", "k_E1",
                                  "k_E2", "eps_code", "relu")])


def quantize(x, bits, mode=ISEG_Q_SQ, status=None, out_dtype=None):
    """Codes in the narrowest of int8 / int16 / int32 that holds `bits`, or in
    out_dtype (a torch integer dtype at least that wide)."""
    w = 8 if bits <= 8 else 16 if bits <= 16 else 32
    if out_dtype is not None:
        w = {torch.int8: 8, torch.int16: 16, torch.int32: 32}[out_dtype]
        if (w == 8 and bits > 8) or (w == 16 and bits > 16):
            raise ValueError("out_dtype too narrow for bits")
    dt = {8: (torch.int8, ISEG_I8), 16: (torch.int16, ISEG_I16), 32: (torch.int32, ISEG_I32)}[w]
    out = torch.empty(x.shape, dtype=dt[0], device=x.device)
    e = _out_exp(x.device)
    ws = workspace(x.device).get(lib().iseg_quantize_ws(x.numel()))
    iseg_quantize(x.contiguous(), bits, mode, dt[1], out, e, ws, status)
    return out, e


def requant(acc, acc_exp, bits=8, stochastic=False, keep_scale=True, seed=0, tensor_id=0, step=0,
            status=None):
    in_dt = {torch.int32: ISEG_I32, torch.int64: ISEG_I64}[acc.dtype]
    od, odt = (torch.int8, ISEG_I8) if bits <= 8 else (torch.int16, ISEG_I16)
    out = torch.empty(acc.shape, dtype=od, device=acc.device)
    e = _out_exp(acc.device)
    ws = workspace(acc.device).get(lib().iseg_requant_ws(acc.numel()))
    iseg_requant(acc.contiguous(), in_dt, acc_exp, bits, int(stochastic), int(keep_scale), seed,
                 tensor_id, step, odt, out, e, ws, status)
    return out, e


def conv_fwd(x, x_exp, w, w_exp, stride=1, pad=0, dil=1, out_mode=ISEG_OUT_Q8, status=None):
    N, H, W, Cc = x.shape
    K, R, S, _ = w.shape
    g = geom(N, H, W, Cc, K, R, S, stride, pad, dil)
    P, Q = conv_out_hw(g)
    y = torch.empty((N, P, Q, K), dtype=torch.int8 if out_mode == ISEG_OUT_Q8 else torch.int32,
                    device=x.device)
    e = _out_exp(x.device)
    ws = workspace(x.device).get(lib().iseg_conv_fwd_ws(C.byref(g), out_mode))
    _maybe_arm(ISEG_KID_CONV_FWD, (N, H, W, Cc, K, R, g.stride_h, g.pad_h, g.dil_h))
    iseg_conv_fwd(x, x_exp, w, w_exp, g, out_mode, y, e, ws, status)
    return y, e


def conv_bwd_data(dy, dy_exp, w, w_exp, x_shape, stride=1, pad=0, dil=1, out_mode=ISEG_OUT_Q8,
                  status=None, wt=None, wt_kind=ISEG_WT_NONE):
    N, H, W, Cc = x_shape
    K, R, S, _ = w.shape
    g = geom(N, H, W, Cc, K, R, S, stride, pad, dil)
    dx = torch.empty((N, H, W, Cc), dtype=torch.int8 if out_mode == ISEG_OUT_Q8 else torch.int32,
                     device=dy.device)
    e = _out_exp(dy.device)
    ws = workspace(dy.device).get(lib().iseg_conv_bwd_data_ws(C.byref(g), out_mode))
    _maybe_arm(ISEG_KID_CONV_BWD_DATA, (N, H, W, Cc, K, R, g.stride_h, g.pad_h, g.dil_h))
    if wt is None:
        iseg_conv_bwd_data(dy, dy_exp, w, w_exp, g, out_mode, dx, e, ws, status)
    else:
        iseg_conv_bwd_data_t(dy, dy_exp, w, w_exp, wt, wt_kind, g, out_mode, dx, e, ws, status)
    return dx, e


def conv_bwd_weight(dy, dy_exp, x, x_exp, w_shape, stride=1, pad=0, dil=1, g_mode=ISEG_G_KEEP,
                    bits=8, seed=0, tensor_id=0, step=0, status=None, out=None):
    N, H, W, Cc = x.shape
    K, R, S, _ = w_shape
    g = geom(N, H, W, Cc, K, R, S, stride, pad, dil)
    if out is None:
        dw = torch.empty((K, R, S, Cc), dtype=torch.int64 if g_mode == ISEG_G_RAW else torch.int8,
                         device=x.device)
        e = _out_exp(x.device)
    else:
        dw, e = out
    ws = workspace(x.device).get(lib().iseg_conv_bwd_weight_ws(C.byref(g), g_mode))
    _maybe_arm(ISEG_KID_CONV_WGRAD, (N, H, W, Cc, K, R, g.stride_h, g.pad_h, g.dil_h))
    iseg_conv_bwd_weight(dy, dy_exp, x, x_exp, g, g_mode, bits, seed, tensor_id, step, dw, e, ws,
                         status)
    return dw, e


def bn_fwd(x, x_exp, gamma_q, beta_q, cfg=None, saved=None, status=None):
    """L1BN forward of int8 codes, or of int32 raw conv sums (the wide input)."""
    Cc = x.shape[-1]
    M = x.numel() // Cc
    cfg = cfg or bn_cfg()
    if x.dtype == torch.int32:
        y = torch.empty(x.shape, dtype=torch.int8, device=x.device)
        e = _out_exp(x.device)
        if saved is None:
            saved = torch.empty(lib().iseg_bn_i32_saved_bytes(Cc), dtype=torch.uint8, device=x.device)
        ws = workspace(x.device).get(lib().iseg_bn_fwd_i32_ws(M, Cc))
        iseg_bn_fwd_i32(x, x_exp, M, Cc, gamma_q, beta_q, cfg, y, e, saved, ws, status)
        return y, e, saved
    y = torch.empty_like(x)
    e = _out_exp(x.device)
    if saved is None:
        saved = torch.empty(lib().iseg_bn_saved_bytes(Cc), dtype=torch.uint8, device=x.device)
    ws = workspace(x.device).get(lib().iseg_bn_fwd_ws(M, Cc))
    for kid in (ISEG_KID_BN_FWD_APPLY, ISEG_KID_BN_FWD_STATS1, ISEG_KID_BN_FWD_STATS2):
        _maybe_arm(kid, (M, Cc))
    iseg_bn_fwd(x, x_exp, M, Cc, gamma_q, beta_q, cfg, y, e, saved, ws, status)
    return y, e, saved


def bn_bwd(dy, dy_exp, x, gamma_q, saved, cfg=None, status=None, dgb_out=None):
    Cc = x.shape[-1]
    M = x.numel() // Cc
    cfg = cfg or bn_cfg()
    dx = torch.empty(x.shape, dtype=torch.int8, device=x.device)
    e = _out_exp(x.device)
    if dgb_out is None:
        dg = torch.empty(Cc, dtype=torch.int64, device=x.device)
        db = torch.empty(Cc, dtype=torch.int64, device=x.device)
        dge, dbe = _out_exp(x.device), _out_exp(x.device)
    else:
        dg, db, dge, dbe = dgb_out
    if x.dtype == torch.int32:
        ws = workspace(x.device).get(lib().iseg_bn_bwd_i32_ws(M, Cc))
        iseg_bn_bwd_i32(dy, dy_exp, x, M, Cc, gamma_q, cfg, saved, dx, e, dg, db, dge, dbe, ws, status)
        return dx, e, dg, db, dge, dbe
    ws = workspace(x.device).get(lib().iseg_bn_bwd_ws(M, Cc))
    for kid in (ISEG_KID_BN_BWD_APPLY, ISEG_KID_BN_BWD_STATS):
        _maybe_arm(kid, (M, Cc))
    iseg_bn_bwd(dy, dy_exp, x, M, Cc, gamma_q, cfg, saved, dx, e, dg, db, dge, dbe, ws, status)
    return dx, e, dg, db, dge, dbe


def bn_saved_view(saved, Cc):
    """Named views of the saved-state buffer (layout of iseg.h)."""
    def al(v):
        return (v + 255) // 256 * 256
    off = 256
    out = {"hdr": saved[:64].view(torch.int32)}
    for name in ("n_mu", "n_sigma", "den", "qmin", "qmax", "t0", "p0", "mlo", "mhi"):
        out[name] = saved[off:off + 4 * Cc].view(torch.int32)
        off += al(4 * Cc)
    out["xcode"] = saved[off:off + 512 * Cc].view(torch.int16).view(Cc, 256)
    off += al(512 * Cc)
    out["flags"] = saved[off:off + 256 * Cc].view(Cc, 256)
    off += al(256 * Cc)
    out["acode"] = saved[off:off + 256 * Cc].view(torch.int8).view(Cc, 256)
    off += al(256 * Cc)
    out["bwd_entry"] = saved[off:off + 1024 * Cc].view(torch.int32).view(Cc, 256)
    return out


def weight_update(master, g, g_exp, lr_shift, master_exp=-23, k_U=24, k_W=8, w_q=None, status=None):
    if w_q is None:
        w_q = torch.empty(master.shape, dtype=torch.int8, device=master.device)
    iseg_weight_update(master, g, g_exp, lr_shift, master_exp, k_U, k_W, w_q, status)
    return w_q


def weight_quant(master, k_U=24, k_W=8):
    w_q = torch.empty(master.shape, dtype=torch.int8, device=master.device)
    iseg_weight_quant(master, k_U, k_W, w_q)
    return w_q


def maxpool_fwd(x, x_exp, k, stride, pad=0):
    N, H, W, Cc = x.shape
    P = (H + 2 * pad - k) // stride + 1
    Q = (W + 2 * pad - k) // stride + 1
    y = torch.empty((N, P, Q, Cc), dtype=torch.int8, device=x.device)
    e = _out_exp(x.device)
    iseg_maxpool_fwd(x, x_exp, k, stride, pad, y, e)
    return y, e


def maxpool_bwd(dy, dy_exp, x, k, stride, pad=0, bits=8, status=None):
    N, H, W, Cc = x.shape
    dx = torch.empty_like(x)
    e = _out_exp(x.device)
    ws = workspace(x.device).get(lib().iseg_maxpool_bwd_ws(N, H, W, Cc))
    _maybe_arm(ISEG_KID_MAXPOOL_BWD, (N, H, W, Cc))
    iseg_maxpool_bwd(dy, dy_exp, x, k, stride, pad, bits, dx, e, ws, status)
    return dx, e


def sum_requant(ins, in_exps, relu=False, exp_add=None, bcast=None, bits=8, status=None):
    """SQ(ReLU?(sum of the inputs)); the first input fixes the shape [N,H,W,C]
    (a broadcast input is [N,1,1,C])."""
    ref = next(t for t, b in zip(ins, bcast or [0] * len(ins)) if not b)
    N, H, W, Cc = ref.shape
    out = torch.empty_like(ref)
    e = _out_exp(ref.device)
    ws = workspace(ref.device).get(lib().iseg_sum_requant_ws(N, H * W, Cc))
    iseg_sum_requant(ins, in_exps, exp_add, bcast, N, H * W, Cc, int(relu), bits, out, e, ws, status)
    return out, e


def sum_requant_relu_mask(ins, in_exps, masks, mask_exps, exp_add=None, bits=8, status=None):
    """sum_requant (no ReLU, no broadcast) followed by relu_mask_bwd with the
    mask inputs, in one call: (codes, exponent)."""
    N, H, W, Cc = ins[0].shape
    out = torch.empty_like(ins[0])
    e = _out_exp(ins[0].device)
    ws = workspace(ins[0].device).get(lib().iseg_sum_requant_ws(N, H * W, Cc))
    iseg_sum_requant_relu_mask(ins, in_exps, exp_add, N, H * W, Cc, bits, masks, mask_exps, out, e, ws, status)
    return out, e


def relu_mask_bwd(dy, ins, in_exps, status=None):
    dx = torch.empty_like(dy)
    iseg_relu_mask_bwd(dy, ins, in_exps, None, dy.shape[-1], dx, status)
    return dx


def concat_requant(ins, in_exps, bits=8, status=None):
    """Channel concatenation of [N,H,W,C_i] tensors (a [N,1,1,C_i] part is
    broadcast to H x W), SQ to `bits`."""
    N = ins[0].shape[0]
    H = max(t.shape[1] for t in ins)
    W = max(t.shape[2] for t in ins)
    widths = [t.shape[3] for t in ins]
    bc = [int(tuple(t.shape[1:3]) != (H, W)) for t in ins]
    out = torch.empty((N, H, W, sum(widths)), dtype=torch.int8, device=ins[0].device)
    e = _out_exp(ins[0].device)
    ws = workspace(ins[0].device).get(lib().iseg_concat_requant_ws(len(ins)))
    iseg_concat_requant(ins, in_exps, widths, bc, N, H * W, bits, out, e, ws, status)
    return out, e


def concat_split(dy, widths, skip=None):
    """Channel slices of dy (None where skip[i])."""
    N, H, W, _ = dy.shape
    outs = [None if (skip and skip[i]) else
            torch.empty((N, H, W, c), dtype=torch.int8, device=dy.device)
            for i, c in enumerate(widths)]
    iseg_concat_split(dy, N * H * W, widths, outs)
    return outs


def spatial_sum(x, x_exp, divisor=1, c0=0, Cc=None, bits=8, status=None):
    """SQ(sum over H x W of channels [c0, c0 + Cc) / divisor) -> [N,1,1,Cc]."""
    N, H, W, ldc = x.shape
    Cc = ldc - c0 if Cc is None else Cc
    out = torch.empty((N, 1, 1, Cc), dtype=torch.int8, device=x.device)
    e = _out_exp(x.device)
    ws = workspace(x.device).get(lib().iseg_spatial_sum_ws(N, H * W, Cc))
    iseg_spatial_sum(x, x_exp, N, H * W, ldc, c0, Cc, divisor, bits, out, e, ws, status)
    return out, e


def gap_fwd(x, x_exp, bits=8, status=None):
    """Global average pooling over H x W -> [N,1,1,C] (SQ of the exact mean)."""
    return spatial_sum(x, x_exp, x.shape[1] * x.shape[2], bits=bits, status=status)


def gap_bwd(dy, dy_exp, H, W, bits=8, status=None):
    """Backward of the mean over H x W: SQ(dy / (H W)), [N,1,1,C], to be
    broadcast over H x W by the consumer."""
    return spatial_sum(dy, dy_exp, H * W, bits=bits, status=status)


def softmax_ce(logits, logit_exp, labels, bits=8, want_grad=False, status=None):
    """Loss (device double), optional float64 gradient, and E1 = SQ(gradient)."""
    N, h, w, K = logits.shape
    _, H, W = labels.shape
    dev = logits.device
    loss = torch.empty(1, dtype=torch.float64, device=dev)
    grad = torch.empty((N, h, w, K), dtype=torch.float64, device=dev) if want_grad else None
    err = torch.empty((N, h, w, K), dtype=torch.int8, device=dev)
    e = _out_exp(dev)
    ws = workspace(dev).get(lib().iseg_softmax_ce_ws(N, h, w, K, H, W))
    iseg_softmax_ce(logits, logit_exp, labels, N, h, w, K, H, W, bits, loss, grad, err, e, ws, status)
    return loss, grad, err, e


def wt_kind(x_shape, w_shape, stride=1, pad=0, dil=1):
    """Transposed-weight layout the backward-data of this conv uses."""
    N, H, W, Cc = x_shape
    K, R, S, _ = w_shape
    return iseg_conv_bwd_data_wt_kind(geom(N, H, W, Cc, K, R, S, stride, pad, dil))


def wt_table(entries, device):
    """Device array of iseg_wt_desc for iseg_weight_transpose_multi.  entries:
    (w [K,R,S,C] int8, wt same size, kind); returns (table, n, total_tiles)."""
    n = len(entries)
    host = (WtDesc * max(n, 1))()
    tiles = 0
    for i, (w, wt, kind) in enumerate(entries):
        K, R, S, Cc = w.shape
        d = host[i]
        d.w, d.wt = w.data_ptr(), wt.data_ptr()
        d.K, d.RS, d.C, d.kind = K, R * S, Cc, kind
        d.tile_begin = tiles
        tiles += ((Cc + 63) // 64) * ((K + 63) // 64) * R * S
    raw = torch.frombuffer(bytearray(bytes(host)), dtype=torch.uint8)
    return raw.to(device), n, tiles


def update_table(entries, device):
    """Device array of iseg_update_desc for iseg_update_multi.  entries: dicts
    with master, w_q, g, g_exp, kind, master_exp and, for ISEG_UPD_RAW,
    tensor_id, g_q, g_q_exp (torch tensors; their storage must stay alive);
    optional k_w, the tensor's own Q_W width (0 = the call's k_W)."""
    n = len(entries)
    host = (UpdateDesc * max(n, 1))()
    for i, e in enumerate(entries):
        d = host[i]
        d.master = e["master"].data_ptr()
        d.w_q = e["w_q"].data_ptr()
        d.g = e["g"].data_ptr()
        d.g_exp = e["g_exp"].data_ptr()
        d.g_q = e["g_q"].data_ptr() if e.get("g_q") is not None else None
        d.g_q_exp = e["g_q_exp"].data_ptr() if e.get("g_q_exp") is not None else None
        d.n = e["master"].numel()
        d.kind = e["kind"]
        d.master_exp = e["master_exp"]
        d.tensor_id = e.get("tensor_id", 0)
        d.k_w = e.get("k_w", 0)
    raw = torch.frombuffer(bytearray(bytes(host)), dtype=torch.uint8)
    return raw.to(device), n


# --------------------------------------------------------------------------
# operators of language models: layer norm, quantizers per row and column,
# int8 products with a scale for each row of either operand, log probabilities
# --------------------------------------------------------------------------
# Matrices are tensors whose last dimension is the row; leading dimensions are
# folded.  Rows may be strided (a slice of a wider buffer); any other layout is
# copied first.  Calls run on the tensors' own device and its current stream.
_FLOATS = {torch.float32: ISEG_F32, torch.float16: ISEG_F16, torch.bfloat16: ISEG_BF16}


def _on_device(f):
    """Run f with its first tensor's device current (the library launches on
    the current device)."""
    first = f.__code__.co_varnames[0]

    @functools.wraps(f)
    def call(*args, **kw):
        x = args[0] if args else kw.get(first)
        if x is None:                    # queries or keys alone: another argument's
            x = next((t for t in (*args, *kw.values()) if isinstance(t, torch.Tensor) and t.get_device() >= 0), None)
        i = x.get_device() if isinstance(x, torch.Tensor) else -1      # f itself refuses what is no tensor
        if i < 0 or i == _raw_device():
            return f(*args, **kw)
        with torch.cuda.device(i):
            return f(*args, **kw)
    return call


def _float_code(t, what):
    c = _FLOATS.get(t.dtype if isinstance(t, torch.Tensor) else t)
    if c is None:
        raise ValueError(f"{what}: float32, float16 or bfloat16 expected")
    return c


def _rows(t, what):
    """(tensor, rows, columns, row stride) of a matrix with dense rows."""
    n = t.dim()
    if n == 2 and t.is_contiguous():
        M, Cc = t.shape
        return t, M, Cc, Cc or 1
    if n < 1:
        raise ValueError(f"{what}: at least one dimension expected")
    Cc = t.shape[-1]
    if n != 2:
        p = t.data_ptr()
        t = t.reshape(math.prod(t.shape[:-1]), Cc)
        if _REC is not None and t.data_ptr() != p:
            raise IsegError(f"{what}: a recorded call needs dense rows")
    M = t.shape[0]
    ld = t.stride(0) if M > 1 else max(Cc, 1)
    if (Cc > 1 and t.stride(1) != 1) or ld < Cc:
        if _REC is not None:
            raise IsegError(f"{what}: a recorded call needs dense rows")
        t = t.contiguous()
        ld = max(Cc, 1)
    return t, M, Cc, ld


def _vec(t, n, dtype, x, what):
    """A dense vector of n elements beside x, or None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() != n or t.get_device() != x.get_device():
        raise ValueError(f"{what}: {n} elements of {dtype} on {x.device} expected")
    if t.is_contiguous():
        return t
    if _REC is not None:
        raise IsegError(f"{what}: a recorded call needs a dense vector")
    return t.contiguous()


def _gpu(x, *ts, status=None):
    if status is not None and (status.dtype != torch.int32 or status.numel() < 1):
        raise ValueError("status: an int32 word expected")       # kernels write to it
    i = x.get_device()
    if i < 0:
        raise ValueError("GPU tensors expected")
    for t in (*ts, status):
        if t is not None and t.get_device() != i:
            raise ValueError("GPU tensors on one device expected")


def _like(t):
    """An uninitialized dense tensor of t's shape and type."""
    return torch.empty_like(t) if t.is_contiguous() else torch.empty(t.shape, dtype=t.dtype, device=t.device)


_NO_WS = {}


def _scratch(x, nbytes):
    """Workspace of a call on x's device: the thread's on this stream, or, under
    graph capture, memory of the graph's own (a graph outlives the stream's workspace,
    and two graphs may replay at once)."""
    if nbytes == 256:                # a call that touches none of it: one for all
        i = x.get_device()
        ws = _NO_WS.get(i)
        if ws is None:
            ws = _NO_WS[i] = torch.empty(256, dtype=torch.uint8, device=x.device)
        return ws
    if torch.cuda.is_current_stream_capturing():
        return torch.empty(nbytes, dtype=torch.uint8, device=x.device)
    return workspace(x.device).get(nbytes)


@functools.lru_cache(maxsize=256)
def _layernorm_geom(M, Cc, x_ld, y_ld, dx_ld, x_dtype, p_dtype, eps):
    return LayernormGeom(M, Cc, x_ld, y_ld, dx_ld, x_dtype, p_dtype, eps, 0)


@functools.lru_cache(maxsize=256)
def _layernorm_bwd_geom(M, Cc, x_ld, y_ld, dx_ld, x_dtype, p_dtype):
    g = LayernormGeom(M, Cc, x_ld, y_ld, dx_ld, x_dtype, p_dtype, 1.0, 0)
    return g, lib().iseg_layernorm_bwd_ws(C.byref(g))


@functools.lru_cache(maxsize=256)
def _quantize_cols_ws(M, Cc):
    return lib().iseg_quantize_cols_ws(M, Cc)


@functools.lru_cache(maxsize=256)
def _matmul_geom(M, N, K, lda, ldb, ldc, out_dtype, unaligned):
    g = MatmulGeom(M, N, K, lda, ldb, ldc, out_dtype, unaligned)
    return g, lib().iseg_matmul_i8_ws(C.byref(g))


@functools.lru_cache(maxsize=256)
def _linear_geom(M, N, K, x_ld, w_ld, codes_ld, y_ld, x_dtype, y_dtype, bits, scale_mode, unaligned):
    g = LinearGeom(M, N, K, x_ld, w_ld, max((codes_ld + 15) // 16 * 16, 16), y_ld, x_dtype, y_dtype, bits,
                   scale_mode, unaligned, 0)
    return g, lib().iseg_linear_i8_fwd_ws(C.byref(g))


@functools.lru_cache(maxsize=256)
def _linear_bwd_geom(M, N, K, dy_ld, a_ld, w_ld, wt_ld, out_ld, dy_dtype, out_dtype, bits, scale_mode, unaligned):
    g = LinearBwdGeom(M, N, K, dy_ld, a_ld, w_ld, wt_ld, out_ld, out_ld, dy_dtype, out_dtype, bits, scale_mode,
                      unaligned, 0)
    return g, lib().iseg_linear_i8_bwd_ws(C.byref(g))


@functools.lru_cache(maxsize=256)
def _logprob_geom(M, V, ld, out_ld, dtype, token_dtype, top_k):
    g = LogprobGeom(M, V, ld, out_ld, dtype, token_dtype, top_k, 0)
    return g, lib().iseg_logprob_fwd_ws(C.byref(g))


@_on_device
def layernorm_fwd(x, gamma=None, beta=None, eps=1e-5, status=None):
    """Layer norm over the last dimension: (y, mean, rstd), the statistics
    float32 with one element per row.  gamma and beta of one float type."""
    xd = _float_code(x, "x")
    xr, M, Cc, ld = _rows(x, "x")
    if Cc < 1:
        raise ValueError("x: empty rows")
    if not (eps > 0 and math.isfinite(eps)):
        raise ValueError("eps: positive and finite expected")
    p = gamma if gamma is not None else beta
    # without either, the kernels of x's own type: those of float32 parameters
    # keep shorter rows of 16-bit types in registers
    pd = _float_code(p, "gamma, beta") if p is not None else xd
    gamma = _vec(gamma, Cc, p.dtype if p is not None else None, x, "gamma")
    beta = _vec(beta, Cc, p.dtype if p is not None else None, x, "beta")
    _gpu(x, status=status)
    y = _like(x)
    mean = torch.empty(M if x.dim() == 2 else x.shape[:-1], dtype=torch.float32, device=x.device)
    rstd = torch.empty_like(mean)
    iseg_layernorm_fwd(xr, gamma, beta, _layernorm_geom(M, Cc, ld, Cc, Cc, xd, pd, eps), y, mean, rstd, status)
    return y, mean, rstd


@_on_device
def layernorm_bwd(dy, x, gamma, mean, rstd, want_params=True):
    """(dx, dgamma, dbeta) of layernorm_fwd; dgamma and dbeta take gamma's type
    (float32 without gamma) and are None without want_params."""
    xd = _float_code(x, "x")
    if dy.dtype != x.dtype or dy.shape != x.shape:
        raise ValueError("dy: x's shape and type expected")
    xr, M, Cc, ld = _rows(x, "x")
    dr, _, _, dld = _rows(dy, "dy")
    if Cc < 1:
        raise ValueError("x: empty rows")
    pdt = gamma.dtype if gamma is not None else torch.float32
    pd = _float_code(pdt, "gamma")
    gamma = _vec(gamma, Cc, pdt, x, "gamma")
    mean = _vec(mean, M, torch.float32, x, "mean")
    rstd = _vec(rstd, M, torch.float32, x, "rstd")
    _gpu(x, dy)
    dx = _like(x)
    dgamma = torch.empty(Cc, dtype=pdt, device=x.device) if want_params else None
    dbeta = torch.empty_like(dgamma) if want_params else None
    g, wsb = _layernorm_bwd_geom(M, Cc, ld, dld, Cc, xd, pd)
    iseg_layernorm_bwd(dr, xr, gamma, mean, rstd, g, dx, dgamma, dbeta, _scratch(x, wsb))
    return dx, dgamma, dbeta


def _codes_matrix(rows, cols, device):
    """int8 [rows, cols] in rows of a multiple of 16 bytes (the alignment that
    the products' wide loads take)."""
    if cols % 16 == 0:
        return torch.empty(rows, cols, dtype=torch.int8, device=device)
    return torch.empty((rows, (cols + 15) // 16 * 16), dtype=torch.int8, device=device)[:, :cols]


def _quant_args(bits, scale_mode):
    if not 2 <= bits <= 8:
        raise ValueError("bits: 2 to 8 expected")
    if scale_mode not in (ISEG_SCALE_MAX, ISEG_SCALE_POW2):
        raise ValueError("scale_mode: ISEG_SCALE_MAX or ISEG_SCALE_POW2 expected")


@_on_device
def quantize_rows(x, bits=8, scale_mode=ISEG_SCALE_MAX, mul=None, status=None):
    """Codes and a scale for each row of x [..., C] (times mul [C]): int8
    [M, C] with M the folded rows, and float32 [M]."""
    xd = _float_code(x, "x")
    _quant_args(bits, scale_mode)
    xr, M, Cc, ld = _rows(x, "x")
    mul = _vec(mul, Cc, torch.float32, x, "mul")
    _gpu(x, status=status)
    codes = _codes_matrix(M, Cc, x.device)
    scale = torch.empty(M, dtype=torch.float32, device=x.device)
    iseg_quantize_rows(xr, xd, M, Cc, ld, mul, bits, scale_mode, codes, codes.stride(0), scale, status)
    return codes, scale


@_on_device
def quantize_cols(x, bits=8, scale_mode=ISEG_SCALE_MAX, mul=None, want_sums=False, status=None):
    """Codes and a scale for each column of x [..., C] (times mul [M], one for
    each folded row): int8 [C, M], transposed, and float32 [C]; with want_sums
    also the plain column sums of x, float32 [C] (None without)."""
    xd = _float_code(x, "x")
    _quant_args(bits, scale_mode)
    xr, M, Cc, ld = _rows(x, "x")
    mul = _vec(mul, M, torch.float32, x, "mul")
    _gpu(x, status=status)
    codes = _codes_matrix(Cc, M, x.device)
    scale = torch.empty(Cc, dtype=torch.float32, device=x.device)
    sums = torch.empty(Cc, dtype=torch.float32, device=x.device) if want_sums else None
    iseg_quantize_cols(xr, xd, M, Cc, ld, mul, bits, scale_mode, codes, codes.stride(0), scale, sums,
                       _scratch(x, _quantize_cols_ws(M, Cc)), status)
    return codes, scale, sums


def _code_rows(t, what):
    if t.dtype != torch.int8 or t.dim() != 2:
        raise ValueError(f"{what}: an int8 matrix expected")
    return _rows(t, what)


@_on_device
def transpose_i8(codes):
    """int8 [C, M] from int8 [M, C]."""
    cr, M, Cc, ld = _code_rows(codes, "codes")
    _gpu(codes)
    out = _codes_matrix(Cc, M, codes.device)
    iseg_transpose_i8(cr, M, Cc, ld, out, out.stride(0))
    return out


@_on_device
def matmul_i8(a, b, a_scale=None, b_scale=None, bias=None, out_dtype=torch.float32):
    """a_scale[m] b_scale[n] sum_k a[m, k] b[n, k] + bias[n] of int8 matrices
    a [M, K] and b [N, K]: [M, N] of out_dtype."""
    od = _float_code(out_dtype, "out_dtype")
    ar, M, K, lda = _code_rows(a, "a")
    br, N, Kb, ldb = _code_rows(b, "b")
    if K != Kb:
        raise ValueError("a and b: rows of one length expected")
    if K > 131071:
        raise ValueError("a and b: rows of at most 131071 codes expected")
    a_scale = _vec(a_scale, M, torch.float32, a, "a_scale")
    b_scale = _vec(b_scale, N, torch.float32, a, "b_scale")
    bias = _vec(bias, N, torch.float32, a, "bias")
    _gpu(a, b)
    out = torch.empty(M, N, dtype=out_dtype, device=a.device)
    g, wsb = _matmul_geom(M, N, K, lda, ldb, max(N, 1), od, int((ar.data_ptr() | br.data_ptr()) & 15 != 0))
    iseg_matmul_i8(ar, a_scale, br, b_scale, bias, g, out, _scratch(a, wsb))
    return out


@_on_device
def linear_i8_fwd(x, w, w_scale=None, bias=None, bits=8, scale_mode=ISEG_SCALE_MAX, out_dtype=None, status=None):
    """A linear layer in integers: x [..., K] quantized per row, then the
    product with the weight codes w [N, K].  Returns (y [..., N] of out_dtype,
    by default x's, the codes and scales of x, which the backward needs)."""
    if x.dim() < 1 or w.dim() != 2 or x.shape[-1] != w.shape[1]:
        raise ValueError("x and w: rows of one length expected")
    out_dtype = x.dtype if out_dtype is None else out_dtype
    xd, od = _float_code(x, "x"), _float_code(out_dtype, "out_dtype")
    _quant_args(bits, scale_mode)
    xr, M, K, x_ld = _rows(x, "x")
    wr, N, _, w_ld = _code_rows(w, "w")
    if K > 131071:
        raise ValueError("x and w: rows of at most 131071 elements expected")
    dev = x.device
    w_scale = _vec(w_scale, N, torch.float32, x, "w_scale")
    bias = _vec(bias, N, torch.float32, x, "bias")
    _gpu(x, w, status=status)
    codes = _codes_matrix(M, K, dev)
    scale = torch.empty(M, dtype=torch.float32, device=dev)
    y = torch.empty(*x.shape[:-1], N, dtype=out_dtype, device=dev)
    g, wsb = _linear_geom(M, N, K, x_ld, w_ld, codes.stride(0) if K else 16, max(N, 1), xd, od, bits, scale_mode,
                          int(wr.data_ptr() & 15 != 0))
    iseg_linear_i8_fwd(xr, wr, w_scale, bias, g, codes, scale, y, _scratch(x, wsb), status)
    return y, codes, scale


@_on_device
def linear_i8_bwd(dy, a, a_scale, w, w_scale=None, w_t=None, bits=8, scale_mode=ISEG_SCALE_MAX, out_dtype=None,
                  want_input=True, want_weight=True, want_bias=False, status=None):
    """Backward of linear_i8_fwd with straight-through quantizers, its products
    in integers too: (dx, dw, dbias), None where not wanted.
      dx = Q_rows(dy w_scale) w, dw = Q_cols(dy a_scale)^T a, dbias = sum dy
    a, a_scale: the forward's codes and scales; w_t: the transposed weight
    codes (transpose_i8), which a program keeps between updates.  dx [M, K] and
    dw [N, K] have out_dtype (by default dy's), dbias is float32."""
    out_dtype = dy.dtype if out_dtype is None else out_dtype
    dd, od = _float_code(dy, "dy"), _float_code(out_dtype, "out_dtype")
    _quant_args(bits, scale_mode)
    dr, M, N, dy_ld = _rows(dy, "dy")
    ar, Ma, K, a_ld = _code_rows(a, "a")
    wr, Nw, Kw, w_ld = _code_rows(w, "w")
    if Ma != M or Nw != N or Kw != K:
        raise ValueError("dy [..., N], a [M, K] and w [N, K] expected")
    if (want_input and N > 131071) or (want_weight and M > 131071):
        raise ValueError("dy: reductions of at most 131071 expected")
    tr, wt_ld = None, 0
    if w_t is not None:
        tr, Kt, Nt, wt_ld = _code_rows(w_t, "w_t")
        if Kt != K or Nt != N:
            raise ValueError("w_t: the transposed w expected")
    dev = dy.device
    a_scale = _vec(a_scale, M, torch.float32, dy, "a_scale")
    w_scale = _vec(w_scale, N, torch.float32, dy, "w_scale")
    _gpu(dy, a, w, w_t, status=status)
    dx = torch.empty(M, K, dtype=out_dtype, device=dev) if want_input else None
    dw = torch.empty(N, K, dtype=out_dtype, device=dev) if want_weight else None
    dbias = torch.empty(N, dtype=torch.float32, device=dev) if want_bias else None
    g, wsb = _linear_bwd_geom(M, N, K, dy_ld, a_ld, w_ld, wt_ld, max(K, 1), dd, od, bits, scale_mode,
                              0 if tr is None else int(tr.data_ptr() & 15 != 0))
    iseg_linear_i8_bwd(dr, ar, a_scale, wr, w_scale, tr, g, dx, dw, dbias, _scratch(dy, wsb), status)
    return dx, dw, dbias


def _tokens(tokens, logits):
    if tokens.dtype not in (torch.int32, torch.int64) or tokens.shape != logits.shape[:-1]:
        raise ValueError("tokens: int32 or int64 of the logits' leading shape expected")
    if tokens.device != logits.device:
        raise ValueError("tokens: on the logits' device expected")
    if not tokens.is_contiguous():
        if _REC is not None:
            raise IsegError("tokens: a recorded call needs a dense tensor")
        tokens = tokens.contiguous()
    return tokens, ISEG_I32 if tokens.dtype == torch.int32 else ISEG_I64


@_on_device
def logprob_fwd(logits, tokens, top_k=0, want_entropy=True, status=None):
    """Log probabilities of the given tokens under logits [..., V]: (logprob,
    lse, entropy, top_ids, top_logprob), float32 and int32, the last two
    [..., top_k] (None if top_k = 0; entropy None without want_entropy)."""
    dt = _float_code(logits, "logits")
    lr, M, V, ld = _rows(logits, "logits")
    tokens, td = _tokens(tokens, logits)
    if V < 1:
        raise ValueError("logits: empty rows")
    if not 0 <= top_k <= min(64, V):
        raise ValueError("top_k: 0 to 64, and at most the logits of a row expected")
    _gpu(logits, tokens, status=status)
    shape, dev = logits.shape[:-1], logits.device
    g, wsb = _logprob_geom(M, V, ld, V, dt, td, top_k)
    logprob = torch.empty(M if logits.dim() == 2 else shape, dtype=torch.float32, device=dev)
    lse = torch.empty_like(logprob)
    entropy = torch.empty_like(logprob) if want_entropy else None
    ids = torch.empty(*shape, top_k, dtype=torch.int32, device=dev) if top_k else None
    tlp = torch.empty_like(ids, dtype=torch.float32) if top_k else None
    iseg_logprob_fwd(lr, tokens, g, logprob, lse, entropy, ids, tlp, _scratch(logits, wsb), status)
    return logprob, lse, entropy, ids, tlp


@_on_device
def logprob_bwd(logits, tokens, lse, entropy, g_logprob=None, g_entropy=None, status=None):
    """Gradient w.r.t. the logits of sum(g_logprob logprob) + sum(g_entropy
    entropy), given logprob_fwd's lse and entropy; one of the gradients may be
    None."""
    dt = _float_code(logits, "logits")
    lr, M, V, ld = _rows(logits, "logits")
    tokens, td = _tokens(tokens, logits)
    if V < 1:
        raise ValueError("logits: empty rows")
    if g_logprob is None and g_entropy is None:
        raise ValueError("g_logprob or g_entropy expected")
    if lse is None or (g_entropy is not None and entropy is None):
        raise ValueError("the forward's lse and, with g_entropy, its entropy expected")
    lse = _vec(lse, M, torch.float32, logits, "lse")
    entropy = _vec(entropy, M, torch.float32, logits, "entropy")
    g_logprob = _vec(g_logprob, M, torch.float32, logits, "g_logprob")
    g_entropy = _vec(g_entropy, M, torch.float32, logits, "g_entropy")
    _gpu(logits, tokens, status=status)
    dx = _like(logits)
    g, _ = _logprob_geom(M, V, ld, V, dt, td, 0)
    iseg_logprob_bwd(lr, tokens, lse, entropy, g_logprob, g_entropy, g, dx, status)
    return dx


# --------------------------------------------------------------------------
# a serving step over a cache held in 4 bits
# --------------------------------------------------------------------------
# Head tensors are [T, H, D] with any strides between tokens and heads (slices
# of one projection's rows serve as they are); only their last dimension has to
# be dense, or they are copied first.
def _heads(t, what, D=None):
    """(tensor, token stride, head stride) of a [T, H, D] tensor with dense heads."""
    if t.dim() != 3 or (D is not None and t.shape[2] != D):
        raise ValueError(f"{what}: [tokens, heads, {'D' if D is None else D}] expected")
    if t.shape[2] > 1 and t.stride(2) != 1:
        if _REC is not None:
            raise IsegError(f"{what}: a recorded call needs dense heads")
        t = t.contiguous()
    return t, t.stride(0), t.stride(1)


def _ints(t, n, x, what, dtypes=(torch.int32,)):
    """A dense vector of n whole numbers beside x."""
    if not isinstance(t, torch.Tensor) or t.dtype not in dtypes or t.numel() != n or t.get_device() != x.get_device():
        names = " or ".join(str(d)[6:] for d in dtypes)
        raise ValueError(f"{what}: {n} elements of {names} on {x.device} expected")
    if t.is_contiguous():
        return t
    if _REC is not None:
        raise IsegError(f"{what}: a recorded call needs a dense vector")
    return t.contiguous()


_INTS = (torch.int32, torch.int64)


@functools.lru_cache(maxsize=256)
def _page_map_geom(B, T, max_pages, table_ld, F, n_pages, page):
    g = PageMapGeom(B, T, max_pages, table_ld, F, n_pages, page, 0)
    return g, lib().iseg_page_map_ws(C.byref(g))


@_on_device
def page_map(ctx, count, table, held, free_pages, n_free, page, n_pages, n_tokens, in_place=False, status=None):
    """The step's pages, slots and positions from the requests' lengths (all
    int32): (q_start [B + 1], kv_len [B], positions [n_tokens], slots
    [n_tokens], held [B], n_free [1]).  ctx and count [B]: tokens before the
    step and new ones; table [B, max_pages], which gets the pages taken from
    the end of free_pages; held [B]: pages of each request so far.  n_tokens:
    rows of the step, at least sum(count).  in_place: held and n_free are
    updated and returned themselves, as a captured step wants it."""
    if not isinstance(ctx, torch.Tensor) or ctx.dim() != 1:
        raise ValueError("ctx: a vector of int32 expected")
    B = ctx.numel()
    if table.dim() != 2 or table.dtype != torch.int32 or table.shape[0] != B or (table.shape[1] > 1 and table.stride(1) != 1) or \
            (B > 1 and table.stride(0) < table.shape[1]):
        raise ValueError("table: int32 [requests, pages] with dense rows expected")
    if page < 1 or n_pages < 0 or n_tokens < 0:
        raise ValueError("page, n_pages, n_tokens: sizes expected")
    if n_pages * page > 1 << 31:
        raise ValueError("n_pages: slots of 32 bits expected")
    _gpu(ctx, table, status=status)
    if in_place and not (held.is_contiguous() and n_free.is_contiguous()):
        raise ValueError("in_place: dense held and n_free expected")
    ctx, count, held = _ints(ctx, B, ctx, "ctx"), _ints(count, B, ctx, "count"), _ints(held, B, ctx, "held")
    F = free_pages.numel()
    free_pages, n_free = _ints(free_pages, F, ctx, "free_pages"), _ints(n_free, 1, ctx, "n_free")
    # one allocation: the host's time is what a decoding step's call takes
    sizes = (B + 1, B, n_tokens, n_tokens) if in_place else (B + 1, B, n_tokens, n_tokens, B, 1)
    outs = torch.empty(sum(sizes), dtype=torch.int32, device=ctx.device).split(sizes)
    q_start, kv_len, positions, slots = outs[:4]
    held_out, n_free_out = (held, n_free) if in_place else outs[4:]
    g, wsb = _page_map_geom(B, n_tokens, table.shape[1], table.stride(0) if B > 1 else max(table.shape[1], 1), F, n_pages, page)
    iseg_page_map(ctx, count, held, free_pages, n_free, g, table, q_start, kv_len, positions, slots, held_out,
                  n_free_out, _scratch(ctx, wsb), status)
    return q_start, kv_len, positions, slots, held_out, n_free_out


def rope_frequencies(rope_dim, base=10000.0, factor=1.0, stretch=None, device="cuda"):
    """inv_freq [rope_dim / 2] float32 of qk_norm_rope_fwd: base^(-2 i / rope_dim).
    For contexts `factor` times as long as those trained on, positions are
    interpolated: every frequency over factor, or, with stretch = (length, slow,
    fast), only those that turn less than `slow` times within the trained
    length; those of more than `fast` turns stay, the ones between blend
    linearly in their turns."""
    if rope_dim < 2 or rope_dim % 2 or not base > 0 or not factor > 0:
        raise ValueError("rope_dim: even and positive, base and factor: positive expected")
    f = torch.pow(torch.tensor(float(base), dtype=torch.float64), -torch.arange(0, rope_dim, 2, dtype=torch.float64) / rope_dim)
    keep = torch.zeros_like(f)
    if stretch is not None:
        length, slow, fast = stretch
        if not (length > 0 and fast > slow >= 0):
            raise ValueError("stretch: (trained length, slow, fast) turns with fast > slow expected")
        keep = ((length * f / (2 * math.pi) - slow) / (fast - slow)).clamp(0, 1)
    return (f * keep + f / factor * (1 - keep)).float().to(device)


def _rope_args(q, k, positions, inv_freq, gamma_q, gamma_k, norm):
    if q is None and k is None:
        raise ValueError("q or k expected")
    x = q if q is not None else k
    if not isinstance(x, torch.Tensor) or x.dim() != 3:
        raise ValueError("q: [tokens, heads, D] expected")
    dt, T, D = _float_code(x, "q"), x.shape[0], x.shape[2]
    if D < 1 or D > 512:
        raise ValueError("q: heads of 1 to 512 elements expected")
    if k is not None and (k.dim() != 3 or k.dtype != x.dtype or k.shape[0] != T or k.shape[2] != D):
        raise ValueError("k: q's tokens, head size and type expected")
    n = inv_freq.numel() if inv_freq is not None else 0
    if 2 * n > D:
        raise ValueError("inv_freq: at most half a head's elements expected")
    inv_freq = _vec(inv_freq, n, torch.float32, x, "inv_freq")
    if n:
        positions = _ints(positions, T, x, "positions", _INTS)
    p = gamma_q if gamma_q is not None else gamma_k
    if p is not None and not norm:
        raise ValueError("gamma: norm expected")
    pd = _float_code(p, "gamma") if p is not None else dt
    pt = p.dtype if p is not None else x.dtype
    gamma_q, gamma_k = _vec(gamma_q, D, pt, x, "gamma_q"), _vec(gamma_k, D, pt, x, "gamma_k")
    pos64 = ISEG_I64 if n and positions.dtype == torch.int64 else ISEG_I32
    return x, T, D, dt, pd, pt, 2 * n, positions if n else None, pos64, inv_freq if n else None, gamma_q, gamma_k


@functools.lru_cache(maxsize=256)
def _rope_geom(*a):
    g = QkNormRopeGeom(*a)
    return g, lib().iseg_qk_norm_rope_bwd_ws(C.byref(g))


def _dense_like(t):
    return None if t is None else t.new_empty(t.shape)


def _hd(t):
    return 0 if t is None else t.shape[1]


@_on_device
def qk_norm_rope_fwd(q, k, positions, inv_freq, gamma_q=None, gamma_k=None, eps=1e-6, pairs=False, norm=True,
                     mscale=1.0, in_place=False, status=None):
    """Norm of every head of q [T, Hq, D] and k [T, Hk, D] (x gamma / sqrt(mean
    x^2 + eps); not without norm) and the rotation of its first 2 len(inv_freq)
    elements by positions [T]: (yq, yk).  pairs: neighbours rotate together
    instead of halves.  Either of q and k may be None, inv_freq None for the norm
    alone; in_place writes to q and k themselves."""
    x, T, D, dt, pd, _, R, positions, pos64, inv_freq, gamma_q, gamma_k = _rope_args(q, k, positions, inv_freq, gamma_q, gamma_k, norm)
    if not (eps >= 0 and math.isfinite(eps) and math.isfinite(mscale)):
        raise ValueError("eps, mscale: finite, eps not negative expected")
    _gpu(x, k, status=status)
    s = []
    ins = []
    for t, what in ((q, "q"), (k, "k")):
        if t is None:
            ins.append(None)
            s += (0, 0)
            continue
        if in_place and D > 1 and t.stride(2) != 1:
            raise ValueError(f"{what}: dense heads expected for in_place")
        t, ld, hs = _heads(t, what)
        ins.append(t)
        s += (ld, hs)
    yq, yk = ins if in_place else (_dense_like(q), _dense_like(k))
    o = s if in_place else [_hd(q) * D, D, _hd(k) * D, D]
    g, _ = _rope_geom(T, _hd(q), _hd(k), D, *s, *o, 0, 0, 0, 0, dt, pd, pos64, R, int(pairs), int(norm), eps, mscale)
    iseg_qk_norm_rope_fwd(ins[0], ins[1], positions, inv_freq, gamma_q, gamma_k, g, yq, yk, status)
    return yq, yk


@_on_device
def qk_norm_rope_bwd(dyq, dyk, q, k, positions, inv_freq, gamma_q=None, gamma_k=None, eps=1e-6, pairs=False,
                     norm=True, mscale=1.0, want_params=True):
    """(dq, dk, dgamma_q, dgamma_k) of qk_norm_rope_fwd, the last two of gamma's
    type (q's without gamma), None without norm or want_params."""
    x, T, D, dt, pd, pt, R, positions, pos64, inv_freq, gamma_q, gamma_k = _rope_args(q, k, positions, inv_freq, gamma_q, gamma_k, norm)
    if not (eps >= 0 and math.isfinite(eps) and math.isfinite(mscale)):
        raise ValueError("eps, mscale: finite, eps not negative expected")
    s, ds, ins, grads = [], [], [], []
    for t, d, what in ((q, dyq, "q"), (k, dyk, "k")):
        if t is None:
            ins.append(None)
            grads.append(None)
            s += (0, 0)
            ds += (0, 0)
            continue
        if d is None or d.shape != t.shape or d.dtype != t.dtype:
            raise ValueError(f"dy{what}: {what}'s shape and type expected")
        t, ld, hs = _heads(t, what)
        d, dld, dhs = _heads(d, "dy" + what)
        ins.append(t)
        grads.append(d)
        s += (ld, hs)
        ds += (dld, dhs)
    _gpu(x, k, dyq, dyk)
    dq, dk = _dense_like(q), _dense_like(k)
    want = want_params and norm
    dgq = torch.empty(D, dtype=pt, device=x.device) if want and q is not None else None
    dgk = torch.empty(D, dtype=pt, device=x.device) if want and k is not None else None
    g, wsb = _rope_geom(T, _hd(q), _hd(k), D, *s, *ds, _hd(q) * D, D, _hd(k) * D, D, dt, pd, pos64, R, int(pairs), int(norm), eps, mscale)
    iseg_qk_norm_rope_bwd(grads[0], grads[1], ins[0], ins[1], positions, inv_freq, gamma_q, gamma_k, g, dq, dk, dgq, dgk,
                          _scratch(x, wsb))
    return dq, dk, dgq, dgk


class Kv4Cache(NamedTuple):
    """Keys and values of n_pages pages in 4 bits (the layout of iseg.h)."""
    k: torch.Tensor                # [n_pages, H, page, W / 2] uint8
    k_scale: torch.Tensor          # [n_pages, H, page] float32
    v: torch.Tensor                # [n_pages, H, page / 16, 8 W] uint8
    v_scale: torch.Tensor          # [n_pages, H, page] float32


def _kv4_width(D):
    return (D + 31) // 32 * 32 if D <= 128 else (D + 63) // 64 * 64


def kv4_cache(n_pages, heads, dim, page=64, device="cuda"):
    """A cache of zeros."""
    if n_pages < 0 or heads < 1 or not 1 <= dim <= 256 or page < 16 or page % 16 or page > 8192:
        raise ValueError("kv4_cache: heads >= 1, dim of 1 to 256, page a multiple of 16 up to 8192 expected")
    if n_pages * page > 1 << 31:
        raise ValueError("n_pages: slots of 32 bits expected")
    W = _kv4_width(dim)
    one = functools.partial(torch.ones, n_pages, heads, page, device=device)
    return Kv4Cache(torch.full((n_pages, heads, page, W // 2), 136, dtype=torch.uint8, device=device), one(),
                    torch.full((n_pages, heads, page // 16, 8 * W), 136, dtype=torch.uint8, device=device), one())


def _kv4_check(cache, D, x):
    """(tensors, n_pages, heads, page) of a cache for heads of D elements beside x."""
    k, ks, v, vs = cache
    if not 1 <= D <= 256:
        raise ValueError("heads of 1 to 256 elements expected")
    W = _kv4_width(D)
    if k.dim() != 4 or k.shape[3] * 2 != W:
        raise ValueError(f"cache: rows of {W // 2} bytes expected for heads of {D} elements")
    P, H, page, _ = k.shape
    if k.dtype != torch.uint8 or v.dtype != torch.uint8 or ks.dtype != torch.float32 or vs.dtype != torch.float32 or \
            page < 16 or page % 16 or page > 8192 or tuple(v.shape) != (P, H, page // 16, 8 * W) or \
            tuple(ks.shape) != (P, H, page) or tuple(vs.shape) != (P, H, page):
        raise ValueError("cache: the four tensors of kv4_cache expected")
    if not (k.is_contiguous() and v.is_contiguous() and ks.is_contiguous() and vs.is_contiguous()):
        raise ValueError("cache: dense tensors expected")
    if (k.data_ptr() | v.data_ptr() | ks.data_ptr() | vs.data_ptr()) & 15:
        raise ValueError("cache: tensors at multiples of 16 bytes expected")
    if P * page > 1 << 31:
        raise ValueError("cache: slots of 32 bits expected")
    _gpu(x, k, ks, v, vs)
    return P, H, page


@functools.lru_cache(maxsize=256)
def _kv4_geom(*a):
    return Kv4Geom(*a)


@_on_device
def kv4_write(k, v, slots, cache, scale_mode=ISEG_SCALE_MAX, status=None):
    """Keys and values [T, H, D] of tokens into their slots [T] (int32 or int64;
    negative ones are skipped) of a Kv4Cache."""
    dt = _float_code(k, "k")
    if v.shape != k.shape or v.dtype != k.dtype:
        raise ValueError("v: k's shape and type expected")
    if scale_mode not in (ISEG_SCALE_MAX, ISEG_SCALE_POW2):
        raise ValueError("scale_mode: ISEG_SCALE_MAX or ISEG_SCALE_POW2 expected")
    k, k_ld, k_hs = _heads(k, "k")
    v, v_ld, v_hs = _heads(v, "v")
    T, H, D = k.shape
    slots = _ints(slots, T, k, "slots", _INTS)
    _gpu(k, v, status=status)
    P, Hc, page = _kv4_check(cache, D, k)
    if H != Hc:
        raise ValueError("k: the cache's heads expected")
    g = _kv4_geom(T, H, D, k_ld, k_hs, v_ld, v_hs, P, page, dt, ISEG_I64 if slots.dtype == torch.int64 else ISEG_I32, scale_mode)
    iseg_kv4_write(k, v, slots, g, *cache, status)


@_on_device
def kv4_read(slots, cache, dim=None, dtype=torch.float32, status=None):
    """(k, v), each [T, H, dim] of dtype: the values at slots [T], zeros for
    negative ones.  dim: elements of a head (the cache's stored width without)."""
    if not isinstance(slots, torch.Tensor) or slots.dtype not in _INTS or slots.dim() != 1:
        raise ValueError("slots: a vector of int32 or int64 expected")
    dt = _float_code(dtype, "dtype")
    D = cache[0].shape[-1] * 2 if dim is None else dim
    P, H, page = _kv4_check(cache, D, slots)
    T = slots.numel()
    slots = _ints(slots, T, slots, "slots", _INTS)
    _gpu(slots, status=status)
    k = torch.empty(T, H, D, dtype=dtype, device=slots.device)
    v = torch.empty_like(k)
    g = _kv4_geom(T, H, D, H * D, D, H * D, D, P, page, dt, ISEG_I64 if slots.dtype == torch.int64 else ISEG_I32, 0)
    iseg_kv4_read(*cache, slots, g, k, v, status)
    return k, v


@functools.lru_cache(maxsize=256)
def _kv4_attention_geom(*a):
    g = Kv4AttentionGeom(*a)
    return g, lib().iseg_kv4_attention_ws(C.byref(g))


@_on_device
def kv4_attention(q, cache, table, q_start, kv_len, scale=None, causal=True, window=0, max_q=0, max_kv=0,
                  want_lse=True, out=None, status=None):
    """Attention of q [T, Hq, D], the new tokens of B requests one after the
    other (q_start [B + 1]), over the kv_len [B] tokens that each has in a
    Kv4Cache under table [B, pages]: (out like q, lse float32 [T, Hq], None
    without want_lse).  A request's queries are its last tokens; causal: each sees
    no key after its own, window > 0: only that many up to its own.  max_q, max_kv:
    bounds of the requests' new and cached tokens, where the caller has them (0:
    T and all of table); a request of more than max_q is left out.  scale: 1 / sqrt(D) without.  Rows of no request keep
    what `out` holds; there lse is unspecified."""
    dt = _float_code(q, "q")
    q, q_ld, q_hs = _heads(q, "q")
    T, Hq, D = q.shape
    if D % 8 or D > 256 or D < 1:
        raise ValueError("q: heads of a multiple of 8 up to 256 elements expected")
    P, H, page = _kv4_check(cache, D, q)
    if Hq < 1 or Hq % H:
        raise ValueError("q: a multiple of the cache's heads expected")
    if table.dim() != 2 or table.dtype != torch.int32 or (table.shape[1] > 1 and table.stride(1) != 1) or \
            (table.shape[0] > 1 and table.stride(0) < table.shape[1]):
        raise ValueError("table: int32 [requests, pages] with dense rows expected")
    B = table.shape[0]
    q_start, kv_len = _ints(q_start, B + 1, q, "q_start"), _ints(kv_len, B, q, "kv_len")
    scale = 1 / math.sqrt(D) if scale is None else scale
    if not (scale > 0 and math.isfinite(scale)):
        raise ValueError("scale: positive and finite expected")
    if window < 0 or max_q < 0 or max_kv < 0:
        raise ValueError("window, max_q, max_kv: not negative expected")
    _gpu(q, table, status=status)
    if out is None:
        out = torch.empty(T, Hq, D, dtype=q.dtype, device=q.device)
    elif out.shape != q.shape or out.dtype != q.dtype or out.get_device() != q.get_device() or (D > 1 and out.stride(2) != 1):
        raise ValueError("out: q's shape and type with dense heads expected")
    lse = torch.empty(T, Hq, dtype=torch.float32, device=q.device) if want_lse else None
    g, wsb = _kv4_attention_geom(T, B, Hq, H, D, q_ld, q_hs, out.stride(0), out.stride(1), P, table.shape[1],
                                 table.stride(0) if B > 1 else max(table.shape[1], 1), max_q, max_kv, window, page, dt, int(causal), scale)
    if wsb == 0:
        raise ValueError("kv4_attention: sizes beyond one launch")
    iseg_kv4_attention(q, *cache, table, q_start, kv_len, g, out, lse, _scratch(q, wsb), status)
    return out, lse


@functools.lru_cache(maxsize=256)
def _verify_geom(*a):
    g = VerifyGeom(*a)
    return g, lib().iseg_verify_drafts_ws(C.byref(g))


def _distributions(t, what):
    if t.shape[2] > 1 and t.stride(2) != 1:
        if _REC is not None:
            raise IsegError(f"{what}: a recorded call needs dense rows")
        t = t.contiguous()
    return t, t.stride(0), t.stride(1)


@_on_device
def verify_drafts(target, draft, tokens, n_draft, u, u_sample, status=None):
    """Drafted tokens [B, S] against the target's probabilities [B, S + 1, V] and
    those they were drawn from, draft [B, S, V] (None: each was certain): (out
    [B, S + 1] int32, the accepted tokens, one more, then -1; accepted [B]
    int32).  n_draft [B] int32: drafts of each request; u [B, S] and u_sample
    [B] float32: uniform random numbers of [0, 1)."""
    dt = _float_code(target, "target")
    if target.dim() != 3 or target.shape[1] < 1 or target.shape[2] < 1:
        raise ValueError("target: [requests, drafts + 1, tokens] expected")
    B, S, V = target.shape[0], target.shape[1] - 1, target.shape[2]
    if draft is not None and (draft.dtype != target.dtype or tuple(draft.shape) != (B, S, V)):
        raise ValueError("draft: target's type and one row less expected")
    target, t_bs, t_ld = _distributions(target, "target")
    d_bs = d_ld = 0
    if draft is not None:
        draft, d_bs, d_ld = _distributions(draft, "draft")
    if tokens.shape != (B, S) or u.shape != (B, S):
        raise ValueError("tokens, u: [requests, drafts] expected")
    tokens = _ints(tokens, B * S, target, "tokens", _INTS)
    n_draft = _ints(n_draft, B, target, "n_draft")
    u, u_sample = _vec(u, B * S, torch.float32, target, "u"), _vec(u_sample, B, torch.float32, target, "u_sample")
    _gpu(target, draft, status=status)
    out = torch.empty(B, S + 1, dtype=torch.int32, device=target.device)
    accepted = torch.empty(B, dtype=torch.int32, device=target.device)
    g, wsb = _verify_geom(B, S, V, t_bs, t_ld, d_bs, d_ld, dt, ISEG_I64 if tokens.dtype == torch.int64 else ISEG_I32)
    iseg_verify_drafts(target, draft, tokens, n_draft, u, u_sample, g, out, accepted, _scratch(target, wsb), status)
    return out, accepted

"""ctypes loader for libloract.so.  Fails loudly when the library has not been built."""
from __future__ import annotations

import ctypes
import os

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG_DIR, "libloract.so")


class LoractParams(ctypes.Structure):
    """Mirror of `loract_params` in include/loract.h."""
    _fields_ = [
        ("m", ctypes.c_int64),
        ("n", ctypes.c_int64),
        ("ldx", ctypes.c_int64),
        ("k", ctypes.c_int32),
        ("l", ctypes.c_int32),
        ("t", ctypes.c_int32),
        ("x_dtype", ctypes.c_int32),
        ("factor_dtype", ctypes.c_int32),
        ("seed", ctypes.c_uint64),
    ]


class LoractLinearParams(ctypes.Structure):
    """Mirror of `loract_linear_params` in include/loract.h (api.py packs the same bytes)."""
    _fields_ = [(f, ctypes.c_int64) for f in ("m", "n_in", "n_out", "ldx", "ldw", "ldr", "ldy", "ldz", "ldp")] + \
               [(f, ctypes.c_int32) for f in ("dtype", "out_dtype", "w_layout", "act", "r_lora")] + \
               [("lora_scale", ctypes.c_float), ("p_drop", ctypes.c_double), ("seed", ctypes.c_uint64)]


class LoractQkParams(ctypes.Structure):
    """Mirror of `loract_qk_params` in include/loract.h (api.py packs the same bytes)."""
    _fields_ = [("m", ctypes.c_int64)] + \
               [(f, ctypes.c_int32) for f in ("heads_q", "heads_k", "d", "rot", "interleaved", "dtype")] + \
               [("n_pos", ctypes.c_int64), ("eps", ctypes.c_float)] + \
               [(f, ctypes.c_int64) for f in ("q_token", "q_head", "k_token", "k_head", "qo_token", "qo_head", "ko_token",
                                              "ko_head", "dq_token", "dq_head", "dk_token", "dk_head")]


class LoractAdamwParams(ctypes.Structure):
    """Mirror of `loract_adamw_params` in include/loract.h (api.py packs the same bytes)."""
    _fields_ = [(f, ctypes.c_double) for f in ("lr", "beta1", "beta2", "eps", "weight_decay")] + \
               [("step", ctypes.c_int64), ("seed", ctypes.c_uint64)] + \
               [(f, ctypes.c_int32) for f in ("p_dtype", "g_dtype", "state_bits")]


class LoractLogprobParams(ctypes.Structure):
    """Mirror of `loract_logprob_params` in include/loract.h (api.py packs the same bytes)."""
    _fields_ = [(f, ctypes.c_int64) for f in ("m", "n", "ld", "ldg")] + \
               [(f, ctypes.c_int32) for f in ("dtype", "target_bits", "top", "reserved")] + [("temperature", ctypes.c_double)]


class LoractRequestsParams(ctypes.Structure):
    """Mirror of `loract_requests_params` in include/loract.h (api.py packs the same bytes)."""
    _fields_ = [(f, ctypes.c_int64) for f in ("m", "n_in", "n_out", "adapters", "ldx", "ldr", "ldy")] + \
               [(f, ctypes.c_int32) for f in ("dtype", "out_dtype", "r", "reserved")]


_P = ctypes.POINTER
_vp, _i32, _i64, _u64, _sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_size_t

# name -> (restype, argtypes); one entry per symbol declared in include/loract.h
SIGNATURES = {
    "loract_version": (ctypes.c_char_p, []),
    "loract_strerror": (ctypes.c_char_p, [ctypes.c_int]),
    "loract_last_hip_error": (ctypes.c_char_p, []),
    "loract_sample_indices": (ctypes.c_int, [_i64, _i32, _u64, _P(_i32)]),
    "loract_workspace_bytes": (ctypes.c_int, [_P(LoractParams), _P(_sz)]),
    "loract_compress": (ctypes.c_int, [_vp, _P(LoractParams), _P(_i32), _vp, _vp, _vp, _sz, _vp, _vp]),
    "loract_compress_adaptive": (ctypes.c_int, [_vp, _P(LoractParams), _P(_i32), ctypes.c_double, _vp, _vp, _vp,
                                                _vp, _sz, _vp, _vp]),
    "loract_reconstruct": (ctypes.c_int, [_vp, _vp, _i64, _i64, _i32, _i32, _vp, _i64, _i32, _vp]),
    "loract_lora_grad_workspace_bytes": (ctypes.c_int, [_i64, _i64, _i32, _i64, _i32, _P(_sz)]),
    "loract_lora_grad": (ctypes.c_int, [_vp, _vp, _i64, _i64, _i32, _i32, _vp, _i64, _vp, _i32, _i32,
                                        ctypes.c_float, _vp, _vp, _sz, _vp]),
    "loract_static_scratch_bytes": (_sz, []),
    "loract_lora_grad_static": (ctypes.c_int, [_vp, _vp, _i64, _i64, _i32, _i32, _vp, _i64, _vp, _i32, _i32,
                                               ctypes.c_float, _vp, _vp]),
    "loract_rsvd": (ctypes.c_int, [_vp, _P(LoractParams), _vp, _vp, _vp, _vp, _sz, _vp, _vp]),
    "loract_gaussian_omega_t": (ctypes.c_int, [_vp, _i32, _i64, _i32, _u64, _vp]),
    "loract_prenorm_forward": (ctypes.c_int, [_vp, _i64, _i64, _i64, _i32, _vp, ctypes.c_float, _vp, _i64,
                                              _vp, _vp]),
    "loract_prenorm_backward": (ctypes.c_int, [_vp, _i64, _i64, _i64, _i32, _vp, _vp, _vp, _i64, _vp,
                                               _i64, _vp]),
    "loract_dropout": (ctypes.c_int, [_vp, _i64, _vp, _i64, _i64, _i64, _i32, ctypes.c_double, _u64, _vp, _i64, _vp]),
    "loract_linear_workspace_bytes": (ctypes.c_int, [_vp, _P(_sz)]),
    "loract_linear": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "loract_linear_backward_workspace_bytes": (ctypes.c_int, [_vp, _P(_sz)]),
    "loract_linear_backward": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "loract_rope_table": (ctypes.c_int, [_vp, _i64, _i32, ctypes.c_double, _i64, _vp]),
    "loract_qknorm_rope_workspace_bytes": (ctypes.c_int, [_vp, _P(_sz)]),
    "loract_qknorm_rope_forward": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "loract_qknorm_rope_backward": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                                   _vp, _vp, _vp, _sz, _vp]),
    "loract_adamw": (ctypes.c_int, [_vp, _vp, _vp, _vp, _i64, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "loract_token_logprobs_workspace_bytes": (ctypes.c_int, [_vp, _P(_sz)]),
    "loract_token_logprobs": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "loract_token_logprobs_backward": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "loract_token_logprobs_grad": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "loract_lora_requests_workspace_bytes": (ctypes.c_int, [_vp, _P(_sz)]),
    "loract_lora_requests": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "loract_profile_begin": (ctypes.c_int, []),
    "loract_profile_end": (ctypes.c_int, []),
    "loract_profile_count": (ctypes.c_int, []),
    "loract_profile_get": (ctypes.c_int, [ctypes.c_int, ctypes.c_char_p, ctypes.c_int,
                                          _P(ctypes.c_double), _P(_i64)]),
}

_lib = None


def load() -> ctypes.CDLL:
    """Load the shared library once and attach the C signatures."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            "libloract.so is missing (%s). Build it with `python -m paper_2509_23472_amd.build` "
            "or __graft_entry__.build(); there is no CPU fallback." % LIB_PATH)
    lib = ctypes.CDLL(LIB_PATH)
    for name, (restype, argtypes) in SIGNATURES.items():
        fn = getattr(lib, name)          # AttributeError if the symbol is not exported
        fn.restype = restype
        fn.argtypes = argtypes
    _lib = lib
    return lib

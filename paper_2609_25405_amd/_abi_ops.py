"""ctypes mirror of include/orthrus/kv8.h and include/orthrus/score.h: the structs and the entry
points, same names.  Argument marshalling only; the library is the one ``_abi`` loads."""
from __future__ import annotations

from ctypes import POINTER, Structure, c_double, c_float, c_int, c_int32, c_int64, c_size_t, c_void_p

from . import _abi

ORTHRUS_DEVERR_STALE = 4
ORTHRUS_MAX_TOP = 64


class orthrus_kv8(Structure):
    _fields_ = [("k_cache", c_void_p), ("v_cache", c_void_p), ("k_scale", c_void_p), ("v_scale", c_void_p),
                ("block_table", c_void_p), ("n_layers", c_int32), ("n_pages", c_int32), ("n_seq", c_int32),
                ("max_blocks", c_int32)]


class orthrus_head_shape(Structure):
    _fields_ = [("n_q_heads", c_int32), ("n_kv_heads", c_int32), ("head_dim", c_int32), ("page_size", c_int32),
                ("dtype", c_int32), ("rot_dims", c_int32), ("interleaved", c_int32), ("rope_base", c_float),
                ("rope_magnitude", c_float), ("norm_eps", c_float), ("rope_freq", POINTER(c_double))]


class orthrus_segment(Structure):
    _fields_ = [("seq", c_int32), ("offset", c_int32), ("len", c_int32)]


# name -> (restype, argtypes); every symbol the two headers declare
SIGNATURES = {
    "orthrus_rows_create": (c_int, [POINTER(orthrus_head_shape), POINTER(c_void_p)]),
    "orthrus_rows_destroy": (None, [c_void_p]),
    "orthrus_rows_workspace_bytes": (c_size_t, [c_void_p, c_int32, c_int32, c_int32]),
    "orthrus_rows_plan": (c_int, [c_void_p, POINTER(orthrus_kv8), c_void_p, c_int32, c_void_p, c_size_t, c_void_p]),
    "orthrus_rows_items": (c_int, [c_void_p, POINTER(orthrus_kv8), c_void_p, c_int32, POINTER(c_int32), c_void_p, c_int32]),
    "orthrus_kv8_append": (c_int, [c_void_p, POINTER(orthrus_kv8), c_int32, c_void_p, c_int32, c_int64, c_void_p, c_void_p,
                                   c_void_p, c_int64, c_void_p]),
    "orthrus_kv8_read": (c_int, [c_void_p, POINTER(orthrus_kv8), c_int32, c_void_p, c_void_p, c_void_p]),
    "orthrus_kv8_attend": (c_int, [c_void_p, POINTER(orthrus_kv8), c_int32, c_void_p, c_int64, c_float, c_void_p, c_int64,
                                   c_void_p]),
    "orthrus_step_kv8_bytes": (c_size_t, [c_void_p, c_void_p, c_int32, c_int32, c_int32, c_int32]),
    "orthrus_step_kv8": (c_int, [c_void_p, c_void_p, POINTER(_abi.orthrus_batch), POINTER(orthrus_kv8), POINTER(orthrus_kv8),
                                 c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "orthrus_logprobs_bytes": (c_size_t, [c_int32, c_int32, c_int32]),
    "orthrus_logprobs": (c_int, [c_void_p, c_int64, c_int32, c_int32, c_void_p, c_int32, c_void_p, c_void_p, c_void_p,
                                 c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
}

_lib = None


def load():
    """The library with these entry points' types set (raises if it is missing)."""
    global _lib
    if _lib is None:
        lib = _abi.load()
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib

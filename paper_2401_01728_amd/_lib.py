"""Loads librv.so (and librvgen.so) with ctypes.  No fallbacks: a missing library is an error."""
import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "librv.so")
GEN_PATH = os.path.join(HERE, "inputs", "librvgen.so")

c_void_p, c_int, c_int32, c_int64, c_size_t, c_float, c_uint32, c_uint64 = (
    ctypes.c_void_p, ctypes.c_int, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t,
    ctypes.c_float, ctypes.c_uint32, ctypes.c_uint64)


class StageDesc(ctypes.Structure):
    _fields_ = [("kind", c_int32), ("dtype", c_int32), ("n_layers", c_int32),
                ("dims", ctypes.POINTER(c_int64)), ("microbatch", c_int32), ("tau", c_int32),
                ("eta", c_float), ("ln_eps", c_float), ("stream", c_void_p)]


class LossDesc(ctypes.Structure):
    _fields_ = [("x", c_void_p), ("ldx", c_int64), ("w", c_void_p), ("ldw", c_int64), ("label", c_void_p),
                ("T", c_int32), ("d", c_int32), ("V", c_int32), ("rows", c_int32), ("scale", c_float),
                ("row_scale", c_void_p), ("loss", c_void_p), ("lse", c_void_p), ("dx", c_void_p), ("lddx", c_int64),
                ("dw", c_void_p), ("master", c_void_p), ("master_out", c_void_p), ("version", c_void_p),
                ("eta", c_float), ("work", c_void_p), ("work_bytes", c_size_t), ("stream", c_void_p)]


# every symbol include/rv.h declares: name -> (restype, argtypes)
SYMBOLS = {
    "rv_stage_create": (c_int, [ctypes.POINTER(StageDesc), ctypes.POINTER(c_void_p)]),
    "rv_stage_destroy": (c_int, [c_void_p]),
    "rv_stage_num_params": (c_size_t, [c_void_p]),
    "rv_stage_in_flight": (c_int, [c_void_p]),
    "rv_stage_set_params": (c_int, [c_void_p, c_void_p, c_size_t]),
    "rv_stage_set_optimizer": (c_int, [c_void_p, c_float, c_float]),
    "rv_stage_set_accumulation": (c_int, [c_void_p, c_int]),
    "rv_stage_defer_update": (c_int, [c_void_p, c_int]),
    "rv_cluster_sync": (c_int, [c_void_p, c_int, c_int, c_int]),
    "rv_cluster_sync_fork": (c_int, [c_void_p, c_int, c_int, c_int, c_int, c_void_p]),
    "rv_cluster_sync_join": (c_int, [c_void_p, c_int]),
    "rv_stage_get_params": (c_int, [c_void_p, c_void_p, c_size_t]),
    "rv_stage_last_grad": (c_int, [c_void_p, c_void_p, c_size_t]),
    "rv_stage_keep_grad": (c_int, [c_void_p, c_int]),
    "rv_stage_forward": (c_int, [c_void_p, c_int64, c_void_p, c_void_p]),
    "rv_stage_backward": (c_int, [c_void_p, c_int64, c_void_p, c_void_p]),
    "rv_stage_step": (c_int, [c_void_p, c_int64, c_void_p, c_void_p, c_int64, c_void_p, c_void_p]),
    "rv_block_update": (c_int, [c_void_p, c_void_p, c_size_t, c_float, c_void_p, c_void_p]),
    "rv_block_update_momentum": (c_int, [c_void_p, c_void_p, c_void_p, c_size_t, c_float, c_float, c_float, c_void_p,
                                         c_void_p]),
    "rv_cluster_average": (c_int, [ctypes.POINTER(c_void_p), c_int, c_size_t, c_int, c_void_p, c_int,
                                   c_void_p, c_int, c_float, c_void_p]),
    "rv_cluster_average_v": (c_int, [ctypes.POINTER(c_void_p), c_int, c_size_t, ctypes.POINTER(c_int64), c_int,
                                     c_void_p, c_int, c_void_p, c_int, c_float, c_void_p]),
    "rv_loss_work": (c_int, [c_int, c_int, c_int, c_int64, c_int, c_int, ctypes.POINTER(c_size_t)]),
    "rv_loss_forward": (c_int, [ctypes.POINTER(LossDesc)]),
    "rv_loss_step": (c_int, [ctypes.POINTER(LossDesc)]),
    "rv_stage_profile": (c_int, [c_void_p, c_int]),
    "rv_stage_profile_read": (c_int, [c_void_p, ctypes.POINTER(c_int), ctypes.POINTER(c_float)]),
    "rv_strerror": (ctypes.c_char_p, [c_int]),
}

# per-kernel entry points declared in include/rv_kernels.h
KERNEL_SYMBOLS = {
    "rv_k_gemm_wgrad_grouped": (c_int, [c_int, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int,
                                        c_void_p, c_void_p]),
    "rv_k_gemm_wgrad_update": (c_int, [c_int, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int,
                                       c_void_p, c_void_p, c_void_p, c_float, c_void_p]),
    "rv_k_gemm_bf16": (c_int, [c_void_p, c_int64, c_int, c_void_p, c_int64, c_int, c_int, c_int, c_int, c_int,
                               c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_int64, c_void_p, c_int,
                               c_void_p]),
    "rv_k_gemm_part": (c_int, [c_void_p, c_int64, c_void_p, c_int64, c_int, c_int, c_int, c_int, c_int, c_int, c_void_p, c_void_p]),
    "rv_k_gemm_bf16_blocks": (c_int, [c_void_p, c_int, c_int, c_void_p, c_int, c_int, c_int, c_int, c_int, c_int, c_void_p, c_void_p, c_int,
                                      c_void_p, c_void_p, c_void_p, c_int, c_int, c_void_p]),
    "rv_k_stage_less_work": (c_int, [c_void_p]),
    "rv_k_gemm_part_form": (c_int, [c_int, c_int, c_int, c_void_p, c_void_p]),
    "rv_k_layernorm_fwd_parts": (c_int, [c_void_p, c_int, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                         c_void_p, c_int, c_int, c_float, c_void_p]),
    "rv_k_layernorm_bwd_parts": (c_int, [c_void_p, c_int, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                         c_int, c_int, c_int, c_void_p]),
    "rv_k_layernorm_fwd": (c_int, [c_void_p, c_int, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                   c_int, c_int, c_float, c_void_p]),
    "rv_k_layernorm_bwd": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                   c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_int, c_void_p]),
    "rv_k_attention_fwd": (c_int, [c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_void_p]),
    "rv_k_attention_bwd": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_int, c_int,
                                   c_int, c_void_p]),
    "rv_k_cross_attention_work": (c_int, [c_int] * 7 + [ctypes.POINTER(c_size_t)]),
    "rv_k_cross_attention_fwd": (c_int, [c_void_p, c_int64] * 3 + [c_void_p, c_void_p, c_int64, c_void_p] + [c_int] * 6
                                 + [c_void_p, c_size_t, c_void_p]),
    "rv_k_cross_attention_bwd": (c_int, [c_void_p, c_int64] * 3 + [c_void_p] + [c_void_p, c_int64] * 2 + [c_void_p]
                                 + [c_void_p, c_int64] * 3 + [c_int] * 6 + [c_void_p, c_size_t, c_void_p]),
    "rv_k_attention_bwd_static": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_int, c_int,
                                          c_int, c_void_p]),
}

GEN_SYMBOLS = {
    "rvgen_fill_normal": (c_int, [c_void_p, c_uint64, c_uint32, c_uint32, c_float, c_float, c_uint64,
                                  c_float, c_int, c_void_p]),
    "rvgen_fill_uniform": (c_int, [c_void_p, c_uint64, c_uint32, c_uint32, c_float, c_float, c_uint64,
                                   c_void_p]),
}

_lib = None
_gen = None


def _load(path, table):
    if not os.path.exists(path):
        raise RuntimeError(
            "%s is not built; run `python -m paper_2401_01728_amd.build` (there is no fallback path)" % path)
    lib = ctypes.CDLL(path)
    for name, (res, args) in table.items():
        fn = getattr(lib, name)          # AttributeError if the symbol is missing
        fn.restype, fn.argtypes = res, args
    return lib


def lib():
    global _lib
    if _lib is None:
        _lib = _load(LIB_PATH, {**SYMBOLS, **KERNEL_SYMBOLS})
    return _lib


def genlib():
    global _gen
    if _gen is None:
        _gen = _load(GEN_PATH, GEN_SYMBOLS)
    return _gen

"""ctypes loader for libcure.so (include/cure.h).

The library is built in-tree by ``paper_2608_00531_gb300.build``.  Loading
fails loudly when it is missing: there is no CPU fallback anywhere in the
package.
"""
from __future__ import annotations

import ctypes as C
import os

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libcure.so")

CURE_OK = 0
STATUS = {0: "CURE_OK", 1: "CURE_ERR_INVALID_ARG", 2: "CURE_ERR_CAPACITY", 3: "CURE_ERR_CUDA",
          4: "CURE_ERR_DEVICE_FAULT", 5: "CURE_ERR_UNSUPPORTED"}

DEVERR_PAGE, DEVERR_SLOT, DEVERR_NODES, DEVERR_TOKEN, DEVERR_TIMEOUT = 0x1, 0x2, 0x4, 0x8, 0x10

# every entry point the header declares
EXPORTS = ("cure_score_draft", "cure_build_tree", "cure_tree_attn", "cure_tree_attn_workspace_size",
           "cure_accept", "cure_lm_head_argmax", "cure_lm_head_workspace_size", "cure_selftest_wait_timeout",
           "cure_selftest_lm_head_timeout", "cure_selftest_prompt_timeout", "cure_selftest_attn_route",
           "cure_sample_target", "cure_resync_kv", "cure_rope_init", "cure_rope_init_freqs", "cure_rope_qkv",
           "cure_append_kv", "cure_prompt_attn", "cure_prompt_attn_workspace_size", "cure_device_error",
           "cure_rope_qkv_axes", "cure_append_kv_axes", "cure_append_kv8", "cure_prompt_attn8",
           "cure_prompt_attn8_workspace_size", "cure_tree_attn8", "cure_tree_attn8_workspace_size", "cure_resync_kv8",
           "cure_selftest_prompt8_timeout", "cure_selftest_tree8_timeout", "cure_save_kv8", "cure_save_kv8_size", "cure_restore_kv8", "cure_status_string", "cure_abi_version")


class TreeParams(C.Structure):
    _fields_ = [("batch", C.c_int32), ("block", C.c_int32), ("topk", C.c_int32),
                ("tau", C.c_float), ("budget", C.c_int32), ("branches", C.c_int32),
                ("repair_depth", C.c_int32), ("max_ufp", C.c_int32),
                ("margin_scale", C.c_float), ("branch_min", C.c_int32),
                ("max_depth", C.c_int32), ("beam", C.c_int32)]


class KVDesc(C.Structure):
    _fields_ = [("layout", C.c_int32), ("heads_kv", C.c_int32), ("head_dim", C.c_int32),
                ("page_size", C.c_int32), ("max_len", C.c_int32), ("num_pages", C.c_int32),
                ("block_table", C.c_void_p)]


class Rope(C.Structure):
    _fields_ = [("style", C.c_int32), ("rot_dim", C.c_int32), ("amplitude", C.c_float), ("reserved", C.c_int32),
                ("turns", C.c_uint64 * 64)]


class RopeScaling(C.Structure):
    _fields_ = [("kind", C.c_int32), ("reserved", C.c_int32), ("factor", C.c_double), ("low", C.c_double),
                ("high", C.c_double), ("original", C.c_double)]


class RopeAxes(C.Structure):
    _fields_ = [("axes", C.c_int32), ("reserved", C.c_int32), ("axis", C.c_uint8 * 64)]


class CureError(RuntimeError):
    def __init__(self, fn: str, code: int, detail: str = ""):
        super().__init__(f"{fn} returned {STATUS.get(code, code)}" + (f": {detail}" if detail else ""))
        self.code = code


_lib = None

P = C.c_void_p
I32 = C.c_int32
I64 = C.c_int64


def load() -> C.CDLL:
    """Load libcure.so once; raise when it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with "
                          "`python -c 'import __graft_entry__ as g; g.build()'`")
    lib = C.CDLL(LIB_PATH)
    lib.cure_score_draft.argtypes = [P, I32, I32, I32, P, P, P, P, P]
    lib.cure_build_tree.argtypes = [C.POINTER(TreeParams), P, P, P, P, P, P, P, P, P, P, P, P, P, P]
    lib.cure_tree_attn.argtypes = [P, P, P, P, P, C.POINTER(KVDesc), P, P, P, I32, I32, I32,
                                   C.c_float, P, P, C.c_size_t, P]
    lib.cure_tree_attn_workspace_size.argtypes = [I32, I32, I32, C.POINTER(KVDesc)]
    lib.cure_tree_attn_workspace_size.restype = C.c_size_t
    lib.cure_accept.argtypes = [P, P, I32, I32, I32, I32, P, P, P, P, P, P, P, P, P, P, P]
    lib.cure_sample_target.argtypes = [P, P, C.c_float, I32, I32, I32, P, P, P]
    lib.cure_lm_head_argmax.argtypes = [P, P, I32, I32, I32, P, P, P, C.c_size_t, P]
    lib.cure_lm_head_workspace_size.argtypes = [I32, I32]
    lib.cure_lm_head_workspace_size.restype = C.c_size_t
    lib.cure_selftest_wait_timeout.argtypes = [C.c_int64, P]
    lib.cure_selftest_wait_timeout.restype = C.c_int
    lib.cure_selftest_lm_head_timeout.argtypes = [P, P, I32, I32, I32, P, P, C.c_size_t, I32, C.c_int64, P]
    lib.cure_selftest_lm_head_timeout.restype = C.c_int
    lib.cure_selftest_attn_route.argtypes = [I32, I32, I32, C.POINTER(KVDesc), I32, C.POINTER(I32)]
    lib.cure_selftest_attn_route.restype = C.c_int
    lib.cure_resync_kv.argtypes = [I32, C.POINTER(C.c_void_p), C.POINTER(C.c_void_p),
                                   C.POINTER(KVDesc), P, P, I32, I32, I32, P, P, P, P, P, P, P,
                                   P, P, P]
    lib.cure_rope_init.argtypes = [C.POINTER(Rope), I32, I32, C.c_double, C.POINTER(RopeScaling), C.c_float]
    lib.cure_rope_init_freqs.argtypes = [C.POINTER(Rope), I32, I32, C.POINTER(C.c_double), C.c_float]
    lib.cure_rope_qkv.argtypes = [P, P, P, I64, I64, I64, I32, I32, I32, I32, P, C.POINTER(Rope), P, P, C.c_float,
                                  P, P, P, I64, I64, I64, P]
    lib.cure_append_kv.argtypes = [P, P, P, I64, I64, I64, I32, I32, I32, P, P, P, C.POINTER(KVDesc), P, P,
                                   C.POINTER(Rope), P, P, C.c_float, P, I64, P]
    lib.cure_prompt_attn.argtypes = [P, P, P, C.POINTER(KVDesc), P, P, I32, I32, I32, C.c_float, P, P, C.c_size_t, P]
    lib.cure_selftest_prompt_timeout.argtypes = [*lib.cure_prompt_attn.argtypes[:-1], I32, I32, P]
    lib.cure_prompt_attn_workspace_size.argtypes = [I32, I32, I32, C.POINTER(KVDesc)]
    lib.cure_prompt_attn_workspace_size.restype = C.c_size_t
    lib.cure_rope_qkv_axes.argtypes = [P, P, P, I64, I64, I64, I32, I32, I32, I32, P, C.POINTER(RopeAxes),
                                       C.POINTER(Rope), P, P, C.c_float, P, P, P, I64, I64, I64, P]
    lib.cure_append_kv_axes.argtypes = [P, P, P, I64, I64, I64, I32, I32, I32, P, P, P, C.POINTER(RopeAxes),
                                        C.POINTER(KVDesc), P, P, C.POINTER(Rope), P, P, C.c_float, P, I64, P]
    lib.cure_append_kv8.argtypes = [P, P, P, I64, I64, I64, I32, I32, I32, P, P, P, C.POINTER(RopeAxes),
                                    C.POINTER(KVDesc), P, P, P, P, C.POINTER(Rope), P, P, C.c_float, P, I64, P]
    lib.cure_prompt_attn8.argtypes = [P, P, P, P, P, C.POINTER(KVDesc), P, P, I32, I32, I32, C.c_float, P, P, C.c_size_t,
                                      P]
    lib.cure_prompt_attn8_workspace_size.argtypes = [I32, I32, I32, C.POINTER(KVDesc)]
    lib.cure_prompt_attn8_workspace_size.restype = C.c_size_t
    lib.cure_tree_attn8.argtypes = [P, P, P, P, P, C.POINTER(KVDesc), P, P, P, I32, I32, I32, C.c_float, P, P, C.c_size_t,
                                    P]
    lib.cure_tree_attn8_workspace_size.argtypes = [I32, I32, I32, C.POINTER(KVDesc)]
    lib.cure_tree_attn8_workspace_size.restype = C.c_size_t
    lib.cure_resync_kv8.argtypes = [I32, C.POINTER(C.c_void_p), C.POINTER(C.c_void_p), C.POINTER(C.c_void_p),
                                    C.POINTER(C.c_void_p), C.POINTER(KVDesc), P, P, I32, I32, I32, P, P, P, P, P, P, P, P,
                                    P, P]
    lib.cure_save_kv8.argtypes = [I32, C.POINTER(C.c_void_p), C.POINTER(C.c_void_p), C.POINTER(C.c_void_p),
                                  C.POINTER(C.c_void_p), C.POINTER(KVDesc), I32, P, P, C.c_size_t, P]
    lib.cure_restore_kv8.argtypes = lib.cure_save_kv8.argtypes
    lib.cure_save_kv8_size.argtypes = [I32, I32, C.POINTER(KVDesc)]
    lib.cure_save_kv8_size.restype = C.c_size_t
    lib.cure_selftest_prompt8_timeout.argtypes = [*lib.cure_prompt_attn8.argtypes[:-1], I32, I32, P]
    lib.cure_selftest_tree8_timeout.argtypes = [*lib.cure_tree_attn8.argtypes[:-1], I32, I32, P]
    lib.cure_device_error.argtypes = [P, C.POINTER(I32)]
    lib.cure_status_string.argtypes = [C.c_int]
    lib.cure_status_string.restype = C.c_char_p
    lib.cure_abi_version.restype = I32
    for name in ("cure_score_draft", "cure_build_tree", "cure_tree_attn", "cure_accept",
                 "cure_resync_kv", "cure_device_error", "cure_sample_target", "cure_lm_head_argmax",
                 "cure_rope_init", "cure_rope_init_freqs", "cure_rope_qkv", "cure_append_kv", "cure_prompt_attn",
                 "cure_rope_qkv_axes", "cure_append_kv_axes", "cure_append_kv8", "cure_prompt_attn8", "cure_tree_attn8",
                 "cure_resync_kv8", "cure_save_kv8", "cure_restore_kv8"):
        getattr(lib, name).restype = C.c_int
    _lib = lib
    return lib


def check(fn: str, code: int) -> None:
    if code != CURE_OK:
        raise CureError(fn, code)

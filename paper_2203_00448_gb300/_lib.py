"""ctypes loader for libmemplan.so (the C ABI declared in include/memplan.h).

Loads the in-tree library only.  There is no fallback: if the library is
missing the import of any compute entry point raises.
"""
from __future__ import annotations

import ctypes
import os

from .build import LIB_PATH

OK, EINVAL, EOVERFLOW, ECUDA, ETIMEOUT, ENOMEM, EINTERNAL = range(7)
FIT_FIRST, FIT_BEST = 0, 1

# Every symbol include/memplan.h declares.
EXPORTS = (
    "mp_live_profile",
    "mp_plan_workspace_bytes",
    "mp_plan_greedy_by_size",
    "mp_plan_greedy_by_size_static",
    "mp_plan_and_validate",
    "mp_host_path_bytes",
    "mp_plan_and_validate_host",
    "mp_validate_workspace_bytes",
    "mp_validate_plan",
    "mp_peak",
    "mp_bump_workspace_bytes",
    "mp_plan_bump",
    "mp_optimal_workspace_bytes",
    "mp_plan_optimal",
    "mp_breadth_workspace_bytes",
    "mp_plan_greedy_by_breadth",
    "mp_slab_layout",
    "mp_replay_workspace_bytes",
    "mp_replay_plan",
    "mp_kv_write",
    "mp_kv_read",
    "mp_kv_attend_workspace_bytes",
    "mp_kv_attend",
    "mp_kv_four_write",
    "mp_kv_four_read",
    "mp_kv_four_attend_workspace_bytes",
    "mp_kv_four_attend",
    "mp_kv_extend_workspace_bytes",
    "mp_kv_extend",
    "mp_rotary",
    "mp_status_string",
    "mp_abi_version",
)


class MpBatch(ctypes.Structure):
    """Mirror of struct mp_batch."""

    _fields_ = [
        ("n_traces", ctypes.c_int32),
        ("max_tensors", ctypes.c_int32),
        ("max_steps", ctypes.c_int32),
        ("reserved0", ctypes.c_int32),
        ("n_tensors", ctypes.c_int64),
        ("n_steps", ctypes.c_int64),
        ("trace_ptr", ctypes.c_void_p),
        ("steps", ctypes.c_void_p),
        ("profile_ptr", ctypes.c_void_p),
        ("alloc_step", ctypes.c_void_p),
        ("free_step", ctypes.c_void_p),
        ("size_bytes", ctypes.c_void_p),
    ]


class MpHostResults(ctypes.Structure):
    """Mirror of struct mp_host_results."""

    _fields_ = [(name, ctypes.c_void_p) for name in
                ("profile", "peak_lb", "offsets", "plan_peak", "verdict", "conflict", "trace_status")]


class MpKvCache(ctypes.Structure):
    """Mirror of struct mp_kv_cache."""

    _fields_ = [(n, ctypes.c_int32) for n in ("n_blocks", "block_tokens", "n_heads", "head_dim")] + \
        [(n, ctypes.c_void_p) for n in ("k", "v", "k_scale", "v_scale")]


class MpKvBatch(ctypes.Structure):
    """Mirror of struct mp_kv_batch."""

    _fields_ = [(n, ctypes.c_int32) for n in ("n_seqs", "max_blocks", "max_tokens", "max_len")] + \
        [("n_tokens", ctypes.c_int64)] + [(n, ctypes.c_void_p) for n in ("table", "lens", "token_ptr")]


class MpTokens(ctypes.Structure):
    """Mirror of struct mp_tokens."""

    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("n_heads", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class MpKv4Cache(ctypes.Structure):
    """Mirror of struct mp_kv4_cache."""

    _fields_ = [(n, ctypes.c_int32) for n in ("n_blocks", "block_tokens", "n_heads", "head_dim")] + \
        [(n, ctypes.c_void_p) for n in ("k", "v")]


class MpKvBlocks(ctypes.Structure):
    """Mirror of struct mp_kv_blocks."""

    _fields_ = [(n, ctypes.c_int32) for n in ("n_seqs", "max_blocks", "block_tokens", "n_blocks")] + \
        [(n, ctypes.c_void_p) for n in ("table", "free", "first", "room")]


class MpKvExtension(ctypes.Structure):
    """Mirror of struct mp_kv_extension."""

    _fields_ = [("n_tokens", ctypes.c_int64), ("max_tokens", ctypes.c_int32), ("max_len", ctypes.c_int32)] + \
        [(n, ctypes.c_void_p) for n in ("lens", "n_free", "n_new", "lens_out", "n_free_out", "step_lens", "token_ptr",
                                        "positions", "slots", "seq_status")]


class MpRotation(ctypes.Structure):
    """Mirror of struct mp_rotation."""

    _fields_ = [("dim", ctypes.c_int32), ("layout", ctypes.c_int32), ("turns", ctypes.c_void_p), ("amplitude", ctypes.c_float)]


HOST_PATH_MAX_CHUNKS = 64
SLAB_ALIGN = 256  # MP_SLAB_ALIGN


class MemplanError(RuntimeError):
    def __init__(self, fn: str, status: int):
        super().__init__(f"{fn} returned {status_string(status)}")
        self.status = status


_lib = None


def load(path: str = LIB_PATH):
    """Loads libmemplan.so and declares the signatures; raises if it is absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with paper_2203_00448_gb300.build.build() "
                           "(there is no CPU fallback)")
    lib = ctypes.CDLL(path)
    P, BP = ctypes.c_void_p, ctypes.POINTER(MpBatch)
    i32, sz = ctypes.c_int32, ctypes.c_size_t
    lib.mp_live_profile.argtypes = [BP, P, P, P, P]
    lib.mp_live_profile.restype = i32
    lib.mp_plan_workspace_bytes.argtypes = [BP]
    lib.mp_plan_workspace_bytes.restype = sz
    lib.mp_plan_greedy_by_size.argtypes = [BP, i32, P, P, P, P, sz, P]
    lib.mp_plan_greedy_by_size.restype = i32
    lib.mp_plan_greedy_by_size_static.argtypes = [BP, i32, P, P, P, P]
    lib.mp_plan_greedy_by_size_static.restype = i32
    lib.mp_plan_and_validate.argtypes = [BP, i32, P, P, P, P, P, P, P, P, sz, P]
    lib.mp_plan_and_validate.restype = i32
    lib.mp_host_path_bytes.argtypes = [BP, i32]
    lib.mp_host_path_bytes.restype = sz
    lib.mp_plan_and_validate_host.argtypes = [BP, i32, ctypes.POINTER(MpHostResults), i32, P, sz, P, P, P]
    lib.mp_plan_and_validate_host.restype = i32
    lib.mp_validate_workspace_bytes.argtypes = [BP]
    lib.mp_validate_workspace_bytes.restype = sz
    lib.mp_validate_plan.argtypes = [BP, P, P, P, P, P, sz, P]
    lib.mp_validate_plan.restype = i32
    lib.mp_peak.argtypes = [BP, P, P, P, P]
    lib.mp_peak.restype = i32
    lib.mp_bump_workspace_bytes.argtypes = [BP]
    lib.mp_bump_workspace_bytes.restype = sz
    lib.mp_plan_bump.argtypes = [BP, P, P, P, P, sz, P]
    lib.mp_plan_bump.restype = i32
    lib.mp_optimal_workspace_bytes.argtypes = [BP]
    lib.mp_optimal_workspace_bytes.restype = sz
    lib.mp_plan_optimal.argtypes = [BP, P, P, P, P, sz, P]
    lib.mp_plan_optimal.restype = i32
    lib.mp_breadth_workspace_bytes.argtypes = [BP]
    lib.mp_breadth_workspace_bytes.restype = sz
    lib.mp_plan_greedy_by_breadth.argtypes = [BP, i32, P, P, P, P, sz, P]
    lib.mp_plan_greedy_by_breadth.restype = i32
    lib.mp_slab_layout.argtypes = [BP, P, P, P, P, P, P]
    lib.mp_slab_layout.restype = i32
    lib.mp_replay_workspace_bytes.argtypes = [BP]
    lib.mp_replay_workspace_bytes.restype = sz
    lib.mp_replay_plan.argtypes = [BP, P, P, P, ctypes.c_int64, P, P, P, P, sz, P]
    lib.mp_replay_plan.restype = i32
    CP, KP, TP = (ctypes.POINTER(t) for t in (MpKvCache, MpKvBatch, MpTokens))
    lib.mp_kv_write.argtypes = [CP, KP, TP, TP, P, P]
    lib.mp_kv_write.restype = i32
    lib.mp_kv_read.argtypes = [CP, KP, TP, TP, P, P]
    lib.mp_kv_read.restype = i32
    lib.mp_kv_attend_workspace_bytes.argtypes = [CP, KP, i32]
    lib.mp_kv_attend_workspace_bytes.restype = sz
    lib.mp_kv_attend.argtypes = [CP, KP, TP, ctypes.c_float, i32, i32, TP, P, P, P, sz, P]
    lib.mp_kv_attend.restype = i32
    CP4, XP, EP, RP = (ctypes.POINTER(t) for t in (MpKv4Cache, MpKvBlocks, MpKvExtension, MpRotation))
    lib.mp_kv_four_write.argtypes = [CP4, KP, TP, TP, P, P]
    lib.mp_kv_four_write.restype = i32
    lib.mp_kv_four_read.argtypes = [CP4, KP, TP, TP, P, P]
    lib.mp_kv_four_read.restype = i32
    lib.mp_kv_four_attend_workspace_bytes.argtypes = [CP4, KP, i32]
    lib.mp_kv_four_attend_workspace_bytes.restype = sz
    lib.mp_kv_four_attend.argtypes = [CP4, KP, TP, ctypes.c_float, i32, i32, TP, P, P, P, sz, P]
    lib.mp_kv_four_attend.restype = i32
    lib.mp_kv_extend_workspace_bytes.argtypes = [XP]
    lib.mp_kv_extend_workspace_bytes.restype = sz
    lib.mp_kv_extend.argtypes = [XP, EP, P, sz, P]
    lib.mp_kv_extend.restype = i32
    lib.mp_rotary.argtypes = [RP, P, ctypes.c_int64, i32, TP, TP, TP, TP, i32, P]
    lib.mp_rotary.restype = i32
    lib.mp_status_string.argtypes = [i32]
    lib.mp_status_string.restype = ctypes.c_char_p
    lib.mp_abi_version.argtypes = []
    lib.mp_abi_version.restype = i32
    _lib = lib
    return lib


def status_string(status: int) -> str:
    try:
        return load().mp_status_string(int(status)).decode()
    except RuntimeError:
        return f"status {status}"

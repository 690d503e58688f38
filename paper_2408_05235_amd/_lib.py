"""ctypes declarations of the C ABI in include/tl.h and the library loader.

The shared library is built in-tree (``paper_2408_05235_amd/lib/libtl.so``).
Loading never falls back to anything else: if the library is missing it is
built once; if it cannot be built or loaded an ImportError is raised.
"""
from __future__ import annotations

import ctypes
import os

from . import build as _build

P = ctypes.c_void_p
i32, i64, u32, f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32, ctypes.c_float

TL_OK, TL_EINVAL, TL_ENOMEM, TL_EDEVICE, TL_EUNSUPPORTED = 0, 1, 2, 3, 4
FLAG_BAD_REQUEST, FLAG_LOST, FLAG_OVERCOMMIT, FLAG_OVERFLOW, FLAG_UNSORTED = 1, 2, 4, 8, 16
FLAG_BAD_CANDIDATE = 32
STATUS_OK, STATUS_INFEASIBLE, STATUS_LOST, STATUS_INVALID = 0, 1, 2, 3
ADMIT_OK, ADMIT_LOST, ADMIT_QUEUE_CAPACITY, ADMIT_QUEUE_TBT, ADMIT_QUEUE_E2E, ADMIT_INVALID = 0, 1, 2, 3, 4, 5
BF16, F16 = 1, 2
PAGES_OK, PAGES_NONE_FREE, PAGES_TABLE_FULL, PAGES_BAD = 0, 1, 2, 3
MAX_HEAD_DIM = 256
MAX_HORIZON, MAX_BLOCK_TOKENS, MAX_FREQS, MAX_FEATURES, MAX_DEPTH = 8192, 65536, 4096, 4, 14

EXPORTED = ("tl_abi_version", "tl_last_error", "tl_forest_create", "tl_forest_destroy",
            "tl_project", "tl_forest_predict", "tl_forest_predict_grid", "tl_select_freq", "tl_admit",
            "tl_select_freq_binary", "tl_adjust_lengths", "tl_lattice_create", "tl_lattice_destroy",
            "tl_lattice_bytes", "tl_lattice_predict_grid", "tl_forest_predict_grid_noalloc",
            "tl_kv_append", "tl_attend", "tl_attend_workspace_bytes", "tl_pages_work_words", "tl_pages_extend",
            "tl_pages_fork", "tl_pages_free", "tl_pages_compact", "tl_pages_copy")


class ProjectArgs(ctypes.Structure):
    _fields_ = [
        ("struct_size", u32), ("horizon", i32), ("n_scenarios", i64), ("n_requests", i64),
        ("block_tokens", i32), ("n_freqs", i32), ("n_features", i32), ("reserved", i32),
        ("req_offset", P), ("prompt_len", P), ("generated", P), ("remaining", P),
        ("arrival_iter", P), ("deadline_ns", P), ("lost", P), ("kv_capacity", P),
        ("batch_cap", P), ("batch", P), ("kv", P), ("deadline_at", P), ("n_iters", P),
        ("flags", P), ("freqs_mhz", P), ("engine_size", P), ("rows", P),
    ]


class AdmitArgs(ctypes.Structure):
    _fields_ = [
        ("struct_size", u32), ("reserved", u32), ("proj", ProjectArgs), ("forest", P),
        ("max_freq_mhz", f32), ("engine_size", P), ("tbt_slo_ns", P), ("cand_prompt", P),
        ("cand_len", P), ("cand_deadline_ns", P), ("ips", P), ("decision", P), ("lattice", P),
    ]


class KvView(ctypes.Structure):
    _fields_ = [
        ("struct_size", u32), ("dtype", i32), ("n_kv_heads", i32), ("head_dim", i32), ("page_tokens", i32),
        ("table_width", i32), ("n_pages", i64), ("n_seqs", i64), ("page_stride", i64), ("head_stride", i64),
        ("token_stride", i64), ("key_pages", P), ("value_pages", P), ("page_table", P), ("length", P),
    ]


class KvAppendArgs(ctypes.Structure):
    _fields_ = [
        ("struct_size", u32), ("reserved", u32), ("cache", KvView), ("n_tokens", i64), ("q_offset", P), ("key", P),
        ("value", P), ("key_token_stride", i64), ("key_head_stride", i64), ("value_token_stride", i64),
        ("value_head_stride", i64), ("granted", P),
    ]


class AttendArgs(ctypes.Structure):
    _fields_ = [
        ("struct_size", u32), ("n_heads", i32), ("cache", KvView), ("n_tokens", i64), ("q_offset", P), ("query", P),
        ("query_token_stride", i64), ("query_head_stride", i64), ("scale", f32), ("window", i32), ("sinks", i32),
        ("max_length", i32), ("out", P), ("lse", P), ("workspace", P), ("workspace_bytes", ctypes.c_uint64),
        ("granted", P),
    ]


class Pages(ctypes.Structure):
    _fields_ = [
        ("struct_size", u32), ("page_tokens", i32), ("n_pages", i64), ("n_slots", i64), ("table_width", i32),
        ("reserved", i32), ("ref", P), ("page_table", P), ("length", P), ("granted", P),
    ]


class TLError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"tl status {status}: {message}")
        self.status = status


_lib = None


def lib():
    """The loaded libtl.so (built first if it does not exist yet)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_build.LIB_PATH):
        _build.build_library()
    try:
        L = ctypes.CDLL(_build.LIB_PATH)
    except OSError as e:
        raise ImportError(f"cannot load {_build.LIB_PATH}: {e}") from e
    L.tl_abi_version.argtypes = []
    L.tl_abi_version.restype = i32
    L.tl_last_error.argtypes = []
    L.tl_last_error.restype = ctypes.c_char_p
    L.tl_forest_create.argtypes = [i32, i32, i32, f32, P, P, P, ctypes.POINTER(P)]
    L.tl_forest_create.restype = ctypes.c_int
    L.tl_forest_destroy.argtypes = [P]
    L.tl_forest_destroy.restype = None
    L.tl_project.argtypes = [ctypes.POINTER(ProjectArgs), P]
    L.tl_project.restype = ctypes.c_int
    L.tl_forest_predict.argtypes = [P, P, i64, P, P]
    L.tl_forest_predict.restype = ctypes.c_int
    L.tl_forest_predict_grid.argtypes = [P, i64, i32, i32, P, P, P, P, P, P]
    L.tl_forest_predict_grid.restype = ctypes.c_int
    L.tl_forest_predict_grid_noalloc.argtypes = [P, i64, i32, i32, P, P, P, P, P, P]
    L.tl_forest_predict_grid_noalloc.restype = ctypes.c_int
    L.tl_select_freq.argtypes = [P, i64, i32, i32, P, P, P, P, P, P, P]
    L.tl_select_freq.restype = ctypes.c_int
    L.tl_select_freq_binary.argtypes = [P, i64, i32, i32] + [P] * 14
    L.tl_select_freq_binary.restype = ctypes.c_int
    L.tl_lattice_create.argtypes = [P, i32, P, i32, P, i32, i32, P, ctypes.POINTER(P)]
    L.tl_lattice_create.restype = ctypes.c_int
    L.tl_lattice_destroy.argtypes = [P]
    L.tl_lattice_destroy.restype = None
    L.tl_lattice_bytes.argtypes = [P]
    L.tl_lattice_bytes.restype = ctypes.c_uint64
    L.tl_lattice_predict_grid.argtypes = [P, i64, i32, P, P, P, P, P]
    L.tl_lattice_predict_grid.restype = ctypes.c_int
    L.tl_adjust_lengths.argtypes = [i64, i64] + [P] * 8
    L.tl_adjust_lengths.restype = ctypes.c_int
    L.tl_admit.argtypes = [ctypes.POINTER(AdmitArgs), P]
    L.tl_admit.restype = ctypes.c_int
    L.tl_kv_append.argtypes = [ctypes.POINTER(KvAppendArgs), P]
    L.tl_kv_append.restype = ctypes.c_int
    L.tl_attend.argtypes = [ctypes.POINTER(AttendArgs), P]
    L.tl_attend.restype = ctypes.c_int
    L.tl_attend_workspace_bytes.argtypes = [ctypes.POINTER(AttendArgs)]
    L.tl_attend_workspace_bytes.restype = ctypes.c_uint64
    L.tl_pages_work_words.argtypes = [ctypes.POINTER(Pages)]
    L.tl_pages_work_words.restype = ctypes.c_uint64
    L.tl_pages_extend.argtypes = [ctypes.POINTER(Pages)] + [P] * 4
    L.tl_pages_extend.restype = ctypes.c_int
    L.tl_pages_fork.argtypes = [ctypes.POINTER(Pages), i64] + [P] * 7
    L.tl_pages_fork.restype = ctypes.c_int
    L.tl_pages_free.argtypes = [ctypes.POINTER(Pages), i64, P, P]
    L.tl_pages_free.restype = ctypes.c_int
    L.tl_pages_compact.argtypes = [ctypes.POINTER(Pages)] + [P] * 7
    L.tl_pages_compact.restype = ctypes.c_int
    L.tl_pages_copy.argtypes = [P, i64, i64, i64, i32, i64, P, P, i64, P, P]
    L.tl_pages_copy.restype = ctypes.c_int
    _lib = L
    return L


def check(status):
    if status != TL_OK:
        msg = lib().tl_last_error()
        raise TLError(status, msg.decode() if msg else "")
    return status

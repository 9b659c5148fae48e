"""Python binding of libmma.so -- multipath host<->GPU copies on one MI355X.

Argument marshalling only: every function forwards to the C entry point of the
same name in ``include/mma.h``; all data movement runs in the library's HIP
kernels and SDMA submissions. PyTorch provides device memory and streams.

``import torch`` happens before the library is loaded so that libmma.so binds to
the HIP runtime already in the process (one runtime, shared streams). If the
library has not been built this import fails loudly -- there is no fallback.
"""
from __future__ import annotations

import ctypes
import importlib.util
import os
from typing import Iterable, List, Optional, Sequence, Tuple

import numpy as np
import torch  # noqa: F401  (loads the process's HIP runtime first)

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmma.so")

MMA_OK = 0
MMA_ERR_NOT_INITIALIZED = -1
MMA_ERR_INVALID_ARG = -2
MMA_ERR_NOT_PINNED = -3
MMA_ERR_HIP = -4
MMA_ERR_TRANSFER_FAILED = -6
MMA_ERR_TIMEOUT = -10
MMA_ERR_NO_MEMORY = -8
MMA_ERR_INTERNAL = -11
MMA_H2D = 0
MMA_D2H = 1
MMA_PATH_CU = 0x80000000
MMA_DUPLEX_UNCHANGED = 0xFFFFFFFF  # duplex_paths_*: keep the direction's own paths
MMA_ENGINE_NAP_OFF = 0xFFFFFFFF  # engine_nap_us: the engine threads poll without sleeping
MMA_KV_LAYOUT_PIECE = 0
MMA_KV_LAYOUT_XPACKED = 1
MMA_KV_LAYOUT_HND = 2
MMA_CONTROL_HOST = 0
MMA_CONTROL_DEVICE = 1
MMA_NUM_PATHS = 17
MMA_FAULT_ENGINE_STALL_US = 1
MMA_FAULT_SDMA_SUBMIT_FAIL = 2
MMA_FAULT_ENGINE_IGNORE = 3
MMA_FAULT_DEVICE_SIGNAL_HOLD = 4
MMA_FAULT_POOL_NO_TABLE = 5
MMA_COPY_NOT_ENQUEUED = 0
MMA_COPY_RETIRED = 1
MMA_COPY_IN_FLIGHT = 2
MMA_TASK_CU_ONLY = 1
MMA_TASK_SDMA_ONLY = 2

MMA_TYPE_BF16 = 0
MMA_TYPE_F16 = 1
MMA_TYPE_F8 = 2
MMA_TYPE_F32 = 3
MMA_ROPE_NONE = 0
MMA_ROPE_LINEAR = 1
MMA_ROPE_BASE = 2
MMA_ROPE_RAMP = 3
MMA_ROPE_BANDS = 4

STATUS = {
    0: "MMA_OK", -1: "MMA_ERR_NOT_INITIALIZED", -2: "MMA_ERR_INVALID_ARG", -3: "MMA_ERR_NOT_PINNED",
    -4: "MMA_ERR_HIP", -5: "MMA_ERR_HSA", -6: "MMA_ERR_TRANSFER_FAILED", -7: "MMA_ERR_ALREADY_INITIALIZED",
    -8: "MMA_ERR_NO_MEMORY", -9: "MMA_ERR_BUFFER_TOO_SMALL", -10: "MMA_ERR_TIMEOUT", -11: "MMA_ERR_INTERNAL",
}


class MMAError(RuntimeError):
    def __init__(self, status: int, func: str, detail: str):
        self.status = status
        self.name = STATUS.get(status, str(status))
        super().__init__(f"{func}: {self.name}: {detail}")


class mma_config_t(ctypes.Structure):
    _fields_ = [("chunk_bytes", ctypes.c_uint64), ("fallback_bytes", ctypes.c_uint64),
                ("small_bytes", ctypes.c_uint64), ("queue_depth", ctypes.c_uint32),
                ("cu_queue_depth", ctypes.c_uint32), ("backoff_depth", ctypes.c_uint32),
                ("path_mask_h2d", ctypes.c_uint32), ("path_mask_d2h", ctypes.c_uint32),
                ("cu_workgroups", ctypes.c_uint32), ("cu_sub_bytes", ctypes.c_uint32),
                ("watchdog_ms", ctypes.c_uint32), ("static_split", ctypes.c_uint32),
                ("static_cu_percent", ctypes.c_uint32), ("sdma_merge_tasks", ctypes.c_uint32),
                ("cu_whole_bytes", ctypes.c_uint32), ("cu_whole_bytes_d2h", ctypes.c_uint32),
                ("control", ctypes.c_uint32), ("duplex_paths_h2d", ctypes.c_uint32),
                ("duplex_paths_d2h", ctypes.c_uint32), ("engine_nap_us", ctypes.c_uint32)]

    def as_dict(self):
        return {k: getattr(self, k) for k, _ in self._fields_}


class mma_copy_desc_t(ctypes.Structure):
    _fields_ = [("dst", ctypes.c_void_p), ("src", ctypes.c_void_p), ("bytes", ctypes.c_uint64)]


class mma_kv_layout_t(ctypes.Structure):
    _fields_ = [("num_layers", ctypes.c_uint32), ("block_tokens", ctypes.c_uint32),
                ("kv_heads", ctypes.c_uint32), ("head_dim", ctypes.c_uint32),
                ("elem_bytes", ctypes.c_uint32), ("gpu_num_blocks", ctypes.c_uint32),
                ("host_num_slots", ctypes.c_uint32), ("gpu_layout", ctypes.c_uint32)]


class mma_stats_t(ctypes.Structure):
    _fields_ = [("transfers", ctypes.c_uint64), ("failed_transfers", ctypes.c_uint64),
                ("path_bytes", ctypes.c_uint64 * MMA_NUM_PATHS), ("path_tasks", ctypes.c_uint64 * MMA_NUM_PATHS),
                ("staging_bytes", ctypes.c_uint64), ("sdma_submit_failures", ctypes.c_uint64),
                ("engine_cpu_ns", ctypes.c_uint64), ("engine_wall_busy_ns", ctypes.c_uint64),
                ("sdma_foreign_busy_skips", ctypes.c_uint64), ("sdma_congestion_backoffs", ctypes.c_uint64),
                ("sdma_commands", ctypes.c_uint64),
                ("sdma_engines_h2d", ctypes.c_uint32), ("sdma_engines_d2h", ctypes.c_uint32),
                ("cu_path_enabled", ctypes.c_uint32), ("reserved", ctypes.c_uint32),
                ("pool_launches", ctypes.c_uint64), ("engine_naps", ctypes.c_uint64)]

    def as_dict(self):
        d = {k: getattr(self, k) for k, _ in self._fields_ if k not in ("reserved", "path_bytes", "path_tasks")}
        d["path_bytes"] = list(self.path_bytes)
        d["path_tasks"] = list(self.path_tasks)
        return d


class mma_trace_rec_t(ctypes.Structure):
    _fields_ = [("seq", ctypes.c_uint64), ("dir", ctypes.c_int32), ("kind", ctypes.c_int32),
                ("bytes", ctypes.c_uint64), ("tasks", ctypes.c_uint64),
                ("t_api_ns", ctypes.c_uint64), ("t_submit_ns", ctypes.c_uint64), ("t_started_ns", ctypes.c_uint64),
                ("t_first_sdma_ns", ctypes.c_uint64), ("t_last_task_ns", ctypes.c_uint64),
                ("t_complete_ns", ctypes.c_uint64), ("t_retire_ns", ctypes.c_uint64),
                ("path_tasks", ctypes.c_uint64 * MMA_NUM_PATHS), ("failed", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]

    def as_dict(self):
        d = {k: getattr(self, k) for k, _ in self._fields_ if k not in ("reserved", "path_tasks")}
        d["path_tasks"] = list(self.path_tasks)
        return d


class mma_plan_entry_t(ctypes.Structure):
    _fields_ = [("item", ctypes.c_uint64), ("offset", ctypes.c_uint64), ("bytes", ctypes.c_uint64),
                ("flags", ctypes.c_uint32), ("reserved", ctypes.c_uint32)]


class mma_kv_seqs_t(ctypes.Structure):
    _fields_ = [("block_table", ctypes.c_void_p), ("lens", ctypes.c_void_p), ("q_start", ctypes.c_void_p),
                ("num_seqs", ctypes.c_uint32), ("table_stride", ctypes.c_uint32),
                ("max_tokens", ctypes.c_uint32), ("max_len", ctypes.c_uint32)]


class mma_rows_t(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_uint64), ("head_stride", ctypes.c_uint64)]


class mma_rope_t(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_uint32), ("kind", ctypes.c_uint32), ("base", ctypes.c_double),
                ("factor", ctypes.c_double), ("original_len", ctypes.c_double), ("low", ctypes.c_double),
                ("high", ctypes.c_double)]


class mma_kv_append_t(ctypes.Structure):
    _fields_ = [("q", mma_rows_t), ("k", mma_rows_t), ("v", mma_rows_t), ("q_out", mma_rows_t),
                ("positions", ctypes.c_void_p), ("rope", ctypes.c_void_p), ("q_weight", ctypes.c_void_p),
                ("k_weight", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("num_tokens", ctypes.c_uint32), ("q_heads", ctypes.c_uint32), ("type", ctypes.c_uint32),
                ("cache_type", ctypes.c_uint32), ("rot_dim", ctypes.c_uint32), ("rope_rows", ctypes.c_uint32),
                ("interleaved", ctypes.c_uint32), ("eps", ctypes.c_float)]


class mma_kv_attention_t(ctypes.Structure):
    _fields_ = [("q", mma_rows_t), ("out", mma_rows_t), ("tree", ctypes.c_void_p), ("lse", ctypes.c_void_p),
                ("scores_in", ctypes.c_void_p), ("scores_out", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_uint64),
                ("num_tokens", ctypes.c_uint32), ("q_heads", ctypes.c_uint32), ("type", ctypes.c_uint32),
                ("cache_type", ctypes.c_uint32), ("tree_words", ctypes.c_uint32), ("scores_stride", ctypes.c_uint32),
                ("scale", ctypes.c_float), ("decay", ctypes.c_float)]


class mma_kv_shape_t(ctypes.Structure):
    _fields_ = [("slopes", ctypes.c_void_p), ("prefix", ctypes.c_void_p), ("max_prefix", ctypes.c_uint32),
                ("window", ctypes.c_uint32), ("softcap", ctypes.c_float)]


class mma_kv_commit_t(ctypes.Structure):
    _fields_ = [("accepted", ctypes.c_void_p), ("counts", ctypes.c_void_p), ("lens_out", ctypes.c_void_p),
                ("scores", ctypes.c_void_p), ("accepted_stride", ctypes.c_uint32), ("scores_stride", ctypes.c_uint32)]


class mma_kv_evict_t(ctypes.Structure):
    _fields_ = [("dst_table", ctypes.c_void_p), ("scores", ctypes.c_void_p), ("entries", ctypes.c_void_p),
                ("scores_out", ctypes.c_void_p), ("lens_out", ctypes.c_void_p), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_uint64), ("dst_stride", ctypes.c_uint32),
                ("scores_stride", ctypes.c_uint32), ("keep", ctypes.c_uint32), ("sinks", ctypes.c_uint32),
                ("recent", ctypes.c_uint32)]


class mma_beam_select_t(ctypes.Structure):
    _fields_ = [("logits", ctypes.c_void_p), ("scores", ctypes.c_void_p), ("done", ctypes.c_void_p),
                ("tokens", ctypes.c_void_p), ("parents", ctypes.c_void_p), ("scores_out", ctypes.c_void_p),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_uint64), ("row_stride", ctypes.c_uint64),
                ("batch", ctypes.c_uint32), ("beams", ctypes.c_uint32), ("vocab", ctypes.c_uint32),
                ("keep", ctypes.c_uint32), ("type", ctypes.c_uint32), ("done_token", ctypes.c_int32)]


class mma_kv_fork_t(ctypes.Structure):
    _fields_ = [("parents", ctypes.c_void_p), ("grow", ctypes.c_void_p), ("refs", ctypes.c_void_p),
                ("refs_out", ctypes.c_void_p), ("table_out", ctypes.c_void_p), ("lens_out", ctypes.c_void_p),
                ("free_out", ctypes.c_void_p), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_uint64),
                ("num_children", ctypes.c_uint32), ("out_stride", ctypes.c_uint32)]


class mma_kv_compact_t(ctypes.Structure):
    _fields_ = [("block_table", ctypes.c_void_p), ("table_out", ctypes.c_void_p), ("refs", ctypes.c_void_p),
                ("refs_out", ctypes.c_void_p), ("moved", ctypes.c_void_p), ("held_out", ctypes.c_void_p),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_uint64), ("num_seqs", ctypes.c_uint32),
                ("table_stride", ctypes.c_uint32)]


_P = ctypes.c_void_p
_U64 = ctypes.c_uint64
_I32 = ctypes.c_int32
_U32 = ctypes.c_uint32
_S = ctypes.c_int32

# name -> (argtypes, restype)
_SIGNATURES = {
    "mma_config_default": ([ctypes.POINTER(mma_config_t)], _S),
    "mma_init": ([ctypes.c_int, ctypes.POINTER(mma_config_t)], _S),
    "mma_finalize": ([], _S),
    "mma_get_config": ([ctypes.POINTER(mma_config_t)], _S),
    "mma_synchronize": ([_U32], _S),
    "mma_host_alloc": ([_U64, ctypes.POINTER(_P)], _S),
    "mma_host_free": ([_P], _S),
    "mma_memcpy_async": ([_P, _P, _U64, _I32, _P], _S),
    "mma_memcpy": ([_P, _P, _U64, _I32], _S),
    "mma_memcpy_stream": ([_P, _P, _U64, _I32, _P, ctypes.POINTER(_I32)], _S),
    "mma_weights_load": ([ctypes.POINTER(mma_copy_desc_t), _U64, _I32, _P], _S),
    # the layer array and the two tables go as plain addresses: a ctypes pointer cast costs
    # microseconds per call, as much as a small transfer's whole host-side set-up
    "mma_kv_fetch": ([ctypes.POINTER(mma_kv_layout_t), _P, _P, _P, _P, _U64, _P], _S),
    "mma_kv_offload": ([ctypes.POINTER(mma_kv_layout_t), _P, _P, _P, _P, _U64, _P], _S),
    "mma_kv_fetch_noalloc": ([ctypes.POINTER(mma_kv_layout_t), _P, _P, _P, _P, _U64, _P], _S),
    "mma_digest_u32": ([_P, _U64, _P, _P], _S),
    "mma_rope_table": ([ctypes.POINTER(mma_rope_t), _U64, _P], _S),
    "mma_kv_append": ([ctypes.POINTER(mma_kv_layout_t), _P, ctypes.POINTER(mma_kv_seqs_t),
                       ctypes.POINTER(mma_kv_append_t), _P], _S),
    "mma_kv_attention": ([ctypes.POINTER(mma_kv_layout_t), _P, ctypes.POINTER(mma_kv_seqs_t),
                          ctypes.POINTER(mma_kv_attention_t), _P], _S),
    "mma_kv_attention_workspace": ([ctypes.POINTER(mma_kv_layout_t), ctypes.POINTER(mma_kv_seqs_t),
                                    ctypes.POINTER(mma_kv_attention_t), ctypes.POINTER(_U64)], _S),
    "mma_kv_attention_shaped": ([ctypes.POINTER(mma_kv_layout_t), _P, ctypes.POINTER(mma_kv_seqs_t),
                                 ctypes.POINTER(mma_kv_attention_t), ctypes.POINTER(mma_kv_shape_t), _P], _S),
    "mma_kv_attention_shaped_workspace": ([ctypes.POINTER(mma_kv_layout_t), ctypes.POINTER(mma_kv_seqs_t),
                                           ctypes.POINTER(mma_kv_attention_t), ctypes.POINTER(mma_kv_shape_t),
                                           ctypes.POINTER(_U64)], _S),
    "mma_kv_commit": ([ctypes.POINTER(mma_kv_layout_t), _P, ctypes.POINTER(mma_kv_seqs_t),
                       ctypes.POINTER(mma_kv_commit_t), _P], _S),
    "mma_kv_evict": ([ctypes.POINTER(mma_kv_layout_t), _P, ctypes.POINTER(mma_kv_seqs_t),
                      ctypes.POINTER(mma_kv_evict_t), _P], _S),
    "mma_kv_evict_workspace": ([ctypes.POINTER(mma_kv_layout_t), ctypes.POINTER(mma_kv_seqs_t), ctypes.POINTER(_U64)], _S),
    "mma_beam_select": ([ctypes.POINTER(mma_beam_select_t), _P], _S),
    "mma_beam_select_workspace": ([ctypes.POINTER(mma_beam_select_t), ctypes.POINTER(_U64)], _S),
    "mma_kv_fork": ([ctypes.POINTER(mma_kv_layout_t), _P, ctypes.POINTER(mma_kv_seqs_t), ctypes.POINTER(mma_kv_fork_t), _P],
                    _S),
    "mma_kv_fork_workspace": ([ctypes.POINTER(mma_kv_fork_t), ctypes.POINTER(_U64)], _S),
    "mma_kv_compact": ([ctypes.POINTER(mma_kv_layout_t), _P, ctypes.POINTER(mma_kv_compact_t), _P], _S),
    "mma_kv_compact_workspace": ([ctypes.POINTER(mma_kv_layout_t), ctypes.POINTER(_U64)], _S),
    "mma_get_stats": ([ctypes.POINTER(mma_stats_t)], _S),
    "mma_reset_stats": ([], _S),
    "mma_status_str": ([_S], ctypes.c_char_p),
    "mma_last_error": ([], ctypes.c_char_p),
    "mma_clear_error": ([], _S),
    "mma_plan_list": ([ctypes.POINTER(_U64), _U64, _U64, _U64, _U64, ctypes.POINTER(mma_plan_entry_t), _U64,
                       ctypes.POINTER(_U64)], _S),
    "mma_plan_kv": ([_U64, _U32, _U64, _U64, ctypes.POINTER(mma_plan_entry_t), _U64, ctypes.POINTER(_U64)], _S),
    "mma_validate_kv_tables": ([ctypes.POINTER(_I32), _U32, ctypes.POINTER(_I32), _U32, _U64], _S),
    "mma_kv_layout_sizes": ([ctypes.POINTER(mma_kv_layout_t), ctypes.POINTER(_U64), ctypes.POINTER(_U64),
                             ctypes.POINTER(_U64), ctypes.POINTER(_U64)], _S),
    "mma_trace_enable": ([_I32], _S),
    "mma_trace_read": ([ctypes.POINTER(mma_trace_rec_t), _U64, ctypes.POINTER(_U64)], _S),
    "mma_test_set_fault": ([_I32, _U64], _S),
}


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python paper_2512_16056_amd/build.py`")
    lib = ctypes.CDLL(LIB_PATH)
    for name, (args, res) in _SIGNATURES.items():
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = res
    return lib


lib = _load()


def _check(status: int, func: str) -> None:
    if status != MMA_OK:
        raise MMAError(status, func, lib.mma_last_error().decode(errors="replace"))


def _ptr(x) -> int:
    """Device/host address of an int, torch tensor, numpy array or PinnedBuffer."""
    if x is None:
        return 0
    if isinstance(x, int):
        return x
    if isinstance(x, torch.Tensor):
        return x.data_ptr()
    if isinstance(x, np.ndarray):
        return x.ctypes.data
    if isinstance(x, PinnedBuffer):
        return x.ptr
    raise TypeError(f"cannot take the address of {type(x)}")


# The handle of torch's current stream, without building a Stream object: the two calls take
# 0.2 us, torch.cuda.current_stream() and is_available() 3.4 us, as much as the rest of a small
# copy's call.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(s) -> int:
    if s is None:
        if _raw_stream is not None and _raw_device is not None and torch.cuda.is_initialized():
            return _raw_stream(_raw_device())
        return torch.cuda.current_stream().cuda_stream if torch.cuda.is_available() else 0
    if isinstance(s, int):
        return s
    return s.cuda_stream


def _i32(a) -> np.ndarray:
    if type(a) is np.ndarray and a.dtype == np.int32 and a.ndim and a.flags.c_contiguous:
        return a
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32))


# ------------------------------------------------------------------ lifecycle
def mma_config_default() -> mma_config_t:
    c = mma_config_t()
    _check(lib.mma_config_default(ctypes.byref(c)), "mma_config_default")
    return c


def mma_init(device: int = 0, cfg: Optional[mma_config_t] = None, **overrides) -> None:
    """Initialise on `device`. cfg=None and no overrides: defaults + MMA_* environment."""
    if overrides and cfg is None:
        cfg = mma_config_t()
    for k, v in overrides.items():
        setattr(cfg, k, v)
    _check(lib.mma_init(device, ctypes.byref(cfg) if cfg is not None else None), "mma_init")


def mma_finalize() -> None:
    _check(lib.mma_finalize(), "mma_finalize")


def mma_get_config() -> mma_config_t:
    c = mma_config_t()
    _check(lib.mma_get_config(ctypes.byref(c)), "mma_get_config")
    return c


def mma_synchronize(timeout_ms: int = 60000) -> None:
    _check(lib.mma_synchronize(timeout_ms), "mma_synchronize")


# ------------------------------------------------------------------ host memory
def mma_host_alloc(nbytes: int) -> int:
    p = ctypes.c_void_p()
    _check(lib.mma_host_alloc(nbytes, ctypes.byref(p)), "mma_host_alloc")
    return p.value or 0


def mma_host_free(ptr: int) -> None:
    _check(lib.mma_host_free(ptr), "mma_host_free")


class PinnedBuffer:
    """Owner of an mma_host_alloc allocation with a zero-copy numpy uint8 view."""

    def __init__(self, nbytes: int):
        self.nbytes = int(nbytes)
        self.ptr = mma_host_alloc(self.nbytes) if self.nbytes else 0
        self.array = (np.ctypeslib.as_array((ctypes.c_uint8 * self.nbytes).from_address(self.ptr))
                      if self.nbytes else np.zeros(0, np.uint8))

    def free(self) -> None:
        if self.ptr:
            self.array = None
            mma_host_free(self.ptr)
            self.ptr = 0

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.free()


# ------------------------------------------------------------------ transfers
def mma_memcpy_async(dst, src, nbytes: int, direction: int, stream=None) -> None:
    _check(lib.mma_memcpy_async(_ptr(dst), _ptr(src), nbytes, direction, _stream(stream)), "mma_memcpy_async")


def mma_memcpy(dst, src, nbytes: int, direction: int) -> None:
    """Blocking copy on the legacy default stream; returns once the data has arrived."""
    _check(lib.mma_memcpy(_ptr(dst), _ptr(src), nbytes, direction), "mma_memcpy")


def mma_memcpy_stream(dst, src, nbytes: int, direction: int, stream=None) -> int:
    """Blocking copy ordered on `stream`; returns the outcome (MMA_COPY_*). A failure raises MMAError,
    whose `outcome` attribute is set."""
    out = ctypes.c_int32(-1)
    st = lib.mma_memcpy_stream(_ptr(dst), _ptr(src), nbytes, direction, _stream(stream), ctypes.byref(out))
    try:
        _check(st, "mma_memcpy_stream")
    except MMAError as e:
        e.outcome = out.value
        raise
    return out.value


def mma_weights_load(copies: Sequence[Tuple[object, object, int]], direction: int, stream=None) -> None:
    """copies: (dst, src, nbytes) triples."""
    n = len(copies)
    arr = (mma_copy_desc_t * max(n, 1))()
    for i, (d, s, b) in enumerate(copies):
        arr[i].dst, arr[i].src, arr[i].bytes = _ptr(d), _ptr(s), int(b)
    _check(lib.mma_weights_load(arr, n, direction, _stream(stream)), "mma_weights_load")


def kv_layout(num_layers, block_tokens, kv_heads, head_dim, elem_bytes, gpu_num_blocks, host_num_slots,
              gpu_layout: int = 0) -> mma_kv_layout_t:
    return mma_kv_layout_t(num_layers, block_tokens, kv_heads, head_dim, elem_bytes, gpu_num_blocks,
                           host_num_slots, gpu_layout)


def layer_table(gpu_layers) -> ctypes.Array:
    """The per-layer GPU base addresses as the C array the KV calls take. A caller that moves
    KV between the same layer tensors many times can build it once and pass it as
    `gpu_layers`; a fresh one costs about 0.3 us per layer."""
    if isinstance(gpu_layers, ctypes.Array):
        return gpu_layers
    ptrs = [_ptr(t) for t in gpu_layers]
    return (ctypes.c_void_p * max(len(ptrs), 1))(*ptrs)


def mma_kv_fetch(layout: mma_kv_layout_t, host_pool, gpu_layers, host_slots, gpu_blocks, stream=None) -> None:
    hs, gb = _i32(host_slots), _i32(gpu_blocks)
    if hs.size != gb.size:
        raise ValueError("host_slots and gpu_blocks differ in length")
    lt = layer_table(gpu_layers)  # a local, so the array outlives the call
    _check(lib.mma_kv_fetch(ctypes.byref(layout), _ptr(host_pool), lt,
                            hs.ctypes.data, gb.ctypes.data, hs.size, _stream(stream)), "mma_kv_fetch")


def mma_kv_fetch_noalloc(layout: mma_kv_layout_t, host_pool, gpu_layers, host_slots, gpu_blocks,
                         stream=None) -> None:
    hs, gb = _i32(host_slots), _i32(gpu_blocks)
    if hs.size != gb.size:
        raise ValueError("host_slots and gpu_blocks differ in length")
    lt = layer_table(gpu_layers)  # a local, so the array outlives the call
    _check(lib.mma_kv_fetch_noalloc(ctypes.byref(layout), _ptr(host_pool), lt,
                                    hs.ctypes.data, gb.ctypes.data, hs.size, _stream(stream)),
           "mma_kv_fetch_noalloc")


def mma_kv_offload(layout: mma_kv_layout_t, host_pool, gpu_layers, gpu_blocks, host_slots, stream=None) -> None:
    gb, hs = _i32(gpu_blocks), _i32(host_slots)
    if hs.size != gb.size:
        raise ValueError("host_slots and gpu_blocks differ in length")
    lt = layer_table(gpu_layers)  # a local, so the array outlives the call
    _check(lib.mma_kv_offload(ctypes.byref(layout), _ptr(host_pool), lt,
                              gb.ctypes.data, hs.ctypes.data, hs.size, _stream(stream)), "mma_kv_offload")


def mma_digest_u32(dev_ptr, nbytes: int, dev_out, stream=None) -> None:
    _check(lib.mma_digest_u32(_ptr(dev_ptr), nbytes, _ptr(dev_out), _stream(stream)), "mma_digest_u32")


# ------------------------------------------------------------------ operators on the paged cache
_TYPES = {torch.bfloat16: MMA_TYPE_BF16, torch.float16: MMA_TYPE_F16}

def _want(name: str, t: torch.Tensor, dtype, shape=None) -> int:
    """Address of a contiguous tensor of the given type and, where given, shape."""
    if t.dtype is not dtype or not t.is_contiguous() or not t.is_cuda or (shape is not None and t.shape != shape):
        raise ValueError(f"{name}: a contiguous {dtype} GPU tensor{'' if shape is None else f' of shape {shape}'} is "
                         f"wanted, got {t.dtype} {tuple(t.shape)} on {t.device}, strides {t.stride()}")
    return t.data_ptr()


def _empty_on(stream, shape, dtype, device) -> torch.Tensor:
    """A new tensor whose memory is `stream`'s (a torch stream, a handle, or None for the current one)."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


class KVSeqs:
    """The sequences of a call (``mma_kv_seqs_t``) and the tensors that it points to. Built once per step, or
    kept while its tensors' addresses and the two bounds stay: what the tensors hold may change between calls. Tokens
    of a sequence past max_tokens (1 unless given to kv_seqs) are left out of a call, their rows of an attention's output
    unwritten; max_len also sets how attention cuts its work, so it is best near the longest sequence."""

    def __init__(self, block_table: torch.Tensor, lens: torch.Tensor, q_start: Optional[torch.Tensor] = None, *,
                 max_tokens: int, max_len: int):
        if block_table.dim() != 2:
            raise ValueError("block_table: [sequences][blocks] is wanted")
        n, width = block_table.shape
        self.tensors = block_table, lens, q_start
        self.num_seqs, self.max_tokens, self.max_len = n, max_tokens, max_len
        self.device = block_table.device
        self.c = mma_kv_seqs_t(_want("block_table", block_table, torch.int32), _want("lens", lens, torch.int32, (n,)),
                               0 if q_start is None else _want("q_start", q_start, torch.int32, (n + 1,)), n, width,
                               max_tokens, max_len)
        self.address = ctypes.addressof(self.c)


def kv_seqs(block_table, lens, q_start=None, *, max_tokens: int = 1, max_len: int) -> KVSeqs:
    return KVSeqs(block_table, lens, q_start, max_tokens=max_tokens, max_len=max_len)


def mma_rope_table(rows: int, rot_dim: int, base: float = 10000.0, kind: int = MMA_ROPE_NONE, factor: float = 1.0,
                   original_len: float = 0.0, low: float = 1.0, high: float = 32.0) -> np.ndarray:
    """float32 [rows][rot_dim]: cosines, then sines, of each position (host memory)."""
    out = np.empty((rows, rot_dim), np.float32)
    r = mma_rope_t(rot_dim, kind, base, factor, original_len, low, high)
    _check(lib.mma_rope_table(ctypes.byref(r), rows, out.ctypes.data), "mma_rope_table")
    return out


def mma_kv_append(layout: mma_kv_layout_t, layer, seqs: KVSeqs, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                  positions: Optional[torch.Tensor] = None, rope: Optional[torch.Tensor] = None, *,
                  q_out: Optional[torch.Tensor] = None, interleaved: bool = False,
                  q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                  k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None,
                  stream=None) -> torch.Tensor:
    """Normalise and rotate q and k, write k and v into `layer`; returns the queries (q_out, or a new tensor)."""
    if stream is not None and q_out is None:
        q_out = _empty_on(stream, q.shape, q.dtype, q.device)
    return _kv_ops.append(layout, layer, seqs.address, q, k, v, positions, rope, q_out, interleaved, q_weight, k_weight,
                          eps, k_scale, v_scale, _stream(stream))


def mma_kv_attention(layout: mma_kv_layout_t, layer, seqs: KVSeqs, q: torch.Tensor, *,
                     out: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                     tree: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                     scores_in: Optional[torch.Tensor] = None, scores_out: Optional[torch.Tensor] = None,
                     decay: float = 1.0, k_scale: Optional[torch.Tensor] = None,
                     v_scale: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                     softcap: float = 0.0, window: int = 0, slopes: Optional[torch.Tensor] = None,
                     prefix: Optional[torch.Tensor] = None, max_prefix: Optional[int] = None,
                     stream=None) -> torch.Tensor:
    """Attention of the call's tokens over their sequences' entries; returns `out` (or a new tensor). `tree`: int64
    [tokens][words] bits. `scale`: 1 / sqrt(head_dim) unless given. `workspace`: a uint8 tensor of
    kv_attention_workspace() bytes of the call's shape or more; a new one of the stream's unless given.

    Scores have the shape of ``mma_kv_shape_t``: capped (`softcap`), less `slopes` (float32 [heads]) times the distance, seen
    within `window` entries up to the token's own, and in both directions within `prefix` (int32 [sequences]) entries, of
    which no sequence has more than `max_prefix` (max_len unless given). Tokens of the prefix see ahead in it: for first entries
    that only stay in sight of a window, they go in a call without one."""
    if stream is not None:
        if out is None:
            out = _empty_on(stream, q.shape, q.dtype, q.device)
        if workspace is None:
            need = kv_attention_workspace(layout, seqs, q.shape[0], q.shape[1], q.dtype, scores_out is not None, window=window,
                                          prefix=prefix is not None, max_prefix=max_prefix, softcap=softcap,
                                          slopes=slopes is not None)
            workspace = _empty_on(stream, (need,), torch.uint8, q.device)
    return _kv_ops.attention(layout, layer, seqs.address, q, out, scale, tree, lse, scores_in, scores_out, decay, k_scale,
                             v_scale, workspace, _stream(stream), softcap, window, slopes, prefix, max_prefix)


def kv_attention_workspace(layout: mma_kv_layout_t, seqs: KVSeqs, num_tokens: int, q_heads: int, dtype: torch.dtype,
                           scores: bool = False, *, window: int = 0, prefix: bool = False,
                           max_prefix: Optional[int] = None, softcap: float = 0.0, slopes: bool = False) -> int:
    """Bytes of workspace of an attention call of these sizes and this shape (of `prefix` and `slopes`, whether the call has
    them): with a window a call needs fewer, with slopes or a cap it may need more."""
    kind = _TYPES.get(dtype)
    if kind is None:
        raise ValueError(f"queries of {dtype}: bfloat16 or float16 is wanted")
    a = mma_kv_attention_t(num_tokens=num_tokens, q_heads=q_heads, type=kind, scores_out=1 if scores else None,
                           cache_type=MMA_TYPE_F8 if layout.elem_bytes == 1 else kind)
    need = _U64()
    shape = mma_kv_shape_t(slopes=1 if slopes else None, prefix=1 if prefix else None,
                           max_prefix=seqs.max_len if max_prefix is None else max_prefix, window=window, softcap=softcap)
    _check(lib.mma_kv_attention_shaped_workspace(layout, seqs.c, a, shape, need), "mma_kv_attention_shaped_workspace")
    return need.value


def _moved_layer(t, layout: mma_kv_layout_t) -> None:
    """A layer whose entries are moved as they are: bytes (an integer type) or a type that caches hold, contiguous."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        return
    held = (torch.float8_e4m3fn,) if layout.elem_bytes == 1 else (torch.bfloat16, torch.float16)
    if not t.is_contiguous() or not (t.dtype in held or not (t.dtype.is_floating_point or t.dtype.is_complex)):
        raise ValueError(f"layer: a contiguous tensor of {held} or of bytes is wanted, got {t.dtype}, strides {t.stride()}")


def mma_kv_commit(layout: mma_kv_layout_t, layers, seqs: KVSeqs, accepted: torch.Tensor, counts: torch.Tensor, *,
                  scores=None, scores_stride: Optional[int] = None, stream=None) -> torch.Tensor:
    """Move the accepted drafted entries together in every layer (in place); returns the new lengths. `layers`,
    `scores`: tensors, or a layer_table (then scores_stride is needed)."""
    if not isinstance(layers, ctypes.Array):
        layers = list(layers)
        for t in layers:
            _moved_layer(t, layout)
    if scores is not None and not isinstance(scores, ctypes.Array):
        if not len(scores):
            raise ValueError("scores: a tensor of each layer is wanted")
        shape = tuple(scores[0].shape)
        if len(shape) != 3 or shape[:2] != (seqs.num_seqs, layout.kv_heads):
            raise ValueError(f"scores: [{seqs.num_seqs}][{layout.kv_heads}][entries] is wanted, got {shape}")
        for t in scores:
            _want("scores", t, torch.float32, shape)
        scores_stride = shape[2]
    if scores is not None:
        scores = layer_table(scores)
        if scores_stride is None:
            raise ValueError("a table of scores needs scores_stride")
    lens = None if stream is None else _empty_on(stream, (seqs.num_seqs,), torch.int32, seqs.device)
    return _kv_ops.commit(layout, layer_table(layers), seqs.address, accepted, counts, scores, scores_stride, lens,
                          _stream(stream))


def kv_evict_workspace(layout: mma_kv_layout_t, seqs: KVSeqs) -> int:
    """Bytes of workspace of an eviction call."""
    need = _U64()
    _check(lib.mma_kv_evict_workspace(layout, seqs.c, need), "mma_kv_evict_workspace")
    return need.value


def mma_kv_evict(layout: mma_kv_layout_t, layer, seqs: KVSeqs, dst_table: torch.Tensor, scores: torch.Tensor, keep: int,
                 *, sinks: int = 0, recent: int = 0, workspace: Optional[torch.Tensor] = None,
                 stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Keep the `keep` entries of each sequence and KV head that attention went to, moved into the blocks of
    dst_table; returns (entries kept, their scores, new lengths). `workspace`: a uint8 tensor of kv_evict_workspace()
    bytes or more; a new one of the stream's unless given."""
    _moved_layer(layer, layout)
    entries = kept = lens = None
    if stream is not None:
        shape = (seqs.num_seqs, layout.kv_heads, keep)
        entries, kept = (_empty_on(stream, shape, t, seqs.device) for t in (torch.int32, torch.float32))
        lens = _empty_on(stream, shape[:1], torch.int32, seqs.device)
        if workspace is None:
            workspace = _empty_on(stream, (kv_evict_workspace(layout, seqs),), torch.uint8, seqs.device)
    return _kv_ops.evict(layout, layer, seqs.address, dst_table, scores, keep, sinks, recent, entries, kept, lens,
                         workspace, _stream(stream))


def beam_select_workspace(batch: int, beams: int, vocab: int, keep: int, dtype: torch.dtype) -> int:
    """Bytes of workspace of a selection of these sizes."""
    kind = {**_TYPES, torch.float32: MMA_TYPE_F32}.get(dtype)
    if kind is None:
        raise ValueError(f"logits of {dtype}: bfloat16, float16 or float32 is wanted")
    need = _U64()
    a = mma_beam_select_t(batch=batch, beams=beams, vocab=vocab, keep=keep, type=kind)
    _check(lib.mma_beam_select_workspace(a, need), "mma_beam_select_workspace")
    return need.value


def mma_beam_select(logits: torch.Tensor, scores: torch.Tensor, keep: int, *, done: Optional[torch.Tensor] = None,
                    done_token: int = 0, out: Optional[Tuple[torch.Tensor, torch.Tensor, torch.Tensor]] = None,
                    workspace: Optional[torch.Tensor] = None,
                    stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """The `keep` best continuations of each request over its beams and the vocabulary: (tokens, parents, scores), each
    [requests][keep]. `logits`: [requests * beams][vocabulary] or [requests][beams][vocabulary]; `scores`: float32
    [requests][beams]; `done`: uint8 or bool of that shape, beams that have ended and stay as they are with `done_token`;
    `out`: the three results' tensors. Parents are rows of `logits`: what mma_kv_fork takes."""
    tokens, parents, best = (None, None, None) if out is None else out
    if stream is not None:
        shape = (scores.shape[0], keep)
        if out is None:
            tokens, parents, best = (_empty_on(stream, shape, t, scores.device) for t in (torch.int32, torch.int32, torch.float32))
        if workspace is None:
            need = beam_select_workspace(*scores.shape, logits.shape[-1], keep, logits.dtype)
            workspace = _empty_on(stream, (need,), torch.uint8, scores.device)
    return _kv_ops.beam_select(logits, scores, keep, done, done_token, tokens, parents, best, workspace, _stream(stream))


def _moved_layers(layers, layout: mma_kv_layout_t) -> ctypes.Array:
    if isinstance(layers, ctypes.Array):
        return layers
    layers = list(layers)
    for t in layers:
        _moved_layer(t, layout)
    return layer_table(layers)


def mma_kv_fork(layout: mma_kv_layout_t, layers, seqs: KVSeqs, parents: torch.Tensor, refs: torch.Tensor, *,
                grow: Optional[torch.Tensor] = None, width: Optional[int] = None,
                out: Optional[Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]] = None,
                workspace: Optional[torch.Tensor] = None,
                stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]:
    """Children that go on from `parents` (int32, sequences of the call; -1: none): whole blocks shared by count, the open one
    kept or copied in every layer, blocks for `grow` (int32) tokens more; sequences without children give theirs
    back. Returns (block table [children][width], lengths, counts of the blocks, [1]: blocks that are free). `refs`: int32
    [blocks], how often tables hold each. `out`: the four results' tensors, of which the counts may be `refs`."""
    table, lens, counts, left = (None,) * 4 if out is None else out
    if stream is not None:
        n = parents.shape[0]
        if out is None:
            wide = seqs.c.table_stride if width is None else width
            table, lens, counts, left = (_empty_on(stream, s, torch.int32, refs.device) for s in ((n, wide), (n,), refs.shape, (1,)))
        if workspace is None:
            workspace = _empty_on(stream, (12 * n,), torch.uint8, refs.device)
    return _kv_ops.fork(layout, _moved_layers(layers, layout), seqs.address, parents, refs, grow, width, table, lens, counts, left,
                        workspace, _stream(stream))


def mma_kv_compact(layout: mma_kv_layout_t, layers, table: torch.Tensor, refs: torch.Tensor, *,
                   out: Optional[Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]] = None,
                   workspace: Optional[torch.Tensor] = None,
                   stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]:
    """Held blocks (those that `refs` counts) moved to the lowest places of the pool, in every layer. Returns (the block
    table, the counts, where each block is now, [1]: how many are held). `out`: the four results' tensors, of which
    the first two may be `table` and `refs`."""
    new, counts, moved, held = (None,) * 4 if out is None else out
    if stream is not None:
        if out is None:
            new, counts, moved, held = (_empty_on(stream, s, torch.int32, refs.device)
                                        for s in (table.shape, refs.shape, refs.shape, (1,)))
        if workspace is None:
            need = _U64()
            _check(lib.mma_kv_compact_workspace(layout, need), "mma_kv_compact_workspace")
            workspace = _empty_on(stream, (need.value,), torch.uint8, refs.device)
    return _kv_ops.compact(layout, _moved_layers(layers, layout), table, refs, new, counts, moved, held, workspace,
                           _stream(stream))


def _load_kv_ops():
    """The operators' binding, a compiled module next to libmma.so, given the library's entry points."""
    path = os.path.join(_HERE, "_kv_ops.so")
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with `python paper_2512_16056_amd/build.py`")
    spec = importlib.util.spec_from_file_location("_kv_ops", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    names = ("kv_append", "kv_attention", "kv_attention_workspace", "kv_commit", "kv_evict", "kv_evict_workspace",
             "kv_attention_shaped", "kv_attention_shaped_workspace", "beam_select", "beam_select_workspace", "kv_fork",
             "kv_fork_workspace", "kv_compact", "kv_compact_workspace")
    m.attach(*(ctypes.cast(getattr(lib, "mma_" + x), _P).value for x in names), _check, _ptr)
    return m


_kv_ops = _load_kv_ops()


# ------------------------------------------------------------------ status
def mma_get_stats() -> dict:
    s = mma_stats_t()
    _check(lib.mma_get_stats(ctypes.byref(s)), "mma_get_stats")
    return s.as_dict()


def mma_reset_stats() -> None:
    _check(lib.mma_reset_stats(), "mma_reset_stats")


def mma_status_str(status: int) -> str:
    return lib.mma_status_str(status).decode()


def mma_last_error() -> str:
    return lib.mma_last_error().decode(errors="replace")


def mma_clear_error() -> None:
    _check(lib.mma_clear_error(), "mma_clear_error")


def mma_trace_enable(on: bool = True) -> None:
    _check(lib.mma_trace_enable(1 if on else 0), "mma_trace_enable")


def mma_trace_read(cap: int = 65536) -> List[dict]:
    buf = (mma_trace_rec_t * cap)()
    n = _U64()
    _check(lib.mma_trace_read(buf, cap, ctypes.byref(n)), "mma_trace_read")
    return [buf[i].as_dict() for i in range(n.value)]


def mma_test_set_fault(kind: int, value: int) -> None:
    _check(lib.mma_test_set_fault(kind, value), "mma_test_set_fault")


# ------------------------------------------------------------------ host-only
def _plan_call(fn, name, *args) -> List[Tuple[int, int, int, int]]:
    n = _U64()
    _check(fn(*args, None, 0, ctypes.byref(n)), name)
    out = (mma_plan_entry_t * max(n.value, 1))()
    _check(fn(*args, out, n.value, ctypes.byref(n)), name)
    return [(out[i].item, out[i].offset, out[i].bytes, out[i].flags) for i in range(n.value)]


def mma_plan_list(sizes: Iterable[int], chunk: int, fallback: int, small: int) -> List[Tuple[int, int, int, int]]:
    s = np.ascontiguousarray(np.asarray(list(sizes), dtype=np.uint64))
    return _plan_call(lib.mma_plan_list, "mma_plan_list", s.ctypes.data_as(ctypes.POINTER(_U64)), s.size,
                      chunk, fallback, small)


def mma_plan_kv(n_blocks: int, pieces_per_block: int, piece_bytes: int, chunk: int):
    return _plan_call(lib.mma_plan_kv, "mma_plan_kv", n_blocks, pieces_per_block, piece_bytes, chunk)


def mma_validate_kv_tables(src, src_count: int, dst, dst_count: int) -> bool:
    s, d = _i32(src), _i32(dst)
    if s.size != d.size:
        return False
    st = lib.mma_validate_kv_tables(s.ctypes.data_as(ctypes.POINTER(_I32)), src_count,
                                    d.ctypes.data_as(ctypes.POINTER(_I32)), dst_count, s.size)
    return st == MMA_OK


def mma_kv_layout_sizes(layout: mma_kv_layout_t) -> dict:
    """Bytes of one piece, one host slot, the host pool and one GPU layer tensor; MMAError if the
    layout is invalid or a size does not fit 64 bits."""
    out = [_U64() for _ in range(4)]
    _check(lib.mma_kv_layout_sizes(ctypes.byref(layout), *[ctypes.byref(v) for v in out]), "mma_kv_layout_sizes")
    return dict(zip(("piece", "slot", "pool", "layer"), (v.value for v in out)))

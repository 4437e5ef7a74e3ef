"""ctypes binding of libcompresskv (include/compresskv.h).

Argument marshalling only: every step of the compression path runs in the
library's CUDA kernels.  PyTorch supplies device memory and streams.  There
is no fallback: if the library is missing or fails to load, importing the
binding raises.
"""
from __future__ import annotations

import ctypes
import os
import struct
from ctypes import POINTER, c_float, c_int32, c_int64, c_size_t, c_void_p

import numpy as np
import torch

from . import _build

CKV_OK = 0
CKV_ERR_INVALID_ARG = -1
CKV_ERR_UNSUPPORTED = -2
CKV_ERR_BUDGET = -3
CKV_ERR_EMPTY_SRH_GROUP = -4
CKV_ERR_WORKSPACE = -5
CKV_ERR_CUDA = -6
CKV_ERR_DEVICE_TIMEOUT = -7
CKV_ERR_DEVICE_INDEX = -8
CKV_ERR_STATIC_SCRATCH = -9
STATIC_SCRATCH_BYTES = 16 * 1024 * 1024
CKV_DTYPE_F16 = 0
CKV_DTYPE_BF16 = 1
CKV_POOL_AVG = 0
CKV_POOL_MAX = 1
CKV_SELECT_PER_GROUP = 0
CKV_SELECT_PER_LAYER = 1
KERNEL_KINDS = {1: "score", 2: "combine", 3: "select", 4: "gather", 5: "fused", 6: "q4_write",
                7: "q4_attend", 8: "q4_evict", 9: "rope", 10: "paged_write", 11: "paged_gather",
                12: "paged_attend"}
ROPE_SCALINGS = {None: 0, "linear": 1, "base": 2, "waves": 3, "ramp": 4}
Q4_TILE = 32  # a 4-bit cache's capacity is a multiple of this

EXPORTED = (
    "compresskv_workspace_size",
    "compresskv_workspace_init",
    "compresskv_output_layout",
    "compresskv_score",
    "compresskv_select",
    "compresskv_gather",
    "compresskv_compress_layer",
    "compresskv_compress_layers",
    "compresskv_compress_layer_noalloc",
    "compresskv_compress_layer_lse",
    "compresskv_compress_layers_lse",
    "compresskv_compress_layer_head_budgets",
    "compresskv_read_device_status",
    "compresskv_debug_stall_next_fused_call",
    "compresskv_debug_stall_next_q4_attend",
    "compresskv_debug_stall_next_paged_attend",
    "compresskv_allocate_layer_budgets",
    "compresskv_status_string",
    "compresskv_q4_workspace_size",
    "compresskv_q4_workspace_init",
    "compresskv_q4_append",
    "compresskv_q4_gather",
    "compresskv_q4_attend",
    "compresskv_q4_evict",
    "compresskv_rope_frequencies",
    "compresskv_rope_init",
    "compresskv_rope_apply",
    "compresskv_paged_append",
    "compresskv_paged_gather",
    "compresskv_paged_workspace_size",
    "compresskv_paged_workspace_init",
    "compresskv_paged_attend",
)


class CkvTrace(ctypes.Structure):
    _fields_ = [("events", POINTER(c_void_p)), ("kinds", POINTER(c_int32)),
                ("capacity", c_int32), ("count", c_int32), ("launches", c_int64)]


class CkvProblem(ctypes.Structure):
    _fields_ = [("batch", c_int32), ("num_q_heads", c_int32), ("num_kv_heads", c_int32),
                ("head_dim", c_int32), ("window", c_int32), ("pool_width", c_int32),
                ("dtype", c_int32), ("pool_kind", c_int32), ("scale", c_float),
                ("selection", c_int32), ("cu_seqlens", POINTER(c_int32)),
                ("kv_token_stride", c_int64), ("kv_head_stride", c_int64),
                ("q_batch_stride", c_int64), ("q_head_stride", c_int64),
                ("q_win_stride", c_int64), ("trace", POINTER(CkvTrace))]


class CkvQ4Cache(ctypes.Structure):
    _fields_ = [("batch", c_int32), ("num_kv_heads", c_int32), ("head_dim", c_int32),
                ("capacity", c_int32), ("k_codes", c_void_p), ("v_codes", c_void_p),
                ("k_params", c_void_p), ("v_params", c_void_p), ("positions", c_void_p),
                ("weights", c_void_p), ("lengths", c_void_p), ("trace", POINTER(CkvTrace))]


class CkvQ4Rows(ctypes.Structure):
    _fields_ = [("dtype", c_int32), ("rows_per_seq", c_int32), ("cu_rows", c_void_p),
                ("token_stride", c_int64), ("head_stride", c_int64)]


class CkvQ4Queries(ctypes.Structure):
    _fields_ = [("num_q_heads", c_int32), ("num_queries", c_int32), ("dtype", c_int32),
                ("accumulate", c_int32), ("scale", c_float),
                ("q_batch_stride", c_int64), ("q_head_stride", c_int64),
                ("q_query_stride", c_int64), ("out_batch_stride", c_int64),
                ("out_head_stride", c_int64), ("out_query_stride", c_int64)]


class CkvRope(ctypes.Structure):
    _fields_ = [("rot_dim", c_int32), ("interleaved", c_int32), ("scale", c_float),
                ("reserved", c_int32), ("turns", ctypes.c_uint64 * 64)]


class CkvRopeRows(ctypes.Structure):
    _fields_ = [("rows", c_int32), ("num_q_heads", c_int32), ("num_k_heads", c_int32),
                ("dtype", c_int32), ("backward", c_int32), ("reserved", c_int32),
                ("q_token_stride", c_int64), ("q_head_stride", c_int64),
                ("k_token_stride", c_int64), ("k_head_stride", c_int64),
                ("q_out_token_stride", c_int64), ("q_out_head_stride", c_int64),
                ("k_out_token_stride", c_int64), ("k_out_head_stride", c_int64),
                ("trace", POINTER(CkvTrace))]


class CkvPagedCache(ctypes.Structure):
    _fields_ = [("batch", c_int32), ("num_kv_heads", c_int32), ("head_dim", c_int32),
                ("dtype", c_int32), ("page_size", c_int32), ("num_pages", c_int32),
                ("table_width", c_int32), ("reserved", c_int32), ("k_pages", c_void_p),
                ("v_pages", c_void_p), ("page_stride", c_int64), ("slot_stride", c_int64),
                ("head_stride", c_int64), ("table", c_void_p), ("table_stride", c_int64),
                ("lengths", c_void_p), ("trace", POINTER(CkvTrace))]


class CkvPagedRows(ctypes.Structure):
    _fields_ = [("rows_per_seq", c_int32), ("num_q_heads", c_int32), ("cu_rows", c_void_p),
                ("kv_token_stride", c_int64), ("kv_head_stride", c_int64),
                ("q_token_stride", c_int64), ("q_head_stride", c_int64),
                ("q_out_token_stride", c_int64), ("q_out_head_stride", c_int64)]


class CkvPagedQueries(ctypes.Structure):
    _fields_ = [("num_q_heads", c_int32), ("rows_per_seq", c_int32), ("cu_rows", c_void_p),
                ("causal", c_int32), ("scale", c_float), ("q_token_stride", c_int64),
                ("q_head_stride", c_int64), ("out_token_stride", c_int64),
                ("out_head_stride", c_int64)]


# What a call describes of its rows, packed as the structures above (native alignment;
# filling a ctypes structure takes twice as long).
_ROPE_ROWS = struct.Struct("6i8qP")
_PAGED_ROWS = struct.Struct("2iP6q")
_PAGED_QUERIES = struct.Struct("2iPif4q")
assert (_ROPE_ROWS.size, _PAGED_ROWS.size, _PAGED_QUERIES.size) == tuple(
    ctypes.sizeof(t) for t in (CkvRopeRows, CkvPagedRows, CkvPagedQueries))


class CompressKVError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {status_string(code)} ({code})")
        self.code = code


_LIB = None
_FAST = {}


def library_path() -> str:
    return _build.LIB_PATH


def load(build_if_missing: bool = True) -> ctypes.CDLL:
    """Load libcompresskv (building it first if it is absent or stale)."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = library_path()
    if build_if_missing and _build.needs_build():
        _build.build()
    if not os.path.exists(path):
        raise RuntimeError(f"libcompresskv not built ({path}); run __graft_entry__.build()")
    lib = ctypes.CDLL(path)
    vp, pp = c_void_p, POINTER(CkvProblem)
    i32p = POINTER(c_int32)
    sig = {
        "compresskv_workspace_size": (c_size_t, [pp]),
        "compresskv_workspace_init": (c_int32, [vp, c_size_t, vp]),
        "compresskv_output_layout": (c_int32, [pp, i32p, i32p, i32p]),
        "compresskv_score": (c_int32, [pp, vp, vp, vp, vp, vp, c_size_t, vp]),
        "compresskv_select": (c_int32, [pp, vp, i32p, vp, i32p, vp, vp, c_size_t, vp]),
        "compresskv_gather": (c_int32, [pp, vp, i32p, vp, vp, vp, vp, vp, vp]),
        "compresskv_compress_layer": (c_int32, [pp, vp, vp, vp, vp, i32p, vp, i32p, vp, vp,
                                                 vp, vp, vp, c_size_t, vp]),
        "compresskv_compress_layers": (c_int32, [pp, c_int32, vp, vp, vp, vp, i32p, vp, i32p, vp,
                                                  vp, vp, vp, vp, c_size_t, vp]),
        "compresskv_compress_layer_noalloc": (c_int32, [pp, vp, vp, vp, vp, i32p, vp, i32p, vp,
                                                         vp, vp, vp, vp, vp]),
        "compresskv_compress_layer_lse": (c_int32, [pp, vp, vp, vp, vp, c_int64, c_int64, vp, i32p,
                                                     vp, i32p, vp, vp, vp, vp, vp, c_size_t, vp]),
        "compresskv_compress_layers_lse": (c_int32, [pp, c_int32, vp, vp, vp, vp, c_int64,
                                                      c_int64, vp, i32p, vp, i32p, vp, vp, vp,
                                                      vp, vp, c_size_t, vp]),
        "compresskv_compress_layer_head_budgets": (c_int32, [pp, vp, vp, vp, vp, i32p, vp, i32p,
                                                              vp, vp, vp, vp, vp, c_size_t, vp]),
        "compresskv_read_device_status": (c_int32, [vp, vp, i32p]),
        "compresskv_debug_stall_next_fused_call": (c_int32, [ctypes.c_longlong]),
        "compresskv_debug_stall_next_q4_attend": (c_int32, [ctypes.c_longlong]),
        "compresskv_debug_stall_next_paged_attend": (c_int32, [ctypes.c_longlong]),
        "compresskv_allocate_layer_budgets": (c_int32, [POINTER(ctypes.c_double), c_int32,
                                                        c_int64, c_int32, c_int32, i32p]),
        "compresskv_status_string": (ctypes.c_char_p, [c_int32]),
        "compresskv_q4_workspace_size": (c_size_t, [vp, c_int32, c_int32]),
        "compresskv_q4_workspace_init": (c_int32, [vp, c_size_t, vp]),
        "compresskv_q4_append": (c_int32, [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]),
        "compresskv_q4_gather": (c_int32, [pp, vp, c_int32, vp, i32p, vp, vp, vp, vp, vp, vp, vp]),
        "compresskv_q4_attend": (c_int32, [vp, vp, vp, vp, vp, vp, vp, c_size_t, vp]),
        "compresskv_q4_evict": (c_int32, [vp, c_int32, vp, c_int32, c_int32, vp, c_size_t, vp]),
        "compresskv_rope_frequencies": (c_int32, [c_int32, ctypes.c_double, c_int32,
                                                  ctypes.c_double, ctypes.c_double,
                                                  ctypes.c_double, ctypes.c_double, vp]),
        "compresskv_rope_init": (c_int32, [vp, c_int32, c_int32, vp, ctypes.c_double]),
        "compresskv_rope_apply": (c_int32, [vp, vp, vp, vp, vp, vp, vp, vp]),
        "compresskv_paged_append": (c_int32, [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]),
        "compresskv_paged_gather": (c_int32, [vp, vp, c_int32, vp, vp, vp, vp, vp]),
        "compresskv_paged_workspace_size": (c_size_t, [vp, c_int32, c_int32]),
        "compresskv_paged_workspace_init": (c_int32, [vp, c_size_t, vp]),
        "compresskv_paged_attend": (c_int32, [vp, vp, vp, vp, vp, vp, vp, c_size_t, vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
        # the wrappers below pass plain addresses: a second prototype of the
        # same function that takes them as integers
        fast = lib[name]
        fast.restype = res
        fast.argtypes = [vp if a in (pp, i32p) else a for a in args]
        _FAST[name] = fast
    _LIB = lib
    return lib


def _fast(name: str):
    if _LIB is None:
        load()
    return _FAST[name]


def status_string(code: int) -> str:
    return load().compresskv_status_string(int(code)).decode()


def _check(code: int, what: str):
    if code != CKV_OK:
        raise CompressKVError(code, what)


def _ptr(t) -> c_void_p:
    if t is None:
        return c_void_p(None)
    return c_void_p(t.data_ptr())


def _stream(stream) -> c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    return c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def _raw_stream(stream) -> int:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _addr(t):
    return None if t is None else t.data_ptr()


def _data(a: np.ndarray) -> int:
    """Address of an array's first element (a.ctypes.data takes 1 us)."""
    try:
        return ctypes.addressof(ctypes.c_char.from_buffer(a))
    except (TypeError, ValueError):  # read-only or empty
        return a.ctypes.data


def _host_i32(arr) -> np.ndarray:
    """`arr` as contiguous int32 (kept alive by the caller over the C call)."""
    return np.ascontiguousarray(arr, dtype=np.int32)


def _i32(arr) -> tuple:
    a = np.ascontiguousarray(np.asarray(arr, dtype=np.int32))
    return a, a.ctypes.data_as(POINTER(c_int32))


class Problem:
    """One layer's problem description (wraps ``ckv_problem``).

    ``q_win`` is ``[B, H_q, W, d]`` and ``k`` is ``[T, H_kv, d]`` (any
    strides with ``d`` contiguous); only shapes, strides and dtype are read.
    """

    def __init__(self, q_win: torch.Tensor, k: torch.Tensor, cu_seqlens, window: int,
                 pool_width: int, scale: float = 0.0, trace: "Trace | None" = None,
                 selection: str = "group", pool: str = "avg"):
        """``selection``: "group" (each KV group keeps its own SRH heads'
        choice) or "layer" (one choice per sequence shared by every group);
        ``pool``: "avg" or "max" (each SRH head max-pooled, then summed)."""
        if k.dtype not in (torch.float16, torch.bfloat16) or q_win.dtype != k.dtype:
            raise CompressKVError(CKV_ERR_INVALID_ARG, "Q and K must share an f16/bf16 dtype")
        self._cu, cu_ptr = _i32(cu_seqlens)
        self.trace = trace
        s = CkvProblem()
        s.batch = len(self._cu) - 1
        s.num_q_heads = q_win.shape[1]
        s.num_kv_heads = k.shape[1]
        s.head_dim = k.shape[2]
        s.window = int(window)
        s.pool_width = int(pool_width)
        s.dtype = CKV_DTYPE_BF16 if k.dtype == torch.bfloat16 else CKV_DTYPE_F16
        if pool not in ("avg", "max"):
            raise CompressKVError(CKV_ERR_INVALID_ARG, "pool must be 'avg' or 'max'")
        s.pool_kind = CKV_POOL_MAX if pool == "max" else CKV_POOL_AVG
        s.scale = float(scale)
        if selection not in ("group", "layer"):
            raise CompressKVError(CKV_ERR_INVALID_ARG, "selection must be 'group' or 'layer'")
        s.selection = CKV_SELECT_PER_LAYER if selection == "layer" else CKV_SELECT_PER_GROUP
        s.cu_seqlens = cu_ptr
        s.kv_token_stride = k.stride(0)
        s.kv_head_stride = k.stride(1)
        s.q_batch_stride = q_win.stride(0)
        s.q_head_stride = q_win.stride(1)
        s.q_win_stride = q_win.stride(2)
        s.trace = ctypes.pointer(trace.struct) if trace is not None else None
        self.struct = s
        self.batch = s.batch
        self.num_kv_heads = s.num_kv_heads

    @property
    def ref(self):
        return ctypes.byref(self.struct)

    @property
    def addr(self) -> int:
        return ctypes.addressof(self.struct)


class Trace:
    """Launch trace: ``capacity`` launches bracketed by CUDA events."""

    def __init__(self, capacity: int):
        """``capacity`` = 0 only counts launches (no events are recorded)."""
        self.events = [torch.cuda.Event(enable_timing=True) for _ in range(2 * capacity)]
        for e in self.events:  # torch creates the CUDA event on its first record
            e.record()
        if capacity:
            torch.cuda.synchronize()
        self._ev = (c_void_p * max(1, 2 * capacity))(*[e.cuda_event for e in self.events])
        self._kinds = (c_int32 * max(1, capacity))()
        self.struct = CkvTrace(ctypes.cast(self._ev, POINTER(c_void_p)),
                               ctypes.cast(self._kinds, POINTER(c_int32)), capacity, 0, 0)

    def reset(self):
        self.struct.count = 0
        self.struct.launches = 0

    @property
    def launches(self) -> int:
        return int(self.struct.launches)

    def records(self):
        """[(kind name, elapsed ms)] for the recorded launches (call after a sync)."""
        out = []
        for i in range(self.struct.count):
            out.append((KERNEL_KINDS.get(self._kinds[i], "?"),
                        self.events[2 * i].elapsed_time(self.events[2 * i + 1])))
        return out


def workspace_size(problem: Problem) -> int:
    n = load().compresskv_workspace_size(problem.ref)
    if n == 0:
        raise CompressKVError(CKV_ERR_INVALID_ARG, "compresskv_workspace_size")
    return int(n)


def workspace(problem: Problem, device=None, stream=None) -> torch.Tensor:
    """A zero-status workspace tensor for ``problem`` (256-byte aligned)."""
    n = workspace_size(problem)
    ws = torch.empty(n, dtype=torch.uint8, device=device or "cuda")
    assert ws.data_ptr() % 256 == 0
    _check(load().compresskv_workspace_init(_ptr(ws), n, _stream(stream)), "workspace_init")
    return ws


def output_layout(problem: Problem, budgets):
    b, bp = _i32(budgets)
    cu_prefix = np.zeros(problem.batch + 1, np.int32)
    cu_out = np.zeros(problem.batch + 1, np.int32)
    _check(load().compresskv_output_layout(problem.ref, bp,
                                           cu_prefix.ctypes.data_as(POINTER(c_int32)),
                                           cu_out.ctypes.data_as(POINTER(c_int32))),
           "output_layout")
    return cu_prefix, cu_out


def _mask(srh_mask, problem: "Problem", n_masks: int = 1):
    """SRH masks as host bytes; the library reads n_masks * num_q_heads of them."""
    m = np.asarray(srh_mask)
    if m.dtype != np.uint8:
        m = m.astype(np.uint8)
    m = np.ascontiguousarray(m)
    if n_masks >= 1 and m.size != n_masks * problem.struct.num_q_heads:
        what = ("srh_mask must have num_q_heads entries" if n_masks == 1
                else "srh_masks must be [n_masks, num_q_heads]")
        raise CompressKVError(CKV_ERR_INVALID_ARG, what)
    return m


def _check_lse(problem: "Problem", lse_win, k, rows: int):
    """lse_win must be a float32 device tensor on K's device, [rows, H_q, W]
    with contiguous window rows: the scoring kernel reads every (sequence,
    SRH head, window row) element through the given strides."""
    W = int(problem.struct.window)
    shape = (int(rows), int(problem.struct.num_q_heads), W)
    if (not isinstance(lse_win, torch.Tensor) or lse_win.dtype != torch.float32
            or not lse_win.is_cuda or lse_win.device != k.device or tuple(lse_win.shape) != shape
            or lse_win.stride(2) != 1 or (shape[1] > 1 and lse_win.stride(1) < W)
            or (shape[0] > 1 and lse_win.stride(0) < 1)):
        raise CompressKVError(CKV_ERR_INVALID_ARG,
                              f"lse_win must be a float32 CUDA tensor on K's device of shape "
                              f"{shape} with contiguous window rows")


def score(problem: Problem, q_win, k, srh_mask, raw, ws, stream=None):
    m = _mask(srh_mask, problem)
    _check(_fast("compresskv_score")(problem.addr, _addr(q_win), _addr(k), _data(m),
                                     _addr(raw), _addr(ws), ws.numel(), _raw_stream(stream)),
           "compresskv_score")


def select(problem: Problem, raw, budgets, indices, ws, pooled=None, stream=None) -> np.ndarray:
    b = _host_i32(budgets)
    cu_out = np.zeros(problem.batch + 1, np.int32)
    _check(_fast("compresskv_select")(problem.addr, _addr(raw), _data(b), _addr(indices),
                                      _data(cu_out), _addr(pooled), _addr(ws), ws.numel(),
                                      _raw_stream(stream)), "compresskv_select")
    return cu_out


def gather(problem: Problem, indices, cu_out, k, v, k_out, v_out, ws=None, stream=None):
    c = _host_i32(cu_out)
    _check(_fast("compresskv_gather")(problem.addr, _addr(indices), _data(c), _addr(k),
                                      _addr(v), _addr(k_out), _addr(v_out), _addr(ws),
                                      _raw_stream(stream)), "compresskv_gather")


def compress_layer(problem: Problem, q_win, k, v, srh_mask, budgets, indices, k_out, v_out, ws,
                   raw=None, pooled=None, stream=None) -> np.ndarray:
    m = _mask(srh_mask, problem)
    b = _host_i32(budgets)
    cu_out = np.zeros(problem.batch + 1, np.int32)
    _check(_fast("compresskv_compress_layer")(
        problem.addr, _addr(q_win), _addr(k), _addr(v), _data(m), _data(b),
        _addr(indices), _data(cu_out), _addr(k_out), _addr(v_out), _addr(raw), _addr(pooled),
        _addr(ws), ws.numel(), _raw_stream(stream)), "compresskv_compress_layer")
    return cu_out


def compress_layers(problem: Problem, n_masks: int, q_win, k, v, srh_masks, budgets, indices,
                    k_out, v_out, ws, raw=None, pooled=None, stream=None) -> np.ndarray:
    """Several layers in one call: ``problem``'s batch packs ``n_masks`` blocks
    of sequences (block l = layer l: K ``[n_layers*T, H_kv, d]``, Q window
    ``[n_layers*B, H_q, W, d]``, cu_seqlens repeated per layer with offset
    l*T) and block l selects with ``srh_masks[l]`` (``[n_masks, H_q]``);
    budgets ``[n_layers*B]``; outputs as for compress_layer on that batch."""
    n_masks = int(n_masks)
    m = _mask(srh_masks, problem, n_masks)
    b = _host_i32(budgets)
    cu_out = np.zeros(problem.batch + 1, np.int32)
    _check(_fast("compresskv_compress_layers")(
        problem.addr, n_masks, _addr(q_win), _addr(k), _addr(v), _data(m), _data(b),
        _addr(indices), _data(cu_out), _addr(k_out), _addr(v_out), _addr(raw), _addr(pooled),
        _addr(ws), ws.numel(), _raw_stream(stream)), "compresskv_compress_layers")
    return cu_out


def compress_layer_noalloc(problem: Problem, q_win, k, v, srh_mask, budgets, indices, k_out,
                           v_out, raw=None, pooled=None, device_status=None,
                           stream=None) -> np.ndarray:
    """compress_layer without a workspace: the library's static scratch is
    used (for callers that cannot allocate device memory)."""
    m = _mask(srh_mask, problem)
    b = _host_i32(budgets)
    cu_out = np.zeros(problem.batch + 1, np.int32)
    _check(_fast("compresskv_compress_layer_noalloc")(
        problem.addr, _addr(q_win), _addr(k), _addr(v), _data(m), _data(b),
        _addr(indices), _data(cu_out), _addr(k_out), _addr(v_out), _addr(raw), _addr(pooled),
        _addr(device_status), _raw_stream(stream)), "compresskv_compress_layer_noalloc")
    return cu_out


def allocate_layer_budgets(layer_errors, total_budget: int, min_budget: int = 32,
                           max_budget: int = 0) -> np.ndarray:
    """Per-layer budgets from offline layer errors (Sec. 3.4); host only.
    `max_budget` <= 0 selects 3 * total_budget / n_layers."""
    err = np.ascontiguousarray(np.asarray(layer_errors, dtype=np.float64))
    out = np.zeros(err.size, dtype=np.int32)
    _check(load().compresskv_allocate_layer_budgets(
        err.ctypes.data_as(POINTER(ctypes.c_double)), int(err.size), int(total_budget),
        int(min_budget), int(max_budget), out.ctypes.data_as(POINTER(c_int32))),
        "compresskv_allocate_layer_budgets")
    return out


def compress_layer_lse(problem: Problem, q_win, k, v, lse_win, srh_mask, budgets, indices, k_out,
                       v_out, ws, raw=None, pooled=None, stream=None) -> np.ndarray:
    """compress_layer with the window queries' log-sum-exp given:
    ``lse_win`` is a float32 ``[B, H_q, W]`` tensor (window rows contiguous)."""
    _check_lse(problem, lse_win, k, problem.batch)
    m = _mask(srh_mask, problem)
    b = _host_i32(budgets)
    cu_out = np.zeros(problem.batch + 1, np.int32)
    _check(_fast("compresskv_compress_layer_lse")(
        problem.addr, _addr(q_win), _addr(k), _addr(v), _addr(lse_win), lse_win.stride(0),
        lse_win.stride(1), _data(m), _data(b), _addr(indices), _data(cu_out),
        _addr(k_out), _addr(v_out), _addr(raw), _addr(pooled), _addr(ws), ws.numel(),
        _raw_stream(stream)), "compresskv_compress_layer_lse")
    return cu_out


def compress_layers_lse(problem: Problem, n_masks: int, q_win, k, v, lse_win, srh_masks, budgets,
                        indices, k_out, v_out, ws, raw=None, pooled=None,
                        stream=None) -> np.ndarray:
    """compress_layers with the window queries' log-sum-exp given, packed like
    the batch: ``lse_win`` is float32 ``[n_layers*B, H_q, W]``."""
    _check_lse(problem, lse_win, k, problem.batch)
    n_masks = int(n_masks)
    m = _mask(srh_masks, problem, n_masks)
    b = _host_i32(budgets)
    cu_out = np.zeros(problem.batch + 1, np.int32)
    _check(_fast("compresskv_compress_layers_lse")(
        problem.addr, n_masks, _addr(q_win), _addr(k), _addr(v), _addr(lse_win),
        lse_win.stride(0), lse_win.stride(1), _data(m), _data(b), _addr(indices),
        _data(cu_out), _addr(k_out), _addr(v_out), _addr(raw), _addr(pooled), _addr(ws),
        ws.numel(), _raw_stream(stream)), "compresskv_compress_layers_lse")
    return cu_out


def head_budget_layout(problem: Problem, group_budgets) -> tuple[np.ndarray, int]:
    """Host-side output layout of compress_layer_head_budgets: cu_out
    ``[H_kv, B+1]`` (group-major packing) and the total number of rows."""
    b = np.asarray(group_budgets, dtype=np.int64).reshape(problem.batch, problem.num_kv_heads)
    lens = np.diff(np.asarray(problem._cu, dtype=np.int64))
    kept = np.minimum(b, lens[:, None])
    cu = np.zeros((problem.num_kv_heads, problem.batch + 1), dtype=np.int32)
    row = 0
    for g in range(problem.num_kv_heads):
        for s in range(problem.batch):
            cu[g, s] = row
            row += int(kept[s, g])
        cu[g, problem.batch] = row
    return cu, row


def compress_layer_head_budgets(problem: Problem, q_win, k, v, srh_mask, group_budgets, indices,
                                k_out, v_out, ws, raw=None, pooled=None,
                                stream=None) -> np.ndarray:
    """compress_layer with a budget per (sequence, KV group): ``group_budgets``
    is ``[B, H_kv]``; outputs are packed group-major (see head_budget_layout);
    returns cu_out ``[H_kv, B+1]``."""
    m = _mask(srh_mask, problem)
    b = _host_i32(group_budgets)
    cu_out = np.zeros((problem.num_kv_heads, problem.batch + 1), np.int32)
    _check(_fast("compresskv_compress_layer_head_budgets")(
        problem.addr, _addr(q_win), _addr(k), _addr(v), _data(m), _data(b),
        _addr(indices), _data(cu_out), _addr(k_out), _addr(v_out), _addr(raw), _addr(pooled),
        _addr(ws), ws.numel(), _raw_stream(stream)), "compresskv_compress_layer_head_budgets")
    return cu_out


def debug_stall_next_fused_call(wait_ns: int) -> None:
    """Test hook: the next persistent-kernel call stalls on purpose and stops
    with CKV_ERR_DEVICE_TIMEOUT after `wait_ns` (see the header)."""
    _check(load().compresskv_debug_stall_next_fused_call(ctypes.c_longlong(int(wait_ns))),
           "compresskv_debug_stall_next_fused_call")


def debug_stall_next_q4_attend(wait_ns: int) -> None:
    """Test hook: one warp of the next q4_attend stalls on purpose and stops its
    CTA after wait_ns (0 cancels)."""
    _check(load().compresskv_debug_stall_next_q4_attend(ctypes.c_longlong(int(wait_ns))),
           "compresskv_debug_stall_next_q4_attend")


def debug_stall_next_paged_attend(wait_ns: int) -> None:
    """Test hook: a CTA of the next paged_attend stalls on purpose and stops
    after wait_ns (0 cancels)."""
    _check(load().compresskv_debug_stall_next_paged_attend(ctypes.c_longlong(int(wait_ns))),
           "compresskv_debug_stall_next_paged_attend")


def read_device_status(ws, stream=None) -> int:
    out = c_int32(0)
    _check(load().compresskv_read_device_status(_ptr(ws), _stream(stream), ctypes.byref(out)),
           "read_device_status")
    return int(out.value)


class LayerOutputs:
    """Device buffers for one compressed layer, sized from the budgets."""

    def __init__(self, problem: Problem, budgets, head_dim: int, dtype, device, scores=True):
        cu_prefix, cu_out = output_layout(problem, budgets)
        H = problem.num_kv_heads
        self.cu_prefix, self.cu_out = cu_prefix, cu_out
        self.indices = torch.empty((H, int(cu_out[-1])), dtype=torch.int32, device=device)
        self.k_out = torch.empty((int(cu_out[-1]), H, head_dim), dtype=dtype, device=device)
        self.v_out = torch.empty_like(self.k_out)
        self.raw = torch.empty((H, int(cu_prefix[-1])), dtype=torch.float32, device=device) if scores else None
        self.pooled = torch.empty_like(self.raw) if scores else None


# ------------------------------------------------------------------ 4-bit cache
def _invalid(what: str):
    raise CompressKVError(CKV_ERR_INVALID_ARG, what)


def _q4_int(x, what: str) -> int:
    """A number that a call takes as int32 (ctypes would drop its upper bits)."""
    x = int(x)
    if not -2 ** 31 <= x < 2 ** 31:
        _invalid(f"{what} does not fit 32 bits")
    return x


def _q4_dtype(t: torch.Tensor) -> int:
    if t.dtype not in (torch.float16, torch.bfloat16):
        _invalid("rows and queries must be f16 or bf16")
    return CKV_DTYPE_BF16 if t.dtype == torch.bfloat16 else CKV_DTYPE_F16


class Q4Cache:
    """A 4-bit KV cache over the caller's tensors (wraps ``ckv_q4_cache``).

    ``k_codes`` / ``v_codes`` are uint8 ``[B, H_kv, capacity, 64]`` (byte b:
    channel 2b in the low half), ``k_params`` / ``v_params`` bfloat16
    ``[B, H_kv, capacity, 8]`` (four scales, four minima, each of 32 channels),
    ``positions`` int32 and ``weights`` float32 ``[B, H_kv, capacity]`` (the
    latter may be None), ``lengths`` int32 ``[B, H_kv]``; all contiguous, on one
    device, the capacity a multiple of 32.  The tensors stay the caller's and
    are kept alive by this object."""

    def __init__(self, k_codes, v_codes, k_params, v_params, positions, lengths, weights=None,
                 trace: "Trace | None" = None):
        if k_codes.dim() != 4:
            _invalid("k_codes must be [B, H_kv, capacity, 64]")
        lead = tuple(k_codes.shape[:3])
        want = [("k_codes", k_codes, torch.uint8, lead + (64,)),
                ("v_codes", v_codes, torch.uint8, lead + (64,)),
                ("k_params", k_params, torch.bfloat16, lead + (8,)),
                ("v_params", v_params, torch.bfloat16, lead + (8,)),
                ("positions", positions, torch.int32, lead),
                ("lengths", lengths, torch.int32, lead[:2])]
        if weights is not None:
            want.append(("weights", weights, torch.float32, lead))
        for name, t, dtype, shape in want:
            if (t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous()
                    or t.device != k_codes.device):
                _invalid(f"{name} must be a contiguous {dtype} tensor {shape} on k_codes' device")
            setattr(self, name, t)
        self.weights = weights
        self.trace = trace
        self.batch, self.num_kv_heads, self.capacity = lead
        self.device = k_codes.device
        self.index = k_codes.get_device()  # (-1: host memory)
        s = CkvQ4Cache(self.batch, self.num_kv_heads, 128, self.capacity, _addr(k_codes),
                       _addr(v_codes), _addr(k_params), _addr(v_params), _addr(positions),
                       _addr(weights), _addr(lengths),
                       ctypes.pointer(trace.struct) if trace is not None else None)
        self.struct = s
        self.addr = ctypes.addressof(s)

    def sequences(self, first: int, count: int) -> "Q4Cache":
        """Sequences ``first .. first + count - 1`` as a cache of their own (a
        layer of a cache that packs its layers); the memory is shared."""
        first, count = int(first), int(count)
        if first < 0 or count < 1 or first + count > self.batch:
            _invalid("sequences outside the cache")
        cut = slice(first, first + count)
        return Q4Cache(self.k_codes[cut], self.v_codes[cut], self.k_params[cut],
                       self.v_params[cut], self.positions[cut], self.lengths[cut],
                       None if self.weights is None else self.weights[cut], self.trace)


def q4_cache(batch: int, num_kv_heads: int, capacity: int, device=None, weights: bool = True,
             trace: "Trace | None" = None) -> Q4Cache:
    """An empty 4-bit cache; ``capacity`` is rounded up to a multiple of 32."""
    cap = -(-int(capacity) // Q4_TILE) * Q4_TILE
    lead = (int(batch), int(num_kv_heads), cap)
    device = device or "cuda"

    def empty(shape, dtype):
        return torch.empty(shape, dtype=dtype, device=device)

    return Q4Cache(empty(lead + (64,), torch.uint8), empty(lead + (64,), torch.uint8),
                   empty(lead + (8,), torch.bfloat16), empty(lead + (8,), torch.bfloat16),
                   empty(lead, torch.int32),
                   torch.zeros(lead[:2], dtype=torch.int32, device=device),
                   empty(lead, torch.float32) if weights else None, trace)


def _q4_call(name: str, cache, stream, *args):
    """Enqueues on `stream` (default: the current stream of the cache's device)."""
    if cache.index < 0:
        _invalid("the cache must be in device memory")
    _device_call(name, cache.index, stream, *args)


def _device_call(name: str, index: int, stream, *args):
    if index < 0:
        _invalid("tensors must be in device memory")
    fn = _FAST.get(name) or _fast(name)
    if stream is None:
        stream = torch._C._cuda_getCurrentRawStream(index)
    else:
        stream = _raw_stream(stream)
    if index == torch._C._cuda_getDevice():
        code = fn(*args, stream)
    else:
        with torch.cuda.device(index):
            code = fn(*args, stream)
    if code != CKV_OK:
        raise CompressKVError(code, name)


def _q4_on_device(cache: Q4Cache, what: str, *tensors):
    index = cache.index
    for t in tensors:
        if t is not None and t.get_device() != index:
            _invalid(f"{what} must be on the cache's device")


def _q4_rows(cache: Q4Cache, k, v):
    """(dtype, shape, strides) of the rows."""
    shape, strides = k.shape, k.stride()
    if len(shape) != 3 or shape[1] != cache.num_kv_heads or shape[2] != 128 or v.shape != shape:
        _invalid("k and v must be [rows, H_kv, 128]")
    if v.dtype != k.dtype or strides[2] != 1 or (
            v.stride() != strides  # (a dimension of one element has a stride that means nothing)
            and any(n > 1 and a != b for n, a, b in zip(shape, strides, v.stride()))):
        _invalid("k and v must share their dtype and strides, head_dim contiguous")
    if v.get_device() not in (cache.index, -1):  # (-1: page-locked host memory)
        _invalid("v must be on the cache's device")
    return _q4_dtype(k), shape, strides


def _q4_values(t, like, shape, what):
    if t is not None and (t.dtype != like.dtype or t.shape != shape or not t.is_contiguous()):
        _invalid(f"{what} must be contiguous {tuple(shape)} in the rows' dtype")


def _q4_i32(cache, t, shape, what):
    if t is not None and (t.dtype != torch.int32 or t.shape != shape or not t.is_contiguous()):
        _invalid(f"{what} must be a contiguous int32 tensor {tuple(shape)}")


def q4_workspace_size(cache: Q4Cache, num_q_heads: int = 0, num_queries: int = 0) -> int:
    n = _fast("compresskv_q4_workspace_size")(cache.addr, _q4_int(num_q_heads, "num_q_heads"),
                                              _q4_int(num_queries, "num_queries"))
    if n == 0:
        raise CompressKVError(CKV_ERR_INVALID_ARG, "compresskv_q4_workspace_size")
    return int(n)


def q4_workspace(cache: Q4Cache, num_q_heads: int = 0, num_queries: int = 0,
                 stream=None) -> torch.Tensor:
    """A zero-status workspace for q4_attend with these heads and query tokens
    (or fewer) and q4_evict; without them for q4_evict alone."""
    if cache.device.type != "cuda":
        _invalid("the cache must be in device memory")
    n = q4_workspace_size(cache, num_q_heads, num_queries)
    ws = torch.empty(n, dtype=torch.uint8, device=cache.device)
    assert ws.data_ptr() % 256 == 0
    with torch.cuda.device(cache.device):
        _check(_fast("compresskv_q4_workspace_init")(ws.data_ptr(), n, _raw_stream(stream)),
               "compresskv_q4_workspace_init")
    return ws


def q4_append(cache: Q4Cache, k, v, positions, cu_rows=None, start=None, k_values=None,
              v_values=None, device_status=None, stream=None) -> None:
    """Quantises rows of new tokens into the cache.  ``k`` / ``v`` are
    ``[rows, H_kv, 128]`` packed by sequence (``cu_rows``: host ``[B+1]``; None:
    the same number for each), ``positions`` int32 ``[rows]`` (negative: padding
    behind a sequence's rows), ``start`` int32 ``[B, H_kv]`` (default: the
    cache's lengths); ``k_values`` / ``v_values`` receive what the codes stand
    for."""
    dtype, shape, strides = _q4_rows(cache, k, v)
    rows = shape[0]
    _q4_i32(cache, positions, (rows,), "positions")
    _q4_i32(cache, start, (cache.batch, cache.num_kv_heads), "start")
    _q4_i32(cache, device_status, (1,), "device_status")
    _q4_values(k_values, k, shape, "k_values")
    _q4_values(v_values, k, shape, "v_values")
    r = CkvQ4Rows(dtype, 0, None, strides[0] if rows > 1 else cache.num_kv_heads * 128,
                  strides[1] if cache.num_kv_heads > 1 else 128)
    if cu_rows is None:
        if rows % cache.batch:
            _invalid("the rows do not divide by the sequences: give cu_rows")
        r.rows_per_seq = rows // cache.batch
    else:
        cu = _host_i32(cu_rows)
        if cu.shape != (cache.batch + 1,) or int(cu[-1]) != rows:
            _invalid("cu_rows must be [B+1] and end at the rows of k")
        r.cu_rows = _data(cu)
    _q4_on_device(cache, "k, positions, start, values and status", k, positions, start, k_values,
                  v_values, device_status)
    _q4_call("compresskv_q4_append", cache, stream, cache.addr, ctypes.addressof(r), _addr(k), _addr(v),
             _addr(positions), _addr(start), _addr(k_values), _addr(v_values),
             _addr(device_status))


def q4_gather(problem: Problem, cache: Q4Cache, indices, cu_out, k, v, raw=None, k_values=None,
              v_values=None, ws=None, stream=None) -> None:
    """Quantises the retained rows of a compression into the cache, from slot 0
    of each unit.  ``indices`` / ``cu_out`` as compress_layer(s) or select give
    them (``[H_kv, rows]``, ``[B+1]``), or as compress_layer_head_budgets does
    (``[rows]``, ``[H_kv, B+1]``); ``raw``: the raw scores become the rows' first
    weights; ``k_values`` / ``v_values`` as k_out / v_out of the compression."""
    dtype, shape, strides = _q4_rows(cache, k, v)
    s = problem.struct
    if (s.batch != cache.batch or s.num_kv_heads != cache.num_kv_heads or s.dtype != dtype
            or s.kv_token_stride != strides[0] or s.kv_head_stride != strides[1]
            or shape[0] < int(problem._cu[-1])):
        _invalid("k, v and the cache must be those of the problem")
    cu = _host_i32(cu_out)
    H, B = cache.num_kv_heads, cache.batch
    group_major = cu.ndim == 2
    if cu.shape != ((H, B + 1) if group_major else (B + 1,)):
        _invalid("cu_out must be [B+1], or [H_kv, B+1] for budgets per KV group")
    rows = int(cu.reshape(-1)[-1])
    _q4_i32(cache, indices, (rows,) if group_major else (H, rows), "indices")
    shape = (rows, 128) if group_major else (rows, H, 128)
    _q4_values(k_values, k, shape, "k_values")
    _q4_values(v_values, k, shape, "v_values")
    if raw is not None:
        n = int(np.maximum(np.diff(problem._cu) - s.window, 0).sum())
        if raw.dtype != torch.float32 or tuple(raw.shape) != (H, n) or not raw.is_contiguous():
            _invalid(f"raw must be a contiguous float32 tensor {(H, n)}")
    _q4_on_device(cache, "k, indices, raw, values and workspace", k, indices, raw, k_values,
                  v_values, ws)
    _q4_call("compresskv_q4_gather", cache, stream, problem.addr, cache.addr, int(group_major),
             _addr(indices), _data(cu), _addr(k), _addr(v), _addr(raw), _addr(k_values),
             _addr(v_values), _addr(ws))


def q4_attend(cache: Q4Cache, q, out, ws, q_positions=None, scale: float = 0.0, lse=None,
              accumulate: bool = False, stream=None) -> None:
    """Attention of ``q`` ``[B, H_q, n, 128]`` (n query tokens a sequence, any
    strides with head_dim contiguous) over the cache into ``out`` (same shape
    and dtype).  ``q_positions`` int32 ``[B, n]``: a slot is seen where its
    position is not above the query's (default: every slot in use is seen);
    ``lse`` float32 ``[B, H_q, n]``; ``accumulate`` adds each slot's attention to
    the cache's weights."""
    if q.dim() != 4 or q.shape[0] != cache.batch or q.shape[3] != 128 or out.shape != q.shape:
        _invalid("q and out must be [B, H_q, n, 128]")
    if out.dtype != q.dtype or q.stride(3) != 1 or out.stride(3) != 1:
        _invalid("q and out must share their dtype, head_dim contiguous")
    B, hq, n = q.shape[:3]
    _q4_i32(cache, q_positions, (B, n), "q_positions")
    if lse is not None and (lse.dtype != torch.float32 or tuple(lse.shape) != (B, hq, n)
                            or not lse.is_contiguous()):
        _invalid("lse must be a contiguous float32 [B, H_q, n]")
    qs, os_ = q.stride(), out.stride()
    # a dimension of one element has a stride that means nothing
    one = (B == 1, hq == 1, n == 1)
    a = CkvQ4Queries(hq, n, _q4_dtype(q), int(bool(accumulate)), float(scale),
                     *(128 if one[i] else qs[i] for i in range(3)),
                     *(128 if one[i] else os_[i] for i in range(3)))
    _q4_on_device(cache, "q, out, q_positions, lse and workspace", q, out, q_positions, lse, ws)
    _q4_call("compresskv_q4_attend", cache, stream, cache.addr, ctypes.addressof(a), _addr(q),
             _addr(q_positions), _addr(out), _addr(lse), _addr(ws), ws.numel())


def q4_evict(cache: Q4Cache, budget, ws, sinks: int = 0, recent: int = 0, stream=None) -> None:
    """Evicts, in place, every unit's slots beyond ``budget`` (an int, or an
    int32 device tensor ``[B, H_kv]``) with the least accumulated weight; slots
    at positions below ``sinks`` and the ``recent`` newest positions stay."""
    budgets = None
    if isinstance(budget, torch.Tensor):
        budgets, budget = budget, 0
        _q4_i32(cache, budgets, (cache.batch, cache.num_kv_heads), "budget")
    _q4_on_device(cache, "budget and workspace", budgets, ws)
    _q4_call("compresskv_q4_evict", cache, stream, cache.addr, _q4_int(budget, "budget"), _addr(budgets),
             _q4_int(sinks, "sinks"), _q4_int(recent, "recent"), _addr(ws), ws.numel())


# ------------------------------------------------------------ rotary positions
def rope_frequencies(rot_dim: int = 128, base: float = 10000.0, scaling: "str | None" = None,
                     factor: float = 1.0, original_length: float = 0.0, low: float = 1.0,
                     high: float = 4.0) -> np.ndarray:
    """Rotary frequencies (float64 ``[rot_dim / 2]``, radians a position), plain or
    scaled for contexts ``factor`` times as long: "linear" (positions
    interpolated), "base" (a larger base), "waves" / "ramp" (only the waves that
    make few turns over ``original_length``; see the header)."""
    if scaling not in ROPE_SCALINGS:
        _invalid(f"scaling must be one of {list(ROPE_SCALINGS)}")
    f = np.zeros(64, np.float64)
    rot_dim = _q4_int(rot_dim, "rot_dim")
    _check(_fast("compresskv_rope_frequencies")(rot_dim, float(base), ROPE_SCALINGS[scaling],
                                                float(factor), float(original_length), float(low),
                                                float(high), f.ctypes.data),
           "compresskv_rope_frequencies")
    return f[:rot_dim // 2]


class Rope:
    """A rotary table (wraps ``ckv_rope``): pairs (i, i + rot_dim / 2) of a head's
    first ``rot_dim`` channels, or (2i, 2i + 1) where ``interleaved``, turn by
    position times frequency and are multiplied by ``scale``.  ``frequencies``
    (float64 ``[rot_dim / 2]``) replaces those of rope_frequencies."""

    def __init__(self, rot_dim: int = 128, base: float = 10000.0, interleaved: bool = False,
                 scaling: "str | None" = None, factor: float = 1.0, original_length: float = 0.0,
                 low: float = 1.0, high: float = 4.0, scale: float = 1.0, frequencies=None):
        rot_dim = _q4_int(rot_dim, "rot_dim")
        if frequencies is None:
            f = rope_frequencies(rot_dim, base, scaling, factor, original_length, low, high)
        else:
            f = np.ascontiguousarray(frequencies, np.float64)
            if f.shape != (rot_dim // 2,):
                _invalid("frequencies must be [rot_dim / 2]")
        self.rot_dim, self.interleaved, self.frequencies = rot_dim, bool(interleaved), f.copy()
        self.struct = CkvRope()
        self.addr = ctypes.addressof(self.struct)
        _check(_fast("compresskv_rope_init")(self.addr, rot_dim, int(self.interleaved), f.ctypes.data,
                                             float(scale)), "compresskv_rope_init")


def _head_rows(t, rows, what, dtype):
    """(heads, token stride, head stride) of rows [rows, heads, 128]."""
    if t.dim() != 3:
        _invalid(f"{what} must be [rows, heads, 128]")
    n, heads, d = t.shape
    token, head, one = t.stride()
    if n != rows or d != 128 or one != 1 or t.dtype != dtype or rows >= 1 << 31:
        _invalid(f"{what} must be {dtype} [{rows}, heads, 128], head_dim contiguous")
    # a dimension of one element has a stride that means nothing
    return (heads, token if rows > 1 else (heads or 1) * 128, head if heads > 1 else 128)


def _rows_i32(t, rows, what):
    if t is not None and (t.dtype != torch.int32 or t.shape != (rows,) or not t.is_contiguous()):
        _invalid(f"{what} must be a contiguous int32 tensor {(rows,)}")


def rope_apply(rope: Rope, positions, q, k=None, q_out=None, k_out=None, backward: bool = False,
               trace: "Trace | None" = None, stream=None) -> None:
    """Rotates ``q`` ``[rows, H_q, 128]`` (and ``k`` ``[rows, H_k, 128]``) by
    ``positions`` (int32 ``[rows]``), in place or into ``q_out`` / ``k_out``;
    ``backward``: by minus the angles (the gradient)."""
    rows, dtype = q.shape[0], q.dtype
    if q_out is None:
        q_out = q
    index = q.get_device()
    hq, qt, qh = _head_rows(q, rows, "q", dtype)
    ho, qot, qoh = (hq, qt, qh) if q_out is q else _head_rows(q_out, rows, "q_out", dtype)
    if ho != hq:
        _invalid("q_out must have q's shape")
    hk, kt, kh, kot, koh = 0, 0, 0, 0, 0
    if k is not None:
        if k_out is None:
            k_out = k
        hk, kt, kh = _head_rows(k, rows, "k", dtype)
        ho, kot, koh = (hk, kt, kh) if k_out is k else _head_rows(k_out, rows, "k_out", dtype)
        if ho != hk:
            _invalid("k_out must have k's shape")
        if k.get_device() != index or k_out.get_device() != index:
            _invalid("q, k, positions and outputs must be on one device")
    elif k_out is not None:
        _invalid("k_out without k")
    _rows_i32(positions, rows, "positions")
    if q_out.get_device() != index or positions.get_device() != index:
        _invalid("q, k, positions and outputs must be on one device")
    x = _ROPE_ROWS.pack(rows, hq, hk, _q4_dtype(q), 1 if backward else 0, 0, qt, qh, kt, kh, qot, qoh, kot,
                        koh, 0 if trace is None else ctypes.addressof(trace.struct))
    _device_call("compresskv_rope_apply", index, stream, rope.addr, x, positions.data_ptr(),
                 q.data_ptr() if hq else None, k.data_ptr() if hk else None,
                 q_out.data_ptr() if hq else None, k_out.data_ptr() if hk else None)


# ----------------------------------------------------------------- paged cache
class PagedCache:
    """A paged 16-bit KV cache over the caller's tensors (wraps
    ``ckv_paged_cache``).

    ``k_pages`` / ``v_pages`` are f16 or bf16 ``[pages, page_size, H_kv, 128]``
    (any strides, 128 contiguous: a pool kept as ``[pages, H_kv, page_size, 128]``
    is passed as its transpose(1, 2)), ``table`` int32 ``[B, width]`` (the pages
    of each sequence in order), ``lengths`` int32 ``[B]`` (slots in use; negative:
    the sequence is not there); all on one device.  The tensors stay the caller's
    and are kept alive by this object."""

    def __init__(self, k_pages, v_pages, table, lengths, trace: "Trace | None" = None):
        if k_pages.dim() != 4 or k_pages.shape[3] != 128 or k_pages.stride(3) != 1:
            _invalid("k_pages must be [pages, page_size, H_kv, 128], head_dim contiguous")
        dtype = _q4_dtype(k_pages)
        shape, strides = k_pages.shape, k_pages.stride()
        if v_pages.dtype != k_pages.dtype or v_pages.shape != shape or any(
                n > 1 and a != b for n, a, b in zip(shape, strides, v_pages.stride())):
            _invalid("v_pages must share k_pages' dtype, shape and strides")
        if table.dtype != torch.int32 or table.dim() != 2 or (table.shape[1] > 1 and table.stride(1) != 1):
            _invalid("table must be int32 [B, width], its rows contiguous")
        if lengths.dtype != torch.int32 or lengths.shape != table.shape[:1] or not lengths.is_contiguous():
            _invalid("lengths must be a contiguous int32 [B]")
        if any(t.device != k_pages.device for t in (v_pages, table, lengths)):
            _invalid("pages, table and lengths must be on one device")
        self.k_pages, self.v_pages, self.table, self.lengths = k_pages, v_pages, table, lengths
        self.trace, self.dtype = trace, k_pages.dtype
        self.num_pages, self.page_size, self.num_kv_heads = shape[:3]
        self.batch, self.table_width = table.shape
        self.capacity = self.table_width * self.page_size
        self.device = k_pages.device
        self.index = k_pages.get_device()
        # a dimension of one element has a stride that means nothing
        head = strides[2] if shape[2] > 1 else 128
        slot = strides[1] if shape[1] > 1 else 128
        page = strides[0] if shape[0] > 1 else max(head * shape[2], slot * shape[1])
        self.struct = CkvPagedCache(self.batch, self.num_kv_heads, 128, dtype, self.page_size,
                                    self.num_pages, self.table_width, 0, _addr(k_pages),
                                    _addr(v_pages), page, slot, head, _addr(table),
                                    table.stride(0) if self.batch > 1 else self.table_width,
                                    _addr(lengths),
                                    ctypes.pointer(trace.struct) if trace is not None else None)
        self.addr = ctypes.addressof(self.struct)

    def sequences(self, first: int, count: int) -> "PagedCache":
        """Sequences ``first .. first + count - 1`` as a cache of their own over
        the same pool."""
        first, count = int(first), int(count)
        if first < 0 or count < 1 or first + count > self.batch:
            _invalid("sequences outside the cache")
        cut = slice(first, first + count)
        return PagedCache(self.k_pages, self.v_pages, self.table[cut], self.lengths[cut], self.trace)


def paged_cache(batch: int, num_kv_heads: int, capacity: int, page_size: int = 64,
                dtype=torch.bfloat16, device=None, trace: "Trace | None" = None) -> PagedCache:
    """An empty paged cache with a pool of its own, in which every sequence has
    pages for ``capacity`` slots."""
    batch, heads, page = int(batch), int(num_kv_heads), int(page_size)
    width = -(-int(capacity) // page)
    device = device or "cuda"
    pools = [torch.empty((batch * width, heads, page, 128), dtype=dtype, device=device).transpose(1, 2)
             for _ in range(2)]
    table = torch.arange(batch * width, dtype=torch.int32, device=device).view(batch, width)
    return PagedCache(*pools, table, torch.zeros(batch, dtype=torch.int32, device=device), trace)


def _paged_rows(cache: PagedCache, rows: int, cu_rows):
    """(rows a sequence, cu_rows to keep alive, its address)."""
    if cu_rows is None:
        if rows % cache.batch:
            _invalid("the rows do not divide by the sequences: give cu_rows")
        return rows // cache.batch, None, None
    cu = _host_i32(cu_rows)
    if cu.shape != (cache.batch + 1,) or int(cu[-1]) != rows:
        _invalid("cu_rows must be [B+1] and end at the rows")
    return 0, cu, _data(cu)


def paged_append(cache: PagedCache, k, v, cu_rows=None, start=None, rope: "Rope | None" = None,
                 positions=None, q=None, q_out=None, device_status=None, stream=None) -> None:
    """Writes rows of new tokens, ``k`` / ``v`` ``[rows, H_kv, 128]`` packed by
    sequence (``cu_rows``: host ``[B+1]``; None: the same number for each), to
    the slots from ``start`` (int32 ``[B]``; default: the lengths) on, and sets
    the lengths.  With a ``rope`` K is rotated on the way, and ``q`` ``[rows, H_q,
    128]`` into ``q_out`` (default: in place), by ``positions`` (int32 ``[rows]``;
    default: the slots)."""
    rows = k.shape[0]
    heads, kt, kh = _head_rows(k, rows, "k", cache.dtype)
    if heads != cache.num_kv_heads or _head_rows(v, rows, "v", cache.dtype) != (heads, kt, kh):
        _invalid("k and v must be [rows, H_kv, 128] of the same strides")
    hq, qt, qh, qot, qoh = 0, 0, 0, 0, 0
    if q is not None:
        if rope is None:
            _invalid("q needs a rope")
        hq, qt, qh = _head_rows(q, rows, "q", cache.dtype)
        if q_out is None:
            q_out = q
        ho, qot, qoh = (hq, qt, qh) if q_out is q else _head_rows(q_out, rows, "q_out", cache.dtype)
        if ho != hq:
            _invalid("q_out must have q's shape")
    elif q_out is not None:
        _invalid("q_out without q")
    _rows_i32(start, cache.batch, "start")
    _rows_i32(positions, rows, "positions")
    _rows_i32(device_status, 1, "device_status")
    _q4_on_device(cache, "rows, start, positions and status", k, v, start, positions, q, q_out,
                  device_status)
    each, cu, at = _paged_rows(cache, rows, cu_rows)
    r = _PAGED_ROWS.pack(each, hq, at or 0, kt, kh, qt, qh, qot, qoh)
    _q4_call("compresskv_paged_append", cache, stream, cache.addr, r, _addr(k),
             _addr(v), _addr(start), None if rope is None else rope.addr, _addr(positions),
             _addr(q) if hq else None, _addr(q_out) if hq else None, _addr(device_status))


def paged_gather(cache: PagedCache, k_out, v_out=None, cu_rows=None, start=None, device_status=None,
                 stream=None) -> None:
    """Reads rows back: sequence s's slots from ``start`` (int32 ``[B]``; default
    0) on, into ``k_out`` / ``v_out`` ``[rows, H_kv, 128]`` (contiguous; either
    may be None), packed by sequence as ``cu_rows`` says (host ``[B+1]``; None:
    the same number for each)."""
    like = k_out if k_out is not None else v_out
    if like is None:
        _invalid("k_out or v_out is needed")
    rows = like.shape[0]
    for t in (k_out, v_out):
        if t is not None and (t.dtype != cache.dtype or t.shape != (rows, cache.num_kv_heads, 128)
                              or not t.is_contiguous()):
            _invalid("k_out and v_out must be contiguous [rows, H_kv, 128] in the cache's dtype")
    _rows_i32(start, cache.batch, "start")
    _rows_i32(device_status, 1, "device_status")
    _q4_on_device(cache, "outputs, start and status", k_out, v_out, start, device_status)
    each, cu, at = _paged_rows(cache, rows, cu_rows)
    _q4_call("compresskv_paged_gather", cache, stream, cache.addr, at, each, _addr(start), _addr(k_out),
             _addr(v_out), _addr(device_status))


def paged_workspace_size(cache: PagedCache, num_q_heads: int, num_queries: int) -> int:
    n = _fast("compresskv_paged_workspace_size")(cache.addr, _q4_int(num_q_heads, "num_q_heads"),
                                                 _q4_int(num_queries, "num_queries"))
    if n == 0:
        raise CompressKVError(CKV_ERR_INVALID_ARG, "compresskv_paged_workspace_size")
    return int(n)


def paged_workspace(cache: PagedCache, num_q_heads: int, num_queries: int, stream=None) -> torch.Tensor:
    """A zero-status workspace for paged_attend with these heads and at most
    ``num_queries`` query tokens of a sequence."""
    if cache.device.type != "cuda":
        _invalid("the cache must be in device memory")
    n = paged_workspace_size(cache, num_q_heads, num_queries)
    ws = torch.empty(n, dtype=torch.uint8, device=cache.device)
    assert ws.data_ptr() % 256 == 0
    with torch.cuda.device(cache.device):
        _check(_fast("compresskv_paged_workspace_init")(ws.data_ptr(), n, _raw_stream(stream)),
               "compresskv_paged_workspace_init")
    return ws


def paged_attend(cache: PagedCache, q, out, ws, cu_rows=None, start=None, scale: float = 0.0, lse=None,
                 causal: bool = True, stream=None) -> None:
    """Attention of ``q`` ``[rows, H_q, 128]``, packed by sequence (``cu_rows``:
    host ``[B+1]``; None: the same number for each), over the cache into ``out``
    (same shape and dtype).  Token i of a sequence stands at slot ``start`` + i
    (int32 ``[B]``; default: the sequence's newest slots) and sees the slots up
    to its own, or all in use where not ``causal``.  ``lse`` float32 ``[H_q,
    rows]``."""
    rows = q.shape[0]
    hq, qt, qh = _head_rows(q, rows, "q", cache.dtype)
    ho, ot, oh = _head_rows(out, rows, "out", cache.dtype)
    if ho != hq:
        _invalid("out must have q's shape")
    if lse is not None and (lse.dtype != torch.float32 or lse.shape != (hq, rows)
                            or not lse.is_contiguous()):
        _invalid("lse must be a contiguous float32 [H_q, rows]")
    _rows_i32(start, cache.batch, "start")
    _q4_on_device(cache, "q, out, start, lse and workspace", q, out, start, lse, ws)
    if not -3e38 < scale < 3e38:
        _invalid("scale must be a finite number")
    each, cu, at = _paged_rows(cache, rows, cu_rows)
    a = _PAGED_QUERIES.pack(hq, each, at or 0, 1 if causal else 0, scale, qt, qh, ot, oh)
    _q4_call("compresskv_paged_attend", cache, stream, cache.addr, a, _addr(q),
             _addr(start), _addr(out), _addr(lse), _addr(ws), ws.numel())

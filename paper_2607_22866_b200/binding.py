"""ctypes binding of libgmagnus.so.  Names mirror the C ABI (gm_spgemm_plan -> spgemm_plan ...).

Argument marshalling only: device arrays are torch tensors, their data_ptr() values go straight
into the gm_csr structs, and the library's device allocations are served by torch's caching
allocator through the gm_set_allocator hook, so results come back as torch tensors without a copy.
There is no fallback: if the library cannot be loaded, importing this module fails.
"""
from __future__ import annotations

import ctypes
import os
import struct
import threading
from dataclasses import dataclass

import numpy as np
import torch

from . import build as _build

GM_MAX_LEVELS = 8
EXPORTED_SYMBOLS = [
    "gm_set_allocator", "gm_planner_params", "gm_planner_batches", "gm_spgemm_plan", "gm_spgemm_plan_ex", "gm_spgemm_execute",
    "gm_spgemm_host", "gm_plan_get_info", "gm_exec_get_stats", "gm_plan_set_timing",
    "gm_plan_get_row_products", "gm_row_products_noalloc", "gm_route_plan", "gm_route_status",
    "gm_route_destroy", "gm_route_product", "gm_route_product_dx", "gm_route_product_dw", "gm_route_sum",
    "gm_route_sum_grads", "gm_block_quantize", "gm_route_product_scaled", "gm_csr_free", "gm_plan_destroy", "gm_status_string", "gm_last_error",
]


class GmError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str):
        super().__init__(f"{where} failed: {status_string(status)} ({status}): {detail}")
        self.status = status


class _CSR(ctypes.Structure):
    _fields_ = [("n_rows", ctypes.c_int64), ("n_cols", ctypes.c_int64), ("nnz", ctypes.c_int64),
                ("row_ptr", ctypes.c_void_p), ("col_idx", ctypes.c_void_p), ("vals", ctypes.c_void_p),
                ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class PlanOpts(ctypes.Structure):
    """gm_plan_opts: zero means "derive it"."""
    _fields_ = [("tau", ctypes.c_int64), ("chunk_width", ctypes.c_int32), ("max_fanout", ctypes.c_int32),
                ("acc_ctas_per_sm", ctypes.c_int32), ("stage_elems", ctypes.c_int64),
                ("c_capacity", ctypes.c_int64), ("separate_histogram", ctypes.c_int32),
                ("validate_inputs", ctypes.c_int32), ("single_stream", ctypes.c_int32),
                ("level0_multisplit", ctypes.c_int32), ("small_chunk_max", ctypes.c_int32),
                ("mid_chunk_max", ctypes.c_int32), ("expand_staging", ctypes.c_int32),
                ("debug_spin_limit", ctypes.c_int32), ("expand_order", ctypes.c_int32), ("early_exit", ctypes.c_int32)]


class Params(ctypes.Structure):
    _fields_ = [("tau", ctypes.c_int64), ("light_slots", ctypes.c_int32), ("chunk_width", ctypes.c_int32),
                ("chunks_required", ctypes.c_int32), ("max_fanout", ctypes.c_int32), ("n_levels", ctypes.c_int32),
                ("fanout", ctypes.c_int32 * GM_MAX_LEVELS), ("shift", ctypes.c_int32 * GM_MAX_LEVELS),
                ("acc_ctas_per_sm", ctypes.c_int32), ("acc_block_threads", ctypes.c_int32)]

    def levels(self):
        return [int(self.fanout[i]) for i in range(self.n_levels)]


class PlanInfo(ctypes.Structure):
    _fields_ = [("params", Params), ("n_rows", ctypes.c_int64), ("n_cols_c", ctypes.c_int64),
                ("products_total", ctypes.c_int64), ("products_heavy", ctypes.c_int64),
                ("products_max_row", ctypes.c_int64), ("rows_heavy", ctypes.c_int64),
                ("rows_light", ctypes.c_int64), ("rows_empty", ctypes.c_int64), ("nnz_a_heavy", ctypes.c_int64),
                ("c_nnz_upper", ctypes.c_int64), ("n_batches", ctypes.c_int64), ("stage_elems", ctypes.c_int64),
                ("workspace_bytes", ctypes.c_int64), ("light_bin_rows", ctypes.c_int64 * 8),
                ("launches", ctypes.c_int64), ("level0_direct", ctypes.c_int64), ("heavy_tasks", ctypes.c_int64),
                ("task_ctas_per_sm", ctypes.c_int64)]


class ExecStats(ctypes.Structure):
    _fields_ = [("c_nnz", ctypes.c_int64), ("c_nnz_heavy", ctypes.c_int64), ("c_capacity", ctypes.c_int64), ("staged_products", ctypes.c_int64),
                ("final_chunks", ctypes.c_int64), ("launches", ctypes.c_int64),
                ("small_chunk_products", ctypes.c_int64), ("small_chunk_entries", ctypes.c_int64),
                ("ms_light_symbolic", ctypes.c_float), ("ms_light_numeric", ctypes.c_float),
                ("ms_expand", ctypes.c_float), ("ms_histogram", ctypes.c_float), ("ms_multisplit", ctypes.c_float),
                ("ms_accumulate", ctypes.c_float), ("ms_gather", ctypes.c_float), ("ms_scan", ctypes.c_float),
                ("ms_total", ctypes.c_float), ("ms_small_chunks", ctypes.c_float), ("ms_mid_chunks", ctypes.c_float),
                ("panel_rows", ctypes.c_float), ("reserved", ctypes.c_float * 2), ("mid_chunk_products", ctypes.c_int64), ("mid_chunk_entries", ctypes.c_int64),
                ("early_exit_products", ctypes.c_int64), ("early_exit_chunks", ctypes.c_int64),
                ("split_products", ctypes.c_int64)]


_ALLOC_FN = ctypes.CFUNCTYPE(ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_void_p)
_FREE_FN = ctypes.CFUNCTYPE(None, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p)

_lib = None
_lock = threading.Lock()
_live: dict[int, torch.Tensor] = {}   # device blocks handed to the library, by address
_alloc_cb = None
_free_cb = None


def _torch_alloc(nbytes, stream, user):
    try:
        t = torch.empty(max(int(nbytes), 16), dtype=torch.uint8, device="cuda")
    except Exception:  # out of memory: the library turns NULL into GM_ERR_OOM
        return None
    _live[t.data_ptr()] = t
    return t.data_ptr()


def _torch_free(ptr, stream, user):
    _live.pop(ptr, None)


def load_library(install_torch_allocator: bool = True):
    """Loads (building it first if needed) libgmagnus.so and declares the C signatures."""
    global _lib, _alloc_cb, _free_cb
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is not None:
            return _lib
        path = _build.build()
        lib = ctypes.CDLL(path)
        vp, i64, i32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t
        P = ctypes.POINTER
        lib.gm_set_allocator.argtypes = [_ALLOC_FN, _FREE_FN, vp]
        lib.gm_planner_params.argtypes = [i64, i32, sz, P(PlanOpts), P(Params)]
        lib.gm_planner_batches.argtypes = [vp, i64, i64, vp, i64]
        lib.gm_planner_batches.restype = i64
        lib.gm_spgemm_plan.argtypes = [P(_CSR), P(_CSR), sz, P(vp)]
        lib.gm_spgemm_plan_ex.argtypes = [P(_CSR), P(_CSR), sz, P(PlanOpts), vp, P(vp)]
        lib.gm_spgemm_execute.argtypes = [vp, vp, P(_CSR)]
        lib.gm_spgemm_host.argtypes = [P(_CSR), P(_CSR), sz, P(PlanOpts), P(_CSR), i64]
        lib.gm_plan_get_info.argtypes = [vp, P(PlanInfo)]
        lib.gm_exec_get_stats.argtypes = [vp, P(ExecStats)]
        lib.gm_plan_set_timing.argtypes = [vp, ctypes.c_int]
        lib.gm_plan_get_row_products.argtypes = [vp, vp, vp]
        lib.gm_row_products_noalloc.argtypes = [P(_CSR), P(_CSR), vp, vp]
        D = vp  # a packed gm_dense
        lib.gm_route_plan.argtypes = [P(_CSR), vp, vp, vp, vp, vp, P(vp)]
        lib.gm_route_status.argtypes = [vp]
        lib.gm_route_destroy.argtypes = [vp]
        lib.gm_route_destroy.restype = None
        lib.gm_route_product.argtypes = [vp, D, ctypes.c_int, D, D, vp]
        lib.gm_route_product_dx.argtypes = [vp, D, D, ctypes.c_int, D, vp, vp]
        lib.gm_route_product_dw.argtypes = [vp, D, D, ctypes.c_int, D, vp]
        lib.gm_route_sum.argtypes = [vp, D, ctypes.c_int, D, vp]
        lib.gm_route_sum_grads.argtypes = [vp, D, D, D, vp, vp]
        lib.gm_block_quantize.argtypes = [D, ctypes.c_int, D, D, vp]
        lib.gm_route_product_scaled.argtypes = [vp, D, D, ctypes.c_int, D, D, D, vp]
        lib.gm_csr_free.argtypes = [P(_CSR)]
        lib.gm_csr_free.restype = None
        lib.gm_plan_destroy.argtypes = [vp]
        lib.gm_plan_destroy.restype = None
        lib.gm_status_string.argtypes = [ctypes.c_int]
        lib.gm_status_string.restype = ctypes.c_char_p
        lib.gm_last_error.argtypes = []
        lib.gm_last_error.restype = ctypes.c_char_p
        if install_torch_allocator and torch.cuda.is_available():
            _alloc_cb, _free_cb = _ALLOC_FN(_torch_alloc), _FREE_FN(_torch_free)
            lib.gm_set_allocator(_alloc_cb, _free_cb, None)
        _lib = lib
        return lib


def status_string(status: int) -> str:
    return load_library().gm_status_string(status).decode()


def _check(status: int, where: str):
    if status != 0:
        raise GmError(status, where, load_library().gm_last_error().decode())


@dataclass
class DeviceCSR:
    """CSR matrix in device memory: int64 row_ptr, int32 col, float32/float64 val (torch tensors)."""
    n_rows: int
    n_cols: int
    row_ptr: torch.Tensor
    col: torch.Tensor
    val: torch.Tensor
    nnz: int | None = None

    def __post_init__(self):
        if self.nnz is None:
            self.nnz = int(self.col.numel())

    @staticmethod
    def from_host(M, device="cuda") -> "DeviceCSR":
        """M: any object with n_rows, n_cols, row_ptr, col, val numpy arrays."""
        return DeviceCSR(M.n_rows, M.n_cols, torch.from_numpy(M.row_ptr).to(device),
                         torch.from_numpy(M.col).to(device), torch.from_numpy(M.val).to(device), int(M.row_ptr[-1]))

    def _struct(self) -> _CSR:
        assert self.row_ptr.dtype == torch.int64 and self.col.dtype == torch.int32
        assert self.val.dtype in (torch.float32, torch.float64)
        assert self.row_ptr.is_contiguous() and self.col.is_contiguous() and self.val.is_contiguous()
        return _CSR(self.n_rows, self.n_cols, self.nnz, self.row_ptr.data_ptr(), self.col.data_ptr(),
                    self.val.data_ptr(), 0 if self.val.dtype == torch.float32 else 1, 0)


def planner_params(c_cols: int, dtype, smem_bytes: int, opts: PlanOpts | None = None) -> Params:
    """gm_planner_params: host-only parameter selection (Section III-D)."""
    out = Params()
    code = 0 if np.dtype(dtype) == np.float32 else 1
    _check(load_library().gm_planner_params(c_cols, code, smem_bytes, ctypes.byref(opts) if opts else None,
                                            ctypes.byref(out)), "gm_planner_params")
    return out


def planner_batches(heavy_prefix: np.ndarray, stage_elems: int) -> list[int]:
    """gm_planner_batches: boundaries (heavy-row positions) of the staging-buffer batches."""
    hp = np.ascontiguousarray(heavy_prefix, dtype=np.int64)
    n = hp.size - 1
    out = np.zeros(n + 2, dtype=np.int64)
    rc = load_library().gm_planner_batches(hp.ctypes.data, n, stage_elems, out.ctypes.data, out.size)
    if rc < 0:
        raise GmError(int(rc), "gm_planner_batches", "a row exceeds stage_elems")
    return out[: rc + 1].tolist()


def _stream_ptr(stream) -> int:
    if stream is None:  # (without building a Stream object: a few microseconds that a small product feels)
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return int(stream.cuda_stream)


class Plan:
    """Owner of a gm_plan*.  Keeps A and B alive, since the plan borrows their arrays."""

    def __init__(self, handle, A: DeviceCSR, B: DeviceCSR):
        self._h, self.A, self.B = handle, A, B

    def info(self) -> PlanInfo:
        out = PlanInfo()
        _check(load_library().gm_plan_get_info(self._h, ctypes.byref(out)), "gm_plan_get_info")
        return out

    def stats(self) -> ExecStats:
        out = ExecStats()
        _check(load_library().gm_exec_get_stats(self._h, ctypes.byref(out)), "gm_exec_get_stats")
        return out

    def set_timing(self, enable: bool):
        _check(load_library().gm_plan_set_timing(self._h, int(enable)), "gm_plan_set_timing")

    def row_products(self, stream=None) -> torch.Tensor:
        out = torch.empty(self.A.n_rows, dtype=torch.int64, device=self.A.row_ptr.device)
        _check(load_library().gm_plan_get_row_products(self._h, out.data_ptr(), _stream_ptr(stream)),
               "gm_plan_get_row_products")
        return out

    def destroy(self):
        if self._h:
            load_library().gm_plan_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


NOALLOC_MAX_NNZ_A = 1048576


def row_products_noalloc(A: DeviceCSR, B: DeviceCSR, out: torch.Tensor, stream=None) -> torch.Tensor:
    """gm_row_products_noalloc: IP_i for every row of A, written into the caller's int64 device tensor
    `out` (A.n_rows entries).  The library allocates nothing; nnz(A) is limited to NOALLOC_MAX_NNZ_A."""
    assert out.dtype == torch.int64 and out.is_contiguous() and out.numel() >= A.n_rows
    a = A._struct()
    b = a if B is A else B._struct()
    _check(load_library().gm_row_products_noalloc(ctypes.byref(a), ctypes.byref(b), out.data_ptr(),
                                                  _stream_ptr(stream)), "gm_row_products_noalloc")
    return out


def spgemm_plan(A: DeviceCSR, B: DeviceCSR, smem_bytes: int = 232448, opts: PlanOpts | None = None,
                stream=None) -> Plan:
    """gm_spgemm_plan_ex on the current (or given) torch stream."""
    lib = load_library()
    h = ctypes.c_void_p()
    a = A._struct()
    b = a if B is A else B._struct()
    _check(lib.gm_spgemm_plan_ex(ctypes.byref(a), ctypes.byref(b), smem_bytes,
                                 ctypes.byref(opts) if opts else None, _stream_ptr(stream), ctypes.byref(h)),
           "gm_spgemm_plan")
    return Plan(h, A, B)


def _wrap(ptr: int, numel: int, dtype) -> torch.Tensor:
    t = _live.pop(ptr).view(dtype)
    return t if t.numel() == numel else t[:numel]


def spgemm_execute(plan: Plan, stream=None) -> DeviceCSR:
    """gm_spgemm_execute; the result's arrays are torch tensors over the library's allocations."""
    lib = load_library()
    c = _CSR()
    _check(lib.gm_spgemm_execute(plan._h, _stream_ptr(stream), ctypes.byref(c)), "gm_spgemm_execute")
    vdt = torch.float32 if c.dtype == 0 else torch.float64
    return DeviceCSR(c.n_rows, c.n_cols, _wrap(c.row_ptr, c.n_rows + 1, torch.int64),
                     _wrap(c.col_idx, c.nnz, torch.int32), _wrap(c.vals, c.nnz, vdt), int(c.nnz))


def spgemm(A: DeviceCSR, B: DeviceCSR, smem_bytes: int = 232448, opts: PlanOpts | None = None, stream=None):
    """plan + execute + destroy; returns (C, PlanInfo, ExecStats)."""
    plan = spgemm_plan(A, B, smem_bytes, opts, stream)
    try:
        C = spgemm_execute(plan, stream)
        return C, plan.info(), plan.stats()
    finally:
        plan.destroy()


def _host_struct(M, keep: list) -> _CSR:
    rp = np.ascontiguousarray(M.row_ptr, dtype=np.int64)
    ci = np.ascontiguousarray(M.col, dtype=np.int32)
    va = np.ascontiguousarray(M.val)
    keep += [rp, ci, va]
    return _CSR(M.n_rows, M.n_cols, int(rp[-1]), rp.ctypes.data, ci.ctypes.data, va.ctypes.data,
                0 if va.dtype == np.float32 else 1, 0)


def spgemm_host(A, B, out_row_ptr: np.ndarray, out_col: np.ndarray, out_val: np.ndarray,
                smem_bytes: int = 232448, opts: PlanOpts | None = None) -> int:
    """gm_spgemm_host: A, B and the output buffers are HOST arrays (numpy; pinned if they wrap pinned
    torch tensors).  Returns nnz(C); raises GmError(GM_ERR_CAPACITY) if the buffers are too small."""
    keep: list = []
    a, b = _host_struct(A, keep), _host_struct(B, keep)
    c = _CSR(0, 0, 0, out_row_ptr.ctypes.data, out_col.ctypes.data, out_val.ctypes.data, a.dtype, 0)
    cap = min(out_col.size, out_val.size)
    _check(load_library().gm_spgemm_host(ctypes.byref(a), ctypes.byref(b), smem_bytes,
                                         ctypes.byref(opts) if opts else None, ctypes.byref(c), cap),
           "gm_spgemm_host")
    return int(c.nnz)


# ---------------------------------------------------------------------------------------------------------------------
# Routed products: R (DeviceCSR) picks blocks of a dense factor.  No autograd graph is recorded; gradients have calls of their own.
# (Marshalling is kept short here: a product of a few rows takes the GPU about as long as it takes the host to call it.)
# ---------------------------------------------------------------------------------------------------------------------
_DTYPES = {torch.float32: 0, torch.float64: 1, torch.bfloat16: 2, torch.float16: 3, torch.float8_e4m3fn: 4}
_byref = ctypes.byref


_pack_dense = struct.Struct("=7q2i").pack  # a gm_dense


def _dense(t: torch.Tensor, where: str, device: torch.device) -> bytes:
    if t.device != device:
        raise GmError(-1, where, f"a tensor on {t.device}, the others on {device}")
    shape, stride = t.shape, t.stride()
    if len(shape) == 2:
        return _pack_dense(t.data_ptr(), 1, shape[0], shape[1], 0, stride[0], stride[1], _DTYPES.get(t.dtype, -1), 0)
    return _pack_dense(t.data_ptr(), *shape, *stride, _DTYPES.get(t.dtype, -1), 0)


def _result(t: torch.Tensor, rows: int, cols: int) -> bytes:
    """A contiguous matrix that the call has just made."""
    return _pack_dense(t.data_ptr(), 1, rows, cols, 0, cols, 1, _DTYPES.get(t.dtype, -1), 0)


def _empty(like: torch.Tensor, rows: int, cols: int, dtype) -> torch.Tensor:
    return like.new_empty((rows, cols)) if dtype is None else like.new_empty((rows, cols), dtype=dtype)


def _dims(t: torch.Tensor, where: str, name: str, dims: int):
    if t.dim() != dims:
        raise GmError(-2, where, f"{name}: {t.dim()} dimensions instead of {dims}")


_current_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else None
_current_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else None


def _on_cuda(where: str, device: torch.device):
    if device.type != "cuda":
        raise GmError(-1, where, f"tensors on {device}: a CUDA device expected")


def _there(call, device: torch.device, stream, *args, **kwargs):
    """The same call with the tensors' device and the given stream made current, so that what it allocates belongs to that stream; the
    inputs' memory is not given to others before the stream is done with it."""
    if stream is not None and stream.device != device:
        raise GmError(-1, call.__name__, f"a stream of {stream.device}, the tensors on {device}")
    with torch.cuda.device(device), torch.cuda.stream(stream):
        if stream is not None:
            for a in args:
                for t in (a.row_ptr, a.col, a.val) if isinstance(a, DeviceCSR) else (a,):
                    if isinstance(t, torch.Tensor) and t.is_cuda:
                        t.record_stream(stream)
        return call(*args, **kwargs)


class Route:
    """Owner of a gm_route*: the entries of R in the order of their columns.

    offsets (n_cols + 1, int64): first place of every column, and behind the last one the number of routed entries;
    rows, order (nnz, int32): row and entry of R at every place; pos (nnz, int32): place of every entry.
    Keeps R alive, whose row_ptr and val it borrows: values may change in place; calls that read an array of R that has been
    replaced are refused.  It may go before its work is done, and status() goes with it.  A graph reads R's arrays at every replay, and
    those of the route if the route was made before the capture: keep R, and such a route, as long as the graph."""

    def __init__(self, handle, R: DeviceCSR, stream: int, memory: torch.Tensor):
        self._h, self.R, self._stream, self._memory = handle, R, stream, memory
        self.n_rows, self.n_cols, self.nnz, self.device = R.n_rows, R.n_cols, R.nnz, memory.device
        self._index = self.device.index
        self._row_ptr, self._val = R.row_ptr, R.val  # what the library has the addresses of
        self._at = R.row_ptr.data_ptr(), R.val.data_ptr()

    def _reads(self, where: str, val: bool):
        """R's arrays must be the ones that the route was made of, wherever a call reads them."""
        if self.R.row_ptr.data_ptr() != self._at[0] or (val and self.R.val.data_ptr() != self._at[1]):
            raise GmError(-1, where, "R has got other arrays since its route was made: change values in place, or make another route")

    def _places(self, k: int) -> torch.Tensor:
        first = 2 * (self.n_cols + 1) + k * self.nnz
        return self._memory[first: first + self.nnz]

    @property
    def offsets(self) -> torch.Tensor:
        return self._memory[: 2 * (self.n_cols + 1)].view(torch.int64)

    @property
    def rows(self) -> torch.Tensor:
        return self._places(0)

    @property
    def order(self) -> torch.Tensor:
        return self._places(1)

    @property
    def pos(self) -> torch.Tensor:
        return self._places(2)

    def status(self):
        """Raises GmError(GM_ERR_TIMEOUT) if a kernel of a finished call on this route gave up a wait."""
        _check(load_library().gm_route_status(self._h), "gm_route_status")

    def _current_stream(self) -> int:
        stream = _current_raw_stream(self._index)
        if stream != self._stream:  # not the one its memory belongs to
            s = torch.cuda.current_stream(self.device)
            for t in (self._memory, self._row_ptr, self._val):
                t.record_stream(s)
        return stream

    def destroy(self):
        if self._h:
            load_library().gm_route_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def route_plan(R: DeviceCSR, stream=None) -> Route:
    """gm_route_plan: the entries of R (float32 values, at most 2048 columns) in the order of their columns.  An entry whose
    column is outside [0, R.n_cols) is routed nowhere."""
    where = "gm_route_plan"
    device = R.row_ptr.device
    _on_cuda(where, device)
    if stream is not None or device.index != _current_device():
        return _there(route_plan, device, stream, R)
    if R.col.device != device or R.val.device != device:
        raise GmError(-1, where, "R's arrays are on different devices")
    if R.n_cols < 0 or R.nnz < 0 or R.row_ptr.numel() < R.n_rows + 1 or R.col.numel() < R.nnz or R.val.numel() < R.nnz:
        raise GmError(-1, where, "R's arrays are shorter than its sizes say")
    n_off = 2 * (R.n_cols + 1)
    memory = torch.empty(n_off + 3 * R.nnz, dtype=torch.int32, device=device)
    st, h, at = _current_raw_stream(device.index), ctypes.c_void_p(), memory.data_ptr()
    rows = at + 4 * n_off
    _check(load_library().gm_route_plan(_byref(R._struct()), at, rows, rows + 4 * R.nnz, rows + 8 * R.nnz, st, _byref(h)), where)
    return Route(h, R, st, memory)


def route_product(route: Route, X: torch.Tensor, W: torch.Tensor, by_entry: bool = False, dtype=None, stream=None) -> torch.Tensor:
    """gm_route_product: P[p] = X[row of place p] @ W[its column].T, (nnz, N), in `dtype` (default: X's).  X (n_rows, K), or with
    by_entry (nnz, K) with a row for each place; W (n_cols, N, K); bf16 or f16."""
    where, device = "gm_route_product", route.device
    if stream is not None or route._index != _current_device():
        return _there(route_product, device, stream, route, X, W, by_entry, dtype)
    _dims(X, where, "X", 2)
    _dims(W, where, "W", 3)
    N = W.shape[1]
    P = _empty(X, route.nnz, N, dtype)
    _check(load_library().gm_route_product(route._h, _dense(X, where, device), by_entry, _dense(W, where, device),
                                           _result(P, route.nnz, N), route._current_stream()), where)
    return P


def route_product_dx(route: Route, dP: torch.Tensor, W: torch.Tensor, by_entry: bool = False, dtype=None, stream=None) -> torch.Tensor:
    """gm_route_product_dx: the gradient of route_product with respect to X, (n_rows, K), or (nnz, K) with by_entry."""
    where, device = "gm_route_product_dx", route.device
    if stream is not None or route._index != _current_device():
        return _there(route_product_dx, device, stream, route, dP, W, by_entry, dtype)
    _dims(dP, where, "dP", 2)
    _dims(W, where, "W", 3)
    if not by_entry:
        route._reads(where, False)
    rows, K = route.nnz if by_entry else route.n_rows, W.shape[2]
    dX = _empty(dP, rows, K, dtype)
    terms = None if by_entry else torch.empty(route.nnz * (K + 7 & ~7), dtype=torch.float32, device=device)
    _check(load_library().gm_route_product_dx(route._h, _dense(dP, where, device), _dense(W, where, device), by_entry, _result(dX, rows, K),
                                              terms.data_ptr() if terms is not None else None, route._current_stream()), where)
    return dX


def route_product_dw(route: Route, dP: torch.Tensor, X: torch.Tensor, by_entry: bool = False, dtype=None, stream=None) -> torch.Tensor:
    """gm_route_product_dw: the gradient of route_product with respect to W, (n_cols, N, K)."""
    where, device = "gm_route_product_dw", route.device
    if stream is not None or route._index != _current_device():
        return _there(route_product_dw, device, stream, route, dP, X, by_entry, dtype)
    _dims(dP, where, "dP", 2)
    _dims(X, where, "X", 2)
    dW = torch.empty((route.n_cols, dP.shape[1], X.shape[1]), dtype=dtype or dP.dtype, device=device)
    _check(load_library().gm_route_product_dw(route._h, _dense(dP, where, device), _dense(X, where, device), by_entry,
                                              _dense(dW, where, device), route._current_stream()), where)
    return dW


def route_sum(route: Route, P: torch.Tensor, weighted: bool = True, dtype=None, stream=None) -> torch.Tensor:
    """gm_route_sum: Y[i] = sum over the entries of row i of R of their row of P, times R's value if `weighted`.  P (nnz, N) by place."""
    where, device = "gm_route_sum", route.device
    if stream is not None or route._index != _current_device():
        return _there(route_sum, device, stream, route, P, weighted, dtype)
    _dims(P, where, "P", 2)
    route._reads(where, weighted)
    Y = _empty(P, route.n_rows, P.shape[1], dtype)
    _check(load_library().gm_route_sum(route._h, _dense(P, where, device), weighted, _result(Y, route.n_rows, P.shape[1]), route._current_stream()), where)
    return Y


def route_sum_grads(route: Route, dY: torch.Tensor, P: torch.Tensor, stream=None) -> tuple[torch.Tensor, torch.Tensor]:
    """gm_route_sum_grads: gradients of the weighted route_sum, dP (nnz, N) by place and dval (nnz,) float32 by entry of R."""
    where, device = "gm_route_sum_grads", route.device
    if stream is not None or route._index != _current_device():
        return _there(route_sum_grads, device, stream, route, dY, P)
    _dims(dY, where, "dY", 2)
    _dims(P, where, "P", 2)
    route._reads(where, True)
    dP = _empty(P, route.nnz, P.shape[1], None)
    dval = torch.empty(route.nnz, dtype=torch.float32, device=device)
    _check(load_library().gm_route_sum_grads(route._h, _dense(dY, where, device), _dense(P, where, device), _result(dP, route.nnz, P.shape[1]),
                                             dval.data_ptr(), route._current_stream()), where)
    return dP, dval


def block_quantize(X: torch.Tensor, block_rows: int = 1, stream=None) -> tuple[torch.Tensor, torch.Tensor]:
    """gm_block_quantize: (values in float8_e4m3fn, float32 scales) of X (rows, K) or (blocks, rows, K), bf16 or f16, with a scale for
    each block of block_rows (1 or 128) x 128."""
    where, device = "gm_block_quantize", X.device
    _on_cuda(where, device)
    if stream is not None or device.index != _current_device():
        return _there(block_quantize, device, stream, X, block_rows)
    if block_rows not in (1, 128):
        raise GmError(-1, where, "block_rows: 1 or 128 expected")
    shape = X.shape
    if len(shape) not in (2, 3):
        raise GmError(-2, where, f"X: {len(shape)} dimensions instead of 2 or 3")
    rows, cols = shape[-2], shape[-1]
    s_rows, s_cols = -(-rows // block_rows), -(-cols // 128)
    blocks = shape[0] if len(shape) == 3 else 1
    Q = X.new_empty(shape, dtype=torch.float8_e4m3fn)
    S = X.new_empty((s_rows, s_cols) if len(shape) == 2 else (blocks, s_rows, s_cols), dtype=torch.float32)
    _check(load_library().gm_block_quantize(_dense(X, where, device), block_rows,
                                            _pack_dense(Q.data_ptr(), blocks, rows, cols, rows * cols, cols, 1, 4, 0),
                                            _pack_dense(S.data_ptr(), blocks, s_rows, s_cols, s_rows * s_cols, s_cols, 1, 0, 0),
                                            _current_raw_stream(device.index)), where)
    return Q, S


def route_product_scaled(route: Route, Xq: torch.Tensor, Xs: torch.Tensor, Wq: torch.Tensor, Ws: torch.Tensor, by_entry: bool = False,
                         dtype=torch.bfloat16, stream=None) -> torch.Tensor:
    """gm_route_product_scaled: route_product of float8_e4m3fn factors with scales, as block_quantize gives them: Xs (rows of X, K / 128),
    Ws (n_cols, N / 128, K / 128) or (n_cols, N, K / 128), all rounded up."""
    where, device = "gm_route_product_scaled", route.device
    if stream is not None or route._index != _current_device():
        return _there(route_product_scaled, device, stream, route, Xq, Xs, Wq, Ws, by_entry, dtype)
    for t, name, dims in ((Xq, "Xq", 2), (Xs, "Xs", 2), (Wq, "Wq", 3), (Ws, "Ws", 3)):
        _dims(t, where, name, dims)
    N = Wq.shape[1]
    P = _empty(Xq, route.nnz, N, dtype)
    _check(load_library().gm_route_product_scaled(route._h, _dense(Xq, where, device), _dense(Xs, where, device), by_entry,
                                                  _dense(Wq, where, device), _dense(Ws, where, device), _result(P, route.nnz, N),
                                                  route._current_stream()), where)
    return P

"""Thin binding of libavsg.so: argument marshalling only, by ctypes and, for
the calls of every step, by an extension module (csrc/python_calls.cpp) where
that has been built for this Python.

Every step of the operator runs in the CUDA kernels behind the C ABI
(include/avsg.h).  PyTorch supplies device tensors, pinned host tensors and
streams.  If the library is missing the import of this module still works, but
any use raises: there is no CPU fallback.
"""
from __future__ import annotations

import array
import ctypes
import os
import struct
from typing import List, Optional, Sequence, Union

import numpy as np

from . import build as _build

OK, EINVAL, ENOMEM, ECUDA, ECAPACITY, EDEVICE_STATUS, EUNSUPPORTED = 0, -1, -2, -3, -4, -5, -6
XFER_SM_BALANCED, XFER_COPY_ENGINE, XFER_REQUEST_LEVEL, XFER_ALL_K, XFER_POSITION_LEVEL, XFER_SM_OVERLAP = 0, 1, 2, 3, 4, 5
INDEX_HASH, INDEX_DIRECT, INDEX_PAPER = 0, 1, 2
ROW_BF16, ROW_FP8, ROW_FP4 = 0, 1, 2
LATENT_DIMS, ROPE_DIMS = 512, 64
STATUS_PROBE_EXHAUSTED, STATUS_NO_DEAD_SLOTS, STATUS_BAD_SLOT, STATUS_BAD_SEGMENT, STATUS_BAD_ID, STATUS_WAIT_TIMEOUT = (
    1, 2, 4, 8, 16, 32)
STATUS_LAUNCH_FAILED = 64

EXPORTS = (
    "avsg_create", "avsg_destroy", "avsg_reset", "avsg_reset_async", "avsg_step", "avsg_step_host", "avsg_buffer", "avsg_stats", "avsg_table_stats",
    "avsg_sync_status", "avsg_export_state", "avsg_import_state", "avsg_save_state", "avsg_restore_state",
    "avsg_set_transfer_mode", "avsg_set_timing", "avsg_set_transfer_geometry", "avsg_strerror",
    "avsg_step_noalloc", "avsg_export_hash_state", "avsg_import_hash_state", "avsg_clear_status",
    "avsg_probe_wait_limit", "avsg_host_kv_alloc", "avsg_host_kv_free", "avsg_row_bytes", "avsg_append", "avsg_attend",
)


class AvsgConfig(ctypes.Structure):
    _fields_ = [("num_tables", ctypes.c_uint32), ("buffer_slots", ctypes.c_uint32), ("row_bytes", ctypes.c_uint32),
                ("max_topk", ctypes.c_uint32), ("max_tokens", ctypes.c_uint32), ("max_lifetime", ctypes.c_int32),
                ("transfer_mode", ctypes.c_uint32), ("device", ctypes.c_int32), ("index_mode", ctypes.c_uint32),
                ("max_context", ctypes.c_uint32), ("probe_retries", ctypes.c_uint32), ("hash_a1", ctypes.c_uint32),
                ("hash_a2", ctypes.c_uint32), ("stage_one_cluster", ctypes.c_uint32)]


class AvsgStepArgs(ctypes.Structure):
    _fields_ = [("n", ctypes.c_uint32), ("table_ids", ctypes.c_void_p), ("n_tokens", ctypes.c_uint32),
                ("topk", ctypes.c_uint32), ("indices", ctypes.c_void_p), ("kv_base", ctypes.c_void_p),
                ("row_stride", ctypes.c_void_p), ("verified_len", ctypes.c_void_p), ("slots", ctypes.c_void_p),
                ("hit", ctypes.c_void_p), ("miss_count", ctypes.c_void_p), ("verified_len_dev", ctypes.c_void_p),
                ("kv_rows", ctypes.c_void_p), ("stage_one_done", ctypes.c_void_p),
                ("stage_one_done_value", ctypes.c_uint64), ("arriving", ctypes.c_void_p)]


class AvsgStats(ctypes.Structure):
    _fields_ = [("steps", ctypes.c_uint64), ("tokens", ctypes.c_uint64), ("hits", ctypes.c_uint64),
                ("misses", ctypes.c_uint64), ("rows_copied", ctypes.c_uint64), ("bytes_copied", ctypes.c_uint64),
                ("extra_decays", ctypes.c_uint64), ("last_stage_one_us", ctypes.c_float),
                ("last_transfer_us", ctypes.c_float), ("last_rows", ctypes.c_uint64),
                ("last_stage_one_kernel_us", ctypes.c_float), ("last_transfer_kernel_us", ctypes.c_float),
                ("last_transfer_start_us", ctypes.c_float), ("last_copy_start_us", ctypes.c_float),
                ("last_first_row_us", ctypes.c_float), ("last_first_block_done_us", ctypes.c_float),
                ("last_call_kernel_us", ctypes.c_float), ("reserved", ctypes.c_float)]


class AvsgNoAllocArgs(ctypes.Structure):
    _fields_ = [("n", ctypes.c_uint32), ("n_tokens", ctypes.c_uint32), ("topk", ctypes.c_uint32),
                ("buffer_slots", ctypes.c_uint32), ("row_bytes", ctypes.c_uint32), ("max_lifetime", ctypes.c_int32),
                ("tok", ctypes.c_void_p), ("life", ctypes.c_void_p), ("buffer", ctypes.c_void_p),
                ("indices", ctypes.c_void_p), ("kv_base", ctypes.c_void_p), ("row_stride", ctypes.c_void_p),
                ("verified_len", ctypes.c_void_p), ("slots", ctypes.c_void_p), ("hit", ctypes.c_void_p),
                ("miss_count", ctypes.c_void_p), ("status", ctypes.c_void_p), ("kv_rows", ctypes.c_void_p)]


class AvsgRope(ctypes.Structure):
    _fields_ = [("inv_freq", ctypes.c_double * 32), ("scale", ctypes.c_float), ("halves", ctypes.c_uint32)]


class AvsgAppendArgs(ctypes.Structure):
    _fields_ = [("n", ctypes.c_uint32), ("n_tokens", ctypes.c_uint32), ("row_format", ctypes.c_uint32), ("type", ctypes.c_uint32),
                ("table_ids", ctypes.c_void_p), ("latent", ctypes.c_void_p), ("rope_part", ctypes.c_void_p),
                ("latent_stride", ctypes.c_uint64 * 2), ("rope_stride", ctypes.c_uint64 * 2), ("positions", ctypes.c_void_p),
                ("rows", ctypes.c_void_p), ("kv_base", ctypes.c_void_p), ("kv", ctypes.c_void_p), ("kv_table_stride", ctypes.c_uint64),
                ("row_stride", ctypes.c_void_p), ("kv_rows", ctypes.c_void_p), ("rope", ctypes.c_void_p), ("values", ctypes.c_void_p),
                ("status", ctypes.c_void_p)]


class AvsgAttendArgs(ctypes.Structure):
    _fields_ = [("n", ctypes.c_uint32), ("n_tokens", ctypes.c_uint32), ("topk", ctypes.c_uint32), ("heads", ctypes.c_uint32),
                ("row_format", ctypes.c_uint32), ("buffer_slots", ctypes.c_uint32), ("buffer_row_bytes", ctypes.c_uint64),
                ("table_ids", ctypes.c_void_p), ("buffer", ctypes.c_void_p), ("slots", ctypes.c_void_p), ("q", ctypes.c_void_p),
                ("q_stride", ctypes.c_uint64 * 3), ("out", ctypes.c_void_p), ("out_stride", ctypes.c_uint64 * 3), ("lse", ctypes.c_void_p),
                ("scale", ctypes.c_float), ("softcap", ctypes.c_float), ("ids", ctypes.c_void_p), ("positions", ctypes.c_void_p),
                ("spans", ctypes.c_void_p), ("slopes", ctypes.c_void_p), ("rope", ctypes.c_void_p), ("status", ctypes.c_void_p)]


NOALLOC_MAX_TABLES, NOALLOC_MAX_IDS = 32, 131072


class AvsgError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__("%s (code %d)" % (what, code))
        self.code = code


_lib = _calls = None


def _python_calls():
    """The extension module (built in-tree by build.build_library), or False: another Python than it was built for, or a
    machine that could not build it.  The same calls are then marshalled by ctypes, 2 to 6 us slower."""
    global _calls
    if _calls is None:
        try:
            from . import _python_calls as module
        except ImportError:
            module = False
        else:
            module.set_binding(_addr, _c_array, _set_lengths, _stream_handle, None, None)
        _calls = module
    return _calls


def load_library():
    """Loads libavsg.so (built in-tree by build.build_library); raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_build.LIB):
        raise RuntimeError("libavsg.so is missing: run `python __graft_entry__.py` (needs nvcc) to build it; "
                           "there is no CPU fallback")
    lib = ctypes.CDLL(_build.LIB)
    vp, u32, i32 = ctypes.c_void_p, ctypes.c_uint32, ctypes.c_int
    lib.avsg_create.argtypes, lib.avsg_create.restype = [ctypes.POINTER(AvsgConfig), ctypes.POINTER(vp)], i32
    lib.avsg_destroy.argtypes, lib.avsg_destroy.restype = [vp], i32
    lib.avsg_reset.argtypes, lib.avsg_reset.restype = [vp, vp, u32], i32
    lib.avsg_step.argtypes, lib.avsg_step.restype = [vp, ctypes.POINTER(AvsgStepArgs), vp], i32
    lib.avsg_step_host.argtypes, lib.avsg_step_host.restype = [vp, ctypes.POINTER(AvsgStepArgs), vp], i32
    lib.avsg_buffer.argtypes, lib.avsg_buffer.restype = [vp, u32, ctypes.POINTER(vp)], i32
    lib.avsg_stats.argtypes, lib.avsg_stats.restype = [vp, ctypes.POINTER(AvsgStats)], i32
    lib.avsg_table_stats.argtypes, lib.avsg_table_stats.restype = [vp, u32, ctypes.POINTER(AvsgStats)], i32
    lib.avsg_sync_status.argtypes, lib.avsg_sync_status.restype = [vp, ctypes.POINTER(u32)], i32
    lib.avsg_reset_async.argtypes, lib.avsg_reset_async.restype = [vp, vp, u32, vp], i32
    lib.avsg_clear_status.argtypes, lib.avsg_clear_status.restype = [vp], i32
    lib.avsg_probe_wait_limit.argtypes, lib.avsg_probe_wait_limit.restype = [vp, vp], i32
    lib.avsg_export_state.argtypes, lib.avsg_export_state.restype = [vp, u32, vp, vp], i32
    lib.avsg_import_state.argtypes, lib.avsg_import_state.restype = [vp, u32, vp, vp], i32
    lib.avsg_save_state.argtypes, lib.avsg_save_state.restype = [vp, vp], i32
    lib.avsg_restore_state.argtypes, lib.avsg_restore_state.restype = [vp, vp], i32
    lib.avsg_set_transfer_mode.argtypes, lib.avsg_set_transfer_mode.restype = [vp, u32], i32
    lib.avsg_set_timing.argtypes, lib.avsg_set_timing.restype = [vp, i32], i32
    lib.avsg_set_transfer_geometry.argtypes, lib.avsg_set_transfer_geometry.restype = [vp, u32, u32], i32
    lib.avsg_strerror.argtypes, lib.avsg_strerror.restype = [i32], ctypes.c_char_p
    lib.avsg_step_noalloc.argtypes, lib.avsg_step_noalloc.restype = [ctypes.POINTER(AvsgNoAllocArgs), vp], i32
    lib.avsg_export_hash_state.argtypes, lib.avsg_export_hash_state.restype = [vp, u32, vp, vp], i32
    lib.avsg_import_hash_state.argtypes, lib.avsg_import_hash_state.restype = [vp, u32, vp, vp], i32
    lib.avsg_host_kv_alloc.argtypes = [ctypes.c_size_t, u32, ctypes.POINTER(vp), ctypes.POINTER(ctypes.c_uint64)]
    lib.avsg_host_kv_alloc.restype = i32
    lib.avsg_host_kv_free.argtypes, lib.avsg_host_kv_free.restype = [vp], i32
    lib.avsg_row_bytes.argtypes, lib.avsg_row_bytes.restype = [u32], u32
    lib.avsg_append.argtypes, lib.avsg_append.restype = [vp, ctypes.POINTER(AvsgAppendArgs), vp], i32
    lib.avsg_attend.argtypes, lib.avsg_attend.restype = [vp, ctypes.POINTER(AvsgAttendArgs), vp], i32
    _lib = lib
    return lib


def _check(rc: int, what: str) -> None:
    if rc != OK:
        raise AvsgError(rc, "%s: %s" % (what, load_library().avsg_strerror(rc).decode()))


HOST_KV_HUGE_PAGES = 1


class HostKV:
    """A range from avsg_host_kv_alloc: pinned, device-mapped host bytes, zero-filled, touched by the calling thread."""

    def __init__(self, nbytes: int, huge_pages: bool = True):
        ptr, huge = ctypes.c_void_p(), ctypes.c_uint64()
        _check(load_library().avsg_host_kv_alloc(int(nbytes), HOST_KV_HUGE_PAGES if huge_pages else 0,
                                                 ctypes.byref(ptr), ctypes.byref(huge)), "avsg_host_kv_alloc")
        self.ptr, self.nbytes, self.huge_bytes = int(ptr.value), int(nbytes), int(huge.value)
        self.mapped_bytes = -(-int(nbytes) // (2 << 20)) * (2 << 20)           # what the library registered

    def data_ptr(self) -> int:
        return self.ptr

    def numpy(self):
        """The bytes as a numpy view (no copy); dead after free()."""
        return np.ctypeslib.as_array((ctypes.c_uint8 * self.nbytes).from_address(self.ptr))

    def free(self) -> None:
        if self.ptr:
            ptr, self.ptr = self.ptr, 0
            _check(load_library().avsg_host_kv_free(ptr), "avsg_host_kv_free")

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass


def pinned_empty(nbytes: int, huge_pages: bool = False):
    """Pinned (page-locked, device-mapped) host bytes for a table's host KV: a torch tensor, or with huge_pages a
    HostKV range backed by transparent 2 MiB pages where the kernel grants them (App. G)."""
    if huge_pages:
        return HostKV(nbytes, True)
    import torch
    return torch.empty(int(nbytes), dtype=torch.uint8, pin_memory=True)


def _addr(x) -> int:
    """Address of a torch tensor / numpy array, or an integer address itself."""
    if isinstance(x, int):
        return x
    if hasattr(x, "data_ptr"):
        return int(x.data_ptr())
    if isinstance(x, np.ndarray):
        return int(x.ctypes.data)
    raise TypeError("expected a tensor, an array or an address, got %r" % type(x))


_current_stream_fn = None


def _current_stream() -> int:
    """Handle of the current device's current stream.  torch.cuda.current_stream() builds a Stream object (3.2 us); the
    functions beneath it give the handle in 0.2 us, where the installed torch has them."""
    global _current_stream_fn
    if _current_stream_fn is None:
        import torch
        torch.cuda.init()
        raw, dev = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
        if raw is not None and dev is not None:
            _current_stream_fn = lambda: raw(dev())
            if _python_calls():
                _calls.set_binding(_addr, _c_array, _set_lengths, _stream_handle, raw, dev)     # (the extension asks them itself from now on)
        else:
            _current_stream_fn = lambda: torch.cuda.current_stream().cuda_stream
    return _current_stream_fn()


def _stream_handle(stream) -> Optional[int]:
    if stream is None:
        return _current_stream() or None
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream or None


class _DevView:
    """Wraps a raw device pointer so that torch can view it without a copy."""

    def __init__(self, ptr: int, shape, typestr: str, owner):
        self.__cuda_array_interface__ = {"shape": tuple(shape), "typestr": typestr, "data": (ptr, False),
                                         "version": 3, "strides": None}
        self._owner = owner


class StepOutput:
    __slots__ = ("slots", "hit", "miss_count", "arriving")

    def __init__(self, slots, hit, miss_count, arriving=None):
        self.slots, self.hit, self.miss_count, self.arriving = slots, hit, miss_count, arriving


def _address_of(function) -> int:
    return ctypes.cast(function, ctypes.c_void_p).value


def _addresses(lib):
    return _address_of(lib.avsg_step), _address_of(lib.avsg_step_host)


def _set_lengths(vlen, values) -> None:
    """Verified lengths from any iterable of n numbers."""
    if not isinstance(values, (list, tuple)):
        values = list(values)                            # (an iterator can be read once only)
    try:
        struct.pack_into("=%di" % len(vlen), vlen, 0, *values)
    except struct.error:                                 # not n integers that fit: as the element type converts them
        vlen[:] = [int(v) for v in values]


class PreparedCall:
    """The argument block of one recurring call (same tables, same host KV): built once, re-used per step."""

    def __init__(self, ctx: "Context", table_ids: Sequence[int], kv: Sequence, n_tokens: int, topk: int,
                 row_stride: Optional[Sequence[int]] = None, kv_rows: Optional[Sequence[int]] = None):
        n = len(table_ids)
        assert len(kv) == n
        self.ctx, self.n, self.n_tokens, self.topk = ctx, n, n_tokens, topk
        self._keep = list(kv)
        self._tids = (ctypes.c_uint32 * n)(*[int(t) for t in table_ids])
        self._kv = (ctypes.c_void_p * n)(*[_addr(k) for k in kv])
        self._stride = (ctypes.c_uint64 * n)(*[int(s) for s in row_stride]) if row_stride is not None else None
        self._vlen = (ctypes.c_int32 * n)()
        self._rows = (ctypes.c_uint32 * n)(*[int(r) for r in kv_rows]) if kv_rows is not None else None
        a = AvsgStepArgs()
        a.n, a.n_tokens, a.topk = n, n_tokens, topk
        a.table_ids = ctypes.addressof(self._tids)
        a.kv_base = ctypes.addressof(self._kv)
        a.row_stride = ctypes.addressof(self._stride) if self._stride is not None else None
        a.verified_len = ctypes.addressof(self._vlen)
        a.kv_rows = ctypes.addressof(self._rows) if self._rows is not None else None
        self.args = a
        self._ref = ctypes.byref(a)
        self._cell, self._native = getattr(ctx, "_cell", None), None
        module = _calls if _calls is not None else _python_calls()
        if module and self._cell is not None:            # (a stand-in for a context has no cell: its library is called from here)
            step, step_host = getattr(ctx, "_addresses", None) or _addresses(ctx._lib)
            self._native = module.Call(ctypes.addressof(a), ctypes.addressof(self._vlen), n, ctypes.addressof(self._cell), step, step_host,
                                       self._vlen)

    def run(self, indices, verified_len: Sequence[int], slots, hit=None, miss_count=None, stream=None,
            host: bool = False, stage_one_done=None, arriving=None) -> None:
        """indices / slots / hit / miss_count: tensors (device, or pinned host when host=True) or addresses.
        verified_len: a sequence of n ints, or an int32 CUDA tensor [n] that the kernel reads when it runs
        (what a call captured in a CUDA graph needs when the sequences grow between replays).
        stage_one_done: None or (device int64 tensor or address, value): the word receives the value once the
        slot table, hit mask and miss counts of the whole call are final, while the missed rows still travel.
        arriving: None or a uint8 device tensor like hit: 1 where the row comes with this call's Stage Two."""
        if self._native is not None:
            rc = self._native.run(indices, verified_len, slots, hit, miss_count, stream, stage_one_done, arriving, host)
        else:
            rc = self._run(indices, verified_len, slots, hit, miss_count, stream, host, stage_one_done, arriving)
        if rc != OK:
            _check(rc, "avsg_step")

    def _run(self, indices, verified_len, slots, hit, miss_count, stream, host, stage_one_done, arriving) -> int:
        a = self.args
        a.arriving = _addr(arriving) if arriving is not None else None
        a.stage_one_done, a.stage_one_done_value = (None, 0) if stage_one_done is None else (_addr(stage_one_done[0]), int(stage_one_done[1]))
        a.verified_len_dev = None
        if hasattr(verified_len, "data_ptr"):
            a.verified_len_dev = _addr(verified_len)
        else:
            _set_lengths(self._vlen, verified_len)
        a.indices, a.slots = _addr(indices), _addr(slots)
        a.hit = _addr(hit) if hit is not None else None
        a.miss_count = _addr(miss_count) if miss_count is not None else None
        handle = self.ctx._h if self._cell is None else self._cell.value or None
        lib = self.ctx._lib
        return (lib.avsg_step_host if host else lib.avsg_step)(handle, self._ref, _stream_handle(stream))


class Context:
    """Owns the device state of num_tables tables (see avsg_create)."""

    def __init__(self, num_tables: int, buffer_slots: int, row_bytes: int, max_topk: int, max_tokens: int = 1,
                 max_lifetime: int = 16, transfer_mode: int = XFER_SM_BALANCED, device: int = 0,
                 index_mode: int = INDEX_HASH, max_context: int = 0, probe_retries: int = 0, hash_a1: int = 0,
                 hash_a2: int = 0, stage_one_cluster: int = 0):
        self._lib = load_library()
        self._h = ctypes.c_void_p()
        cfg = AvsgConfig(num_tables, buffer_slots, row_bytes, max_topk, max_tokens, max_lifetime, transfer_mode,
                         device, index_mode, max_context, probe_retries, hash_a1, hash_a2, stage_one_cluster)
        _check(self._lib.avsg_create(ctypes.byref(cfg), ctypes.byref(self._h)), "avsg_create")
        self._cell = ctypes.c_uint64(self._h.value)      # the handle, for prepared calls; 0 when it is closed
        self._addresses = _addresses(self._lib)
        self.num_tables, self.S, self.row_bytes = num_tables, buffer_slots, row_bytes
        self.max_topk, self.max_tokens, self.L, self.device = max_topk, max_tokens, max_lifetime, device

    def close(self) -> None:
        if getattr(self, "_h", None):
            self._cell.value = 0
            self._lib.avsg_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- the hot call ---------------------------------------------------------------------------------
    def prepare(self, table_ids, kv, n_tokens: int, topk: int, row_stride=None, kv_rows=None) -> PreparedCall:
        return PreparedCall(self, table_ids, kv, n_tokens, topk, row_stride, kv_rows)

    def step(self, table_ids, indices, kv, verified_len, row_stride=None, want_hit: bool = True,
             want_miss_count: bool = True, stream=None, kv_rows=None, stage_one_done=None,
             want_arriving: bool = False) -> StepOutput:
        """One decode iteration. indices: int32 CUDA tensor [n, n_tokens, topk]. Returns device tensors."""
        import torch
        assert indices.is_cuda and indices.dtype == torch.int32 and indices.is_contiguous() and indices.dim() == 3
        n, n_q, K = indices.shape
        call = PreparedCall(self, table_ids, kv, n_q, K, row_stride, kv_rows)
        device = indices.get_device()
        on = _stream_of(stream, device)
        slots = _output(indices.shape, torch.int32, device, on)
        hit = _output(indices.shape, torch.uint8, device, on) if want_hit else None
        mc = _output((n, n_q), torch.int32, device, on) if want_miss_count else None
        arriving = _output(indices.shape, torch.uint8, device, on) if want_arriving else None
        call.run(indices, verified_len, slots, hit, mc, stream, stage_one_done=stage_one_done, arriving=arriving)
        out = StepOutput(slots, hit, mc)
        out.arriving = arriving
        return out

    def step_host(self, table_ids, indices, kv, verified_len, row_stride=None, want_hit: bool = True,
                  want_miss_count: bool = True, stream=None) -> StepOutput:
        """Same with host tensors in and out (pinned for asynchrony); returns pinned host tensors."""
        import torch
        assert not indices.is_cuda and indices.dtype == torch.int32 and indices.is_contiguous() and indices.dim() == 3
        n, n_q, K = indices.shape
        call = PreparedCall(self, table_ids, kv, n_q, K, row_stride)
        slots = torch.empty(indices.shape, dtype=torch.int32, pin_memory=True)
        hit = torch.empty(indices.shape, dtype=torch.uint8, pin_memory=True) if want_hit else None
        mc = torch.empty((n, n_q), dtype=torch.int32, pin_memory=True) if want_miss_count else None
        call.run(indices, verified_len, slots, hit, mc, stream, host=True)
        return StepOutput(slots, hit, mc)

    # -- rows into the cache, attention over the buffer -------------------------------------------------
    def append(self, table_ids, latent, rope_part, positions, kv, *, row_format: int, **kw):
        """append() into the caches of this context's tables; problems go to its status word (sync_status)."""
        return append(latent, rope_part, positions, kv, row_format=row_format, _ctx=self, _tables=table_ids, **kw)

    def attend(self, table_ids, q, slots, *, row_format: int, scale: float, **kw):
        """attend() over the buffers of these tables, slots as step() filled them (in the same order of tables)."""
        return attend(q, None, slots, row_format=row_format, scale=scale, _ctx=self, _tables=table_ids, **kw)

    # -- state ----------------------------------------------------------------------------------------
    def reset(self, table_ids: Sequence[int]) -> None:
        ids = (ctypes.c_uint32 * len(table_ids))(*[int(t) for t in table_ids])
        _check(self._lib.avsg_reset(self._h, ids, len(table_ids)), "avsg_reset")

    def reset_async(self, table_ids: Sequence[int], stream=None) -> None:
        """Stream-ordered reset: nothing waits on the host."""
        ids = (ctypes.c_uint32 * len(table_ids))(*[int(t) for t in table_ids])
        _check(self._lib.avsg_reset_async(self._h, ids, len(table_ids), _stream_handle(stream)), "avsg_reset_async")

    def buffer(self, table_id: int):
        """The table's S rows as a uint8 CUDA tensor [S, row_bytes] (a view, no copy)."""
        import torch
        p = ctypes.c_void_p()
        _check(self._lib.avsg_buffer(self._h, table_id, ctypes.byref(p)), "avsg_buffer")
        return torch.as_tensor(_DevView(p.value, (self.S, self.row_bytes), "|u1", self),
                               device="cuda:%d" % self.device)

    def export_state(self, table_id: int):
        tok = np.empty(self.S, np.int32)
        life = np.empty(self.S, np.int8)
        _check(self._lib.avsg_export_state(self._h, table_id, tok.ctypes.data, life.ctypes.data), "avsg_export_state")
        return tok, life

    def import_state(self, table_id: int, tok, life) -> None:
        tok = np.ascontiguousarray(tok, dtype=np.int32)
        life = np.ascontiguousarray(life, dtype=np.int8)
        assert tok.size == self.S and life.size == self.S
        _check(self._lib.avsg_import_state(self._h, table_id, tok.ctypes.data, life.ctypes.data), "avsg_import_state")

    def export_hash_state(self, table_id: int):
        """Paper-literal mode: (c[S] int32, q[S] uint32 packed words)."""
        c = np.empty(self.S, np.int32)
        q = np.empty(self.S, np.uint32)
        _check(self._lib.avsg_export_hash_state(self._h, table_id, c.ctypes.data, q.ctypes.data),
               "avsg_export_hash_state")
        return c, q

    def import_hash_state(self, table_id: int, c, q) -> None:
        c = np.ascontiguousarray(c, dtype=np.int32)
        q = np.ascontiguousarray(q, dtype=np.uint32)
        assert c.size == self.S and q.size == self.S
        _check(self._lib.avsg_import_hash_state(self._h, table_id, c.ctypes.data, q.ctypes.data),
               "avsg_import_hash_state")

    def save_state(self, stream=None) -> None:
        _check(self._lib.avsg_save_state(self._h, _stream_handle(stream)), "avsg_save_state")

    def restore_state(self, stream=None) -> None:
        _check(self._lib.avsg_restore_state(self._h, _stream_handle(stream)), "avsg_restore_state")

    # -- knobs and counters ---------------------------------------------------------------------------
    def set_transfer_mode(self, mode: int) -> None:
        _check(self._lib.avsg_set_transfer_mode(self._h, mode), "avsg_set_transfer_mode")

    def set_timing(self, enable: bool) -> None:
        _check(self._lib.avsg_set_timing(self._h, int(enable)), "avsg_set_timing")

    def set_transfer_geometry(self, blocks: int, threads: int) -> None:
        _check(self._lib.avsg_set_transfer_geometry(self._h, blocks, threads), "avsg_set_transfer_geometry")

    def sync_status(self) -> int:
        """Waits for the device and returns the kernels' status word (0 = no problem was flagged)."""
        w = ctypes.c_uint32(0)
        rc = self._lib.avsg_sync_status(self._h, ctypes.byref(w))
        if rc != EDEVICE_STATUS:
            _check(rc, "avsg_sync_status")
        return w.value

    def clear_status(self) -> None:
        _check(self._lib.avsg_clear_status(self._h), "avsg_clear_status")

    def probe_wait_limit(self, stream=None) -> None:
        """Launches the overlapped transfer kernel alone (its Stage One never comes): it must give up by itself."""
        _check(self._lib.avsg_probe_wait_limit(self._h, _stream_handle(stream)), "avsg_probe_wait_limit")

    def stats(self) -> dict:
        s = AvsgStats()
        _check(self._lib.avsg_stats(self._h, ctypes.byref(s)), "avsg_stats")
        return {name: getattr(s, name) for name, _ in AvsgStats._fields_}

    def table_stats(self, table_id: int) -> dict:
        """Counters of one table (request-level hit rates are averaged from these)."""
        s = AvsgStats()
        _check(self._lib.avsg_table_stats(self._h, table_id, ctypes.byref(s)), "avsg_table_stats")
        return {name: getattr(s, name) for name, _ in AvsgStats._fields_ if not name.startswith("last_")}


_CTYPES = {"Q": ctypes.c_uint64, "I": ctypes.c_uint32, "i": ctypes.c_int32}


def _c_array(kind: str, values, n: int):
    """(owner, address) of a C array of n integers; None: no array.  array.array fills from Python integers at a third of
    a ctypes array's cost; what it does not take (other numbers, another count, values that wrap) goes that way."""
    if values is None:
        return None, None
    if not isinstance(values, (list, tuple)):
        values = list(values)                            # (an iterator can be read once only)
    try:
        out = array.array(kind, values)
        if len(out) == n:
            return out, out.buffer_info()[0]
    except (TypeError, OverflowError):
        pass
    out = (_CTYPES[kind] * n)(*[int(v) for v in values])
    return out, ctypes.addressof(out)


_noalloc_fn = None
_NOALLOC = ctypes.CFUNCTYPE(ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p)


def step_noalloc(tok, life, buffer, indices, kv, verified_len, *, max_lifetime: int = 16, slots, hit=None,
                 miss_count=None, status=None, row_stride=None, stream=None, kv_rows=None) -> None:
    """avsg_step_noalloc: one decode iteration on caller-owned state, for callers that cannot allocate
    (an engine whose own pool holds all device memory, or a path where an allocation's device-wide
    synchronisation is not acceptable).  Every tensor is the caller's; the library allocates nothing and
    keeps its scratch in a fixed array inside the library image.

    tok int32 [n, S], life int8 [n, S], buffer uint8 [n, S, row_bytes], indices int32 [n, n_tokens, topk],
    slots int32 like indices: CUDA tensors on the current device.  kv: one pinned host tensor (or address) per
    table.  Calls that overlap on the GPU race on the shared scratch: keep them on one stream.
    """
    global _noalloc_fn
    if _noalloc_fn is None:
        _noalloc_fn = _address_of(load_library().avsg_step_noalloc)
    module = _python_calls()
    if module:
        rc = module.noalloc(_noalloc_fn, tok, life, buffer, indices, kv, verified_len, max_lifetime, slots, hit, miss_count, status,
                            row_stride, stream, kv_rows)
    else:
        n, S = tok.shape
        _, n_q, K = indices.shape
        kv_owner, kv_at = _c_array("Q", [_addr(k) for k in kv], n)
        length_owner, lengths_at = _c_array("i", verified_len, n)
        stride_owner, strides_at = _c_array("Q", row_stride, n)
        rows_owner, rows_at = _c_array("I", kv_rows, n)
        a = AvsgNoAllocArgs()
        a.n, a.n_tokens, a.topk, a.buffer_slots = n, n_q, K, S
        a.row_bytes, a.max_lifetime = buffer.shape[-1], max_lifetime
        a.tok, a.life, a.buffer, a.indices = _addr(tok), _addr(life), _addr(buffer), _addr(indices)
        a.kv_base, a.row_stride, a.verified_len, a.kv_rows = kv_at, strides_at, lengths_at, rows_at
        a.slots = _addr(slots)
        a.hit = _addr(hit) if hit is not None else None
        a.miss_count = _addr(miss_count) if miss_count is not None else None
        a.status = _addr(status) if status is not None else None
        rc = _NOALLOC(_noalloc_fn)(ctypes.addressof(a), _stream_handle(stream))
    if rc != OK:
        _check(rc, "avsg_step_noalloc")


_ROW_BYTES = {}


def row_bytes(row_format: int) -> int:
    """Bytes of a row of that format: 1152, 656, 400."""
    n = _ROW_BYTES.get(row_format)
    if n is None:
        n = load_library().avsg_row_bytes(row_format)
        if not n:
            raise AvsgError(EINVAL, "row_bytes: no such row format: %r" % (row_format,))
        _ROW_BYTES[row_format] = n
    return n


_ROPE = struct.Struct("=32dfI")


class Rope:
    """Rotation of the last 64 numbers by their position: pair i by the angle position * inv_freq[i], times scale; pairs are
    neighbours, or (halves) 32 apart."""

    def __init__(self, inv_freq: Sequence[float], scale: float = 1.0, halves: bool = False):
        try:
            self.c = AvsgRope.from_buffer_copy(_ROPE.pack(*inv_freq, scale, 1 if halves else 0))
        except struct.error:
            raise AvsgError(EINVAL, "Rope: inv_freq holds %d numbers, scale is one" % (ROPE_DIMS // 2)) from None
        self.address = ctypes.addressof(self.c)


def _need(ok, what: str) -> None:
    if not ok:
        raise AvsgError(EINVAL, what)


def _tensor_at(x, name: str, dtype, shape, device: int) -> int:
    """Address of a contiguous tensor of that type and shape on that device."""
    if x.dtype is dtype and x.shape == shape and x.get_device() == device and x.is_contiguous():
        return x.data_ptr()
    raise AvsgError(EINVAL, "%s: expected a contiguous %s tensor %s on cuda:%d, got %s %s on %s" %
                    (name, dtype, tuple(shape), device, x.dtype, tuple(x.shape), x.device))


def _steps(x, size: int, dims: int):
    """Bytes between the elements of each of the first dimensions (one of a single element may have any stride)."""
    return [size * d if n > 1 else 0 for n, d in zip(x.shape[:dims], x.stride())]


_raw_stream = None


def _stream_of(stream, device: int) -> int:
    """Handle of the stream of a call whose tensors lie on `device`: by default that device's current one."""
    global _raw_stream
    if stream is not None:
        return _stream_handle(stream) or 0
    if _raw_stream is None:
        import torch
        torch.cuda.init()
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda d: torch.cuda.current_stream(d).cuda_stream)
    return _raw_stream(device)


def _output(shape, dtype, device: int, stream: int):
    """An output of a call on that stream.  Its block is one of that stream's (another stream's may still be in use by what is queued
    there), and when the tensor is dropped it waits for what the current stream has queued by then, which reads it."""
    import torch
    if stream == _stream_of(None, device):
        return torch.empty(shape, dtype=dtype, device=device)
    # (1: the handle that CUDA itself has for the default stream)
    on = torch.cuda.ExternalStream(stream, device) if stream > 1 else torch.cuda.default_stream(device)
    with torch.cuda.stream(on):
        out = torch.empty(shape, dtype=dtype, device=device)
    out.record_stream(torch.cuda.current_stream(device))
    return out


# The argument blocks, packed at once: a structure of ctypes filled field by field costs a microsecond for eight of them.
_APPEND = struct.Struct("=4I3Q2Q2Q4QQ5Q")
_ATTEND = struct.Struct("=6I5Q3QQ3QQ2f6Q")


def _packed(layout, what: str, *values) -> bytes:
    try:
        return layout.pack(*values)
    except (struct.error, OverflowError) as e:
        raise AvsgError(EINVAL, "%s: a number does not fit its argument (%s)" % (what, e)) from None


def _status_word(status) -> int:
    """Address of a word that status bits are added to."""
    if hasattr(status, "element_size") and (status.element_size() != 4 or status.numel() == 0):
        raise AvsgError(EINVAL, "status: a word of 32 bits on the call's device is expected, got %s %s" % (status.dtype, tuple(status.shape)))
    return _addr(status)


_ROWS_CALL = ctypes.CFUNCTYPE(ctypes.c_int, ctypes.c_void_p, ctypes.c_char_p, ctypes.c_void_p)
_append_fn = _attend_fn = None
_tensor_calls = False                                # the extension module that makes these calls (csrc/tensor_calls.cpp), where it loads


def _rows_functions():
    global _append_fn, _attend_fn, _tensor_calls
    lib = load_library()
    import torch
    try:
        from . import _tensor_calls as module
    except ImportError:                              # not built: the same calls are marshalled below
        module = None
    _tensor_calls = False
    if module and module.built_for == torch.__version__:
        module.set_library(_address_of(lib.avsg_append), _address_of(lib.avsg_attend), _address_of(lib.avsg_row_bytes))
        _tensor_calls = module
    _append_fn, _attend_fn = _ROWS_CALL(_address_of(lib.avsg_append)), _ROWS_CALL(_address_of(lib.avsg_attend))


def _stream_number(stream):
    return stream if stream is None or type(stream) is int else _stream_handle(stream) or 0


def _rows_in(kv, bytes_: int, stride):
    """Rows that a cache given as a tensor (a HostKV range, a packed array) has room for; None: an address."""
    if hasattr(kv, "element_size"):
        if kv.is_contiguous():
            span = kv.nbytes
            if stride is None:
                return min(span // bytes_, 0x80000000)
        else:
            span = (sum((size - 1) * step for size, step in zip(kv.shape, kv.stride())) + 1) * kv.element_size() if kv.numel() else 0
    elif isinstance(kv, HostKV) or (isinstance(kv, np.ndarray) and kv.flags.c_contiguous):
        span = kv.nbytes
    else:
        return None
    return 0 if span < bytes_ else min((span - bytes_) // (stride or bytes_) + 1, 0x80000000)


def _limits(most, kv_rows):
    """Rows of each cache: `most` (None: no limit known), or fewer where the caller says so."""
    if kv_rows is None:
        return None if all(m is None for m in most) else [0x80000000 if m is None else m for m in most]
    kv_rows = list(kv_rows)
    _need(len(kv_rows) == len(most), "append: one kv_rows per table")
    for m, r in zip(most, kv_rows):
        if m is not None and r > m:
            raise AvsgError(EINVAL, "append: kv_rows says %s rows, the cache has room for %s" % (r, m))
    return kv_rows


def append(latent, rope_part, positions, kv, *, row_format: int, rope: Optional[Rope] = None, rows=None, row_stride=None, kv_rows=None,
           want_values: bool = False, values=None, status=None, stream=None, _ctx=None, _tables=None):
    """avsg_append: the rows of new positions, rotated and quantised on their way into the cache.

    latent [n, n_tokens, 512] and rope_part [n, n_tokens, 64]: CUDA tensors of one type (bf16, fp16, fp32), parts of a wider
    projection too; positions int32 [n, n_tokens], negative = padding; rows int32 like positions: where a token's row goes, if
    not to its position.  kv: a uint8 tensor [n, rows, bytes] (CUDA or pinned), or one pinned or CUDA tensor (or address) per
    table, as avsg_step takes them (a tensor's own bytes are the limit, kv_rows may set a lower one; an address has none but
    kv_rows); a tensor [rows, bytes] is a pool that all tables share.  stream: a torch stream or a handle (default: the current one of
    latent's device).  Returns the values tensor (bf16 [n, n_tokens, 576], what the rows stand for; allocated on that stream; without a
    gradient) where one is wanted, else None."""
    import torch
    if _append_fn is None:
        _rows_functions()
    if _tensor_calls and row_stride is None and kv_rows is None:
        done = _tensor_calls.append(
            None if _ctx is None else _ctx._cell.value or None, _tables, latent, rope_part, positions, kv, row_format, None if rope is None else rope.address,
            rows, bool(want_values), values, None if status is None else _status_word(status), _stream_number(stream))
        if done is not NotImplemented:
            if done[0] != OK:
                _check(done[0], "avsg_append")
            return done[1]
    device, dtype, shape = latent.get_device(), latent.dtype, latent.shape
    if device < 0 or len(shape) != 3 or shape[2] != LATENT_DIMS or latent.stride(2) != 1:
        raise AvsgError(EINVAL, "append: latent is a CUDA tensor [n, n_tokens, 512] with its last numbers side by side")
    n, n_tokens, _ = shape
    kind = 0 if dtype is torch.bfloat16 else 1 if dtype is torch.float16 else 2 if dtype is torch.float32 else -1
    if kind < 0 or rope_part.dtype is not dtype or rope_part.get_device() != device or rope_part.shape != (n, n_tokens, ROPE_DIMS) or \
            rope_part.stride(2) != 1:
        raise AvsgError(EINVAL, "append: rope_part is a tensor [n, n_tokens, 64] of latent's type (bf16, fp16, fp32) and device, with its last "
                                "numbers side by side")
    stream = _stream_of(stream, device)
    size = 4 if kind == 2 else 2
    here = (n, n_tokens)
    kv_base = at = table_step = 0
    keep = []
    if hasattr(kv, "data_ptr") and not isinstance(kv, (list, tuple)):
        full = kv.shape
        bytes_ = row_bytes(row_format)
        if kv.dtype is not torch.uint8 or len(full) not in (2, 3) or full[-1] != bytes_ or kv.stride(-1) != 1 or \
                (len(full) == 3 and full[0] != n) or (kv.is_cuda and kv.get_device() != device):
            raise AvsgError(EINVAL, "append: kv is a uint8 tensor [n, rows, row bytes] or [rows, row bytes] on latent's device or pinned, or a "
                                    "list of caches")
        _need(row_stride is None, "append: row_stride goes with a list of caches")
        at, table_step = kv.data_ptr(), (kv.stride(0) if len(full) == 3 and n > 1 else 0)
        kv_rows = _limits([full[-2]] * n, kv_rows)
        if full[-2] > 1 and kv.stride(-2) != bytes_:
            row_stride = [kv.stride(-2)] * n
    else:
        kv = list(kv)
        _need(len(kv) == n, "append: one cache per table")
        owner, kv_base = _c_array("Q", [_addr(k) for k in kv], n)
        keep.append(owner)
        if row_stride is not None:
            row_stride = list(row_stride)
            _need(len(row_stride) == n, "append: one row_stride per table")
        # a tensor's own bytes are the cache's limit; an address has none
        kv_rows = _limits([_rows_in(k, row_bytes(row_format), None if row_stride is None else row_stride[i]) for i, k in enumerate(kv)], kv_rows)
    strides, strides_at = _c_array("Q", row_stride, n)
    limits, limits_at = _c_array("I", kv_rows, n)
    tables, tables_at = _c_array("I", _tables, n)
    if want_values and values is None:
        values = _output((n, n_tokens, LATENT_DIMS + ROPE_DIMS), torch.bfloat16, device, stream)
    block = _packed(
        _APPEND, "append",
        n, n_tokens, row_format, kind, tables_at or 0, latent.data_ptr(), rope_part.data_ptr(), *_steps(latent, size, 2), *_steps(rope_part, size, 2),
        _tensor_at(positions, "append: positions", torch.int32, here, device),
        0 if rows is None else _tensor_at(rows, "append: rows", torch.int32, here, device), kv_base, at, table_step, strides_at or 0, limits_at or 0,
        0 if rope is None else rope.address,
        0 if values is None else _tensor_at(values, "append: values", torch.bfloat16, (n, n_tokens, LATENT_DIMS + ROPE_DIMS), device),
        0 if status is None else _status_word(status))
    rc = _append_fn(None if _ctx is None else _ctx._h, block, stream)
    if rc != OK:
        _check(rc, "avsg_append")
    return values


def attend(q, buffer, slots, *, row_format: int, scale: float, out=None, lse=None, want_lse: bool = False, softcap: float = 0.0, ids=None,
           positions=None, spans=None, slopes=None, rope: Optional[Rope] = None, status=None, stream=None, _ctx=None, _tables=None):
    """avsg_attend: the sparse attention that reads the rows of `buffer` through the slot table of avsg_step.

    q: bf16 CUDA tensor [n, n_tokens, heads, 576]; buffer: uint8 [n, slots per table, row bytes] (avsg_step_noalloc's state;
    Context.attend reads the context's own); slots int32 [n, n_tokens, topk], negative = padding.  Optional: softcap; ids int32
    like slots with spans int32 [n, n_tokens, 2] (the ids [begin, end) that a query may see) and slopes fp32 [heads] with positions
    int32 [n, n_tokens] (a bias of slope * (id - position)); rope with positions: q's last 64 numbers are rotated here.  stream: a torch stream
    or a handle (default: the current one of q's device), on which outputs that are not given are allocated.
    Returns bf16 [n, n_tokens, heads, 512], and with want_lse the fp32 logarithms [n, n_tokens, heads] too.  For serving: a result has no
    gradient, also where q requires one."""
    import torch
    if _attend_fn is None:
        _rows_functions()
    if _tensor_calls:
        done = _tensor_calls.attend(
            None if _ctx is None else _ctx._cell.value or None, _tables, q, buffer, slots, row_format, scale, out, lse, bool(want_lse), softcap, ids,
            positions, spans, slopes, None if rope is None else rope.address, None if status is None else _status_word(status), _stream_number(stream))
        if done is not NotImplemented:
            if done[0] != OK:
                _check(done[0], "avsg_attend")
            return done[1]
    device, shape, bf16, int32 = q.get_device(), q.shape, torch.bfloat16, torch.int32
    if device < 0 or q.dtype is not bf16 or len(shape) != 4 or shape[3] != LATENT_DIMS + ROPE_DIMS or q.stride(3) != 1:
        raise AvsgError(EINVAL, "attend: q is a bf16 CUDA tensor [n, n_tokens, heads, 576] with its last numbers side by side")
    stream = _stream_of(stream, device)
    n, n_tokens, heads, _ = shape
    _need(slots.dim() == 3, "attend: slots is [n, n_tokens, topk]")
    topk = slots.shape[2]
    ids_like, here = (n, n_tokens, topk), (n, n_tokens)
    tables_at = rows_at = rows = row_step = 0
    if _ctx is None:
        held = buffer.shape
        if buffer.get_device() != device or buffer.dtype is not torch.uint8 or len(held) != 3 or held[0] != n or held[2] != row_bytes(row_format) or \
                buffer.stride(2) != 1 or (n > 1 and held[1] > 1 and buffer.stride(0) != buffer.stride(1) * held[1]):
            raise AvsgError(EINVAL, "attend: buffer is a uint8 tensor [n, slots, row bytes] on q's device, its tables one behind another")
        # (an expanded row has a stride of 0, which the library would take for the bytes of a row)
        if (held[1] > 1 and buffer.stride(1) < held[2]) or (n > 1 and buffer.stride(0) < held[2]):
            raise AvsgError(EINVAL, "attend: rows of buffer share their place")
        # (tables of one row are as far apart as their rows; the stride between rows says nothing then)
        rows_at, rows, row_step = buffer.data_ptr(), held[1], (buffer.stride(1) if held[1] > 1 else buffer.stride(0) if n > 1 else 0)
    else:
        _need(len(_tables) == n, "attend: one table per block of queries")
        owner, tables_at = _c_array("I", _tables, n)
    if out is None:
        out = _output((n, n_tokens, heads, LATENT_DIMS), bf16, device, stream)
        out_steps = (1024 * heads * n_tokens, 1024 * heads, 1024)
    else:
        if out.dtype is not bf16 or out.get_device() != device or out.shape != (n, n_tokens, heads, LATENT_DIMS) or out.stride(3) != 1:
            raise AvsgError(EINVAL, "attend: out is a bf16 tensor [n, n_tokens, heads, 512] on q's device with its last numbers side by side")
        out_steps = _steps(out, 2, 3)
    if want_lse and lse is None:
        lse = _output((n, n_tokens, heads), torch.float32, device, stream)
    block = _packed(
        _ATTEND, "attend",
        n, n_tokens, topk, heads, row_format, rows, row_step, tables_at, rows_at, _tensor_at(slots, "attend: slots", int32, ids_like, device),
        q.data_ptr(), *_steps(q, 2, 3), out.data_ptr(), *out_steps,
        0 if lse is None else _tensor_at(lse, "attend: lse", torch.float32, (n, n_tokens, heads), device), scale, softcap,
        0 if ids is None else _tensor_at(ids, "attend: ids", int32, ids_like, device),
        0 if positions is None else _tensor_at(positions, "attend: positions", int32, here, device),
        0 if spans is None else _tensor_at(spans, "attend: spans", int32, (n, n_tokens, 2), device),
        0 if slopes is None else _tensor_at(slopes, "attend: slopes", torch.float32, (heads,), device),
        0 if rope is None else rope.address, 0 if status is None else _status_word(status))
    rc = _attend_fn(None if _ctx is None else _ctx._h, block, stream)
    if rc != OK:
        _check(rc, "avsg_attend")
    return out if lse is None else (out, lse)

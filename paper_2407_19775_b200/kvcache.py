"""ctypes binding of the 4-bit key/value cache of ``libbq.so`` (the ``bqkv_*`` calls of ``include/bq4.h``), taking torch
tensors.  Argument marshalling only: every step runs in the library's kernels.
"""
from __future__ import annotations

import ctypes
import math

import torch

from .binding import _DT, BqError, Scratch, _check, _dev, _raw_stream, lib
from .bq4 import Codebook4

PATH_AUTO, PATH_GENERAL, PATH_ROWS, PATH_TILES = 0, 1, 2, 3
SYMBOLS = ("bqkv_append", "bqkv_read", "bqkv_attend_workspace", "bqkv_attend", "bqkv_kernel_status", "bqkv_evict_workspace", "bqkv_evict")
kHeader = 1024                                                       # bytes of an attention workspace that start as zeros
_16 = (torch.float16, torch.bfloat16)
_typed = False


class _Cache(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("k_codes", "v_codes", "k_scale", "v_scale", "table", "lens")] +
                [(n, ctypes.c_int) for n in ("n_pages", "kv_heads", "page", "head_dim", "block", "n_seq", "max_pages", "table_stride")])


def _lib() -> ctypes.CDLL:
    global _typed
    L = lib()
    if not _typed:
        vp, sz, i32, i64, f32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_int64, ctypes.c_float
        c = ctypes.POINTER(_Cache)
        L.bqkv_append.argtypes = [c, vp, vp, vp, i32, i64, i64, vp, i32, vp]
        L.bqkv_read.argtypes = [c, vp, vp, i32, vp, vp, i32, vp]
        L.bqkv_attend_workspace.argtypes = [c, i32, i32, i32, i32, i32, ctypes.POINTER(sz)]
        L.bqkv_attend.argtypes = [c, vp, vp, i32, i64, vp, i32, i32, i32, i32, f32, vp, i64, vp, vp, sz, i32, vp]
        L.bqkv_kernel_status.argtypes = [vp, ctypes.POINTER(i32)]
        L.bqkv_evict_workspace.argtypes = [c, i32, ctypes.POINTER(sz)]
        L.bqkv_evict.argtypes = [c, vp, i64, i32, i32, i32, vp, sz, vp]
        _typed = True
    return L


def _rows_of(x: torch.Tensor, name: str, device, dim: int, dtype=None):
    """(rows, heads, elements between rows) of [rows, heads, dim]; the heads of a row have to be contiguous."""
    if x.device != device:
        raise BqError(f"{name} must be a CUDA tensor on the cache's device")
    dt = x.dtype
    if dt not in _16 or (dtype is not None and dt != dtype):
        raise BqError(f"{name} must be float16 or bfloat16" + ("" if dtype is None else f" ({dtype})"))
    shape, stride = x.shape, x.stride()
    if len(shape) != 3 or shape[2] != dim:
        raise BqError(f"{name} must be [rows, heads, {dim}]")
    if shape[0] > 0 and (stride[2] != 1 or (shape[1] > 1 and stride[1] != dim)):
        raise BqError(f"the heads of a row of {name} must be contiguous")
    return shape[0], shape[1], stride[0]


class KvCache4:
    """A paged key/value cache held in 4 bits (``bqkv_cache``) over tensors of the caller.

    k_codes, v_codes: uint8 [pages, kv_heads, page, head_dim / 2]; k_scale, v_scale: bfloat16 [pages, kv_heads, page,
    head_dim / block]; table: int32 [sequences, pages of a sequence] (rows may be strided); lens: int32 [sequences], the
    slots in use, the rows of the present call included.  Rows of table that overlap (an expanded one) are refused.  The caller owns table and lens and may change them between calls.
    Work runs on the current stream of the cache's device."""

    def __init__(self, k_codes: torch.Tensor, v_codes: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor, table: torch.Tensor,
                 lens: torch.Tensor, codebook: Codebook4):
        for name, t, dt in (("k_codes", k_codes, torch.uint8), ("v_codes", v_codes, torch.uint8), ("k_scale", k_scale, torch.bfloat16),
                            ("v_scale", v_scale, torch.bfloat16)):
            _dev(t, name)
            if t.dtype != dt or t.dim() != 4 or t.shape[:3] != k_codes.shape[:3] or t.device != k_codes.device:
                raise BqError(f"{name} must be {dt} [pages, kv_heads, page, ...] like the other pools")
        if v_codes.shape != k_codes.shape or v_scale.shape != k_scale.shape:
            raise BqError("the pools of keys and values must have the same shapes")
        n_pages, self.kv_heads, self.page, half = k_codes.shape
        self.head_dim = 2 * half
        if k_scale.shape[3] < 1 or self.head_dim % k_scale.shape[3] != 0:
            raise BqError("the scales of a row must divide head_dim")
        self.block = self.head_dim // k_scale.shape[3]
        if not table.is_cuda or table.dtype != torch.int32 or table.dim() != 2 or table.device != k_codes.device or (table.shape[1] > 1 and table.stride(1) != 1):
            raise BqError("table must be a CUDA int32 [sequences, pages] tensor with contiguous rows")
        if table.shape[0] > 1 and table.stride(0) < table.shape[1]:
            raise BqError("the rows of table must not overlap")
        _dev(lens, "lens")
        if lens.dtype != torch.int32 or lens.shape != (table.shape[0],) or lens.device != k_codes.device:
            raise BqError("lens must be a CUDA int32 tensor of one entry per sequence")
        self.device = k_codes.device
        self._index = self.device.index
        self.n_seq, self.max_pages = table.shape
        self.capacity = self.max_pages * self.page
        self.table, self.lens, self.codebook = table, lens, codebook
        self._pools = (k_codes, v_codes, k_scale, v_scale)
        self._c = _Cache(*(t.data_ptr() for t in self._pools), table.data_ptr(), lens.data_ptr(), n_pages, self.kv_heads, self.page, self.head_dim,
                         self.block, self.n_seq, self.max_pages, table.stride(0) if self.n_seq > 1 else self.max_pages)
        self._scratch = Scratch(self.device, kHeader)
        self._need = {}
        self._sm = 1.0 / math.sqrt(self.head_dim)
        self._ref = ctypes.byref(self._c)

    @classmethod
    def empty(cls, sequences: int, max_len: int, kv_heads: int, head_dim: int, block: int, codebook: Codebook4, page: int = 64, device=None) -> "KvCache4":
        """A cache with pages of its own for every sequence, all of them empty."""
        dev = torch.device("cuda") if device is None else torch.device(device)
        width = (max_len + page - 1) // page
        codes = [torch.zeros((sequences * width, kv_heads, page, head_dim // 2), dtype=torch.uint8, device=dev) for _ in range(2)]
        scale = [torch.zeros((sequences * width, kv_heads, page, head_dim // block), dtype=torch.bfloat16, device=dev) for _ in range(2)]
        table = torch.arange(sequences * width, dtype=torch.int32, device=dev).view(sequences, width)
        return cls(*codes, *scale, table, torch.zeros(sequences, dtype=torch.int32, device=dev), codebook)

    def _starts(self, starts, n_rows):
        if starts is None:
            if n_rows != self.n_seq:
                raise BqError(f"without starts there is one row per sequence ({self.n_seq}), not {n_rows}")
            return None
        if starts.device != self.device or starts.dtype != torch.int32 or starts.shape != (self.n_seq + 1,) or not starts.is_contiguous():
            raise BqError("starts must be a contiguous CUDA int32 tensor of one entry per sequence and one more, on the cache's device")
        return starts.data_ptr()

    def _run(self, call, what: str, *args) -> None:
        """The call with the cache's device current, on its current stream (the last argument)."""
        if torch.cuda.current_device() == self._index:
            rc = call(self._ref, *args, _raw_stream(self._index))
        else:
            with torch.cuda.device(self.device):
                rc = call(self._ref, *args, _raw_stream(self._index))
        if rc != 0:
            _check(rc, what)

    def append(self, k: torch.Tensor, v: torch.Tensor, starts: torch.Tensor | None = None) -> None:
        """``bqkv_append``: k, v [rows, kv_heads, head_dim] into the last slots of their sequences."""
        n, heads, ks = _rows_of(k, "k", self.device, self.head_dim)
        nv, heads_v, vs = _rows_of(v, "v", self.device, self.head_dim, k.dtype)
        if nv != n or heads != self.kv_heads or heads_v != heads:
            raise BqError(f"k and v must both be [rows, {self.kv_heads}, {self.head_dim}]")
        self._run(_lib().bqkv_append, "bqkv_append", self.codebook.handle, k.data_ptr(), v.data_ptr(), _DT[k.dtype], ks, vs, self._starts(starts, n), n)

    def read(self, starts: torch.Tensor | None, n_rows: int, dtype: torch.dtype):
        """``bqkv_read``: the values (k, v) of the sequences' last rows, [n_rows, kv_heads, head_dim] of ``dtype``."""
        if dtype not in _16:
            raise BqError("dtype must be float16 or bfloat16")
        k = torch.empty((n_rows, self.kv_heads, self.head_dim), dtype=dtype, device=self.device)
        v = torch.empty_like(k)
        self._run(_lib().bqkv_read, "bqkv_read", self.codebook.handle, self._starts(starts, n_rows), n_rows, k.data_ptr(), v.data_ptr(), _DT[dtype])
        return k, v

    def attend(self, q: torch.Tensor, starts: torch.Tensor | None = None, max_new: int = 1, max_len: int = 0, sm_scale: float | None = None,
               weights: torch.Tensor | None = None, out: torch.Tensor | None = None, path: int = PATH_AUTO) -> torch.Tensor:
        """``bqkv_attend``: q [rows, q_heads, head_dim] -> the same shape.  ``max_new`` and ``max_len`` bound (for the launch
        sizes) the rows of a sequence and lens; sm_scale defaults to 1 / sqrt(head_dim).  ``weights`` (float32 [sequences,
        kv_heads, slots]) is added to in place."""
        n, heads, qs = _rows_of(q, "q", self.device, self.head_dim)
        if heads < 1 or heads % self.kv_heads != 0:
            raise BqError(f"q must have a multiple of {self.kv_heads} heads")
        if out is None:
            out = torch.empty((n, heads, self.head_dim), dtype=q.dtype, device=self.device)
        elif out.shape != q.shape or out.device != self.device or out.dtype != q.dtype or not out.is_contiguous():
            raise BqError("out must be contiguous, of q's shape, type and device")
        if weights is not None:
            self._check_weights(weights)
        L = _lib()
        sizes = (n, heads, max_new, max_len, 0 if weights is None else 2 if path == PATH_ROWS else 1)
        need = self._need.get(sizes)
        if need is None:
            size = ctypes.c_size_t()
            _check(L.bqkv_attend_workspace(self._ref, *sizes, ctypes.byref(size)), "bqkv_attend_workspace")
            need = self._need[sizes] = size.value
            if len(self._need) > 1024:                                # ragged batches: sizes keep changing
                self._need.clear()
        held, ws, ws_bytes = self._scratch.take("attend", need)
        self._run(L.bqkv_attend, "bqkv_attend", self.codebook.handle, q.data_ptr(), _DT[q.dtype], qs, self._starts(starts, n), n, heads, max_new, max_len,
                  self._sm if sm_scale is None else sm_scale, None if weights is None else weights.data_ptr(), 0 if weights is None else weights.shape[2],
                  out.data_ptr(), ws, ws_bytes, path)
        return out

    def kernel_status(self) -> int:
        """``bqkv_kernel_status`` over the cache's workspaces: non-zero when a kernel gave up on a bounded wait (reads and clears).
        Workspaces that belong to a graph (captured on a stream that no call had used before) are not among them."""
        found = 0
        for _, address, _ in self._scratch.all("attend"):
            st = ctypes.c_int(0)
            with torch.cuda.device(self.device):
                _check(_lib().bqkv_kernel_status(address, ctypes.byref(st)), "bqkv_kernel_status")
            found = found or int(st.value)
        return found

    def _check_weights(self, weights):
        if (weights.device != self.device or weights.dtype != torch.float32 or weights.dim() != 3 or weights.shape[0] != self.n_seq or
                weights.shape[1] != self.kv_heads or not weights.is_contiguous()):
            raise BqError("weights must be contiguous float32 [sequences, kv_heads, slots] on the cache's device")

    def evict(self, weights: torch.Tensor, budget: int, sinks: int = 0, recent: int = 0) -> None:
        """``bqkv_evict``: every sequence down to ``budget`` slots by accumulated weight; updates the pools, weights and lens."""
        if weights is None:
            raise BqError("evict needs the accumulated weights")
        self._check_weights(weights)
        L = _lib()
        need = self._need.get(budget)
        if need is None:
            size = ctypes.c_size_t()
            _check(L.bqkv_evict_workspace(self._ref, budget, ctypes.byref(size)), "bqkv_evict_workspace")
            need = self._need[budget] = size.value
        held, ws, ws_bytes = self._scratch.take("evict", need)
        self._run(L.bqkv_evict, "bqkv_evict", weights.data_ptr(), weights.shape[2], budget, sinks, recent, ws, ws_bytes)

"""ctypes binding of the 4-bit key/value cache of ``libbq.so`` (the ``bqkv_*`` calls of ``include/bq4.h``), taking torch
tensors.  Argument marshalling only: every step runs in the library's kernels.
"""
from __future__ import annotations

import ctypes
import math

import torch

from .binding import _DT, BqError, _check, _dev, _stream, lib
from .bq4 import Codebook4

PATH_AUTO, PATH_GENERAL, PATH_ROWS, PATH_TILES = 0, 1, 2, 3
SYMBOLS = ("bqkv_append", "bqkv_read", "bqkv_attend_workspace", "bqkv_attend", "bqkv_kernel_status", "bqkv_evict_workspace", "bqkv_evict")
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


def _row_stride(x: torch.Tensor, name: str, device, heads: int, dim: int, dtype=None) -> int:
    """Elements between the rows of [rows, heads, dim]; the heads of a row have to be contiguous."""
    if x.device != device:
        raise BqError(f"{name} must be a CUDA tensor on the cache's device")
    if x.dtype not in _16 or (dtype is not None and x.dtype != dtype):
        raise BqError(f"{name} must be float16 or bfloat16" + ("" if dtype is None else f" ({dtype})"))
    if x.dim() != 3 or x.shape[1] != heads or x.shape[2] != dim:
        raise BqError(f"{name} must be [rows, {heads}, {dim}]")
    if x.shape[0] > 0 and ((dim > 1 and x.stride(2) != 1) or (heads > 1 and x.stride(1) != dim)):
        raise BqError(f"the heads of a row of {name} must be contiguous")
    return x.stride(0)


class KvCache4:
    """A paged key/value cache held in 4 bits (``bqkv_cache``) over tensors of the caller.

    k_codes, v_codes: uint8 [pages, kv_heads, page, head_dim / 2]; k_scale, v_scale: bfloat16 [pages, kv_heads, page,
    head_dim / block]; table: int32 [sequences, pages of a sequence] (rows may be strided); lens: int32 [sequences], the
    slots in use, the rows of the present call included.  The caller owns table and lens and may change them between calls.
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
        _dev(lens, "lens")
        if lens.dtype != torch.int32 or lens.shape != (table.shape[0],) or lens.device != k_codes.device:
            raise BqError("lens must be a CUDA int32 tensor of one entry per sequence")
        self.device = k_codes.device
        self.n_seq, self.max_pages = table.shape
        self.capacity = self.max_pages * self.page
        self.table, self.lens, self.codebook = table, lens, codebook
        self._pools = (k_codes, v_codes, k_scale, v_scale)
        self._c = _Cache(*(t.data_ptr() for t in self._pools), table.data_ptr(), lens.data_ptr(), n_pages, self.kv_heads, self.page, self.head_dim,
                         self.block, self.n_seq, self.max_pages, max(table.stride(0), self.max_pages))
        self._ws = {}

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
        _dev(starts, "starts")
        if starts.device != self.device or starts.dtype != torch.int32 or starts.shape != (self.n_seq + 1,):
            raise BqError("starts must be a CUDA int32 tensor of one entry per sequence and one more")
        return starts.data_ptr()

    def _workspace(self, key: str, nbytes: int) -> torch.Tensor:
        """One scratch buffer per use and stream, kept as long as the cache: calls on different streams do not share one."""
        at = (key, torch.cuda.current_stream(self.device).cuda_stream)
        ws = self._ws.get(at)
        if ws is None or ws.numel() < nbytes + 256:
            ws = self._ws[at] = torch.zeros(nbytes + 256, dtype=torch.uint8, device=self.device)
        off = (-ws.data_ptr()) % 256
        return ws[off:off + nbytes]

    def append(self, k: torch.Tensor, v: torch.Tensor, starts: torch.Tensor | None = None) -> None:
        """``bqkv_append``: k, v [rows, kv_heads, head_dim] into the last slots of their sequences."""
        ks, vs = _row_stride(k, "k", self.device, self.kv_heads, self.head_dim), _row_stride(v, "v", self.device, self.kv_heads, self.head_dim, k.dtype)
        if v.shape != k.shape:
            raise BqError("k and v must have the same shape")
        with torch.cuda.device(self.device):
            rc = _lib().bqkv_append(ctypes.byref(self._c), self.codebook.handle, k.data_ptr(), v.data_ptr(), _DT[k.dtype], ks, vs,
                                    self._starts(starts, k.shape[0]), k.shape[0], _stream(k))
        _check(rc, "bqkv_append")

    def read(self, starts: torch.Tensor | None, n_rows: int, dtype: torch.dtype):
        """``bqkv_read``: the values (k, v) of the sequences' last rows, [n_rows, kv_heads, head_dim] of ``dtype``."""
        if dtype not in _16:
            raise BqError("dtype must be float16 or bfloat16")
        k, v = (torch.empty((n_rows, self.kv_heads, self.head_dim), dtype=dtype, device=self.device) for _ in range(2))
        with torch.cuda.device(self.device):
            rc = _lib().bqkv_read(ctypes.byref(self._c), self.codebook.handle, self._starts(starts, n_rows), n_rows, k.data_ptr(), v.data_ptr(),
                                  _DT[dtype], _stream(k))
        _check(rc, "bqkv_read")
        return k, v

    def attend(self, q: torch.Tensor, starts: torch.Tensor | None = None, max_new: int = 1, max_len: int = 0, sm_scale: float | None = None,
               weights: torch.Tensor | None = None, out: torch.Tensor | None = None, path: int = PATH_AUTO) -> torch.Tensor:
        """``bqkv_attend``: q [rows, q_heads, head_dim] -> the same shape.  ``max_new`` and ``max_len`` bound (for the launch
        sizes) the rows of a sequence and lens; sm_scale defaults to 1 / sqrt(head_dim).  ``weights`` (float32 [sequences,
        kv_heads, slots]) is added to in place."""
        if q.dim() != 3 or q.shape[1] < 1 or q.shape[1] % self.kv_heads != 0:
            raise BqError(f"q must be [rows, a multiple of {self.kv_heads} heads, {self.head_dim}]")
        n, heads = q.shape[:2]
        qs = _row_stride(q, "q", self.device, heads, self.head_dim)
        if out is None:
            out = torch.empty((n, heads, self.head_dim), dtype=q.dtype, device=q.device)
        elif out.shape != q.shape or out.device != q.device or out.dtype != q.dtype:
            raise BqError("out must have q's shape and type")
        self._check_weights(weights)
        L = _lib()
        need = ctypes.c_size_t()
        _check(L.bqkv_attend_workspace(ctypes.byref(self._c), n, heads, max_new, max_len, weights is not None, ctypes.byref(need)), "bqkv_attend_workspace")
        with torch.cuda.device(self.device):
            ws = self._workspace("attend", need.value)
            rc = L.bqkv_attend(ctypes.byref(self._c), self.codebook.handle, q.data_ptr(), _DT[q.dtype], qs, self._starts(starts, n), n, heads, max_new, max_len,
                               1.0 / math.sqrt(self.head_dim) if sm_scale is None else sm_scale, None if weights is None else weights.data_ptr(),
                               0 if weights is None else weights.shape[2], _dev(out, "out").data_ptr(), ws.data_ptr(), ws.numel(), path, _stream(q))
        _check(rc, "bqkv_attend")
        return out

    def kernel_status(self) -> int:
        """``bqkv_kernel_status`` over the cache's workspaces: non-zero when a kernel gave up on a bounded wait (reads and clears)."""
        found = 0
        for (key, _), ws in self._ws.items():
            if key == "attend":
                st = ctypes.c_int(0)
                with torch.cuda.device(self.device):
                    _check(_lib().bqkv_kernel_status(ws.data_ptr() + (-ws.data_ptr()) % 256, ctypes.byref(st)), "bqkv_kernel_status")
                found = found or int(st.value)
        return found

    def _check_weights(self, weights):
        if weights is None:
            return
        _dev(weights, "weights")
        if weights.device != self.device or weights.dtype != torch.float32 or weights.dim() != 3 or weights.shape[:2] != (self.n_seq, self.kv_heads):
            raise BqError("weights must be float32 [sequences, kv_heads, slots]")

    def evict(self, weights: torch.Tensor, budget: int, sinks: int = 0, recent: int = 0) -> None:
        """``bqkv_evict``: every sequence down to ``budget`` slots by accumulated weight; updates the pools, weights and lens."""
        if weights is None:
            raise BqError("evict needs the accumulated weights")
        self._check_weights(weights)
        L = _lib()
        need = ctypes.c_size_t()
        _check(L.bqkv_evict_workspace(ctypes.byref(self._c), budget, ctypes.byref(need)), "bqkv_evict_workspace")
        with torch.cuda.device(self.device):
            ws = self._workspace("evict", need.value)
            rc = L.bqkv_evict(ctypes.byref(self._c), weights.data_ptr(), weights.shape[2], budget, sinks, recent, ws.data_ptr(), ws.numel(), _stream(weights))
        _check(rc, "bqkv_evict")

"""ctypes binding of the mixed-matrix-decomposition calls of ``libbq.so`` (``include/mmd.h``),
taking torch tensors.  Argument marshalling only: every step runs in the library's kernels.
"""
from __future__ import annotations

import ctypes

import numpy as np
import torch

from .binding import _DT, BqError, Scratch, _check, _dev, _stream, lib

PATH_AUTO, PATH_GENERAL, PATH_TENSOR, PATH_TENSOR_TILE, PATH_TENSOR_SOLO, PATH_TENSOR_STREAMK = 0, 1, 2, 3, 4, 5
_TORCH_OF = {0: torch.float32, 1: torch.float16, 2: torch.bfloat16}

SYMBOLS = ("mmd_side_columns", "mmd_select_features", "mmd_rowquant", "mmd_decompose", "mmd_free", "mmd_weights_view",
           "mmd_workspace_layout", "mmd_linear", "mmd_linear_static", "mmd_kernel_status", "mmd_selftest_bounded_wait", "mmd_workspace_bytes_streamk",
           "mmd_norm_rowquant", "mmd_norm_linear", "mmd_adapted_workspace", "mmd_linear_adapted", "mmd_norm_linear_adapted")
SELFTEST_CODE = 77
STATIC_SCRATCH_BYTES = 4 << 20
MAX_RANK = 256
_typed = False


class _Adapters(ctypes.Structure):
    _fields_ = [("a", ctypes.c_void_p), ("b", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("count", ctypes.c_int), ("rank", ctypes.c_int)]


def _lib() -> ctypes.CDLL:
    global _typed
    L = lib()
    if not _typed:
        vp, sz, i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
        L.mmd_side_columns.argtypes = [i32]
        L.mmd_select_features.argtypes = [vp, i32, ctypes.c_float, vp, ctypes.POINTER(i32)]
        L.mmd_rowquant.argtypes = [vp, i32, i32, i32, vp, i32, vp, vp, vp, vp]
        L.mmd_decompose.argtypes = [vp, i32, i32, i32, vp, i32, vp, ctypes.POINTER(vp)]
        L.mmd_free.argtypes = [vp]
        L.mmd_weights_view.argtypes = [vp] + [ctypes.POINTER(vp)] * 4 + [ctypes.POINTER(i32)] * 4
        L.mmd_workspace_layout.argtypes = [vp, i32, ctypes.POINTER(sz), ctypes.POINTER(sz)]
        L.mmd_workspace_bytes_streamk.argtypes = [vp, i32, ctypes.POINTER(sz)]
        L.mmd_linear.argtypes = [vp, vp, i32, vp, i32, vp, sz, i32, vp]
        L.mmd_linear_static.argtypes = [vp, vp, i32, vp, i32, i32, vp]
        L.mmd_kernel_status.argtypes = [vp, ctypes.POINTER(i32)]
        L.mmd_norm_rowquant.argtypes = [vp, vp, vp, ctypes.c_float, i32, i32, i32, vp, i32, vp, vp, vp, vp, vp]
        L.mmd_norm_linear.argtypes = [vp, vp, vp, vp, ctypes.c_float, i32, vp, vp, i32, vp, sz, i32, vp]
        ad = ctypes.POINTER(_Adapters)
        L.mmd_adapted_workspace.argtypes = [vp, i32, i32, i32, i32, ctypes.POINTER(sz)]
        L.mmd_linear_adapted.argtypes = [vp, ad, vp, vp, i32, vp, i32, vp, i32, vp, sz, i32, vp]
        L.mmd_norm_linear_adapted.argtypes = [vp, ad, vp, vp, i32, vp, vp, vp, ctypes.c_float, i32, vp, vp, i32, vp, sz, i32, vp]
        L.mmd_selftest_bounded_wait.argtypes = [vp, ctypes.c_uint, ctypes.POINTER(i32), vp]
        _typed = True
    return L


def mmd_side_columns(n_features: int) -> int:
    return int(_lib().mmd_side_columns(n_features))


def mmd_select_features(feature_absmax, tau: float) -> np.ndarray:
    """``mmd_select_features`` on a host array of per-feature calibration magnitudes."""
    a = np.ascontiguousarray(feature_absmax, np.float32)
    idx = np.empty(a.size, np.int32)
    count = ctypes.c_int(0)
    _check(_lib().mmd_select_features(a.ctypes.data, a.size, float(tau), idx.ctypes.data, ctypes.byref(count)), "mmd_select_features")
    return idx[:count.value].copy()


def mmd_rowquant(v: torch.Tensor, idx: torch.Tensor | None):
    """``mmd_rowquant``: returns (q int8 [R, K], scale float32 [R], side [R, side columns])."""
    _dev(v, "v")
    R, K = v.shape
    ko = 0 if idx is None else idx.numel()
    q = torch.empty((R, K), dtype=torch.int8, device=v.device)
    scale = torch.empty(R, dtype=torch.float32, device=v.device)
    side = torch.empty((R, mmd_side_columns(ko)), dtype=v.dtype, device=v.device)
    with torch.cuda.device(v.device):
        rc = _lib().mmd_rowquant(v.data_ptr(), _DT[v.dtype], R, K, None if ko == 0 else _dev(idx, "idx").data_ptr(), ko, q.data_ptr(),
                                 scale.data_ptr(), side.data_ptr() if ko else None, _stream(v))
    _check(rc, "mmd_rowquant")
    return q, scale, side


def rowquant_into(v: torch.Tensor, idx: torch.Tensor | None, q: torch.Tensor, scale: torch.Tensor, side: torch.Tensor) -> None:
    """``mmd_rowquant`` into caller-provided outputs."""
    R, K = v.shape
    ko = 0 if idx is None else idx.numel()
    with torch.cuda.device(v.device):
        rc = _lib().mmd_rowquant(_dev(v, "v").data_ptr(), _DT[v.dtype], R, K, None if ko == 0 else idx.data_ptr(), ko, q.data_ptr(),
                                 scale.data_ptr(), side.data_ptr() if ko else None, _stream(v))
    _check(rc, "mmd_rowquant")


def _norm_args(x, gamma, residual, h_out):
    """(h_out, pointers of residual and h_out) after the checks the two norm calls share."""
    _dev(x, "x")
    _dev(gamma, "gamma")
    if x.dim() != 2 or gamma.dtype != x.dtype or gamma.shape != (x.shape[1],) or gamma.device != x.device:
        raise BqError("x must be [rows, K] and gamma [K] of the same element type and device")
    if residual is not None:
        _dev(residual, "residual")
        if residual.dtype != x.dtype or residual.shape != x.shape or residual.device != x.device:
            raise BqError("residual must have x's shape, type and device")
        if h_out is None:
            h_out = torch.empty_like(x)
    if h_out is not None:
        _dev(h_out, "h_out")
        if h_out.dtype != x.dtype or h_out.shape != x.shape or h_out.device != x.device:
            raise BqError("h_out must have x's shape, type and device")
    return h_out, None if residual is None else residual.data_ptr(), None if h_out is None else h_out.data_ptr()


def mmd_norm_rowquant(x: torch.Tensor, gamma: torch.Tensor, eps: float, idx: torch.Tensor | None = None, residual: torch.Tensor | None = None,
                      h_out: torch.Tensor | None = None):
    """``mmd_norm_rowquant``: returns (q int8 [R, K], scale float32 [R], side [R, side columns], h).  Without a residual h is x."""
    h_out, pr, ph = _norm_args(x, gamma, residual, h_out)
    R, K = x.shape
    ko = 0 if idx is None else idx.numel()
    if ko and (idx.dtype != torch.int32 or idx.device != x.device):
        raise BqError("idx must be int32 on x's device")
    q = torch.empty((R, K), dtype=torch.int8, device=x.device)
    scale = torch.empty(R, dtype=torch.float32, device=x.device)
    side = torch.empty((R, mmd_side_columns(ko)), dtype=x.dtype, device=x.device)
    with torch.cuda.device(x.device):
        rc = _lib().mmd_norm_rowquant(x.data_ptr(), pr, gamma.data_ptr(), eps, _DT[x.dtype], R, K, None if ko == 0 else _dev(idx, "idx").data_ptr(), ko, ph,
                                      q.data_ptr(), scale.data_ptr(), side.data_ptr() if ko else None, _stream(x))
    _check(rc, "mmd_norm_rowquant")
    return q, scale, side, x if h_out is None else h_out


def _bytes_of(workspace: torch.Tensor, X: torch.Tensor) -> int:
    if _dev(workspace, "workspace").device != X.device:
        raise BqError("the workspace must be on X's device")
    return workspace.numel() * workspace.element_size()


class Adapters:
    """Low-rank adapters of one decomposed layer (``mmd_adapters``) over tensors of the caller, who may change their contents between
    calls: a [count, rank, K], b [count, N, rank] of the layer's element type, scale float32 [count].  rank: a multiple of 16."""

    def __init__(self, a: torch.Tensor, b: torch.Tensor, scale: torch.Tensor):
        for name, t in (("a", a), ("b", b), ("scale", scale)):
            _dev(t, name)
            if t.device != a.device:
                raise BqError("a, b and scale must be on one device")
        if a.dim() != 3 or b.dim() != 3 or b.shape[0] != a.shape[0] or b.shape[2] != a.shape[1] or a.dtype not in (torch.float16, torch.bfloat16) or b.dtype != a.dtype:
            raise BqError("a must be [adapters, rank, K] and b [adapters, N, rank] of one 16-bit type")
        if scale.dtype != torch.float32 or scale.shape != (a.shape[0],):
            raise BqError("scale must be float32, one for each adapter")
        self.count, self.rank, self.K = a.shape
        self.N = b.shape[1]
        if self.count < 1 or self.rank < 16 or self.rank > MAX_RANK or self.rank % 16 != 0:
            raise BqError(f"the rank must be a multiple of 16 up to {MAX_RANK} (pack() pads)")
        self.dtype, self.device = a.dtype, a.device
        self._tensors = (a, b, scale)
        self._c = _Adapters(a.data_ptr(), b.data_ptr(), scale.data_ptr(), self.count, self.rank)
        self._ref = ctypes.byref(self._c)

    @classmethod
    def pack(cls, pairs, scales) -> "Adapters":
        """From a list of (a [rank, K], b [N, rank]) of any ranks: padded with zeros to the largest one's next multiple of 16."""
        pairs = list(pairs)
        if not pairs or len(pairs) != len(scales):
            raise BqError("as many scales as adapters, one at least")
        if any(x.dim() != 2 or y.dim() != 2 or y.shape[1] != x.shape[0] for x, y in pairs):
            raise BqError("an adapter is a [rank, K] and b [N, rank]")
        rank = (max(max(x.shape[0] for x, _ in pairs), 1) + 15) // 16 * 16
        (K, N), first = (pairs[0][0].shape[1], pairs[0][1].shape[0]), pairs[0][0]
        if any(x.shape[1] != K or y.shape[0] != N or x.dtype != first.dtype or y.dtype != first.dtype for x, y in pairs):
            raise BqError("the adapters must be of one layer and one type")
        a, b = first.new_zeros((len(pairs), rank, K)), first.new_zeros((len(pairs), N, rank))
        for i, (x, y) in enumerate(pairs):
            a[i, :x.shape[0]], b[i, :, :x.shape[0]] = x, y
        return cls(a, b, torch.tensor([float(v) for v in scales], dtype=torch.float32, device=first.device))


class DecomposedLinear:
    """Handle of one decomposed weight matrix (``mmd_decompose``) and its linear layer."""

    def __init__(self, W: torch.Tensor, features):
        _dev(W, "W")
        idx = np.ascontiguousarray(features, np.int32)
        self._h = ctypes.c_void_p()
        self.N, self.K = W.shape
        self.dtype = W.dtype
        self.device = W.device
        with torch.cuda.device(W.device):
            rc = _lib().mmd_decompose(W.data_ptr(), _DT[W.dtype], self.N, self.K, idx.ctypes.data if idx.size else None, idx.size,
                                      _stream(W), ctypes.byref(self._h))
        _check(rc, "mmd_decompose")
        self.n_features = int(idx.size)
        self._scratch = Scratch(self.device)
        self._need = {}

    @property
    def handle(self):
        return self._h

    def _output(self, y_out: torch.Tensor | None, M: int, out_dtype: torch.dtype | None, X: torch.Tensor) -> torch.Tensor:
        """y_out after its checks (the kernels write [M, N] elements from its start on), or a new tensor."""
        if y_out is None:
            return torch.empty((M, self.N), dtype=out_dtype or X.dtype, device=X.device)
        _dev(y_out, "y_out")
        if y_out.numel() < M * self.N or y_out.device != X.device:
            raise BqError(f"y_out must have room for [{M}, {self.N}] on X's device")
        if y_out.dtype not in _DT:
            raise BqError("y_out must be float32, float16 or bfloat16")
        return y_out

    def view(self):
        """(q, scale, side, idx) as torch tensors aliasing the handle's device memory."""
        ptr = [ctypes.c_void_p() for _ in range(4)]
        ints = [ctypes.c_int() for _ in range(4)]
        _check(_lib().mmd_weights_view(self._h, *[ctypes.byref(p) for p in ptr], *[ctypes.byref(i) for i in ints]), "mmd_weights_view")
        N, K, ko, _ = (i.value for i in ints)
        sc = mmd_side_columns(ko)

        def alias(p, shape, dtype):
            n = int(np.prod(shape))
            if n == 0:
                return torch.empty(shape, dtype=dtype, device=self.device)
            nbytes = n * torch.empty((), dtype=dtype).element_size()
            iface = {"shape": (nbytes,), "typestr": "|u1", "data": (p.value, False), "version": 3}
            holder = type("DevMem", (), {"__cuda_array_interface__": iface})()
            return torch.as_tensor(holder, device=self.device).view(dtype).view(shape)

        return (alias(ptr[0], (N, K), torch.int8), alias(ptr[1], (N,), torch.float32), alias(ptr[2], (N, sc), self.dtype),
                alias(ptr[3], (ko,), torch.int32))

    def workspace_layout(self, M: int):
        offs = (ctypes.c_size_t * 3)()
        total = ctypes.c_size_t()
        _check(_lib().mmd_workspace_layout(self._h, M, offs, ctypes.byref(total)), "mmd_workspace_layout")
        return tuple(int(o) for o in offs), int(total.value)

    def workspace_bytes(self, M: int) -> int:
        """``mmd_workspace_bytes_streamk``: the workspace size that lets decode-size calls take the stream-K kernel."""
        total = ctypes.c_size_t()
        _check(_lib().mmd_workspace_bytes_streamk(self._h, M, ctypes.byref(total)), "mmd_workspace_bytes_streamk")
        return int(total.value)

    def workspace(self, M: int, streamk: bool = False) -> torch.Tensor:
        """A workspace for M rows (cached, of the current stream); with ``streamk`` also the room the stream-K kernel's slots need."""
        total = self.workspace_bytes(M) if streamk else self.workspace_layout(M)[1]
        buf, address, _ = self._scratch.take("rows", total)
        off = address - buf.data_ptr()
        return buf[off:off + total]

    def check_adapters(self, adapters: Adapters) -> None:
        """Refuses adapters of another layer."""
        if adapters.device != self.device or adapters.dtype != self.dtype or (adapters.K, adapters.N) != (self.K, self.N):
            raise BqError(f"the adapters must be of a {self.K} -> {self.N} layer of {self.dtype} on its device")

    def check_ids(self, ids: torch.Tensor, starts: torch.Tensor | None, M: int) -> int:
        """Refuses what a call of M rows with adapters cannot take as the sequences' adapters and rows; the number of sequences."""
        if ids is None or ids.device != self.device or ids.dtype != torch.int32 or ids.dim() != 1 or not ids.is_contiguous() or ids.shape[0] < 1:
            raise BqError("ids must be a contiguous CUDA int32 tensor, the adapter of every sequence, on the layer's device")
        n_seq = ids.shape[0]
        if starts is None:
            if n_seq != M:
                raise BqError(f"without starts there is one row per sequence ({n_seq}), not {M}")
        elif starts.device != self.device or starts.dtype != torch.int32 or starts.shape != (n_seq + 1,) or not starts.is_contiguous():
            raise BqError("starts must be a contiguous CUDA int32 tensor of one entry per sequence and one more, on the layer's device")
        return n_seq

    def _adapted(self, X: torch.Tensor, adapters: Adapters, ids: torch.Tensor, starts: torch.Tensor | None,
                 workspace: torch.Tensor | None, path: int, y_out: torch.Tensor):
        """(arguments in front of X, workspace address and bytes, what keeps it) of a call with adapters, after its checks."""
        self.check_adapters(adapters)
        if X.device != self.device:
            raise BqError("X must be on the layer's device")
        M = X.shape[0]
        n_seq = self.check_ids(ids, starts, M)
        if workspace is None:
            if path == PATH_AUTO and y_out.data_ptr() % 16 != 0:
                path = PATH_GENERAL
            at = (M, n_seq, adapters.rank, path)
            need = self._need.get(at)
            if need is None:
                if len(self._need) > 1024:
                    self._need.clear()
                size = ctypes.c_size_t()
                _check(_lib().mmd_adapted_workspace(self._h, M, n_seq, adapters.rank, path, ctypes.byref(size)), "mmd_adapted_workspace")
                need = self._need[at] = size.value
            held, ws, ws_bytes = self._scratch.take("adapted", need)
        else:
            held, ws, ws_bytes = workspace, workspace.data_ptr(), _bytes_of(workspace, X)
        return (self._h, adapters._ref, ids.data_ptr(), None if starts is None else starts.data_ptr(), n_seq), ws, ws_bytes, held

    def linear(self, X: torch.Tensor, out_dtype: torch.dtype | None = None, path: int = PATH_AUTO, y_out: torch.Tensor | None = None,
               workspace: torch.Tensor | None = None, adapters: Adapters | None = None, ids: torch.Tensor | None = None,
               starts: torch.Tensor | None = None) -> torch.Tensor:
        """``mmd_linear``: Y = X W^T through the decomposition.  With ``adapters`` (``mmd_linear_adapted``) the rows of sequence s, starts[s] ..
        starts[s + 1] - 1 (None: one each), also go through adapter ids[s] (int32; -1: none)."""
        _dev(X, "X")
        if X.dtype != self.dtype or X.dim() != 2 or X.shape[1] != self.K:
            raise BqError("X must be [M, K] of the weights' element type")
        M = X.shape[0]
        if adapters is not None:
            y_out = self._output(y_out, M, out_dtype, X)
            who, ws, ws_bytes, held = self._adapted(X, adapters, ids, starts, workspace, path, y_out)
            self._run(_lib().mmd_linear_adapted, "mmd_linear_adapted", *who, X.data_ptr(), M, y_out.data_ptr(), _DT[y_out.dtype], ws, ws_bytes, path, _stream(X))
            return y_out
        if ids is not None or starts is not None:
            raise BqError("ids and starts without adapters")
        if workspace is not None:
            held, ws, ws_bytes = workspace, workspace.data_ptr(), _bytes_of(workspace, X)
        elif path == PATH_TENSOR_STREAMK:
            held, ws, ws_bytes = self._scratch.take("rows", self.workspace_bytes(M))
        else:
            held, ws, ws_bytes = self._rows_scratch(M)
        y_out = self._output(y_out, M, out_dtype, X)
        with torch.cuda.device(X.device):
            rc = _lib().mmd_linear(self._h, X.data_ptr(), M, y_out.data_ptr(), _DT[y_out.dtype], ws, ws_bytes, path, _stream(X))
        _check(rc, "mmd_linear")
        return y_out

    def _run(self, call, what: str, *args) -> None:
        """The call with the layer's device current."""
        if torch.cuda.current_device() == self.device.index:
            rc = call(*args)
        else:
            with torch.cuda.device(self.device):
                rc = call(*args)
        if rc != 0:
            _check(rc, what)

    def norm_linear(self, X: torch.Tensor, gamma: torch.Tensor, eps: float, residual: torch.Tensor | None = None, out_dtype: torch.dtype | None = None,
                    path: int = PATH_AUTO, h_out: torch.Tensor | None = None, y_out: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                    adapters: Adapters | None = None, ids: torch.Tensor | None = None, starts: torch.Tensor | None = None):
        """``mmd_norm_linear``: (Y, h) with h = X + residual (X itself without one) and Y = rms_norm(h) * gamma through the layer; ``adapters``,
        ``ids`` and ``starts`` as in linear (``mmd_norm_linear_adapted``)."""
        if X.dtype != self.dtype or X.dim() != 2 or X.shape[1] != self.K:
            raise BqError("X must be [M, K] of the weights' element type")
        h_out, pr, ph = _norm_args(X, gamma, residual, h_out)
        M = X.shape[0]
        if adapters is None and (ids is not None or starts is not None):
            raise BqError("ids and starts without adapters")
        if adapters is not None:
            if y_out is not None and y_out.shape != (M, self.N):
                raise BqError(f"y_out must be [{M}, {self.N}]")
            y_out = self._output(y_out, M, out_dtype, X)
            who, ws, ws_bytes, held = self._adapted(X, adapters, ids, starts, workspace, path, y_out)
            self._run(_lib().mmd_norm_linear_adapted, "mmd_norm_linear_adapted", *who, X.data_ptr(), pr, gamma.data_ptr(), eps, M, ph, y_out.data_ptr(),
                      _DT[y_out.dtype], ws, ws_bytes, path, _stream(X))
            return y_out, X if h_out is None else h_out
        if workspace is not None:
            ws, ws_bytes = workspace.data_ptr(), _bytes_of(workspace, X)
        else:
            held, ws, ws_bytes = self._rows_scratch(M)
        if y_out is not None and y_out.shape != (M, self.N):
            raise BqError(f"y_out must be [{M}, {self.N}]")
        y_out = self._output(y_out, M, out_dtype, X)
        args = (self._h, X.data_ptr(), pr, gamma.data_ptr(), eps, M, ph, y_out.data_ptr(), _DT[y_out.dtype], ws, ws_bytes, path, _stream(X))
        if torch.cuda.current_device() == X.device.index:
            rc = _lib().mmd_norm_linear(*args)
        else:
            with torch.cuda.device(X.device):
                rc = _lib().mmd_norm_linear(*args)
        if rc != 0:
            _check(rc, "mmd_norm_linear")
        return y_out, X if h_out is None else h_out

    def _rows_scratch(self, M: int):
        """The cached workspace for M rows as Scratch.take gives it, its size looked up once per M."""
        need = self._need.get(M)
        if need is None:
            if len(self._need) > 1024:
                self._need.clear()
            need = self._need[M] = self.workspace_layout(M)[1]
        return self._scratch.take("rows", need)

    def linear_static(self, X: torch.Tensor, out_dtype: torch.dtype | None = None, path: int = PATH_AUTO,
                      y_out: torch.Tensor | None = None) -> torch.Tensor:
        """``mmd_linear_static``: the same layer with the library's built-in scratch array (small M only); the call
        itself allocates nothing when ``y_out`` is given."""
        _dev(X, "X")
        if X.dtype != self.dtype or X.dim() != 2 or X.shape[1] != self.K:
            raise BqError("X must be [M, K] of the weights' element type")
        M = X.shape[0]
        y_out = self._output(y_out, M, out_dtype, X)
        with torch.cuda.device(X.device):
            rc = _lib().mmd_linear_static(self._h, X.data_ptr(), M, y_out.data_ptr(), _DT[y_out.dtype], path, _stream(X))
        if rc == 10:
            raise BqError("mmd_linear_static failed with status 10: " + _lib().bq_last_cuda_error().decode())
        _check(rc, "mmd_linear_static")
        return y_out

    def workspace_parts(self, M: int, workspace: torch.Tensor | None = None):
        """(qx, scalex, sidex) views of the workspace after a call with M rows."""
        ws = self.workspace(M) if workspace is None else workspace
        (oq, osc, osd), _ = self.workspace_layout(M)
        sc = mmd_side_columns(self.n_features)
        qx = ws[oq:oq + M * self.K].view(torch.int8).view(M, self.K)
        sx = ws[osc:osc + 4 * M].view(torch.float32)
        sd = ws[osd:osd + 2 * M * sc].view(self.dtype).view(M, sc)
        return qx, sx, sd

    def kernel_status(self) -> int:
        st = ctypes.c_int(0)
        with torch.cuda.device(self.device):
            _check(_lib().mmd_kernel_status(self._h, ctypes.byref(st)), "mmd_kernel_status")
        return int(st.value)

    def selftest_bounded_wait(self, limit_us: int = 2000) -> int:
        """``mmd_selftest_bounded_wait``: lets a bounded wait of the tensor-core kernels run out on purpose (short
        limit, a barrier nothing arms); returns how many threads left through the give-up path."""
        left = ctypes.c_int(-1)
        with torch.cuda.device(self.device):
            _check(_lib().mmd_selftest_bounded_wait(self._h, limit_us, ctypes.byref(left), torch.cuda.current_stream(self.device).cuda_stream),
                   "mmd_selftest_bounded_wait")
        return int(left.value)

    def close(self) -> None:
        if self._h:
            _lib().mmd_free(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

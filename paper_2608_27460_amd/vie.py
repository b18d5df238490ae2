"""Python binding of libvie (include/vie.h): argument marshalling only.

Every step of the head runs in the library's HIP kernels (or, for the offline
index build, its C++ builder); torch only supplies device memory and the
current HIP stream.  There is no fallback: if libvie.so is missing this module
raises on import.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import functools
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("VIE_LIB") or os.path.join(_HERE, "lib", "libvie.so")

OK, EINVAL, ENOMEM, EHIP, EIO, EFORMAT, ESTATE, EUNSUPPORTED = range(8)
F32, BF16 = 0, 1


class VieError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("%s (status %d)" % (message, status))
        self.status = status


class SearchParams(C.Structure):
    _fields_ = [("expand_width", C.c_int32), ("int8_rows", C.c_int32), ("trace_dev", C.c_void_p),
                ("trace_cap", C.c_int32), ("team", C.c_int32), ("workspace_dev", C.c_void_p),
                ("workspace_bytes", C.c_size_t), ("share", C.c_int32)]


class BuildParams(C.Structure):
    _fields_ = [("M", C.c_int32), ("M0", C.c_int32), ("ef_construction", C.c_int32), ("n_threads", C.c_int32),
                ("seed", C.c_uint64), ("select", C.c_int32)]


class GpuBuildParams(C.Structure):
    _fields_ = [("K", C.c_int32), ("M0", C.c_int32), ("chunk_rows", C.c_int64)]


class SamplingParams(C.Structure):
    _fields_ = [("temperature", C.c_double), ("top_p", C.c_double), ("min_p", C.c_double), ("top_k", C.c_int32),
                ("temperature_dev", C.c_void_p), ("top_k_dev", C.c_void_p), ("top_p_dev", C.c_void_p),
                ("min_p_dev", C.c_void_p)]


class IndexDesc(C.Structure):
    _fields_ = [("V", C.c_int64), ("d", C.c_int32), ("dtype", C.c_int32), ("M", C.c_int32), ("M0", C.c_int32),
                ("ef_construction", C.c_int32), ("maxlevel", C.c_int32), ("entry", C.c_int32),
                ("n_upper_blocks", C.c_int64), ("seed", C.c_uint64), ("w_fingerprint", C.c_uint64),
                ("on_device", C.c_int32), ("device", C.c_int32)]


def _load() -> C.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError("libvie.so is not built (%s); run `python -m paper_2608_27460_amd.build`" % LIB_PATH)
    L = C.CDLL(LIB_PATH)
    vp, i32, i64, sz, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t, C.c_float
    st = C.c_int
    sig = {
        "vie_index_build": (st, [vp, i32, i64, i32, C.POINTER(BuildParams), C.POINTER(vp)]),
        "vie_index_build_gpu": (st, [vp, i32, i64, i32, C.POINTER(GpuBuildParams), vp, C.POINTER(vp)]),
        "vie_index_save": (st, [vp, C.c_char_p]),
        "vie_index_load": (st, [C.c_char_p, vp, C.POINTER(vp)]),
        "vie_index_to_device": (st, [vp, vp, vp]),
        "vie_index_info": (st, [vp, C.POINTER(IndexDesc)]),
        "vie_index_export": (st, [vp, vp, vp, vp, vp]),
        "vie_index_free": (None, [vp]),
        "vie_query": (st, [vp, vp, i32, i32, i32, vp, vp, vp, vp]),
        "vie_query_ex": (st, [vp, vp, i32, i32, i32, vp, vp, vp, vp, vp]),
        "vie_query_forced": (st, [vp, vp, i32, i32, i32, vp, vp, i32, vp, vp, vp, vp]),
        "vie_query_workspace": (st, [vp, i32, i32, i32, vp, C.POINTER(sz)]),
        "vie_quantize_rows": (st, [vp, i32, i64, i32, vp, vp, vp]),
        "vie_index_attach_int8": (st, [vp, vp, vp]),
        "vie_dense_topk_workspace": (st, [i64, i32, i32, i32, C.POINTER(sz)]),
        "vie_dense_topk": (st, [vp, i32, i64, i32, vp, i32, i32, vp, vp, vp, sz, vp]),
        "vie_dense_topk_noalloc": (st, [vp, i32, i64, i32, vp, i32, i32, vp, vp, vp]),
        "vie_scatter": (st, [vp, vp, i32, i32, i64, vp, vp]),
        "vie_int8_logits_workspace": (st, [i64, i32, i32, C.POINTER(sz)]),
        "vie_int8_logits": (st, [vp, vp, i64, i32, vp, i32, i32, vp, i32, i64, vp, sz, vp]),
        "vie_sample": (st, [vp, vp, i32, i32, vp, vp, vp, vp, vp, vp]),
        "vie_sample_rows_workspace": (st, [i64, i32, C.POINTER(sz)]),
        "vie_sample_rows": (st, [vp, i32, i64, i64, i32, vp, vp, vp, vp, vp, vp, sz, vp]),
        "vie_distill_workspace": (st, [i64, i32, C.POINTER(sz)]),
        "vie_distill": (st, [vp, i32, i32, i64, i64, vp, vp, i32, f32, vp, vp, vp, sz, vp]),
        "vie_distill_grad": (st, [vp, i32, i32, i64, i64, vp, vp, i32, f32, vp, vp, f32, vp, i64, vp]),
        "vie_distill_step": (st, [vp, i32, i32, i64, i64, vp, vp, i32, f32, vp, f32, vp, vp, i64, vp, sz, vp]),
        "vie_status_string": (C.c_char_p, [st]),
        "vie_last_error": (C.c_char_p, []),
        "vie_version": (i32, []),
    }
    for name, (res, args) in sig.items():
        f = getattr(L, name)
        f.restype = res
        f.argtypes = args
    return L


lib = _load()


def _check(status: int) -> None:
    if status != OK:
        msg = lib.vie_last_error().decode(errors="replace") or lib.vie_status_string(status).decode()
        raise VieError(status, msg)


def _torch():
    import torch
    return torch


def _stream(t) -> C.c_void_p:
    torch = _torch()
    return C.c_void_p(torch.cuda.current_stream(t.device).cuda_stream)


def _raw_stream(device) -> int:
    """The current stream of a device, without the Stream object of _stream (1.8 us of a call)."""
    torch = _torch()
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(device.index) if raw else torch.cuda.current_stream(device).cuda_stream


def _dtype_of_tensor(t) -> int:
    torch = _torch()
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError("W_out / queries must be float32 or bfloat16, got %s" % t.dtype)


def _dev_ptr(t, name: str):
    if not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return C.c_void_p(t.data_ptr())


def host_to_torch(W: np.ndarray, dtype: int):
    """CPU torch tensor view of a synthetic matrix (fp32, or bf16 bit patterns)."""
    torch = _torch()
    W = np.ascontiguousarray(W)
    if dtype == F32:
        return torch.from_numpy(W.astype(np.float32, copy=False))
    return torch.from_numpy(W.view(np.int16)).view(torch.bfloat16)


class Index:
    """An HNSW index over the rows of W_out (Section 3 of the paper)."""

    def __init__(self, handle: C.c_void_p):
        self._h = handle
        self._W_dev = None

    @classmethod
    def build(cls, W: np.ndarray, dtype: int, M: int, ef_construction: int, seed: int = 0, n_threads: int = 0,
              M0: int = 0, select: str = "heuristic") -> "Index":
        W = np.ascontiguousarray(W)
        want = np.float32 if dtype == F32 else np.uint16
        if W.dtype != want or W.ndim != 2:
            raise TypeError("W must be a 2-D %s array" % np.dtype(want).name)
        p = BuildParams(M, M0, ef_construction, n_threads, seed, 0 if select == "heuristic" else 1)
        h = C.c_void_p()
        _check(lib.vie_index_build(W.ctypes.data_as(C.c_void_p), dtype, W.shape[0], W.shape[1], C.byref(p),
                                   C.byref(h)))
        return cls(h)

    @classmethod
    def build_gpu(cls, W_dev, K: int, M0: int, chunk_rows: int = 0) -> "Index":
        """Single-layer batch graph over the rows of the device matrix W_dev
        (vie_index_build_gpu); the index comes back on W_dev's device."""
        torch = _torch()
        dt = _dtype_of_tensor(W_dev)
        V, d = W_dev.shape
        p = GpuBuildParams(K, M0, chunk_rows)
        h = C.c_void_p()
        with torch.cuda.device(W_dev.device):
            _check(lib.vie_index_build_gpu(_dev_ptr(W_dev, "W_dev"), dt, V, d, C.byref(p), _stream(W_dev),
                                           C.byref(h)))
        ix = cls(h)
        ix._W_dev = W_dev
        ix._q8 = None
        return ix

    @classmethod
    def load(cls, path: str, W: np.ndarray | None = None) -> "Index":
        h = C.c_void_p()
        wp = None if W is None else np.ascontiguousarray(W).ctypes.data_as(C.c_void_p)
        _check(lib.vie_index_load(path.encode(), wp, C.byref(h)))
        return cls(h)

    def save(self, path: str) -> None:
        _check(lib.vie_index_save(self._h, path.encode()))

    def info(self) -> dict:
        d = IndexDesc()
        _check(lib.vie_index_info(self._h, C.byref(d)))
        return {f: getattr(d, f) for f, _ in IndexDesc._fields_}

    def export(self) -> dict:
        i = self.info()
        V, M, M0, nb = i["V"], i["M"], i["M0"], i["n_upper_blocks"]
        out = {"levels": np.empty(V, np.uint8), "adj0": np.empty((V, M0), np.int32),
               "upper_off": np.empty(V, np.int32), "upper": np.empty((nb, M), np.int32)}
        _check(lib.vie_index_export(self._h, *(out[k].ctypes.data_as(C.c_void_p) if out[k].size else None
                                               for k in ("levels", "adj0", "upper_off", "upper"))))
        return out

    def to_device(self, W_dev) -> None:
        """Upload the graph to W_dev's device and borrow W_dev (kept alive here)."""
        torch = _torch()
        with torch.cuda.device(W_dev.device):
            _check(lib.vie_index_to_device(self._h, _dev_ptr(W_dev, "W_dev"), _stream(W_dev)))
        self._W_dev = W_dev
        self._q8 = None  # the library detaches int8 rows on every move

    def attach_int8(self, q, scale) -> None:
        """Layer-0 scores from these int8 rows (see quantize_rows); None detaches."""
        if q is None:
            _check(lib.vie_index_attach_int8(self._h, None, None))
            self._q8 = None
            return
        _check(lib.vie_index_attach_int8(self._h, _dev_ptr(q, "q"), _dev_ptr(scale, "scale")))
        self._q8 = (q, scale)

    def _params(self, h, B: int, k: int, ef: int, width: int, int8: bool, trace, team: int,
                share: int = 1) -> SearchParams:
        prm = SearchParams(width, int(int8), None if trace is None else _dev_ptr(trace, "trace"),
                           0 if trace is None else trace.shape[1], team, None, 0, share)
        if team > 1 or share > 1:
            n = C.c_size_t()
            _check(lib.vie_query_workspace(self._h, B, k, ef, C.byref(prm), C.byref(n)))
            ws = getattr(self, "_ws", None)
            if ws is None or ws.numel() < n.value or ws.device != h.device:
                ws = _torch().empty(n.value, dtype=_torch().uint8, device=h.device)
                self._ws = ws
            prm.workspace_dev = _dev_ptr(ws, "workspace")
            prm.workspace_bytes = ws.numel()
        return prm

    def query_into(self, h, k: int, ef: int, ids, logits, stats=None, width: int = 1, int8: bool = False,
                   trace=None, team: int = 1, share: int = 1) -> None:
        """HNSW top-k of h [B, d] into preallocated ids int32 [B, k], logits fp32 [B, k]
        (and stats uint32-as-int32 [B, 2]) on the current stream; width > 1
        expands that many beam entries per layer-0 step, int8 walks layer 0 on
        the attached int8 rows, trace (int32 [B, cap]) receives each query's
        expansions as (layer << 27) | node, team > 1 searches each query with
        that many workgroups, share > 1 lets groups of that many queries
        share the rows they fetch (vie_query_ex; the index keeps the
        workspace, so such searches of one index must not overlap in time)."""
        B = h.shape[0]
        sp = None if stats is None else _dev_ptr(stats, "stats")
        if width == 1 and not int8 and trace is None and team <= 1 and share <= 1:
            _check(lib.vie_query(self._h, _dev_ptr(h, "h"), B, k, ef, _dev_ptr(ids, "ids"),
                                 _dev_ptr(logits, "logits"), sp, _stream(h)))
        else:
            prm = self._params(h, B, k, ef, width, int8, trace, team, share)
            _check(lib.vie_query_ex(self._h, _dev_ptr(h, "h"), B, k, ef, C.byref(prm), _dev_ptr(ids, "ids"),
                                    _dev_ptr(logits, "logits"), sp, _stream(h)))

    def query_forced_into(self, h, k: int, ef: int, forced, ids, logits, stats=None, width: int = 1,
                          int8: bool = False, team: int = 1) -> None:
        """Search plus the forced-inclusion ids (int32 device tensor [n]):
        ids int32 [B, k + n], logits fp32 [B, k + n] (vie_query_forced)."""
        B = h.shape[0]
        n = int(forced.numel())
        sp = None if stats is None else _dev_ptr(stats, "stats")
        prm = self._params(h, B, k, ef, width, int8, None, team)
        fp = _dev_ptr(forced, "forced") if n else None
        _check(lib.vie_query_forced(self._h, _dev_ptr(h, "h"), B, k, ef, C.byref(prm), fp, n, _dev_ptr(ids, "ids"),
                                    _dev_ptr(logits, "logits"), sp, _stream(h)))

    def query(self, h, k: int, ef: int, stats: bool = False, width: int = 1, int8: bool = False,
              trace_cap: int = 0, team: int = 1, share: int = 1):
        """(ids, logits), plus stats if asked, plus the expansion trace
        [B, trace_cap] (-1 past the last expansion) if trace_cap > 0."""
        torch = _torch()
        if h.dim() == 1:
            h = h.unsqueeze(0)
        B = h.shape[0]
        ids = torch.empty((B, k), dtype=torch.int32, device=h.device)
        lg = torch.empty((B, k), dtype=torch.float32, device=h.device)
        st = torch.empty((B, 2), dtype=torch.int32, device=h.device) if stats else None
        tr = torch.full((B, trace_cap), -1, dtype=torch.int32, device=h.device) if trace_cap > 0 else None
        self.query_into(h, k, ef, ids, lg, st, width, int8, tr, team, share)
        out = (ids, lg) + ((st,) if stats else ())
        return out + (tr,) if tr is not None else out

    def close(self) -> None:
        if self._h:
            lib.vie_index_free(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def quantize_rows(W, dtype: int):
    """int8 rows [V, d] and fp32 scales [V] of the device matrix W (vie_quantize_rows)."""
    torch = _torch()
    V, d = W.shape
    q = torch.empty((V, d), dtype=torch.int8, device=W.device)
    sc = torch.empty((V,), dtype=torch.float32, device=W.device)
    _check(lib.vie_quantize_rows(_dev_ptr(W, "W"), dtype, V, d, _dev_ptr(q, "q"), _dev_ptr(sc, "scale"), _stream(W)))
    return q, sc


def dense_topk_workspace_bytes(V: int, d: int, B: int, k: int) -> int:
    n = C.c_size_t()
    _check(lib.vie_dense_topk_workspace(V, d, B, k, C.byref(n)))
    return n.value


def dense_topk_into(W, h, k: int, ids, logits, workspace) -> None:
    """Exact top-k of W h on the current stream; workspace is a uint8 device
    tensor of at least dense_topk_workspace_bytes() bytes."""
    V, d = W.shape
    dt = _dtype_of_tensor(W)
    if _dtype_of_tensor(h) != dt:
        raise TypeError("W and h must have the same dtype")
    _check(lib.vie_dense_topk(_dev_ptr(W, "W"), dt, V, d, _dev_ptr(h, "h"), h.shape[0], k, _dev_ptr(ids, "ids"),
                              _dev_ptr(logits, "logits"), _dev_ptr(workspace, "workspace"), workspace.numel(),
                              _stream(h)))


def dense_topk_noalloc_into(W, h, k: int, ids, logits) -> None:
    """dense_topk_into without a workspace argument: the library's static
    per-GPU workspace (vie_dense_topk_noalloc); calls on one GPU must not
    overlap."""
    V, d = W.shape
    dt = _dtype_of_tensor(W)
    if _dtype_of_tensor(h) != dt:
        raise TypeError("W and h must have the same dtype")
    _check(lib.vie_dense_topk_noalloc(_dev_ptr(W, "W"), dt, V, d, _dev_ptr(h, "h"), h.shape[0], k,
                                      _dev_ptr(ids, "ids"), _dev_ptr(logits, "logits"), _stream(h)))


class DenseHead:
    """Exact dense head over a device W_out with its own workspace."""

    def __init__(self, W, max_batch: int = 8, max_k: int = 1024):
        torch = _torch()
        self.W = W
        V, d = W.shape
        nbytes = dense_topk_workspace_bytes(V, d, max_batch, min(max_k, V))
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=W.device)

    def __call__(self, h, k: int):
        torch = _torch()
        if h.dim() == 1:
            h = h.unsqueeze(0)
        B = h.shape[0]
        ids = torch.empty((B, k), dtype=torch.int32, device=h.device)
        lg = torch.empty((B, k), dtype=torch.float32, device=h.device)
        dense_topk_into(self.W, h, k, ids, lg, self.workspace)
        return ids, lg


def scatter_into(ids, logits, V: int, out) -> None:
    B, k = ids.shape
    _check(lib.vie_scatter(_dev_ptr(ids, "ids"), _dev_ptr(logits, "logits"), B, k, V, _dev_ptr(out, "out"),
                           _stream(ids)))


def scatter(ids, logits, V: int):
    """Full-vocabulary logits [B, V]: -inf except at the retrieved ids (Section 3)."""
    torch = _torch()
    if ids.dim() == 1:
        ids, logits = ids.unsqueeze(0), logits.unsqueeze(0)
    out = torch.empty((ids.shape[0], V), dtype=torch.float32, device=ids.device)
    scatter_into(ids, logits, V, out)
    return out


# ---------------------------------------------------------------------------
# around the head's logits: the int8 head, the token drawn, distillation
# (of which autograd records the losses of distill alone)
# ---------------------------------------------------------------------------

_SAME_DEVICE = contextlib.nullcontext()


def _on(device):
    """A context in which `device` is the current one (entering torch's costs 1.3 us, so only where it is not)."""
    torch = _torch()
    return _SAME_DEVICE if torch.cuda.current_device() == device.index else torch.cuda.device(device)


def _matrix(t, name: str):
    """Pointer, dtype code, rows, row length and row stride of a device matrix of logits."""
    if not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError("%s must be [rows, V] with contiguous rows" % name)
    rows, V = t.shape
    return t.data_ptr(), _dtype_of_tensor(t), rows, V, t.stride(0) if rows > 1 else V


def _values(t, name: str, dtype, shape, device) -> int:
    """Pointer of a contiguous device tensor of this type and shape."""
    if t.dtype is dtype and t.shape == shape and t.is_cuda and t.device == device and t.is_contiguous():
        return t.data_ptr()
    if t.dtype is not dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if t.shape != shape:
        raise ValueError("%s must be %s, got %s" % (name, list(shape), list(t.shape)))
    if t.is_cuda and t.device != device:
        raise ValueError("%s is on %s, not on %s" % (name, t.device, device))
    return _dev_ptr(t, name).value


@functools.lru_cache(maxsize=256)
def _workspace_bytes(query: str, *sizes) -> int:
    n = C.c_size_t()
    _check(getattr(lib, query)(*sizes, C.byref(n)))
    return n.value


def _workspace(nbytes: int, device):
    """A workspace of this call (torch reuses its memory in stream order), and its pointer."""
    if nbytes == 0:
        return None, None
    t = _torch().empty(nbytes, dtype=_torch().uint8, device=device)
    return t, t.data_ptr()


def _overwritten(out) -> None:
    """Lets autograd see that a caller's tensor was written to: a backward pass that saved it then refuses to run."""
    _torch().autograd.graph.increment_version(out)


class Int8Head:
    """Full-vocabulary logits from the int8 rows and scales of quantize_rows.
    The quantized products have no derivative: autograd does not record them."""

    def __init__(self, q, scale):
        torch = _torch()
        if q.dtype != torch.int8 or q.dim() != 2:
            raise TypeError("q must be a 2-D int8 tensor")
        _dev_ptr(q, "q")
        _values(scale, "scale", torch.float32, (q.shape[0],), q.device)
        self.q, self.scale = q, scale

    def __call__(self, h, dtype=None, out=None):
        """Logits [B, V] (vie_int8_logits) of h [B, d], fp32 unless dtype or out says bf16."""
        torch = _torch()
        if h.dim() == 1:
            h = h.unsqueeze(0)
        V, d = self.q.shape
        if h.dim() != 2 or h.shape[1] != d:
            raise ValueError("h must be [B, %d], got %s" % (d, list(h.shape)))
        if h.device != self.q.device:
            raise ValueError("h is on %s, not on %s" % (h.device, self.q.device))
        B, hd = h.shape[0], _dtype_of_tensor(h)
        given = out is not None
        if not given:
            out = torch.empty((B, V), dtype=dtype or torch.float32, device=h.device)
        elif dtype is not None and out.dtype != dtype:
            raise TypeError("out is %s, not %s" % (out.dtype, dtype))
        op, od, rows, cols, ld = _matrix(out, "out")
        if (rows, cols) != (B, V) or out.device != h.device:
            raise ValueError("out must be [%d, %d] on %s" % (B, V, h.device))
        hp = _dev_ptr(h, "h")
        n = _workspace_bytes("vie_int8_logits_workspace", V, d, B)
        with _on(h.device):
            ws, wp = _workspace(n, h.device)
            _check(lib.vie_int8_logits(self.q.data_ptr(), self.scale.data_ptr(), V, d, hp, hd, B, op, od, ld, wp, n,
                                       _raw_stream(h.device)))
        if given:
            _overwritten(out)
        return out


def _sampling(B: int, device, temperature, top_k, top_p, min_p) -> SamplingParams:
    """Each setting is a number, or a device tensor [B] (fp32; top_k int32)."""
    p = SamplingParams(1.0, 1.0, 0.0, 0)
    torch = _torch()
    for name, v in (("temperature", temperature), ("top_k", top_k), ("top_p", top_p), ("min_p", min_p)):
        if isinstance(v, torch.Tensor):
            setattr(p, name + "_dev", _values(v, name, torch.int32 if name == "top_k" else torch.float32, (B,), device))
        else:
            setattr(p, name, max(-1, min(v, 0x7FFFFFFF)) if name == "top_k" else v)
    return p


def _drawn(B: int, device):
    torch = _torch()
    return (torch.empty(B, dtype=torch.int32, device=device), torch.empty(B, dtype=torch.float32, device=device),
            torch.empty(B, dtype=torch.int32, device=device))


def sample(ids, logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token int32, probability fp32, kept candidates int32), each [B], drawn
    from the lists ids int32 [B, k], logits fp32 [B, k] of a head with the
    uniform numbers u fp32 [B] (vie_sample)."""
    torch = _torch()
    if ids.dim() == 1:
        ids, logits = ids.unsqueeze(0), logits.unsqueeze(0)
    if ids.dim() != 2:
        raise ValueError("ids must be [B, k]")
    (B, k), dev = ids.shape, ids.device
    ip = _values(ids, "ids", torch.int32, (B, k), dev)
    lp = _values(logits, "logits", torch.float32, (B, k), dev)
    up = _values(u, "u", torch.float32, (B,), dev)
    prm = _sampling(B, dev, temperature, top_k, top_p, min_p)
    with _on(dev):
        tok, prob, kept = out = _drawn(B, dev)
        _check(lib.vie_sample(ip, lp, B, k, C.byref(prm), up, tok.data_ptr(), prob.data_ptr(), kept.data_ptr(),
                              _raw_stream(dev)))
    return out


def sample_rows(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """sample() over full-vocabulary rows logits [B, V], fp32 or bf16, -inf where masked (vie_sample_rows)."""
    torch = _torch()
    if logits.dim() == 1:
        logits = logits.unsqueeze(0)
    lp, dt, B, V, ld = _matrix(logits, "logits")
    dev = logits.device
    up = _values(u, "u", torch.float32, (B,), dev)
    prm = _sampling(B, dev, temperature, top_k, top_p, min_p)
    n = _workspace_bytes("vie_sample_rows_workspace", V, B)
    with _on(dev):
        tok, prob, kept = out = _drawn(B, dev)
        ws, wp = _workspace(n, dev)
        _check(lib.vie_sample_rows(lp, dt, V, ld, B, C.byref(prm), up, tok.data_ptr(), prob.data_ptr(),
                                   kept.data_ptr(), wp, n, _raw_stream(dev)))
    return out


def _distill_inputs(logits, ids, teacher):
    torch = _torch()
    m = _matrix(logits, "logits")
    N = m[2]
    if ids.dim() != 2:
        raise ValueError("ids must be [N, k]")
    k = ids.shape[1]
    return (m, _values(ids, "ids", torch.int32, (N, k), logits.device),
            _values(teacher, "teacher", torch.float32, (N, k), logits.device), k)


def _grad_of(logits, gloss, out):
    """The gradient's tensor, pointer and row stride, and the pointer of the losses' gradients."""
    torch = _torch()
    N, V = logits.shape
    if out is None:
        out = torch.empty((N, V), dtype=logits.dtype, device=logits.device)
    gp, gd, rows, cols, ld = _matrix(out, "out")
    if (rows, cols) != (N, V) or out.dtype != logits.dtype or out.device != logits.device:
        raise ValueError("out must be like logits")
    return out, gp, ld, None if gloss is None else _values(gloss, "gloss", torch.float32, (N,), logits.device)


@functools.lru_cache(maxsize=None)
def _recorded():
    """Distillation as autograd records it: (the losses of distill, the loss that distill_step returns)."""
    torch = _torch()

    class Losses(torch.autograd.Function):
        @staticmethod
        def forward(ctx, logits, ids, teacher, tau):
            loss, stats = _losses(logits, ids, teacher, tau)
            ctx.save_for_backward(logits, ids, teacher, stats)
            ctx.tau = tau
            ctx.mark_non_differentiable(stats)
            return loss, stats

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, gloss, _):
            logits, ids, teacher, stats = ctx.saved_tensors
            return distill_grad(logits, ids, teacher, stats, ctx.tau, gloss=gloss.contiguous()), None, None, None

    class Given(torch.autograd.Function):
        # (`anchor`: a leaf of its own, so that a loss kept for the log does not keep the logits' graph)
        @staticmethod
        def forward(ctx, anchor, loss):
            return loss.view_as(loss)

        @staticmethod
        def backward(ctx, gloss):
            raise RuntimeError("distill_step gives the gradient of its loss as the second result; "
                               "detach the loss, or take it from distill")

    return Losses, lambda loss: Given.apply(torch.empty(0, requires_grad=True), loss)


def _losses(logits, ids, teacher, tau):
    torch = _torch()
    (lp, dt, N, V, ld), ip, tp, k = _distill_inputs(logits, ids, teacher)
    n = _workspace_bytes("vie_distill_workspace", V, N)
    with _on(logits.device):
        loss = torch.empty(N, dtype=torch.float32, device=logits.device)
        stats = torch.empty((N, 2), dtype=torch.float32, device=logits.device)
        ws, wp = _workspace(n, logits.device)
        _check(lib.vie_distill(lp, dt, N, V, ld, ip, tp, k, tau, loss.data_ptr(), stats.data_ptr(), wp, n,
                               _raw_stream(logits.device)))
    return loss, stats


def distill(logits, ids, teacher, tau: float = 1.0):
    """(loss fp32 [N], stats fp32 [N, 2]) of the student's logits [N, V] (fp32
    or bf16) against a teacher's lists ids int32 [N, k], teacher fp32 [N, k] of
    logits at the temperature tau (vie_distill); stats goes to distill_grad.
    Where the logits require a gradient, autograd's backward pass takes the
    losses' from distill_grad (once differentiable); the teacher gets none, and
    is refused if it requires one.  (Captured into a graph, as any backward
    pass of torch: while no eager graph of the same leaves is alive.)"""
    torch = _torch()
    if torch.is_grad_enabled():
        if teacher.requires_grad:
            raise ValueError("teacher requires a gradient, which distillation does not compute: detach it")
        if logits.requires_grad:
            return _recorded()[0].apply(logits, ids, teacher, tau)
    return _losses(logits, ids, teacher, tau)


def distill_grad(logits, ids, teacher, stats, tau: float = 1.0, gloss=None, weight: float = 1.0, out=None):
    """Gradient of sum_n weight gloss[n] loss[n] (gloss fp32 [N], ones if None)
    in the logits, in their type; out may be logits itself (vie_distill_grad).
    Autograd does not record it."""
    (lp, dt, N, V, ld), ip, tp, k = _distill_inputs(logits, ids, teacher)
    sp = _values(stats, "stats", _torch().float32, (N, 2), logits.device)
    with _on(logits.device):
        grad, gp, gld, glp = _grad_of(logits, gloss, out)
        _check(lib.vie_distill_grad(lp, dt, N, V, ld, ip, tp, k, tau, sp, glp, weight, gp, gld,
                                    _raw_stream(logits.device)))
    if out is not None:
        _overwritten(out)
    return grad


def distill_step(logits, ids, teacher, tau: float = 1.0, gloss=None, weight: float = 1.0, out=None):
    """(loss, gradient): distill and distill_grad at once (vie_distill_step).
    The gradient is the caller's to pass on (logits.backward(gradient)); where
    an input requires one, a backward pass from the loss raises."""
    torch = _torch()
    (lp, dt, N, V, ld), ip, tp, k = _distill_inputs(logits, ids, teacher)
    n = _workspace_bytes("vie_distill_workspace", V, N)
    with _on(logits.device):
        loss = torch.empty(N, dtype=torch.float32, device=logits.device)
        grad, gp, gld, glp = _grad_of(logits, gloss, out)
        ws, wp = _workspace(n, logits.device)
        _check(lib.vie_distill_step(lp, dt, N, V, ld, ip, tp, k, tau, glp, weight, loss.data_ptr(), gp, gld, wp, n,
                                    _raw_stream(logits.device)))
    if out is not None:
        _overwritten(out)
    if (logits.requires_grad or teacher.requires_grad) and torch.is_grad_enabled():
        loss = _recorded()[1](loss)
    return loss, grad

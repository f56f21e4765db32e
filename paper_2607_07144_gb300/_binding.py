"""ctypes binding of libfkv.so (include/fkv.h).  Argument marshalling only:
every step of the archive path runs in the library's CUDA kernels.  PyTorch
supplies device memory and the current CUDA stream."""
from __future__ import annotations

import ctypes
import os
import struct
import threading

import numpy as np
import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libfkv.so")

OK, EINVAL, ERANGE, ENOMEM, ECUDA, ECORRUPT, ETIMEOUT = 0, -1, -2, -3, -4, -5, -6
F32, F16, BF16 = 0, 1, 2
E4M3, INT8 = 0, 1
_FORMAT = {torch.float8_e4m3fn: E4M3, torch.int8: INT8}
_DTYPE = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}
_ERRNAME = {EINVAL: "EINVAL", ERANGE: "ERANGE", ENOMEM: "ENOMEM", ECUDA: "ECUDA",
            ECORRUPT: "ECORRUPT", ETIMEOUT: "ETIMEOUT"}

_lock = threading.Lock()
_lib = None


class FkvError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__("%s (%d): %s" % (_ERRNAME.get(code, "?"), code, msg))
        self.code = code


class _Codebooks(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int), ("n_heads", ctypes.c_int), ("dim", ctypes.c_int),
                ("stages_k", ctypes.c_int), ("stages_v", ctypes.c_int),
                ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("codewords", ctypes.c_int), ("pooled", ctypes.c_int)]


class _Cache(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("dtype", ctypes.c_int), ("batch", ctypes.c_int64),
                ("seq", ctypes.c_int64), ("stride_layer", ctypes.c_int64),
                ("stride_batch", ctypes.c_int64), ("stride_head", ctypes.c_int64),
                ("stride_pos", ctypes.c_int64)]


class _Pages(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("format", ctypes.c_int), ("n_heads", ctypes.c_int),
                ("dim", ctypes.c_int), ("block", ctypes.c_int), ("n_blocks", ctypes.c_int64),
                ("stride_block", ctypes.c_int64), ("stride_head", ctypes.c_int64), ("stride_pos", ctypes.c_int64),
                ("scale_stride_block", ctypes.c_int64), ("scale_stride_head", ctypes.c_int64)]


# fkv_cache, fkv_rows, fkv_plan and fkv_attend, packed: filling a buffer takes a tenth of
# the time of as many ctypes arguments
_CACHE = struct.Struct("@Pi6q")
_ROWS = struct.Struct("@Piqq")
_PLAN = struct.Struct("@10P6q")
_ATTEND = struct.Struct("@9P12q3i2fi")


# name -> (restype, argtypes)
_P, _I, _I64, _D = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_double
SIGNATURES = {
    "fkv_packing_ratio": (_D, [_I]),
    "fkv_max_span_len": (_I, [_D]),
    "fkv_create": (_I, [_I, _D, _I, _P, ctypes.POINTER(_P)]),
    "fkv_destroy": (_I, [_P]),
    "fkv_vertices": (_I, [_P, _P]),
    "fkv_params": (_I, [_P, _P, _P, _P]),
    "fkv_symbol_bytes": (_I, [_P]),
    "fkv_last_error": (ctypes.c_char_p, [_P]),
    "fkv_sync_status": (_I, [_P, _P]),
    "fkv_span_encode": (_I, [_P, _P, _I64, _I64, _I64, _P, _I64, _P]),
    "fkv_span_decode": (_I, [_P, _P, _I64, _I64, _I64, _P, _I64, _P]),
    "fkv_read": (_I, [_P, _P, _I64, _I64, _I64, _P, _I64, _P, _P]),
    "fkv_span_encode_ragged": (_I, [_P, _P, _P, _I64, _P, _P, _P]),
    "fkv_span_decode_ragged": (_I, [_P, _P, _P, _I64, _P, _P, _P]),
    "fkv_read_ragged": (_I, [_P, _P, _P, _P, _I64, _P, _I64, _P, _P]),
    "fkv_suffix_search": (_I, [_P, _P, _I64, _I64, _I64, _P, _I, _P, _I64, _P, _P]),
    "fkv_truncate": (_I, [_P, _P, _I64, _I64, _I64, _I, _I64, _P, _I64, _P, _I64, _P]),
    "fkv_lossy_decode": (_I, [_P, _P, _I64, _P, _I64, _I64, _I64, _I, _I64, _P, _I64, _P]),
    "fkv_lossy_read": (_I, [_P, _P, _I64, _P, _I64, _I64, _I64, _I, _I64, _P, _I64, _P, _P]),
    "fkv_ac_capacity_words": (_I64, [_P, _I64]),
    "fkv_ac_encode": (_I, [_P, _P, _I64, _I64, _I64, _I, _P, _I64, _P, _P]),
    "fkv_ac_decode": (_I, [_P, _P, _I64, _P, _I64, _I64, _I, _P, _I64, _P]),
    "fkv_measure_fp64_rate": (_I, [_P, _P]),
    "fkv_check_bounded_wait": (_I, [_P, _I64, _P, _P]),
    "fkv_record_len": (_I, [_P]),
    "fkv_rvq_encode": (_I, [_P, _I, _P, _I64, _I64, _P, _I64, _I64, _P]),
    "fkv_rvq_decode": (_I, [_P, _P, _I64, _I64, _P, _P, _I64, _P]),
    "fkv_decode_kv": (_I, [_P, _P, _I64, _I64, _P, _P, _I64, _P]),
    "fkv_decode_kv_static": (_I, [_P, _P, _I64, _I64, _P, _P, _I64, _P]),
    "fkv_read_kv": (_I, [_P, _P, _I64, _I64, _I64, _P, _I64, _P, _I, _P]),
    "fkv_cache_upload": (_I, [_P, _P, _P, _I64, _I64, _P]),
    "fkv_page_plan": (_I, [_P, _P, _P]),
    "fkv_page_write": (_I, [_P, _P, _P, _P, _P, _I64, _P]),
    "fkv_page_attend_workspace": (_I64, [_P, _P]),
    "fkv_page_attend": (_I, [_P, _P, _P, _I64, _P]),
    "fkv_page_read": (_I, [_P, _P, _P, _I64, _P, _I64, _I64, _I64, _I64, _I64, _P, _P, _P]),
    "fkv_streams_create": (_I, [_P, _I64, _I64, ctypes.POINTER(_P)]),
    "fkv_streams_destroy": (_I, [_P]),
    "fkv_streams_reset": (_I, [_P]),
    "fkv_streams_info": (_I, [_P, _P, _P, _P, _P]),
    "fkv_append": (_I, [_P, _P, _P, _I64, _I64, _P]),
    "fkv_streams_export": (_I, [_P, _P, _P, _P]),
    "fkv_streams_import": (_I, [_P, _I64, _I64, _P, ctypes.POINTER(_P)]),
}


def lib():
    """The loaded library.  Raises if it has not been built: there is no
    fallback implementation."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(LIB_PATH):
                raise RuntimeError("libfkv.so is not built (run __graft_entry__.build())")
            L = ctypes.CDLL(LIB_PATH)
            for name, (res, args) in SIGNATURES.items():
                f = getattr(L, name)
                f.restype = res
                f.argtypes = args
            _lib = L
        return _lib


def _stream(stream=None):
    if stream is not None:
        return stream.cuda_stream
    if torch.cuda.is_initialized():
        # the handle alone: building a Stream object takes 3 us of a call's 15
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return torch.cuda.current_stream().cuda_stream


def _ptr(t: torch.Tensor):
    return t.data_ptr()


def _rows(t: torch.Tensor, unit: int = 1) -> int:
    """Row stride of a [rows, ...] tensor in units of `unit` elements; a
    single row has no meaningful stride, so report its own extent."""
    if t.shape[0] <= 1:
        return max(1, t.numel() // unit)
    return t.stride(0) // unit


def packing_ratio(N: int) -> float:
    return lib().fkv_packing_ratio(int(N))


def max_span_len(r: float) -> int:
    return lib().fkv_max_span_len(float(r))


def measure_fp64_rate(stream=None) -> float:
    """Binary64 add/mul instructions per second of the current device."""
    v = ctypes.c_double()
    rc = lib().fkv_measure_fp64_rate(ctypes.byref(v), _stream(stream))
    if rc != OK:
        raise FkvError(rc, "fkv_measure_fp64_rate failed")
    return v.value


def cache_view(t: torch.Tensor, host: bool = False) -> _Cache:
    """fkv_cache view of a tensor shaped [n_layers, batch, n_heads, seq, dim]
    (any strides with a contiguous last dimension): a CUDA tensor, or with
    host=True a CPU tensor (pinned for full transfer speed)."""
    st = t.stride()
    if len(st) != 5 or st[4] != 1 or t.is_cuda == host:
        raise ValueError("cache must be a %s tensor [layers, batch, heads, seq, dim] with contiguous dim"
                         % ("CPU" if host else "CUDA"))
    return _Cache(t.data_ptr(), _DTYPE[t.dtype], t.shape[1], t.shape[3], st[0], st[1], st[2], st[3])


_I32, _INT64, _FLOAT = torch.int32, torch.int64, torch.float32


def _vectors(t: torch.Tensor, dim: int, what: str, dev: int):
    """(pointer, dtype, shape, token stride, head stride) of a CUDA tensor [tokens, heads, dim] (contiguous dim)."""
    shape, st, dt = t.shape, t.stride(), _DTYPE.get(t.dtype)
    if len(st) != 3 or st[2] != 1 or shape[2] != dim or dt is None or t.get_device() != dev:
        raise ValueError("%s must be a tensor [tokens, heads, %d] with contiguous dim on cuda:%d" % (what, dim, dev))
    # the stride of a dimension of one is never used, but has to be a valid one
    return t.data_ptr(), dt, shape, st[0] if shape[0] > 1 else dim, st[1] if shape[1] > 1 else dim


def _array(t: torch.Tensor, dtype, numel: int, what: str, dev: int):
    """Pointer of a contiguous array of at least `numel` elements on device `dev`."""
    if t.dtype is not dtype or t.numel() < numel or not t.is_contiguous() or t.get_device() != dev:
        raise ValueError("%s must be a contiguous %s tensor of %d elements on cuda:%d" % (what, dtype, numel, dev))
    return t.data_ptr()


def _table(t: torch.Tensor, n_req: int, dev: int):
    shape, st = t.shape, t.stride()
    if (t.dtype is not _I32 or len(shape) != 2 or shape[0] < n_req or (shape[1] > 1 and st[1] != 1) or
            t.get_device() != dev):
        raise ValueError("block_table must be an int32 tensor [requests, pages] on cuda:%d" % dev)
    return t.data_ptr(), st[0] if shape[0] > 1 else max(1, shape[1]), shape[1]


class Pages:
    """A pool of 8-bit K/V pages (fkv_pages): codes k and v [n_blocks, heads,
    block, dim], torch.float8_e4m3fn or torch.int8, of the same strides (any,
    with a contiguous dim: [n_blocks, block, heads, dim] permuted will do), and
    float32 scales [n_blocks, heads].  The tensors stay the caller's."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor):
        if (k.dim() != 4 or k.shape != v.shape or k.stride() != v.stride() or k.dtype != v.dtype or k.stride(3) != 1 or
                k.dtype not in _FORMAT or not k.is_cuda or any(t.device != k.device for t in (v, k_scale, v_scale))):
            raise ValueError("k and v must be float8_e4m3fn or int8 tensors [blocks, heads, block, dim] of one shape "
                             "and strides, with contiguous dim, and all four on one CUDA device")
        if (k_scale.dtype != torch.float32 or v_scale.dtype != torch.float32 or k_scale.shape != k.shape[:2] or
                v_scale.shape != k.shape[:2] or k_scale.stride() != v_scale.stride()):
            raise ValueError("k_scale and v_scale must be float32 tensors [blocks, heads] of the same strides")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_blocks, self.heads, self.block, self.dim = k.shape
        self.device = k.get_device()
        ss = k_scale.stride()
        # the stride of a dimension of one is never used, but has to be a valid one
        st = [x if n > 1 else self.dim for x, n in zip(k.stride(), k.shape)]
        self._c = _Pages(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), _FORMAT[k.dtype],
                         self.heads, self.dim, self.block, self.n_blocks, st[0], st[1], st[2], ss[0], ss[1])
        self._ref = ctypes.byref(self._c)
        self._addr = ctypes.addressof(self._c)

    @classmethod
    def empty(cls, n_blocks: int, heads: int, block: int, dim: int, dtype=torch.float8_e4m3fn, device="cuda"):
        shape = (n_blocks, heads, block, dim)
        return cls(torch.empty(shape, dtype=dtype, device=device), torch.empty(shape, dtype=dtype, device=device),
                   torch.empty(shape[:2], dtype=torch.float32, device=device),
                   torch.empty(shape[:2], dtype=torch.float32, device=device))


class Context:
    """An fkv_ctx: alphabet N, ratio r (default r_N), span length (default
    floor(44/log2(1/r))) and optional codebooks (k, v) as float32 arrays
    [n_layers, n_heads, stages, N, dim] (N = 256 or 1024 codewords per stage),
    or, pooled (one codebook per layer shared by its heads), arrays
    [n_layers, 1, stages, N, dim] with the head count given as n_heads."""

    def __init__(self, N: int, r: float = None, span_len: int = None, codebooks=None, pooled: bool = False,
                 n_heads: int = None):
        L = lib()
        self.N = int(N)
        self.r = float(r) if r is not None else L.fkv_packing_ratio(self.N)
        self.L = int(span_len) if span_len is not None else L.fkv_max_span_len(self.r)
        self._h = ctypes.c_void_p()
        cbp = None
        if codebooks is not None:
            k, v = (np.ascontiguousarray(a, np.float32) for a in codebooks)
            if (k.ndim != 5 or v.ndim != 5 or k.shape[:2] != v.shape[:2] or k.shape[3:] != v.shape[3:]
                    or (pooled and k.shape[1] != 1)):
                raise ValueError("codebooks must be [layers, heads (1 if pooled), stages, codewords, dim]")
            H = int(n_heads) if pooled else k.shape[1]
            if pooled and n_heads is None:
                raise ValueError("pooled codebooks need n_heads")
            self._cb_arrays = (k, v)          # keep alive during create
            cb = _Codebooks(k.shape[0], H, k.shape[4], k.shape[2], v.shape[2],
                            k.ctypes.data, v.ctypes.data, k.shape[3], int(bool(pooled)))
            cbp = ctypes.byref(cb)
            self.n_layers, self.n_heads, self.dim = k.shape[0], H, k.shape[4]
            self.pooled = bool(pooled)
            self.stages_k, self.stages_v = k.shape[2], v.shape[2]
        rc = L.fkv_create(self.N, self.r, self.L, cbp, ctypes.byref(self._h))
        self._cb_arrays = None
        if rc != OK:
            raise FkvError(rc, "fkv_create(N=%d, r=%r, span_len=%d) rejected" % (self.N, self.r, self.L))
        self._dev = torch.cuda.current_device()
        # argument blocks of the paged calls (calls on one context are serialised)
        self._plan = ctypes.create_string_buffer(_PLAN.size)
        self._rows = [ctypes.create_string_buffer(_ROWS.size) for _ in range(2)]
        self._attend = ctypes.create_string_buffer(_ATTEND.size)
        self._caches = [ctypes.create_string_buffer(_CACHE.size) for _ in range(2)]
        self._attend_need = {}
        # symbols are uint8 up to N = 256, uint16 above; torch.int16 holds the
        # uint16 symbols bit for bit (every symbol is below 1024)
        self.sym_bytes = L.fkv_symbol_bytes(self._h)
        self.sym_dtype = torch.uint8 if self.sym_bytes == 1 else torch.int16

    # -- plumbing
    def _check(self, rc):
        if rc != OK:
            raise FkvError(rc, lib().fkv_last_error(self._h).decode())

    def _sym(self, t: torch.Tensor) -> torch.Tensor:
        if t.element_size() != self.sym_bytes:
            raise ValueError("symbols of this context are %d-byte integers, got %s" % (self.sym_bytes, t.dtype))
        return t

    def close(self):
        if self._h:
            lib().fkv_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def handle(self):
        return self._h

    # -- ABI calls
    def vertices(self) -> np.ndarray:
        out = np.empty((self.N, 2), np.float64)
        self._check(lib().fkv_vertices(self._h, out.ctypes.data))
        return out

    def record_len(self) -> int:
        return lib().fkv_record_len(self._h)

    def sync_status(self, stream=None) -> int:
        return lib().fkv_sync_status(self._h, _stream(stream))

    def check_bounded_wait(self, limit_ns: int, stream=None) -> list:
        """fkv_check_bounded_wait: the six results, as ints."""
        res = (ctypes.c_int32 * 6)()
        self._check(lib().fkv_check_bounded_wait(self._h, int(limit_ns), res, _stream(stream)))
        return list(res)

    def n_spans(self, n: int) -> int:
        return (int(n) + self.L - 1) // self.L

    def span_encode(self, sym: torch.Tensor, pts: torch.Tensor = None, stream=None) -> torch.Tensor:
        """sym [n_streams, n] (sym_dtype) -> pts float64 [n_streams, spans, 2]."""
        ns, n = self._sym(sym).shape
        if pts is None:
            pts = torch.empty((ns, self.n_spans(n), 2), dtype=torch.float64, device=sym.device)
        self._check(lib().fkv_span_encode(self._h, _ptr(sym), ns, n, _rows(sym), _ptr(pts), _rows(pts, 2),
                                          _stream(stream)))
        return pts

    def span_decode(self, pts: torch.Tensor, n: int, sym: torch.Tensor = None, stream=None) -> torch.Tensor:
        ns = pts.shape[0]
        if sym is None:
            sym = torch.empty((ns, n), dtype=self.sym_dtype, device=pts.device)
        self._sym(sym)
        self._check(lib().fkv_span_decode(self._h, _ptr(pts), ns, n, _rows(pts, 2), _ptr(sym), _rows(sym),
                                          _stream(stream)))
        return sym

    def read(self, pts: torch.Tensor, n: int, req: torch.Tensor, out: torch.Tensor = None, stream=None):
        """req int64 [n_req, 2] = (stream, position) -> symbols [n_req] (sym_dtype)."""
        if out is None:
            out = torch.empty(req.shape[0], dtype=self.sym_dtype, device=pts.device)
        self._sym(out)
        self._check(lib().fkv_read(self._h, _ptr(pts), pts.shape[0], n, _rows(pts, 2), _ptr(req), req.shape[0],
                                   _ptr(out), _stream(stream)))
        return out

    # -- ragged batches (streams of different lengths in one call)
    def ragged_offsets(self, lengths, device="cuda"):
        """Packed offsets for streams of the given lengths: (sym_off, pt_off),
        int64 [n_streams + 1] device tensors (points packed with no slack)."""
        ln = np.asarray(lengths, np.int64).ravel()
        so = np.concatenate([[0], np.cumsum(ln)]).astype(np.int64)
        po = np.concatenate([[0], np.cumsum((ln + self.L - 1) // self.L)]).astype(np.int64)
        return torch.from_numpy(so).to(device), torch.from_numpy(po).to(device)

    def span_encode_ragged(self, sym: torch.Tensor, sym_off: torch.Tensor, pt_off: torch.Tensor,
                           pts: torch.Tensor = None, n_slots: int = None, stream=None) -> torch.Tensor:
        """sym: flat symbols (sym_dtype) of all streams; sym_off, pt_off: int64
        [n_streams + 1] device offsets -> pts float64 [slots, 2] (n_slots, or
        pt_off's last entry read back, a synchronisation, when pts is None)."""
        self._sym(sym)
        ns = sym_off.numel() - 1
        if pts is None:
            slots = int(pt_off[-1].item()) if n_slots is None else int(n_slots)
            pts = torch.empty((max(slots, 1), 2), dtype=torch.float64, device=sym.device)
        self._check(lib().fkv_span_encode_ragged(self._h, _ptr(sym), _ptr(sym_off), ns, _ptr(pts), _ptr(pt_off),
                                                 _stream(stream)))
        return pts

    def span_decode_ragged(self, pts: torch.Tensor, pt_off: torch.Tensor, sym_off: torch.Tensor,
                           sym: torch.Tensor = None, n_sym: int = None, stream=None) -> torch.Tensor:
        ns = sym_off.numel() - 1
        if sym is None:
            n = int(sym_off[-1].item()) if n_sym is None else int(n_sym)
            sym = torch.empty(max(n, 1), dtype=self.sym_dtype, device=pts.device)
        self._sym(sym)
        self._check(lib().fkv_span_decode_ragged(self._h, _ptr(pts), _ptr(pt_off), ns, _ptr(sym), _ptr(sym_off),
                                                 _stream(stream)))
        return sym

    def read_ragged(self, pts: torch.Tensor, pt_off: torch.Tensor, sym_off: torch.Tensor, req: torch.Tensor,
                    out: torch.Tensor = None, stream=None) -> torch.Tensor:
        """req int64 [n_req, 2] = (stream, position within it) -> symbols [n_req]."""
        if out is None:
            out = torch.empty(req.shape[0], dtype=self.sym_dtype, device=pts.device)
        self._sym(out)
        self._check(lib().fkv_read_ragged(self._h, _ptr(pts), _ptr(pt_off), _ptr(sym_off), sym_off.numel() - 1,
                                          _ptr(req), req.shape[0], _ptr(out), _stream(stream)))
        return out

    def suffix_search(self, pts: torch.Tensor, n: int, query, cap: int = 1 << 16, match: torch.Tensor = None,
                      counts: torch.Tensor = None, stream=None):
        """Sec. 5 in-place retrieval: spans whose last len(query) symbols equal
        the query.  Returns (match int64 [min(count, cap), 2] = (stream, span)
        in no particular order, number of matches, number of candidates); reads
        the two counts back (a device synchronisation on `stream`)."""
        q = np.asarray(query).ravel()
        if q.size and (q.min() < 0 or q.max() >= 1 << (8 * self.sym_bytes)):
            raise ValueError("query symbol does not fit the symbol width")
        q = np.ascontiguousarray(q.astype(np.uint8 if self.sym_bytes == 1 else np.uint16))
        if match is None:
            match = torch.empty((max(cap, 1), 2), dtype=torch.int64, device=pts.device)
        if counts is None:
            counts = torch.empty(2, dtype=torch.int64, device=pts.device)
        self._check(lib().fkv_suffix_search(self._h, _ptr(pts), pts.shape[0], n, _rows(pts, 2),
                                            q.ctypes.data_as(ctypes.c_void_p), q.size, _ptr(match), cap,
                                            _ptr(counts), _stream(stream)))
        c = counts.cpu().tolist()
        return match[:min(c[0], cap)], c[0], c[1]

    # -- Sec. 6 probability-weighted maps (arithmetic coding)
    def ac_encode(self, sym: torch.Tensor, adaptive: bool = True, words: torch.Tensor = None,
                  nbits: torch.Tensor = None, stream=None):
        """sym [n_streams, n] -> (words int32 [n_streams, capacity] holding the
        uint32 code words, nbits int64 [n_streams])."""
        ns, n = self._sym(sym).shape
        cap = lib().fkv_ac_capacity_words(self._h, n)
        if words is None:
            words = torch.zeros((ns, cap), dtype=torch.int32, device=sym.device)
        if nbits is None:
            nbits = torch.empty(ns, dtype=torch.int64, device=sym.device)
        self._check(lib().fkv_ac_encode(self._h, _ptr(sym), ns, n, _rows(sym), int(bool(adaptive)), _ptr(words),
                                        _rows(words), _ptr(nbits), _stream(stream)))
        return words, nbits

    def ac_decode(self, words: torch.Tensor, nbits: torch.Tensor, n: int, adaptive: bool = True,
                  sym: torch.Tensor = None, stream=None) -> torch.Tensor:
        ns = words.shape[0]
        if sym is None:
            sym = torch.empty((ns, n), dtype=self.sym_dtype, device=words.device)
        self._sym(sym)
        self._check(lib().fkv_ac_decode(self._h, _ptr(words), _rows(words), _ptr(nbits), ns, n, int(bool(adaptive)),
                                        _ptr(sym), _rows(sym), _stream(stream)))
        return sym

    # -- Sec. 4 lossy archive
    def lossy_geometry(self, n: int, bits: int, keep_exact: int):
        """(truncated spans T, code words per stream, exact tail spans)."""
        S = self.n_spans(n)
        T = max(0, S - int(keep_exact))
        return T, (2 * T * int(bits) + 31) // 32, S - T

    def truncate(self, pts: torch.Tensor, n: int, bits: int, keep_exact: int, codes: torch.Tensor = None,
                 tail: torch.Tensor = None, stream=None):
        """pts float64 [n_streams, spans, 2] -> (codes int32 [n_streams, words]
        holding the uint32 code words, tail float64 [n_streams, S - T, 2])."""
        ns = pts.shape[0]
        T, words, ts = self.lossy_geometry(n, bits, keep_exact)
        if codes is None:
            codes = torch.empty((ns, max(words, 1)), dtype=torch.int32, device=pts.device)
        if tail is None:
            tail = torch.empty((ns, max(ts, 1), 2), dtype=torch.float64, device=pts.device)
        self._check(lib().fkv_truncate(self._h, _ptr(pts), ns, n, _rows(pts, 2), int(bits), int(keep_exact),
                                       _ptr(codes), _rows(codes), _ptr(tail), _rows(tail, 2), _stream(stream)))
        return codes, tail

    def lossy_decode(self, codes: torch.Tensor, tail: torch.Tensor, n: int, bits: int, keep_exact: int,
                     sym: torch.Tensor = None, stream=None) -> torch.Tensor:
        ns = codes.shape[0]
        if sym is None:
            sym = torch.empty((ns, n), dtype=self.sym_dtype, device=codes.device)
        self._sym(sym)
        self._check(lib().fkv_lossy_decode(self._h, _ptr(codes), _rows(codes), _ptr(tail), _rows(tail, 2), ns, n,
                                           int(bits), int(keep_exact), _ptr(sym), _rows(sym), _stream(stream)))
        return sym

    def lossy_read(self, codes: torch.Tensor, tail: torch.Tensor, n: int, bits: int, keep_exact: int,
                   req: torch.Tensor, out: torch.Tensor = None, stream=None) -> torch.Tensor:
        if out is None:
            out = torch.empty(req.shape[0], dtype=self.sym_dtype, device=codes.device)
        self._sym(out)
        self._check(lib().fkv_lossy_read(self._h, _ptr(codes), _rows(codes), _ptr(tail), _rows(tail, 2),
                                         codes.shape[0], n, int(bits), int(keep_exact), _ptr(req), req.shape[0],
                                         _ptr(out), _stream(stream)))
        return out

    def rvq_encode(self, kv: int, x: torch.Tensor, t0: int, t1: int, sym: torch.Tensor, rec0: int = 0, stream=None):
        """x: cache [layers, batch, heads, seq, dim]; sym: [batch*layers, >= (rec0+t1-t0)*R] of sym_dtype."""
        self._sym(sym)
        c = cache_view(x)
        self._check(lib().fkv_rvq_encode(self._h, int(kv), ctypes.byref(c), t0, t1, _ptr(sym), _rows(sym), rec0,
                                         _stream(stream)))
        return sym

    def rvq_decode(self, sym: torch.Tensor, n_rec: int, k_out: torch.Tensor = None, v_out: torch.Tensor = None,
                   t0: int = 0, stream=None):
        self._sym(sym)
        ck = cache_view(k_out) if k_out is not None else None
        cv = cache_view(v_out) if v_out is not None else None
        self._check(lib().fkv_rvq_decode(self._h, _ptr(sym), _rows(sym), n_rec,
                                         ctypes.byref(ck) if ck else None, ctypes.byref(cv) if cv else None,
                                         t0, _stream(stream)))

    def decode_kv(self, pts: torch.Tensor, n_rec: int, k_out: torch.Tensor = None, v_out: torch.Tensor = None,
                  t0: int = 0, stream=None):
        ck = cache_view(k_out) if k_out is not None else None
        cv = cache_view(v_out) if v_out is not None else None
        self._check(lib().fkv_decode_kv(self._h, _ptr(pts), n_rec, _rows(pts, 2),
                                        ctypes.byref(ck) if ck else None, ctypes.byref(cv) if cv else None,
                                        t0, _stream(stream)))

    def decode_kv_static(self, pts: torch.Tensor, n_rec: int, k_out: torch.Tensor = None,
                         v_out: torch.Tensor = None, t0: int = 0, stream=None):
        """decode_kv without any device allocation: the decoded symbols go
        through the library's fixed 16 MiB scratch array (for callers whose
        device memory must all come from their own allocator)."""
        ck = cache_view(k_out) if k_out is not None else None
        cv = cache_view(v_out) if v_out is not None else None
        self._check(lib().fkv_decode_kv_static(self._h, _ptr(pts), n_rec, _rows(pts, 2),
                                               ctypes.byref(ck) if ck else None, ctypes.byref(cv) if cv else None,
                                               t0, _stream(stream)))

    def cache_upload(self, src_host: torch.Tensor, dst: torch.Tensor, t0: int, t1: int, stream=None):
        """Copy positions [t0, t1) of a host cache (CPU tensor, pinned) into a device cache."""
        cs, cd = cache_view(src_host, host=True), cache_view(dst)
        self._check(lib().fkv_cache_upload(self._h, ctypes.byref(cs), ctypes.byref(cd), t0, t1, _stream(stream)))
        return dst

    def read_kv(self, pts: torch.Tensor, n_rec: int, req: torch.Tensor, out: torch.Tensor, stream=None):
        """req int64 [n_req, 2] = (stream, record) -> out [n_req, 2, heads, dim]."""
        self._check(lib().fkv_read_kv(self._h, _ptr(pts), pts.shape[0], n_rec, _rows(pts, 2), _ptr(req),
                                      req.shape[0], _ptr(out), _DTYPE[out.dtype], _stream(stream)))
        return out

    # -- paged 8-bit cache (all tensors on the context's device)
    def _on(self, pages: Pages) -> int:
        if pages.device != self._dev:
            raise ValueError("the pages are on cuda:%d, the context on cuda:%d" % (pages.device, self._dev))
        return self._dev

    def _empty(self, shape, dtype, stream) -> torch.Tensor:
        """Memory for a call on `stream`: the allocator gives out what is free, and takes it back, in that
        stream's order, not in the current one's."""
        if stream is None:
            return torch.empty(shape, dtype=dtype, device=self._dev)
        with torch.cuda.stream(stream):
            return torch.empty(shape, dtype=dtype, device=self._dev)

    def page_plan(self, n_new: torch.Tensor, kv_len: torch.Tensor, block_table: torch.Tensor, free: torch.Tensor,
                  taken: torch.Tensor, block: int, cu: torch.Tensor, slots: torch.Tensor, positions: torch.Tensor,
                  kv_len_out: torch.Tensor = None, taken_out: torch.Tensor = None, stream=None):
        """Pages, slots and positions of n_new[r] more tokens of every request
        (n_new[r] < 0: it ends) whose first kv_len[r] positions are in pages of
        `block`.  int32 arrays, slots int64; block_table [requests, pages] and the
        stack `free` are updated, kv_len and taken in place unless their outputs
        are given.  slots and positions may have more rows than there are tokens:
        -1 behind the last."""
        n, rows = n_new.numel(), slots.numel()
        dev = self._dev
        tp, ts, tw = _table(block_table, n, dev)
        if positions.numel() != rows:
            raise ValueError("slots and positions must have the same length")
        lp, kp = _array(kv_len, _I32, n, "kv_len", dev), _array(taken, _I32, 1, "taken", dev)
        _PLAN.pack_into(
            self._plan, 0, _array(n_new, _I32, n, "n_new", dev), lp, tp, _array(free, _I32, 0, "free", dev), kp,
            _array(cu, _I32, n + 1, "cu", dev), _array(slots, _INT64, 0, "slots", dev), _array(positions, _I32, 0, "positions", dev),
            lp if kv_len_out is None else _array(kv_len_out, _I32, n, "kv_len_out", dev),
            kp if taken_out is None else _array(taken_out, _I32, 1, "taken_out", dev), n, ts, tw, free.numel(), rows, block)
        rc = lib().fkv_page_plan(self._h, self._plan, _stream(stream))
        if rc != OK:
            self._check(rc)

    def page_write(self, pages: Pages, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, stream=None):
        """Quantise k and v [tokens, heads, dim] into the pages' slots (int64 [tokens], negative: skipped)."""
        dev = self._on(pages)
        kp, kd, shape, kt, kh = _vectors(k, pages.dim, "k", dev)
        vp, vd, vshape, vt, vh = _vectors(v, pages.dim, "v", dev)
        n = shape[0]
        if vshape != shape or shape[1] != pages.heads:
            raise ValueError("k and v must be [tokens, %d, %d]" % (pages.heads, pages.dim))
        _ROWS.pack_into(self._rows[0], 0, kp, kd, kt, kh)
        _ROWS.pack_into(self._rows[1], 0, vp, vd, vt, vh)
        rc = lib().fkv_page_write(self._h, pages._addr, self._rows[0], self._rows[1],
                                  _array(slots, _INT64, n, "slots", dev), n, _stream(stream))
        if rc != OK:
            self._check(rc)

    def page_attend(self, pages: Pages, q: torch.Tensor, cu: torch.Tensor, kv_len: torch.Tensor,
                    block_table: torch.Tensor, max_new: int, max_len: int, out: torch.Tensor = None,
                    lse: torch.Tensor = None, scale: float = None, causal: bool = True, window: int = 0,
                    sinks: int = 0, softcap: float = 0.0, slopes: torch.Tensor = None, prefix: torch.Tensor = None,
                    workspace: torch.Tensor = None, stream=None) -> torch.Tensor:
        """Attention of q [tokens, query heads, dim] (rows cu[r] .. cu[r+1] the
        last tokens of request r's kv_len[r] positions) over the pages; scale
        defaults to dim ** -0.5.  max_new and max_len bound every request's new
        tokens and positions.  lse: float32 [tokens, query heads] or None.  out and
        the workspace are taken from torch's allocator, on the call's stream, unless
        given."""
        dev = self._on(pages)
        n = kv_len.numel()
        dim = pages.dim
        qp, qd, shape, qt, qh = _vectors(q, dim, "q", dev)
        T, Hq = shape[0], shape[1]
        if out is None:
            out = self._empty((T, Hq, dim), q.dtype, stream)
        op, od, oshape, ot, oh = _vectors(out, dim, "out", dev)
        if oshape != shape or od != qd:
            raise ValueError("out must have q's shape and type")
        tp, ts, tw = _table(block_table, n, dev)
        buf = self._attend
        _ATTEND.pack_into(
            buf, 0, pages._addr, qp, op, 0 if lse is None else _array(lse, _FLOAT, T * Hq, "lse", dev),
            _array(cu, _I32, n + 1, "cu", dev), _array(kv_len, _I32, n, "kv_len", dev), tp,
            0 if slopes is None else _array(slopes, _FLOAT, Hq, "slopes", dev),
            0 if prefix is None else _array(prefix, _I32, n, "prefix", dev), qt, qh, ot, oh, T, n, ts, tw, max_new, max_len,
            window, sinks, qd, Hq, causal, dim ** -0.5 if scale is None else scale, softcap, 0)
        L = lib()
        # the workspace's size depends on these alone, in a call that is not refused
        key = (T, Hq, n, max_new, max_len, window, sinks, prefix is None, pages.heads, dim)
        need = self._attend_need.get(key)
        if need is None:
            need = L.fkv_page_attend_workspace(self._h, buf)
        ws = nb = 0
        if workspace is not None:
            if workspace.get_device() != dev or not workspace.is_contiguous():
                raise ValueError("workspace must be a contiguous tensor on cuda:%d" % dev)
            ws, nb = workspace.data_ptr(), workspace.numel() * workspace.element_size()
        elif need:
            workspace = self._empty((need,), torch.uint8, stream)
            ws, nb = workspace.data_ptr(), need
        rc = L.fkv_page_attend(self._h, buf, ws, nb, _stream(stream))
        if rc != OK:
            self._check(rc)
        if key not in self._attend_need:
            if len(self._attend_need) >= 4096:
                self._attend_need.clear()
            self._attend_need[key] = need
        return out

    def page_read(self, pages: Pages, kv_len: torch.Tensor, block_table: torch.Tensor, t0: int, t1: int,
                  layer: int = 0, k_out: torch.Tensor = None, v_out: torch.Tensor = None, stream=None):
        """Rebuild positions [t0, min(t1, kv_len[r])) of request r into sequence r
        of a layer of the caches k_out and v_out [layers, batch, heads, seq, dim]."""
        dev = self._on(pages)
        n = kv_len.numel()
        tp, ts, tw = _table(block_table, n, dev)
        views = [0, 0]
        for i, x in enumerate((k_out, v_out)):
            if x is None:
                continue
            shape, st, dt = x.shape, x.stride(), _DTYPE.get(x.dtype)
            if (len(shape) != 5 or shape[2] != pages.heads or shape[4] != pages.dim or st[4] != 1 or dt is None or
                    not 0 <= layer < shape[0] or x.get_device() != dev):
                raise ValueError("caches must be CUDA tensors [layers, batch, %d, seq, %d] with contiguous dim that "
                                 "hold the layer" % (pages.heads, pages.dim))
            _CACHE.pack_into(self._caches[i], 0, x.data_ptr(), dt, shape[1], shape[3], st[0], st[1], st[2], st[3])
            views[i] = self._caches[i]
        rc = lib().fkv_page_read(self._h, pages._addr, _array(kv_len, _I32, n, "kv_len", dev), n, tp, ts, tw, t0, t1, layer,
                                 views[0] or None, views[1] or None, _stream(stream))
        if rc != OK:
            self._check(rc)


class Streams:
    """An fkv_streams set: n_streams library-owned appendable streams."""

    def __init__(self, ctx: Context, n_streams: int, capacity: int = 0, _handle=None):
        self.ctx = ctx
        self._h = ctypes.c_void_p()
        if _handle is not None:
            self._h = _handle
        else:
            ctx._check(lib().fkv_streams_create(ctx.handle, n_streams, capacity, ctypes.byref(self._h)))

    @classmethod
    def import_(cls, ctx: Context, length: int, host_pts: np.ndarray):
        h = ctypes.c_void_p()
        p = np.ascontiguousarray(host_pts, np.float64)
        ctx._check(lib().fkv_streams_import(ctx.handle, p.shape[0], length, p.ctypes.data, ctypes.byref(h)))
        return cls(ctx, p.shape[0], _handle=h)

    def info(self):
        ns, ln, st = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64()
        p = ctypes.c_void_p()
        lib().fkv_streams_info(self._h, ctypes.byref(ns), ctypes.byref(ln), ctypes.byref(st), ctypes.byref(p))
        return ns.value, ln.value, st.value, p.value

    def points(self) -> torch.Tensor:
        """A [n_streams, cap_spans, 2] float64 view of the library-owned point
        buffer (valid until the next growing append)."""
        ns, ln, st, p = self.info()
        return _device_view(p, (ns, st, 2))

    @property
    def length(self) -> int:
        return self.info()[1]

    def reset(self):
        lib().fkv_streams_reset(self._h)

    def append(self, sym: torch.Tensor, stream=None):
        """sym [n_streams, m] of the context's sym_dtype."""
        self.ctx._sym(sym)
        self.ctx._check(lib().fkv_append(self.ctx.handle, self._h, _ptr(sym), sym.shape[1], _rows(sym),
                                         _stream(stream)))

    def export(self, stream=None) -> np.ndarray:
        ns, ln, st, p = self.info()
        out = np.empty((ns, self.ctx.n_spans(ln), 2), np.float64)
        length = ctypes.c_int64()
        self.ctx._check(lib().fkv_streams_export(self._h, ctypes.byref(length), out.ctypes.data, _stream(stream)))
        return out

    def close(self):
        if self._h:
            lib().fkv_streams_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _device_view(ptr: int, shape):
    """Wrap a library-owned float64 device buffer as a torch tensor (no copy)."""
    n = int(np.prod(shape))

    class _Holder:
        __cuda_array_interface__ = {"shape": tuple(shape), "typestr": "<f8", "data": (ptr, False),
                                    "version": 3, "strides": None}
    if n == 0:
        return torch.empty(shape, dtype=torch.float64, device="cuda")
    return torch.as_tensor(_Holder(), device="cuda")

"""ctypes binding of libfkv (include/fkv.h), with the C names.

Argument marshalling only: every step of the archive path runs in the HIP
kernels of libfkv.so.  PyTorch provides device memory and the current HIP
stream; what a call makes itself (results, scratch) lies in the memory of the
stream that it runs on, the current one or that of `stream=`, a raw handle.
Importing this module loads the library and raises ImportError when
it has not been built -- there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
from typing import NamedTuple

import numpy as np

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libfkv.so")
if not os.path.exists(_LIB_PATH):
    raise ImportError("libfkv.so is not built (run paper_2607_07144_amd.build.build() or "
                      "__graft_entry__.build()); there is no fallback implementation")
lib = ctypes.CDLL(_LIB_PATH)

FKV_OK = 0
FKV_ERR_INVALID_ARG = -1
FKV_ERR_UNSUPPORTED = -2
FKV_ERR_LAUNCH = -3
FKV_ERR_NO_DEVICE = -4
FKV_ERR_SCRATCH_TOO_SMALL = -5


class fkv_codec(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int32), ("L", ctypes.c_int32), ("r", ctypes.c_double),
                ("r_max", ctypes.c_double)]


class fkv_rvq_desc(ctypes.Structure):
    _fields_ = [("n_streams", ctypes.c_int64), ("T", ctypes.c_int64), ("t_begin", ctypes.c_int64),
                ("t_end", ctypes.c_int64), ("d", ctypes.c_int32), ("S", ctypes.c_int32),
                ("K", ctypes.c_int32), ("n_books", ctypes.c_int32)]


FKV_PAGE_INT8, FKV_PAGE_E4M3 = 0, 1
FKV_ROW_F16, FKV_ROW_BF16 = 0, 1
FKV_ROTATE_HALVES, FKV_ROTATE_PAIRS = 0, 1


class fkv_page_desc(ctypes.Structure):
    _fields_ = [("n_pages", ctypes.c_int64), ("page", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("d", ctypes.c_int32), ("format", ctypes.c_int32)]


class fkv_row_desc(ctypes.Structure):
    _fields_ = [("group", ctypes.c_int64), ("stride_group", ctypes.c_int64), ("stride_token", ctypes.c_int64),
                ("stride_head", ctypes.c_int64), ("type", ctypes.c_int32)]


class fkv_rotate_desc(ctypes.Structure):
    _fields_ = [("n_pos", ctypes.c_int64), ("rot", ctypes.c_int32), ("pairing", ctypes.c_int32),
                ("q_heads", ctypes.c_int32)]


class fkv_attend_desc(ctypes.Structure):
    _fields_ = [("n_req", ctypes.c_int64), ("n_tokens", ctypes.c_int64), ("max_new", ctypes.c_int64),
                ("max_kv", ctypes.c_int64), ("max_pages", ctypes.c_int64), ("q_stride_token", ctypes.c_int64),
                ("q_stride_head", ctypes.c_int64), ("o_stride_token", ctypes.c_int64),
                ("o_stride_head", ctypes.c_int64), ("q_heads", ctypes.c_int32), ("type", ctypes.c_int32),
                ("scale", ctypes.c_float), ("softcap", ctypes.c_float), ("causal", ctypes.c_int32),
                ("window", ctypes.c_int32), ("sinks", ctypes.c_int32)]


class fkv_select_desc(ctypes.Structure):
    _fields_ = [("n_req", ctypes.c_int64), ("n_tokens", ctypes.c_int64), ("max_new", ctypes.c_int64),
                ("max_kv", ctypes.c_int64), ("max_pages", ctypes.c_int64), ("q_stride_token", ctypes.c_int64),
                ("q_stride_head", ctypes.c_int64), ("q_heads", ctypes.c_int32), ("type", ctypes.c_int32),
                ("causal", ctypes.c_int32), ("n_select", ctypes.c_int32), ("keep_first", ctypes.c_int32),
                ("keep_last", ctypes.c_int32)]


_i32, _i64, _dbl, _p, _sz = ctypes.c_int32, ctypes.c_int64, ctypes.c_double, ctypes.c_void_p, ctypes.c_size_t
_PC = ctypes.POINTER(fkv_codec)
_SIGS = {
    "fkv_codec_init": ([_i32, _dbl, _i32, _PC], ctypes.c_int),
    "fkv_codec_table_bytes": ([_PC], _sz),
    "fkv_codec_fill_table": ([_PC, _p], ctypes.c_int),
    "fkv_num_spans": ([_PC, _i64], _i64),
    "fkv_rvq_assign": ([ctypes.POINTER(fkv_rvq_desc), _p, _p, _p, _p, _p, _p, _p], ctypes.c_int),
    "fkv_rvq_assign_stages": ([ctypes.POINTER(fkv_rvq_desc), _i32, _p, _p, _p, _p, _p, _p, _p], ctypes.c_int),
    "fkv_rvq_assign_encode_fused": ([ctypes.POINTER(fkv_rvq_desc), _p], ctypes.c_int),
    "fkv_rvq_assign_groups": ([ctypes.POINTER(fkv_rvq_desc), _p, _i64, _i32, _p, _p, _p, _p, _p, _p, _p],
                              ctypes.c_int),
    "fkv_rvq_assign_encode": ([ctypes.POINTER(fkv_rvq_desc), _p, _p, _p, _PC, _p, _p, _p, _p, _p, _p],
                              ctypes.c_int),
    "fkv_cgr_encode_spans": ([_PC, _p, _p, _i64, _i64, _p, _p], ctypes.c_int),
    "fkv_cgr_decode_spans": ([_PC, _p, _p, _i64, _i64, _p, _p, _p, _i32, _p], ctypes.c_int),
    "fkv_span_lookup": ([_PC, _p, _p, _i64, _i64, _i32, _p, _p, _i64, _p, _p, _p, _p], ctypes.c_int),
    "fkv_rehydrate": ([_PC, _p, _p, _i64, _i64, _i32, _p, _p, _i32, _i32, _i32, _p, _p, _i64, _p, _p, _p, _p],
                      ctypes.c_int),
    "fkv_cgr_append": ([_PC, _p, _p, _i64, _i64, _i64, _p, _i64, _p], ctypes.c_int),
    "fkv_trajectory": ([_PC, _p, _p, _i64, _i64, _i32, _p, _p], ctypes.c_int),
    "fkv_suffix_search": ([_PC, _p, _p, _i64, _i64, _p, _i32, _i32, _p, _i64, _p, _p, _p], ctypes.c_int),
    "fkv_kmeans_accumulate": ([ctypes.POINTER(fkv_rvq_desc), _p, _p, _p, _p, _i32, _p, _p, _p], ctypes.c_int),
    "fkv_kmeans_finalize": ([_i32, _i32, _i32, _i32, _i32, _p, _p, _p, _p], ctypes.c_int),
    "fkv_kmeans_update_noalloc": ([ctypes.POINTER(fkv_rvq_desc), _p, _p, _p, _p, _i32, _p, _p], ctypes.c_int),
    "fkv_kmeans_update_noalloc_bytes": ([_i32, _i32, _i32], _sz),
    "fkv_page_plan": ([_i32, _i64, _p, _p, _p, _i64, _p, _p, _i64, _i64, _p, _p, _p, _p, _p, _p, _p, _p, _p],
                      ctypes.c_int),
    "fkv_page_store": ([_p, _p, _p, _p, _p, _i64, _p, _p, _p, _p, _p, _p], ctypes.c_int),
    "fkv_page_append": ([_p, _p, _p, _p, _p, _p, _p, _p, _p, _p, _i64, _p, _p, _p, _p, _p, _p, _p, _p, _p], ctypes.c_int),
    "fkv_page_load": ([_p, _p, _p, _p, _i64, _p, _p, _p, _p, _p, _p], ctypes.c_int),
    "fkv_page_attend_workspace": ([_p, _p], _sz),
    "fkv_page_attend": ([_p, _p, _p, _p, _p, _p, _p, _p, _p, _p, _p, _p, _p, _p, _p, _sz, _p], ctypes.c_int),
    "fkv_page_select_workspace": ([_p, _p], _sz),
    "fkv_page_select": ([_p, _p, _p, _p, _p, _p, _p, _p, _p, _p, _sz, _p], ctypes.c_int),
    "fkv_page_attend_selected_workspace": ([_p, _p, _i64], _sz),
    "fkv_page_attend_selected": ([_p, _p, _i64, _p, _p, _p, _p, _p, _p, _p, _p, _p, _p, _p, _p, _p, _p, _sz, _p],
                                 ctypes.c_int),
    "fkv_diag_mfma_loop": ([_i32, _i32, _i32, ctypes.c_float, ctypes.c_float, _p, _p], ctypes.c_int),
    "fkv_diag_mfma_loop_flops": ([_i32, _i32], _dbl),
    "fkv_status_string": ([ctypes.c_int], ctypes.c_char_p),
    "fkv_version": ([], ctypes.c_char_p),
}
for _name, (_args, _res) in _SIGS.items():
    _f = getattr(lib, _name)
    _f.argtypes = _args
    _f.restype = _res


class FkvError(RuntimeError):
    def __init__(self, status: int, where: str):
        super().__init__("%s: %s (%d)" % (where, lib.fkv_status_string(status).decode(), status))
        self.status = status


def _check(status: int, where: str) -> None:
    if status != FKV_OK:
        raise FkvError(status, where)


# A small call's time is mostly this marshalling, so it builds no objects that
# it can do without: addresses go to ctypes as plain integers (the argument
# types convert them), and the current stream is read as its raw handle instead
# of through a Stream object.  Measured on the decoding-step eviction of 288
# streams (two calls): 19.7 -> 14.4 us; a lookup of 1500 tokens 11.7 -> 8.9 us.
_TORCH = None


def _torch():
    global _TORCH
    if _TORCH is None:
        import torch
        _TORCH = torch
    return _TORCH


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream):
    if stream is not None:
        return int(stream)
    torch = _TORCH or _torch()
    C = torch._C
    raw = getattr(C, "_cuda_getCurrentRawStream", None)
    if raw is None:
        return torch.cuda.current_stream().cuda_stream
    device = getattr(C, "_cuda_getDevice", None)
    return raw(device() if device is not None else torch.cuda.current_device())


def _need(t, dtype, name):
    try:
        if t.is_cuda and t.dtype is dtype and t.is_contiguous():
            return
    except AttributeError:   # no tensor
        pass
    raise TypeError("%s must be a contiguous CUDA tensor of %s" % (name, dtype))


def _here(*tensors) -> None:
    """Refuses tensors of another device than the current one, whose stream and scratch a call takes."""
    torch = _TORCH or _torch()
    device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)()
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError("tensor on device %d, the current device is %d" % (t.get_device(), device))


def _on(stream, device):
    """torch's stream of a raw handle, to be current while a call makes or clears tensors (torch takes the handle 0 of the
    default stream for a new stream's)."""
    cuda = (_TORCH or _torch()).cuda
    return cuda.stream(cuda.ExternalStream(int(stream), device=device) if stream else cuda.default_stream(device))


def _new(shape, dtype, device, stream, zero=False):
    """A tensor that a call makes, from the memory of the stream that it runs on, as its kernels write it there: of another
    stream's memory, that one's work on what it held before might not be done.  (What reads a result on a third stream
    waits for it, and keeps it until it is done, as with torch.cuda.stream.  The paged calls make theirs in place where no
    stream is given: a small call's time is such lines.)"""
    torch = _TORCH or _torch()
    make = torch.zeros if zero else torch.empty
    if stream is None:
        return make(shape, dtype=dtype, device=device)
    with _on(stream, device):
        return make(shape, dtype=dtype, device=device)


def _clear(t, stream) -> None:
    """Zeros, on the stream that the call runs on."""
    if stream is None:
        t.zero_()
        return
    with _on(stream, t.device):
        t.zero_()


# ------------------------------------------------------------------ codec

class Codec:
    """Host codec parameters (a fkv_codec) plus the device table built from them."""

    def __init__(self, N: int, r_scale: float = 0.98, L_override: int = 0):
        self.c = fkv_codec()
        _check(lib.fkv_codec_init(N, r_scale, L_override, ctypes.byref(self.c)), "fkv_codec_init")
        self._table = None

    N = property(lambda self: self.c.N)
    L = property(lambda self: self.c.L)
    r = property(lambda self: self.c.r)
    r_max = property(lambda self: self.c.r_max)

    def n_spans(self, n_sym: int) -> int:
        return int(lib.fkv_num_spans(ctypes.byref(self.c), n_sym))

    def host_table(self) -> np.ndarray:
        n = lib.fkv_codec_table_bytes(ctypes.byref(self.c))
        buf = np.zeros(n, np.uint8)
        _check(lib.fkv_codec_fill_table(ctypes.byref(self.c), buf.ctypes.data), "fkv_codec_fill_table")
        return buf

    def table(self, device="cuda"):
        """The device copy of the table (built once per Codec)."""
        if self._table is None:
            torch = _torch()
            self._table = torch.from_numpy(self.host_table()).to(device)
        return self._table


def fkv_codec_init(N: int, r_scale: float = 0.98, L_override: int = 0) -> Codec:
    return Codec(N, r_scale, L_override)


# ------------------------------------------------------------------ a2: residual VQ

def fkv_rvq_assign(x, books, stream_book, t_begin: int, t_end: int, symbols=None, residual=None,
                   want_residual: bool = False, n_bad=None, n_stages=None, stream=None):
    """x f16 [n_streams][T][d], books f16 [n_books][S][K][d], stream_book i32 [n_streams] (all CUDA).
    Returns (symbols u8 [n_streams][(t_end-t_begin)*S], residual f32 or None).  With n_stages (1..S),
    only the first n_stages stages are assigned (fkv_rvq_assign_stages): the other symbol bytes are left
    as they are and the residual is the one after n_stages stages."""
    torch = _torch()
    _need(x, torch.float16, "x")
    _need(books, torch.float16, "books")
    _need(stream_book, torch.int32, "stream_book")
    ns, T, d = x.shape
    nb, S, K, d2 = books.shape
    if d2 != d or stream_book.shape != (ns,):
        raise ValueError("shape mismatch between x, books and stream_book")
    Ta = t_end - t_begin
    if symbols is None:
        symbols = _new((ns, Ta * S), torch.uint8, x.device, stream)
    _need(symbols, torch.uint8, "symbols")
    if symbols.numel() != ns * Ta * S:
        raise ValueError("symbols has the wrong size")
    if residual is None and want_residual:
        residual = _new((ns, Ta, d), torch.float32, x.device, stream)
    if residual is not None:
        _need(residual, torch.float32, "residual")
        if residual.numel() != ns * Ta * d:
            raise ValueError("residual has the wrong size")
    if n_bad is not None:
        _need(n_bad, torch.int32, "n_bad")
    desc = fkv_rvq_desc(ns, T, t_begin, t_end, d, S, K, nb)
    if n_stages is None:
        _check(lib.fkv_rvq_assign(ctypes.byref(desc), _ptr(x), _ptr(books), _ptr(stream_book), _ptr(symbols),
                                  _ptr(residual), _ptr(n_bad), _stream(stream)), "fkv_rvq_assign")
    else:
        _check(lib.fkv_rvq_assign_stages(ctypes.byref(desc), n_stages, _ptr(x), _ptr(books), _ptr(stream_book),
                                         _ptr(symbols), _ptr(residual), _ptr(n_bad), _stream(stream)),
               "fkv_rvq_assign_stages")
    return symbols, residual


def book_groups(stream_book) -> "np.ndarray":
    """Host-side grouping for fkv_rvq_assign_groups: the streams of each book that has any, in stream order,
    as int32 [n_used_books][members] (every used book must have the same number of streams)."""
    import numpy as np
    sb = np.asarray(stream_book).reshape(-1)
    order = np.argsort(sb, kind="stable")
    books, counts = np.unique(sb, return_counts=True)
    if counts.size == 0:
        return np.zeros((0, 1), np.int32)
    if (counts != counts[0]).any():
        raise ValueError("books have different numbers of streams")
    return order.reshape(books.size, counts[0]).astype(np.int32)


def fkv_rvq_assign_groups(x, books, stream_book, groups, t_begin: int, t_end: int, symbols=None, residual=None,
                          want_residual: bool = False, n_bad=None, stream=None):
    """fkv_rvq_assign for the streams listed in groups (i32 [n_groups][group_size], CUDA; the members of a
    group share a book), one block per group's tokens.  Returns (symbols, residual or None) in the layout of
    fkv_rvq_assign; streams not listed keep their symbol bytes."""
    torch = _torch()
    _need(x, torch.float16, "x")
    _need(books, torch.float16, "books")
    _need(stream_book, torch.int32, "stream_book")
    _need(groups, torch.int32, "groups")
    ns, T, d = x.shape
    nb, S, K, d2 = books.shape
    if d2 != d or stream_book.shape != (ns,) or groups.dim() != 2:
        raise ValueError("shape mismatch between x, books, stream_book and groups")
    Ta = t_end - t_begin
    if symbols is None:
        symbols = _new((ns, Ta * S), torch.uint8, x.device, stream)
    _need(symbols, torch.uint8, "symbols")
    if symbols.numel() != ns * Ta * S:
        raise ValueError("symbols has the wrong size")
    if residual is None and want_residual:
        residual = _new((ns, Ta, d), torch.float32, x.device, stream)
    if residual is not None:
        _need(residual, torch.float32, "residual")
        if residual.numel() != ns * Ta * d:
            raise ValueError("residual has the wrong size")
    if n_bad is not None:
        _need(n_bad, torch.int32, "n_bad")
    desc = fkv_rvq_desc(ns, T, t_begin, t_end, d, S, K, nb)
    _check(lib.fkv_rvq_assign_groups(ctypes.byref(desc), _ptr(groups), groups.shape[0], groups.shape[1], _ptr(x),
                                     _ptr(books), _ptr(stream_book), _ptr(symbols), _ptr(residual), _ptr(n_bad),
                                     _stream(stream)), "fkv_rvq_assign_groups")
    return symbols, residual


def fkv_rvq_assign_encode_fused(x, books, t_begin: int, t_end: int, symbols=None) -> bool:
    """Whether fkv_rvq_assign_encode runs its single fused kernel for these shapes (True) or the assignment
    and then the span encode (False); symbols is the output tensor the call would get, if any."""
    ns, T, d = x.shape
    nb, S, K, _ = books.shape
    desc = fkv_rvq_desc(ns, T, t_begin, t_end, d, S, K, nb)
    ptr = _ptr(symbols) if symbols is not None else ctypes.c_void_p(256)   # a fresh tensor is aligned
    r = lib.fkv_rvq_assign_encode_fused(ctypes.byref(desc), ptr)
    if r < 0:
        raise FkvError(r, "fkv_rvq_assign_encode_fused")
    return r == 1


def fkv_rvq_assign_encode(codec: Codec, x, books, stream_book, t_begin: int, t_end: int, symbols=None, points=None,
                          residual=None, want_residual: bool = False, n_bad=None, stream=None):
    """Assignment and span encode in one kernel: returns (symbols, points, residual or None), identical to
    fkv_rvq_assign followed by fkv_cgr_encode_spans."""
    torch = _torch()
    _need(x, torch.float16, "x")
    _need(books, torch.float16, "books")
    _need(stream_book, torch.int32, "stream_book")
    ns, T, d = x.shape
    nb, S, K, d2 = books.shape
    if d2 != d or stream_book.shape != (ns,):
        raise ValueError("shape mismatch between x, books and stream_book")
    Ta = t_end - t_begin
    if symbols is None:
        symbols = _new((ns, Ta * S), torch.uint8, x.device, stream)
    _need(symbols, torch.uint8, "symbols")
    if symbols.numel() != ns * Ta * S:
        raise ValueError("symbols has the wrong size")
    n_spans = codec.n_spans(Ta * S)
    if points is None:
        points = _new((ns, n_spans, 2), torch.float64, x.device, stream)
    _need(points, torch.float64, "points")
    if points.numel() != ns * n_spans * 2:
        raise ValueError("points has the wrong size")
    if residual is None and want_residual:
        residual = _new((ns, Ta, d), torch.float32, x.device, stream)
    if residual is not None:
        _need(residual, torch.float32, "residual")
    if n_bad is not None:
        _need(n_bad, torch.int32, "n_bad")
    desc = fkv_rvq_desc(ns, T, t_begin, t_end, d, S, K, nb)
    _check(lib.fkv_rvq_assign_encode(ctypes.byref(desc), _ptr(x), _ptr(books), _ptr(stream_book),
                                     ctypes.byref(codec.c), _ptr(codec.table(x.device)), _ptr(symbols),
                                     _ptr(points), _ptr(residual), _ptr(n_bad), _stream(stream)),
           "fkv_rvq_assign_encode")
    return symbols, points, residual


# ------------------------------------------------------------------ a3: encode

def fkv_cgr_encode_spans(codec: Codec, symbols, points=None, stream=None):
    """symbols u8 [n_streams][n_sym] -> points f64 [n_streams][n_spans][2]."""
    torch = _torch()
    _need(symbols, torch.uint8, "symbols")
    ns, n_sym = symbols.shape
    if points is None:
        points = _new((ns, codec.n_spans(n_sym), 2), torch.float64, symbols.device, stream)
    _need(points, torch.float64, "points")
    if points.numel() != ns * codec.n_spans(n_sym) * 2:
        raise ValueError("points has the wrong size")
    _check(lib.fkv_cgr_encode_spans(ctypes.byref(codec.c), _ptr(codec.table(symbols.device)), _ptr(symbols),
                                    ns, n_sym, _ptr(points), _stream(stream)), "fkv_cgr_encode_spans")
    return points


# ------------------------------------------------------------------ a4: decode

def fkv_cgr_decode_spans(codec: Codec, points, n_sym: int, symbols=None, span_ok=None, n_failed=None,
                         verify: bool = False, stream=None):
    """points f64 [n_streams][n_spans][2] -> symbols u8 [n_streams][n_sym] (span_ok, n_failed optional)."""
    torch = _torch()
    _need(points, torch.float64, "points")
    ns = points.shape[0]
    if points.numel() != ns * codec.n_spans(n_sym) * 2:
        raise ValueError("points does not match n_sym")
    if symbols is None:
        symbols = _new((ns, n_sym), torch.uint8, points.device, stream)
    _need(symbols, torch.uint8, "symbols")
    if span_ok is not None:
        _need(span_ok, torch.uint8, "span_ok")
    if n_failed is not None:
        _need(n_failed, torch.int32, "n_failed")
    _check(lib.fkv_cgr_decode_spans(ctypes.byref(codec.c), _ptr(codec.table(points.device)), _ptr(points),
                                    ns, n_sym, _ptr(symbols), _ptr(span_ok), _ptr(n_failed),
                                    1 if verify else 0, _stream(stream)), "fkv_cgr_decode_spans")
    return symbols


# ------------------------------------------------------------------ a5: lookup

def fkv_span_lookup(codec: Codec, points, n_sym: int, S: int, q_stream, q_token, out=None, q_status=None,
                    n_failed=None, stream=None):
    """Random access: out u8 [n_q][S] with the S symbols of each (stream, token) query."""
    torch = _torch()
    _need(points, torch.float64, "points")
    _need(q_stream, torch.int32, "q_stream")
    _need(q_token, torch.int32, "q_token")
    nq = q_stream.numel()
    if q_token.numel() != nq:
        raise ValueError("q_stream and q_token differ in length")
    if out is None:
        out = _new((nq, S), torch.uint8, points.device, stream)
    _need(out, torch.uint8, "out")
    if q_status is not None:
        _need(q_status, torch.uint8, "q_status")
    if n_failed is not None:
        _need(n_failed, torch.int32, "n_failed")
    ns = points.shape[0]
    _check(lib.fkv_span_lookup(ctypes.byref(codec.c), _ptr(codec.table(points.device)), _ptr(points), ns,
                               n_sym, S, _ptr(q_stream), _ptr(q_token), nq, _ptr(out), _ptr(q_status),
                               _ptr(n_failed), _stream(stream)), "fkv_span_lookup")
    return out


# ------------------------------------------------------------------ rehydrate / append

def fkv_rehydrate(codec: Codec, points, n_sym: int, S: int, books, stream_book, q_stream, q_token, out=None,
                  q_status=None, n_failed=None, stream=None):
    """Reconstruction of archived positions: out f16 [n_q][d], the sum of each queried token's S
    codewords (symbols read back by random access), correctly rounded to binary16."""
    torch = _torch()
    _need(points, torch.float64, "points")
    _need(books, torch.float16, "books")
    _need(stream_book, torch.int32, "stream_book")
    _need(q_stream, torch.int32, "q_stream")
    _need(q_token, torch.int32, "q_token")
    nb, S2, K, d = books.shape
    if S2 != S:
        raise ValueError("books has %d stages, S = %d" % (S2, S))
    nq = q_stream.numel()
    if q_token.numel() != nq:
        raise ValueError("q_stream and q_token differ in length")
    if out is None:
        out = _new((nq, d), torch.float16, points.device, stream)
    _need(out, torch.float16, "out")
    if q_status is not None:
        _need(q_status, torch.uint8, "q_status")
    if n_failed is not None:
        _need(n_failed, torch.int32, "n_failed")
    ns = points.shape[0]
    if stream_book.numel() != ns:
        raise ValueError("stream_book must have one entry per stream")
    _check(lib.fkv_rehydrate(ctypes.byref(codec.c), _ptr(codec.table(points.device)), _ptr(points), ns, n_sym,
                             S, _ptr(books), _ptr(stream_book), nb, K, d, _ptr(q_stream), _ptr(q_token), nq,
                             _ptr(out), _ptr(q_status), _ptr(n_failed), _stream(stream)), "fkv_rehydrate")
    return out


def fkv_cgr_append(codec: Codec, points, n_old: int, sym_new, stream=None):
    """Append sym_new u8 [n_streams][m] to every stream of n_old symbols; points f64
    [n_streams][cap_spans][2] is updated in place."""
    torch = _torch()
    _need(points, torch.float64, "points")
    _need(sym_new, torch.uint8, "sym_new")
    ns, cap = points.shape[0], points.shape[1]
    if sym_new.dim() != 2 or sym_new.shape[0] != ns:
        raise ValueError("sym_new must be [n_streams][m]")
    _check(lib.fkv_cgr_append(ctypes.byref(codec.c), _ptr(codec.table(points.device)), _ptr(points), cap, ns,
                              n_old, _ptr(sym_new), sym_new.shape[1], _stream(stream)), "fkv_cgr_append")
    return points


# ------------------------------------------------------------------ retrieval

def fkv_trajectory(codec: Codec, symbols, W: int = 0, traj=None, stream=None):
    """Per-position index: traj f64 [n_streams][n_sym][2] (W = 0 selects W = L)."""
    torch = _torch()
    _need(symbols, torch.uint8, "symbols")
    ns, n = symbols.shape
    W = W or codec.L
    if traj is None:
        traj = _new((ns, n, 2), torch.float64, symbols.device, stream)
    _need(traj, torch.float64, "traj")
    _check(lib.fkv_trajectory(ctypes.byref(codec.c), _ptr(codec.table(symbols.device)), _ptr(symbols), ns, n, W,
                              _ptr(traj), _stream(stream)), "fkv_trajectory")
    return traj


def fkv_suffix_search(codec: Codec, traj, query, verify: bool = True, max_hits: int = 1 << 20, hits=None,
                      n_hits=None, n_candidates=None, stream=None):
    """Suffix search: returns (hits u32-as-int32 [max_hits][2], n_hits int32 [1], n_candidates int32 [1]);
    the first min(n_hits, max_hits) rows of hits are (stream, position) pairs in no particular order."""
    torch = _torch()
    _need(traj, torch.float64, "traj")
    _need(query, torch.uint8, "query")
    ns, n = traj.shape[0], traj.shape[1]
    if hits is None:
        hits = _new((max(max_hits, 1), 2), torch.int32, traj.device, stream)
    _need(hits, torch.int32, "hits")
    if n_hits is None:
        n_hits = _new(1, torch.int32, traj.device, stream, zero=True)
    if n_candidates is None:
        n_candidates = _new(1, torch.int32, traj.device, stream, zero=True)
    _check(lib.fkv_suffix_search(ctypes.byref(codec.c), _ptr(codec.table(traj.device)), _ptr(traj), ns, n,
                                 _ptr(query), query.numel(), 1 if verify else 0, _ptr(hits), max_hits,
                                 _ptr(n_hits), _ptr(n_candidates), _stream(stream)), "fkv_suffix_search")
    return hits, n_hits, n_candidates


# ------------------------------------------------------------------ k-means

def fkv_kmeans_step(x, books, stream_book, t_begin: int, t_end: int, symbols, stage: int, sums=None, counts=None,
                    stream=None):
    """One Lloyd update of stage `stage` of `books` (in place) from an assignment `symbols`;
    returns (books, counts).  sums int64 [n_books][K][d] and counts int32 [n_books][K] are
    workspace (zeroed here)."""
    torch = _torch()
    _need(x, torch.float16, "x")
    _need(books, torch.float16, "books")
    _need(stream_book, torch.int32, "stream_book")
    _need(symbols, torch.uint8, "symbols")
    ns, T, d = x.shape
    nb, S, K, d2 = books.shape
    if d2 != d or stream_book.shape != (ns,) or symbols.numel() != ns * (t_end - t_begin) * S:
        raise ValueError("shape mismatch")
    if sums is None:
        sums = _new((nb, K, d), torch.int64, x.device, stream, zero=True)
    else:
        _clear(sums, stream)
    if counts is None:
        counts = _new((nb, K), torch.int32, x.device, stream, zero=True)
    else:
        _clear(counts, stream)
    desc = fkv_rvq_desc(ns, T, t_begin, t_end, d, S, K, nb)
    st = _stream(stream)
    _check(lib.fkv_kmeans_accumulate(ctypes.byref(desc), _ptr(x), _ptr(books), _ptr(stream_book), _ptr(symbols),
                                     stage, _ptr(sums), _ptr(counts), st), "fkv_kmeans_accumulate")
    _check(lib.fkv_kmeans_finalize(nb, S, K, d, stage, _ptr(sums), _ptr(counts), _ptr(books), st),
           "fkv_kmeans_finalize")
    return books, counts


def fkv_kmeans_update_noalloc(x, books, stream_book, t_begin: int, t_end: int, symbols, stage: int, counts=None,
                              stream=None):
    """fkv_kmeans_step without caller workspace: the cluster sums and counts live in the library's fixed
    device scratch (no allocation in the call).  Updates `books` in place; counts int32 [n_books][K] is
    filled when given.  Returns books."""
    torch = _torch()
    _need(x, torch.float16, "x")
    _need(books, torch.float16, "books")
    _need(stream_book, torch.int32, "stream_book")
    _need(symbols, torch.uint8, "symbols")
    ns, T, d = x.shape
    nb, S, K, d2 = books.shape
    if d2 != d or stream_book.shape != (ns,) or symbols.numel() != ns * (t_end - t_begin) * S:
        raise ValueError("shape mismatch")
    if counts is not None:
        _need(counts, torch.int32, "counts")
        if counts.numel() != nb * K:
            raise ValueError("counts must have n_books * K entries")
    desc = fkv_rvq_desc(ns, T, t_begin, t_end, d, S, K, nb)
    _check(lib.fkv_kmeans_update_noalloc(ctypes.byref(desc), _ptr(x), _ptr(books), _ptr(stream_book), _ptr(symbols),
                                         stage, _ptr(counts), _stream(stream)), "fkv_kmeans_update_noalloc")
    return books


# ------------------------------------------------------------------ paged 8-bit cache

class Pages(NamedTuple):
    """A pool of pages: k int8 or float8_e4m3fn [n_pages][heads][page][d], v the same type
    [n_pages][heads][page // 16][d][16], scales f32 [n_pages][heads][2].  Calls take any such triple."""
    k: object
    v: object
    scales: object


class PagePlan(NamedTuple):
    """What fkv_page_plan gives a step: slots i64 [n_tokens], positions i32 [n_tokens], q_start i32 [n_req + 1],
    kv_end i32 [n_req], head i32 [1] (the free-list entry that the requests served reach up to, refused ones before
    them counted; not the next step's head), next_head i32 [1] (the next step's head: entries handed out by now),
    status u8 [n_req] (0: served).  A refused request's rows keep their place in q_start, with slots of -1: attention
    takes them for the last tokens that the cache holds of it, so leave its results out by status."""
    slots: object
    positions: object
    q_start: object
    kv_end: object
    head: object
    next_head: object
    status: object


def fkv_pages(n_pages: int, page: int, heads: int, d: int, dtype=None, device="cuda") -> Pages:
    """An empty pool of n_pages pages of `page` tokens; dtype torch.int8 (default) or torch.float8_e4m3fn."""
    torch = _torch()
    dtype = dtype or torch.int8
    pages = Pages(torch.zeros((n_pages, heads, page, d), dtype=torch.uint8, device=device).view(dtype),
                  torch.zeros((n_pages, heads, page // 16, d, 16), dtype=torch.uint8, device=device).view(dtype),
                  torch.zeros((n_pages, heads, 2), dtype=torch.float32, device=device))
    _page_desc(pages)
    return pages


def _page_desc(pages) -> fkv_page_desc:
    torch = _TORCH or _torch()
    k, v, scales = pages
    code = k.dtype
    if code is torch.int8:
        kind = FKV_PAGE_INT8
    elif code is torch.float8_e4m3fn:
        kind = FKV_PAGE_E4M3
    else:
        raise TypeError("pages hold int8 or float8_e4m3fn codes")
    if not (k.is_cuda and k.is_contiguous() and v.is_cuda and v.dtype is code and v.is_contiguous() and scales.is_cuda
            and scales.dtype is torch.float32 and scales.is_contiguous()):
        _need(k, code, "pages.k")
        _need(v, code, "pages.v")
        _need(scales, torch.float32, "pages.scales")
    if k.dim() != 4:
        raise ValueError("pages.k must be [n_pages][heads][page][d]")
    n, heads, page, d = k.shape
    if v.shape != (n, heads, page // 16, d, 16) or scales.shape != (n, heads, 2):
        raise ValueError("shape mismatch between pages.k, pages.v and pages.scales")
    return fkv_page_desc(n, page, heads, d, kind)


def _row_type(dtype, name) -> int:
    torch = _TORCH or _torch()
    if dtype is torch.float16:
        return FKV_ROW_F16
    if dtype is torch.bfloat16:
        return FKV_ROW_BF16
    raise TypeError("%s must be float16 or bfloat16" % name)


def _rows(t, slots, heads: int, d: int, name) -> fkv_row_desc:
    """Rows [n][heads][d] of slots [n], or [b][heads][t][d] of slots [b][t]; strided, contiguous in d."""
    shape, stride = t.shape, t.stride()
    if not t.is_cuda or stride[-1] != 1:
        raise TypeError("%s must be CUDA rows of %d contiguous elements" % (name, d))
    kind, at = _row_type(t.dtype, name), slots.shape
    if len(at) == 1 and shape == (at[0], heads, d):
        return fkv_row_desc(shape[0] or 1, 0, stride[0], stride[1], kind)
    if len(at) == 2 and shape == (at[0], heads, at[1], d):
        return fkv_row_desc(shape[2] or 1, stride[0], stride[2], stride[1], kind)
    raise ValueError("%s must be [n][heads][d] for slots [n] or [b][heads][t][d] for slots [b][t]" % name)


def fkv_page_plan(page: int, kv_len, new_len, free_pages, head, tables, n_tokens: int, n_bad=None,
                  stream=None) -> PagePlan:
    """Block tables and slot map of a step: kv_len, new_len i32 [n_req], free_pages i32 [n_free], head i32 [1] or
    None, tables i32 [n_req][max_pages] (new entries written in place), n_tokens rows of the step."""
    torch = _TORCH or _torch()
    i32 = torch.int32
    _need(kv_len, i32, "kv_len")
    _need(new_len, i32, "new_len")
    _need(free_pages, i32, "free_pages")
    _need(tables, i32, "tables")
    if head is not None:
        _need(head, i32, "head")
    if n_bad is not None:
        _need(n_bad, i32, "n_bad")
    n_req, width = kv_len.numel(), tables.shape
    if new_len.numel() != n_req or len(width) != 2 or width[0] != n_req:
        raise ValueError("shape mismatch between kv_len, new_len and tables")
    # one allocation for the outputs: int64 slots first, then the int32 arrays, then the bytes; the addresses go to
    # the call as offsets, and the tensors are made while the kernel runs
    r4 = (n_req + 3) // 4
    sizes = (2 * n_tokens, n_tokens, n_req + 1, n_req, 1, 1, r4)
    size = 3 * n_tokens + 2 * n_req + 3 + r4
    buf = torch.empty(size, dtype=i32, device=kv_len.device) if stream is None else _new(size, i32, kv_len.device, stream)
    at = buf.data_ptr()
    rows = at + 12 * n_tokens          # q_start
    ends = rows + 4 * n_req + 4        # kv_end
    marks = ends + 4 * n_req           # head, next_head, status
    _check(lib.fkv_page_plan(page, n_req, kv_len.data_ptr(), new_len.data_ptr(), free_pages.data_ptr(),
                             free_pages.numel(), _ptr(head), tables.data_ptr(), width[1], n_tokens, at,
                             at + 8 * n_tokens, rows, ends, marks, marks + 4, marks + 8, _ptr(n_bad),
                             _stream(stream)), "fkv_page_plan")
    slots, positions, q_start, kv_end, head_out, next_head, status = buf.split_with_sizes(sizes)
    status = status.view(torch.uint8)
    return PagePlan(slots.view(torch.int64), positions, q_start, kv_end, head_out, next_head,
                    status if n_req == 4 * r4 else status[:n_req])


def fkv_page_store(pages, k, v, slots, n_bad=None, stream=None):
    """Writes rows into the pages' slots: k, v f16 or bf16 [n][heads][d] for slots i64 [n], or [b][heads][t][d] for
    slots [b][t]; any strides, contiguous in d."""
    torch = _TORCH or _torch()
    desc = _page_desc(pages)
    _need(slots, torch.int64, "slots")
    if n_bad is not None:
        _need(n_bad, torch.int32, "n_bad")
    heads, d = desc.heads, desc.d
    rk, rv = _rows(k, slots, heads, d, "k"), _rows(v, slots, heads, d, "v")
    ref = ctypes.byref
    _check(lib.fkv_page_store(ref(desc), ref(rk), ref(rv), k.data_ptr(), v.data_ptr(), slots.numel(),
                              slots.data_ptr(), pages[0].data_ptr(), pages[1].data_ptr(), pages[2].data_ptr(),
                              _ptr(n_bad), _stream(stream)), "fkv_page_store")


def fkv_boxes(pages):
    """Boxes of a pool's pages, for fkv_page_append and fkv_page_select: codes of the pages' type
    [n_pages][heads][2][d], the smallest and largest of each key channel."""
    torch = _TORCH or _torch()
    n, heads, _, d = pages[0].shape
    return torch.zeros((n, heads, 2, d), dtype=torch.uint8, device=pages[0].device).view(pages[0].dtype)


def fkv_rotation_table(n_pos: int, rot: int, base: float = 10000.0, device="cuda"):
    """A table for fkv_page_append, f32 [n_pos][rot // 2][2]: cosines and sines of the angles p * base ** (-2 i / rot),
    formed in 64 bits.  Tables of other frequencies, or with a factor, are made the same way."""
    torch = _TORCH or _torch()
    freq = base ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=device) / rot)
    angle = torch.arange(n_pos, dtype=torch.float64, device=device)[:, None] * freq
    return torch.stack((angle.cos(), angle.sin()), -1).float()


def _need_boxes(boxes, pages) -> None:
    k = pages[0]
    _need(boxes, k.dtype, "boxes")
    n, heads, _, d = k.shape
    if boxes.shape != (n, heads, 2, d):
        raise ValueError("boxes must be [n_pages][heads][2][d]")


def fkv_page_append(pages, k, v, slots, positions=None, table=None, q=None, q_out=None, pairs: bool = False,
                    boxes=None, n_bad=None, stream=None):
    """Writes rows into the pages' slots as fkv_page_store does, the key rows turned by their positions on the way, and
    turns the query rows: k, v, q f16 or bf16 [n][heads][d] for slots i64 [n] and positions i32 [n], or [b][heads][t][d]
    for [b][t]; table f32 [n_pos][rot // 2][2] (fkv_rotation_table), None for no rotation; channels (i, i + rot // 2) are
    turned together, or (2i, 2i + 1) with pairs.  boxes (fkv_boxes) of the pages written are formed of the codes that they then
    hold.  Returns the query rows (q_out, which may be q; by default new ones), or None without q."""
    torch = _TORCH or _torch()
    desc = _page_desc(pages)
    _need(slots, torch.int64, "slots")
    if n_bad is not None:
        _need(n_bad, torch.int32, "n_bad")
    heads, d = desc.heads, desc.d
    rk, rv = _rows(k, slots, heads, d, "k"), _rows(v, slots, heads, d, "v")
    rotate = rq = ro = None
    n_pos = rot = q_heads = 0
    if table is not None:
        _need(table, torch.float32, "table")
        if table.dim() != 3 or table.shape[2] != 2:
            raise ValueError("table must be [n_pos][rot // 2][2]")
        n_pos, rot = table.shape[0], 2 * table.shape[1]
        if positions is None:
            raise TypeError("a rotation needs positions")
        _need(positions, torch.int32, "positions")
        if positions.shape != slots.shape:
            raise ValueError("positions and slots differ in shape")
    if q is not None:
        if q.dim() != len(slots.shape) + 2:
            raise ValueError("q must be [n][q_heads][d] for slots [n] or [b][q_heads][t][d] for slots [b][t]")
        q_heads = q.shape[1]
        rq = _rows(q, slots, q_heads, d, "q")
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if stream is None else _new(q.shape, q.dtype, q.device, stream)
        ro = _rows(q_out, slots, q_heads, d, "q_out")
    elif q_out is not None:
        raise TypeError("q_out without q")
    if boxes is not None:
        _need_boxes(boxes, pages)
    _here(*pages, k, v, slots, positions, table, q, q_out, boxes, n_bad)
    ref = ctypes.byref
    if rot or rq is not None:
        rotate = ref(fkv_rotate_desc(n_pos, rot, FKV_ROTATE_PAIRS if pairs else FKV_ROTATE_HALVES, q_heads))
    _check(lib.fkv_page_append(ref(desc), rotate, None if rq is None else ref(rq), None if ro is None else ref(ro),
                               ref(rk), ref(rv), _ptr(q), _ptr(q_out), k.data_ptr(), v.data_ptr(), slots.numel(),
                               slots.data_ptr(), _ptr(positions) if rot else None, _ptr(table) if rot else None,
                               pages[0].data_ptr(), pages[1].data_ptr(), pages[2].data_ptr(), _ptr(boxes), _ptr(n_bad),
                               _stream(stream)), "fkv_page_append")
    return q_out


def fkv_page_load(pages, slots, dtype=None, k=None, v=None, stream=None):
    """Reads the slots' rows back: returns (k, v) in f16 or bf16, [n][heads][d] for slots [n] and
    [b][heads][t][d] for slots [b][t].  With k or v given, those are written (and no other)."""
    torch = _TORCH or _torch()
    desc = _page_desc(pages)
    _need(slots, torch.int64, "slots")
    heads, d = desc.heads, desc.d
    if k is None and v is None:
        at = slots.shape
        shape = (at[0], heads, d) if len(at) == 1 else (at[0], heads, at[1], d)
        dtype = dtype or torch.float16
        if stream is None:
            k = torch.empty(shape, dtype=dtype, device=slots.device)
            v = torch.empty(shape, dtype=dtype, device=slots.device)
        else:
            k, v = (_new(shape, dtype, slots.device, stream) for _ in "kv")
        rk = rv = _rows(k, slots, heads, d, "k")
    else:
        rk = _rows(k, slots, heads, d, "k") if k is not None else None
        rv = _rows(v, slots, heads, d, "v") if v is not None else None
    ref = ctypes.byref
    _check(lib.fkv_page_load(ref(desc), pages[0].data_ptr(), pages[1].data_ptr(), pages[2].data_ptr(), slots.numel(),
                             slots.data_ptr(), None if rk is None else ref(rk), None if rv is None else ref(rv),
                             _ptr(k), _ptr(v), _stream(stream)), "fkv_page_load")
    return k, v


def _q_rows(pages, q, tables, kv_len, q_start):
    """The checks that the calls for long contexts share over requests' query rows (fkv_page_attend makes them in place: a
    small call's time is these lines, and helpers cost it 0.6 of 11.5 us): (page desc, row type, requests, columns of a table,
    q's shape and strides)."""
    torch = _TORCH or _torch()
    desc = _page_desc(pages)
    if not isinstance(q, torch.Tensor) or not q.is_cuda or q.dim() != 3:
        raise TypeError("q must be a CUDA tensor [n_tokens][q_heads][d]")
    shape, stride = q.shape, q.stride()
    if shape[2] != desc.d or stride[2] != 1:
        raise TypeError("q must have rows of %d contiguous elements" % desc.d)
    i32, kind = torch.int32, _row_type(q.dtype, "q")
    _need(tables, i32, "tables")
    _need(kv_len, i32, "kv_len")
    _need(q_start, i32, "q_start")
    n_req, width = kv_len.numel(), tables.shape
    if len(width) != 2 or width[0] != n_req or q_start.numel() != n_req + 1:
        raise ValueError("shape mismatch between tables, kv_len and q_start")
    return desc, kind, n_req, width[1], shape, stride


def _masks(n: int, q_heads: int, n_req: int, slopes, prefix, first) -> None:
    """Checks of the attention calls' optional tensors."""
    torch = _TORCH or _torch()
    if prefix is not None:
        _need(prefix, torch.int32, "prefix")
        if prefix.numel() != n_req:
            raise ValueError("prefix must have one entry per request")
    if first is not None:
        _need(first, torch.int32, "first")
        if first.numel() != n:
            raise ValueError("first must have one entry per row of q")
    if slopes is not None:
        _need(slopes, torch.float32, "slopes")
        if slopes.numel() != q_heads:
            raise ValueError("slopes must have one entry per query head")


def fkv_page_select(pages, boxes, q, tables, kv_len, q_start, max_new: int, max_kv: int, n_select: int, keep_first: int = 1,
                    keep_last: int = 1, causal: bool = True, selected=None, workspace=None, stream=None):
    """The pages that each query token is to attend to: of those that it sees, the first keep_first, the last keep_last
    and the n_select - keep_first - keep_last others with the largest bounds on their keys' scores (all, where there are
    no more).  boxes (fkv_boxes, kept by fkv_page_append); q, tables, kv_len, q_start, max_new, max_kv as for
    fkv_page_attend.  Returns i32 [n_tokens][heads][n_select]: columns of the token's row of tables, ascending, -1 after
    the last; rows of no request are left as they were.  workspace: uint8 scratch of fkv_page_select_workspace bytes, for
    callers that keep one."""
    torch = _TORCH or _torch()
    desc, kind, n_req, width, shape, q_stride = _q_rows(pages, q, tables, kv_len, q_start)
    _need_boxes(boxes, pages)
    n, q_heads, _ = shape
    sel = fkv_select_desc(n_req, n, max_new, max_kv, width, q_stride[0], q_stride[1], q_heads, kind, 1 if causal else 0,
                          n_select, keep_first, keep_last)
    if selected is None:
        selected = _new((n, desc.heads, max(n_select, 1)), torch.int32, q.device, stream)
    else:
        _need(selected, torch.int32, "selected")
        if selected.shape != (n, desc.heads, n_select):
            raise ValueError("selected must be [n_tokens][heads][n_select]")
    _here(*pages, boxes, q, tables, kv_len, q_start, selected, workspace)
    ref = ctypes.byref
    if workspace is not None:
        _need(workspace, torch.uint8, "workspace")
    else:
        need = lib.fkv_page_select_workspace(ref(desc), ref(sel))
        if need:
            workspace = _new(need, torch.uint8, q.device, stream)
    _check(lib.fkv_page_select(ref(desc), ref(sel), boxes.data_ptr(), pages[2].data_ptr(), q.data_ptr(), tables.data_ptr(),
                               kv_len.data_ptr(), q_start.data_ptr(), selected.data_ptr(), _ptr(workspace),
                               0 if workspace is None else workspace.numel(), _stream(stream)), "fkv_page_select")
    return selected


def fkv_page_select_workspace(pages, q, n_req: int, max_pages: int, max_new: int, max_kv: int, n_select: int) -> int:
    """Bytes of scratch that fkv_page_select of these shapes takes (0: none)."""
    desc = _page_desc(pages)
    sel = fkv_select_desc(n_req, q.shape[0], max_new, max_kv, max_pages, 0, 0, q.shape[1], _row_type(q.dtype, "q"), 1, n_select,
                          0, 0)
    return int(lib.fkv_page_select_workspace(ctypes.byref(desc), ctypes.byref(sel)))


def fkv_page_attend_selected(pages, q, tables, kv_len, q_start, selected, max_new: int, max_kv: int, scale=None,
                             softcap: float = 0.0, causal: bool = True, window: int = 0, sinks: int = 0, slopes=None,
                             prefix=None, first=None, out=None, lse=None, want_lse: bool = False, workspace=None,
                             stream=None):
    """fkv_page_attend over the pages that selected i32 [n_tokens][heads][n] lists for each query token and KV head
    (fkv_page_select's result; columns of the token's row of tables in any order, an entry that is none lists nothing).
    Returns (out, lse or None).  workspace: uint8 scratch of fkv_page_attend_selected_workspace bytes."""
    torch = _TORCH or _torch()
    desc, kind, n_req, width, shape, q_stride = _q_rows(pages, q, tables, kv_len, q_start)
    _need(selected, torch.int32, "selected")
    at = selected.shape
    if len(at) != 3 or at[0] != shape[0] or at[1] != desc.heads:
        raise ValueError("selected must be [n_tokens][heads][n]")
    n, q_heads, d = shape
    if slopes is not None or prefix is not None or first is not None:
        _masks(n, q_heads, n_req, slopes, prefix, first)
    if out is None:
        out = torch.empty(shape, dtype=q.dtype, device=q.device) if stream is None else _new(shape, q.dtype, q.device, stream)
        o_stride = (q_heads * d, d)
    else:
        if not out.is_cuda or out.shape != shape or out.dtype is not q.dtype or out.stride(2) != 1:
            raise TypeError("out must be a CUDA tensor of q's shape and type, contiguous in d")
        o_stride = out.stride()
    if lse is not None:
        _need(lse, torch.float32, "lse")
        if lse.numel() != n * q_heads:
            raise ValueError("lse has the wrong size")
    elif want_lse:
        size = (n, q_heads)   # (a slice of q's shape takes torch half a microsecond)
        lse = torch.empty(size, dtype=torch.float32, device=q.device) if stream is None else _new(size, torch.float32, q.device, stream)
    _here(*pages, q, tables, kv_len, q_start, selected, slopes, prefix, first, out, lse, workspace)
    att = fkv_attend_desc(n_req, n, max_new, max_kv, width, q_stride[0], q_stride[1], o_stride[0], o_stride[1], q_heads, kind,
                          d ** -0.5 if scale is None else scale, softcap, 1 if causal else 0, window, sinks)
    ref = ctypes.byref
    if workspace is not None:
        _need(workspace, torch.uint8, "workspace")
    else:
        need = lib.fkv_page_attend_selected_workspace(ref(desc), ref(att), at[2])
        if need:
            workspace = _new(need, torch.uint8, q.device, stream)
    _check(lib.fkv_page_attend_selected(ref(desc), ref(att), at[2], selected.data_ptr(), pages[0].data_ptr(),
                                        pages[1].data_ptr(), pages[2].data_ptr(), q.data_ptr(), tables.data_ptr(),
                                        kv_len.data_ptr(), q_start.data_ptr(), _ptr(slopes), _ptr(prefix), _ptr(first),
                                        out.data_ptr(), _ptr(lse), _ptr(workspace),
                                        0 if workspace is None else workspace.numel(), _stream(stream)),
           "fkv_page_attend_selected")
    return out, lse


def fkv_page_attend_selected_workspace(pages, q, n_req: int, max_pages: int, max_new: int, max_kv: int, n_selected: int) -> int:
    """Bytes of scratch that fkv_page_attend_selected of these shapes takes (0: none)."""
    desc = _page_desc(pages)
    n, q_heads, d = q.shape
    att = fkv_attend_desc(n_req, n, max_new, max_kv, max_pages, 0, 0, 0, 0, q_heads, _row_type(q.dtype, "q"), 1.0, 0.0, 1, 0, 0)
    return int(lib.fkv_page_attend_selected_workspace(ctypes.byref(desc), ctypes.byref(att), n_selected))


def fkv_page_attend(pages, q, tables, kv_len, q_start, max_new: int, max_kv: int, scale=None, softcap: float = 0.0,
                    causal: bool = True, window: int = 0, sinks: int = 0, slopes=None, prefix=None, first=None,
                    out=None, lse=None, want_lse: bool = False, workspace=None, stream=None):
    """Attention of q f16 or bf16 [n_tokens][q_heads][d] (any strides, contiguous in d) over the pages that tables
    i32 [n_req][max_pages] lists: request r holds kv_len[r] tokens, the last q_start[r+1] - q_start[r] of which are
    its rows of q.  max_new and max_kv bound the rows and tokens of a request (host values: they set the launch).
    scale defaults to d ** -0.5; slopes f32 [q_heads], prefix i32 [n_req], first i32 [n_tokens].  Returns
    (out, lse or None).  workspace: uint8 scratch of fkv_page_attend_workspace bytes, for callers that keep one;
    without it the call takes its scratch from torch's allocator, on the stream it runs on."""
    torch = _TORCH or _torch()
    desc = _page_desc(pages)
    if not isinstance(q, torch.Tensor) or not q.is_cuda or q.dim() != 3:
        raise TypeError("q must be a CUDA tensor [n_tokens][q_heads][d]")
    (n, q_heads, d), q_stride = q.shape, q.stride()
    if d != desc.d or q_stride[2] != 1:
        raise TypeError("q must have rows of %d contiguous elements" % desc.d)
    i32, kind = torch.int32, _row_type(q.dtype, "q")
    _need(tables, i32, "tables")
    _need(kv_len, i32, "kv_len")
    _need(q_start, i32, "q_start")
    n_req, width = kv_len.numel(), tables.shape
    if len(width) != 2 or width[0] != n_req or q_start.numel() != n_req + 1:
        raise ValueError("shape mismatch between tables, kv_len and q_start")
    if slopes is not None or prefix is not None or first is not None:
        _masks(n, q_heads, n_req, slopes, prefix, first)
    if out is None:
        out = torch.empty((n, q_heads, d), dtype=q.dtype, device=q.device) if stream is None else _new(q.shape, q.dtype, q.device, stream)
        o_stride = (q_heads * d, d)
    else:
        if not out.is_cuda or out.shape != q.shape or out.dtype is not q.dtype or out.stride(2) != 1:
            raise TypeError("out must be a CUDA tensor of q's shape and type, contiguous in d")
        o_stride = out.stride()
    if lse is not None:
        _need(lse, torch.float32, "lse")
        if lse.numel() != n * q_heads:
            raise ValueError("lse has the wrong size")
    elif want_lse:
        size = (n, q_heads)   # (a slice of q's shape takes torch half a microsecond)
        lse = torch.empty(size, dtype=torch.float32, device=q.device) if stream is None else _new(size, torch.float32, q.device, stream)
    att = fkv_attend_desc(n_req, n, max_new, max_kv, width[1], q_stride[0], q_stride[1], o_stride[0], o_stride[1], q_heads, kind,
                          d ** -0.5 if scale is None else scale, softcap, 1 if causal else 0, window, sinks)
    ref = ctypes.byref
    if workspace is not None:
        _need(workspace, torch.uint8, "workspace")
    else:
        need = lib.fkv_page_attend_workspace(ref(desc), ref(att))
        if need:
            workspace = _new(need, torch.uint8, q.device, stream)
    _check(lib.fkv_page_attend(ref(desc), ref(att), pages[0].data_ptr(), pages[1].data_ptr(), pages[2].data_ptr(),
                               q.data_ptr(), tables.data_ptr(), kv_len.data_ptr(), q_start.data_ptr(), _ptr(slopes),
                               _ptr(prefix), _ptr(first), out.data_ptr(), _ptr(lse), _ptr(workspace),
                               0 if workspace is None else workspace.numel(), _stream(stream)), "fkv_page_attend")
    return out, lse


def fkv_page_attend_workspace(pages, q, n_req: int, max_pages: int, max_new: int, max_kv: int, window: int = 0,
                              sinks: int = 0) -> int:
    """Bytes of scratch that fkv_page_attend of these shapes takes (0: none)."""
    desc = _page_desc(pages)
    n, q_heads, d = q.shape
    att = fkv_attend_desc(n_req, n, max_new, max_kv, max_pages, 0, 0, 0, 0, q_heads, _row_type(q.dtype, "q"), 1.0, 0.0,
                          1, window, sinks)
    return int(lib.fkv_page_attend_workspace(ctypes.byref(desc), ctypes.byref(att)))


def fkv_diag_mfma_loop(n_blocks: int, iters: int, out=None, random_operands: bool = False, a: float = 1.0,
                       b: float = 1.0, stream=None):
    """Measurement aid: n_blocks blocks of back-to-back v_mfma_f32_32x32x16_f16 from registers (no memory
    traffic).  Returns (out, flops): out float32 [1] holds block 0's accumulator sum (4 * 16 * iters * a * b
    for constant operands when exact), flops the launch's FLOP count.  random_operands alternates two
    pseudo-random operand sets per lane, as real data would."""
    torch = _torch()
    if out is None:
        out = _new(1, torch.float32, "cuda", stream)
    _need(out, torch.float32, "out")
    _check(lib.fkv_diag_mfma_loop(n_blocks, iters, 1 if random_operands else 0, a, b, _ptr(out), _stream(stream)),
           "fkv_diag_mfma_loop")
    return out, lib.fkv_diag_mfma_loop_flops(n_blocks, iters)


def fkv_version() -> str:
    return lib.fkv_version().decode()

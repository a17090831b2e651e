"""Thin ctypes binding of the serving side of liboccam (include/occam_cache.h): rotary
positions, the paged 8-bit key/value cache, attention over it, and its page operations.

The functions mirror the C entry points and, like those of :mod:`.occam`, take torch
tensors, write into tensors that the caller passes, and enqueue on
``torch.cuda.current_stream()`` of the tensors' device unless a stream is given.
:class:`Pages`, :class:`Layer`, :func:`plan` and :func:`workspace` only allocate device
memory; nothing here synchronises with the device.

A serving step::

    pages = cache.Pages(num_pages, 64, num_seqs, max_pages)
    layers = [cache.Layer(pages, num_kv_heads, head_dim) for _ in range(L)]
    cache.reserve(pages, batch, plan)                 # once, for all layers
    for layer in layers:
        cache.rotate(rotary, positions, [q, k])       # in place
        cache.append(pages, layer, batch, plan, k, v)
        cache.attend(pages, layer, batch, q, out, ws, lse=row_lse, max_tokens=longest)

and after ``occam.prune`` has chosen a sequence's survivors::

    cache.keep(pages, seq, span_start, span_len, kept_idx, kept_offsets, plan)
    for layer in layers:
        cache.move(pages, layer, plan, kept_idx, kept_offsets)
"""
from __future__ import annotations

import ctypes
import struct

import torch

from . import occam

HALVES, ADJACENT = 0, 1
FULL, BAD_SEQ, TOO_LONG, BAD_SPAN, BAD_ROWS = 1, 2, 4, 8, 16     # bits of Pages.status

EXPORTS = ("occam_rotary_init", "occam_rotate", "occam_pages_plan_size",
           "occam_cache_storage_size", "occam_pages_reset", "occam_pages_reserve",
           "occam_pages_fork", "occam_pages_free", "occam_pages_keep", "occam_cache_append",
           "occam_cache_read", "occam_cache_move", "occam_cache_workspace_size",
           "occam_cache_attend")

_i32, _i64, _sz, _vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_void_p


class _Pages(ctypes.Structure):
    _fields_ = [("num_pages", _i32), ("page_tokens", _i32), ("num_seqs", _i32),
                ("max_pages", _i32), ("table", _vp), ("length", _vp), ("refs", _vp),
                ("taken", _vp), ("status", _vp)]


class _Cache(ctypes.Structure):
    _fields_ = [("num_kv_heads", _i32), ("head_dim", _i32), ("k", _vp), ("v", _vp),
                ("k_scale", _vp), ("v_scale", _vp)]


class _Batch(ctypes.Structure):
    _fields_ = [("n", _i32), ("seq", _vp), ("rows", _i32), ("row_offsets", _vp),
                ("max_rows", _i32)]


class _Rotary(ctypes.Structure):
    _fields_ = [("head_dim", _i32), ("pairs", _i32), ("axes", _i32), ("layout", _i32),
                ("turn", ctypes.c_uint64 * 128), ("axis", ctypes.c_uint8 * 128)]


class _Heads(ctypes.Structure):
    _fields_ = [("src", _vp), ("dst", _vp), ("heads", _i32), ("src_row_stride", _i64),
                ("dst_row_stride", _i64)]


class _Attention(ctypes.Structure):
    _fields_ = [("num_heads", _i32), ("causal", _i32), ("softmax_scale", ctypes.c_float),
                ("max_tokens", _i32)]


_lib = None


def lib():
    """liboccam.so with the argument types of these entry points."""
    global _lib
    if _lib is None:
        L = occam.lib()
        P, C, B = (ctypes.POINTER(t) for t in (_Pages, _Cache, _Batch))
        A, R = ctypes.POINTER(_Attention), ctypes.POINTER(_Rotary)
        for name, args in dict(
                occam_rotary_init=[R, _i32, _i32, _i32, _i32, ctypes.POINTER(ctypes.c_double),
                                   ctypes.POINTER(ctypes.c_uint8)],
                occam_rotate=[R, _i32, _vp, _i32, _i32, _i32, _vp, _vp],
                occam_pages_reset=[P, _vp],
                occam_pages_reserve=[P, B, _vp, _sz, _vp],
                occam_pages_fork=[P, _i32, _vp, _vp, _vp, _sz, _vp],
                occam_pages_free=[P, _i32, _vp, _vp],
                occam_pages_keep=[P, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp],
                occam_cache_append=[P, C, B, _vp, _sz, _i32, _vp, _i64, _vp, _i64, _vp],
                occam_cache_read=[P, C, B, _vp, _i32, _vp, _i64, _vp, _i64, _vp],
                occam_cache_move=[P, C, _i32, _vp, _sz, _vp, _vp, _vp],
                occam_cache_attend=[P, C, B, A, _vp, _i64, _vp, _i64, _vp, _vp, _sz, _vp]).items():
            getattr(L, name).argtypes = args
            getattr(L, name).restype = _i32
        for name, args in dict(occam_pages_plan_size=[P, _i32],
                               occam_cache_storage_size=[P, _i32, _i32],
                               occam_cache_workspace_size=[P, C, B, A]).items():
            getattr(L, name).argtypes = args
            getattr(L, name).restype = _sz
        _lib = L
    return _lib


_raw_stream = torch._C._cuda_getCurrentRawStream
_current = torch._C._cuda_getDevice
_heads = struct.Struct("PPi4xqq").pack          # an occam_heads


# Devices are compared by index (a tensor elsewhere than on a GPU has -1): what a call costs
# on the host is much of what a small one costs at all.
def _enqueue(fn, index, stream, *args):
    """Call ``fn(*args, stream)`` with device ``index`` current and raise on an error status."""
    if stream is None:
        stream = _raw_stream(index)
    elif isinstance(stream, torch.cuda.Stream):
        stream = stream.cuda_stream
    if index == _current():
        st = fn(*args, stream)
    else:
        with torch.cuda.device(index):
            st = fn(*args, stream)
    if st:
        raise occam.OccamError(st, occam.status_string(st))


def _bad(msg):
    raise occam.OccamError(occam.ERR_INVALID_ARG, msg)


_I32, _F32 = torch.int32, torch.float32


def _ints(t, index, name, at_least=0):
    """Pointer of an int32 device vector (None stays None)."""
    if t is None:
        return None
    if t.dtype is not _I32 or t.get_device() != index or not t.is_contiguous() or (
            at_least and t.numel() < at_least):
        _bad("%s must be a contiguous int32 tensor on GPU %s with at least %d elements" % (name, index, at_least))
    return t.data_ptr()


def _rows(t, index, name, heads, dim, dtype):
    """(pointer, row stride, rows) of a tensor [rows, heads, dim] whose heads are packed."""
    shape = t.shape
    if len(shape) == 3 and t.dtype is dtype and t.get_device() == index:
        n, h, w = shape
        if h == heads and w == dim:
            s0, s1, s2 = t.stride()
            if not n or ((s2 == 1 or dim == 1) and (s1 == dim or heads == 1)):
                return t.data_ptr(), (s0 if n > 1 else heads * dim), n
    _bad("%s must be a [rows, %d, %d] tensor of %s on GPU %s with packed heads" % (name, heads, dim, dtype, index))


_DTYPES = {torch.float32: occam.F32, torch.bfloat16: occam.BF16}


# ------------------------------------------------------------------------------ rotary
def sections(sizes):
    """The axis of every pair where the axes' pairs lie one after the other."""
    return [a for a, n in enumerate(sizes) for _ in range(n)]


def interleaved(sizes):
    """The axis of every pair where the axes take turns, one pair each, until an axis has
    its share; what is left goes to axis 0."""
    total, axes = sum(sizes), len(sizes)
    return [p % axes if p // axes < sizes[p % axes] else 0 for p in range(total)]


class Rotary:
    """occam_rotary: ``inv_freq`` radians per position of every pair, ``axis`` its axis
    (default: axis 0)."""

    def __init__(self, head_dim, inv_freq, axis=None, axes=1, adjacent=False):
        self.c, self.head_dim, self.axes = _Rotary(), int(head_dim), int(axes)
        freq = [float(f) for f in inv_freq]
        if axis is not None and (len(axis) != len(freq) or any(not 0 <= int(a) < 256 for a in axis)):
            _bad("axis must name one axis for every pair")
        st = lib().occam_rotary_init(
            ctypes.byref(self.c), int(head_dim), len(freq), int(axes), ADJACENT if adjacent else HALVES,
            (ctypes.c_double * max(len(freq), 1))(*freq),
            None if axis is None else (ctypes.c_uint8 * max(len(freq), 1))(*[int(a) for a in axis]))
        if st != occam.OK:
            raise occam.OccamError(st, occam.status_string(st))
        self.ref = ctypes.byref(self.c)


def rotate(rotary, positions, src, dst=None, inverse=False, stream=None):
    """occam_rotate of the tensors ``src`` ([rows, heads, head_dim] each, one dtype) into
    ``dst`` (None: in place).  ``positions``: int32 [rows, axes] (or [rows] for one axis)."""
    dst = src if dst is None else dst
    if not src or len(src) != len(dst) or len(src) > occam.MAX_ROW_TENSORS:
        _bad("src and dst must be lists of 1 to %d tensors" % occam.MAX_ROW_TENSORS)
    x, d = src[0], rotary.head_dim
    index, dt, rows = x.get_device(), x.dtype, x.shape[0] if x.dim() else 0
    if dt not in _DTYPES or index < 0 or positions.numel() != rows * rotary.axes:
        _bad("positions must have %d axes for every row, tensors float32 or bfloat16 on a GPU" % rotary.axes)
    heads = b""
    for t, o in zip(src, dst):
        n = t.shape[1] if t.dim() == 3 else 0
        ps, ss, r = _rows(t, index, "src", n, d, dt)
        pd, sd, q = (ps, ss, r) if o is t else _rows(o, index, "dst", n, d, dt)
        if r != rows or q != rows:
            _bad("every tensor must have the same rows")
        heads += _heads(ps, pd, n, ss, sd)
    if rows == 0:
        return
    _enqueue(lib().occam_rotate, index, stream, rotary.ref, rows, _ints(positions, index, "positions"),
             1 if inverse else 0, _DTYPES[dt], len(src), heads)


# ------------------------------------------------------------------------------- pages
class Pages:
    """occam_pages with its device arrays, reset on the current stream.  ``length`` and
    ``table`` may be read between calls; ``status`` holds the sticky failure bits."""

    def __init__(self, num_pages, page_tokens, num_seqs, max_pages, device="cuda"):
        device = torch.device(device)
        if device.type != "cuda":
            _bad("the pages must be on a GPU")
        if device.index is None:
            device = torch.device("cuda", torch.cuda.current_device())
        self.device, self.index = device, device.index
        self.num_pages, self.page_tokens = int(num_pages), int(page_tokens)
        self.num_seqs, self.max_pages = int(num_seqs), int(max_pages)
        self.c = _Pages(self.num_pages, self.page_tokens, self.num_seqs, self.max_pages)
        self.ref = ctypes.byref(self.c)
        if lib().occam_pages_plan_size(self.ref, 1) == 0:
            _bad("invalid pages")
        i32 = dict(dtype=torch.int32, device=device)
        self.table = torch.zeros(self.num_seqs, self.max_pages, **i32)
        self.length = torch.zeros(self.num_seqs, **i32)
        self.refs = torch.zeros(self.num_pages, **i32)
        self.taken = torch.zeros((self.num_pages + 31) // 32, **i32)
        self.status = torch.zeros(1, **i32)
        for name in ("table", "length", "refs", "taken", "status"):
            setattr(self.c, name, getattr(self, name).data_ptr())
        reset(self)


class Layer:
    """occam_cache: one layer's storage for the pages."""

    def __init__(self, pages, num_kv_heads, head_dim):
        self.num_kv_heads, self.head_dim = int(num_kv_heads), int(head_dim)
        self.num_pages, self.page_tokens, self.index = pages.num_pages, pages.page_tokens, pages.index
        size = lib().occam_cache_storage_size(pages.ref, self.num_kv_heads, self.head_dim)
        if size == 0:
            _bad("invalid layer")
        dev = pages.device
        self.k = torch.empty(size, dtype=torch.uint8, device=dev)
        self.v = torch.empty(size, dtype=torch.uint8, device=dev)
        self.k_scale = torch.empty(pages.num_pages, self.num_kv_heads, dtype=torch.float32, device=dev)
        self.v_scale = torch.empty_like(self.k_scale)
        self.c = _Cache(self.num_kv_heads, self.head_dim, self.k.data_ptr(), self.v.data_ptr(),
                        self.k_scale.data_ptr(), self.v_scale.data_ptr())
        self.ref = ctypes.byref(self.c)


class Batch:
    """occam_batch: ``n`` sequences (slots ``seq``, or 0 .. n-1) with ``rows`` rows each, or
    with the packed rows that the int32 device prefix ``row_offsets`` ([n+1]) gives them, at
    most ``max_rows`` each (a bound of at least 1; :data:`BAD_ROWS` where they pass it)."""

    def __init__(self, n, rows=1, seq=None, row_offsets=None, max_rows=0):
        self.n, self.seq, self.row_offsets = int(n), seq, row_offsets     # kept alive
        self.rows = int(rows)
        self.index = None
        for t, least, name in ((seq, self.n, "seq"), (row_offsets, self.n + 1, "row_offsets")):
            if t is not None:
                self.index = t.get_device() if self.index is None else self.index
                _ints(t, self.index, name, least)
        self.c = _Batch(self.n, None if seq is None else seq.data_ptr(), self.rows,
                        None if row_offsets is None else row_offsets.data_ptr(), int(max_rows))
        self.ref = ctypes.byref(self.c)

    def check(self, index, rows=None):
        """The batch's tensors are on GPU ``index``, and tensors of ``rows`` rows hold its rows."""
        if self.index is not None and self.index != index:
            _bad("the batch's tensors must be on GPU %s" % index)
        if rows is not None and self.row_offsets is None and rows < self.n * self.rows:
            _bad("the batch has %d rows, a tensor %d" % (self.n * self.rows, rows))


def plan(pages, n):
    """Memory for the plan of :func:`reserve`, :func:`fork` and :func:`keep` of up to ``n``
    sequences."""
    size = lib().occam_pages_plan_size(pages.ref, int(n))
    if size == 0:
        _bad("invalid plan")
    return torch.zeros(size // 4, dtype=torch.int32, device=pages.device)


def _plan(pages, p):
    return _ints(p, pages.index, "plan"), p.numel() * 4


def reset(pages, stream=None):
    _enqueue(lib().occam_pages_reset, pages.index, stream, pages.ref)


def reserve(pages, batch, plan, stream=None):
    batch.check(pages.index)
    _enqueue(lib().occam_pages_reserve, pages.index, stream, pages.ref, batch.ref, *_plan(pages, plan))


def fork(pages, src, dst, plan, stream=None):
    n, dev = src.numel(), pages.index
    _enqueue(lib().occam_pages_fork, dev, stream, pages.ref, n, _ints(src, dev, "src"),
             _ints(dst, dev, "dst", n), *_plan(pages, plan))


def free(pages, seq, stream=None):
    dev = pages.index
    _enqueue(lib().occam_pages_free, dev, stream, pages.ref, seq.numel(), _ints(seq, dev, "seq"))


def _lists(kept_idx, kept_offsets, dev):
    """Pointers of the survivors' lists.  A list of no survivors may have no address: the
    offsets' stands for it (nothing reads it)."""
    idx, offsets = _ints(kept_idx, dev, "kept_idx"), _ints(kept_offsets, dev, "kept_offsets")
    return offsets if idx == 0 else idx, offsets


def keep(pages, seq, span_start, span_len, kept_idx, kept_offsets, plan, stream=None):
    n = seq.numel()
    if kept_offsets.numel() != n + 1:             # move() takes n from it
        _bad("kept_offsets must have %d elements" % (n + 1))
    dev = pages.index
    _enqueue(lib().occam_pages_keep, dev, stream, pages.ref, n, _ints(seq, dev, "seq"),
             _ints(span_start, dev, "span_start", n), _ints(span_len, dev, "span_len", n),
             *_lists(kept_idx, kept_offsets, dev), *_plan(pages, plan))


# ------------------------------------------------------------------------------- rows
def _layer(pages, layer):
    """The device of the pages, whose numbers the layer has storage for."""
    if layer.num_pages < pages.num_pages or layer.page_tokens != pages.page_tokens or layer.index != pages.index:
        _bad("the layer must have been made for these pages")
    return pages.index


def append(pages, layer, batch, plan, k, v, stream=None):
    """occam_cache_append: ``k`` and ``v`` [rows, num_kv_heads, head_dim], float32 or bfloat16."""
    dev, dt = _layer(pages, layer), k.dtype
    if dt not in _DTYPES:
        _bad("k and v must be float32 or bfloat16 tensors")
    kp, ks, n = _rows(k, dev, "k", layer.num_kv_heads, layer.head_dim, dt)
    vp, vs, m = _rows(v, dev, "v", layer.num_kv_heads, layer.head_dim, dt)
    if n != m:
        _bad("k and v must have the same rows")
    batch.check(dev, n)
    if n == 0:
        return
    _enqueue(lib().occam_cache_append, dev, stream, pages.ref, layer.ref, batch.ref, *_plan(pages, plan),
             _DTYPES[dt], kp, ks, vp, vs)


def read(pages, layer, batch, k, v=None, start=None, stream=None):
    """occam_cache_read into ``k`` and ``v`` (either may be None), float32 or bfloat16."""
    dev = _layer(pages, layer)
    x = k if k is not None else v
    if x is None or x.dtype not in _DTYPES:
        _bad("k or v must be a float32 or bfloat16 tensor")
    dt, kp, ks, vp, vs = x.dtype, None, 0, None, 0
    if k is not None:
        kp, ks, n = _rows(k, dev, "k", layer.num_kv_heads, layer.head_dim, dt)
        batch.check(dev, n)
    if v is not None:
        vp, vs, n = _rows(v, dev, "v", layer.num_kv_heads, layer.head_dim, dt)
        batch.check(dev, n)
        if n != x.shape[0]:
            _bad("k and v must have the same rows")
    if x.shape[0] == 0:
        return
    _enqueue(lib().occam_cache_read, dev, stream, pages.ref, layer.ref, batch.ref,
             _ints(start, dev, "start", batch.n), _DTYPES[dt], kp, ks, vp, vs)


def move(pages, layer, plan, kept_idx, kept_offsets, stream=None):
    """occam_cache_move with the plan and the lists of :func:`keep`."""
    dev = _layer(pages, layer)
    _enqueue(lib().occam_cache_move, dev, stream, pages.ref, layer.ref, kept_offsets.numel() - 1,
             *_plan(pages, plan), *_lists(kept_idx, kept_offsets, dev))


# --------------------------------------------------------------------------- attention
def workspace_size(pages, layer, batch, num_heads, max_tokens=0) -> int:
    at = _Attention(int(num_heads), 1, 0.0, int(max_tokens))
    return int(lib().occam_cache_workspace_size(pages.ref, layer.ref, batch.ref, ctypes.byref(at)))


def workspace(pages, layer, batch, num_heads, max_tokens=0):
    """Memory for :func:`attend` of this batch; calls that may overlap need one each."""
    n = workspace_size(pages, layer, batch, num_heads, max_tokens)
    if n == 0:
        _bad("invalid attention (workspace size 0)")
    return torch.empty(n, dtype=torch.uint8, device=pages.device)


def attend(pages, layer, batch, q, out, ws, lse=None, causal=True, softmax_scale=0.0, max_tokens=0,
           stream=None):
    """occam_cache_attend: ``q`` and ``out`` bfloat16 [rows, num_heads, head_dim], ``lse``
    float32 [rows, num_heads] or None.  ``q`` and ``out`` must not overlap.  ``max_tokens``: a
    bound of the lengths (0: what the tables hold), as for :func:`workspace`; a near one lets
    the call choose the faster form."""
    dev, H = _layer(pages, layer), q.shape[1] if q.dim() == 3 else 0
    qp, qs, n = _rows(q, dev, "q", H, layer.head_dim, torch.bfloat16)
    op, os, m = _rows(out, dev, "out", H, layer.head_dim, torch.bfloat16)
    batch.check(dev, n)
    if n != m or ws.get_device() != dev or not ws.is_contiguous():
        _bad("q and out must have the same rows, and the workspace be contiguous on the pages' device")
    if lse is not None and (lse.dtype is not _F32 or lse.get_device() != dev or not lse.is_contiguous() or
                            lse.numel() < n * H):
        _bad("lse must be a contiguous float32 tensor [rows, %d] on GPU %s" % (H, dev))
    if n == 0:
        return
    at = _Attention(H, 1 if causal else 0, float(softmax_scale), int(max_tokens))
    _enqueue(lib().occam_cache_attend, dev, stream, pages.ref, layer.ref, batch.ref, ctypes.byref(at), qp, qs,
             op, os, None if lse is None else lse.data_ptr(), ws.data_ptr(), ws.nbytes)

"""The paged 4-bit cache: thin ctypes binding of include/kve_pages.h.

``Pages`` bundles the buffers of a cache; the functions have the names and the
meaning of the C calls without their ``kve_`` prefix.  As in ``binding``, they
check shapes, types and devices, allocate outputs and workspaces that the caller
does not pass, and forward raw device pointers and the current HIP stream (or
``stream``; what is allocated here then belongs to that stream).
"""

from __future__ import annotations

import ctypes
import functools
from dataclasses import dataclass, field

from . import binding as kb
from .binding import LIB


class _CPages(ctypes.Structure):
    """kve_pages_t"""
    _fields_ = [(n, ctypes.c_void_p) for n in ("pool", "refs", "table", "held", "length")] + [
        (n, ctypes.c_int) for n in ("L", "n_pages", "Hkv", "d", "page", "S", "M")]


@functools.lru_cache(maxsize=None)
def page_bytes(page: int, d: int) -> int:
    """Bytes of a page of one layer and KV head (0 if page or d is invalid)."""
    return int(LIB.kve_page_bytes(page, d))


@dataclass(frozen=True)
class Pages:
    """A paged cache (kve_pages_t): device tensors

      pool    uint8 [L, n_pages, Hkv, page_bytes(page, d)]
      refs    int32 [n_pages]   sequences that hold a page
      table   int32 [S, M]      page numbers of each slot's sequence
      held    int32 [S]         pages that it holds
      length  int32 [S]         its tokens

    An empty cache has refs, held and length all zero (pipeline.alloc_pages makes
    one).  part: the pool holds some of the layers that share the bookkeeping
    (``layers``), and pages_fork does not take it."""
    pool: object
    refs: object
    table: object
    held: object
    length: object
    page: int
    d: int
    part: bool = False
    c: object = field(init=False, repr=False, compare=False)      # kve_pages_t
    index: int = field(init=False, repr=False, compare=False)     # the device's

    def __post_init__(self):
        torch = kb._torch()
        pool = self.pool
        if pool.dim() != 4 or pool.dtype != torch.uint8:
            raise ValueError("pool must be uint8 [L, n_pages, Hkv, page_bytes]")
        L, n_pages, Hkv, have = pool.shape
        nb = page_bytes(self.page, self.d)
        if nb == 0:
            raise ValueError(f"page={self.page} must be a power of two in [32, 1024] and d={self.d} 64 or 128")
        if have != nb:
            raise ValueError(f"pool has pages of {have} bytes, page={self.page} and d={self.d} make {nb}")
        if self.table.dim() != 2:
            raise ValueError("table must be int32 [S, M]")
        S, M = self.table.shape
        object.__setattr__(self, "index", pool.get_device())
        if self.index < 0 or not pool.is_contiguous():
            raise ValueError("pool must be a contiguous device tensor")
        object.__setattr__(self, "c", _CPages(
            pool.data_ptr(), _ints(self.refs, (n_pages,), "refs", self), _ints(self.table, (S, M), "table", self),
            _ints(self.held, (S,), "held", self), _ints(self.length, (S,), "length", self), L, n_pages, Hkv, self.d,
            self.page, S, M))

    @property
    def L(self) -> int:
        return self.c.L

    @property
    def Hkv(self) -> int:
        return self.c.Hkv

    def layers(self, l0: int, l1: int) -> "Pages":
        """The rows of layers [l0, l1), with the same bookkeeping: a decode step takes
        layer after layer.  What changes the bookkeeping is called once for all of
        them; pages_fork, which copies rows too, takes all layers only."""
        pool = self.pool[l0:l1]
        return Pages(pool, self.refs, self.table, self.held, self.length, self.page, self.d,
                     self.part or pool.shape[0] != self.L)


def _four_bit(pages):
    """Refuses a cache of another format for a call on four-bit rows."""
    if not isinstance(pages, Pages):
        raise ValueError("the cache must be a Pages")


def _on(pages: Pages, stream):
    """The stream to launch on; the cache's device must be the current one."""
    torch = kb._torch()
    if pages.index != torch._C._cuda_getDevice():
        raise ValueError(f"the cache is on {pages.pool.device}, the current device is {torch.cuda.current_device()}")
    return torch._C._cuda_getCurrentRawStream(pages.index) if stream is None else stream.cuda_stream


def _new(make, stream):
    """make(), an allocation that belongs to ``stream`` (None: the current one)."""
    if stream is None:
        return make()
    with kb._torch().cuda.stream(stream):
        return make()


def _workspace(pages, size, workspace, stream):
    """(tensor, its pointer and bytes): the caller's workspace, or one made here of
    size() bytes.  The tensor has to live until the call is enqueued."""
    torch = kb._torch()
    if workspace is None:
        nbytes = size()
        workspace = _new(lambda: torch.empty(nbytes, dtype=torch.uint8, device=pages.pool.device), stream)
    elif workspace.get_device() != pages.index or not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous on the cache's device")
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _ints(t, shape, name, pages, optional=False):
    """Pointer of a contiguous int32 device tensor of the given shape, or None."""
    if t is None and optional:
        return None
    if t.dtype is not kb._torch().int32 or t.shape != shape:
        raise ValueError(f"{name} must be int32 {list(shape)}")
    if t.get_device() != pages.index or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous on the cache's device")
    return t.data_ptr()


def _rows(k, v, pages):
    """(B, T, then pointer and strides of both, dtype code) of row tensors [L, B, Hkv, T, d]."""
    shape = k.shape
    if v.shape != shape or v.dtype is not k.dtype:
        raise ValueError("v must match k")
    if len(shape) != 5 or shape[0] != pages.c.L or shape[2] != pages.c.Hkv or shape[4] != pages.d:
        raise ValueError(f"k and v must be [L={pages.L}, B, Hkv={pages.Hkv}, T, d={pages.d}]")
    if k.get_device() != pages.index or v.get_device() != pages.index:
        raise ValueError("k or v is not on the cache's device")
    at = []
    for t, name in ((k, "k"), (v, "v")):
        if t.is_contiguous():
            at += [t.data_ptr(), None]
        else:
            p, st = kb._view(t, name)
            at += [p, ctypes.byref(st)]
    return (shape[1], shape[3], *at, kb._dtype_code(k))


def pages_workspace_size(n_pages: int, S: int, n: int) -> int:
    return int(LIB.kve_pages_workspace_size(n_pages, S, n))


def _book(pages, n, out, missing, name, workspace, stream):
    """Outputs and workspace of a bookkeeping call on n entries: (out, missing, workspace, their
    pointers and the workspace's bytes)."""
    torch = kb._torch()
    if out is None:
        out = _new(lambda: torch.empty(n, dtype=torch.int32, device=pages.pool.device), stream)
    if missing is None:
        missing = _new(lambda: torch.empty(1, dtype=torch.int32, device=pages.pool.device), stream)
    ws, wp, wsb = _workspace(pages, lambda: pages_workspace_size(pages.c.n_pages, pages.c.S, n), workspace, stream)
    return out, missing, ws, (_ints(out, (n,), name, pages), _ints(missing, (1,), "missing", pages), wp, wsb)


def pages_extend(pages: Pages, add, seq=None, start=None, missing=None, workspace=None, stream=None):
    """Room for add[i] more tokens in the sequence of slot seq[i] (slot i without
    seq): pages reserved, lengths advanced.  Returns (start, missing): the lengths
    before, -1 where an entry was refused, and the pages that were lacking."""
    n = add.numel()
    st = _on(pages, stream)
    start, missing, _ws, at = _book(pages, n, start, missing, "start", workspace, stream)
    kb._check(LIB.kve_pages_extend(ctypes.byref(pages.c), _ints(seq, (n,), "seq", pages, True),
                                   _ints(add, (n,), "add", pages), n, *at, st))
    return start, missing


def pages_fork(pages: Pages, src, dst, done=None, missing=None, workspace=None, stream=None):
    """Slot dst[i] becomes a continuation of the sequence in slot src[i].  Returns
    (done, missing): 1 per entry, 0 where it was refused, and the pages lacking.
    Takes all layers of the cache: the others would lack the rows that are copied."""
    _four_bit(pages)
    if pages.part:
        raise ValueError("a fork takes all layers of the cache")
    n = src.numel()
    st = _on(pages, stream)
    done, missing, _ws, at = _book(pages, n, done, missing, "done", workspace, stream)
    kb._check(LIB.kve_pages_fork(ctypes.byref(pages.c), _ints(src, (n,), "src", pages),
                                 _ints(dst, (n,), "dst", pages), n, *at, st))
    return done, missing


def pages_free(pages: Pages, seq=None, stream=None):
    """Empties the slots seq (all slots without it) and returns their pages."""
    n = pages.c.S if seq is None else seq.numel()
    kb._check(LIB.kve_pages_free(ctypes.byref(pages.c), _ints(seq, (n,), "seq", pages, True), n, _on(pages, stream)))


def pages_append(k, v, pages: Pages, start, n_new=None, seq=None, stream=None):
    """Packs the first n_new[b] (all without it) of the rows k, v [L, B, Hkv, T, d]
    into positions start[b] on of the sequence in slot seq[b]; views as for
    kv_compact_strided."""
    _four_bit(pages)
    B, T, kp, ks, vp, vs, dt = _rows(k, v, pages)
    kb._check(LIB.kve_pages_append(kp, ks, vp, vs, dt, B, T, _ints(n_new, (B,), "n_new", pages, True),
                                   _ints(start, (B,), "start", pages), _ints(seq, (B,), "seq", pages, True),
                                   ctypes.byref(pages.c), _on(pages, stream)))


def _compact_args(k, v, idx, count, pages, start, seq):
    _four_bit(pages)
    B, N, kp, ks, vp, vs, dt = _rows(k, v, pages)
    shape = (pages.c.L, B, pages.c.Hkv)
    k_cap = idx.shape[-1]
    return (kp, ks, vp, vs, dt, B, N, _ints(idx, shape + (k_cap,), "idx", pages), _ints(count, shape, "count", pages),
            k_cap, _ints(start, (B,), "start", pages), _ints(seq, (B,), "seq", pages, True), ctypes.byref(pages.c))


def pages_compact(k, v, idx, count, pages: Pages, start, seq=None, stream=None):
    """kv_compact into pages: rows idx[l, b, j, :count[l, b, j]] of k, v
    [L, B, Hkv, N, d] packed into positions start[b] on of the sequence in slot
    seq[b]."""
    kb._check(LIB.kve_pages_compact(*_compact_args(k, v, idx, count, pages, start, seq), _on(pages, stream)))


def check_compact(k, v, idx, count, pages: Pages, start, seq=None):
    """Raises what pages_compact would raise, launching nothing; returns the call's
    arguments for run_compact (the tensors have to live until then)."""
    args = _compact_args(k, v, idx, count, pages, start, seq)
    st = _on(pages, None)
    B, k_cap = args[5], args[9]
    kb._check(LIB.kve_pages_compact(*args[:7], None, args[8], 0, *args[10:], st))    # of no rows: checks alone
    if pages.c.L * B * pages.c.Hkv * (k_cap // 64 + 1) >= 1 << 24:    # workgroups of 64 rows in one launch
        raise ValueError("too many rows for one call")
    return args


def run_compact(args, pages: Pages, stream=None):
    """pages_compact with the arguments that check_compact returned."""
    kb._check(LIB.kve_pages_compact(*args, _on(pages, stream)))


def pages_select(pages: Pages, src, idx, count, dst, start, stream=None):
    """A second eviction: rows idx[l, b, j, :count[l, b, j]] of the sequence in
    slot src[b] moved, unchanged, to positions start[b] on of slot dst[b]."""
    _four_bit(pages)
    B, k_cap = src.numel(), idx.shape[-1]
    shape = (pages.L, B, pages.Hkv)
    kb._check(LIB.kve_pages_select(ctypes.byref(pages.c), B, _ints(src, (B,), "src", pages),
                                   _ints(idx, shape + (k_cap,), "idx", pages), _ints(count, shape, "count", pages),
                                   k_cap, _ints(dst, (B,), "dst", pages), _ints(start, (B,), "start", pages),
                                   _on(pages, stream)))


def pages_read(pages: Pages, T: int, seq=None, start=None, count=None, dtype=None, k_out=None, v_out=None,
               stream=None):
    """Key and value rows [L, B, Hkv, T, d] of the sequences in slots seq (all
    slots without it): T rows from start[b] (0), count[b] (T) of them.  Outputs
    are of ``dtype`` (bfloat16) unless given; rows that the sequence does not
    have stay as they were, zero in outputs made here."""
    _four_bit(pages)
    torch = kb._torch()
    B = pages.c.S if seq is None else seq.numel()
    shape = (pages.c.L, B, pages.c.Hkv, T, pages.d)
    st = _on(pages, stream)
    for name, t in (("k_out", k_out), ("v_out", v_out)):
        if t is not None:
            dtype = t.dtype if dtype is None else dtype
            if t.shape != shape or t.dtype is not dtype or t.get_device() != pages.index or not t.is_contiguous():
                raise ValueError(f"{name} must be {dtype} {list(shape)}, contiguous on the cache's device")
    dtype = torch.bfloat16 if dtype is None else dtype
    if k_out is None:
        k_out = _new(lambda: torch.zeros(shape, dtype=dtype, device=pages.pool.device), stream)
    if v_out is None:
        v_out = _new(lambda: torch.zeros(shape, dtype=dtype, device=pages.pool.device), stream)
    kb._check(LIB.kve_pages_read(ctypes.byref(pages.c), kb._dtype_code(k_out), B, T,
                                 _ints(seq, (B,), "seq", pages, True), _ints(start, (B,), "start", pages, True),
                                 _ints(count, (B,), "count", pages, True), k_out.data_ptr(), v_out.data_ptr(), st))
    return k_out, v_out


def decode_pages_workspace_size(L, B, Hq, Hkv, max_tokens, d) -> int:
    return int(LIB.kve_decode_pages_workspace_size(L, B, Hq, Hkv, max_tokens, d))


def decode_pages(q, pages: Pages, max_tokens: int | None = None, seq=None, scale: float = 0.0, out=None,
                 workspace=None, stream=None):
    """decode_attention over paged sequences: q [L, B, Hq, d] attends to the rows
    of the sequences in slots seq (slot b without it) -> float32 [L, B, Hq, d].
    max_tokens bounds the lengths (default: what the table can hold); the work is
    split by it.  A workspace made for the largest call serves smaller ones."""
    _four_bit(pages)
    torch = kb._torch()
    shape = q.shape
    if len(shape) != 4 or shape[0] != pages.c.L or shape[3] != pages.d or q.get_device() != pages.index or \
            not q.is_contiguous():
        raise ValueError(f"q must be [L={pages.L}, B, Hq, d={pages.d}], contiguous on the cache's device")
    L, B, Hq, d = shape
    if max_tokens is None:
        max_tokens = pages.c.M * pages.page
    st = _on(pages, stream)
    if out is None:
        out = _new(lambda: torch.empty(shape, dtype=torch.float32, device=q.device), stream)
    elif out.shape != shape or out.dtype is not torch.float32 or out.get_device() != pages.index or \
            not out.is_contiguous():
        raise ValueError("out must be float32 [L, B, Hq, d], contiguous on the cache's device")
    _ws, wp, wsb = _workspace(pages, lambda: decode_pages_workspace_size(L, B, Hq, pages.Hkv, max_tokens, d),
                              workspace, stream)
    kb._check(LIB.kve_decode_pages(q.data_ptr(), kb._dtype_code(q), ctypes.byref(pages.c), B, Hq, int(max_tokens),
                                   _ints(seq, (B,), "seq", pages, True), float(scale), out.data_ptr(), wp, wsb, st))
    return out

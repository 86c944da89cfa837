"""The paged 8-bit cache: thin ctypes binding of include/kve_blocks.h.

``Blocks`` bundles the buffers of a cache, ``Rotation`` the angles that new keys
and queries are turned by; the functions have the names and the meaning of the C
calls without their ``kve_`` prefix.  pages_extend and pages_free take a Blocks
as they take a Pages: the bookkeeping is the same.  Shapes, types and devices are
checked, outputs and workspaces that the caller does not pass are allocated, and
raw device pointers and the current HIP stream (or ``stream``; what is allocated
here then belongs to that stream) are forwarded.
"""

from __future__ import annotations

import ctypes
import functools
from dataclasses import dataclass, field

from . import binding as kb
from .binding import LIB
from .pages import _CPages, _ints, _new, _on, _rows, _workspace


class _CRotation(ctypes.Structure):
    """kve_rotation_t"""
    _fields_ = [(n, ctypes.c_void_p) for n in ("cos", "sin", "position")] + \
        [(n, ctypes.c_int) for n in ("P", "r", "pairs")]


@functools.lru_cache(maxsize=None)
def block_bytes(page: int, d: int) -> int:
    """Bytes of a block, a page of one layer and KV head (0 if page or d is invalid)."""
    return int(LIB.kve_block_bytes(page, d))


@dataclass(frozen=True)
class Blocks:
    """A paged 8-bit cache (a kve_pages_t with blocks in its pool): device tensors

      pool    uint8 [L, n_pages, Hkv, block_bytes(page, d)]
      refs, table, held, length   as of a Pages

    An empty cache has refs, held and length all zero (pipeline.alloc_blocks makes
    one)."""
    pool: object
    refs: object
    table: object
    held: object
    length: object
    page: int
    d: int
    c: object = field(init=False, repr=False, compare=False)      # kve_pages_t
    index: int = field(init=False, repr=False, compare=False)     # the device's

    def __post_init__(self):
        torch = kb._torch()
        pool = self.pool
        if pool.dim() != 4 or pool.dtype != torch.uint8:
            raise ValueError("pool must be uint8 [L, n_pages, Hkv, block_bytes]")
        L, n_pages, Hkv, have = pool.shape
        nb = block_bytes(self.page, self.d)
        if nb == 0:
            raise ValueError(f"page={self.page} must be 32, 64 or 128 and d={self.d} 64 or 128")
        if have != nb:
            raise ValueError(f"pool has blocks of {have} bytes, page={self.page} and d={self.d} make {nb}")
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

    def layers(self, l0: int, l1: int) -> "Blocks":
        """The blocks of layers [l0, l1), with the same bookkeeping: a decode step takes
        layer after layer.  What changes the bookkeeping is called once for all."""
        return Blocks(self.pool[l0:l1], self.refs, self.table, self.held, self.length, self.page, self.d)


@dataclass(frozen=True)
class Rotation:
    """The angles of positions: cos and sin float32 [P, r / 2] (device) turn the first
    r channels of a row at position p, channels i and i + r / 2 as a pair, or with
    ``pairs`` channels 2 i and 2 i + 1."""
    cos: object
    sin: object
    pairs: bool = False

    def __post_init__(self):
        torch = kb._torch()
        if self.cos.dim() != 2 or self.cos.shape != self.sin.shape:
            raise ValueError("cos and sin must be float32 [P, r / 2]")
        for t in (self.cos, self.sin):
            if t.dtype is not torch.float32 or not t.is_cuda or not t.is_contiguous():
                raise ValueError("cos and sin must be contiguous float32 device tensors")


def _blocks(x):
    if not isinstance(x, Blocks):
        raise ValueError("the cache must be a Blocks")
    return x


def blocks_append(k, v, blocks: Blocks, start, n_new=None, seq=None, rotation: Rotation | None = None, position=None,
                  q=None, q_out=None, stream=None):
    """Writes the first n_new[b] (all without it) of the rows k, v [L, B, Hkv, T, d]
    into positions start[b] on of the sequence in slot seq[b], the keys turned by
    ``rotation`` at position int32 [B, T]; views as for kv_compact_strided.  With q
    [L, B, Hq, T, d], a view, returns the queries turned alike (q_out, dense)."""
    torch = kb._torch()
    _blocks(blocks)
    B, T, kp, ks, vp, vs, dt = _rows(k, v, blocks)
    st = _on(blocks, stream)
    rot = None
    if (rotation is None) != (position is None):
        raise ValueError("a rotation and the tokens' positions go together")
    if rotation is not None:
        if rotation.cos.get_device() != blocks.index or rotation.sin.get_device() != blocks.index:
            raise ValueError("cos or sin is not on the cache's device")
        P, half = rotation.cos.shape
        rot = ctypes.byref(_CRotation(rotation.cos.data_ptr(), rotation.sin.data_ptr(),
                                      _ints(position, (B, T), "position", blocks), P, 2 * half, int(rotation.pairs)))
    qp, qs, Hq, op = None, None, 0, None
    if q is None and q_out is not None:
        raise ValueError("q_out without q")
    if q is not None:
        if rotation is None:
            raise ValueError("queries are turned: they need a rotation")
        if q.dim() != 5 or q.shape[0] != blocks.c.L or q.shape[1] != B or q.shape[3:] != (T, blocks.d) or \
                q.dtype is not k.dtype or q.get_device() != blocks.index:
            raise ValueError(f"q must be [L={blocks.L}, B={B}, Hq, T={T}, d={blocks.d}] of k's type "
                             "on the cache's device")
        Hq = q.shape[2]
        if q.is_contiguous():
            qp = q.data_ptr()
        else:
            qp, qst = kb._view(q, "q")
            qs = ctypes.byref(qst)
        if q_out is None:
            q_out = _new(lambda: torch.empty(q.shape, dtype=q.dtype, device=q.device), stream)
        elif q_out.shape != q.shape or q_out.dtype is not q.dtype or q_out.get_device() != blocks.index or \
                not q_out.is_contiguous():
            raise ValueError("q_out must be as q, contiguous on the cache's device")
        op = q_out.data_ptr()
        if q.numel() == 0:
            qp = op = None
    kb._check(LIB.kve_blocks_append(kp, ks, vp, vs, dt, B, T, _ints(n_new, (B,), "n_new", blocks, True),
                                    _ints(start, (B,), "start", blocks), _ints(seq, (B,), "seq", blocks, True),
                                    ctypes.byref(blocks.c), rot, qp, qs, Hq, op, st))
    return q_out


def _compact_args(k, v, idx, count, blocks, start, seq):
    B, N, kp, ks, vp, vs, dt = _rows(k, v, _blocks(blocks))
    shape = (blocks.c.L, B, blocks.c.Hkv)
    k_cap = idx.shape[-1]
    return (kp, ks, vp, vs, dt, B, N, _ints(idx, shape + (k_cap,), "idx", blocks), _ints(count, shape, "count", blocks),
            k_cap, _ints(start, (B,), "start", blocks), _ints(seq, (B,), "seq", blocks, True), ctypes.byref(blocks.c))


def blocks_compact(k, v, idx, count, blocks: Blocks, start, seq=None, stream=None):
    """kv_compact into blocks: rows idx[l, b, j, :count[l, b, j]] of k, v
    [L, B, Hkv, N, d] written into positions start[b] on of the sequence in slot
    seq[b]."""
    kb._check(LIB.kve_blocks_compact(*_compact_args(k, v, idx, count, blocks, start, seq), _on(blocks, stream)))


def check_compact(k, v, idx, count, blocks: Blocks, start, seq=None):
    """Raises what blocks_compact would raise, launching nothing; returns the call's
    arguments for run_compact (the tensors have to live until then)."""
    args = _compact_args(k, v, idx, count, blocks, start, seq)
    st = _on(blocks, None)
    B, k_cap = args[5], args[9]
    kb._check(LIB.kve_blocks_compact(*args[:7], None, args[8], 0, *args[10:], st))    # of no rows: checks alone
    # workgroups, for the keys and the values of each block that the rows can touch, in one launch
    if 2 * blocks.c.L * B * blocks.c.Hkv * ((k_cap + blocks.page - 2) // blocks.page + 1) >= 1 << 24:
        raise ValueError("too many rows for one call")
    return args


def run_compact(args, blocks: Blocks, stream=None):
    """blocks_compact with the arguments that check_compact returned."""
    kb._check(LIB.kve_blocks_compact(*args, _on(blocks, stream)))


def _outputs(blocks, shape, dtype, names, outs, stream):
    """(dtype, outputs) of a call that reads the cache: the caller's, or zeros."""
    torch = kb._torch()
    for name, t in zip(names, outs):
        if t is not None:
            dtype = t.dtype if dtype is None else dtype
            if t.shape != shape or t.dtype is not dtype or t.get_device() != blocks.index or not t.is_contiguous():
                raise ValueError(f"{name} must be {dtype} {list(shape)}, contiguous on the cache's device")
    dtype = torch.bfloat16 if dtype is None else dtype
    return tuple(_new(lambda: torch.zeros(shape, dtype=dtype, device=blocks.pool.device), stream) if t is None else t
                 for t in outs)


def blocks_read(blocks: Blocks, T: int, seq=None, start=None, count=None, dtype=None, k_out=None, v_out=None,
                stream=None):
    """Key and value rows [L, B, Hkv, T, d] of the sequences in slots seq (all
    slots without it): T rows from start[b] (0), count[b] (T) of them.  Outputs
    are of ``dtype`` (bfloat16) unless given; rows that the sequence does not
    have stay as they were, zero in outputs made here."""
    _blocks(blocks)
    B = blocks.c.S if seq is None else seq.numel()
    st = _on(blocks, stream)
    k_out, v_out = _outputs(blocks, (blocks.c.L, B, blocks.c.Hkv, T, blocks.d), dtype, ("k_out", "v_out"),
                            (k_out, v_out), stream)
    kb._check(LIB.kve_blocks_read(ctypes.byref(blocks.c), kb._dtype_code(k_out), B, T,
                                  _ints(seq, (B,), "seq", blocks, True), _ints(start, (B,), "start", blocks, True),
                                  _ints(count, (B,), "count", blocks, True), k_out.data_ptr(), v_out.data_ptr(), st))
    return k_out, v_out


def blocks_bounds(blocks: Blocks, n: int, seq=None, first=None, dtype=None, lo_out=None, hi_out=None, stream=None):
    """Smallest and largest keys [L, B, Hkv, n, d] of blocks first[b] (0) on of the
    sequences in slots seq (all slots without it); outputs as for blocks_read."""
    _blocks(blocks)
    B = blocks.c.S if seq is None else seq.numel()
    st = _on(blocks, stream)
    lo_out, hi_out = _outputs(blocks, (blocks.c.L, B, blocks.c.Hkv, n, blocks.d), dtype, ("lo_out", "hi_out"),
                              (lo_out, hi_out), stream)
    kb._check(LIB.kve_blocks_bounds(ctypes.byref(blocks.c), kb._dtype_code(lo_out), B, n,
                                    _ints(seq, (B,), "seq", blocks, True), _ints(first, (B,), "first", blocks, True),
                                    lo_out.data_ptr(), hi_out.data_ptr(), st))
    return lo_out, hi_out


def _queries(q, blocks, max_tokens):
    """(L, B, Hq, T, max_tokens) of queries [L, B, Hq, T, d], or [L, B, Hq, d] of one token."""
    _blocks(blocks)
    shape = q.shape
    if len(shape) not in (4, 5) or shape[0] != blocks.c.L or shape[-1] != blocks.d or \
            q.get_device() != blocks.index or not q.is_contiguous():
        raise ValueError(f"q must be [L={blocks.L}, B, Hq, T, d={blocks.d}], contiguous on the cache's device")
    T = shape[3] if len(shape) == 5 else 1
    return shape[0], shape[1], shape[2], T, blocks.c.M * blocks.page if max_tokens is None else int(max_tokens)


@functools.lru_cache(maxsize=1024)
def blocks_top_workspace_size(L, B, Hkv, T, max_tokens, page) -> int:
    return int(LIB.kve_blocks_top_workspace_size(L, B, Hkv, T, max_tokens, page))


def blocks_top(q, blocks: Blocks, k: int, first: int = 1, last: int = 1, max_tokens: int | None = None, seq=None,
               start=None, out=None, workspace=None, stream=None):
    """The k blocks of each query token and KV head whose keys' bounds allow the
    highest product with its queries, the ``first`` and ``last`` ones of the
    sequence among them: q [L, B, Hq, T, d] (or [L, B, Hq, d]) -> int32
    [L, B, Hkv, T, k], ascending, then -1.  What a token sees is as for
    decode_blocks, which takes the result as ``top``.  max_tokens bounds the lengths
    (default: what the table can hold)."""
    torch = kb._torch()
    L, B, Hq, T, max_tokens = _queries(q, blocks, max_tokens)
    st = _on(blocks, stream)
    shape = (L, B, blocks.c.Hkv, T, k)
    if out is None:
        out = _new(lambda: torch.empty(shape, dtype=torch.int32, device=q.device), stream)
    _ws, wp, wsb = _workspace(blocks, lambda: blocks_top_workspace_size(L, B, blocks.c.Hkv, T, max_tokens, blocks.page),
                              workspace, stream)
    kb._check(LIB.kve_blocks_top(q.data_ptr(), kb._dtype_code(q), ctypes.byref(blocks.c), B, Hq, T, max_tokens,
                                 _ints(start, (B,), "start", blocks, True), _ints(seq, (B,), "seq", blocks, True),
                                 k, first, last, _ints(out, shape, "out", blocks), wp, wsb, st))
    return out


@functools.lru_cache(maxsize=1024)
def decode_blocks_workspace_size(L, B, Hq, Hkv, T, d) -> int:
    return int(LIB.kve_decode_blocks_workspace_size(L, B, Hq, Hkv, T, d))


def decode_blocks(q, blocks: Blocks, max_tokens: int | None = None, seq=None, start=None, top=None,
                  scale: float = 0.0, out=None, workspace=None, stream=None):
    """Attention of query tokens q [L, B, Hq, T, d] (or [L, B, Hq, d], one token) to
    the sequences in slots seq (slot b without it) -> float32 of q's shape.  Token t
    sees the rows before position start[b] + t + 1, without ``start`` that of the
    sequence's last T tokens; with ``top`` int32 [L, B, Hkv, T, k] only those of the
    blocks it names (blocks_top).  max_tokens bounds the lengths (default: what the
    table can hold); the work is split by it.  A workspace made for the largest call
    serves smaller ones."""
    torch = kb._torch()
    L, B, Hq, T, max_tokens = _queries(q, blocks, max_tokens)
    st = _on(blocks, stream)
    if out is None:
        out = _new(lambda: torch.empty(q.shape, dtype=torch.float32, device=q.device), stream)
    elif out.shape != q.shape or out.dtype is not torch.float32 or out.get_device() != blocks.index or \
            not out.is_contiguous():
        raise ValueError("out must be float32 of q's shape, contiguous on the cache's device")
    k, tp = 0, None
    if top is not None:
        k = top.shape[-1]
        tp = _ints(top, (L, B, blocks.c.Hkv, T, k), "top", blocks)
    _ws, wp, wsb = _workspace(blocks, lambda: decode_blocks_workspace_size(L, B, Hq, blocks.c.Hkv, T, blocks.d),
                              workspace, stream)
    kb._check(LIB.kve_decode_blocks(q.data_ptr(), kb._dtype_code(q), ctypes.byref(blocks.c), B, Hq, T, max_tokens,
                                    _ints(start, (B,), "start", blocks, True), _ints(seq, (B,), "seq", blocks, True),
                                    tp, k, float(scale), out.data_ptr(), wp, wsb, st))
    return out

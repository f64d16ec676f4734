"""The rollout's key-value cache in pages, attention over it, and drafted tokens: the
binding of that part of include/rr.h.

A rollout's token step, next to the products of ``products.py``: ``rr_cache_extend``
takes pages for the step's tokens, ``rr_cache_append`` writes a layer's keys and values,
``rr_attend`` is the attention over them; ``rr_accept`` holds drafted tokens against the
model's probabilities, and ``rr_cache_truncate`` takes the refused ones back.  Samples of
one prompt share its pages (``rr_cache_fork``), and ``rr_cache_compact`` moves the pages in
use to the front.  As in ``rr.py``, every step runs in the CUDA library; this module checks and
marshals arguments.
"""
from __future__ import annotations

import ctypes

from .products import _stream_of, _torch_type
from .rr import RR_OK, _check, _DST_DTYPES, _lib, _sig, _stream, _vp

_i32, _i64, _f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_float


class _Cache(ctypes.Structure):
    _fields_ = [("layers", _i32), ("n_kv", _i32), ("dim", _i32), ("page_tokens", _i32),
                ("n_pages", _i32), ("max_seqs", _i32), ("max_pages", _i32), ("dtype", _i32)]


_PC, _P64 = ctypes.POINTER(_Cache), ctypes.POINTER(_i64)

_sig("rr_cache_bytes", [_PC, _P64, _P64, _P64])
_sig("rr_cache_clear", [_PC, _vp, _vp])
_sig("rr_cache_fork", [_PC, _vp, _vp, _vp, _i32, _vp])
_sig("rr_cache_extend", [_PC, _vp, _vp, _vp, _vp, _i32, _vp])
_sig("rr_cache_append", [_PC, _vp, _vp, _i32, _vp, _i64, _vp, _i64, _i32, _vp, _vp, _i32, _vp])
_sig("rr_cache_truncate", [_PC, _vp, _vp, _vp, _i32, _vp])
_sig("rr_cache_compact", [_PC, _vp, _vp, _vp])
_sig("rr_cache_check", [_PC, _vp, _vp])
_sig("rr_attend_workspace", [_PC, _i32, _P64])
_sig("rr_attend", [_PC, _vp, _vp, _i32, _vp, _i64, _i32, _i32, _vp, _i64, _vp, _vp, _vp, _i32, _f32,
                   _vp, _i64, _vp])
_sig("rr_accept", [_vp, _i64, _vp, _i64, _vp, _vp, _vp, _vp, _i32, _i32, _i32, _vp, _vp, _vp, _vp])

_types = None


def _torch_types():
    """(int32, float32), without an import in every call."""
    global _types
    if _types is None:
        import torch
        _types = (torch.int32, torch.float32)
    return _types


class Cache:
    """Keys and values of up to max_seqs sequences, in pages of page_tokens tokens.

    ``pages`` [n_pages, layers, 2, n_kv, page_tokens, pitch]: keys, then values; allocated
    on the current device if not given.  ``pitch`` is dim, rounded up to a multiple of 8.
    ``book``: an int32 tensor with all that says which sequence holds which page; a copy
    of it, put back, undoes the calls in between, as long as the pages that they gave
    away have not been written.  Views of it: ``table`` [max_seqs, max_pages] (a sequence's
    pages in order; behind its last one -1), ``lengths`` [max_seqs] (tokens) and ``refs`` [n_pages]
    (how many sequences hold a page; 0: it is free).  A new cache is empty."""

    def __init__(self, layers: int, n_kv: int, dim: int, n_pages: int, max_seqs: int,
                 max_pages: int, page_tokens: int = 16, dtype: str = "bf16", pages=None):
        import torch
        if dtype not in _DST_DTYPES:
            raise ValueError(f"dtype must be one of {sorted(_DST_DTYPES)}, not {dtype!r}")
        self._c = _Cache(layers, n_kv, dim, page_tokens, n_pages, max_seqs, max_pages,
                         _DST_DTYPES[dtype])
        self._ref = ctypes.byref(self._c)
        one, pitch, book = _i64(), _i64(), _i64()
        _check(_lib.rr_cache_bytes(self._ref, ctypes.byref(one), ctypes.byref(pitch),
                                   ctypes.byref(book)), "rr_cache_bytes")
        self.layers, self.n_kv, self.dim, self.page_tokens = layers, n_kv, dim, page_tokens
        self.n_pages, self.max_seqs, self.max_pages = n_pages, max_seqs, max_pages
        self.dtype, self.torch_dtype = dtype, _torch_type(dtype)
        self.pitch, self.page_bytes = pitch.value, one.value
        shape = (n_pages, layers, 2, n_kv, page_tokens, self.pitch)
        if pages is None:
            pages = torch.empty(shape, dtype=self.torch_dtype, device="cuda")
        if pages.dtype != self.torch_dtype or tuple(pages.shape) != shape or \
                not pages.is_contiguous():
            raise ValueError(f"pages: expected a contiguous {self.torch_dtype} tensor of {shape}")
        self.pages = pages
        self.book = torch.zeros(book.value // 4, dtype=torch.int32, device=pages.device)

        def part(at, *shape):
            n = 1
            for d in shape:
                n *= d
            return self.book[at:at + n].view(shape), at + (n + 3) // 4 * 4

        self.table, at = part(64, max_seqs, max_pages)
        self.lengths, at = part(at, max_seqs)
        self.refs, _ = part(at, n_pages)
        self.table.fill_(-1)
        # The first call may come on another stream than these.
        if pages.is_cuda and not torch.cuda.is_current_stream_capturing():
            torch.cuda.current_stream(pages.device).synchronize()
        self._p, self._b = pages.data_ptr(), self.book.data_ptr()


def _ints(x, n, what: str) -> int:
    """The address of a contiguous int32 tensor of n elements."""
    if x.dtype is not _torch_types()[0] or x.numel() != n or not x.is_contiguous():
        raise ValueError(f"{what}: expected a contiguous int32 tensor of {n}")
    return x.data_ptr()


def _list(x, what: str):
    if x.dim() != 1:
        raise ValueError(f"{what}: shape {tuple(x.shape)}, expected [n]")
    n = x.numel()
    return _ints(x, n, what), n


def _vectors(x, heads: int, cache: Cache, what: str):
    """(rows, row stride) of [rows, heads, dim], or [rows, heads * dim]."""
    if x.dtype is not cache.torch_dtype:
        raise ValueError(f"{what}: elements of {x.dtype}, expected {cache.torch_dtype}")
    dim, cols = cache.dim, heads * cache.dim
    shape = x.shape
    if len(shape) == 3 and shape[1] == heads and shape[2] == dim:
        n = shape[0]
        if x.is_contiguous():
            return n, cols
        ld, inner, head = x.stride()
        ok = (head == 1 or dim == 1) and (inner == dim or heads == 1)
    elif len(shape) == 2 and shape[1] == cols:
        n = shape[0]
        if x.is_contiguous():
            return n, cols
        ld, inner = x.stride()
        ok = inner == 1 or cols == 1
    else:
        raise ValueError(f"{what}: shape {tuple(shape)}, expected [n, {heads}, {dim}]")
    if not ok:
        raise ValueError(f"{what}: the elements of a row must be contiguous")
    if n <= 1:
        ld = cols
    if ld < cols:
        raise ValueError(f"{what}: rows overlap")
    return n, ld


def rr_cache_clear(cache: Cache, stream=None) -> None:
    """Makes the cache empty: no sequence holds a token, all pages are free, no mark is left."""
    st = _lib.rr_cache_clear(cache._ref, cache._b, _stream_of(cache.book, stream))
    if st != RR_OK:
        _check(st, "rr_cache_clear")


def rr_cache_fork(cache: Cache, parents, children, stream=None) -> None:
    """children[i], an empty sequence, comes to hold parents[i]'s tokens: its pages, shared.
    A parent may be listed more than once.  Asynchronous on `stream`, as all calls on a
    cache are but ``rr_cache_check``."""
    p, n = _list(parents, "parents")
    c = _ints(children, n, "children")
    st = _lib.rr_cache_fork(cache._ref, cache._b, p, c, n, _stream_of(parents, stream))
    if st != RR_OK:
        _check(st, "rr_cache_fork")


def rr_cache_extend(cache: Cache, seqs, starts=None, stream=None) -> None:
    """Room for new tokens of the listed sequences, starts[i + 1] - starts[i] of sequence
    seqs[i] (one each without starts): their lengths grow, and the pool's lowest free pages are
    taken as needed.  A partly filled page that others hold too is copied first."""
    s, n = _list(seqs, "seqs")
    at = None if starts is None else _ints(starts, n + 1, "starts")
    st = _lib.rr_cache_extend(cache._ref, cache._p, cache._b, s, at, n, _stream_of(seqs, stream))
    if st != RR_OK:
        _check(st, "rr_cache_extend")


def rr_cache_append(cache: Cache, layer: int, k, v, seqs, starts=None, stream=None) -> None:
    """One layer's keys and values [rows, n_kv, dim] of the sequences' newest tokens: rows
    starts[i] .. starts[i + 1] - 1 are the last ones of seqs[i] (without starts, row i is the
    last one of seqs[i]).  A sequence whose rows are not all there is left out and marks the cache."""
    rows, ldk = _vectors(k, cache.n_kv, cache, "k")
    m, ldv = _vectors(v, cache.n_kv, cache, "v")
    if m != rows:
        raise ValueError(f"v: {m} rows, k has {rows}")
    s, n = _list(seqs, "seqs")
    at = None if starts is None else _ints(starts, n + 1, "starts")
    st = _lib.rr_cache_append(cache._ref, cache._p, cache._b, layer, k.data_ptr(), ldk, v.data_ptr(),
                              ldv, rows, s, at, n, _stream_of(k, stream))
    if st != RR_OK:
        _check(st, "rr_cache_append")


def rr_cache_truncate(cache: Cache, seqs, drop=None, stream=None) -> None:
    """Takes the last drop[i] tokens of seqs[i] back (without drop, all of them): pages
    that no token is left in are given up."""
    s, n = _list(seqs, "seqs")
    d = None if drop is None else _ints(drop, n, "drop")
    st = _lib.rr_cache_truncate(cache._ref, cache._b, s, d, n, _stream_of(seqs, stream))
    if st != RR_OK:
        _check(st, "rr_cache_truncate")


def rr_cache_compact(cache: Cache, stream=None) -> None:
    """Moves pages in use to the front of the pool, so that the free ones are its end."""
    st = _lib.rr_cache_compact(cache._ref, cache._p, cache._b, _stream_of(cache.pages, stream))
    if st != RR_OK:
        _check(st, "rr_cache_compact")


def rr_cache_check(cache: Cache, stream=None) -> None:
    """Raise if a call on this cache found its lists or the table out of range, or the pool
    without room (waits for `stream`).  Such a call was not done, nor were those after it, and the
    cache is as it was; ``rr_cache_append`` and ``rr_attend`` left out what did not fit, after which
    only they go on."""
    _check(_lib.rr_cache_check(cache._ref, cache._b, _stream_of(cache.pages, stream)),
           "rr_cache_check")


class AttendWorkspace:
    """Device workspace of ``rr_attend`` with n_q query heads on a cache, or on any of the
    same head size, ready on every stream.  Calls that overlap in time need one each."""

    def __init__(self, cache: Cache, n_q: int):
        import torch
        need = _i64()
        _check(_lib.rr_attend_workspace(cache._ref, n_q, ctypes.byref(need)), "rr_attend_workspace")
        self.nbytes, self.n_q = need.value, n_q
        self.data = torch.zeros(self.nbytes, dtype=torch.uint8, device=cache.pages.device)
        # The first call may come on another stream than the zeros.
        if self.data.is_cuda and not torch.cuda.is_current_stream_capturing():
            torch.cuda.current_stream(self.data.device).synchronize()
        self._p = self.data.data_ptr()


def rr_attend(cache: Cache, layer: int, q, out, seqs, workspace: AttendWorkspace, starts=None,
              lse=None, scale=None, stream=None) -> None:
    """Attention of the sequences' newest tokens, rows of q [rows, n_q, dim] as for
    ``rr_cache_append``, over one layer's keys and values; a token sees the tokens up to itself.
    ``lse`` (float32 [rows, n_q]) receives ln(sum exp(score)).  scale: dim ** -0.5 if not given.
    Rows of q that belong to no listed sequence are left as they are in out and lse."""
    n_q = workspace.n_q
    rows, ldq = _vectors(q, n_q, cache, "q")
    m, ldo = _vectors(out, n_q, cache, "out")
    if m != rows:
        raise ValueError(f"out: {m} rows, q has {rows}")
    s, n = _list(seqs, "seqs")
    at = None if starts is None else _ints(starts, n + 1, "starts")
    e = None
    if lse is not None:
        if lse.dtype is not _torch_types()[1] or tuple(lse.shape) != (rows, n_q) or \
                not lse.is_contiguous():
            raise ValueError(f"lse: expected a contiguous float32 tensor of [{rows}, {n_q}]")
        e = lse.data_ptr()
    st = _lib.rr_attend(cache._ref, cache._p, cache._b, layer, q.data_ptr(), ldq, n_q, rows,
                        out.data_ptr(), ldo, e, s, at, n,
                        cache.dim ** -0.5 if scale is None else scale,
                        workspace._p, workspace.nbytes, _stream_of(q, stream))
    if st != RR_OK:
        _check(st, "rr_attend")


def _probabilities(x, what: str):
    if x.dtype is not _torch_types()[1]:
        raise ValueError(f"{what}: elements of {x.dtype}, expected float32")
    if x.dim() != 2 or (x.stride(1) != 1 and x.shape[1] > 1):
        raise ValueError(f"{what}: expected [rows, vocab] with contiguous rows")
    rows, vocab = x.shape
    ld = x.stride(0) if rows > 1 else vocab
    if ld < vocab:
        raise ValueError(f"{what}: rows overlap")
    return rows, vocab, ld


def _floats(x, n: int, what: str) -> int:
    if x.dtype is not _torch_types()[1] or x.numel() != n or not x.is_contiguous():
        raise ValueError(f"{what}: expected a contiguous float32 tensor of {n}")
    return x.data_ptr()


def rr_accept(p, drafts, u, v, accepted, tokens, q=None, starts=None, rejected=None,
              stream=None) -> None:
    """Drafted tokens held against the model's probabilities p [rows, vocab] (float32).

    Rows starts[i] .. starts[i + 1] - 1 are those of sequence i: one for each draft and one
    more.  Draft drafts[r] is accepted if u[r] q[r, draft] < p[r, draft], as long as all before
    it were; the next token comes from max(p - q, 0) where a draft was refused, else from
    p, by the number v[i] of [0, 1).  Without q, drafts are sure (q is 1 at the draft); without
    starts, every row is a sequence without drafts (drafts and u may be None).
    accepted and rejected (int32 [n]): how many drafts were; tokens (int32 [rows]): the accepted
    ones, the next one, then -1."""
    rows, vocab, ldp = _probabilities(p, "p")
    pq, ldq = None, 0
    if q is not None:
        m, cols, ldq = _probabilities(q, "q")
        if (m, cols) != (rows, vocab):
            raise ValueError(f"q: shape {(m, cols)}, p has {(rows, vocab)}")
        pq = q.data_ptr()
    n = accepted.numel()
    at = pd = pu = None
    if starts is not None:
        at = _ints(starts, n + 1, "starts")
        pd, pu = _ints(drafts, rows, "drafts"), _floats(u, rows, "u")
    st = _lib.rr_accept(p.data_ptr(), ldp, pq, ldq, pd, at, pu, _floats(v, n, "v"), rows, n, vocab,
                        _ints(accepted, n, "accepted"), _ints(tokens, rows, "tokens"),
                        None if rejected is None else _ints(rejected, n, "rejected"),
                        _stream_of(p, stream))
    if st != RR_OK:
        _check(st, "rr_accept")

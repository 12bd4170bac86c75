"""What a decoder that serves drafted tokens runs between their logits and the
next step: probabilities, verification, accepted slots, copied pages and the
table of pages.

Like the rest of the package this only marshals arguments to the C ABI of
include/af1.h, which has the formulas, the layouts and the errors. Tensors are
on the current CUDA device; index tensors are int32. `stream` (default: the
current one) takes the work; a tensor that a call allocates belongs to it. No
call waits for the device, so that a whole step can be captured in a graph.
"""
from __future__ import annotations

import ctypes

import torch

from . import AF1Error, _check, _i64, _ptr, _vp, last_error
from .attention import (KVCache, _declare, _dtype, _empty, _f32, _F32, _i32, _I32, _index, _pages, _steps,
                        _stream_handle)

_DISTINCT = 1


class _ProbsArgs(ctypes.Structure):
    _fields_ = [("logits", _vp), ("rows", _i64), ("vocab", _i64), ("ld", _i64), ("probs", _vp), ("probs_ld", _i64),
                ("temperature", _vp), ("top_k", _vp), ("min_p", _vp), ("all_temperature", _f32), ("all_top_k", _i32),
                ("all_min_p", _f32), ("dtype", _i32)]


class _VerifyArgs(ctypes.Structure):
    _fields_ = [("probs", _vp), ("probs_seq", _i64), ("probs_node", _i64), ("draft", _vp), ("draft_seq", _i64),
                ("draft_node", _i64), ("tokens", _vp), ("parents", _vp), ("counts", _vp), ("uniforms", _vp),
                ("path", _vp), ("lengths", _vp), ("following", _vp), ("sequences", _i64), ("nodes", _i64),
                ("vocab", _i64), ("flags", _i32), ("reserved", _i32)]


class _TableDesc(ctypes.Structure):
    _fields_ = [("table", _vp), ("refs", _vp), ("sequences", _i64), ("columns", _i64), ("ld", _i64), ("pages", _i64),
                ("page_size", _i32), ("reserved", _i32)]


_P = ctypes.POINTER
_token_probs = _declare("af1_token_probs", _P(_ProbsArgs), _vp)
_verify_tree = _declare("af1_verify_tree", _P(_VerifyArgs), _vp)
_kv_compact = _declare("af1_kv_compact", _P(_vp), _i64, _vp, _i64, _i64, _i64, _vp, _vp, _i64, _vp, _vp)
_kv_copy = _declare("af1_kv_copy", _P(_vp), _i64, _vp, _i64, _vp)
_pages_fork = _declare("af1_pages_fork", _P(_TableDesc), _vp, _vp)
_pages_workspace = _declare("af1_pages_workspace_bytes", _P(_TableDesc), restype=_i64)
_pages_reserve = _declare("af1_pages_reserve", _P(_TableDesc), _vp, _vp, _vp, _vp, _vp, _i64, _vp)
_pages_release = _declare("af1_pages_release", _P(_TableDesc), _vp, _vp)


# -- probabilities -------------------------------------------------------------------


def _setting(value, what: str, rows: int, dtype):
    """(pointer, value for all rows) of a number or of a tensor of the rows' own."""
    if not isinstance(value, torch.Tensor):
        return 0, float(value)
    if value.dtype is not dtype or value.shape != (rows,) or not value.is_contiguous():
        raise ValueError(f"{what} must be a number or a contiguous {dtype} tensor of shape {(rows,)}")
    return value.data_ptr(), 0


def token_probs(logits: torch.Tensor, temperature=1.0, top_k=0, min_p=0.0, out: torch.Tensor | None = None,
                stream=None) -> torch.Tensor:
    """Probabilities (rows, vocab), float32, of rows of logits, float16 or
    float32, after the temperature (0: greedy), of the top_k largest (0: all)
    that are at least min_p times as likely as the largest (af1_token_probs).
    Each setting is a number, or a tensor (rows,) of the rows' own: float32,
    top_k int32. out: float32, with rows of its own, or float32 logits themselves."""
    ld = _steps(logits, "logits", 2)[0]
    dt = _dtype(logits, "logits")
    rows, vocab = logits.shape
    settings = [_setting(temperature, "temperature", rows, _F32), _setting(top_k, "top_k", rows, _I32),
                _setting(min_p, "min_p", rows, _F32)]
    k = settings[1][1]
    if k != int(k) or not -(1 << 31) <= k < 1 << 31:
        raise ValueError("top_k must be a whole number of 32 bits")
    if out is None:
        out = _empty((rows, vocab), _F32, logits.device, stream)
    elif out.shape != logits.shape or out.dtype is not _F32:
        raise ValueError("out must be float32 with the shape of logits")
    out_ld = _steps(out, "out", 2)[0]
    if rows == 0:
        return out
    a = _ProbsArgs(logits.data_ptr(), rows, vocab, ld if rows > 1 else vocab, out.data_ptr(),
                   out_ld if rows > 1 else vocab, settings[0][0], settings[1][0], settings[2][0], settings[0][1], int(k),
                   settings[2][1], dt)
    _check(_token_probs(ctypes.byref(a), _stream_handle(stream)))
    return out


# -- verification --------------------------------------------------------------------


def verify_tree(probs: torch.Tensor, tokens: torch.Tensor, parents: torch.Tensor, uniforms: torch.Tensor,
                draft: torch.Tensor | None = None, counts: torch.Tensor | None = None, distinct: bool = False,
                out=None, stream=None):
    """(path, lengths, following) of drafted trees (af1_verify_tree): the
    accepted nodes of every sequence from node 0 on, then -1 (sequences, nodes);
    how many they are; the token that follows.

    probs: the target's probabilities behind every node, float32 (sequences,
    nodes, vocab). tokens, parents: int32 (sequences, nodes); node 0 is the last
    token and the root. uniforms: float32 (sequences, nodes), number 0 for the
    token that follows. draft: the probabilities that every node's children were
    drawn from, like probs; None: the children are guesses. distinct: siblings
    were drawn without repetition. counts: nodes of each sequence's tree. out:
    three contiguous int32 tensors for the results; without them a call takes
    the host 10 us more."""
    ps = _steps(probs, "probs", 3)
    sequences, nodes, vocab = probs.shape
    if probs.dtype is not _F32:
        raise ValueError("probs must be float32")
    qs = (0, 0, 1)
    if draft is not None:
        qs = _steps(draft, "draft", 3)
        if draft.dtype is not _F32 or draft.shape != probs.shape:
            raise ValueError("draft must be float32 with the shape of probs")
    elif distinct:
        raise ValueError("distinct without draft")
    if uniforms.dtype is not _F32 or uniforms.shape != (sequences, nodes) or not uniforms.is_contiguous():
        raise ValueError(f"uniforms must be a contiguous float32 tensor of shape {(sequences, nodes)}")
    tp, pp = _index(tokens, "tokens", (sequences, nodes)), _index(parents, "parents", (sequences, nodes))
    cp = _index(counts, "counts", (sequences,))
    if out is None:
        device = probs.device
        path = _empty((sequences, nodes), _I32, device, stream)
        lengths, following = _empty((sequences,), _I32, device, stream), _empty((sequences,), _I32, device, stream)
    else:
        path, lengths, following = out
        _index(path, "out[0]", (sequences, nodes))
        _index(lengths, "out[1]", (sequences,))
        _index(following, "out[2]", (sequences,))
    if sequences == 0:
        return path, lengths, following
    a = _VerifyArgs(probs.data_ptr(), ps[0], ps[1], _ptr(draft), qs[0], qs[1], tp, pp, cp, uniforms.data_ptr(),
                    path.data_ptr(), lengths.data_ptr(), following.data_ptr(), sequences, nodes, vocab,
                    _DISTINCT if distinct else 0, 0)
    _check(_verify_tree(ctypes.byref(a), _stream_handle(stream)))
    return path, lengths, following


# -- accepted slots and copied pages -------------------------------------------------


def _handles(caches):
    """The handles of one cache or of several (a model's layers)."""
    if isinstance(caches, KVCache):
        caches = (caches,)
    return (_vp * len(caches))(*[c._h for c in caches]), len(caches)


def kv_compact(caches, pages: torch.Tensor, first: torch.Tensor, index: torch.Tensor, counts: torch.Tensor,
               stream=None) -> None:
    """Move slot first + index[j] of every sequence to first + j, j < counts,
    in one KVCache or in a list of them that share the table `pages`
    (af1_kv_compact): with the path and the lengths of verify_tree, the accepted
    tokens come to lie behind the prefix. first, counts: (sequences,); index:
    (sequences, nodes)."""
    handles, n = _handles(caches)
    pp, sequences, columns, ld = _pages(pages)
    if index.dim() != 2:
        raise ValueError("index must be (sequences, nodes)")
    nodes = index.shape[1]
    _check(_kv_compact(handles, n, pp, sequences, columns, ld, _index(first, "first", (sequences,)),
                       _index(index, "index", (sequences, nodes)), nodes, _index(counts, "counts", (sequences,)),
                       _stream_handle(stream)))


def kv_copy(caches, copies: torch.Tensor, stream=None) -> None:
    """Copy the first rows of pages in one KVCache or in a list of them
    (af1_kv_copy). copies: (entries, 3), source page, target page and rows, as
    PageTable.reserve gives them."""
    handles, n = _handles(caches)
    if copies.dim() != 2:
        raise ValueError("copies must be (entries, 3)")
    entries = copies.shape[0]
    _check(_kv_copy(handles, n, _index(copies, "copies", (entries, 3)), entries, _stream_handle(stream)))


# -- the table -----------------------------------------------------------------------


class PageTable:
    """The table of a batch's pages over the caller's tensors, shared by the
    caches of a model's layers: `table`, int32 (sequences, columns), -1 where
    there is no page, and `refs`, int32 (pages,), how many entries hold each page
    (0: free; what the caller adds keeps a page). Both are changed in place, in
    the order of the stream; fork, reserve and release keep refs right."""

    def __init__(self, table: torch.Tensor, refs: torch.Tensor, page_size: int):
        pp, sequences, columns, ld = _pages(table)
        if refs.dim() != 1:
            raise ValueError("refs must be (pages,)")
        rp = _index(refs, "refs", (refs.shape[0],))
        self._d = _TableDesc(pp, rp, sequences, columns, ld, refs.shape[0], page_size, 0)
        size = _pages_workspace(ctypes.byref(self._d))
        if size < 0:
            raise AF1Error(int(size), last_error())
        self.table, self.refs, self.page_size = table, refs, page_size
        self._workspace_bytes = size
        # (workspace, copies, lacking) for each stream that has had a reserve call, which writes them before it reads them:
        # made at the first one, in that stream's order, and filled by nothing else.
        self._buffers = {}

    @classmethod
    def empty(cls, sequences: int, columns: int, pages: int, page_size: int, device=None):
        """A table without pages, over tensors of its own, which are filled in
        the order of the current stream."""
        device = device or torch.device("cuda", torch.cuda.current_device())
        return cls(torch.full((sequences, columns), -1, dtype=_I32, device=device),
                   torch.zeros(pages, dtype=_I32, device=device), page_size)

    def _per_sequence(self, t: torch.Tensor, what: str) -> int:
        return _index(t, what, (self.table.shape[0],))

    def fork(self, parents: torch.Tensor, stream=None) -> None:
        """Row s becomes what row parents[s] was, its pages shared; a row with
        no parent (-1) gives up its pages (af1_pages_fork)."""
        _check(_pages_fork(ctypes.byref(self._d), self._per_sequence(parents, "parents"), _stream_handle(stream)))

    def reserve(self, first: torch.Tensor, counts: torch.Tensor, copies: torch.Tensor | None = None,
                lacking: torch.Tensor | None = None, stream=None):
        """Pages of the sequences' own for counts slots from `first` on
        (af1_pages_reserve). Returns (copies, lacking): what kv_copy has to copy
        before these slots are written, (sequences, 3), and the number of pages
        that were lacking, (1,); if it is not 0, no page has changed hands. Where
        they are not given they are tensors that the table has for this stream,
        and hold until the next call on it."""
        fp, cp = self._per_sequence(first, "first"), self._per_sequence(counts, "counts")
        sequences, device = self.table.shape[0], self.table.device
        op, lp = _index(copies, "copies", (sequences, 3)), _index(lacking, "lacking", (1,))
        handle = _stream_handle(stream)
        own = self._buffers.get(handle)
        if own is None:
            own = self._buffers[handle] = (_empty((self._workspace_bytes,), torch.uint8, device, stream),
                                           _empty((sequences, 3), _I32, device, stream), _empty((1,), _I32, device, stream))
        workspace = own[0]
        if copies is None:
            copies = own[1]
            op = copies.data_ptr()
        if lacking is None:
            lacking = own[2]
            lp = lacking.data_ptr()
        _check(_pages_reserve(ctypes.byref(self._d), fp, cp, op, lp, workspace.data_ptr(), self._workspace_bytes, handle))
        return copies, lacking

    def release(self, lens: torch.Tensor, stream=None) -> None:
        """Give up the pages behind each sequence's first lens slots (0: all of
        them) (af1_pages_release)."""
        _check(_pages_release(ctypes.byref(self._d), self._per_sequence(lens, "lens"), _stream_handle(stream)))

"""What a decoder step runs around its linears: rotary positions, a paged cache
of keys and values in 16, 8 or 4 bits, attention of drafted tokens over it,
and the scores of tokens.

Like the rest of the package this only marshals arguments to the C ABI of
include/af1.h, which has the formulas, the layouts and the errors. Tensors are
on the current CUDA device; index tensors are int32. `stream` (default: the
current one) takes the work; a tensor that a call allocates belongs to it.
"""
from __future__ import annotations

import ctypes
import math

import torch

from . import AF1_F16, AF1_F32, AF1Error, _check, _i64, _lib, _ptr, _vp, last_error

_i32 = ctypes.c_int32
_f32 = ctypes.c_float
_f64 = ctypes.c_double

KINDS = {"f16": 0, "int8": 1, "e4m3": 2, "int4": 3}
SCALINGS = {None: 0, "linear": 1, "base": 2, "bands": 3, "ramp": 4}
_INTERLEAVED, _BACKWARD = 1, 2


class _RopeParams(ctypes.Structure):
    _fields_ = [("length", _i64), ("dim", _i32), ("scaling", _i32), ("base", _f64), ("factor", _f64), ("low", _f64),
                ("high", _f64), ("original", _f64), ("attention", _f64)]


class _RopeArgs(ctypes.Structure):
    _fields_ = [("x", _vp), ("y", _vp), ("positions", _vp), ("table", _vp), ("tokens", _i64), ("heads", _i64),
                ("dim", _i64), ("rope_dim", _i64), ("length", _i64), ("x_token", _i64), ("x_head", _i64),
                ("y_token", _i64), ("y_head", _i64), ("dtype", _i32), ("flags", _i32)]


class _KvDesc(ctypes.Structure):
    _fields_ = [("pages", _i64), ("page_size", _i32), ("kv_heads", _i32), ("head_dim", _i32), ("kind", _i32),
                ("k", _vp), ("v", _vp), ("k_scale", _vp), ("v_scale", _vp)]


class _AppendArgs(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("k_token", _i64), ("k_head", _i64), ("v_token", _i64), ("v_head", _i64),
                ("seq", _vp), ("slot", _vp), ("positions", _vp), ("pages", _vp), ("tokens", _i64),
                ("sequences", _i64), ("page_columns", _i64), ("pages_ld", _i64), ("table", _vp), ("length", _i64),
                ("rope_dim", _i64), ("q", _vp), ("q_out", _vp), ("q_heads", _i64), ("q_token", _i64),
                ("q_head", _i64), ("qo_token", _i64), ("qo_head", _i64), ("k_out", _vp), ("v_out", _vp),
                ("dtype", _i32), ("flags", _i32)]


class _TreeArgs(ctypes.Structure):
    _fields_ = [("q", _vp), ("q_seq", _i64), ("q_node", _i64), ("q_head", _i64), ("out", _vp), ("o_seq", _i64),
                ("o_node", _i64), ("o_head", _i64), ("lse", _vp), ("pages", _vp), ("lens", _vp), ("counts", _vp),
                ("mask", _vp), ("mask_seq", _i64), ("sequences", _i64), ("nodes", _i64), ("q_heads", _i64),
                ("page_columns", _i64), ("pages_ld", _i64), ("scale", _f32), ("out_dtype", _i32)]


class _LogprobArgs(ctypes.Structure):
    _fields_ = [("logits", _vp), ("rows", _i64), ("vocab", _i64), ("ld", _i64), ("tokens", _vp), ("given", _i64),
                ("logprobs", _vp), ("entropy", _vp), ("top_logprobs", _vp), ("top_ids", _vp), ("top", _i32),
                ("dtype", _i32), ("temperature", _f32), ("reserved", _i32)]


def _declare(name, *args, restype=ctypes.c_int):
    f = getattr(_lib, name)
    f.argtypes, f.restype = list(args), restype
    return f


_P = ctypes.POINTER
_rope_frequencies = _declare("af1_rope_frequencies", _P(_RopeParams), _P(_f64), _P(_f64))
_rope_table = _declare("af1_rope_table", _P(_RopeParams), _vp, _vp)
_rope = _declare("af1_rope", _P(_RopeArgs), _vp)
_kv_create = _declare("af1_kv_create", _P(_KvDesc), _P(_vp))
_kv_free = _declare("af1_kv_free", _vp, restype=None)
_kv_append = _declare("af1_kv_append", _vp, _P(_AppendArgs), _vp)
_kv_read = _declare("af1_kv_read", _vp, _vp, _i64, _i64, _i64, _vp, _i64, _i64, _vp, _vp, ctypes.c_int, _vp)
_tree_mask = _declare("af1_tree_mask", _vp, _i64, _i64, _vp, _vp)
_tree_workspace = _declare("af1_tree_workspace_bytes", _vp, _i64, _i64, _i64, restype=_i64)
_tree_attention = _declare("af1_tree_attention", _vp, _P(_TreeArgs), _vp, _i64, _vp)
_token_logprobs = _declare("af1_token_logprobs", _P(_LogprobArgs), _vp)
# Of the runtime that the library is linked to; a slice of a tensor and its zero_() take the host 5 us more.
_memset = _declare("cudaMemsetAsync", _vp, ctypes.c_int, ctypes.c_size_t, _vp)


# What torch.cuda.current_stream().cuda_stream gives, without building the stream object (3 us of a call's 14); a
# torch without these functions takes the public way.
_raw_stream, _raw_device = (getattr(torch._C, f, None) for f in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))


def _stream_handle(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None or _raw_device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_raw_device())


# Bytes at the front of a workspace that are zero between calls.
_WORKSPACE_HEAD = 65792

_F16, _F32, _I32 = torch.float16, torch.float32, torch.int32
_KINDS_OF = {_F16: AF1_F16, _F32: AF1_F32}


def _dtype(t: torch.Tensor, what: str) -> int:
    kind = _KINDS_OF.get(t.dtype)
    if kind is None:
        raise ValueError(f"{what} must be float16 or float32")
    return kind


def _steps(t: torch.Tensor, what: str, dims: int):
    """Strides of all axes; the last one is 1. Axes of one entry have stride 0."""
    s = t.stride()
    if len(s) != dims or (s[-1] != 1 and t.shape[-1] > 1):
        raise ValueError(f"{what} must be {dims}-D with unit stride along its last axis")
    n = t.shape
    if 1 in n:
        return [0 if n[i] == 1 else s[i] for i in range(dims)]
    return s


def _index(t, what: str, shape) -> int:
    """Pointer of a contiguous int32 tensor of this shape, 0 for None."""
    if t is None:
        return 0
    if t.dtype is not _I32 or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous int32 tensor of shape {tuple(shape)}")
    return t.data_ptr()


def _empty(shape, dtype, device, stream) -> torch.Tensor:
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):  # the allocator may hand the memory on in that stream's order
        return torch.empty(shape, dtype=dtype, device=device)


def _pages(t: torch.Tensor):
    s = t.stride()
    if t.dtype is not _I32 or len(s) != 2 or (s[1] != 1 and t.shape[1] > 1):
        raise ValueError("pages must be a 2-D int32 tensor with contiguous rows")
    rows, columns = t.shape
    return t.data_ptr(), rows, columns, s[0] if rows > 1 else columns


# -- rotary positions ----------------------------------------------------------------


def _params(length, dim, base, scaling, factor, low, high, original, attention):
    if scaling not in SCALINGS:
        raise ValueError(f"scaling must be one of {list(SCALINGS)}")
    low = 1.0 if low is None else low
    high = (32.0 if scaling == "ramp" else 4.0) if high is None else high
    return _RopeParams(length, dim, SCALINGS[scaling], base, factor, low, high, original, attention)


def rope_frequencies(dim: int, base: float = 10000.0, scaling=None, factor: float = 1.0, low: float | None = None,
                     high: float | None = None, original: float = 0.0, attention: float = 0.0):
    """(list of dim / 2 frequencies, factor of cos and sin): af1_rope_frequencies, on the host.
    low, high: by default 1 and 4 for "bands", 1 and 32 for "ramp"."""
    p = _params(1, dim, base, scaling, factor, low, high, original, attention)
    freq, att = (_f64 * 128)(), _f64()
    _check(_rope_frequencies(ctypes.byref(p), freq, ctypes.byref(att)))
    return list(freq)[: dim // 2], att.value


def rope_table(length: int, dim: int, base: float = 10000.0, scaling=None, factor: float = 1.0,
               low: float | None = None, high: float | None = None, original: float = 0.0, attention: float = 0.0,
               device=None, stream=None) -> torch.Tensor:
    """cos and sin of positions 0 .. length - 1, float32 (length, dim / 2, 2)
    (af1_rope_table). scaling: None, "linear", "base", "bands" or "ramp";
    low, high: by default 1 and 4 for "bands", 1 and 32 for "ramp"."""
    p = _params(length, dim, base, scaling, factor, low, high, original, attention)
    table = _empty((max(length, 0), max(dim, 0) // 2, 2), torch.float32,
                   device or torch.device("cuda", torch.cuda.current_device()), stream)
    _check(_rope_table(ctypes.byref(p), table.data_ptr(), _stream_handle(stream)))
    return table


def _table(t: torch.Tensor):
    shape = t.shape
    if t.dtype is not _F32 or len(shape) != 3 or shape[2] != 2 or not t.is_contiguous():
        raise ValueError("the rotary table must be a contiguous float32 tensor (length, pairs, 2)")
    return t.data_ptr(), shape[0], 2 * shape[1]


def rope(x: torch.Tensor, positions: torch.Tensor, table: torch.Tensor, out: torch.Tensor | None = None,
         interleaved: bool = False, backward: bool = False, stream=None) -> torch.Tensor:
    """x (tokens, heads, dim) with the first 2 table.shape[1] entries of every
    head rotated to the tokens' positions (af1_rope); float16 or float32, out
    may be x. backward: the gradient of x from that of the output."""
    xs = _steps(x, "x", 3)
    dt = _dtype(x, "x")
    if out is None:
        out = _empty(x.shape, x.dtype, x.device, stream)
    elif out.shape != x.shape or out.dtype != x.dtype:
        raise ValueError("out must have the shape and dtype of x")
    ys = _steps(out, "out", 3)
    tokens, heads, dim = x.shape
    tp, length, rope_dim = _table(table)
    if heads == 0 or tokens == 0:
        return out
    a = _RopeArgs(x.data_ptr(), out.data_ptr(), _index(positions, "positions", (tokens,)), tp, tokens, heads, dim,
                  rope_dim, length, xs[0], xs[1], ys[0], ys[1], dt, (_INTERLEAVED if interleaved else 0) | (_BACKWARD if backward else 0))
    _check(_rope(ctypes.byref(a), _stream_handle(stream)))
    return out


# -- the paged cache --------------------------------------------------------------------


class KVCache:
    """A paged cache over the caller's tensors (af1_kv_create):

    kind    k, v                                          k_scale, v_scale
    f16     float16 (pages, kv_heads, page, dim)          None
    int8    int8                                          float32 (pages, kv_heads, page)
    e4m3    float8_e4m3fn                                 float32 (pages, kv_heads, page)
    int4    uint8 (pages, kv_heads, page, dim / 2)        float16 (pages, kv_heads, page, dim / 32, 2)

    all contiguous. The tensors are kept alive by this object. Sequences are
    rows of a table `pages` (sequences, columns) of int32 page numbers."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale=None, v_scale=None):
        self._h = None
        kinds = {torch.float16: "f16", torch.int8: "int8", torch.float8_e4m3fn: "e4m3", torch.uint8: "int4"}
        if k.dtype not in kinds or k.dim() != 4 or v.shape != k.shape or v.dtype != k.dtype:
            raise ValueError("k and v must be 4-D float16, int8, float8_e4m3fn or uint8 tensors of one shape")
        self.kind = kinds[k.dtype]
        self.pages, self.kv_heads, self.page_size = k.shape[:3]
        self.head_dim = k.shape[3] * (2 if self.kind == "int4" else 1)
        lead = tuple(k.shape[:3])
        want = {"f16": None, "int4": (torch.float16, lead + (self.head_dim // 32, 2))}.get(
            self.kind, (torch.float32, lead))
        for s in (k_scale, v_scale):
            if (s is None) != (want is None) or (s is not None and (s.dtype != want[0] or tuple(s.shape) != want[1])):
                raise ValueError(f"k_scale and v_scale of an {self.kind} cache must be {want}")
        for t in (k, v, k_scale, v_scale):
            if t is not None and not t.is_contiguous():
                raise ValueError("the cache's tensors must be contiguous")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        d = _KvDesc(self.pages, self.page_size, self.kv_heads, self.head_dim, KINDS[self.kind], _ptr(k), _ptr(v),
                    _ptr(k_scale), _ptr(v_scale))
        h = _vp()
        _check(_kv_create(ctypes.byref(d), ctypes.byref(h)))
        self._h = h.value

    @classmethod
    def empty(cls, pages: int, page_size: int, kv_heads: int, head_dim: int, kind: str = "int8", device=None):
        """A cache of zeros over tensors of its own."""
        if kind not in KINDS:
            raise ValueError(f"kind must be one of {list(KINDS)}")
        device = device or torch.device("cuda", torch.cuda.current_device())
        dtype = {"f16": torch.float16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn, "int4": torch.uint8}[kind]
        lead = (pages, kv_heads, page_size)
        parts = []
        for _ in "kv":
            parts.append(torch.zeros(lead + (head_dim // 2 if kind == "int4" else head_dim,), dtype=torch.uint8 if
                                     kind == "e4m3" else dtype, device=device).view(dtype))
        scales = [None, None]
        if kind == "int4":
            scales = [torch.zeros(lead + (head_dim // 32, 2), dtype=torch.float16, device=device) for _ in "kv"]
        elif kind != "f16":
            scales = [torch.zeros(lead, dtype=torch.float32, device=device) for _ in "kv"]
        return cls(*parts, *scales)

    def append(self, k: torch.Tensor, v: torch.Tensor, pages: torch.Tensor, seq: torch.Tensor, slot: torch.Tensor,
               rope: torch.Tensor | None = None, positions: torch.Tensor | None = None, q: torch.Tensor | None = None,
               q_out: torch.Tensor | None = None, interleaved: bool = False, k_out: torch.Tensor | None = None,
               v_out: torch.Tensor | None = None, stream=None):
        """Write k and v (tokens, kv_heads, head_dim), float16 or float32, to
        slot[i] of sequence seq[i] (af1_kv_append); keys are rotated with the
        table `rope` to `positions` (default: the slots). q (tokens, heads,
        head_dim) is rotated to the same positions; returns it as float16
        (q_out, allocated if not given), or None. k_out, v_out: float16
        (tokens, kv_heads, head_dim), receive the values that the cache holds."""
        ks, vs = _steps(k, "k", 3), _steps(v, "v", 3)
        dt = _dtype(k, "k")
        tokens = k.shape[0]
        shape = (tokens, self.kv_heads, self.head_dim)
        if k.shape != shape or v.shape != shape or v.dtype != k.dtype:
            raise ValueError(f"k and v must have shape {shape} and one dtype")
        for t in (k_out, v_out):
            if t is not None and (t.shape != shape or t.dtype != torch.float16 or not t.is_contiguous()):
                raise ValueError(f"k_out and v_out must be contiguous float16 tensors of shape {shape}")
        heads, qs, qos = 0, (0, 0, 1), (0, 0, 1)
        if q is not None:
            qs, heads = _steps(q, "q", 3), q.shape[1]
            if q.shape != (tokens, heads, self.head_dim) or q.dtype != k.dtype:
                raise ValueError("q must have k's tokens, head size and dtype")
            if q_out is None:
                q_out = _empty(q.shape, torch.float16, q.device, stream)
            elif q_out.shape != q.shape or q_out.dtype != torch.float16:
                raise ValueError("q_out must be float16 with the shape of q")
            qos = _steps(q_out, "q_out", 3)
        elif q_out is not None:
            raise ValueError("q_out without q")
        if tokens == 0:
            return q_out
        if q is not None and heads == 0:
            raise ValueError("q has no heads")
        tp, length, rope_dim = _table(rope) if rope is not None else (0, 0, 0)
        one = (tokens,)
        pp, sequences, columns, ld = _pages(pages)
        a = _AppendArgs(k.data_ptr(), v.data_ptr(), ks[0], ks[1], vs[0], vs[1], _index(seq, "seq", one),
                        _index(slot, "slot", one), _index(positions, "positions", one), pp, tokens, sequences,
                        columns, ld, tp, length, rope_dim, _ptr(q), _ptr(q_out), heads, qs[0], qs[1], qos[0],
                        qos[1], _ptr(k_out), _ptr(v_out), dt, _INTERLEAVED if interleaved else 0)
        _check(_kv_append(self._h, ctypes.byref(a), _stream_handle(stream)))
        return q_out

    def read(self, pages: torch.Tensor, lens: torch.Tensor, first: int = 0, count: int | None = None,
             dtype=torch.float16, k_out: torch.Tensor | None = None, v_out: torch.Tensor | None = None, stream=None):
        """(k, v) of slots first .. first + count - 1 of every sequence, each
        (sequences, count, kv_heads, head_dim) of dtype float16 or float32;
        slots at lens[sequence] and after are zeros (af1_kv_read). count
        defaults to the table's capacity after `first`."""
        pp, sequences, columns, ld = _pages(pages)
        if count is None:
            count = max(0, columns * self.page_size - first)
        shape = (sequences, count, self.kv_heads, self.head_dim)
        outs = []
        for t in (k_out, v_out):
            if t is None:
                t = _empty(shape, dtype, pages.device, stream)
            elif t.shape != shape or not t.is_contiguous():
                raise ValueError(f"k_out and v_out must be contiguous tensors of shape {shape}")
            outs.append(t)
        dt = _dtype(outs[0], "k_out")
        if outs[1].dtype != outs[0].dtype:
            raise ValueError("k_out and v_out must have one dtype")
        _check(_kv_read(self._h, pp, sequences, columns, ld, _index(lens, "lens", (sequences,)), first, count,
                        outs[0].data_ptr(), outs[1].data_ptr(), dt, _stream_handle(stream)))
        return outs[0], outs[1]

    def workspace_bytes(self, sequences: int, nodes: int, heads: int) -> int:
        v = _tree_workspace(self._h, sequences, nodes, heads)
        if v < 0:
            raise AF1Error(int(v), last_error())
        return int(v)

    def make_workspace(self, q: torch.Tensor, pages: torch.Tensor | None = None) -> torch.Tensor:
        """A workspace for tree_attention calls with queries of q's shape, or
        with fewer rows for each cached head; what has to be zero is. pages:
        the table of these calls, only checked against q."""
        if pages is not None and _pages(pages)[1] != q.shape[0]:
            raise ValueError("pages must have one row for each sequence")
        size = self.workspace_bytes(q.shape[0], q.shape[1], q.shape[2])
        if not q.is_cuda:
            return torch.zeros(size, dtype=torch.uint8, device=q.device)
        workspace = torch.empty(size, dtype=torch.uint8, device=q.device)
        if _memset(workspace.data_ptr(), 0, _WORKSPACE_HEAD, _stream_handle(None)) != 0:
            raise AF1Error(-6, "cudaMemsetAsync failed")
        return workspace

    def tree_attention(self, q: torch.Tensor, pages: torch.Tensor, lens: torch.Tensor,
                       mask: torch.Tensor | None = None, counts: torch.Tensor | None = None,
                       scale: float | None = None, out: torch.Tensor | None = None, lse: torch.Tensor | None = None,
                       workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
        """Attention of the nodes q (sequences, nodes, heads, head_dim),
        float16, over slots 0 .. lens - 1 and over the nodes' own slots as
        `mask` says (af1_tree_attention). mask: int32 (sequences or 1, nodes,
        words) from tree_mask, or None: each node sees the nodes up to itself.
        At most 1024 sequences and 64 nodes. counts: nodes of each sequence's
        tree. scale: default
        1 / sqrt(head_dim). out: float16 (default) or float32, the shape of q.
        lse: float32 (sequences, nodes, heads), optional."""
        qs = _steps(q, "q", 4)
        sequences, nodes, heads, dim = q.shape
        if q.dtype != torch.float16 or dim != self.head_dim:
            raise ValueError("q must be float16 with the cache's head size")
        if out is None:
            out = _empty(q.shape, torch.float16, q.device, stream)
        elif out.shape != q.shape:
            raise ValueError("out must have the shape of q")
        os = _steps(out, "out", 4)
        pp, rows, columns, ld = _pages(pages)
        if rows != sequences:
            raise ValueError("pages must have one row for each sequence")
        mask_seq = 0
        if mask is not None:
            if mask.dim() != 3 or mask.shape[0] not in (1, sequences):
                raise ValueError("mask must be (sequences or 1, nodes, words)")
            words = (nodes + 31) // 32
            mp = _index(mask, "mask", (mask.shape[0], nodes, words))
            mask_seq = nodes * words if mask.shape[0] == sequences else 0
        else:
            mp = 0
        if lse is not None and (lse.dtype != torch.float32 or lse.shape != q.shape[:3] or not lse.is_contiguous()):
            raise ValueError("lse must be a contiguous float32 tensor (sequences, nodes, heads)")
        if sequences == 0:
            return out
        if workspace is None:
            if stream is None:
                workspace = self.make_workspace(q)
            else:
                with torch.cuda.stream(stream):
                    workspace = self.make_workspace(q)
        a = _TreeArgs(q.data_ptr(), qs[0], qs[1], qs[2], out.data_ptr(), os[0], os[1], os[2], _ptr(lse), pp, _index(lens, "lens", (sequences,)),
                      _index(counts, "counts", (sequences,)), mp, mask_seq, sequences, nodes, heads, columns, ld,
                      1.0 / math.sqrt(dim) if scale is None else scale, _dtype(out, "out"))
        _check(_tree_attention(self._h, ctypes.byref(a), workspace.data_ptr(),
                               workspace.numel() * workspace.element_size(), _stream_handle(stream)))
        return out

    def free(self) -> None:
        if getattr(self, "_h", None):
            _kv_free(self._h)
            self._h = None

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass


def tree_mask(parents: torch.Tensor, stream=None) -> torch.Tensor:
    """Mask words (sequences, nodes, (nodes + 31) / 32) of trees given by the
    parents (sequences, nodes) of their nodes, negative for the children of
    the last cached token (af1_tree_mask)."""
    if parents.dim() != 2:
        raise ValueError("parents must be (sequences, nodes)")
    sequences, nodes = parents.shape
    mask = _empty((sequences, nodes, (nodes + 31) // 32), torch.int32, parents.device, stream)
    _check(_tree_mask(_index(parents, "parents", (sequences, nodes)), sequences, nodes, mask.data_ptr(),
                      _stream_handle(stream)))
    return mask


# -- scores ---------------------------------------------------------------------------------


def token_logprobs(logits: torch.Tensor, tokens: torch.Tensor | None = None, top: int = 0, temperature: float = 1.0,
                   stream=None):
    """Of rows of logits (rows, vocab), float16 or float32: (logprobs, entropy)
    or, with `top`, (logprobs, entropy, top_logprobs, top_ids)
    (af1_token_logprobs). tokens: int32 (rows, given), or None (logprobs is
    then (rows, 0))."""
    ld = _steps(logits, "logits", 2)[0]
    dt = _dtype(logits, "logits")
    rows, vocab = logits.shape
    if tokens is not None and (tokens.dim() != 2 or tokens.shape[0] != rows):
        raise ValueError("tokens must be (rows, given)")
    given = 0 if tokens is None else tokens.shape[1]
    device = logits.device
    logprobs = _empty((rows, given), _F32, device, stream)
    entropy = _empty((rows,), _F32, device, stream)
    best = ids = None
    if top:
        best, ids = _empty((rows, top), _F32, device, stream), _empty((rows, top), _I32, device, stream)
    if rows > 0:
        a = _LogprobArgs(logits.data_ptr(), rows, vocab, ld if rows > 1 else vocab,
                         _index(tokens, "tokens", (rows, given)) if given else 0, given,
                         logprobs.data_ptr() if given else 0, entropy.data_ptr(), _ptr(best), _ptr(ids), top, dt,
                         temperature, 0)
        _check(_token_logprobs(ctypes.byref(a), _stream_handle(stream)))
    return (logprobs, entropy, best, ids) if top else (logprobs, entropy)

"""Serving from the key-value cache in K-means codes (include/kmeans.h): Python binding.

    kmeans_kv_rotate(q, k, positions, frequencies, interleaved=False, inverse=False,
                     amplitude=1.0, out=None) -> (q, k)
    kmeans_kv_attend_tokens(cache, q, bounds, table, lengths, scale=None, cap=0.0,
                            slopes=None, window=0, prefixes=None, starts=None, out=None,
                            lse=None, ws=None) -> (out, lse)
    kmeans_kv_weigh(cache, q, lse, bounds, table, lengths, weights=None, scale=None,
                    cap=0.0, slopes=None, window=0, prefixes=None, starts=None) -> weights
    kmeans_kv_evict(cache, weights, table, lengths, keep, recent=0, first=0, to=None)
        -> (kept, lengths, weights)

As in kv.py, everything runs on the current stream of the tensors' device, no call
waits for it or reads device data back, and no call carries a gradient (that of
kmeans_kv_rotate is the call with inverse=True on the outputs' gradients).
"""
from __future__ import annotations

import ctypes
import math

import torch

from . import KmeansError, KMEANS_EUNSUPPORTED, _lib
from . import kv as _kv
from .kv import (KVCodes, _TYPES, _apart, _call, _current_device, _Desc, _ints, _no_gradient,
                 _raw_stream, _rows, _strides, _target)

_INTERLEAVED, _INVERSE = 1, 2           # KMEANS_KV_INTERLEAVED, KMEANS_KV_INVERSE


class _Turn(ctypes.Structure):
    """kmeans_kv_turn_t"""
    _fields_ = [("positions", ctypes.c_void_p), ("frequencies", ctypes.c_void_p),
                ("tokens", ctypes.c_int64), ("dim", ctypes.c_int32), ("half", ctypes.c_int32),
                ("type", ctypes.c_int32), ("flags", ctypes.c_uint32),
                ("amplitude", ctypes.c_float)]


class _Tokens(ctypes.Structure):
    """kmeans_kv_tokens_t"""
    _fields_ = [("bounds", ctypes.c_void_p), ("table", ctypes.c_void_p),
                ("table_stride", ctypes.c_int64), ("table_pages", ctypes.c_int64),
                ("lengths", ctypes.c_void_p), ("starts", ctypes.c_void_p),
                ("prefixes", ctypes.c_void_p), ("slopes", ctypes.c_void_p),
                ("tokens", ctypes.c_int64), ("seqs", ctypes.c_int32), ("q_heads", ctypes.c_int32),
                ("window", ctypes.c_int32), ("scale", ctypes.c_float), ("cap", ctypes.c_float)]


class _Evict(ctypes.Structure):
    """kmeans_kv_evict_t"""
    _fields_ = [("table", ctypes.c_void_p), ("table_stride", ctypes.c_int64),
                ("table_pages", ctypes.c_int64), ("lengths", ctypes.c_void_p),
                ("weights", ctypes.c_void_p), ("weights_seq", ctypes.c_int64),
                ("weights_head", ctypes.c_int64), ("positions", ctypes.c_int64),
                ("seqs", ctypes.c_int32), ("keep", ctypes.c_int32), ("recent", ctypes.c_int32),
                ("first", ctypes.c_int32), ("to", ctypes.c_void_p), ("to_stride", ctypes.c_int64),
                ("to_pages", ctypes.c_int64)]


def _bind():
    p, i64, i32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t
    d, t = ctypes.POINTER(_Desc), ctypes.POINTER(_Tokens)
    x = [p, i64, i64, i32, p, i64, i64]
    _lib.kmeans_kv_rotate.argtypes = [ctypes.POINTER(_Turn), *x, *x, p]
    _lib.kmeans_kv_rotate.restype = ctypes.c_int
    _lib.kmeans_kv_attend_tokens_workspace_bytes.argtypes = [d, t]
    _lib.kmeans_kv_attend_tokens_workspace_bytes.restype = sz
    _lib.kmeans_kv_attend_tokens.argtypes = [d, t, p, i64, i64, p, i64, i64, p, p, sz, p]
    _lib.kmeans_kv_attend_tokens.restype = ctypes.c_int
    _lib.kmeans_kv_weigh.argtypes = [d, t, p, i64, i64, p, p, i64, i64, i64, i32, p]
    _lib.kmeans_kv_weigh.restype = ctypes.c_int
    _lib.kmeans_kv_evict.argtypes = [d, ctypes.POINTER(_Evict), p, p, p, i64, i64, p]
    _lib.kmeans_kv_evict.restype = ctypes.c_int
    if _kv._fast is not None:
        _kv._fast.bind_serve(*(ctypes.cast(f, ctypes.c_void_p).value
                               for f in (_lib.kmeans_kv_rotate,
                                         _lib.kmeans_kv_attend_tokens_workspace_bytes,
                                         _lib.kmeans_kv_attend_tokens, _lib.kmeans_kv_weigh,
                                         _lib.kmeans_kv_evict)))


_bind()


class _Like:
    """What the checks of kv.py ask of a cache, of a tensor that stands alone."""

    def __init__(self, t):
        self.dtype, self.device, self.index, self.dim = t.dtype, t.device, t.get_device(), t.shape[2]


def _here(index, device, fn, name, *args):
    """fn on a device and its current stream."""
    if _current_device() == index:
        rc = fn(*args, _raw_stream(index))
    else:
        with torch.cuda.device(device):
            rc = fn(*args, _raw_stream(index))
    if rc:
        raise KmeansError(name, rc)


def kmeans_kv_rotate(q: torch.Tensor, k: torch.Tensor | None, positions: torch.Tensor,
                     frequencies: torch.Tensor, interleaved: bool = False, inverse: bool = False,
                     amplitude: float = 1.0, out=None):
    """Turns queries and keys by their positions (rotary positions).

    q, k         [tokens, heads, dim], bfloat16 or float16, both alike but for
                 their heads (k may be None); dim a multiple of 8 up to 512
    positions    int64 [tokens]
    frequencies  float64 [pairs], radians to a position; 2 * pairs <= dim features
                 of every head are turned, the others copied; constants, as
                 everywhere here: those that need a gradient are refused
    interleaved  pairs are features (2i, 2i + 1), else (i, i + pairs)
    inverse      by the negative angle: what takes gradients of the outputs to
                 those of q and k
    amplitude    factor of the turned features

    Returns the turned tensors (q, k). `out` may supply them, among them q and k
    themselves, or others of the same memory with the same strides."""
    flags = (_INTERLEAVED if interleaved else 0) | (_INVERSE if inverse else 0)
    if _kv._fast is not None and out is None:
        index = _current_device()
        got = _kv._fast.rotate(index, _raw_stream(index), q, k, positions, frequencies, flags,
                               amplitude)
        if type(got) is tuple:
            return got
        if got is not None:
            raise KmeansError("kmeans_kv_rotate", got)
    if not (isinstance(q, torch.Tensor) and q.is_cuda and q.dim() == 3 and q.dtype in _TYPES):
        raise ValueError("q must be a bfloat16 or float16 [tokens, heads, dim] tensor on a GPU")
    like = _Like(q)
    if not (isinstance(frequencies, torch.Tensor) and frequencies.dtype is torch.float64
            and frequencies.dim() == 1 and frequencies.get_device() == like.index):
        raise ValueError("frequencies must be a float64 [pairs] tensor on q's GPU")
    _no_gradient(frequencies, "frequencies")
    tokens = q.shape[0]
    positions = _ints(like, positions, torch.int64, tokens, "positions")
    frequencies = frequencies.contiguous()
    outs = (None, None) if out is None else out
    args, got, kept = [], [], []
    for t, o, what in ((q, outs[0], "q"), (k, outs[1], "k")):
        if t is None:
            args += [None, 0, 0, 0, None, 0, 0]
            got.append(None)
            continue
        in_place = o is t
        rows, at, shape, a, b = _rows(like, t, what)
        _no_gradient(rows, what)
        if shape[0] != tokens:
            raise ValueError(f"k must have {tokens} tokens, as q has")
        kept.append(rows)
        if in_place and rows is not t:
            raise ValueError(f"{what} in place needs contiguous features and rows on 16 bytes")
        if o is None and t.is_contiguous() and rows is t:
            o = torch.empty_like(t)
            to, oa, ob = o.data_ptr(), a, b
        else:
            o, to, oa, ob = _target(like, o, shape, what)
        if at and o.data_ptr() == at:       # in place, whichever tensor says so
            a, b, oa, ob = *_strides(rows)[:2], *_strides(o)[:2]
            if (a, b) != (oa, ob):
                raise ValueError(f"out for {what} begins where {what} does, with other strides")
        args += [at, a, b, shape[1], to, oa, ob]
        got.append(o)
    if 2 * frequencies.shape[0] > like.dim:
        raise ValueError("more features are turned than a head has")
    turn = _Turn(positions.data_ptr(), frequencies.data_ptr(), tokens, like.dim,
                 frequencies.shape[0], _TYPES[q.dtype], flags, amplitude)
    _here(like.index, like.device, _lib.kmeans_kv_rotate, "kmeans_kv_rotate", turn, *args)
    return tuple(got)


def _table(cache, table, seqs, what="table"):
    if not (isinstance(table, torch.Tensor) and table.dtype is torch.int32 and table.dim() == 2
            and table.get_device() == cache.index and table.shape[0] == seqs):
        raise ValueError(f"{what} must be an int32 [{seqs}, pages] tensor on the cache's GPU")
    return table if table.stride(1) == 1 else table.contiguous()


def _new_tokens(cache, q, bounds, table, lengths, scale, cap, slopes, window, prefixes, starts):
    """kmeans_kv_tokens_t, q as the library takes it, and what must live until the call."""
    q, qp, shape, qa, qb = _rows(cache, q, "q")
    _no_gradient(q, "q")
    tokens, q_heads, _ = shape
    if q_heads < 1 or q_heads % cache.heads:
        raise ValueError(f"q must have a multiple of {cache.heads} heads")
    lengths = _ints(cache, lengths, torch.int32, None, "lengths")
    seqs = lengths.shape[0]
    bounds = _ints(cache, bounds, torch.int32, seqs + 1, "bounds")
    table = _table(cache, table, seqs)
    if prefixes is not None:
        prefixes = _ints(cache, prefixes, torch.int32, seqs, "prefixes")
    if starts is not None:
        starts = _ints(cache, starts, torch.int32, tokens, "starts")
    if slopes is not None:
        slopes = _ints(cache, slopes, torch.float32, q_heads, "slopes")
        _no_gradient(slopes, "slopes")
    if not 0 <= window < 1 << 31:
        raise ValueError("window must be a number of positions, or 0")
    t = _Tokens(bounds.data_ptr(), table.data_ptr(), table.stride(0), table.shape[1],
                lengths.data_ptr(), None if starts is None else starts.data_ptr(),
                None if prefixes is None else prefixes.data_ptr(),
                None if slopes is None else slopes.data_ptr(), tokens, seqs, q_heads, window,
                scale, cap)
    if t.table_pages == 0:              # no position anywhere
        lengths = torch.zeros_like(lengths)
        table = torch.zeros((seqs, 1), dtype=torch.int32, device=cache.device)
        t.lengths, t.table, t.table_stride, t.table_pages = (lengths.data_ptr(), table.data_ptr(),
                                                             1, 1)
    return t, q, qp, qa, qb, (q, bounds, table, lengths, starts, prefixes, slopes)


def kmeans_kv_attend_tokens_workspace_bytes(cache: KVCodes, tokens: int, seqs: int, q_heads: int,
                                            table_pages: int) -> int:
    """Bytes that kmeans_kv_attend_tokens takes for its workspace; 0 if it refuses."""
    t = _Tokens(table_pages=max(table_pages, 1), tokens=tokens, seqs=seqs, q_heads=q_heads)
    return int(_lib.kmeans_kv_attend_tokens_workspace_bytes(cache._ref, t))


def kmeans_kv_attend_tokens(cache: KVCodes, q: torch.Tensor, bounds: torch.Tensor,
                            table: torch.Tensor, lengths: torch.Tensor, scale: float | None = None,
                            cap: float = 0.0, slopes: torch.Tensor | None = None, window: int = 0,
                            prefixes: torch.Tensor | None = None,
                            starts: torch.Tensor | None = None, out=None, lse=None,
                            ws: torch.Tensor | None = None):
    """Attention of many new tokens of every sequence over its cached positions, their
    own among them (they have been written before).

    q         [tokens, q_heads, dim], q_heads a multiple of the cache's heads
    bounds    int32 [seqs + 1], ascending: sequence b has the tokens bounds[b] to
              bounds[b + 1] - 1, the last of its positions
    table     int32 [seqs, pages of a sequence]: page numbers
    lengths   int32 [seqs]: cached positions, the new tokens' included
    scale     of the scores, 1 / sqrt(dim) if None
    cap       scores become cap * tanh(score / cap), 0: they do not; scale / cap is
              0 or a normal fp32 number, as most caps up to 1e36 make it
    slopes    float32 [q_heads]: a score loses slope * distance in positions
    window    a token sees its own position and the window - 1 before it, 0: all
    prefixes  int32 [seqs]: first positions that every token of a sequence sees
    starts    int32 [tokens]: the first position that a token sees (its document's,
              or what padding leaves)

    Returns (out, lse): out like q, lse float32 [tokens, q_heads], the logarithm of
    the sum of the scores' exponentials (-inf, with out 0, where nothing is seen).
    Tokens outside every sequence are not written. `out` and `lse` may supply the
    tensors, `ws` the workspace (kmeans_kv_attend_tokens_workspace_bytes)."""
    if scale is None:
        scale = 1.0 / math.sqrt(cache.dim)
    if (_kv._fast is not None and out is None and lse is None and ws is None
            and _current_device() == cache.index):
        got = _kv._fast.attend_tokens(cache._at, cache.k_centres, _raw_stream(cache.index), q, bounds,
                                      table, lengths, scale, cap, slopes, window, prefixes, starts)
        if type(got) is tuple:
            return got
        if got is not None:
            raise KmeansError("kmeans_kv_attend_tokens", got)
    t, q, qp, qa, qb, _keep = _new_tokens(cache, q, bounds, table, lengths, scale, cap, slopes,
                                          window, prefixes, starts)
    shape = q.shape
    if out is None and q.is_contiguous():
        out, oa, ob = torch.empty_like(q), qa, qb
        op = out.data_ptr()
    else:
        out, op, oa, ob = _target(cache, out, shape, "out")
    if lse is None:
        lse = torch.empty(shape[:2], dtype=torch.float32, device=cache.device)
    elif not (lse.dtype is torch.float32 and lse.shape == shape[:2] and lse.is_contiguous()
              and lse.get_device() == cache.index):
        raise ValueError(f"lse must be a contiguous float32 {tuple(shape[:2])} tensor on the "
                         "cache's GPU")
    else:
        _no_gradient(lse, "lse")
    if t.seqs == 0 or t.tokens == 0:
        return out, lse
    if ws is None:
        nbytes = int(_lib.kmeans_kv_attend_tokens_workspace_bytes(cache._ref, t))
        if nbytes == 0:
            raise KmeansError("kmeans_kv_attend_tokens", KMEANS_EUNSUPPORTED)
        ws = torch.empty(nbytes, dtype=torch.uint8, device=cache.device)
    else:
        if ws.get_device() != cache.index or not ws.is_contiguous():
            raise ValueError("ws must be a contiguous tensor on the cache's GPU")
        nbytes = ws.numel() * ws.element_size()
    _call(cache, _lib.kmeans_kv_attend_tokens, "kmeans_kv_attend_tokens", t, qp, qa, qb, op, oa, ob,
          lse.data_ptr(), ws.data_ptr(), nbytes)
    return out, lse


def _weights(cache, w, seqs, what):
    """A float32 [seqs, heads, positions] tensor with contiguous rows, and its strides."""
    if not (isinstance(w, torch.Tensor) and w.dtype is torch.float32 and w.dim() == 3
            and w.get_device() == cache.index and w.shape[0] == seqs
            and w.shape[1] == cache.heads):
        raise ValueError(f"{what} must be a float32 [{seqs}, {cache.heads}, positions] tensor on "
                         "the cache's GPU")
    _no_gradient(w, what)
    a, b, c = _strides(w)
    return a, b, c == 1 or w.shape[2] <= 1


def kmeans_kv_weigh(cache: KVCodes, q: torch.Tensor, lse: torch.Tensor, bounds: torch.Tensor,
                    table: torch.Tensor, lengths: torch.Tensor,
                    weights: torch.Tensor | None = None, scale: float | None = None,
                    cap: float = 0.0, slopes: torch.Tensor | None = None, window: int = 0,
                    prefixes: torch.Tensor | None = None, starts: torch.Tensor | None = None):
    """The weight that the attention of new tokens gave to every cached position:
    weights[b, h, i] is the sum of exp(score - lse) over the new tokens of sequence b and
    the query heads of key-value head h.

    lse      float32 [tokens, q_heads] that kmeans_kv_attend_tokens (or kmeans_kv_attend)
             returned with the same arguments
    weights  float32 [seqs, heads, positions], which the sums are added to; None: a new
             tensor with as many positions as a row of table has
    others   as of kmeans_kv_attend_tokens

    Returns weights."""
    if scale is None:
        scale = 1.0 / math.sqrt(cache.dim)
    if _kv._fast is not None and weights is None and _current_device() == cache.index:
        got = _kv._fast.weigh(cache._at, cache.k_centres, _raw_stream(cache.index), q, bounds, table,
                              lengths, lse, scale, cap, slopes, window, prefixes, starts)
        if type(got) is tuple:
            return got[0]
        if got is not None:
            raise KmeansError("kmeans_kv_weigh", got)
    t, q, qp, qa, qb, _keep = _new_tokens(cache, q, bounds, table, lengths, scale, cap, slopes,
                                          window, prefixes, starts)
    if not (isinstance(lse, torch.Tensor) and lse.dtype is torch.float32
            and lse.shape == q.shape[:2] and lse.get_device() == cache.index):
        raise ValueError(f"lse must be a float32 {tuple(q.shape[:2])} tensor on the cache's GPU")
    _no_gradient(lse, "lse")
    lse = lse.contiguous()
    add = weights is not None
    if not add:
        weights = torch.empty((t.seqs, cache.heads, table.shape[1] * cache.page),
                              dtype=torch.float32, device=cache.device)
    a, b, rows = _weights(cache, weights, t.seqs, "weights")
    if not rows or not _apart(t.seqs, a, cache.heads, b, weights.shape[2]):
        raise ValueError("weights needs contiguous positions, and no two elements in one place")
    if weights.numel():
        _call(cache, _lib.kmeans_kv_weigh, "kmeans_kv_weigh", t, qp, qa, qb, lse.data_ptr(),
              weights.data_ptr(), a, b, weights.shape[2], int(add))
    return weights


def kmeans_kv_evict(cache: KVCodes, weights: torch.Tensor, table: torch.Tensor,
                    lengths: torch.Tensor, keep: int, recent: int = 0, first: int = 0,
                    to: torch.Tensor | None = None):
    """Brings every sequence of more than `keep` positions down to `keep`: each head keeps
    the last `recent`, the first `first`, and the positions of the largest weight between
    (ties go to the lowest position).

    weights  float32 [seqs, heads, positions] (kmeans_kv_weigh)
    table    int32 [seqs, pages of a sequence]; no two sequences share a page that is
             written to
    lengths  int32 [seqs]: cached positions
    to       int32 [seqs, pages]: pages, none of them in table, that take the codes that
             are kept

    Without `to` the codes move to the front of the sequence's own pages, and weights and
    lengths are written in place; with it both are new tensors, and the table's pages
    stay as they are. Returns (kept, lengths, weights): kept int32 [seqs, heads, keep], the
    positions in their order, -1 past the last; weights those of the kept positions, then
    zeros."""
    if _kv._fast is not None and _current_device() == cache.index:
        got = _kv._fast.evict(cache._at, cache.k_centres, _raw_stream(cache.index), weights, table,
                              lengths, keep, recent, first, to)
        if type(got) is tuple:
            return got
        if got is not None:
            raise KmeansError("kmeans_kv_evict", got)
    lengths = _ints(cache, lengths, torch.int32, None, "lengths") if to is not None else lengths
    if to is None and not (isinstance(lengths, torch.Tensor) and lengths.dtype is torch.int32
                           and lengths.get_device() == cache.index and lengths.dim() == 1
                           and lengths.is_contiguous()):
        raise ValueError("lengths must be a contiguous 1-D int32 tensor on the cache's GPU")
    seqs = lengths.shape[0]
    a, b, rows = _weights(cache, weights, seqs, "weights")
    positions = weights.shape[2]
    table = _table(cache, table, seqs)
    if to is None:
        if not rows or not _apart(seqs, a, cache.heads, b, positions):
            raise ValueError("weights needs contiguous positions, and no two elements in one place")
        new_lengths, new_weights, oa, ob = lengths, weights, a, b
    else:
        if not rows:
            weights = weights.contiguous()
            a, b, _ = _weights(cache, weights, seqs, "weights")
        to = _table(cache, to, seqs, "to")
        new_lengths = torch.empty_like(lengths)
        new_weights = torch.empty((seqs, cache.heads, positions), dtype=torch.float32,
                                  device=cache.device)
        oa, ob = cache.heads * positions, positions
    if not (1 <= keep < 1 << 31 and 0 <= recent < 1 << 31 and 0 <= first < 1 << 31
            and recent + first <= keep):
        raise ValueError("keep must be at least 1, and recent + first at most keep")
    kept = torch.empty((seqs, cache.heads, keep), dtype=torch.int32, device=cache.device)
    if seqs and table.shape[1] == 0:    # no position anywhere
        return kept.fill_(-1), new_lengths.zero_(), new_weights.zero_()
    e = _Evict(table.data_ptr(), table.stride(0), table.shape[1], lengths.data_ptr(),
               weights.data_ptr(), a, b, positions, seqs, keep, recent, first,
               None if to is None else to.data_ptr(), 0 if to is None else to.stride(0),
               0 if to is None else to.shape[1])
    if seqs:
        _call(cache, _lib.kmeans_kv_evict, "kmeans_kv_evict", e, kept.data_ptr(),
              new_lengths.data_ptr(), new_weights.data_ptr(), oa, ob)
    return kept, new_lengths, new_weights

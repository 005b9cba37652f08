"""The key-value cache in K-means codes (include/kmeans.h): Python binding.

    cache = KVCodes.empty(k_centres, v_centres, pages, page)
    kmeans_kv_write(cache, k, v, slots)
    kmeans_kv_read(cache, slots, out=None) -> (k, v)
    kmeans_kv_attend(cache, q, table, lengths, scale=None, starts=None, out=None,
                     lse=None, ws=None) -> (out, lse)

Everything runs on the current stream of the cache's device; no call waits for
it or reads device data back. No call carries a gradient: keys and values are
written as constants, the codes and centres are constants, and a query or an
output that needs a gradient is refused (torch.no_grad() says that it does not).
"""
from __future__ import annotations

import ctypes
import math
import warnings

import torch
from torch.autograd import forward_ad

from . import KmeansError, KMEANS_EUNSUPPORTED, _lib

# The usual calls in C++. Without it, or with one built for another torch, every
# call takes the steps below: the same results, 4 to 7 us later.
try:
    from . import _kv_call as _fast
    _without = None
    if getattr(_fast, "torch_version", None) != str(torch.__version__):
        _fast, _without = None, f"it was not built for torch {torch.__version__}"
except ImportError as e:
    _fast, _without = None, str(e)

# a tenth of the time of torch.cuda.current_stream and current_device, which
# small calls would mostly consist of
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                      lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)

_TYPES = {torch.bfloat16: 0, torch.float16: 1}      # KMEANS_KV_BF16, KMEANS_KV_FP16


class _Desc(ctypes.Structure):
    """kmeans_kv_t"""
    _fields_ = [("k_centres", ctypes.c_void_p), ("v_centres", ctypes.c_void_p),
                ("k_codes", ctypes.c_void_p), ("v_codes", ctypes.c_void_p),
                ("pages", ctypes.c_int64), ("page", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("dim", ctypes.c_int32), ("sub", ctypes.c_int32), ("K", ctypes.c_int32),
                ("type", ctypes.c_int32)]


def _bind():
    p, i64, i32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t
    d = ctypes.POINTER(_Desc)
    _lib.kmeans_kv_write.argtypes = [d, p, i64, i64, p, i64, i64, p, i64, p]
    _lib.kmeans_kv_write.restype = ctypes.c_int
    _lib.kmeans_kv_read.argtypes = [d, p, i64, p, i64, i64, p, i64, i64, p]
    _lib.kmeans_kv_read.restype = ctypes.c_int
    _lib.kmeans_kv_attend_workspace_bytes.argtypes = [d, i32, i32, i64]
    _lib.kmeans_kv_attend_workspace_bytes.restype = sz
    _lib.kmeans_kv_attend.argtypes = [d, p, i64, i64, i32, i32, p, i64, i64, p, p, ctypes.c_float,
                                      p, i64, i64, p, p, sz, p]
    _lib.kmeans_kv_attend.restype = ctypes.c_int
    if _fast is not None:
        _fast.bind(*(ctypes.cast(f, ctypes.c_void_p).value
                     for f in (_lib.kmeans_kv_write, _lib.kmeans_kv_read,
                               _lib.kmeans_kv_attend_workspace_bytes, _lib.kmeans_kv_attend)))


_bind()


class KVCodes:
    """A paged cache of codes and the centres they name.

    k_centres, v_centres  [heads, dim / sub, K, sub], bfloat16 or float16
    k_codes               [pages, heads, page, dim / sub], uint8
    v_codes               [pages, heads, dim / sub, page], uint8

    all contiguous on one GPU. The tensors are kept, not copied: what is written
    to them is what the calls see. Other tensors, or other sizes, are another
    KVCodes: these attributes cannot be set."""

    _KEPT = frozenset(("k_centres", "v_centres", "k_codes", "v_codes", "pages", "page", "heads",
                       "dim", "sub", "K", "dtype", "device", "index"))

    def __setattr__(self, name, value):
        # the library has their addresses and sizes; an operation in place, which ends
        # by setting what was there, is none of this
        if name in self._KEPT and self.__dict__.get(name, value) is not value:
            raise AttributeError(f"{name} of a KVCodes cannot be set: make another")
        object.__setattr__(self, name, value)

    def __delattr__(self, name):
        raise AttributeError(f"{name} of a KVCodes cannot be deleted")

    def __init__(self, k_centres, v_centres, k_codes, v_codes):
        tensors = (k_centres, v_centres, k_codes, v_codes)
        if not all(isinstance(t, torch.Tensor) and t.is_cuda and t.dim() == 4
                   and t.is_contiguous() and t.device == k_centres.device for t in tensors):
            raise ValueError("centres and codes must be contiguous 4-D tensors on one GPU")
        if k_centres.dtype not in _TYPES or v_centres.dtype != k_centres.dtype:
            raise ValueError("centres must be bfloat16 or float16, both alike")
        if k_codes.dtype != torch.uint8 or v_codes.dtype != torch.uint8:
            raise ValueError("codes must be uint8")
        heads, S, K, sub = k_centres.shape
        pages, _, page, _ = k_codes.shape
        if (v_centres.shape != k_centres.shape or k_codes.shape != (pages, heads, page, S)
                or v_codes.shape != (pages, heads, S, page)):
            raise ValueError("shapes of centres and codes do not belong together")
        self.k_centres, self.v_centres, self.k_codes, self.v_codes = tensors
        self.pages, self.page, self.heads, self.dim, self.sub, self.K = (
            pages, page, heads, S * sub, sub, K)
        self.dtype, self.device = k_centres.dtype, k_centres.device
        self._desc = _Desc(*(t.data_ptr() for t in tensors), pages, page, heads, S * sub, sub, K,
                           _TYPES[self.dtype])
        self._ref = ctypes.byref(self._desc)
        self._at = ctypes.addressof(self._desc)
        self.index = k_centres.get_device()
        self._ws_bytes = {}
        # the library says what it takes; it looks at no pointer here
        if not self.attend_workspace_bytes(1, heads, 1):
            raise KmeansError("KVCodes", KMEANS_EUNSUPPORTED)
        if _fast is None:
            warnings.warn("_kv_call cannot be used, the cache's calls take 4 to 7 us longer "
                          f"(`python paper_1402_3788_amd/build.py` builds it): {_without}",
                          RuntimeWarning, stacklevel=2)

    @classmethod
    def empty(cls, k_centres, v_centres, pages: int, page: int):
        """A cache of `pages` pages of `page` tokens, all codes 0."""
        if not (isinstance(k_centres, torch.Tensor) and k_centres.dim() == 4):
            raise ValueError("centres must be [heads, dim / sub, K, sub]")
        heads, S = k_centres.shape[:2]
        codes = [torch.zeros(shape, dtype=torch.uint8, device=k_centres.device)
                 for shape in ((pages, heads, page, S), (pages, heads, S, page))]
        return cls(k_centres, v_centres, *codes)

    def attend_workspace_bytes(self, seqs: int, q_heads: int, table_pages: int) -> int:
        """Bytes that kmeans_kv_attend takes for its workspace; 0 if it refuses."""
        key = (seqs, q_heads, table_pages)
        nbytes = self._ws_bytes.get(key)
        if nbytes is None:
            nbytes = int(_lib.kmeans_kv_attend_workspace_bytes(self._ref, *key))
            if len(self._ws_bytes) < 4096:
                self._ws_bytes[key] = nbytes
        return nbytes


def _no_gradient(t, what):
    """Refuses a tensor whose gradient the caller would miss without a word."""
    if (t.requires_grad and torch.is_grad_enabled()) or (
            forward_ad._current_level >= 0 and forward_ad.unpack_dual(t).tangent is not None):
        raise ValueError(f"{what} needs a gradient, which these calls do not carry: detach it, "
                         "or call them under torch.no_grad()")


def _strides(t):
    """t's strides; 0 for a dimension of one, whose stride leads nowhere and may
    be any number."""
    return tuple(s if n > 1 else 0 for n, s in zip(t.shape[:2], t.stride())) + t.stride()[2:]


def _rows(cache, t, what):
    """t as the library takes it, [n, heads, dim] with its features contiguous
    and its rows on 16 bytes (a copy where it is not), its address, its shape
    and its two strides."""
    if not (isinstance(t, torch.Tensor) and t.dtype is cache.dtype
            and t.get_device() == cache.index and t.dim() == 3 and t.shape[2] == cache.dim):
        raise ValueError(f"{what} must be a [n, heads, {cache.dim}] tensor of the cache's type "
                         "on its GPU")
    a, b, c = t.stride()
    at = t.data_ptr()
    if c != 1 or (a | b) & 7 or at & 15:
        t = t.contiguous()
        if t.data_ptr() & 15:
            t = t.clone()
        a, b, c = _strides(t)
        at = t.data_ptr()
    return t, at, t.shape, a, b


def _apart(n, a, heads, b, dim):
    """Whether rows of dim features, n of them a apart for each of the heads b apart,
    have no element in common."""
    if heads * b <= a and b >= dim:             # the usual ones
        return True
    if n == 0 or heads == 0:
        return True
    (n, a), (heads, b) = sorted(((n, a), (heads, b)), key=lambda x: x[1] if x[0] > 1 else 0)
    if n == 1:
        return heads == 1 or b >= dim
    if a < dim:
        return False
    if (n - 1) * a + dim <= b:                  # one run of rows ends before the next
        return True
    # runs that lie among each other: the rows next to j b of the first run
    return all(j * b - i * a >= dim and (i + 1 == n or (i + 1) * a - j * b >= dim)
               for j in range(1, heads) for i in (min(j * b // a, n - 1),))


def _target(cache, t, shape, what):
    """An output that the caller gave, or a new one; its address and strides."""
    if t is None:
        t = torch.empty(shape, dtype=cache.dtype, device=cache.device)
        return t, t.data_ptr(), shape[1] * shape[2], shape[2]
    if not (isinstance(t, torch.Tensor) and tuple(t.shape) == tuple(shape)
            and t.dtype is cache.dtype and t.get_device() == cache.index):
        raise ValueError(f"{what} must be {tuple(shape)} of the cache's type on its GPU")
    _no_gradient(t, what)
    a, b, c = t.stride()
    if (a | b) & 7:
        a, b, c = _strides(t)
    if c != 1 or (a | b) & 7 or t.data_ptr() & 15 or not _apart(shape[0], a, shape[1], b, shape[2]):
        raise ValueError(f"{what} needs contiguous features, rows on 16 bytes, and no two "
                         "elements in one place")
    return t, t.data_ptr(), a, b


def _ints(cache, t, dtype, n, what):
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == cache.index
            and t.dim() == 1 and (n is None or t.shape[0] == n)):
        raise ValueError(f"{what} must be a 1-D {dtype} tensor"
                         + ("" if n is None else f" of {n}") + " on the cache's GPU")
    return t if t.is_contiguous() else t.contiguous()


def _call(cache, fn, name, *args):
    """fn on the cache's device and current stream."""
    if _current_device() == cache.index:
        rc = fn(cache._ref, *args, _raw_stream(cache.index))
    else:
        with torch.cuda.device(cache.device):
            rc = fn(cache._ref, *args, _raw_stream(cache.index))
    if rc:
        raise KmeansError(name, rc)


def kmeans_kv_write(cache: KVCodes, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor):
    """Encodes the tokens k, v ([n, heads, dim]) into the slots of `slots` (int64
    [n]; page number * page + place). A token whose slot is negative or past
    the cache is left out."""
    if _fast is not None and _current_device() == cache.index:
        rc = _fast.write(cache._at, cache.k_centres, _raw_stream(cache.index), k, v, slots)
        if rc == 0:
            return
        if rc is not None:
            raise KmeansError("kmeans_kv_write", rc)
    slots = _ints(cache, slots, torch.int64, None, "slots")
    n = slots.shape[0]
    k, kp, shape, ka, kb = _rows(cache, k, "k")
    v, vp, v_shape, va, vb = _rows(cache, v, "v")
    if shape[0] != n or shape[1] != cache.heads or v_shape != shape:
        raise ValueError(f"k and v must be [{n}, {cache.heads}, {cache.dim}], as slots and the "
                         "cache are")
    _call(cache, _lib.kmeans_kv_write, "kmeans_kv_write", kp, ka, kb, vp, va, vb,
          slots.data_ptr(), n)


def kmeans_kv_read(cache: KVCodes, slots: torch.Tensor, out=None):
    """The keys and values in the slots of `slots` (int64 [n]), as the centres
    that their codes name: (k, v), each [n, heads, dim]; zeros for a slot that
    is not in the cache. `out` may supply both tensors."""
    if _fast is not None and out is None and _current_device() == cache.index:
        got = _fast.read(cache._at, cache.k_centres, _raw_stream(cache.index), slots)
        if type(got) is tuple:
            return got
        if got is not None:
            raise KmeansError("kmeans_kv_read", got)
    slots = _ints(cache, slots, torch.int64, None, "slots")
    n = slots.shape[0]
    shape = (n, cache.heads, cache.dim)
    k, v = (None, None) if out is None else out
    k, kp, ka, kb = _target(cache, k, shape, "k")
    v, vp, va, vb = _target(cache, v, shape, "v")
    _call(cache, _lib.kmeans_kv_read, "kmeans_kv_read", slots.data_ptr(), n, kp, ka, kb, vp, va,
          vb)
    return k, v


def kmeans_kv_attend(cache: KVCodes, q: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor,
                     scale: float | None = None, starts: torch.Tensor | None = None, out=None,
                     lse=None, ws: torch.Tensor | None = None):
    """Attention of one new token of every sequence over its cached positions.

    q        [seqs, q_heads, dim], q_heads a multiple of the cache's heads
    table    int32 [seqs, pages of a sequence]: page numbers
    lengths  int32 [seqs]: cached positions
    scale    of the scores, 1 / sqrt(dim) if None
    starts   int32 [seqs]: the first attended position, 0 if None

    Returns (out, lse): out like q, lse float32 [seqs, q_heads], the logarithm
    of the sum of the scores' exponentials (-inf, with out 0, where nothing is
    attended). `out` and `lse` may supply the tensors, `ws` the workspace
    (cache.attend_workspace_bytes)."""
    if scale is None:
        scale = 1.0 / math.sqrt(cache.dim)
    if (_fast is not None and out is None and lse is None and ws is None
            and _current_device() == cache.index):
        got = _fast.attend(cache._at, cache.k_centres, _raw_stream(cache.index), q, table, lengths,
                           scale, starts)
        if type(got) is tuple:
            return got
        if got is not None:
            raise KmeansError("kmeans_kv_attend", got)
    q, qp, shape, qa, qb = _rows(cache, q, "q")
    _no_gradient(q, "q")
    seqs, q_heads, dim = shape
    if q_heads < 1 or q_heads % cache.heads:
        raise ValueError(f"q must have a multiple of {cache.heads} heads")
    if not (isinstance(table, torch.Tensor) and table.dtype is torch.int32 and table.dim() == 2
            and table.get_device() == cache.index and table.shape[0] == seqs):
        raise ValueError(f"table must be an int32 [{seqs}, pages] tensor on the cache's GPU")
    row, one = table.stride()
    if one != 1:
        table = table.contiguous()
        row = table.stride(0)
    lengths = _ints(cache, lengths, torch.int32, seqs, "lengths")
    if starts is not None:
        starts = _ints(cache, starts, torch.int32, seqs, "starts")
    if out is None and q.is_contiguous():
        out, oa, ob = torch.empty_like(q), qa, qb
        op = out.data_ptr()
    else:
        out, op, oa, ob = _target(cache, out, shape, "out")
    if lse is None:
        lse = torch.empty((seqs, q_heads), dtype=torch.float32, device=cache.device)
    elif not (lse.dtype is torch.float32 and tuple(lse.shape) == (seqs, q_heads)
              and lse.is_contiguous() and lse.get_device() == cache.index):
        raise ValueError(f"lse must be a contiguous float32 [{seqs}, {q_heads}] tensor on the "
                         "cache's GPU")
    else:
        _no_gradient(lse, "lse")
    width = table.shape[1]
    if width == 0 or seqs == 0:         # no position anywhere
        return out.zero_(), lse.fill_(-math.inf)
    if ws is None:
        nbytes = cache.attend_workspace_bytes(seqs, q_heads, width)
        if nbytes == 0:
            raise KmeansError("kmeans_kv_attend", KMEANS_EUNSUPPORTED)
        ws = torch.empty(nbytes, dtype=torch.uint8, device=cache.device)
    else:
        if ws.get_device() != cache.index or not ws.is_contiguous():
            raise ValueError("ws must be a contiguous tensor on the cache's GPU")
        nbytes = ws.numel() * ws.element_size()
    _call(cache, _lib.kmeans_kv_attend, "kmeans_kv_attend", qp, qa, qb, seqs, q_heads,
          table.data_ptr(), row, width, lengths.data_ptr(),
          None if starts is None else starts.data_ptr(),
          scale, op, oa, ob, lse.data_ptr(), ws.data_ptr(), nbytes)
    return out, lse

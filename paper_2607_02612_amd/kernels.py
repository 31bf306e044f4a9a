"""Python binding of the kernel-level entry points (fusion_test_* in
include/fusion.h): argument marshalling only.  Tensors are passed as device
pointers; the per-sample row offsets and merge counts are host arrays.

Each function runs one step of the pipeline with the library's HIP kernels
on caller-supplied packed ragged buffers and returns device tensors, ordered
on the current stream.  The scratch of a call is a tensor of torch's caching
allocator, so a call neither allocates device memory itself nor waits for the
stream; the caller's tensors are recorded on it, except by gemm.

For long sequences and token caches: window_attention (a sliding window over
packed rows), TokenCache with cache_append, paged_attention (one new token per
sequence, adding up the attention weight of each cached token) and cache_evict
(the tokens with the most weight stay).  TokenCache4 holds a cache in 4 bits,
cache_append_rotary turns queries and keys by their position on their way in,
and block_attention reads the pages that PageBounds and the query choose.  They
compute no gradients.
"""
from __future__ import annotations

import ctypes
import struct
from ctypes import byref, c_double, c_float

import numpy as np
import torch
from torch.autograd import forward_ad

from . import _native
from ._native import FusionCache, FusionPackedOut, FusionRagged, FusionScales, check

EPI = {"store": 0, "gelu": 1, "resid": 2, "f32": 3}


def _ptr(t):
    return None if t is None else t.data_ptr()


def _host_i32(a):
    a = np.ascontiguousarray(np.asarray(a, dtype=np.int32))
    return a, a.ctypes.data_as(ctypes.c_void_p)


def _stream(*used):
    """The current stream, for a call that leaves work on it; `used` are the
    caller's tensors that it uses from now on (they may belong to another
    stream: their memory is not given out again before that work is done)."""
    s = torch.cuda.current_stream()
    for t in used:
        if t is not None:
            t.record_stream(s)
    return s.cuda_stream


def _workspace(B, M, dev):
    """Scratch for one call."""
    n = _native.lib().fusion_test_workspace_bytes(B, M)
    return torch.empty(max(n, 256), dtype=torch.uint8, device=dev), n


def _need(t, name, dtype):
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous {dtype} GPU tensor")


def gemm(A, W, bias, epi, out, rows=None):
    """out <- epi(A W^T + bias).  A [M, K], W [N, K]: both bfloat16 (bf16
    path) or both float32; bias float32 [N]; out in the storage type
    (store / gelu) or float32 (resid / f32).  Like a torch operator with out=
    it leaves record_stream of tensors from another stream to the caller
    (recording the five takes 1.6 us of a call of 9)."""
    prec = {torch.bfloat16: 1, torch.float32: 0}[A.dtype]
    _need(A, "A", A.dtype)
    _need(W, "W", A.dtype)
    _need(bias, "bias", torch.float32)
    _need(out, "out", out.dtype)
    if rows is not None:
        _need(rows, "rows", torch.int32)
    M, K = A.shape
    N = W.shape[0]
    if W.shape[1] != K or bias.shape[0] != N or out.shape[1] < N:
        raise ValueError("operand shapes do not match")
    if rows is None and out.shape[0] < M:
        raise ValueError("out has fewer rows than A")
    check(_native.lib().fusion_test_gemm(prec, A.data_ptr(), K, W.data_ptr(), N, K, M,
                                         bias.data_ptr(), EPI[epi], out.data_ptr(),
                                         out.shape[1], _ptr(rows), _stream()))
    return out


def attention(qkv, size, cu, heads, prop_attn=True, cls_tmax=None):
    """Per-sample MHSA over packed rows; returns (out [M, d] like qkv,
    cls_scores [B, heads, tmax] float32 or None)."""
    prec = {torch.bfloat16: 1, torch.float32: 0}[qkv.dtype]
    _need(qkv, "qkv", qkv.dtype)
    _need(size, "size", torch.float32)
    cu_h, cu_p = _host_i32(cu)
    B = len(cu_h) - 1
    M, d3 = qkv.shape
    if M != cu_h[-1] or size.shape[0] != M:
        raise ValueError("rows do not match the offsets")
    d = d3 // 3
    out = torch.empty(M, d, dtype=qkv.dtype, device=qkv.device)
    cls = None
    if cls_tmax is not None:
        cls = torch.empty((B, heads, cls_tmax), dtype=torch.float32, device=qkv.device)
    ws, n = _workspace(B, M, qkv.device)
    check(_native.lib().fusion_test_attention_ws(prec, qkv.data_ptr(), size.data_ptr(), cu_p, B,
                                                 heads, d, int(bool(prop_attn)), out.data_ptr(),
                                                 _ptr(cls), cls_tmax or 0, ws.data_ptr(), n,
                                                 _stream(qkv, size)))
    return out, cls


def _ragged(x, size, origin, cu):
    _need(x, "x", torch.float32)
    _need(size, "size", torch.float32)
    _need(origin, "origin", torch.int32)
    cu_h, cu_p = _host_i32(cu)
    if x.shape[0] != cu_h[-1] or size.shape[0] != x.shape[0] or origin.shape[0] != x.shape[0]:
        raise ValueError("rows do not match the offsets")
    rg = FusionRagged(x.data_ptr(), size.data_ptr(), origin.data_ptr(), cu_p,
                      len(cu_h) - 1, x.shape[1])
    return rg, cu_h


def _packed(M, B, dev, fill=False):
    """Output buffers; `fill`: for an entry point that leaves the entries past
    the survivors as they are."""
    def buf(n, dtype=torch.int32):
        return torch.full((n,), -1, dtype=dtype, device=dev) if fill else \
            torch.empty((n,), dtype=dtype, device=dev)

    o = dict(rows=buf(M), size=buf(M, torch.float32), origin=buf(M), cu=buf(B + 1), live=buf(B),
             counts=buf(2))
    po = FusionPackedOut(*(o[k].data_ptr() for k in ("rows", "size", "origin", "cu", "live",
                                                     "counts")))
    return o, po


def merge(x, size, origin, cu, r, id_stride, noalloc=False):
    """Bipartite merge of r[i] pairs per sample (x updated in place); returns
    (packed output dict, merge_dst [B, id_stride] int32).  noalloc: the
    variant whose scratch is the library's static device array."""
    rg, cu_h = _ragged(x, size, origin, cu)
    B = len(cu_h) - 1
    r_h, r_p = _host_i32(r)
    if len(r_h) != B:
        raise ValueError("one merge count per sample")
    M, dev = x.shape[0], x.device
    o, po = _packed(M, B, dev, fill=noalloc)
    if noalloc:
        md = torch.full((B, id_stride), -1, dtype=torch.int32, device=dev)
        check(_native.lib().fusion_test_merge_noalloc(byref(rg), r_p, id_stride, md.data_ptr(),
                                                      byref(po), _stream(x, size, origin)))
        return o, md
    md = torch.empty((B, id_stride), dtype=torch.int32, device=dev)
    ws, n = _workspace(B, M, dev)
    check(_native.lib().fusion_test_merge_ws(byref(rg), r_p, id_stride, md.data_ptr(), byref(po),
                                             ws.data_ptr(), n, _stream(x, size, origin)))
    return o, md


def topk_compact(x, size, origin, cu, keep_ratio, scores=None, heads=1, prune_w=None,
                 prune_b=None, exit_logits=None, delta=1.0, ln=None, precision=1):
    """Exit check (optional), top-k prune and re-compaction; returns (packed
    output dict, logits, exit_block, ln_out)."""
    rg, cu_h = _ragged(x, size, origin, cu)
    B, M, d = len(cu_h) - 1, x.shape[0], x.shape[1]
    dev = x.device
    tmax = 0
    if scores is not None:
        _need(scores, "scores", torch.float32)
        if scores.shape[0] != B or scores.shape[1] != heads:
            raise ValueError("scores must be [batch, heads, tmax]")
        tmax = scores.shape[2]
    C = 0
    logits = exit_block = None
    if exit_logits is not None:
        _need(exit_logits, "exit_logits", torch.float32)
        C = exit_logits.shape[1]
        logits = torch.empty((B, C), dtype=torch.float32, device=dev)
        exit_block = torch.empty((B,), dtype=torch.int32, device=dev)
    ln_out = None
    ln_g = ln_b = None
    if ln is not None:
        ln_g, ln_b = ln
        ln_out = torch.empty(M, d, dtype=torch.bfloat16 if precision == 1 else torch.float32,
                             device=dev)
    o, po = _packed(M, B, dev)
    ws, n = _workspace(B, M, dev)
    check(_native.lib().fusion_test_topk_compact_ws(
        byref(rg), _ptr(scores), heads, tmax, _ptr(prune_w), _ptr(prune_b), c_double(keep_ratio),
        _ptr(exit_logits), C, c_float(delta), _ptr(logits), _ptr(exit_block), precision,
        _ptr(ln_g), _ptr(ln_b), _ptr(ln_out), byref(po), ws.data_ptr(), n,
        _stream(x, size, origin, scores, exit_logits, prune_w, prune_b, ln_g, ln_b)))
    return o, logits, exit_block, ln_out


# ------------------------------------------- long sequences, token caches --
# (the host's part of a small call is longer than the kernels': the helpers
# below ask torch for as little as they can)
_PREC = {torch.bfloat16: 1, torch.float32: 0}
_PIECE = {torch.bfloat16: 7, torch.float32: 3}  # strides are multiples of one more
_STREAMS = {}


def _current(dev, *used):
    """Handle of the current stream of GPU `dev`, with `used` recorded on it.
    torch.cuda.current_stream makes an object, which takes 2.6 us; here each
    stream's is made once."""
    raw = torch._C._cuda_getCurrentRawStream(dev)
    s = _STREAMS.get((dev, raw))
    if s is None:
        s = _STREAMS[dev, raw] = torch.cuda.current_stream(dev)
    for t in used:
        if t is not None:
            t.record_stream(s)
    return raw


def _no_grad(t, name):
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} requires a gradient, and none is computed: detach it")
    if forward_ad._current_level >= 0 and forward_ad.unpack_dual(t).tangent is not None:
        raise ValueError(f"{name} carries a tangent, and none is computed: pass its primal")


def _heads(t, name, dtype, heads, dh):
    """Checks a [rows, heads, dh] tensor of any row and head strides in whole
    16-byte pieces; returns its address and the two strides."""
    shape = t.shape if isinstance(t, torch.Tensor) else ()
    if len(shape) != 3 or shape[1] != heads or shape[2] != dh:
        raise ValueError(f"{name} must be a tensor [rows, {heads}, {dh}]")
    if t.dtype is not dtype:
        raise ValueError(f"{name} must be {dtype}")
    _no_grad(t, name)
    row, head, one = t.stride()
    p = t.data_ptr()
    if one != 1 or (row | head) & _PIECE[dtype] or p & 15:
        raise ValueError(f"{name} must have contiguous heads, and strides and a base in whole "
                         "16-byte pieces")
    return p, row, head


def _here(*tensors):
    """The current GPU, whose current stream the call uses; all tensors are on
    it."""
    dev = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"tensors must be on the current GPU (cuda:{dev}), got {t.device}")
    return dev


def _offsets(cu):
    """Host row offsets as int32 and their address (the library checks their
    order)."""
    a = cu if isinstance(cu, np.ndarray) else np.asarray(cu)
    if a.ndim != 1 or len(a) < 2 or a.dtype.kind not in "iu":
        raise ValueError("offsets must be [batch + 1] whole numbers")
    if a.dtype != np.int32:
        if a.min() < 0 or a.max() > 1 << 30:
            raise ValueError("offsets must be in 0 .. 2^30")
        a = a.astype(np.int32)
    if not (a.flags.c_contiguous and a.flags.writeable):
        a = a.copy()
    return a, ctypes.addressof(ctypes.c_char.from_buffer(a))


def _count(v, name, lowest=0, most=1 << 30):
    """A whole number; beyond `most` (rows of a sequence, or the last position
    there is) it makes no difference."""
    if type(v) is int and lowest <= v <= most:
        return v
    try:
        n = int(v)
    except (OverflowError, TypeError, ValueError):  # infinite, no number, NaN
        n = None
    if n is None or n != v or n < lowest:
        raise ValueError(f"{name} must be a whole number, at least {lowest}")
    return min(n, most)


_LAST = (1 << 31) - 1  # position


_Strides2, _Strides4, _Strides6 = (ctypes.c_int64 * n for n in (2, 4, 6))
_rotary_rows = struct.Struct("13q3i4x").pack  # fusion_rotary_rows


def _out(out, rows, heads, dh, like):
    if out is None:
        return like.new_empty((rows, heads, dh))
    _need(out, "out", like.dtype)
    _no_grad(out, "out")
    if tuple(out.shape) != (rows, heads, dh) or out.data_ptr() % 16:
        raise ValueError(f"out must be a 16-byte aligned tensor [{rows}, {heads}, {dh}]")
    _here(out)
    return out


def _span(t):
    """Address of a tensor's first element, and that past its last one."""
    last = sum((n - 1) * s for n, s in zip(t.shape, t.stride())) if t.numel() else -1
    return t.data_ptr(), t.data_ptr() + (last + 1) * t.element_size()


def _clear(first, past, spans):
    """Memory that is written and the spans of other tensors have no byte in common."""
    for a, z in spans:
        if a < past and first < z:
            raise ValueError("tensors that are written must not overlap the others")


def _beside(out, *inputs):
    """A tensor that is written and the span of each other one, from its first
    element to its last, have no memory in common."""
    _clear(*_span(out), map(_span, inputs))


def window_attention(q, k, v, cu, window=None, sinks=0, causal=True, size=None, out=None):
    """Attention of packed rows: row i of a sample sees its rows j <= i with
    i - j < window or j < sinks; with causal=False those with |i - j| < window
    or j < sinks (the first rows are seen by all, but see their own window
    only).  window None: no limit.  q [M, heads, dh], k and v
    [M, kv_heads, dh], bfloat16 or float32, dh a multiple of 8 up to 128, any
    row and head strides in whole 16-byte pieces (views of one product's
    output, say); cu: host offsets [batch + 1] (samples may be empty), rows
    from cu[-1] on take no part; size: float32 [M], scores += ln(size), a size
    of 0 hides the row.  Returns out [M, heads, dh]: rows that see nothing are
    zero, rows from cu[-1] on are left as they were (zero if out is None); a
    given out does not overlap the inputs."""
    if not isinstance(q, torch.Tensor) or q.dim() != 3 or q.dtype not in _PREC:
        raise ValueError("q must be a bfloat16 or float32 tensor [rows, heads, dh]")
    M, heads, dh = q.shape
    kv_heads = k.shape[1] if isinstance(k, torch.Tensor) and k.dim() == 3 else 0
    qp, q_row, q_head = _heads(q, "q", q.dtype, heads, dh)
    kp, k_row, k_head = _heads(k, "k", q.dtype, kv_heads, dh)
    vp, v_row, v_head = _heads(v, "v", q.dtype, kv_heads, dh)
    if k.shape[0] != M or v.shape[0] != M:
        raise ValueError("q, k and v must have the same rows")
    if size is not None:
        _need(size, "size", torch.float32)
        _no_grad(size, "size")
        if tuple(size.shape) != (M,):
            raise ValueError("one size per row")
    dev = _here(q, k, v, size)
    cu_h, cu_p = _offsets(cu)
    if cu_h[-1] > M:
        raise ValueError("offsets must end within the rows")
    window = 0 if window is None else _count(window, "window", 1)
    rows = int(cu_h[-1])
    fresh = out is None
    out = _out(out, M, heads, dh, q)
    if fresh and rows < M:
        out[max(rows, 0):].zero_()
    check(_native.lib().fusion_window_attention(
        _PREC[q.dtype], qp, kp, vp, _Strides6(q_row, q_head, k_row, k_head, v_row, v_head),
        _ptr(size), cu_p, len(cu_h) - 1, heads, kv_heads, dh, window, _count(sinks, "sinks"),
        1 if causal else 0, out.data_ptr(), _current(dev, q, k, v, size, None if fresh else out)))
    return out


def _apart(t, name):
    """The elements of a tensor lie apart from each other."""
    extent = t.shape[3]
    for st, n in sorted(zip(t.stride()[:3], t.shape[:3])):
        if n > 1 and st < extent:
            raise ValueError(f"{name} must not overlap itself")
        extent = st * (n - 1) + extent if n > 1 else extent


class TokenCache:
    """A paged cache of keys and values with the attention weight that each
    cached token has drawn; holds the caller's tensors and their checks.

    k, v [pages, page_size, kv_heads, dh], bfloat16 or float32, contiguous
    heads, other strides free in whole 16-byte pieces; table int32 [batch,
    max_pages], the pages of each sequence (numbers outside the pages: none);
    length, seen int32 [batch]: slots in use, tokens appended so far; weight
    float32 and pos int32 [batch, max_pages * page_size]: attention weight and
    position of the token in each slot.  length = seen = 0 is an empty
    sequence; while they are equal, pos of slot x must be x.  The calls below
    update k, v, length, seen, weight and pos in place, and the caller may
    too, in stream order.  Pages that a call writes must not be shared."""

    # entry points that take the cache, and what follows it in their arguments
    _names = "fusion_paged_attention", "fusion_cache_evict"
    _scales, _more = None, ()

    def __init__(self, k, v, table, length, seen, weight, pos):
        if not isinstance(k, torch.Tensor) or k.dim() != 4 or k.dtype not in _PREC:
            raise ValueError("k must be a bfloat16 or float32 tensor [pages, page_size, "
                             "kv_heads, dh]")
        self._pages(k, v)
        self._take((k, v, table, length, seen, weight, pos), k.dtype, k.shape[3])
        self._bytes(self._names[1], 1)  # the library's checks

    @staticmethod
    def _pages(k, v):
        for t, name in ((k, "k"), (v, "v")):
            if not isinstance(t, torch.Tensor) or t.shape != k.shape or t.dtype != k.dtype:
                raise ValueError("k and v must have the same shape and type")
            if not t.is_cuda:
                raise ValueError(f"{name} must be on a GPU")
            _apart(t, name)
            if t.stride(3) != 1 or t.data_ptr() % 16 or \
                    any(st * t.element_size() % 16 for st in t.stride()[:3]):
                raise ValueError(f"{name} must have contiguous heads, and strides and a base in "
                                 "whole 16-byte pieces")

    def _take(self, tensors, dtype, dh):
        """Checks what every cache has; `tensors`: k, v, table, length, seen,
        weight, pos and the tensors of a kind of cache."""
        k, v, table, length, seen, weight, pos = tensors[:7]
        pages, page_size, kv_heads = k.shape[:3]
        for t, name in ((table, "table"), (length, "length"), (seen, "seen"), (pos, "pos")):
            _need(t, name, torch.int32)
        _need(weight, "weight", torch.float32)
        if table.dim() != 2:
            raise ValueError("table must be [batch, max_pages]")
        batch, max_pages = table.shape
        if tuple(length.shape) != (batch,) or tuple(seen.shape) != (batch,):
            raise ValueError("length and seen must be [batch]")
        if tuple(weight.shape) != (batch, max_pages * page_size) or pos.shape != weight.shape:
            raise ValueError("weight and pos must be [batch, max_pages * page_size]")
        self._tensors = tensors
        if any(t.requires_grad for t in self._tensors):
            raise ValueError("the cache's tensors are written in place and have no gradients")
        for t, name in zip(self._tensors, ("k", "v", "table", "length", "seen", "weight", "pos",
                                           "k_scale", "v_scale")):
            _no_grad(t, name)
        if any(t.device != k.device for t in self._tensors):
            raise ValueError("the cache's tensors must be on one GPU")
        self._c = FusionCache(k.data_ptr(), v.data_ptr(), k.stride()[:3], v.stride()[:3],
                              table.data_ptr(), length.data_ptr(), seen.data_ptr(),
                              weight.data_ptr(), pos.data_ptr(), _PREC[dtype], batch, pages,
                              page_size, max_pages, kv_heads, dh)
        self._ref = byref(self._c)
        self._attend, self._evict = (getattr(_native.lib(), name) for name in self._names)
        self._space, self._streams = {}, set()
        self._spans = [_span(t) for t in tensors]
        self.batch, self.kv_heads, self.dh, self.dtype = batch, kv_heads, dh, dtype
        self.capacity, self.device = max_pages * page_size, k.device
        self._index = k.get_device()

    @classmethod
    def empty(cls, batch, capacity, kv_heads, dh, page_size=64, dtype=torch.bfloat16):
        """An empty cache on the current GPU with pages for `capacity` tokens
        of every sequence."""
        n = -(-capacity // page_size)
        dev = torch.device("cuda", torch.cuda.current_device())
        kv = [torch.empty((batch * n, page_size, kv_heads, dh), dtype=dtype, device=dev)
              for _ in range(2)]
        i32 = [torch.zeros(shape, dtype=torch.int32, device=dev)
               for shape in ((batch,), (batch,), (batch, n * page_size))]
        return cls(*kv, torch.arange(batch * n, dtype=torch.int32, device=dev).view(batch, n),
                   i32[0], i32[1],
                   torch.zeros((batch, n * page_size), dtype=torch.float32, device=dev), i32[2])

    k, v, table, length, seen, weight, pos = (
        property(lambda self, i=i: self._tensors[i]) for i in range(7))

    def _bytes(self, entry, *args):
        """Workspace of a call, asked once."""
        key = (entry, *args)
        if key not in self._space:
            n = getattr(_native.lib(), entry + "_workspace_bytes")(self._ref, *self._more, *args)
            if n == 0:
                check(-1)
            self._space[key] = n
        return self._space[key]

    def _ready(self, *used):
        """Handle of the current stream, with the caller's tensors recorded on
        it; the cache's own are recorded on each stream once, which holds
        until they are freed."""
        if torch.cuda.current_device() != self._index:
            raise ValueError(f"the cache is on {self.device}, not on the current GPU")
        raw = _current(self._index, *used)
        if raw not in self._streams:
            _current(self._index, *self._tensors)
            self._streams.add(raw)
        return raw

    def _workspace(self, entry, *args):
        n = self._bytes(entry, *args)
        return torch.empty(n, dtype=torch.uint8, device=self.device), n


class TokenCache4(TokenCache):
    """A TokenCache that holds its keys and values in 4 bits: e2m1 numbers (0,
    1/2, 1, 3/2, 2, 3, 4, 6 and a sign) times a power of two for each 32 dims of a
    head, 4.25 bits a value.

    k, v uint8 [pages, page_size, kv_heads, dh / 2], two codes a byte, the lower
    dim in the lower half, dh a multiple of 32 up to 128; k_scale, v_scale uint8
    [pages, page_size, kv_heads, dh / 32], s in 2 .. 252 for a scale of
    2^(s - 127), 255: the block is NaN; strides as in a TokenCache, those of the
    scales in whole bytes.
    Attention sums in fp32 with weights of up to 2^8: values of n visible tokens are
    within its range up to s = 244 - log2(n) (magnitudes of 2^120 / n), larger ones may
    give infinity or NaN.
    dtype: of the rows that come in, of queries and of outputs.  cache_append,
    cache_append_rotary, paged_attention, cache_evict, PageBounds and
    block_attention take it as they take a TokenCache; rows are rounded to 4
    bits when they are appended."""
    _names = "fusion_cache4_attention", "fusion_cache4_evict"

    def __init__(self, k, v, k_scale, v_scale, table, length, seen, weight, pos,
                 dtype=torch.bfloat16):
        if dtype not in _PREC:
            raise ValueError("rows must be bfloat16 or float32")
        if not isinstance(k, torch.Tensor) or k.dim() != 4 or k.dtype != torch.uint8 or k.shape[3] % 16:
            raise ValueError("k must be a uint8 tensor [pages, page_size, kv_heads, dh / 2], dh a "
                             "multiple of 32")
        self._pages(k, v)
        for t, name in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            if not isinstance(t, torch.Tensor) or t.dtype != torch.uint8 or \
                    tuple(t.shape) != (*k.shape[:3], k.shape[3] // 16):
                raise ValueError(f"{name} must be a uint8 tensor [pages, page_size, kv_heads, dh / 32]")
            if t.shape[3] > 1 and t.stride(3) != 1:
                raise ValueError(f"{name} must have contiguous heads")
            _apart(t, name)
        self._take((k, v, table, length, seen, weight, pos, k_scale, v_scale), dtype, 2 * k.shape[3])
        self._s = FusionScales(k_scale.data_ptr(), v_scale.data_ptr(), k_scale.stride()[:3],
                               v_scale.stride()[:3])
        self._scales = byref(self._s)
        self._more = (self._scales,)
        self._bytes(self._names[1], 1)  # the library's checks

    @classmethod
    def empty(cls, batch, capacity, kv_heads, dh, page_size=64, dtype=torch.bfloat16):
        """An empty cache on the current GPU with pages for `capacity` tokens of
        every sequence.  In memory the heads of a page come before its tokens, so
        that what a key head reads of a page lies together."""
        if dh < 32 or dh % 32:
            raise ValueError("dh must be a multiple of 32")
        n = -(-capacity // page_size)
        dev = torch.device("cuda", torch.cuda.current_device())
        u8 = [torch.zeros((batch * n, kv_heads, page_size, w), dtype=torch.uint8,
                          device=dev).transpose(1, 2) for w in (dh // 2, dh // 2, dh // 32, dh // 32)]
        i32 = [torch.zeros(shape, dtype=torch.int32, device=dev)
               for shape in ((batch,), (batch,), (batch, n * page_size))]
        return cls(*u8, torch.arange(batch * n, dtype=torch.int32, device=dev).view(batch, n),
                   i32[0], i32[1],
                   torch.zeros((batch, n * page_size), dtype=torch.float32, device=dev), i32[2],
                   dtype=dtype)

    k_scale, v_scale = (property(lambda self, i=i: self._tensors[i]) for i in (7, 8))


def cache_append(cache, k, v, cu=None):
    """Append key and value rows [rows, kv_heads, dh]: one per sequence, or
    rows cu[i] .. cu[i+1]-1 to sequence i (cu: host offsets, rows from cu[-1]
    on take no part; no row lies in a slot that the call writes).  Their weight
    starts at 0, that of a prompt's rows too; rows past a sequence's capacity are
    dropped."""
    kp, k_row, k_head = _heads(k, "k", cache.dtype, cache.kv_heads, cache.dh)
    vp, v_row, v_head = _heads(v, "v", cache.dtype, cache.kv_heads, cache.dh)
    _here(k, v)
    cu_p = None
    if cu is not None:
        cu_h, cu_p = _offsets(cu)
        if len(cu_h) != cache.batch + 1:
            raise ValueError("offsets must be [batch + 1]")
    rows = k.shape[0]
    if v.shape[0] != rows or (rows != cache.batch if cu is None else rows < cu_h[-1]):
        raise ValueError("rows do not match the sequences")
    if cache._scales is not None:
        r = _rotary_rows(0, kp, vp, 0, 0, k_row, k_head, v_row, v_head, 0, 0, 0, 0, 0, 0, 0)
        check(_native.lib().fusion_cache_append_rotary(cache._ref, cache._scales, r, cu_p,
                                                       cache._ready(k, v)))
        return
    check(_native.lib().fusion_cache_append(cache._ref, kp, vp,
                                            _Strides4(k_row, k_head, v_row, v_head), cu_p,
                                            cache._ready(k, v)))


def paged_attention(q, cache, window=None, sinks=0, accumulate=True, out=None):
    """Attention of each sequence's newest token (appended before; of several
    rows appended at once the last one) over its cached tokens; with a window,
    over those among the last `window` positions or the first `sinks`.
    q [batch, heads, dh]; returns out like q, contiguous (a given out does not
    overlap the inputs).  accumulate: cache.weight grows by the mean over the
    heads of the attention probabilities."""
    if not isinstance(q, torch.Tensor) or q.dim() != 3 or q.shape[0] != cache.batch:
        raise ValueError("q must be a tensor [batch, heads, dh]")
    heads = q.shape[1]
    qp, q_row, q_head = _heads(q, "q", cache.dtype, heads, cache.dh)
    window = 0 if window is None else _count(window, "window", 1, _LAST)
    _here(q)
    fresh = out is None
    out = _out(out, cache.batch, heads, cache.dh, q)
    acc = 1 if accumulate else 0
    stream = cache._ready(q, None if fresh else out)
    ws, n = cache._workspace(cache._names[0], heads, acc)
    check(cache._attend(
        cache._ref, *cache._more, qp, _Strides2(q_row, q_head), heads, window,
        _count(sinks, "sinks", 0, _LAST), acc,
        out.data_ptr(), ws.data_ptr(), n, stream))
    return out


def cache_evict(cache, budget, sinks=0, recent=0):
    """Bring every sequence down to `budget` tokens: the first `sinks` and
    last `recent` positions stay, and the others by accumulated weight, equal
    ones by the lower slot (tokens that have drawn nothing yet, such as a
    prompt's before the first steps, are equal).  A token past the budget
    that no page holds leaves first.  Returns src int32 [batch, budget]: the
    slot from which each slot's token came, -1 past the sequence's length."""
    budget, sinks = _count(budget, "budget", 1, _LAST), _count(sinks, "sinks", 0, _LAST)
    recent = _count(recent, "recent", 0, _LAST)
    if budget > 1 << 30:
        raise ValueError("budget must be at most 2^30")
    if sinks + recent > budget:
        raise ValueError("sinks and recent do not fit the budget")
    stream = cache._ready()
    ws, n = cache._workspace(cache._names[1], budget)
    src = cache.table.new_empty((cache.batch, budget))
    check(cache._evict(cache._ref, *cache._more, budget, sinks, recent, src.data_ptr(),
                       ws.data_ptr(), n, stream))
    return src


def cache_append_rotary(cache, q, k, v, freq, cu=None, interleaved=False, drop=None, rotated_k=False,
                        out=None):
    """cache_append of rows whose queries q [rows, heads, dh] and keys are turned
    by their position on the way.  freq: float32 [n] on the GPU, radians per
    position, n a multiple of 4 with 2 n <= dh (none: nothing turns): at position
    p dims j and j + n (interleaved: 2j and 2j + 1) turn by the angle p freq[j], a
    product in 64 bits; dims from 2 n on stay.  drop: int32 [batch] on the GPU or
    None; so many of each sequence's newest tokens leave before, such as drafted
    ones that were not kept (they lie in its last slots unless an eviction has
    moved them).  Returns (turned queries, turned keys): both contiguous, rows
    from cu[-1] on zero; the keys, as window_attention takes them, only with
    `rotated_k`, else None; a given out takes the queries, lies apart from the
    inputs and the cache's tensors, and its rows from cu[-1] on are left as they
    were.  No input overlaps what the call writes of the cache (drop may be its
    length or seen).

    Queries come back for all rows, but attention over the cache is that of one
    query a sequence, its newest token's (paged_attention, block_attention), and
    window_attention reads packed rows: drafts, or a later part of a prompt, all
    attend what the cache holds only if they are appended one at a time."""
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q must be a tensor [rows, heads, dh]")
    rows, heads = q.shape[:2]
    dh = cache.dh
    qp, q_row, q_head = _heads(q, "q", cache.dtype, heads, dh)
    kp, k_row, k_head = _heads(k, "k", cache.dtype, cache.kv_heads, dh)
    vp, v_row, v_head = _heads(v, "v", cache.dtype, cache.kv_heads, dh)
    _need(freq, "freq", torch.float32)
    _no_grad(freq, "freq")
    half = freq.shape[0] if freq.dim() == 1 else -1
    if half < 0 or half % 4 or 2 * half > dh:
        raise ValueError("freq must hold a multiple of 4 frequencies, for no more dims than a head has")
    if drop is not None:
        _need(drop, "drop", torch.int32)
        if tuple(drop.shape) != (cache.batch,):
            raise ValueError("drop must be [batch]")
    _here(q, k, v, freq, drop)
    cu_p, used = None, rows
    if cu is not None:
        cu_h, cu_p = _offsets(cu)
        if len(cu_h) != cache.batch + 1:
            raise ValueError("offsets must be [batch + 1]")
        used = int(cu_h[-1])
    if k.shape[0] != rows or v.shape[0] != rows or (rows != cache.batch if cu is None else rows < used):
        raise ValueError("rows do not match the sequences")
    fresh = out is None
    out = _out(out, rows, heads, dh, q)
    if not fresh:
        _beside(out, q, k, v, freq, *(() if drop is None else (drop,)))
        _clear(*_span(out), cache._spans)
    keys = k.new_empty((rows, cache.kv_heads, dh)) if rotated_k else None
    if used < rows:
        for t in (out if fresh else None, keys):
            if t is not None:
                t[max(used, 0):].zero_()
    r = _rotary_rows(qp, kp, vp, q_row, q_head, k_row, k_head, v_row, v_head, out.data_ptr(),
                     0 if keys is None else keys.data_ptr(), freq.data_ptr(),
                     0 if drop is None else drop.data_ptr(), heads, half, 1 if interleaved else 0)
    check(_native.lib().fusion_cache_append_rotary(
        cache._ref, cache._scales, r, cu_p,
        cache._ready(q, k, v, freq, drop, None if fresh else out)))
    return out, keys


class PageBounds:
    """The least and the greatest value of each dim of the keys of every page of
    a cache, by which block_attention chooses pages: lo, hi [pages, kv_heads, dh]
    of the cache's dtype.  Made for what the cache holds, or from given tensors
    as they are, apart from each other and from the cache's.  update() brings
    them up to date: after the cache has changed and before block_attention.  A
    page that sequences share is bounded by what one of them holds of it, so each
    should hold all of it."""

    def __init__(self, cache, lo=None, hi=None):
        shape = (cache.k.shape[0], cache.kv_heads, cache.dh)
        self.cache, given = cache, lo is not None or hi is not None
        if not given:
            lo, hi = (torch.zeros(shape, dtype=cache.dtype, device=cache.device) for _ in range(2))
        for t, name in ((lo, "lo"), (hi, "hi")):
            _need(t, name, cache.dtype)
            _no_grad(t, name)
            if t.requires_grad:
                raise ValueError("bounds are written in place and have no gradients")
            if tuple(t.shape) != shape or t.device != cache.device or t.data_ptr() % 16:
                raise ValueError(f"{name} must be a 16-byte aligned tensor {list(shape)} on the cache's GPU")
        _beside(lo, hi)
        for t in (lo, hi):
            _clear(*_span(t), cache._spans)
        self.lo, self.hi, self._streams = lo, hi, set()
        if not given:
            self.update()

    def _ready(self, *used):
        raw = self.cache._ready(*used)
        if raw not in self._streams:
            _current(self.cache._index, self.lo, self.hi)
            self._streams.add(raw)
        return raw

    def update(self, new=None):
        """Bounds of the pages that hold the newest `new` slots of each sequence,
        at least as many as rows were appended since (None: of all its pages, as
        after an eviction)."""
        new = 0 if new is None else _count(new, "new", 1)
        c = self.cache
        check(_native.lib().fusion_page_bounds(c._ref, c._scales, self.lo.data_ptr(), self.hi.data_ptr(),
                                               new, self._ready()))


def block_attention(q, cache, bounds, blocks, first=0, recent=1, out=None):
    """paged_attention of each sequence's newest token over `blocks` pages that
    each key head chooses: the sequence's `first` and `recent` ones, and of the
    others those whose keys can score highest by their bounds with one of the key
    head's queries (equal ones: the lower page).  Sequences of no more pages
    are attended whole.  Weights stay as they are.  bounds: PageBounds of the
    cache, up to date.  Returns (out like q, contiguous, a given one apart from
    q, the bounds and the cache's tensors; chosen int32 [batch, kv_heads, blocks],
    the pages by their place in the sequence, ascending, then -1)."""
    if not isinstance(q, torch.Tensor) or q.dim() != 3 or q.shape[0] != cache.batch:
        raise ValueError("q must be a tensor [batch, heads, dh]")
    heads = q.shape[1]
    qp, q_row, q_head = _heads(q, "q", cache.dtype, heads, cache.dh)
    if not isinstance(bounds, PageBounds) or bounds.cache is not cache:
        raise ValueError("bounds must be the PageBounds of the cache")
    blocks, first = _count(blocks, "blocks", 1, _LAST), _count(first, "first", 0, _LAST)
    recent = _count(recent, "recent", 1, _LAST)
    if blocks > 1 << 30:
        raise ValueError("blocks must be at most 2^30")
    if first + recent > blocks:
        raise ValueError("first and recent do not fit the blocks")
    _here(q)
    fresh = out is None
    out = _out(out, cache.batch, heads, cache.dh, q)
    if not fresh:
        _beside(out, q, bounds.lo, bounds.hi)
        _clear(*_span(out), cache._spans)
    stream = bounds._ready(q, None if fresh else out)
    key = ("fusion_block_attention", heads, blocks)
    n = cache._space.get(key)
    if n is None:
        n = _native.lib().fusion_block_attention_workspace_bytes(cache._ref, cache._scales, heads, blocks)
        if n == 0:
            check(-1)
        cache._space[key] = n
    ws = torch.empty(n, dtype=torch.uint8, device=cache.device)
    chosen = cache.table.new_empty((cache.batch, cache.kv_heads, blocks))
    check(_native.lib().fusion_block_attention(
        cache._ref, cache._scales, bounds.lo.data_ptr(), bounds.hi.data_ptr(), qp,
        _Strides2(q_row, q_head), heads, blocks, first, recent, out.data_ptr(), chosen.data_ptr(),
        ws.data_ptr(), n, stream))
    return out, chosen

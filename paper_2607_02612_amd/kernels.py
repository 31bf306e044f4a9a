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
(the tokens with the most weight stay).  They compute no gradients.
"""
from __future__ import annotations

import ctypes
from ctypes import byref, c_double, c_float

import numpy as np
import torch
from torch.autograd import forward_ad

from . import _native
from ._native import FusionCache, FusionPackedOut, FusionRagged, check

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


def _out(out, rows, heads, dh, like):
    if out is None:
        return like.new_empty((rows, heads, dh))
    _need(out, "out", like.dtype)
    _no_grad(out, "out")
    if tuple(out.shape) != (rows, heads, dh) or out.data_ptr() % 16:
        raise ValueError(f"out must be a 16-byte aligned tensor [{rows}, {heads}, {dh}]")
    _here(out)
    return out


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

    def __init__(self, k, v, table, length, seen, weight, pos):
        if not isinstance(k, torch.Tensor) or k.dim() != 4 or k.dtype not in _PREC:
            raise ValueError("k must be a bfloat16 or float32 tensor [pages, page_size, "
                             "kv_heads, dh]")
        for t, name in ((k, "k"), (v, "v")):
            if not isinstance(t, torch.Tensor) or t.shape != k.shape or t.dtype != k.dtype:
                raise ValueError("k and v must have the same shape and type")
            if not t.is_cuda:
                raise ValueError(f"{name} must be on a GPU")
            extent = t.shape[3]
            for st, n in sorted(zip(t.stride()[:3], t.shape[:3])):
                if n > 1 and st < extent:
                    raise ValueError(f"{name} must not overlap itself")
                extent = st * (n - 1) + extent if n > 1 else extent
            if t.stride(3) != 1 or t.data_ptr() % 16 or \
                    any(st * t.element_size() % 16 for st in t.stride()[:3]):
                raise ValueError(f"{name} must have contiguous heads, and strides and a base in "
                                 "whole 16-byte pieces")
        pages, page_size, kv_heads, dh = k.shape
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
        self._tensors = (k, v, table, length, seen, weight, pos)
        if any(t.requires_grad for t in self._tensors):
            raise ValueError("the cache's tensors are written in place and have no gradients")
        for t, name in zip(self._tensors, ("k", "v", "table", "length", "seen", "weight", "pos")):
            _no_grad(t, name)
        if any(t.device != k.device for t in self._tensors):
            raise ValueError("the cache's tensors must be on one GPU")
        self._c = FusionCache(k.data_ptr(), v.data_ptr(), k.stride()[:3], v.stride()[:3],
                              table.data_ptr(), length.data_ptr(), seen.data_ptr(),
                              weight.data_ptr(), pos.data_ptr(), _PREC[k.dtype], batch, pages,
                              page_size, max_pages, kv_heads, dh)
        self._ref = byref(self._c)
        self._space, self._streams = {}, set()
        self.batch, self.kv_heads, self.dh, self.dtype = batch, kv_heads, dh, k.dtype
        self.capacity, self.device = max_pages * page_size, k.device
        self._index = k.get_device()
        self._bytes("fusion_cache_evict_workspace_bytes", 1)  # the library's checks

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
            n = getattr(_native.lib(), entry)(self._ref, *args)
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


def cache_append(cache, k, v, cu=None):
    """Append key and value rows [rows, kv_heads, dh]: one per sequence, or
    rows cu[i] .. cu[i+1]-1 to sequence i (cu: host offsets, rows from cu[-1]
    on take no part).  Their weight starts at 0, that of a prompt's rows too;
    rows past a sequence's capacity are dropped."""
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
    check(_native.lib().fusion_cache_append(cache._ref, kp, vp,
                                            _Strides4(k_row, k_head, v_row, v_head), cu_p,
                                            cache._ready(k, v)))


def paged_attention(q, cache, window=None, sinks=0, accumulate=True, out=None):
    """Attention of each sequence's newest token (appended before) over its
    cached tokens; with a window, over those among the last `window` positions
    or the first `sinks`.  q [batch, heads, dh]; returns out like q,
    contiguous (a given out does not overlap the inputs).  accumulate:
    cache.weight grows by the mean over the heads of the attention
    probabilities."""
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
    ws, n = cache._workspace("fusion_paged_attention_workspace_bytes", heads, acc)
    check(_native.lib().fusion_paged_attention(
        cache._ref, qp, _Strides2(q_row, q_head), heads, window,
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
    ws, n = cache._workspace("fusion_cache_evict_workspace_bytes", budget)
    src = cache.table.new_empty((cache.batch, budget))
    check(_native.lib().fusion_cache_evict(cache._ref, budget, sinks, recent, src.data_ptr(),
                                           ws.data_ptr(), n, stream))
    return src

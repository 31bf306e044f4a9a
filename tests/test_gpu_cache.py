"""Windowed attention and token caches (kernels.window_attention, TokenCache,
cache_append, paged_attention, cache_evict) against plain NumPy in 64 bits.

Tolerances.  u = eps / 2 of a type is the most a rounding changes a value
relative to it (bf16 2^-8, fp32 2^-24).  A score is a sum of dh products, so
its fp32 error is at most ds = (dh + 8) 2^-24 scale sum |q||k| + 8 2^-24 |s|
(the last part: the factors and the added logarithm); a probability's relative
error is then 2 ds (its own and the sum's) + (n + 16) 2^-24 (n additions, the
exponential, the division), and on the bf16 path one rounding, 2^-8, before it
multiplies V.  With A = sum p |v| the output is off by at most
  u |out| + (u_p + 2 ds + (n + 16) 2^-24) A,   u_p = 2^-8 (bf16) or 0 (fp32).
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24
UNIT = {"bf16": 2.0 ** -8, "fp32": U32}


@pytest.fixture(scope="module")
def torch_cuda():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _kern():
    from paper_2607_02612_amd import kernels
    return kernels


def _dt(torch, dtype):
    return {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]


def _np(t):
    return t.detach().double().cpu().numpy()


def _normal(torch, rng, dtype, *shape):
    a = torch.from_numpy(rng.standard_normal(shape).astype(np.float32))
    return a.cuda().to(_dt(torch, dtype))


def _attend(q, k, v, see, extra, dtype):
    """One head in 64 bits: (out, probabilities, bound of |out error|, bound
    of the probabilities' relative error).  q [T, dh], k, v [S, dh], see
    [T, S]; values of unseen keys are not touched."""
    dh, scale = q.shape[1], 1 / math.sqrt(q.shape[1])
    kz = np.where(see.any(0)[:, None], k, 0.0)
    vz = np.where(see.any(0)[:, None], v, 0.0)
    s = q @ kz.T * scale + extra
    ds = (dh + 8) * U32 * scale * (np.abs(q) @ np.abs(kz).T) + \
        8 * U32 * np.where(see & np.isfinite(s), np.abs(s), 0)
    s = np.where(see, s, -np.inf)
    top = s.max(1, keepdims=True, initial=-np.inf)
    e = np.exp(s - np.where(np.isfinite(top), top, 0))
    l = e.sum(1, keepdims=True)
    p = np.divide(e, l, out=np.zeros_like(e), where=l > 0)
    rel = 2 * np.where(see, ds, 0).max(1, initial=0.0) + (see.sum(1) + 16) * U32
    out = p @ vz
    up = UNIT["bf16"] if dtype == "bf16" else 0.0
    tol = UNIT[dtype] * np.abs(out) + (up + rel)[:, None] * (p @ np.abs(vz))
    return out, p, tol, rel


def _window_ref(q, k, v, cu, window, sinks, causal, size, dtype):
    out = np.zeros(q.shape)
    tol = np.zeros(q.shape)
    g = q.shape[1] // k.shape[1]
    for a, b in zip(cu[:-1], cu[1:]):
        i, j = np.arange(b - a)[:, None], np.arange(b - a)[None]
        near = np.abs(i - j) < window if window else np.ones((b - a, b - a), bool)
        see = near | (j < sinks)
        if causal:
            see &= j <= i
        extra = np.zeros(b - a)
        if size is not None:
            see = see & (size[a:b] > 0)[None]
            extra = np.log(np.where(size[a:b] > 0, size[a:b], 1))
        for h in range(q.shape[1]):
            o, _, t, _ = _attend(q[a:b, h], k[a:b, h // g], v[a:b, h // g], see, extra, dtype)
            out[a:b, h], tol[a:b, h] = o, t
    return out, tol


def _close(got, ref, tol, what=""):
    assert np.isfinite(got).all(), what
    worst = float((np.abs(got - ref) - tol).max(initial=-1.0))
    assert worst <= 0, (what, worst, float(np.abs(got - ref).max()))


# --------------------------------------------------------- window_attention --
WINDOW = [  # lengths, heads, kv_heads, dh, window, sinks, causal, sizes
    ([1], 1, 1, 8, None, 0, True, False),
    ([197], 6, 6, 64, 49, 1, False, False),
    ([577, 1, 290], 3, 3, 64, 97, 1, False, True),
    ([0, 5, 0, 0, 130, 1, 0], 4, 2, 64, 3, 2, True, False),
    ([63, 64, 65, 128, 129, 2], 4, 1, 128, 64, 0, True, False),
    ([31, 32, 33, 300], 5, 1, 80, 1, 0, True, False),
    ([257, 16, 15, 17], 2, 2, 24, 1, 5, False, True),
    ([700], 8, 2, 128, 100, 200, True, False),
    ([511, 90], 6, 3, 96, None, 0, False, True),
    ([1030, 3], 2, 1, 128, None, 0, True, False),
    ([400, 20], 20, 1, 64, 1000, 3, True, True),
    ([333], 3, 1, 128, 65, 70, False, False),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", range(len(WINDOW)))
def test_window_attention(torch_cuda, case, dtype):
    torch = torch_cuda
    lengths, hq, hkv, dh, window, sinks, causal, sizes = WINDOW[case]
    print(f"[window] {dtype} {WINDOW[case]}", flush=True)
    rng = np.random.default_rng(case)
    cu = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    M = int(cu[-1])
    qkv = _normal(torch, rng, dtype, M, hq + 2 * hkv, dh)  # views of one buffer
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    size = None
    if sizes:  # some tokens hidden, of the last sample all
        size = rng.integers(0, 5, size=M).astype(np.float32)
        size[cu[-2]:] = 0
    dsize = None if size is None else torch.from_numpy(size).cuda()
    got = _kern().window_attention(q, k, v, cu, window, sinks, causal, dsize)
    assert got.dtype == q.dtype and got.shape == q.shape and got.is_contiguous()
    ref, tol = _window_ref(_np(q), _np(k), _np(v), cu, window, sinks, causal, size, dtype)
    _close(_np(got), ref, tol)
    if sizes:
        assert not got[int(cu[-2]):].any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_window_attention_large_scores(torch_cuda, dtype):
    """Scores of several hundred, of either sign, overflow without the maximum."""
    torch = torch_cuda
    rng = np.random.default_rng(3)
    q, k, v = (_normal(torch, rng, dtype, 150, 2, 64) for _ in range(3))
    q, k = q * 16, k * 16
    k[:, 1] -= 40 * torch.sign(q[:1, 1])
    cu = np.array([0, 70, 150], np.int32)
    got = _kern().window_attention(q, k, v, cu, 40, 2)
    ref, tol = _window_ref(_np(q), _np(k), _np(v), cu, 40, 2, True, None, dtype)
    _close(_np(got), ref, tol)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dh", [64, 128])
def test_window_attention_unseen_values_have_no_influence(torch_cuda, dtype, causal, dh):
    """Infinities and NaN in rows that a query does not see leave its output
    bit for bit; so do other samples and hidden rows."""
    torch = torch_cuda
    rng = np.random.default_rng(4)
    cu = np.array([0, 200, 330], np.int32)
    q, k, v = (_normal(torch, rng, dtype, 330, 2, dh) for _ in range(3))
    size = torch.ones(330, device="cuda")
    size[250] = 0
    window, sinks = 20, 3
    kern = _kern()
    want = kern.window_attention(q, k, v, cu, window, sinks, causal, size)
    i = np.arange(330)
    for bad in (5, 77, 130, 250):
        for value in (float("nan"), float("inf"), -float("inf")):
            kb, vb = k.clone(), v.clone()
            kb[bad], vb[bad] = value, value
            vb[bad, :, ::3] = -value
            got = kern.window_attention(q, kb, vb, cu, window, sinks, causal, size)
            same = (i >= 200) != (bad >= 200)
            near = (i - bad < window) & (i >= bad) if causal else np.abs(i - bad) < window
            clean = torch.from_numpy(same | ~near | (bad == 250)).cuda()
            assert torch.equal(got[clean], want[clean]), (bad, value)


def test_window_attention_strides_out_and_padding(torch_cuda):
    """Heads-first layouts, a given out, rows behind the last sample."""
    torch = torch_cuda
    rng = np.random.default_rng(5)
    cu = np.array([0, 50, 120], np.int32)
    base = [_normal(torch, rng, "bf16", h, 140, 64) for h in (4, 2, 2)]
    q, k, v = (t.transpose(0, 1) for t in base)
    kern = _kern()
    want = kern.window_attention(q[:120].contiguous(), k[:120].contiguous(),
                                 v[:120].contiguous(), cu, 33, 1)
    out = torch.full((140, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    got = kern.window_attention(q, k, v, cu, 33, 1, out=out)
    assert got is out and torch.equal(out[:120], want) and bool((out[120:] == 7).all())
    got = kern.window_attention(q, k, v, cu, 33, 1)
    assert torch.equal(got[:120], want) and not got[120:].any()
    one = kern.window_attention(q, k[:, :1].expand(-1, 4, -1), v[:, :1].expand(-1, 4, -1), cu, 33, 1)
    ref = kern.window_attention(q, k[:, :1], v[:, :1], cu, 33, 1)
    assert torch.equal(one, ref)
    assert kern.window_attention(q[:0], k[:0], v[:0], [0, 0, 0]).shape == (0, 4, 64)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_window_attention_ends_within_tiles(torch_cuda, dtype, dh, causal):
    """Windows and first rows that end at, before and after halves of tiles."""
    torch = torch_cuda
    rng = np.random.default_rng(dh + causal)
    cu = np.array([0, 197, 230])
    q, k, v = (_normal(torch, rng, dtype, 230, 1, dh) for _ in range(3))
    for window in (2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 95, 96, 97, 128, 129):
        for sinks in (0, 1, 16, 33):
            got = _kern().window_attention(q, k, v, cu, window, sinks, causal)
            ref, tol = _window_ref(_np(q), _np(k), _np(v), cu, window, sinks, causal, None, dtype)
            _close(_np(got), ref, tol, (window, sinks))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dh", [64, 72, 128])
@pytest.mark.parametrize("rows", [130, 2000])
def test_window_attention_few_and_many_row_tiles(torch_cuda, dtype, dh, rows):
    """Calls whose waves share the keys of a row tile, and calls of many row
    tiles, with infinities and NaN in rows that are not seen."""
    torch = torch_cuda
    rng = np.random.default_rng(rows + dh)
    q, k, v = (_normal(torch, rng, dtype, rows + 61, 9, dh) for _ in range(3))
    cu = [0, rows, rows + 61]
    v[rows + 20] = float("nan")
    v[rows + 21] = float("-inf")
    k[rows + 20:rows + 22] = float("inf")
    size = torch.ones(rows + 61, device="cuda")
    size[rows + 20:rows + 22] = 0
    for heads, causal in ((1, True), (9, False)):
        got = _kern().window_attention(q[:, :heads], k[:, :heads], v[:, :heads], cu, 70, 3, causal, size)
        kz, vz = _np(k[:, :heads]), _np(v[:, :heads])
        kz[~np.isfinite(kz)] = 0
        vz[~np.isfinite(vz)] = 0
        ref, tol = _window_ref(_np(q[:, :heads]), kz, vz, cu, 70, 3, causal, _np(size), dtype)
        _close(_np(got), ref, tol)


@pytest.mark.parametrize("B", [127, 128, 129, 256, 448, 1000])
def test_window_attention_many_samples(torch_cuda, B):
    """More samples than one launch describes."""
    torch = torch_cuda
    rng = np.random.default_rng(B)
    cu = np.concatenate([[0], np.cumsum(rng.integers(0, 9, size=B))]).astype(np.int32)
    q, k, v = (_normal(torch, rng, "bf16", int(cu[-1]), 2, 64) for _ in range(3))
    got = _kern().window_attention(q, k, v, cu, 4, 1)
    ref, tol = _window_ref(_np(q), _np(k), _np(v), cu, 4, 1, True, None, "bf16")
    _close(_np(got), ref, tol)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_window_attention_offsets_past_32_bits(torch_cuda, dtype):
    """Rows so far apart that element offsets pass 2^31."""
    torch = torch_cuda
    rng = np.random.default_rng(6)
    n, gap = 600, 1 << 22  # 600 rows of 2^22 elements: 2.5e9
    big = torch.empty(n * gap, dtype=_dt(torch, dtype), device="cuda")
    qkv = [_normal(torch, rng, dtype, n, 2, 64) for _ in range(3)]
    far = []
    for x, t in enumerate(qkv):
        view = big.as_strided((n, 2, 64), (gap, 64, 1), 1024 * x)
        view.copy_(t)
        far.append(view)
    cu = [0, 1, n]
    kern = _kern()
    assert torch.equal(kern.window_attention(*far, cu, 100, 2), kern.window_attention(*qkv, cu, 100, 2))


# ------------------------------------------------------------------ caches --
def _cache(torch, rng, dtype, lengths, hkv, dh, page, cap, evicted=False, heads_first=False,
           seen=None):
    """A cache with shuffled pages and random contents."""
    B, n = len(lengths), -(-cap // page)
    pages = B * n + 2
    if heads_first:
        k, v = (_normal(torch, rng, dtype, pages, hkv, page, dh).transpose(1, 2) for _ in range(2))
    else:
        k, v = (_normal(torch, rng, dtype, pages, page, hkv, dh) for _ in range(2))
    table = torch.from_numpy(rng.permutation(pages)[:B * n].reshape(B, n).astype(np.int32)).cuda()
    i32 = lambda a: torch.from_numpy(np.asarray(a, np.int32)).cuda()
    length = np.asarray(lengths)
    pos = np.tile(np.arange(n * page), (B, 1))
    if evicted:
        seen = 3 * length + 2
        for b in range(B):
            pos[b, :length[b]] = rng.permutation(seen[b])[:length[b]]
    weight = torch.from_numpy(np.exp(rng.standard_normal((B, n * page))).astype(np.float32)).cuda()
    return _kern().TokenCache(k, v, table, i32(length), i32(length if seen is None else seen), weight,
                              i32(pos))


def _rows(cache, b, n):
    """Keys, values and `stored` marks of slots 0 .. n-1 in 64 bits."""
    page = cache.k.shape[1]
    x = np.arange(n)
    t = cache.table[b].long()
    ok = (t >= 0) & (t < cache.k.shape[0])
    t = t.clamp(0, cache.k.shape[0] - 1)[:-(-n // page)]
    k, v = (_np(a[t]).reshape(-1, *a.shape[2:])[:n] for a in (cache.k, cache.v))
    return k, v, ok.cpu().numpy()[x // page]


def _paged_ref(q, cache, window, sinks, dtype):
    B, hq, dh = q.shape
    g = hq // cache.kv_heads
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    add, add_tol = np.zeros(cache.weight.shape), np.zeros(cache.weight.shape)
    length = np.clip(cache.length.cpu().numpy(), 0, cache.capacity)
    seen, pos = cache.seen.cpu().numpy(), cache.pos.cpu().numpy()
    for b in range(B):
        n = int(length[b])
        k, v, see = _rows(cache, b, n)
        if window:
            see = see & ((pos[b, :n] > int(seen[b]) - 1 - window) | (pos[b, :n] < sinks))
        for h in range(hq):
            o, p, t, rel = _attend(q[b, h][None], k[:, h // g], v[:, h // g], see[None], 0.0, dtype)
            out[b, h], tol[b, h] = o[0], t[0]
            add[b, :n] += p[0] / hq
            add_tol[b, :n] += p[0] / hq * (rel[0] + (hq + 2) * U32)
    return out, tol, add, add_tol


PAGED = [  # lengths, heads, kv_heads, dh, page, capacity, window, sinks, evicted
    ([1], 1, 1, 8, 16, 16, None, 0, False),
    ([777], 6, 6, 64, 16, 777, None, 0, False),
    ([0, 5, 64, 65, 130, 1], 4, 2, 64, 27, 140, None, 0, False),
    ([300, 17, 0, 299], 8, 1, 128, 1, 300, 50, 3, True),
    ([2000, 3], 32, 8, 128, 16, 2000, None, 0, True),
    ([1500, 900, 40], 20, 4, 80, 64, 1536, 100, 4, False),
    ([700, 64], 40, 2, 24, 48, 720, 1, 0, False),
    ([513], 16, 2, 96, 128, 600, 1000, 2, True),
    ([4099, 17], 12, 12, 64, 27, 4099, 1000, 4, True),
    ([260, 33, 31], 17, 1, 128, 32, 288, 70, 90, False),
    ([3000], 6, 6, 64, 64, 3008, 257, 1, False),
    ([60000], 64, 64, 8, 64, 60000, 100000, 2, True),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", range(len(PAGED)))
def test_paged_attention(torch_cuda, case, dtype):
    torch = torch_cuda
    lengths, hq, hkv, dh, page, cap, window, sinks, evicted = PAGED[case]
    print(f"[paged] {dtype} {PAGED[case]}", flush=True)
    rng = np.random.default_rng(100 + case)
    c = _cache(torch, rng, dtype, lengths, hkv, dh, page, cap, evicted, heads_first=case % 2 == 1)
    wide = _normal(torch, rng, dtype, len(lengths), hq + 3, dh)
    q = wide[:, 1:hq + 1] if dh * wide.element_size() % 16 == 0 else wide[:, :hq]
    out, tol, add, add_tol = _paged_ref(_np(q), c, window, sinks, dtype)
    before = _np(c.weight)
    kern = _kern()
    got = kern.paged_attention(q, c, window, sinks, accumulate=False)
    assert np.array_equal(_np(c.weight), before)
    _close(_np(got), out, tol)
    given = torch.empty_like(got)
    assert kern.paged_attention(q, c, window, sinks, out=given) is given
    assert torch.equal(given, got)
    w = _np(c.weight)
    assert (np.abs(w - before - add) <= add_tol + U32 * (before + add)).all()
    assert np.array_equal(w[add == 0], before[add == 0])
    # each visible sequence hands out one unit of weight
    some = out.any((1, 2))
    assert np.allclose((w - before).sum(1)[some], 1, atol=1e-3)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_paged_attention_hidden_and_odd_contents(torch_cuda, dtype):
    """NaN and infinities in slots past the length, out of the window, in
    pages that no table entry names; page numbers outside the pages; lengths
    outside the capacity; one page named twice."""
    torch = torch_cuda
    rng = np.random.default_rng(7)
    c = _cache(torch, rng, dtype, [100, 130, 200, 60, 128], 2, 64, 16, 200, evicted=False)
    q = _normal(torch, rng, dtype, 5, 6, 64)
    pages = c.k.shape[0]
    c.table[1, 2], c.table[1, 5], c.table[3, 0], c.table[3, 3] = -1, pages, 1 << 30, -(1 << 31)
    c.table[4, 3] = c.table[4, 6]
    c.length[2] = 5000
    c.seen[2] = 5000
    c.length[0], c.seen[0] = -3, -3
    for window, sinks in ((None, 0), (40, 2)):
        out, tol, add, add_tol = _paged_ref(_np(q), c, window, sinks, dtype)
        assert not out[0].any()
        used = torch.zeros(pages, 16, dtype=torch.bool)
        length = np.clip(c.length.cpu().numpy(), 0, c.capacity)
        seen, pos = c.seen.cpu().numpy(), c.pos.cpu().numpy()
        for b in range(5):
            for x in range(length[b]):
                p = int(c.table[b, x // 16])
                if 0 <= p < pages and (not window or pos[b, x] > seen[b] - 1 - window or
                                       pos[b, x] < sinks):
                    used[p, x % 16] = True
        for value in (float("nan"), float("inf")):
            k, v = c.k.clone(), c.v.clone()
            k[~used.cuda()], v[~used.cuda()] = value, value
            w = c.weight.clone()
            d = _kern().TokenCache(k, v, c.table, c.length, c.seen, w, c.pos)
            _close(_np(_kern().paged_attention(q, d, window, sinks)), out, tol, (window, value))
            err = np.abs(_np(w) - _np(c.weight) - add)
            assert (err <= add_tol + U32 * (_np(c.weight) + add)).all()


@pytest.mark.parametrize("B", [63, 64, 65, 200, 1024, 1025, 2100])
def test_paged_attention_many_sequences(torch_cuda, B):
    """Around the sequences that a wave looks at together and those up to
    which the work is split over lengths, empty ones among them."""
    torch = torch_cuda
    rng = np.random.default_rng(B)
    lengths = [int(v) for v in rng.integers(0, 90, size=B)]
    lengths[-1] = 0
    c = _cache(torch, rng, "bf16", lengths, 1, 64, 16, 96, evicted=True)
    q = _normal(torch, rng, "bf16", B, 2, 64)
    before = _np(c.weight)
    out, tol, add, add_tol = _paged_ref(_np(q), c, 60, 2, "bf16")
    _close(_np(_kern().paged_attention(q, c, 60, 2)), out, tol)
    assert (np.abs(_np(c.weight) - before - add) <= add_tol + U32 * (before + add)).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_paged_attention_caches_in_and_out_of_order(torch_cuda, dtype):
    """Sequences with and without evicted tokens in turn, several to a wave."""
    torch = torch_cuda
    rng = np.random.default_rng(77)
    lengths = rng.integers(0, 300, size=40)
    seen = lengths + np.where(np.arange(40) % 3 == 1, rng.integers(1, 90, size=40), 0)
    cache = _cache(torch, rng, dtype, lengths, 64, 8, 16, 304, seen=seen)
    q = _normal(torch, rng, dtype, 40, 64, 8)
    before = _np(cache.weight)
    got = _kern().paged_attention(q, cache, 100, 3)
    ref, tol, add, add_tol = _paged_ref(_np(q), cache, 100, 3, dtype)
    _close(_np(got), ref, tol)
    after = before + add
    _close(_np(cache.weight), after, add_tol + U32 * np.abs(after))


@pytest.mark.parametrize("seen", [-(1 << 31), 0, (1 << 31) - 1])
def test_extreme_positions(torch_cuda, seen):
    """Positions and counts at the ends of their type: no wrapped sums."""
    torch = torch_cuda
    rng = np.random.default_rng(15)
    c = _cache(torch, rng, "bf16", [70, 40], 1, 64, 16, 80, seen=[seen, seen])
    ends = np.array([-(1 << 31), -1, 0, 1, (1 << 31) - 2, (1 << 31) - 1])
    pos = rng.choice(ends, size=c.pos.shape).astype(np.int32)
    c.pos.copy_(torch.from_numpy(pos))
    q = _normal(torch, rng, "bf16", 2, 3, 64)
    for window, sinks in ((1, 0), (5, 1), (1 << 30, 0)):
        out, tol, _, _ = _paged_ref(_np(q), c, window, sinks, "bf16")
        _close(_np(_kern().paged_attention(q, c, window, sinks)), out, tol, window)
    w = c.weight.cpu().numpy()
    want = [_evict_ref(n, seen, w[b], pos[b], c.capacity, 30, 1, 20)[0] for b, n in enumerate((70, 40))]
    assert np.array_equal(_kern().cache_evict(c, 30, 1, 20).cpu().numpy(), np.array(want))


def test_paged_attention_offsets_past_32_bits(torch_cuda):
    """Pages so far apart that element offsets pass 2^31, and byte offsets 2^32."""
    torch = torch_cuda
    rng = np.random.default_rng(8)
    c = _cache(torch, rng, "bf16", [300, 290], 2, 64, 16, 304, evicted=True)
    pages, gap = c.k.shape[0], 1 << 26
    big = torch.empty(pages * gap, dtype=torch.bfloat16, device="cuda")
    k = big.as_strided(c.k.shape, (gap, 128, 64, 1), 0)
    v = big.as_strided(c.k.shape, (gap, 128, 64, 1), 1 << 20)
    k.copy_(c.k), v.copy_(c.v)
    w = c.weight.clone()
    far = _kern().TokenCache(k, v, c.table, c.length.clone(), c.seen.clone(), w, c.pos.clone())
    q = _normal(torch, rng, "bf16", 2, 4, 64)
    kern = _kern()
    assert torch.equal(kern.paged_attention(q, far), kern.paged_attention(q, c))
    assert torch.equal(w, c.weight)
    new = [_normal(torch, rng, "bf16", 2, 2, 64) for _ in range(2)]
    for x in (far, c):
        kern.cache_append(x, *new)
    assert torch.equal(kern.cache_evict(far, 200, 1, 8), kern.cache_evict(c, 200, 1, 8))
    assert torch.equal(far.k, c.k) and torch.equal(far.v, c.v)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("counts", [None, [0, 3, 40, 1, 200, 7], [70, 0, 0, 0, 0, 33]])
def test_cache_append(torch_cuda, dtype, counts):
    """Ragged rows, none, more than fit, into a page that is not there."""
    torch = torch_cuda
    print(f"[append] {dtype} {counts}", flush=True)
    rng = np.random.default_rng(9)
    lengths = [0, 5, 60, 96, 30, 95]
    c = _cache(torch, rng, dtype, lengths, 3, 40, 27, 100, evicted=False,
               seen=[0, 50, 60, 200, 30, 95], heads_first=counts is None)
    c.table[2, 3] = -1
    c.table[4, 2] = c.k.shape[0]
    n = np.ones(6, int) if counts is None else np.array(counts)
    rows = _normal(torch, rng, dtype, int(n.sum()), 6, 40)
    k, v = rows[:, :3], rows[:, 3:]
    state = {x: _np(getattr(c, x)) for x in ("k", "v", "weight", "pos", "length", "seen")}
    table, r = c.table.cpu().numpy(), 0
    for b in range(6):
        for i in range(n[b]):
            x = int(state["length"][b])
            if x < c.capacity:
                state["weight"][b, x], state["pos"][b, x] = 0, state["seen"][b]
                p = table[b, x // 27]
                if 0 <= p < c.k.shape[0]:
                    state["k"][p, x % 27], state["v"][p, x % 27] = _np(k[r]), _np(v[r])
                state["length"][b] += 1
                state["seen"][b] += 1
            r += 1
    cu = None if counts is None else np.concatenate([[0], np.cumsum(n)])
    if counts is not None:  # rows behind the last sequence take no part
        k, v = (torch.cat([t, t[:3]]) for t in (k, v))
    _kern().cache_append(c, k, v, cu)
    for x in state:
        assert np.array_equal(_np(getattr(c, x)), state[x]), x


@pytest.mark.parametrize("B,most", [(255, 8), (256, 9), (257, 8), (600, 20)])
def test_cache_append_many_sequences(torch_cuda, B, most):
    """More sequences than one launch describes, few rows each or more."""
    torch = torch_cuda
    rng = np.random.default_rng(B)
    n = rng.integers(0, most + 1, size=B)
    n[3] = most
    lengths = rng.integers(0, 12, size=B)
    c = _cache(torch, rng, "bf16", lengths, 1, 16, 16, 32, seen=lengths + 5)
    k, v = (_normal(torch, rng, "bf16", int(n.sum()), 1, 16) for _ in range(2))
    cu = np.concatenate([[0], np.cumsum(n)])
    _kern().cache_append(c, k, v, cu)
    assert np.array_equal(c.length.cpu().numpy(), lengths + n)
    assert np.array_equal(c.seen.cpu().numpy(), lengths + 5 + n)
    pos, w = c.pos.cpu().numpy(), c.weight.cpu().numpy()
    for b in range(B):
        new = slice(lengths[b], lengths[b] + n[b])
        kc, vc, _ = _rows(c, b, int(lengths[b] + n[b]))
        assert np.array_equal(kc[new], _np(k[cu[b]:cu[b + 1]]))
        assert np.array_equal(vc[new], _np(v[cu[b]:cu[b + 1]]))
        assert np.array_equal(pos[b, new], lengths[b] + 5 + np.arange(n[b])) and not w[b, new].any()


def _evict_ref(length, seen, weight, pos, cap, budget, sinks, recent):
    """src and moves of one sequence."""
    n = max(0, min(length, cap))
    src = np.full(budget, -1)
    src[:min(n, budget)] = np.arange(min(n, budget))
    if n <= budget:
        return src, []
    p, w, seen = pos[:n].astype(np.int64), weight[:n].astype(np.float64), int(seen)
    safe = (p < sinks) | (p >= seen - recent)
    order = sorted(range(n), key=lambda x: (not safe[x], math.isnan(w[x]) and not safe[x],
                                            0 if safe[x] or math.isnan(w[x]) else -w[x], x))
    keep = np.zeros(n, bool)
    keep[order[:budget]] = True
    moves = list(zip(np.flatnonzero(~keep[:budget]), budget + np.flatnonzero(keep[budget:])))
    for d, s in moves:
        src[d] = s
    return src, moves


EVICT = [  # lengths, capacity, page, budget, sinks, recent, weights
    ([10], 16, 16, 4, 1, 2, "normal"),
    ([0, 1, 64, 65, 100, 128], 128, 27, 64, 4, 8, "normal"),
    ([1500, 1024, 1025, 3000], 3000, 16, 1024, 4, 100, "normal"),
    ([1100, 2047], 2048, 64, 1, 0, 1, "normal"),
    ([900, 500], 900, 1, 300, 0, 0, "equal"),
    ([900, 500], 900, 64, 300, 2, 298, "few"),
    ([800, 801], 801, 32, 333, 3, 5, "odd"),
    ([5000, 257], 5000, 48, 256, 0, 0, "few"),
    ([100, 30], 128, 16, 500, 0, 0, "normal"),
    ([20000, 16385], 20000, 64, 16384, 4, 64, "normal"),
    ([70000, 10], 70001, 128, 1000, 4, 64, "normal"),
]


@pytest.mark.parametrize("case", range(len(EVICT)))
def test_cache_evict(torch_cuda, case):
    """Kept sets, moves and contents are exactly those of a plain sort, for
    equal weights, few distinct ones, infinities, NaN and zeros of both signs."""
    torch = torch_cuda
    lengths, cap, page, budget, sinks, recent, kind = EVICT[case]
    print(f"[evict] {EVICT[case]}", flush=True)
    rng = np.random.default_rng(200 + case)
    dtype = "bf16" if case % 2 else "fp32"
    c = _cache(torch, rng, dtype, lengths, 2, 24, page, cap, evicted=True,
               heads_first=case % 3 == 1)
    if case == 2:
        c.table[0, 3] = -1  # moves into or out of a page that is not there
    w = c.weight.cpu().numpy().copy()
    if kind == "equal":
        w[:] = 0.5
    elif kind == "few":
        w = rng.integers(0, 4, size=w.shape).astype(np.float32)
    elif kind == "odd":
        w = rng.choice(np.array([0.0, -0.0, np.inf, -np.inf, np.nan, 1e-40, -1.0, 2.0], np.float32),
                       size=w.shape)
    c.weight.copy_(torch.from_numpy(w))
    state = {x: (getattr(c, x).float() if x in "kv" else getattr(c, x)).cpu().numpy().copy()
             for x in ("k", "v", "weight", "pos", "length", "seen")}
    table, pages = c.table.cpu().numpy(), c.k.shape[0]
    want = []
    for b in range(len(lengths)):
        src, moves = _evict_ref(lengths[b], state["seen"][b], w[b], state["pos"][b], c.capacity, budget,
                                sinks, recent)
        want.append(src)
        for d, s in moves:
            state["weight"][b, d], state["pos"][b, d] = state["weight"][b, s], state["pos"][b, s]
            pd, ps = table[b, d // page], table[b, s // page]
            if 0 <= pd < pages and 0 <= ps < pages:
                for x in "kv":
                    state[x][pd, d % page] = state[x][ps, s % page]
        state["length"][b] = min(lengths[b], budget)
    src = _kern().cache_evict(c, budget, sinks, recent)
    assert np.array_equal(src.cpu().numpy(), np.array(want))
    for x in state:
        got = getattr(c, x)
        got = (got.float() if x in "kv" else got).cpu().numpy()
        assert np.array_equal(got, state[x], equal_nan=True), x


# ---------------------------------------------------------------- together --
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_prompt_decode_and_evict_together(torch_cuda, dtype):
    """A prompt by windowed attention, its rows appended, then steps that
    append, attend and evict; the last prompt row equals the cache's answer,
    and every step the 64-bit one for the tokens that the evictions left."""
    torch = torch_cuda
    rng = np.random.default_rng(11)
    kern = _kern()
    lengths, hq, hkv, dh, window, sinks, budget = [90, 1, 40], 8, 2, 64, 50, 2, 60
    cu = np.concatenate([[0], np.cumsum(lengths)])
    q, k, v = (_normal(torch, rng, dtype, int(cu[-1]), h, dh) for h in (hq, hkv, hkv))
    prompt = kern.window_attention(q, k, v, cu, window, sinks)
    c = kern.TokenCache.empty(3, 100, hkv, dh, page_size=16, dtype=_dt(torch, dtype))
    kern.cache_append(c, k, v, cu)
    last = torch.tensor(cu[1:] - 1, device="cuda")
    out, tol, _, _ = _paged_ref(_np(q[last]), c, window, sinks, dtype)
    got = kern.paged_attention(q[last], c, window, sinks)
    _close(_np(got), out, tol)
    # both are within the bound of the same sum
    assert (np.abs(_np(got) - _np(prompt[last])) <= 2 * tol).all()
    token = [[int(a + i) for i in range(b - a)] for a, b in zip(cu[:-1], cu[1:])]  # row of each slot
    rows_k, rows_v = _np(k), _np(v)
    for step in range(30):
        src = kern.cache_evict(c, budget, sinks, 8).cpu().numpy()
        qs, ks, vs = (_normal(torch, rng, dtype, 3, h, dh) for h in (hq, hkv, hkv))
        kern.cache_append(c, ks, vs)
        w = window if step % 2 else None
        got = kern.paged_attention(qs, c, w, sinks)
        rows_k, rows_v = np.concatenate([rows_k, _np(ks)]), np.concatenate([rows_v, _np(vs)])
        for b in range(3):
            token[b] = [token[b][x] for x in src[b] if x >= 0] + [len(rows_k) - 3 + b]
            n = int(c.length[b])
            assert n == len(token[b])
            kc, vc, _ = _rows(c, b, n)
            assert np.array_equal(kc, rows_k[token[b]]) and np.array_equal(vc, rows_v[token[b]])
        out, tol, _, _ = _paged_ref(_np(qs), c, w, sinks, dtype)
        _close(_np(got), out, tol, step)
    assert c.length.cpu().tolist() == [61, 31, 61] and c.seen.cpu().tolist() == [120, 31, 70]


def test_steps_captured_in_a_graph(torch_cuda):
    """A captured step (append, attention, eviction), replayed several times
    with eager work in between, equals eager steps of a second cache."""
    torch = torch_cuda
    rng = np.random.default_rng(12)
    kern = _kern()
    a = _cache(torch, rng, "bf16", [64, 80, 3], 2, 64, 16, 96, evicted=True)
    rng = np.random.default_rng(12)
    b = _cache(torch, rng, "bf16", [64, 80, 3], 2, 64, 16, 96, evicted=True)
    q, k, v = (_normal(torch, rng, "bf16", 3, h, 64) for h in (4, 2, 2))
    out = torch.empty(3, 4, 64, dtype=torch.bfloat16, device="cuda")
    cu = np.array([0, 1, 3], np.int32)

    def step(c, out):
        kern.cache_append(c, k, v)
        kern.paged_attention(q, c, 60, 2, out=out)
        return kern.cache_evict(c, 64, 2, 4), kern.window_attention(q, q, q, cu, 2, 0)

    ref = torch.empty_like(out)
    src_b, win_b = step(b, ref)  # also warms up what a first call loads
    state = [t.clone() for t in a._tensors]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        src, win = step(a, out)
    assert all(torch.equal(x, y) for x, y in zip(a._tensors, state))  # capture runs nothing
    for replay in range(4):
        if replay:
            q.copy_(_normal(torch, rng, "bf16", 3, 4, 64))
            k.copy_(_normal(torch, rng, "bf16", 3, 2, 64))
            src_b, win_b = step(b, ref)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref) and torch.equal(src, src_b) and torch.equal(win, win_b), replay
        assert all(torch.equal(x, y) for x, y in zip(a._tensors, b._tensors)), replay


def test_calls_on_a_side_stream_record_their_tensors(torch_cuda, monkeypatch):
    """Tensors of another stream are recorded; two streams at once with a
    cache each give what one after the other gives."""
    torch = torch_cuda
    used = set()
    record = torch.Tensor.record_stream
    monkeypatch.setattr(torch.Tensor, "record_stream",
                        lambda t, s: (used.add((t.data_ptr(), s.cuda_stream)), record(t, s))[1])
    kern = _kern()
    made = []
    for _ in range(3):
        rng = np.random.default_rng(13)
        c = _cache(torch, rng, "bf16", [500, 60], 2, 64, 16, 600, evicted=True)
        made.append((c, *(_normal(torch, rng, "bf16", 2, h, 64) for h in (4, 2, 2))))

    def steps(c, q, k, v):
        outs = []
        for _ in range(5):
            kern.cache_append(c, k, v)
            outs.append(kern.paged_attention(q, c))
            outs.append(kern.window_attention(q, k, v, [0, 2]))
        return outs, kern.cache_evict(c, 50, 1, 1)

    want, src = steps(*made[0])
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for s, m in zip(streams, made[1:]):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append(steps(*m))
    torch.cuda.synchronize()
    for (outs, e), s, m in zip(got, streams, made[1:]):
        assert all(torch.equal(x, y) for x, y in zip(outs, want)) and torch.equal(e, src)
        assert {(t.data_ptr(), s.cuda_stream) for t in (*m[0]._tensors, *m[1:])} <= used


def test_refusals_on_the_gpu(torch_cuda):
    torch = torch_cuda
    from paper_2607_02612_amd import FusionError
    kern = _kern()
    rng = np.random.default_rng(14)
    c = _cache(torch, rng, "bf16", [20, 5], 2, 64, 16, 32)
    n = lambda *s: _normal(torch, rng, "bf16", *s)
    q, k = n(2, 4, 64), n(2, 2, 64)
    for call in [
        lambda: kern.window_attention(q, k, k, [0, 3]),                     # past the rows
        lambda: kern.window_attention(q, k, k, [0, 2], window=0),
        lambda: kern.window_attention(q, k, k, [0, 2], window=1.5),
        lambda: kern.window_attention(q, k, k, [0, 2], sinks=-1),
        lambda: kern.window_attention(q, k, k, [0, 2.0]),
        lambda: kern.window_attention(q, k, k, np.array([0, (1 << 32) + 2])),
        lambda: kern.window_attention(q, k.float(), k, [0, 2]),
        lambda: kern.window_attention(q, k[:1], k, [0, 1]),
        lambda: kern.window_attention(q, k, k, [0, 2], size=torch.ones(2)),  # host tensor
        lambda: kern.window_attention(q, k, k, [0, 2], out=q[:, :2]),
        lambda: kern.window_attention(q.half(), k.half(), k.half(), [0, 2]),
        lambda: kern.window_attention(q.requires_grad_(), k, k, [0, 2]),
        lambda: kern.window_attention(q.detach(), k, k, [0, 2], size=torch.ones(
            2, device="cuda", requires_grad=True)),
        lambda: kern.cache_append(c, k, k, [0, 2, 3]),
        lambda: kern.window_attention(n(2, 4, 68)[:, :, 4:], k, k, [0, 2]),  # base, strides
        lambda: kern.paged_attention(n(3, 4, 64), c),
        lambda: kern.paged_attention(n(2, 4, 32), c),
        lambda: kern.paged_attention(q.detach(), c, window=-1),
        lambda: kern.cache_append(c, k[:1], k[:1]),
        lambda: kern.cache_append(c, k, k, [0, 2]),
        lambda: kern.cache_evict(c, 0),
        lambda: kern.cache_evict(c, 4, 3, 2),
        lambda: kern.TokenCache(*c._tensors[:2], c.table.long(), *c._tensors[3:]),
        lambda: kern.TokenCache(*c._tensors[:5], c.weight[:, :16].contiguous(), c.pos),
        lambda: kern.TokenCache(c.k[:1].expand(4, -1, -1, -1), *c._tensors[1:]),
    ]:
        with pytest.raises(ValueError):
            call()
    q = q.detach()
    for call in [
        lambda: kern.window_attention(n(2, 3, 64), k, k, [0, 2]),           # heads
        lambda: kern.window_attention(q, k, k, [0, 2, 1]),                  # order
        lambda: kern.window_attention(q, k, k, [1, 2]),
        lambda: kern.window_attention(n(2, 1, 136), n(2, 1, 136), n(2, 1, 136), [0, 2]),
        lambda: kern.paged_attention(n(2, 3, 64), c),
    ]:
        with pytest.raises(FusionError):
            call()
    with torch.no_grad():
        kern.window_attention(q.requires_grad_(), k, k, [0, 2])

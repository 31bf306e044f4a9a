"""Token caches in 4 bits (kernels.TokenCache4 with cache_append, paged_attention
and cache_evict) against plain NumPy in 64 bits.

What is held is compared bit by bit: the rounding to e2m1 is exact arithmetic.
Attention is compared with that of the held values.  Keys and values are exact
in bf16, fp32 queries and weights are sums of three bf16 numbers (24 bits), so
the tolerances are those of test_gpu_cache.py; a sum of three products for one
has at most 3 dh additions, which (dh + 8) 2^-24 sum |q||k| still covers, as the
parts after the first are below 2^-8 of it."""
import numpy as np
import pytest

from test_gpu_cache import (EVICT, PAGED, _attend, _close, _dt, _evict_ref, _kern, _normal,  # noqa: F401
                            _np, U32, torch_cuda)

pytestmark = pytest.mark.gpu
GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


# ------------------------------------------------------------- plain form --
def quantise(x):
    """x [.., dh] in 64 bits -> codes [.., dh], scales [.., dh / 32]."""
    b = np.asarray(x, np.float64).reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    top = np.abs(b).max(-1)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.clip(np.floor(np.log2(top)) - 2, -125, 125)
    bad = ~np.isfinite(b).all(-1)
    e = np.where(bad, 0, e)
    a = np.where(bad[..., None], 0, b) / 2.0 ** e[..., None]
    far = np.abs(np.abs(a)[..., None] - GRID)
    code = (far + np.array([0, 1e-9] * 4)).argmin(-1)  # of two as near the even one
    code = code | np.where(np.signbit(a), 8, 0)
    return (np.where(bad[..., None], 0, code).reshape(x.shape).astype(np.uint8),
            np.where(bad, 255, e + 127).astype(np.uint8))


def values(codes, scales):
    """codes [.., dh / 2] bytes, scales [.., dh / 32] -> [.., dh] in 64 bits."""
    c = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1, 32)
    v = np.where(c & 8, -1.0, 1.0) * GRID[c & 7]
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (v * s[..., None]).reshape(*codes.shape[:-1], -1)


def held(cache):
    """Keys and values of all pages, [pages, page_size, kv_heads, dh]."""
    return [values(getattr(cache, x).cpu().numpy(), getattr(cache, x + "_scale").cpu().numpy())
            for x in "kv"]


def cache4(torch, rng, dtype, lengths, hkv, dh, page, cap, evicted=False, heads_first=True, seen=None):
    """A cache with shuffled pages and random contents."""
    B, n = len(lengths), -(-cap // page)
    pages = B * n + 2
    shape = (pages, hkv, page) if heads_first else (pages, page, hkv)
    u8 = lambda lo, hi, w: torch.from_numpy(rng.integers(lo, hi, (*shape, w), dtype=np.uint8)).cuda()
    ts = [u8(0, 256, dh // 2), u8(0, 256, dh // 2), u8(122, 128, dh // 32), u8(120, 131, dh // 32)]
    if heads_first:
        ts = [t.transpose(1, 2) for t in ts]
    table = torch.from_numpy(rng.permutation(pages)[:B * n].reshape(B, n).astype(np.int32)).cuda()
    i32 = lambda a: torch.from_numpy(np.asarray(a, np.int32)).cuda()
    length = np.asarray(lengths)
    pos = np.tile(np.arange(n * page), (B, 1))
    if evicted:
        seen = 3 * length + 2
        for b in range(B):
            pos[b, :length[b]] = rng.permutation(seen[b])[:length[b]]
    weight = torch.from_numpy(np.exp(rng.standard_normal((B, n * page))).astype(np.float32)).cuda()
    return _kern().TokenCache4(*ts, table, i32(length), i32(length if seen is None else seen), weight,
                               i32(pos), dtype=_dt(torch, dtype))


def slots(cache, kv, b, n):
    """Keys, values and `stored` marks of slots 0 .. n-1 of a sequence."""
    page = cache.k.shape[1]
    t = cache.table[b].cpu().numpy().astype(np.int64)
    ok = (t >= 0) & (t < cache.k.shape[0])
    x = np.arange(n)
    at = np.clip(t, 0, cache.k.shape[0] - 1)[x // page]
    return kv[0][at, x % page], kv[1][at, x % page], ok[x // page]


def paged_ref(q, cache, window, sinks, dtype, chosen=None):
    """out, its tolerance, added weights, theirs; `chosen` [B, kv_heads, blocks]:
    pages that are attended."""
    B, hq, dh = q.shape
    g = hq // cache.kv_heads
    kv = held(cache) if cache.k.dtype.itemsize == 1 else [_np(cache.k), _np(cache.v)]
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    add, add_tol = np.zeros(cache.weight.shape), np.zeros(cache.weight.shape)
    length = np.clip(cache.length.cpu().numpy(), 0, cache.capacity)
    seen, pos = cache.seen.cpu().numpy(), cache.pos.cpu().numpy()
    for b in range(B):
        n = int(length[b])
        k, v, see = slots(cache, kv, b, n)
        if window:
            see = see & ((pos[b, :n] > int(seen[b]) - 1 - window) | (pos[b, :n] < sinks))
        for h in range(hq):
            s = see
            if chosen is not None:
                s = see & np.isin(np.arange(n) // cache.k.shape[1], chosen[b, h // g])
            o, p, t, rel = _attend(q[b, h][None], k[:, h // g], v[:, h // g], s[None], 0.0, dtype)
            out[b, h], tol[b, h] = o[0], t[0]
            add[b, :n] += p[0] / hq
            add_tol[b, :n] += p[0] / hq * (rel[0] + (hq + 2) * U32)
    return out, tol, add, add_tol


# ----------------------------------------------------------------- append --
def _odd_rows(rng, rows, heads, dh):
    """Rows with ties, both zeros, the ends of the range, infinities and NaN."""
    x = rng.standard_normal((rows, heads, dh)).astype(np.float32)
    x[::5] = rng.choice(np.array([0, -0.0, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, 7, -5, -2.5, 6, 4]),
                        size=x[::5].shape)
    x[1::7] *= np.float32(2.0) ** rng.integers(-110, 110, size=(len(x[1::7]), heads, 1))
    x[2::11] = 0
    x[3::11, :, ::2] = -0.0
    x[3::11, :, 1::2] = 0
    x[4::11, :, :8] = 3.3e38
    x[5::11, 0, 3] = np.inf
    x[6::11, -1, -2] = np.nan
    x[7::11, 0, 5] = -np.inf
    return x


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dh", [32, 64, 96, 128])
@pytest.mark.parametrize("counts", [None, [0, 3, 40, 1, 200, 7], [5, 0, 8, 0, 0, 2]])
def test_append_rounds_to_four_bits(torch_cuda, dtype, dh, counts):
    """Ragged rows, none, more than fit, into a page that is not there."""
    torch = torch_cuda
    print(f"[append4] {dtype} {dh} {counts}", flush=True)
    rng = np.random.default_rng(dh)
    lengths = [0, 5, 60, 96, 30, 95]
    c = cache4(torch, rng, dtype, lengths, 3, dh, 27, 100, seen=[0, 50, 60, 200, 30, 95],
               heads_first=counts is None)
    c.table[2, 3] = -1
    c.table[4, 2] = c.k.shape[0]
    n = np.ones(6, int) if counts is None else np.array(counts)
    rows = torch.from_numpy(_odd_rows(rng, int(n.sum()), 6, dh)).cuda().to(c.dtype)
    k, v = rows[:, :3], rows[:, 3:]
    want = {x: getattr(c, x).cpu().numpy().copy()
            for x in ("k", "v", "k_scale", "v_scale", "weight", "pos", "length", "seen")}
    new = [quantise(_np(t)) for t in (k, v)]
    table, r = c.table.cpu().numpy(), 0
    for b in range(6):
        for i in range(n[b]):
            x = int(want["length"][b])
            if x < c.capacity:
                want["weight"][b, x], want["pos"][b, x] = 0, want["seen"][b]
                p = table[b, x // 27]
                if 0 <= p < c.k.shape[0]:
                    for t, (codes, scales) in zip("kv", new):
                        want[t][p, x % 27] = codes[r, :, ::2] | codes[r, :, 1::2] << 4
                        want[t + "_scale"][p, x % 27] = scales[r]
                want["length"][b] += 1
                want["seen"][b] += 1
            r += 1
    cu = None if counts is None else np.concatenate([[0], np.cumsum(n)])
    if counts is not None:  # rows behind the last sequence take no part
        k, v = (torch.cat([t, t[:2]]) for t in (k, v))
    _kern().cache_append(c, k, v, cu)
    for x in want:
        assert np.array_equal(getattr(c, x).cpu().numpy(), want[x]), x


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_append_rounds_every_value(torch_cuda, dtype):
    """Each bf16 number (fp32: and what lies beside it) under a block's largest
    value of 4 to 8, and subnormal numbers."""
    torch = torch_cuda
    bits = np.arange(1 << 16, dtype=np.uint32) << 16
    x = bits.view(np.float32)
    x = x[np.abs(x) < 8]
    if dtype == "fp32":
        near = np.concatenate([GRID, (GRID[1:] + GRID[:-1]) / 2, [7]]).astype(np.float32)
        near = np.concatenate([np.nextafter(near, np.float32(9)), np.nextafter(near, np.float32(-9)), near])
        x = np.concatenate([x, near, -near])
    x = np.concatenate([x, np.zeros(-len(x) % 31, np.float32)]).reshape(-1, 31)
    for top in (4.0, 7.75):
        rows = np.concatenate([np.full((len(x), 1), top, np.float32), x], 1)
        rows = np.concatenate([rows, np.zeros((-len(rows) % 4, 32), np.float32)]).reshape(-1, 4, 32)
        small = rows[:50] * np.float32(2.0) ** -127  # subnormal: below the least scale
        rows = np.concatenate([rows, small])
        k = torch.from_numpy(rows).cuda().to(_dt(torch, dtype))
        c = _kern().TokenCache4.empty(1, len(rows), 4, 32, dtype=_dt(torch, dtype))
        _kern().cache_append(c, k, -k, [0, len(rows)])
        for t, want in (("k", quantise(_np(k))), ("v", quantise(_np(-k)))):
            at = torch.arange(len(rows), device="cuda")
            got = getattr(c, t)[at // 64, at % 64].cpu().numpy()
            assert np.array_equal(got, want[0][..., ::2] | want[0][..., 1::2] << 4)
            assert np.array_equal(getattr(c, t + "_scale")[at // 64, at % 64].cpu().numpy(), want[1])


# -------------------------------------------------------------- attention --
FOURS = [c for c in PAGED if c[3] % 32 == 0] + [
    ([300, 0, 31, 32, 33], 4, 4, 32, 27, 300, None, 0, False),
    ([90, 500], 34, 2, 32, 16, 512, 60, 2, True),
    ([2000, 64, 7], 24, 8, 96, 64, 2048, None, 0, False),
    ([513, 5, 64, 65, 0], 16, 2, 96, 128, 600, None, 0, True),
    ([700, 64], 40, 2, 32, 48, 720, None, 0, False),
    ([1300, 15], 17, 1, 128, 32, 1312, None, 0, False),
    ([1300, 130, 63], 12, 2, 128, 16, 1312, None, 0, False),
    ([4100], 8, 8, 32, 80, 4160, None, 0, False),
    ([3000, 1], 33, 11, 64, 16, 3008, None, 0, True),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", range(len(FOURS)))
def test_paged_attention_over_four_bits(torch_cuda, case, dtype):
    torch = torch_cuda
    lengths, hq, hkv, dh, page, cap, window, sinks, evicted = FOURS[case]
    print(f"[paged4] {dtype} {FOURS[case]}", flush=True)
    rng = np.random.default_rng(400 + case)
    c = cache4(torch, rng, dtype, lengths, hkv, dh, page, cap, evicted, heads_first=case % 2 == 0)
    q = _normal(torch, rng, dtype, len(lengths), hq + 3, dh)[:, 1:hq + 1]
    out, tol, add, add_tol = paged_ref(_np(q), c, window, sinks, dtype)
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


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dh", [32, 64, 96, 128])
def test_hidden_and_odd_contents(torch_cuda, dtype, dh):
    """NaN blocks in slots past the length, out of the window, in pages that no
    table entry names; page numbers outside the pages; lengths outside the
    capacity; NaN blocks that are seen."""
    torch = torch_cuda
    rng = np.random.default_rng(7)
    c = cache4(torch, rng, dtype, [100, 130, 200, 60, 128], 2, dh, 16, 200)
    q = _normal(torch, rng, dtype, 5, 6, dh)
    pages = c.k.shape[0]
    c.table[1, 2], c.table[1, 5], c.table[3, 0], c.table[3, 3] = -1, pages, 1 << 30, -(1 << 31)
    c.length[2], c.seen[2], c.length[0], c.seen[0] = 5000, 5000, -3, -3
    kern = _kern()
    for window, sinks in ((None, 0), (40, 2)):
        out, tol, add, add_tol = paged_ref(_np(q), c, window, sinks, dtype)
        assert not out[0].any()
        used = torch.zeros(pages, 16, dtype=torch.bool)
        length = np.clip(c.length.cpu().numpy(), 0, c.capacity)
        seen, pos = c.seen.cpu().numpy(), c.pos.cpu().numpy()
        for b in range(5):
            for x in range(length[b]):
                p = int(c.table[b, x // 16])
                if 0 <= p < pages and (not window or pos[b, x] > seen[b] - 1 - window or pos[b, x] < sinks):
                    used[p, x % 16] = True
        ks, vs, w = c.k_scale.clone(), c.v_scale.clone(), c.weight.clone()
        ks[~used.cuda()], vs[~used.cuda()] = 255, 255
        d = kern.TokenCache4(c.k, c.v, ks, vs, c.table, c.length, c.seen, w, c.pos, dtype=c.dtype)
        _close(_np(kern.paged_attention(q, d, window, sinks)), out, tol, window)
        assert (np.abs(_np(w) - _np(c.weight) - add) <= add_tol + U32 * (_np(c.weight) + add)).all()
        # a visible value block of NaN: its 32 dims are NaN, for all heads that read it
        at = int(c.table[4, 7])  # slot 115 of sequence 4, in the window
        vs[at, 3, 1, dh // 32 - 1] = 255
        got = _np(kern.paged_attention(q, d, window, sinks, accumulate=False))
        hole = np.zeros(out.shape, bool)
        hole[4, 3:, dh - 32:] = True
        assert np.isnan(got[hole]).all()
        _close(np.where(hole, 0, got), np.where(hole, 0, out), tol)
        # a visible key block of NaN: the rows that see it are NaN
        ks[at, 3, 0, 0] = 255
        got = _np(kern.paged_attention(q, d, window, sinks, accumulate=False))
        assert np.isnan(got[4, :3]).all() and not np.isnan(got[:4]).any()


@pytest.mark.parametrize("B", [64, 65, 1024, 1025, 2100])
def test_many_sequences(torch_cuda, B):
    torch = torch_cuda
    rng = np.random.default_rng(B)
    lengths = [int(v) for v in rng.integers(0, 90, size=B)]
    lengths[-1] = 0
    c = cache4(torch, rng, "bf16", lengths, 1, 64, 16, 96, evicted=True)
    q = _normal(torch, rng, "bf16", B, 2, 64)
    before = _np(c.weight)
    out, tol, add, add_tol = paged_ref(_np(q), c, 60, 2, "bf16")
    _close(_np(_kern().paged_attention(q, c, 60, 2)), out, tol)
    assert (np.abs(_np(c.weight) - before - add) <= add_tol + U32 * (before + add)).all()


def test_large_scores_and_values(torch_cuda):
    """Scores of several hundred, of either sign, and scales at the ends.

    A weight relative to the largest is an fp32 number, and so are the three
    parts of it: below 2^-126 each of the four is flushed to zero.  The sum of
    weights is at least 1 beside them, so the output is off by at most 4 2^-126
    sum |v| more, which values of 2^115 make visible."""
    torch = torch_cuda
    rng = np.random.default_rng(3)
    for dtype in ("bf16", "fp32"):
        c = cache4(torch, rng, dtype, [150, 90], 2, 64, 16, 160)
        c.k_scale.add_(4)
        c.v_scale[...] = torch.from_numpy(rng.choice(np.array([2, 3, 120, 240], np.uint8),
                                                     size=tuple(c.v_scale.shape))).cuda()
        q = _normal(torch, rng, dtype, 2, 4, 64) * 8
        out, tol, _, _ = paged_ref(_np(q), c, None, 0, dtype)
        kv = held(c)
        for b, n in enumerate((150, 90)):
            tol[b] += 2.0 ** -124 * np.abs(slots(c, kv, b, n)[1]).sum(0).repeat(2, 0)
        _close(_np(_kern().paged_attention(q, c)), out, tol)


# --------------------------------------------------------------- eviction --
@pytest.mark.parametrize("case", range(len(EVICT)))
def test_cache_evict_of_four_bits(torch_cuda, case):
    """Kept sets and moved bytes are those of a plain sort."""
    torch = torch_cuda
    lengths, cap, page, budget, sinks, recent, kind = EVICT[case]
    rng = np.random.default_rng(500 + case)
    c = cache4(torch, rng, "bf16", lengths, 2, (32, 96, 128)[case % 3], page, cap, evicted=True,
               heads_first=case % 2 == 0)
    w = c.weight.cpu().numpy().copy()
    if kind == "equal":
        w[:] = 0.5
    c.weight.copy_(torch.from_numpy(w))
    names = ("k", "v", "k_scale", "v_scale")
    want = {x: getattr(c, x).cpu().numpy().copy() for x in (*names, "weight", "pos", "length", "seen")}
    table, pages, srcs = c.table.cpu().numpy(), c.k.shape[0], []
    for b in range(len(lengths)):
        src, moves = _evict_ref(lengths[b], want["seen"][b], w[b], want["pos"][b], c.capacity, budget,
                                sinks, recent)
        srcs.append(src)
        for d, s in moves:
            want["weight"][b, d], want["pos"][b, d] = want["weight"][b, s], want["pos"][b, s]
            for x in names:
                want[x][table[b, d // page], d % page] = want[x][table[b, s // page], s % page]
        want["length"][b] = min(lengths[b], budget)
    src = _kern().cache_evict(c, budget, sinks, recent)
    assert np.array_equal(src.cpu().numpy(), np.array(srcs))
    for x in want:
        assert np.array_equal(getattr(c, x).cpu().numpy(), want[x]), x
    assert pages == c.k.shape[0]


# ------------------------------------------------------- far apart, refusals --
def test_offsets_past_32_bits(torch_cuda):
    """Pages so far apart that byte offsets pass 2^32."""
    torch = torch_cuda
    rng = np.random.default_rng(8)
    c = cache4(torch, rng, "bf16", [300, 290], 2, 64, 16, 304, evicted=True, heads_first=False)
    pages, gap = c.k.shape[0], 1 << 28
    big = torch.empty(pages * gap, dtype=torch.uint8, device="cuda")
    far = []
    for i, t in enumerate((c.k, c.v, c.k_scale, c.v_scale)):
        view = big.as_strided(t.shape, (gap, 2 * t.shape[3], t.shape[3], 1), i << 20)
        view.copy_(t)
        far.append(view)
    w = c.weight.clone()
    f = _kern().TokenCache4(*far, c.table, c.length.clone(), c.seen.clone(), w, c.pos.clone())
    q = _normal(torch, rng, "bf16", 2, 4, 64)
    kern = _kern()
    assert torch.equal(kern.paged_attention(q, f), kern.paged_attention(q, c))
    assert torch.equal(w, c.weight)
    new = [_normal(torch, rng, "bf16", 2, 2, 64) for _ in range(2)]
    for x in (f, c):
        kern.cache_append(x, *new)
    assert torch.equal(kern.cache_evict(f, 200, 1, 8), kern.cache_evict(c, 200, 1, 8))
    for a, b in zip(f._tensors, c._tensors):
        assert torch.equal(a, b)


def test_refusals(torch_cuda):
    torch = torch_cuda
    kern = _kern()
    rng = np.random.default_rng(14)
    c = cache4(torch, rng, "bf16", [20, 5], 2, 64, 16, 32, heads_first=False)
    ts = list(c._tensors)
    rest = ts[2:7]
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda")
    P = c.k.shape[0]
    for call in [
        lambda: kern.TokenCache4(c.k.float(), c.v, c.k_scale, c.v_scale, *rest),
        lambda: kern.TokenCache4(c.k[..., :24], c.v[..., :24], c.k_scale, c.v_scale, *rest),
        lambda: kern.TokenCache4(c.k, c.v, c.k_scale[..., :1], c.v_scale, *rest),
        lambda: kern.TokenCache4(c.k, c.v, c.k_scale.int(), c.v_scale, *rest),
        lambda: kern.TokenCache4(c.k, c.v, c.k_scale.cpu(), c.v_scale, *rest),
        lambda: kern.TokenCache4(c.k, c.v, c.k_scale, c.v_scale, *rest, dtype=torch.float16),
        lambda: kern.TokenCache4(u8(P, 16, 2, 33)[..., 1:], c.v, c.k_scale, c.v_scale, *rest),
        lambda: kern.TokenCache4(c.k[:1].expand(P, -1, -1, -1), c.v, c.k_scale, c.v_scale, *rest),
        lambda: kern.TokenCache4(c.k, c.v, c.k_scale[:1].expand(P, -1, -1, -1), c.v_scale, *rest),
        lambda: kern.TokenCache4(c.k, c.v, c.k_scale, c.v_scale, rest[0].long(), *rest[1:]),
        lambda: kern.paged_attention(_normal(torch, rng, "fp32", 2, 4, 64), c),
        lambda: kern.cache_append(c, *(_normal(torch, rng, "bf16", 2, 2, 32) for _ in range(2))),
    ]:
        with pytest.raises(ValueError):
            call()
    with pytest.raises(kern._native.FusionError):  # 160-wide heads
        kern.TokenCache4(u8(P, 16, 2, 80), u8(P, 16, 2, 80), u8(P, 16, 2, 5), u8(P, 16, 2, 5), *rest)

"""Page bounds and attention over chosen pages (kernels.PageBounds,
block_attention) against plain NumPy in 64 bits.

Bounds are least and greatest values of what is held: compared bit by bit.  The
choice is compared with that of scores summed in 64 bits and rounded to 32; sums
of 64 bits in another order are off by 2^-52 of sum |q||k|, so the reference
checks that no unchosen page comes nearer than that to a chosen one unless their
scores are equal exactly.  Attention over the chosen pages has the tolerances of
test_gpu_cache.py."""
import numpy as np
import pytest

from test_gpu_cache import _cache, _close, _dt, _kern, _normal, _np, torch_cuda  # noqa: F401
from test_gpu_cache4 import cache4, held, paged_ref

pytestmark = pytest.mark.gpu


def make(torch, rng, bits, *args, **kw):
    dtype = bits.split("/")[0]
    return (cache4 if "/" in bits else _cache)(torch, rng, dtype, *args, **kw)


def keys_of(cache):
    return held(cache)[0] if cache.k.dtype.itemsize == 1 else _np(cache.k)


def bounds_ref(cache, lo, hi, newest=None):
    k, page = keys_of(cache), cache.k.shape[1]
    length = np.clip(cache.length.cpu().numpy(), 0, cache.capacity)
    table = cache.table.cpu().numpy()
    for b, n in enumerate(length):
        first = 0 if newest is None else max(0, n - newest) // page
        for p in range(first, -(-n // page)):
            at = table[b, p]
            if 0 <= at < len(k):
                rows = k[at, :min(page, n - p * page)]
                lo[at] = np.fmin.reduce(rows, axis=0, initial=np.inf)
                hi[at] = np.fmax.reduce(rows, axis=0, initial=-np.inf)
    return lo, hi


def choose_ref(q, cache, lo, hi, blocks, first, recent):
    """chosen [B, kv_heads, blocks]"""
    B, hq, _ = q.shape
    g, page = hq // cache.kv_heads, cache.k.shape[1]
    length = np.clip(cache.length.cpu().numpy(), 0, cache.capacity)
    table = cache.table.cpu().numpy()
    chosen = np.full((B, cache.kv_heads, blocks), -1)
    for b, n in enumerate(length):
        pages = -(-n // page)
        t = table[b, :pages]
        there = (t >= 0) & (t < len(lo))
        at = np.where(there, t, 0)
        for h in range(cache.kv_heads):
            if pages <= blocks:
                chosen[b, h, :pages] = np.arange(pages)
                continue
            qh = q[b, h * g:(h + 1) * g, None]
            with np.errstate(invalid="ignore", over="ignore"):
                s = np.where(qh >= 0, qh * hi[at, h], qh * lo[at, h]).sum(-1)
                err = 2.0 ** -50 * np.abs(np.where(qh >= 0, qh * hi[at, h], qh * lo[at, h])).sum(-1).max(0)
                f = s.astype(np.float32)
                f = np.where(np.isnan(f).any(0), np.nan, f.max(0))
            p = np.arange(pages)
            rank = np.where(np.isnan(f), 2, 1)
            rank[~there] = 0
            rank[(p < first) | (p >= pages - recent)] = 3
            key = np.where(rank == 1, f, 0)
            order = np.lexsort((p, -key, -rank))
            take, leave = order[:blocks], order[blocks:]
            i, j = take[-1], leave[0]
            assert rank[i] != 1 or rank[j] != 1 or f[i] == f[j] or \
                f[i] - f[j] > 2 * max(np.nan_to_num(err[i]), np.nan_to_num(err[j])), "too near to tell"
            chosen[b, h] = np.sort(take)
    return chosen


BITS = ["bf16", "fp32", "bf16/4", "fp32/4"]


@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("hkv,dh,page", [(1, 8, 1), (2, 64, 16), (3, 96, 27), (40, 128, 5), (8, 128, 64),
                                         (5, 32, 300)])
def test_bounds(torch_cuda, bits, hkv, dh, page):
    """All pages, those of the newest slots, pages that are not there, NaN."""
    torch = torch_cuda
    if "/" in bits and dh % 32:
        pytest.skip("4 bits hold blocks of 32 dims")
    print(f"[bounds] {bits} {hkv} {dh} {page}", flush=True)
    rng = np.random.default_rng(dh + page)
    cap = max(40, 3 * page + 1)
    lengths = [0, 1, page, min(cap, 2 * page + 1), cap, cap + 9, -2]
    c = make(torch, rng, bits, lengths, hkv, dh, page, cap, seen=[9] * 7)
    c.table[3, 0], c.table[4, 1] = -1, c.k.shape[0]
    if "/" in bits:
        c.k_scale[int(c.table[5, 1]), 0, 0, 0] = 255
    else:
        c.k[int(c.table[5, 1]), 0, 0, 3] = float("nan")
        c.k[int(c.table[4, 0]), 0, -1, 2] = float("inf")
    shape = (c.k.shape[0], hkv, dh)
    lo, hi = bounds_ref(c, np.zeros(shape), np.zeros(shape))
    made = _kern().PageBounds(c)
    assert made.lo.dtype == c.dtype
    assert np.array_equal(_np(made.lo), lo) and np.array_equal(_np(made.hi), hi)
    for newest in (1, page, 2 * page + 3, 1 << 30):
        given = [torch.full(shape, 7.0, dtype=c.dtype, device="cuda") for _ in range(2)]
        lo, hi = bounds_ref(c, np.full(shape, 7.0), np.full(shape, 7.0), newest)
        b = _kern().PageBounds(c, *given)
        assert b.lo is given[0]
        b.update(newest)
        assert np.array_equal(_np(b.lo), lo) and np.array_equal(_np(b.hi), hi), newest


def test_bounds_of_more_pages_than_a_launch_has_rows(torch_cuda):
    """70,000 pages of one token: bounds are the keys."""
    torch = torch_cuda
    rng = np.random.default_rng(3)
    c = _cache(torch, rng, "bf16", [70000], 1, 16, 1, 70000)
    b = _kern().PageBounds(c)
    t = c.table[0].long()
    assert torch.equal(b.lo[t], c.k[t, 0]) and torch.equal(b.hi[t], c.k[t, 0])
    q = _normal(torch, rng, "bf16", 1, 2, 16)
    got, chosen = _kern().block_attention(q, c, b, 1000, 3, 7)
    want = choose_ref(_np(q), c, _np(b.lo), _np(b.hi), 1000, 3, 7)
    assert np.array_equal(chosen.cpu().numpy(), want)
    out, tol, _, _ = paged_ref(_np(q), c, None, 0, "bf16", want)
    _close(_np(got), out, tol)


BLOCKS = [  # lengths, heads, kv_heads, dh, page, capacity, blocks, first, recent
    ([1], 1, 1, 32, 16, 16, 1, 0, 1),
    ([300, 0, 17, 16, 1], 6, 6, 64, 16, 300, 4, 1, 1),
    ([777, 64, 129], 8, 2, 64, 27, 800, 9, 2, 3),
    ([2000, 1999, 40], 32, 8, 128, 16, 2000, 20, 1, 2),
    ([1500, 900, 40], 20, 4, 96, 64, 1536, 8, 0, 1),
    ([700, 64], 40, 1, 128, 1, 720, 33, 4, 8),
    ([5000], 34, 1, 64, 8, 5000, 100, 0, 100),
    ([9000, 8999], 4, 2, 32, 4, 9000, 257, 1, 1),
    ([600, 20], 3, 3, 128, 200, 600, 2, 1, 1),
    ([130, 77], 2, 2, 64, 16, 160, 50, 1, 1),
    ([1500, 40], 40, 1, 64, 16, 1504, 12, 1, 2),
    ([1500, 1499, 16], 16, 2, 128, 64, 1536, 6, 1, 1),
    ([900, 33], 20, 4, 96, 48, 912, 7, 0, 2),
    ([5000, 129, 64], 4, 1, 128, 64, 5056, 30, 1, 1),
]


@pytest.mark.parametrize("bits", BITS)
@pytest.mark.parametrize("case", range(len(BLOCKS)))
def test_block_attention(torch_cuda, case, bits):
    torch = torch_cuda
    lengths, hq, hkv, dh, page, cap, blocks, first, recent = BLOCKS[case]
    dtype = bits.split("/")[0]
    print(f"[blocks] {bits} {BLOCKS[case]}", flush=True)
    rng = np.random.default_rng(700 + case)
    c = make(torch, rng, bits, lengths, hkv, dh, page, cap, heads_first=case % 2 == 0)
    if case == 3:
        c.table[0, 5], c.table[0, 124], c.table[1, 7] = -1, c.k.shape[0], -9
    q = _normal(torch, rng, dtype, len(lengths), hq + 3, dh)[:, 1:hq + 1]
    kern = _kern()
    b = kern.PageBounds(c)
    state = [t.clone() for t in c._tensors]
    got, chosen = kern.block_attention(q, c, b, blocks, first, recent)
    assert all(torch.equal(x, y) for x, y in zip(c._tensors, state))
    want = choose_ref(_np(q), c, _np(b.lo), _np(b.hi), blocks, first, recent)
    assert np.array_equal(chosen.cpu().numpy(), want)
    out, tol, _, _ = paged_ref(_np(q), c, None, 0, dtype, want)
    _close(_np(got), out, tol)
    given = torch.empty_like(got)
    again, same = kern.block_attention(q, c, b, blocks, first, recent, out=given)
    assert again is given and torch.equal(again, got) and torch.equal(same, chosen)


@pytest.mark.parametrize("bits", BITS)
def test_all_pages_are_paged_attention(torch_cuda, bits):
    torch = torch_cuda
    rng = np.random.default_rng(21)
    c = make(torch, rng, bits, [500, 130, 0], 2, 64, 16, 512)
    q = _normal(torch, rng, bits.split("/")[0], 3, 8, 64)
    kern = _kern()
    got, chosen = kern.block_attention(q, c, kern.PageBounds(c), 32)
    assert torch.equal(got, kern.paged_attention(q, c, accumulate=False))
    assert chosen[0].tolist() == [list(range(32))] * 2 and chosen[2].eq(-1).all()


@pytest.mark.parametrize("bits", BITS)
def test_ties_signs_and_no_bounds(torch_cuda, bits):
    """Pages of equal scores (the lower one's count as the higher), scores of
    either sign, zero and minus zero; pages whose keys are infinite or NaN."""
    torch = torch_cuda
    dtype, four = bits.split("/")[0], "/" in bits
    rng = np.random.default_rng(22)
    kern = _kern()
    c = kern.TokenCache4.empty(2, 640, 2, 64, 16, _dt(torch, dtype)) if four else \
        kern.TokenCache.empty(2, 640, 2, 64, 16, _dt(torch, dtype))
    k = torch.from_numpy(rng.choice(np.array([-2, 0, 0, 1, 2]), size=(1280, 2, 64))).cuda().to(c.dtype)
    k[:, 0, 1:] = 0  # few distinct scores
    k[640:, 1] = -k[640:, 1].abs()
    kern.cache_append(c, k, k, [0, 640, 1280])
    for value in (None, float("inf"), float("nan")):
        if value is not None:
            bad = k[:32].clone()
            bad[3, 0, 0] = bad[20, 1, 5] = value
            c.length[0] = c.seen[0] = 608
            kern.cache_append(c, bad, bad, [0, 32, 32])
        b = kern.PageBounds(c)
        q = _normal(torch, rng, dtype, 2, 4, 64).abs()
        q[1, :, ::7] = 0
        q[0, 1] = 0
        q[0, 2] = -q[0, 2]
        for blocks in (2, 5, 17, 38, 39):
            got, chosen = kern.block_attention(q, c, b, blocks, 1, 1)
            want = choose_ref(_np(q), c, _np(b.lo), _np(b.hi), blocks, 1, 1)
            assert np.array_equal(chosen.cpu().numpy(), want), (value, blocks)
            if value is None:
                out, tol, _, _ = paged_ref(_np(q), c, None, 0, dtype, want)
                _close(_np(got), out, tol, blocks)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("pages", [100, 700, 5000])
def test_scores_that_32_bits_cannot_tell_apart(torch_cuda, dtype, pages):
    """Keys that are the same numbers in another order: their sums are equal,
    and sums of 32 bits are not.  Some pages are higher or lower by little more
    than 32 bits hold, some by far."""
    torch = torch_cuda
    rng = np.random.default_rng(pages)
    kern = _kern()
    base = rng.standard_normal(64)
    x = np.stack([rng.permutation(base) for _ in range(pages)])
    x = torch.from_numpy(x.astype(np.float32)).to(_dt(torch, dtype)).double().numpy()
    x[rng.integers(0, pages, pages // 9)] += 2.0 ** -6  # (a bf16 number's last bits, at 2)
    x[rng.integers(0, pages, pages // 9)] -= 2.0 ** -6
    x[rng.integers(0, pages, 3)] += 1
    k = torch.from_numpy(x).cuda().to(_dt(torch, dtype)).repeat_interleave(2, 0).view(-1, 1, 64)
    c = kern.TokenCache.empty(1, 2 * pages, 1, 64, 2, _dt(torch, dtype))
    kern.cache_append(c, k, k, [0, 2 * pages])
    b = kern.PageBounds(c)
    q = torch.ones(1, 3, 64, dtype=c.dtype, device="cuda")
    q[0, 1:] = -4
    q[0, 2, :32] = 4
    for heads in (slice(0, 1), slice(0, 2), slice(0, 3)):
        for blocks in (3, pages // 20, pages // 3, pages - 1):
            _, chosen = kern.block_attention(q[:, heads], c, b, blocks, 1, 1)
            want = choose_ref(_np(q[:, heads]), c, _np(b.lo), _np(b.hi), blocks, 1, 1)
            assert np.array_equal(chosen.cpu().numpy(), want), (heads, blocks)


def test_infinite_values_of_chosen_pages(torch_cuda):
    """An output dimension with infinite values among the attended ones is
    their sum; infinities in pages that are not chosen have no influence."""
    torch = torch_cuda
    rng = np.random.default_rng(23)
    kern = _kern()
    for dtype in ("bf16", "fp32"):
        c = _cache(torch, rng, dtype, [400], 2, 64, 16, 400)
        q = _normal(torch, rng, dtype, 1, 4, 64)
        b = kern.PageBounds(c)
        clean, chosen = kern.block_attention(q, c, b, 6, 1, 1)
        pages = [set(row) for row in chosen[0].tolist()]
        for p in range(25):
            c.v[int(c.table[0, p]), 3, 0, 5 if p in pages[0] else 6] = float("inf")
        got, same = kern.block_attention(q, c, b, 6, 1, 1)
        assert torch.equal(same, chosen)
        hole = torch.zeros(1, 4, 64, dtype=torch.bool, device="cuda")
        hole[:, :2, 5] = True
        assert torch.isposinf(got[hole]).all() and torch.equal(got[~hole], clean[~hole])


@pytest.mark.parametrize("B", [64, 1024, 1025, 2100])
def test_many_sequences(torch_cuda, B):
    torch = torch_cuda
    rng = np.random.default_rng(B)
    lengths = [int(v) for v in rng.integers(0, 90, size=B)]
    c = _cache(torch, rng, "bf16", lengths, 1, 64, 8, 96)
    q = _normal(torch, rng, "bf16", B, 2, 64)
    kern = _kern()
    b = kern.PageBounds(c)
    got, chosen = kern.block_attention(q, c, b, 5, 1, 2)
    want = choose_ref(_np(q), c, _np(b.lo), _np(b.hi), 5, 1, 2)
    assert np.array_equal(chosen.cpu().numpy(), want)
    out, tol, _, _ = paged_ref(_np(q), c, None, 0, "bf16", want)
    _close(_np(got), out, tol)


@pytest.mark.parametrize("bits", ["bf16", "bf16/4"])
def test_steps_captured_in_a_graph(torch_cuda, bits):
    """A captured step (rotated append, bounds, block attention, eviction,
    bounds), replayed several times with eager work in between, equals eager
    steps of a second cache."""
    torch = torch_cuda
    kern = _kern()
    a, b = (make(torch, np.random.default_rng(12), bits, [64, 80, 3], 2, 64, 16, 96, evicted=True)
            for _ in range(2))
    rng = np.random.default_rng(13)
    q, k, v = (_normal(torch, rng, "bf16", 3, h, 64) for h in (4, 2, 2))
    freq = torch.rand(32, device="cuda")
    drop = torch.tensor([0, 1, 0], dtype=torch.int32, device="cuda")
    ba, bb = kern.PageBounds(a), kern.PageBounds(b)

    def step(c, bounds):
        tq, _ = kern.cache_append_rotary(c, q, k, v, freq, drop=drop)
        bounds.update(1)
        out, chosen = kern.block_attention(tq, c, bounds, 3, 1, 1)
        dense = kern.paged_attention(tq, c, 60, 2)
        src = kern.cache_evict(c, 64, 2, 4)
        bounds.update()
        return tq, out, chosen, dense, src

    want = step(b, bb)
    state = [t.clone() for t in a._tensors]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(a, ba)
    assert all(torch.equal(x, y) for x, y in zip(a._tensors, state))  # capture runs nothing
    for replay in range(4):
        if replay:
            for t, h in ((q, 4), (k, 2), (v, 2)):
                t.copy_(_normal(torch, rng, "bf16", 3, h, 64))
            want = step(b, bb)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want)), replay
        assert all(torch.equal(x, y) for x, y in zip(a._tensors, b._tensors)), replay
        assert torch.equal(ba.lo, bb.lo) and torch.equal(ba.hi, bb.hi), replay


def test_side_streams_record_their_tensors(torch_cuda, monkeypatch):
    """Tensors of another stream are recorded; two streams at once with a
    cache each give what one after the other gives."""
    torch = torch_cuda
    used = set()
    record = torch.Tensor.record_stream
    monkeypatch.setattr(torch.Tensor, "record_stream",
                        lambda t, s: (used.add((t.data_ptr(), s.cuda_stream)), record(t, s))[1])
    kern = _kern()
    made = []
    for bits in ("bf16/4", "bf16/4", "bf16/4"):
        rng = np.random.default_rng(13)
        c = make(torch, rng, bits, [500, 60], 2, 64, 16, 600)
        made.append((c, kern.PageBounds(c), torch.linspace(0, 1, 32, device="cuda"),
                     *(_normal(torch, rng, "bf16", 2, h, 64) for h in (4, 2, 2))))

    def steps(c, b, freq, q, k, v):
        outs = []
        for _ in range(5):
            outs.append(kern.cache_append_rotary(c, q, k, v, freq)[0])
            b.update(1)
            outs += kern.block_attention(q, c, b, 7)
        return outs

    want = steps(*made[0])
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for s, m in zip(streams, made[1:]):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append(steps(*m))
    torch.cuda.synchronize()
    for outs, s, m in zip(got, streams, made[1:]):
        assert all(torch.equal(x, y) for x, y in zip(outs, want))
        assert {(t.data_ptr(), s.cuda_stream) for t in (*m[0]._tensors, m[1].lo, m[1].hi, *m[2:])} <= used


def test_refusals(torch_cuda):
    torch = torch_cuda
    kern = _kern()
    rng = np.random.default_rng(14)
    c = _cache(torch, rng, "bf16", [20, 5], 2, 64, 16, 32)
    other = _cache(torch, rng, "bf16", [20, 5], 2, 64, 16, 32)
    q = _normal(torch, rng, "bf16", 2, 4, 64)
    b = kern.PageBounds(c)
    lo = b.lo
    for call in [
        lambda: kern.PageBounds(c, lo), lambda: kern.PageBounds(c, lo, lo.float()),
        lambda: kern.PageBounds(c, lo, lo[:1]), lambda: kern.PageBounds(c, lo.cpu(), lo),
        lambda: kern.PageBounds(c, lo, lo.transpose(0, 1)),
        lambda: kern.PageBounds(c, lo.clone().requires_grad_(), lo),
        lambda: b.update(0), lambda: b.update(1.5), lambda: b.update(-1),
        lambda: kern.block_attention(q, other, b, 2), lambda: kern.block_attention(q, c, lo, 2),
        lambda: kern.block_attention(q, c, b, 0), lambda: kern.block_attention(q, c, b, 2, 2),
        lambda: kern.block_attention(q, c, b, 2, 0, 0), lambda: kern.block_attention(q, c, b, 2, -1),
        lambda: kern.block_attention(q, c, b, 2.5), lambda: kern.block_attention(q, c, b, (1 << 30) + 1),
        lambda: kern.block_attention(q[:1], c, b, 2), lambda: kern.block_attention(q.float(), c, b, 2),
        lambda: kern.block_attention(q, c, b, 2, out=q[:, :2]),
        lambda: kern.block_attention(q, c, b, 2, out=q), lambda: kern.PageBounds(c, lo, lo),
        lambda: kern.block_attention(q, c, b, 2, out=lo.view(-1)[:512].view(2, 4, 64)),
        lambda: kern.block_attention(q.clone().requires_grad_(), c, b, 2),
    ]:
        with pytest.raises(ValueError):
            call()
    with pytest.raises(kern._native.FusionError):
        kern.block_attention(_normal(torch, rng, "bf16", 2, 3, 64), c, b, 2)

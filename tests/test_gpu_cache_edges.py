"""Windowed attention and token caches at their edges: slots without a page, values
that are infinite or NaN and are seen.  Helpers and tolerances are those of
test_gpu_cache.py."""
import numpy as np
import pytest

from test_gpu_cache import (_cache, _close, _kern, _normal, _np, _paged_ref, _rows,  # noqa: F401
                            _window_ref, torch_cuda)

pytestmark = pytest.mark.gpu


# ------------------------------------------------------- slots without a page --
def _stored(cache):
    """Whether each slot's page is there, [batch, capacity]."""
    t = cache.table.cpu().numpy()
    return np.repeat((t >= 0) & (t < cache.k.shape[0]), cache.k.shape[1], 1)


PAGELESS = [  # lengths, capacity, page, budget, sinks, recent, (sequence, pages) without a page
    ([100, 90, 100, 70], 128, 16, 64, 2, 20, [(0, [6]), (1, [5]), (2, [4, 5, 6, 7]), (3, [4])]),
    ([1500, 1100], 1504, 16, 1024, 4, 200, [(0, [80, 93]), (1, [66, 68])]),
    ([20000, 16500], 20000, 64, 16384, 0, 64, [(0, [300, 312]), (1, [257])]),
    ([90, 33], 96, 27, 33, 0, 0, [(0, [1, 2]), (1, [1])]),
]


@pytest.mark.parametrize("case", range(len(PAGELESS)))
def test_cache_evict_drops_tokens_that_are_stored_nowhere(torch_cuda, case):
    """A token in a slot past the budget that has no page has no keys: it
    leaves, whatever its weight and position, and no other token's keys are
    taken for its own."""
    torch = torch_cuda
    lengths, cap, page, budget, sinks, recent, missing = PAGELESS[case]
    print(f"[evict] {PAGELESS[case]}", flush=True)
    rng = np.random.default_rng(300 + case)
    dtype = "bf16" if case % 2 else "fp32"
    c = _cache(torch, rng, dtype, lengths, 2, 24, page, cap)
    for b, pages in missing:
        for i, p in enumerate(pages):
            c.table[b, p] = c.k.shape[0] if i % 2 else -1
    stored, w, pos = _stored(c), _np(c.weight), c.pos.cpu().numpy()
    w[~stored] = 1e6
    c.weight.copy_(torch.from_numpy(w))
    w, seen = _np(c.weight), c.seen.cpu().numpy()
    before = [_rows(c, b, n)[:2] for b, n in enumerate(lengths)]
    got = _kern().cache_evict(c, budget, sinks, recent).cpu().numpy()
    for b, n in enumerate(lengths):
        want = np.arange(budget)
        want[n:] = -1
        if n > budget:
            x = np.arange(n)
            safe = (pos[b, :n] < sinks) | (pos[b, :n] >= seen[b] - recent)
            lost = (x >= budget) & ~stored[b, :n]
            order = np.lexsort((x, np.where(safe, 0, -w[b, :n]), ~safe, lost))
            keep = np.sort(order[:budget])
            want[np.setdiff1d(np.arange(budget), keep)] = keep[keep >= budget]
        assert np.array_equal(got[b], want), b
        m = min(n, budget)
        assert np.array_equal(_np(c.weight)[b, :m], w[b, want[:m]])
        k, v, here = _rows(c, b, m)
        assert np.array_equal(k[here], before[b][0][want[:m]][here])
        assert np.array_equal(v[here], before[b][1][want[:m]][here])
    q = _normal(torch, rng, dtype, len(lengths), 4, 24)
    out, tol, _, _ = _paged_ref(_np(q), c, None, 0, dtype)
    _close(_np(_kern().paged_attention(q, c)), out, tol)


# -------------------------------------------- seen values that are not finite --
def _with_values(out, tol, special, got):
    """Rows that see infinities and NaN have their sum (weights are positive),
    the others the finite answer.  special: sum of those values, 0 where none."""
    odd = special != 0
    assert odd.any() and not odd.all()
    assert np.array_equal(got[odd], special[odd], equal_nan=True)
    _close(np.where(odd, 0, got), np.where(odd, 0, out), tol)


def _shares_keys(dtype, lengths, hq, hkv, dh, window, causal):
    """Which of the two kernels a call takes (share_keys in window.hip)."""
    group = hq // hkv
    hshift = 2 if group % 4 == 0 else 1 if group % 2 == 0 else 0
    rows, parts = (32 if dtype == "bf16" else 16) * (4 >> hshift), 4 if dh <= 64 else 2
    groups, longest = sum(-(-n // rows) for n in lengths) * (hq >> hshift), max(lengths)
    return groups * parts <= 512 or (causal and longest >= 5 * groups and
                                     groups * longest <= 400 * min(window or 1 << 30, longest))


def _copies(shared, dtype, lengths, hq, hkv, dh, window, causal):
    """How often to repeat the samples so that the call's waves share the keys
    of a row tile, or do not."""
    for n in range(1, 400):
        if _shares_keys(dtype, lengths * n, hq, hkv, dh, window, causal) == shared:
            return n
    raise AssertionError("no such call")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hq,hkv,dh", [(2, 2, 64), (8, 2, 72), (4, 2, 128)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("shared", [True, False])
def test_window_attention_seen_infinities_and_nan(torch_cuda, dtype, hq, hkv, dh, causal, shared):
    """Infinities and NaN reach every row that sees them and no other, whether
    all rows of a tile see them or some, and also where the weight is below
    what fp32 holds."""
    torch = torch_cuda
    rng = np.random.default_rng(hq + dh + causal)
    lengths = [200, 0, 130]
    cu1 = np.array([0, 200, 200, 330])
    q, k, v = (_normal(torch, rng, dtype, 330, h, dh) for h in (hq, hkv, hkv))
    size = torch.ones(330, device="cuda")
    size[250] = 0
    for row, value in ((1, "inf"), (5, "-inf"), (77, "inf"), (130, "nan"), (250, "nan"), (328, "-inf")):
        v[row, :, row % 3::7] = float(value)
    vn = _np(v)
    i = np.arange(330)
    for scale in (1, 12):  # 12: scores of hundreds, most weights underflow
        for window, sinks in ((20, 3), (100, 0), (None, 0)):
            see = np.abs(i[:, None] - i) < (window or 1000)
            see |= (i < sinks) | ((i >= 200) & (i < 200 + sinks))
            if causal:
                see &= i <= i[:, None]
            see &= ((i >= 200)[:, None] == (i >= 200)) & (i != 250)
            special = np.zeros((330, hq, dh))
            with np.errstate(invalid="ignore"):
                for row in np.flatnonzero(~np.isfinite(vn).all((1, 2))):
                    special[see[:, row]] += np.where(np.isfinite(vn[row]), 0, vn[row]).repeat(hq // hkv, 0)
            vz = np.where(np.isfinite(vn), vn, 0)
            n = _copies(shared, dtype, lengths, hq, hkv, dh, window, causal)
            out, tol = _window_ref(_np(q * scale), _np(k * scale), vz, cu1, window, sinks, causal,
                                   _np(size), dtype)
            cu = np.concatenate([[0], np.cumsum(lengths * n)])
            got = _kern().window_attention((q * scale).repeat(n, 1, 1), (k * scale).repeat(n, 1, 1),
                                           v.repeat(n, 1, 1), cu, window, sinks, causal, size.repeat(n))
            got = _np(got).reshape(n, 330, hq, dh)
            assert np.array_equal(got, np.broadcast_to(got[:1], got.shape), equal_nan=True)
            _with_values(out, tol, special, got[0])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hq,hkv,dh", [(2, 2, 64), (8, 2, 72), (4, 1, 128)])
@pytest.mark.parametrize("evicted", [True, False])
def test_paged_attention_seen_infinities_and_nan(torch_cuda, dtype, hq, hkv, dh, evicted):
    """Infinities and NaN among the cached values reach the output of a sequence
    that sees them and no other, in sequences of one part and of many, and also
    where their weight is below what fp32 holds."""
    torch = torch_cuda
    rng = np.random.default_rng(hq + dh + evicted)
    c = _cache(torch, rng, dtype, [5000, 1, 77, 0, 300], hkv, dh, 16, 5008, evicted=evicted)
    c.table[4, 3] = -1
    for b, x, value in ((0, 3, "inf"), (0, 2500, "inf"), (0, 4990, "-inf"), (1, 0, "inf"), (2, 40, "nan"),
                        (2, 70, "-inf"), (4, 50, "nan"), (4, 1, "-inf"), (4, 299, "inf")):
        page = int(c.table[b, x // 16])
        if page >= 0:
            c.v[page, x % 16, :, x % 3::7] = float(value)
    clean = c.v.nan_to_num(0, 0, 0)
    pos, seen = c.pos.cpu().numpy(), c.seen.cpu().numpy()
    q1 = _normal(torch, rng, dtype, 5, hq, dh)
    for scale in (1, 40):
        q = q1 * scale
        for window, sinks in ((None, 0), (60, 2), (3000, 0)):
            z = _kern().TokenCache(c.k, clean, c.table, c.length, c.seen, c.weight.clone(), c.pos)
            out, tol, add, add_tol = _paged_ref(_np(q), z, window, sinks, dtype)
            special = np.zeros(out.shape)
            with np.errstate(invalid="ignore"):
                for b in range(5):
                    n = int(c.length[b])
                    _, v, see = _rows(c, b, n)
                    if window:
                        see = see & ((pos[b, :n] > seen[b] - 1 - window) | (pos[b, :n] < sinks))
                    for x in np.flatnonzero(see & ~np.isfinite(v).all((1, 2))):
                        special[b] += np.where(np.isfinite(v[x]), 0, v[x]).repeat(hq // hkv, 0)
            d = _kern().TokenCache(c.k, c.v, c.table, c.length, c.seen, c.weight.clone(), c.pos)
            _with_values(out, tol, special, _np(_kern().paged_attention(q, d, window, sinks)))
            # what a token draws does not depend on its values
            _kern().paged_attention(q, z, window, sinks)
            assert torch.equal(d.weight, z.weight)


# ------------------------------------------------ more work than one launch holds --
def test_window_attention_of_more_workgroups_than_a_launch(torch_cuda):
    """140,000 rows of 4,096 narrow heads: each head equals the same head in a
    call of few heads."""
    torch = torch_cuda
    torch.manual_seed(1)
    rows, heads, dh = 140_000, 4096, 8
    print(f"[window] {rows} rows, {heads} heads of {dh}", flush=True)
    q = torch.randn(rows, heads, dh, dtype=torch.bfloat16, device="cuda")
    k, v = (torch.randn(rows, 1, dh, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cu = [0, 1, 70_001, rows]
    got = _kern().window_attention(q, k, v, cu, 3, 1)
    for h in range(0, heads, 1020):
        assert torch.equal(got[:, h:h + 16], _kern().window_attention(q[:, h:h + 16], k, v, cu, 3, 1)), h


def test_cache_append_of_more_rows_than_a_launch(torch_cuda):
    """2^26 rows and a few more, a wave each."""
    torch = torch_cuda
    torch.manual_seed(2)
    n = [(1 << 26) - 9, 40]
    print(f"[append] {n}", flush=True)
    c = _kern().TokenCache.empty(2, 1 << 26, 1, 8, page_size=1024)
    k, v = (torch.randn(sum(n), 1, 8, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    _kern().cache_append(c, k, v, [0, n[0], sum(n)])
    assert c.length.tolist() == n and c.seen.tolist() == n
    for b, first in enumerate((0, n[0])):
        for have, new in ((c.k, k), (c.v, v)):
            assert torch.equal(have.view(2, -1, 1, 8)[b, :n[b]], new[first:first + n[b]])
        assert torch.equal(c.pos[b, :n[b]], torch.arange(n[b], dtype=torch.int32, device="cuda"))


def test_paged_attention_of_more_workgroups_than_a_launch(torch_cuda):
    """65,536 sequences with 512 heads of their own: each sequence equals the
    same one in a call of few."""
    torch = torch_cuda
    torch.manual_seed(3)
    B, heads, dh = 65_536, 512, 8
    print(f"[paged] {B} sequences, {heads} heads of {dh}", flush=True)
    k, v = (torch.randn(4, 16, heads, dh, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.randn(B, heads, dh, dtype=torch.bfloat16, device="cuda")
    table = torch.arange(B, dtype=torch.int32, device="cuda").view(B, 1) % 4
    length = torch.randint(0, 17, (B,), dtype=torch.int32, device="cuda")
    weight, pos = torch.zeros(B, 16, device="cuda"), torch.arange(16, dtype=torch.int32, device="cuda").repeat(B, 1)
    whole = _kern().TokenCache(k, v, table, length, length.clone(), weight, pos)
    got = _kern().paged_attention(q, whole)
    for b in range(0, B, 13_000):
        s = slice(b, b + 1500)
        w = torch.zeros(len(q[s]), 16, device="cuda")
        part = _kern().TokenCache(k, v, table[s], length[s], length[s].clone(), w, pos[s])
        assert torch.equal(got[s], _kern().paged_attention(q[s], part)), b
        assert torch.equal(weight[s], w), b


# ------------------------------------------------------------- NaN all over --
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dh", [64, 72])
def test_nan_queries_and_rows_of_nan(torch_cuda, dtype, dh):
    """A query that is NaN gives NaN for itself alone; a row of values that is
    NaN throughout gives NaN to what sees it, beside infinities too."""
    torch = torch_cuda
    rng = np.random.default_rng(dh)
    kern = _kern()
    c = _cache(torch, rng, dtype, [700, 3, 1200, 0], 2, dh, 16, 1200)
    q = _normal(torch, rng, dtype, 4, 6, dh)
    want = kern.paged_attention(q, c, accumulate=False)
    bad = q.clone()
    bad[0, 3], bad[1] = float("nan"), float("nan")
    got = kern.paged_attention(bad, c, accumulate=False)
    assert got[0, 3].isnan().all() and got[1].isnan().all()
    ok = torch.ones(4, 6, dtype=torch.bool, device="cuda")
    ok[0, 3], ok[1] = False, False
    assert torch.equal(got[ok], want[ok])
    v = c.v.clone()
    v[int(c.table[2, 40]), 5] = float("nan")
    v[int(c.table[2, 70]), 5, :, ::2] = float("inf")
    d = kern.TokenCache(c.k, v, *c._tensors[2:])
    got = kern.paged_attention(q, d, accumulate=False)
    assert got[2].isnan().all() and torch.equal(got[[0, 1, 3]], want[[0, 1, 3]])

    q, k, v = (_normal(torch, rng, dtype, 300, h, dh) for h in (4, 2, 2))
    want = kern.window_attention(q, k, v, [0, 300], 90, 1)
    q[7, 1] = float("nan")
    v[150] = float("nan")
    v[160, :, ::2] = float("inf")
    got = kern.window_attention(q, k, v, [0, 300], 90, 1)
    odd = torch.zeros(300, 4, dtype=torch.bool, device="cuda")
    odd[7, 1], odd[150:240] = True, True
    assert got[odd].isnan().all()
    odd[240:250] = True
    assert bool((got[240:250, :, ::2] == float("inf")).all())
    assert torch.equal(got[~odd], want[~odd])

"""Token caches at their edges: slots without a page.  Helpers and tolerances are
those of test_gpu_cache.py."""
import numpy as np
import pytest

from test_gpu_cache import (_cache, _close, _kern, _normal, _np, _paged_ref, _rows,  # noqa: F401
                            torch_cuda)

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

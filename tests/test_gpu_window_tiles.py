"""Windowed attention on both sides of the rule that chooses between waves with
a row tile each and waves that share one's keys (share_keys in window.hip,
mirrored by _shares_keys): each case asserts which side it takes, so that a
change of the rule cannot leave a kernel without tests.  Helpers and tolerances
are those of test_gpu_cache.py."""
import numpy as np
import pytest

from test_gpu_cache import _close, _kern, _normal, _np, _window_ref, torch_cuda  # noqa: F401
from test_gpu_cache_edges import _copies, _shares_keys

pytestmark = pytest.mark.gpu

MANY = [  # lengths, heads, kv_heads, dh, window, sinks, causal, sizes: a row tile for each wave
    ([577, 300, 1, 0, 129, 250], 32, 8, 128, 100, 4, True, False),
    ([577, 300, 1, 0, 129, 250], 32, 8, 128, 100, 1, False, True),
    ([600, 500, 300, 40], 32, 8, 128, None, 0, True, False),
    ([1100, 500, 64, 65], 24, 12, 128, 300, 70, False, False),
    ([900, 800, 5], 20, 20, 128, 130, 2, True, False),
    ([1100, 500, 64, 65], 24, 12, 96, 130, 3, False, True),
    ([900, 800, 5], 20, 20, 80, 70, 1, True, False),
    ([600, 500, 300, 40], 32, 4, 104, 257, 0, True, True),
    ([577, 290, 200, 130], 12, 12, 64, 97, 1, False, True),
    ([577, 290, 200, 130], 12, 12, 64, 97, 1, False, False),
    ([500, 333, 1, 0, 64, 129], 16, 4, 64, 64, 0, True, False),
    ([500, 333, 1, 0, 64, 229], 16, 8, 64, 150, 9, True, True),
    ([400, 300, 200, 31, 33], 16, 16, 40, 33, 0, True, False),
    ([400, 300, 200, 31, 33], 18, 9, 24, None, 0, False, True),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", range(len(MANY)))
def test_window_attention_of_many_row_tiles(torch_cuda, case, dtype):
    torch = torch_cuda
    lengths, hq, hkv, dh, window, sinks, causal, sizes = MANY[case]
    print(f"[window] {dtype} {MANY[case]}", flush=True)
    assert not _shares_keys(dtype, lengths, hq, hkv, dh, window, causal)
    rng = np.random.default_rng(400 + case)
    cu = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    M = int(cu[-1])
    qkv = _normal(torch, rng, dtype, M, hq + 2 * hkv, dh)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    size = None
    if sizes:  # some tokens hidden, of the last sample all
        size = rng.integers(0, 5, size=M).astype(np.float32)
        size[cu[-2]:] = 0
    dsize = None if size is None else torch.from_numpy(size).cuda()
    got = _kern().window_attention(q, k, v, cu, window, sinks, causal, dsize)
    ref, tol = _window_ref(_np(q), _np(k), _np(v), cu, window, sinks, causal, size, dtype)
    _close(_np(got), ref, tol)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hq,hkv,dh", [(1, 1, 64), (1, 1, 128), (2, 1, 96), (4, 1, 128), (4, 1, 64)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("shared", [True, False])
def test_window_attention_ends_within_tiles_of_both_kernels(torch_cuda, dtype, hq, hkv, dh, causal, shared):
    """Windows and first rows that end at, before and after parts of tiles; the
    samples repeated until the call takes the kernel that is meant."""
    torch = torch_cuda
    rng = np.random.default_rng(hq + dh + causal)
    lengths = [197, 33]
    q, k, v = (_normal(torch, rng, dtype, 230, h, dh) for h in (hq, hkv, hkv))
    for window in (2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 95, 96, 97, 128, 129):
        for sinks in (0, 1, 16, 33):
            n = _copies(shared, dtype, lengths, hq, hkv, dh, window, causal)
            cu = np.concatenate([[0], np.cumsum(lengths * n)])
            got = _kern().window_attention(*(t.repeat(n, 1, 1) for t in (q, k, v)), cu, window, sinks, causal)
            got = got.view(n, 230, hq, dh)
            assert torch.equal(got, got[:1].expand(n, -1, -1, -1)), (window, sinks)
            ref, tol = _window_ref(_np(q), _np(k), _np(v), np.array([0, 197, 230]), window, sinks, causal,
                                   None, dtype)
            _close(_np(got[0]), ref, tol, (window, sinks))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hq,hkv,dh", [(2, 2, 64), (8, 2, 72), (4, 2, 128)])
@pytest.mark.parametrize("causal", [True, False])
def test_window_attention_unseen_values_have_no_influence_on_many_row_tiles(torch_cuda, dtype, hq, hkv, dh,
                                                                            causal):
    """Infinities and NaN, in keys too, in rows that a query does not see leave
    its output bit for bit, where each wave has a row tile."""
    torch = torch_cuda
    rng = np.random.default_rng(hq + dh + causal)
    lengths, rows, window, sinks = [200, 130], 330, 20, 3
    n = _copies(False, dtype, lengths, hq, hkv, dh, window, causal)
    cu = np.concatenate([[0], np.cumsum(lengths * n)])
    q, k, v = (_normal(torch, rng, dtype, rows * n, h, dh) for h in (hq, hkv, hkv))
    size = torch.ones(rows * n, device="cuda")
    size[250] = 0
    want = _kern().window_attention(q, k, v, cu, window, sinks, causal, size)
    i = np.arange(rows * n)
    for bad in (5, 77, 130, 250):
        for value in (float("nan"), float("inf"), -float("inf")):
            kb, vb = k.clone(), v.clone()
            kb[bad], vb[bad] = value, value
            vb[bad, :, ::3] = -value
            got = _kern().window_attention(q, kb, vb, cu, window, sinks, causal, size)
            start = 0 if bad < 200 else 200
            same = (i >= start) & (i < (200 if bad < 200 else rows))
            near = (i - bad < window) & (i >= bad) if causal else np.abs(i - bad) < window
            clean = torch.from_numpy(~same | ~near | (bad == 250)).cuda()
            assert torch.equal(got[clean], want[clean]), (bad, value)

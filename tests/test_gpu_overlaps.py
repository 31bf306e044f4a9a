"""Calls on token caches refuse tensors that are written and overlap others, and
leave everything as it was (GPU)."""
import numpy as np
import pytest

from test_gpu_cache import _cache, _kern, _normal, torch_cuda  # noqa: F401
from test_gpu_cache4 import cache4

pytestmark = pytest.mark.gpu


def bytes_of(t):
    """A tensor's whole storage."""
    import torch
    return torch.tensor([], dtype=torch.uint8, device=t.device).set_(t.untyped_storage())


def over(t, dtype, *shape):
    """A tensor over another's memory, from its first byte on."""
    n = int(np.prod(shape)) * dtype.itemsize
    b = bytes_of(t)
    return b[:n].view(dtype).view(shape) if len(b) >= n else None


def refuses(c, calls):
    state = [t.clone() for t in c._tensors]
    for call in calls:
        with pytest.raises((ValueError, _kern()._native.FusionError), match="overlap"):
            call()
    assert all(bool((a == b).all()) for a, b in zip(c._tensors, state))


def caches(torch):
    rng = np.random.default_rng(31)
    # (pages enough for bounds to fit into the scales)
    for make in (_cache, cache4):
        c = make(torch, rng, "bf16", [200, 250], 2, 64, 64, 2048)
        yield c, rng


def test_page_bounds(torch_cuda):
    torch = torch_cuda
    for c, rng in caches(torch):
        P = c.k.shape[0]
        free = torch.zeros((P, 2, 64), dtype=torch.bfloat16, device="cuda")
        bad = [t for t in (over(t, c.dtype, P, 2, 64) for t in c._tensors) if t is not None]
        assert len(bad) == (4 if c.k.dtype == torch.uint8 else 2)
        refuses(c, [lambda t=t: _kern().PageBounds(c, t, free) for t in bad])
        refuses(c, [lambda t=t: _kern().PageBounds(c, free, t) for t in bad])
        refuses(c, [lambda: _kern().PageBounds(c, free, free)])
        _kern().PageBounds(c, free, free.clone()).update()


def test_block_attention(torch_cuda):
    torch = torch_cuda
    kern = _kern()
    for c, rng in caches(torch):
        q, bounds = _normal(torch, rng, "bf16", 2, 4, 64), kern.PageBounds(c)
        want, _ = kern.block_attention(q, c, bounds, 2)
        bad = [t for t in (over(t, c.dtype, 2, 4, 64) for t in (*c._tensors, q, bounds.lo, bounds.hi))
               if t is not None]
        refuses(c, [lambda t=t: kern.block_attention(q, c, bounds, 2, out=t) for t in bad])
        out = torch.empty_like(want)
        assert kern.block_attention(q, c, bounds, 2, out=out)[0] is out and torch.equal(out, want)


def test_turned_queries(torch_cuda):
    torch = torch_cuda
    call = _kern().cache_append_rotary
    for c, rng in caches(torch):
        q, k, v = (_normal(torch, rng, "bf16", 2, h, 64) for h in (4, 2, 2))
        freq = torch.rand(512, device="cuda")[:32]
        drop = torch.zeros(512, dtype=torch.int32, device="cuda")[:2]
        bad = [t for t in (over(t, c.dtype, 2, 4, 64) for t in (*c._tensors, freq, drop, q)) if t is not None]
        refuses(c, [lambda t=t: call(c, q, k, v, freq, drop=drop, out=t) for t in bad])
        out = torch.empty_like(q)
        assert call(c, q, k, v, freq, drop=drop, out=out)[0] is out


def test_rows_of_an_append(torch_cuda):
    """Rows from the cache's own memory; all of a sequence's tokens dropped by its length."""
    torch = torch_cuda
    call = _kern().cache_append_rotary
    for c, rng in caches(torch):
        rows = [_normal(torch, rng, "bf16", 2, h, 64) for h in (4, 2, 2)]
        freq, calls = torch.rand(32, device="cuda"), []
        written = [t for t in c._tensors if t is not c.table]
        for t in written:
            for i, h in enumerate((4, 2, 2)):
                bad = over(t, c.dtype, 2, h, 64)
                if bad is not None:
                    calls.append(lambda i=i, bad=bad: call(c, *rows[:i], bad, *rows[i + 1:], freq))
            bad = over(t, torch.float32, 32)
            if bad is not None:
                calls.append(lambda bad=bad: call(c, *rows, bad))
            if t is not c.length and t is not c.seen:
                calls.append(lambda t=t: call(c, *rows, freq, drop=over(t, torch.int32, 2)))
            if c.k.dtype == torch.uint8 and t.nbytes >= 512:
                calls.append(lambda t=t: _kern().cache_append(c, over(t, c.dtype, 2, 2, 64), rows[2]))
        assert len(calls) >= 20
        refuses(c, calls)
        for counts in ([0, 1, 2], [0, 20, 70]):
            want = [call(x, *(t.repeat(35, 1, 1)[:counts[-1]] for t in rows), freq, counts, drop=d)[0]
                    for x, d in ((c, c.length), (c, c.seen))]
            assert torch.equal(*want)
            assert c.length.tolist() == c.seen.tolist() == np.diff(counts).tolist()

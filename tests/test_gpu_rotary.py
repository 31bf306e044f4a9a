"""kernels.cache_append_rotary against plain NumPy in 64 bits.

Tolerances.  With u = eps / 2 of the type (bf16 2^-8, fp32 2^-24) and an angle
whose cosine and sine are rounded to fp32, x cos - y sin as a product and a
fused multiply-add has an error of at most 2^-24 (|x cos| + 2 |y sin|) + 2^-24
of the result, so 4 2^-24 (|x| + |y|) covers it, beside u of the result.  The
angle itself is the same product of 64 bits on both sides, and its reduction is
off by less than 2^-50.  What goes into 4 bits is compared bit by bit with the
rounding of the turned keys that the call gives out."""
import numpy as np
import pytest

from test_gpu_cache import U32, UNIT, _cache, _dt, _kern, _normal, _np, _paged_ref, _close, torch_cuda  # noqa: F401
from test_gpu_cache4 import cache4, paged_ref, quantise

pytestmark = pytest.mark.gpu


def turn(x, pos, freq, pairs):
    """x [rows, heads, dh] turned by positions [rows]: (result, tolerance
    without the rounding to the type)."""
    n = len(freq)
    angle = pos.astype(np.float64)[:, None, None] * freq.astype(np.float32).astype(np.float64)
    c, s = np.cos(angle), np.sin(angle)
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if pairs else (slice(0, n), slice(n, 2 * n))
    out, tol = x.copy(), np.zeros_like(x)
    out[..., a], out[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    tol[..., a] = tol[..., b] = 4 * U32 * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return out, tol


def near(got, want, tol, dtype):
    got = _np(got)
    assert np.isfinite(got).all()
    worst = (np.abs(got - want) - tol - UNIT[dtype] * np.abs(want)).max(initial=-1.0)
    assert worst <= 0, worst


ROTARY = [  # counts (None: one each), heads, kv_heads, dh, n, pairs, drop
    (None, 6, 6, 64, 32, False, None),
    (None, 5, 1, 128, 64, False, [1, 0, 3, 96, 200, -4]),
    ([1, 0, 8, 3, 0, 5], 8, 2, 96, 48, False, [1, 5, 8, 3, 0, 5]),
    ([1, 0, 8, 3, 0, 5], 4, 4, 32, 8, True, None),
    ([0, 3, 40, 1, 200, 7], 4, 2, 64, 16, True, [0, 3, 40, 1, 20, 7]),
    ([70, 0, 0, 0, 0, 33], 12, 3, 128, 20, False, None),
    ([9, 1, 0, 0, 2, 0], 3, 3, 96, 4, False, None),
    ([9, 1, 0, 0, 2, 0], 2, 1, 64, 0, False, [5, 5, 5, 5, 5, 5]),
    ([0, 0, 0, 0, 0, 0], 2, 1, 64, 32, False, [1, 2, 3, 0, 90, 1]),
    (None, 0, 2, 64, 32, True, None),
    (None, 3, 3, 40, 20, False, None),
    ([2, 1, 0, 7, 1, 3], 4, 2, 72, 36, False, [0, 1, 2, 3, 4, 5]),
    ([0, 12, 1, 1, 9, 0], 2, 1, 8, 4, True, None),
    ([0, 12, 1, 1, 9, 0], 5, 5, 120, 28, True, [0, 5, 0, 0, 30, 0]),
]


@pytest.mark.parametrize("bits", ["bf16", "fp32", "bf16/4", "fp32/4"])
@pytest.mark.parametrize("case", range(len(ROTARY)))
def test_append_rotary(torch_cuda, case, bits):
    """Ragged rows, none, more than fit, replaced tokens, pages that are not
    there, positions that are not slots."""
    torch = torch_cuda
    counts, hq, hkv, dh, n, pairs, drop = ROTARY[case]
    dtype, four = bits.split("/")[0], "/" in bits
    if four and dh % 32:
        pytest.skip("4 bits hold blocks of 32 dims")
    print(f"[rotary] {bits} {ROTARY[case]}", flush=True)
    rng = np.random.default_rng(600 + case)
    lengths, seen = [0, 5, 60, 96, 30, 95], [0, 50, 60, 200, 30, (1 << 31) - 400]
    make = cache4 if four else _cache
    c = make(torch, rng, dtype, lengths, hkv, dh, 27, 100, seen=seen)
    c.table[2, 3] = -1
    c.table[4, 2] = c.k.shape[0]
    m = np.ones(6, int) if counts is None else np.array(counts)
    rows = int(m.sum())
    extra = 0 if counts is None else 2
    qkv = _normal(torch, rng, dtype, rows + extra, hq + 2 * hkv, dh)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    freq = (10000.0 ** (-np.arange(n) / max(n, 1))).astype(np.float32)
    names = ("k", "v", "weight", "pos", "length", "seen") + (("k_scale", "v_scale") if four else ())
    want = {x: (_np(getattr(c, x)) if x in "kv" and not four else getattr(c, x).cpu().numpy().copy())
            for x in names}
    cu = None if counts is None else np.concatenate([[0], np.cumsum(m)])
    d = None if drop is None else torch.tensor(drop, dtype=torch.int32, device="cuda")
    got_q, got_k = _kern().cache_append_rotary(c, q, k, v, torch.from_numpy(freq).cuda(), cu, pairs, d,
                                               rotated_k=True)
    assert got_q.is_contiguous() and got_q.shape == q.shape and got_k.shape == k.shape
    assert not got_q[rows:].any() and not got_k[rows:].any()
    at, r, table = np.zeros(rows, np.int64), 0, c.table.cpu().numpy()
    new_k = _np(got_k[:rows])
    if four:
        new_k, new_v = quantise(new_k), quantise(_np(v[:rows]))
    else:
        new_v = _np(v[:rows])
    for b in range(6):
        less = 0 if drop is None else min(max(drop[b], 0), lengths[b])
        want["length"][b] -= less
        want["seen"][b] -= less
        base = int(want["seen"][b])
        for i in range(m[b]):
            x = int(want["length"][b])
            at[r] = base + i
            if x < c.capacity:
                want["weight"][b, x], want["pos"][b, x] = 0, at[r]
                p = table[b, x // 27]
                if 0 <= p < c.k.shape[0]:
                    for t, new in (("k", new_k), ("v", new_v)):
                        if four:
                            want[t][p, x % 27] = new[0][r, :, ::2] | new[0][r, :, 1::2] << 4
                            want[t + "_scale"][p, x % 27] = new[1][r]
                        else:
                            want[t][p, x % 27] = new[r]
                want["length"][b] += 1
                want["seen"][b] += 1
            r += 1
    near(got_q[:rows], *turn(_np(q[:rows]), at, freq, pairs), dtype)
    near(got_k[:rows], *turn(_np(k[:rows]), at, freq, pairs), dtype)
    for x in want:
        have = getattr(c, x)
        have = _np(have) if x in "kv" and not four else have.cpu().numpy()
        assert np.array_equal(have, want[x]), x


@pytest.mark.parametrize("bits", ["fp32", "bf16/4"])
def test_far_positions(torch_cuda, bits):
    """Angles of up to 2^31 radians, where 32 bits hold no part of a turn."""
    torch = torch_cuda
    dtype, four = bits.split("/")[0], "/" in bits
    rng = np.random.default_rng(1)
    seen = [0, 1 << 20, (1 << 30) + 12345, (1 << 31) - 2]
    c = (cache4 if four else _cache)(torch, rng, dtype, [0] * 4, 1, 64, 16, 32, seen=seen)
    q, k = _normal(torch, rng, dtype, 4, 3, 64), _normal(torch, rng, dtype, 4, 1, 64)
    freq = np.concatenate([[1.0, 0.7, 3.1e-5, 2.0], rng.uniform(0, 1, 28)]).astype(np.float32)
    got_q, got_k = _kern().cache_append_rotary(c, q, k, k, torch.from_numpy(freq).cuda(), rotated_k=True)
    near(got_q, *turn(_np(q), np.array(seen), freq, False), dtype)
    near(got_k, *turn(_np(k), np.array(seen), freq, False), dtype)


@pytest.mark.parametrize("bits", ["fp32", "bf16/4"])
def test_steep_frequencies(torch_cuda, bits):
    """Angles of up to 2^50 radians are reduced as well as small ones; past it each pair
    turns by whole quarters, and infinite or NaN frequencies give NaN."""
    torch = torch_cuda
    dtype, four = bits.split("/")[0], "/" in bits
    rng = np.random.default_rng(46)
    seen = rng.integers(1 << 30, (1 << 31) - 1, size=96)
    make = cache4 if four else _cache
    freq = (rng.uniform(1, 2, 32) * 2.0 ** np.repeat(np.arange(11, 19), 4)).astype(np.float32)
    freq[31] = 2.0 ** 19
    q, k = _normal(torch, rng, dtype, 96, 3, 64), _normal(torch, rng, dtype, 96, 1, 64)
    call = lambda f: _kern().cache_append_rotary(make(torch, rng, dtype, [0] * 96, 1, 64, 16, 32, seen=seen),
                                                 q, k, k, torch.from_numpy(f).cuda(), rotated_k=True)
    got_q, got_k = call(freq)
    near(got_q, *turn(_np(q), seen, freq, False), dtype)
    near(got_k, *turn(_np(k), seen, freq, False), dtype)
    steep = freq * np.float32(2.0 ** 22)
    for got, x in zip(call(steep), (q, k)):
        x, y = x[..., :32], x[..., 32:]
        quarters = torch.stack([torch.cat(t, -1) for t in ((x, y), (-y, x), (-x, -y), (y, -x))])
        pair = (quarters == got).view(4, *got.shape[:2], 2, 32).all(3)
        assert bool(pair.any(0).all())
    steep[3], steep[7] = np.inf, np.nan
    for got in call(steep):
        bad = torch.isnan(got)
        assert bool(bad[..., [3, 7, 35, 39]].all()) and int(bad.sum()) == 4 * got[..., 0].numel()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_in_one_or_in_steps(torch_cuda, dtype):
    """Turned keys, appended as they are, are what the call itself appends; a
    row's place in the call does not show; prompts in parts are prompts at once."""
    torch = torch_cuda
    rng = np.random.default_rng(2)
    kern = _kern()
    lengths = [70, 1, 33]
    cu = np.concatenate([[0], np.cumsum(lengths)])
    q, k, v = (_normal(torch, rng, dtype, int(cu[-1]), h, 64) for h in (4, 2, 2))
    freq = torch.rand(32, device="cuda")
    for cls in (kern.TokenCache, kern.TokenCache4):
        made = [cls.empty(3, 80, 2, 64, page_size=16, dtype=_dt(torch, dtype)) for _ in range(3)]
        for m in made:  # (what unused slots hold is not compared)
            m.k.zero_(), m.v.zero_()
        tq, tk = kern.cache_append_rotary(made[0], q, k, v, freq, cu, rotated_k=True)
        kern.cache_append(made[1], tk, v, cu)
        for part in (slice(0, 30), slice(30, 31), slice(31, 80)):  # of each sequence
            take = [np.arange(a, b)[part] for a, b in zip(cu[:-1], cu[1:])]
            r = torch.from_numpy(np.concatenate(take)).cuda()
            sub = np.concatenate([[0], np.cumsum([len(t) for t in take])])
            sq, _ = kern.cache_append_rotary(made[2], q[r], k[r], v[r], freq, sub)
            assert torch.equal(sq, tq[r])
        for m in made[1:]:
            for a, b in zip(m._tensors, made[0]._tensors):
                assert torch.equal(a, b)


def test_given_out_strides_and_side_stream(torch_cuda):
    torch = torch_cuda
    rng = np.random.default_rng(3)
    kern = _kern()
    made = []
    for _ in range(2):
        r = np.random.default_rng(4)
        made.append(_cache(torch, r, "bf16", [20, 5], 2, 64, 16, 60))
    base = [_normal(torch, rng, "bf16", h, 12, 64) for h in (4, 2, 2)]
    q, k, v = (t.transpose(0, 1) for t in base)  # heads first
    freq, cu = torch.rand(20, device="cuda"), [0, 4, 9]
    want, _ = kern.cache_append_rotary(made[0], *(t.contiguous() for t in (q, k, v)), freq, cu)
    out = torch.full((12, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got, none = kern.cache_append_rotary(made[1], q, k, v, freq, cu, out=out)
    s.synchronize()
    assert got is out and none is None and torch.equal(out[:9], want[:9]) and bool((out[9:] == 7).all())
    for a, b in zip(made[0]._tensors, made[1]._tensors):
        assert torch.equal(a, b)


@pytest.mark.parametrize("B,most", [(255, 8), (256, 9), (257, 8), (600, 20)])
def test_many_sequences(torch_cuda, B, most):
    """More sequences than one launch describes, few rows each or more."""
    torch = torch_cuda
    rng = np.random.default_rng(B)
    n = rng.integers(0, most + 1, size=B)
    n[3] = most
    lengths = rng.integers(0, 12, size=B)
    drop = rng.integers(0, 4, size=B)
    c = _cache(torch, rng, "fp32", lengths, 1, 16, 16, 32, seen=lengths + 5)
    q, k, v = (_normal(torch, rng, "fp32", int(n.sum()), h, 16) for h in (2, 1, 1))
    cu = np.concatenate([[0], np.cumsum(n)])
    freq = np.linspace(0, 1, 8, dtype=np.float32)
    got, keys = _kern().cache_append_rotary(c, q, k, v, torch.from_numpy(freq).cuda(), cu,
                                            drop=torch.from_numpy(drop).int().cuda(), rotated_k=True)
    start = lengths - np.minimum(drop, lengths)
    assert np.array_equal(c.length.cpu().numpy(), np.minimum(start + n, 32))
    at = np.concatenate([start[b] + 5 + np.arange(n[b]) for b in range(B)])
    near(got, *turn(_np(q), at, freq, False), "fp32")
    near(keys, *turn(_np(k), at, freq, False), "fp32")


@pytest.mark.parametrize("four", [False, True])
def test_prompt_drafts_and_steps_together(torch_cuda, four):
    """A prompt under window_attention and into the cache, then drafted tokens
    of which some are kept, attention and eviction: at every step the attention
    is that of the tokens that a plain account holds."""
    torch = torch_cuda
    rng = np.random.default_rng(5)
    kern = _kern()
    lengths, hq, hkv, dh, window, sinks = [90, 1, 40], 8, 2, 64, 50, 2
    cu = np.concatenate([[0], np.cumsum(lengths)])
    freq = 100.0 ** (-np.arange(32) / 32)
    fr = torch.from_numpy(freq.astype(np.float32)).cuda()
    c = (kern.TokenCache4 if four else kern.TokenCache).empty(3, 140, hkv, dh, page_size=16)
    q, k, v = (_normal(torch, rng, "bf16", int(cu[-1]), h, dh) for h in (hq, hkv, hkv))
    tq, tk = kern.cache_append_rotary(c, q, k, v, fr, cu, rotated_k=True)
    prompt = kern.window_attention(tq, tk, v, cu, window, sinks)
    last = torch.tensor(cu[1:] - 1, device="cuda")
    got = kern.paged_attention(tq[last], c, window, sinks)
    ref = paged_ref if four else _paged_ref
    out, tol, _, _ = ref(_np(tq[last]), c, window, sinks, "bf16")
    _close(_np(got), out, tol)
    if not four:
        assert (np.abs(_np(got) - _np(prompt[last])) <= 2 * tol).all()
    position = [list(range(n)) for n in lengths]
    drop = torch.zeros(3, dtype=torch.int32, device="cuda")
    for step in range(6):
        drafts = 4
        q, k, v = (_normal(torch, rng, "bf16", 3 * drafts, h, dh) for h in (hq, hkv, hkv))
        tq, _ = kern.cache_append_rotary(c, q, k, v, fr, np.arange(4) * drafts, drop=drop)
        for b in range(3):
            position[b] = position[b][:len(position[b]) - int(drop[b])]
            top = int(c.seen[b]) - drafts
            position[b] += list(range(top, top + drafts))
            n = int(c.length[b])
            assert n == len(position[b]) and c.pos[b, :n].tolist() == position[b]
        at = torch.arange(3, device="cuda") * drafts + drafts - 1
        got = kern.paged_attention(tq[at], c, window if step % 2 else None, sinks)
        out, tol, _, _ = ref(_np(tq[at]), c, window if step % 2 else None, sinks, "bf16")
        _close(_np(got), out, tol, step)
        drop = torch.tensor([step % 4, 2, 0], dtype=torch.int32, device="cuda")
        if step == 3:  # the kept ones stay, the others go before an eviction
            none = [torch.zeros(0, h, dh, dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv)]
            kern.cache_append_rotary(c, *none, fr, [0, 0, 0, 0], drop=drop)
            for b in range(3):
                position[b] = position[b][:len(position[b]) - int(drop[b])]
            src = kern.cache_evict(c, 60, sinks, 8).cpu().numpy()
            position = [[position[b][x] for x in src[b] if x >= 0] for b in range(3)]
            drop = torch.zeros_like(drop)


def test_refusals(torch_cuda):
    torch = torch_cuda
    kern = _kern()
    rng = np.random.default_rng(14)
    c = _cache(torch, rng, "bf16", [20, 5], 2, 64, 16, 32)
    n = lambda *s: _normal(torch, rng, "bf16", *s)
    q, k, f = n(2, 4, 64), n(2, 2, 64), torch.rand(32, device="cuda")
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    state = [t.clone() for t in c._tensors]
    call = kern.cache_append_rotary
    for bad in [
        lambda: call(c, q, k, k, f.double()), lambda: call(c, q, k, k, f.cpu()),
        lambda: call(c, q, k, k, f[:30]), lambda: call(c, q, k, k, torch.rand(36, device="cuda")),
        lambda: call(c, q, k, k, torch.rand(4, 8, device="cuda")), lambda: call(c, q, k, k, None),
        lambda: call(c, q, k, k, torch.rand(64, device="cuda")[::2]),
        lambda: call(c, q, k, k, f.clone().requires_grad_()),
        lambda: call(c, q, k, k, f, drop=i32(1)), lambda: call(c, q, k, k, f, drop=i32(1, 2).long()),
        lambda: call(c, q, k, k, f, drop=[1, 2]), lambda: call(c, q, k, k, f, [0, 1, 3]),
        lambda: call(c, q, k, k, f, [0, 2]), lambda: call(c, q, k[:1], k, f),
        lambda: call(c, q[:1], k, k, f), lambda: call(c, q, k, k.float(), f),
        lambda: call(c, q, k, k, f, out=q[:, :2]), lambda: call(c, q.float(), k, k, f),
        lambda: call(c, n(2, 4, 32), k, k, f), lambda: call(c, None, k, k, f),
        lambda: call(c, q.clone().requires_grad_(), k, k, f),
        lambda: call(c, n(3, 4, 64), n(3, 2, 64), n(3, 2, 64), f),
    ]:
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(kern._native.FusionError):
        call(c, q, k, k, f, [0, 2, 1])
    # in place, and behind the keys by one row of eight values
    both = n(2 * 4 * 64 + 2 * 2 * 64)
    queries, keys = both[256:768].view(2, 4, 64), both[:256].view(2, 2, 64)
    for out, key in ((queries, keys), (both[8:520].view(2, 4, 64), keys), (both[:512].view(2, 4, 64), k)):
        with pytest.raises(ValueError):
            call(c, queries, key, k, f, out=out)
        with pytest.raises(ValueError):
            call(c, q, k, keys, f, out=both[248:760].view(2, 4, 64))
    assert all(torch.equal(a, b) for a, b in zip(c._tensors, state))
    call(c, q, k, keys, f, out=queries)  # beside the values, without a gap

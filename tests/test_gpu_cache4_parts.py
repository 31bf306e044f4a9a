"""Attention over caches in 4 bits (kernels.TokenCache4 with paged_attention and
block_attention) where a wave's part of the work has many tiles: what one tile
hands to the next, scores that wait in LDS for several of them, sequences that begin
and end within a part, and more sequences than the work is split over.

Compared with plain torch in 64 bits on what the cache holds; tolerances as in
test_gpu_cache.py, and for numbers below 2^-126, which become zero: a weight relative to
the largest and the three parts that it is the sum of (4 2^-126 |v| for each token), and a
sum of a tile that is brought to another maximum, in its part and where parts are joined
(2 2^-126 for each tile); the sum of the weights beside them is at least 1."""
import math

import numpy as np
import pytest

from test_gpu_cache import U32, UNIT, _dt, _kern, torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu
E2M1 = [0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6]


def tiles_a_part(cache, hq, dtype, tokens, tile):
    """Tiles of each wave's part: 2 or 3 waves a SIMD (fp32 queries of wide heads: 2)
    of 1,024 SIMDs share the tiles of a unit, a key head and up to 16 of its query heads."""
    if cache.batch > 1024:
        return max(-(-n // tile) for n in tokens)
    units = cache.kv_heads * -(-(hq // cache.kv_heads) // 16)
    ranges = max(1, 1024 * (2 if dtype == "fp32" and cache.dh > 64 else 3) // units)
    return -(-sum(-(-n // tile) for n in tokens) // ranges)


def make(torch, seed, dtype, lengths, hkv, dh, page, evicted=False):
    """A cache with shuffled pages and random contents, its queries' generator."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    B, n = len(lengths), -(-max(lengths) // page)
    pages = B * n + 2
    u8 = lambda lo, hi, w: torch.randint(lo, hi, (pages, hkv, page, w), dtype=torch.uint8, device="cuda",
                                         generator=g).transpose(1, 2)
    ts = [u8(0, 256, dh // 2), u8(0, 256, dh // 2), u8(122, 128, dh // 32), u8(120, 131, dh // 32)]
    table = torch.randperm(pages, generator=g, device="cuda")[:B * n].view(B, n).int()
    length = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    seen, pos = length.clone(), torch.arange(n * page, device="cuda").int().repeat(B, 1)
    if evicted:
        seen = 3 * length + 2
        for b in range(B):
            pos[b, :lengths[b]] = torch.randperm(int(seen[b]), generator=g, device="cuda")[:lengths[b]].int()
    weight = torch.rand((B, n * page), generator=g, device="cuda")
    return _kern().TokenCache4(*ts, table, length, seen, weight, pos, dtype=_dt(torch, dtype)), g


def rows_of(torch, codes, scales):
    """The values [heads, n, dh] in 64 bits of codes [n, heads, dh / 2]."""
    two = torch.tensor([[E2M1[i & 15], E2M1[i >> 4]] for i in range(256)], dtype=torch.float64, device="cuda")
    x = two[codes.int()].reshape(*codes.shape[:2], -1, 32)
    return (x * torch.exp2(scales.double() - 127)[..., None]).flatten(-2).transpose(0, 1).contiguous()


def reference(torch, q, c, dtype, window=None, sinks=0, chosen=None):
    """out, its tolerance, added weights, theirs; `chosen`: pages that are attended."""
    B, hq, dh = q.shape
    page, hkv = c.k.shape[1], c.kv_heads
    scale, up = 1 / math.sqrt(dh), UNIT["bf16"] if dtype == "bf16" else 0.0
    out, tol = (torch.zeros(q.shape, dtype=torch.float64, device="cuda") for _ in range(2))
    add, add_tol = (torch.zeros(c.weight.shape, dtype=torch.float64, device="cuda") for _ in range(2))
    for b, n in enumerate(c.length.tolist()):
        if n == 0:
            continue
        x = torch.arange(n, device="cuda")
        at = c.table[b].long()[x // page], x % page
        k, v = rows_of(torch, c.k[at], c.k_scale[at]), rows_of(torch, c.v[at], c.v_scale[at])
        see = torch.ones((1, n), dtype=torch.bool, device="cuda")
        if window:
            see = ((c.pos[b, :n] > c.seen[b] - 1 - window) | (c.pos[b, :n] < sinks))[None]
        if chosen is not None:
            pages = torch.zeros((hkv, c.table.shape[1] + 1), dtype=torch.bool, device="cuda")
            pages.scatter_(1, chosen[b].long() % pages.shape[1], True)  # (-1: the last, which is none)
            see = pages[:, x // page]
        qb, kt = q[b].double().view(hkv, -1, dh), k.transpose(1, 2).contiguous()
        s = torch.matmul(qb, kt) * scale
        ds = (dh + 8) * U32 * scale * torch.matmul(qb.abs(), kt.abs()) + 8 * U32 * s.abs()
        s = s.masked_fill(~see[:, None], -math.inf)
        e = torch.exp(s - s.amax(-1, keepdim=True).clamp(min=-1e300))
        p = e / e.sum(-1, keepdim=True).clamp(min=1e-300)
        rel = 2 * ds.masked_fill(~see[:, None], 0).amax(-1) + (see.sum(-1)[:, None] + 16) * U32
        o = torch.matmul(p, v)
        t = UNIT[dtype] * o.abs() + (up + rel)[..., None] * torch.matmul(p, v.abs())
        t += 2.0 ** -126 * (4 * torch.matmul(see.double()[:, None], v.abs()) + 2 * (-(-n // 32)))
        out[b], tol[b] = o.view(hq, dh), t.view(hq, dh)
        add[b, :n] = p.sum((0, 1)) / hq
        add_tol[b, :n] = (p * (rel + (hq + 2) * U32)[..., None]).sum((0, 1)) / hq
    return out, tol, add, add_tol


def close(torch, got, want, tol, what):
    assert bool(torch.isfinite(got).all()), what
    worst = float(((got.double() - want).abs() - tol).max())
    assert worst <= 0, (what, worst)


def lengths_of(seed, n, most):
    """0 .. most, with the ends of tiles and pages among them."""
    some = [0, 1, 63, 64, 65, most, 0, 128, 1023]
    return some + [int(x) for x in np.random.default_rng(seed).integers(0, most + 1, size=n - len(some))]


def check(torch, c, q, dtype, window=None, sinks=0):
    out, tol, add, add_tol = reference(torch, q, c, dtype, window, sinks)
    before = c.weight.double()
    got = _kern().paged_attention(q, c, window, sinks)
    close(torch, got, out, tol, "out")
    # (a weight grows by what 128 heads add at a time, each sum rounded once: with h heads
    # it is rounded ceil(h / 128) times, by at most half a step of its last value)
    grown = -(-q.shape[1] // 128)
    off = (c.weight.double() - before - add).abs() - (add_tol + grown * U32 * (before + add))
    assert float(off.max()) <= 0, float(off.max())
    assert torch.equal(c.weight[add == 0].double(), before[add == 0])
    w = c.weight.clone()
    assert torch.equal(_kern().paged_attention(q, c, window, sinks, accumulate=False), got)
    assert torch.equal(c.weight, w)


PARTS = [  # query heads a key head, kv_heads, dh, page, sequences, least tiles a part
    (4, 32, 128, 64, 70, 8),
    (1, 96, 64, 16, 70, 24),
    (1, 48, 128, 128, 70, 11),
    (8, 32, 96, 16, 70, 8),
    (6, 40, 64, 64, 70, 9),
    (16, 32, 128, 128, 70, 8),
    (12, 32, 128, 32, 70, 8),
    (3, 48, 32, 48, 70, 11),
    (20, 20, 64, 64, 70, 9),
    (33, 12, 128, 16, 60, 7),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", range(len(PARTS)))
def test_parts_of_many_tiles(torch_cuda, case, dtype):
    torch = torch_cuda
    group, hkv, dh, page, B, least = PARTS[case]
    print(f"[parts] {dtype} {PARTS[case]}", flush=True)
    lengths = lengths_of(case, B, 1500)
    c, g = make(torch, case, dtype, lengths, hkv, dh, page)
    assert tiles_a_part(c, group * hkv, dtype, lengths, 64) >= least
    q = torch.randn((B, group * hkv, dh), generator=g, device="cuda").to(c.dtype)
    check(torch, c, q, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("group,dh,page", [(4, 128, 64), (1, 64, 16), (8, 128, 16), (16, 64, 64)])
def test_more_sequences_than_the_work_is_split_over(torch_cuda, group, dh, page, dtype):
    """1,030 sequences, each a part of its own, of up to 36 tiles."""
    torch = torch_cuda
    print(f"[parts] 1030 {dtype} {group} {dh} {page}", flush=True)
    lengths = [int(n) for n in np.random.default_rng(dh).integers(0, 200, size=1030)]
    lengths[7], lengths[600], lengths[1029], lengths[5] = 2300, 1500, 1400, 0
    c, g = make(torch, dh, dtype, lengths, 2, dh, page)
    assert tiles_a_part(c, 2 * group, dtype, lengths, 64) == 36
    q = torch.randn((1030, 2 * group, dh), generator=g, device="cuda").to(c.dtype)
    check(torch, c, q, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("group,hkv,dh,page,evicted", [
    (4, 32, 128, 64, True), (1, 64, 64, 16, True), (16, 24, 96, 27, True), (4, 32, 128, 64, False),
    (5, 48, 64, 27, False)])
def test_windows_over_parts_of_many_tiles(torch_cuda, group, hkv, dh, page, evicted, dtype):
    """Slots in order and out of it (whose visible ones are gathered 512 at a time)."""
    torch = torch_cuda
    print(f"[parts] window {dtype} {group} {hkv} {dh} {page} {evicted}", flush=True)
    lengths = lengths_of(hkv, 70, 1500)
    window = 2000 if evicted else 900
    c, g = make(torch, hkv, dtype, lengths, hkv, dh, page, evicted)
    visible = lengths if evicted else [min(n, window + 3) for n in lengths]
    assert tiles_a_part(c, group * hkv, dtype, visible, 32) >= 8
    q = torch.randn((70, group * hkv, dh), generator=g, device="cuda").to(c.dtype)
    check(torch, c, q, dtype, window, 3)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("group,hkv,dh,page", [(4, 32, 128, 64), (1, 64, 64, 16), (8, 32, 96, 32),
                                               (16, 24, 128, 128), (20, 24, 64, 27)])
def test_chosen_pages_of_many_tiles(torch_cuda, group, hkv, dh, page, dtype):
    torch = torch_cuda
    print(f"[parts] blocks {dtype} {group} {hkv} {dh} {page}", flush=True)
    lengths = lengths_of(hkv, 70, 1500)
    blocks = 1000 // page
    c, g = make(torch, hkv, dtype, lengths, hkv, dh, page)
    tokens = [min(n, blocks * page) for n in lengths]
    assert tiles_a_part(c, group * hkv, dtype, tokens, 64 if page % 16 == 0 else 32) >= 6
    q = torch.randn((70, group * hkv, dh), generator=g, device="cuda").to(c.dtype)
    got, chosen = _kern().block_attention(q, c, _kern().PageBounds(c), blocks, 1, 2)
    out, tol, _, _ = reference(torch, q, c, dtype, chosen=chosen)
    close(torch, got, out, tol, "out")
    pages = (torch.tensor(lengths, device="cuda") + page - 1) // page
    assert torch.equal((chosen >= 0).sum(-1), pages.clamp(max=blocks)[:, None].expand(-1, hkv))
    ahead = chosen[..., 1:] > chosen[..., :-1]
    assert bool((ahead | (chosen[..., 1:] < 0)).all()) and bool((chosen < pages[:, None, None]).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("group,hkv,dh,page", [(4, 32, 128, 64), (1, 96, 64, 16), (8, 32, 64, 128),
                                               (16, 32, 128, 16), (4, 32, 64, 27)])
def test_scores_that_grow_along_a_sequence(torch_cuda, group, hkv, dh, page, dtype):
    """Keys whose scales rise every 64 tokens: the maximum that weights refer to is
    raised, and sums so far brought to it, in the middle of a part (27 tokens a page: by
    the kernel of windows and other pages)."""
    torch = torch_cuda
    print(f"[parts] grow {dtype} {group} {hkv} {dh} {page}", flush=True)
    lengths = lengths_of(3, 70, 1500)
    c, g = make(torch, 3, dtype, lengths, hkv, dh, page)
    slot = torch.arange(c.capacity, device="cuda").view(1, -1, page)
    c.k_scale[c.table.long()] = (123 + (slot // 64).clamp(max=8))[..., None, None].to(torch.uint8)
    assert tiles_a_part(c, group * hkv, dtype, lengths, 64) >= 6
    q = torch.randn((70, group * hkv, dh), generator=g, device="cuda").to(c.dtype)
    b = max(range(70), key=lambda b: lengths[b])
    x = torch.arange(576, device="cuda")
    at = c.table[b].long()[x // page], x % page
    k = rows_of(torch, c.k[at], c.k_scale[at])
    s = torch.matmul(q[b].double().view(hkv, group, dh), k.transpose(1, 2).contiguous())
    top = (s / math.sqrt(dh) / math.log(2)).view(hkv, group, 9, 64).amax(-1).cummax(-1).values
    assert float(((top[..., 1:] - top[..., :-1] > 8).sum(-1) >= 2).double().mean()) > 0.5
    check(torch, c, q, dtype)


FAR = [  # page and row strides of codes and of scales: at the last that the tiles of 64 take, and past it
    ((1 << 32) - 16, 64, 1 << 20, 4), (1 << 32, 64, 1 << 20, 4),
    (1 << 20, 64, (1 << 32) - 1, 4), (1 << 20, 64, 1 << 32, 4), (1 << 20, 64, (1 << 32) + 5, 4),
    (1 << 32, (1 << 26) - 16, 1 << 20, 4), (1 << 32, 1 << 26, 1 << 20, 4),
    ((1 << 32) - 16, (1 << 26) - 16, 1 << 20, 4), ((1 << 32) - 16, 1 << 26, 1 << 20, 4),
    (1 << 20, 64, (1 << 32) - 1, (1 << 26) - 1), (1 << 20, 64, (1 << 32) - 1, 1 << 26),
    (1 << 20, 64, (1 << 32) - 1, (1 << 26) + 3),
]


@pytest.mark.parametrize("part", ["k", "v"])
@pytest.mark.parametrize("page,row,scale_page,scale_row", FAR)
def test_strides_at_the_limits_of_the_tiles(torch_cuda, page, row, scale_page, scale_row, part):
    """Strides on both sides of those that tiles of 64 tokens hold in 32 bits, of the
    keys' codes and scales or of the values', give what a compact cache gives."""
    torch = torch_cuda
    print(f"[parts] strides {part} {page:#x} {row:#x} {scale_page:#x} {scale_row:#x}", flush=True)
    places = 64  # (a page's places by row strides of 2^26: 4 GiB)
    c, g = make(torch, 9, "bf16", [128, 70], 2, 64, places)
    q = torch.randn((2, 8, 64), generator=g, device="cuda").to(c.dtype)
    far, big = [], None
    for i, t in enumerate((c.k, c.v, c.k_scale, c.v_scale)):
        w, mine = t.shape[3], i % 2 == "kv".index(part)
        st = (scale_page, scale_row) if i > 1 else (page, row)
        if not mine or st in ((1 << 20, 64), (1 << 20, 4)):
            far.append(t)
            continue
        st = (*st, w, 1)
        big = torch.empty(1 + sum((n - 1) * s for n, s in zip(t.shape, st)), dtype=torch.uint8, device="cuda")
        far.append(big.as_strided(t.shape, st))
        far[-1].copy_(t)
    kern = _kern()
    f = kern.TokenCache4(*far, c.table, c.length.clone(), c.seen.clone(), c.weight.clone(), c.pos.clone())
    out, tol, add, add_tol = reference(torch, q, c, "bf16")
    close(torch, kern.paged_attention(q, f), out, tol, "out")
    off = (f.weight.double() - c.weight.double() - add).abs() - (add_tol + U32 * (c.weight.double() + add))
    assert float(off.max()) <= 0
    got, chosen = kern.block_attention(q, f, kern.PageBounds(f), 1)
    assert torch.equal(chosen[:, :, 0], torch.tensor([[1, 1], [1, 1]], device="cuda"))
    out, tol, _, _ = reference(torch, q, c, "bf16", chosen=chosen)
    close(torch, got, out, tol, "out")
    new = [torch.randn((1, 2, 64), generator=g, device="cuda").to(c.dtype) for _ in "kv"]
    for x in (f, c):
        kern.cache_append(x, *new, [0, 0, 1])
    assert all(torch.equal(a, b) for a, b in zip((f.k, f.v, f.k_scale, f.v_scale), c._tensors[:2] + c._tensors[7:]))
    del f, far, big
    torch.cuda.empty_cache()  # (the memory of one case at a time)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("page", [16, 64, 27])
def test_values_at_the_ends_of_their_range(torch_cuda, page, dtype):
    """Sums are fp32 and the weights in them up to 2^8: n visible values of up to
    6 2^(s - 127) are summed within fp32's range for s up to 244 - log2 n, by windows and
    over chosen pages too.  At the lower end a product of a weight's part (of up to three)
    and a value, or a sum of two, that falls below 2^-126 is lost, 6 n + 4 of them at most
    beside a sum of weights of at least 1."""
    torch = torch_cuda
    kern = _kern()
    for lengths in ([1000, 64, 1, 2, 0], [40, 7, 1, 2, 16]):
        n = max(lengths)
        most = 244 - math.ceil(math.log2(n))
        for scales in ((most, most), (most - 1, most), (2, 2), (2, 40)):
            print(f"[ends] {dtype} {page} {n} {scales}", flush=True)
            c, g = make(torch, n, dtype, lengths, 4, 64, page)
            c.v_scale[...] = torch.randint(scales[0], scales[1] + 1, c.v_scale.shape, generator=g,
                                           device="cuda").to(torch.uint8)
            c.k_scale.add_(2)  # weights of many sizes
            q = torch.randn((5, 16, 64), generator=g, device="cuda").to(c.dtype)
            lost = 2.0 ** -126 * (6 * n + 4)
            out, tol, _, _ = reference(torch, q, c, dtype)
            close(torch, kern.paged_attention(q, c), out, tol + lost, scales)
            out, tol, _, _ = reference(torch, q, c, dtype, 30, 1)
            close(torch, kern.paged_attention(q, c, 30, 1), out, tol + lost, scales)
            got, chosen = kern.block_attention(q, c, kern.PageBounds(c), 3)
            out, tol, _, _ = reference(torch, q, c, dtype, chosen=chosen)
            close(torch, got, out, tol + lost, scales)

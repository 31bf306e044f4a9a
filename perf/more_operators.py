"""Workloads for measuring what serves long streams from a small token cache,
through the public entry points of ``paper_2607_02612_amd.kernels``.

Three kinds of cases:

* ``rotary``: ``cache_append_rotary``, new rows turned by their position and
  appended, in place of the newest tokens of before;
* ``four``: a step over a cache held in 4 bits: ``cache_append_rotary`` into a
  ``TokenCache4``, then ``paged_attention`` of each sequence's newest token.
  The codes that the append leaves come back through the attention that reads
  them, as the values they stand for;
* ``block``: ``PageBounds.update`` for the newest token, then
  ``block_attention`` over the pages that a cheap score selects.

``listed()`` names twelve of them, ``draw()`` gives more of the same ranges,
``exact()`` computes a case in 64 bits, apart from the plain form.
"""
import math

import numpy as np
import torch

own = False  # False: plain torch, in 32 bits and where they lose what matters in 64; True: the library

GPU = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
BASE = 10000.0  # of the frequencies of the rotation
# e2m1 numbers by code (sign, two bits of exponent, one of mantissa)
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]


# ------------------------------------------------------------------ cases --
def listed():
    return [
        # one short stream whose last token is chosen anew: latency
        _rotary("rotary_one", "bf16", 1, 300, 300, 1, 1, 6, 6, 64, 64, False, False),
        # a serving batch, up to five drafted tokens a stream
        _rotary("rotary_drafts", "bf16", 64, 4096, 3, 5, 1, 32, 8, 128, 128, False, False),
        # prompts of very different lengths, whose attention wants turned keys too
        _rotary("rotary_prompts", "bf16", 8, 4096, 1, 4096, 1, 32, 8, 128, 128, False, True),
        # the fp32 path, half of each head turned, in pairs of neighbours
        _rotary("rotary_fp32", "fp32", 16, 1024, 40, 577, 5, 12, 12, 64, 32, True, True),
        # one short stream over 4 bits: latency
        _four("four_one", "bf16", 1, 777, 777, 1, 1, 6, 6, 64, 16, 0, 0, False),
        # a serving batch of ragged lengths, shared key heads
        _four("four_batch", "bf16", 64, 8192, 3, 1, 1, 32, 8, 128, 64, 0, 0, False),
        # two long streams: the work has to be split over the length
        _four("four_long", "bf16", 2, 131072, 100001, 1, 1, 32, 8, 128, 64, 0, 0, False),
        # the next parts of prompts, windowed, over an evicted cache, pages of an odd size
        _four("four_parts_fp32", "fp32", 16, 4099, 317, 301, 7, 12, 4, 96, 27, 1000, 4, True),
        # one stream over small pages: latency
        _block("block_one", "bf16", 1, 16384, 16384, 6, 6, 64, 16, 16, 32, 1, 1),
        # a serving batch, at most 16 pages of 64 tokens a head
        _block("block_batch", "bf16", 64, 8192, 3, 32, 8, 128, 16, 64, 16, 1, 2),
        # two long streams, about a sixteenth of their pages
        _block("block_long", "bf16", 2, 131072, 100001, 32, 8, 128, 16, 64, 128, 1, 4),
        # the same over 4 bits, in the fp32 path
        _block("block_four_fp32", "fp32", 12, 20011, 15, 20, 4, 64, 4, 48, 40, 2, 3),
    ]


def _named(c, name):
    return dict(c, name=name) if name else c


def _rotary(name, dtype, batch, tokens, shortest, new, fewest, q_heads, kv_heads, dh, turned, pairs,
            keys):
    """`tokens`, `shortest`: the longest and the shortest sequence before the
    call; `new`, `fewest`: the most and the fewest rows of one; `turned`: dims
    of a head that turn; `pairs`: dims 2j and 2j + 1 turn together; `keys`: the
    turned keys are asked for."""
    return _named({"kind": "rotary", "dtype": dtype, "batch": batch, "tokens": tokens,
                   "shortest": shortest, "new": new, "fewest": fewest, "q_heads": q_heads,
                   "kv_heads": kv_heads, "dh": dh, "page": 64, "turned": turned, "pairs": pairs,
                   "keys": keys, "bits": 32 if dtype == "fp32" else 16, "evicted": False}, name)


def _four(name, dtype, batch, tokens, shortest, new, fewest, q_heads, kv_heads, dh, page, window,
          sinks, evicted):
    """`evicted`: tokens have left the cache, so its slots are out of order.
    A window of 0: every cached token is visible."""
    return _named({"kind": "four", "dtype": dtype, "batch": batch, "tokens": tokens,
                   "shortest": shortest, "new": new, "fewest": fewest, "q_heads": q_heads,
                   "kv_heads": kv_heads, "dh": dh, "page": page, "turned": dh, "pairs": False,
                   "window": window, "sinks": sinks, "evicted": evicted, "bits": 4}, name)


def _block(name, dtype, batch, tokens, shortest, q_heads, kv_heads, dh, bits, page, blocks, first,
           recent):
    """`blocks`: pages that a key head reads, the `first` and `recent` ones
    among them."""
    return _named({"kind": "block", "dtype": dtype, "batch": batch, "tokens": tokens,
                   "shortest": shortest, "q_heads": q_heads, "kv_heads": kv_heads, "dh": dh,
                   "bits": bits, "page": page, "blocks": blocks, "first": first, "recent": recent,
                   "evicted": False}, name)


def _spread(rng, lo, hi):
    """A whole number in lo .. hi, spread over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


HEADS = [(6, 6, 64), (12, 12, 64), (16, 2, 128), (32, 8, 128), (8, 1, 96), (20, 4, 64), (12, 4, 80)]


def draw(rng):
    kind = rng.choice(["rotary", "four", "block"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    bits = 32 if dtype == "fp32" else 16
    if kind == "four" or kind == "block" and rng.random() < 0.4:
        bits = 4
    q_heads, kv_heads, dh = rng.choice([h for h in HEADS if bits > 4 or h[2] % 32 == 0])
    row = kv_heads * dh * (4 if dtype == "fp32" else 2)
    if kind == "rotary":
        new = rng.choice([1, _spread(rng, 2, 8), _spread(rng, 9, 4096)])
        batch = _spread(rng, 1, 64 if new <= 8 else max(1, min(16, (24 << 20) // (row * new))))
        tokens = new + _spread(rng, 1, 4096)
        fewest = rng.randint(1, new)
        return _rotary(None, dtype, batch, tokens, rng.randint(new, tokens), new, fewest, q_heads,
                       kv_heads, dh, rng.choice([dh, dh // 2]), rng.random() < 0.3, new > 8)
    page = rng.choice([16, 32, 64, 128, 27, 48])
    if kind == "four":
        new = rng.choice([1, 1, _spread(rng, 2, 300)])
        tokens = new + _spread(rng, 100, 131072 - 300)
        batch = _spread(rng, 1, max(1, min(64, (400 << 20) // (row * tokens))))
        window = rng.choice([0, _spread(rng, 16, tokens)])
        return _four(None, dtype, batch, tokens, rng.randint(new, tokens), new, rng.randint(1, new),
                     q_heads, kv_heads, dh, page, window, rng.randint(0, 8) if window else 0,
                     rng.random() < 0.5)
    tokens = _spread(rng, 1000, 131072)
    batch = _spread(rng, 1, max(1, min(64, (400 << 20) // (row * tokens))))
    pages = -(-tokens // page)
    first, recent = rng.randint(0, 2), rng.randint(1, 4)
    most = max(first + recent, min(pages, (100 << 20) // (batch * page * row)))
    return _block(None, dtype, batch, tokens, rng.randint(1, tokens), q_heads, kv_heads, dh, bits,
                  page, _spread(rng, first + recent, most), first, recent)


def _lengths(longest, shortest, n):
    """n whole numbers in shortest .. longest, the first the longest, spread
    evenly in no order (the case alone decides them)."""
    return [longest - int((longest - shortest) * ((i * 0.6180339887498949) % 1.0) + 0.5)
            for i in range(n)]


def _shape(case):
    """Rows of the call by sequence, and the tokens held when it begins (the
    rows that it replaces among them)."""
    n = _lengths(case["tokens"], case["shortest"], case["batch"])
    if "new" not in case:
        return [0] * len(n), n
    new = _lengths(case["new"], case["fewest"], case["batch"])
    return new, [max(a, b) for a, b in zip(n, new)]


# ------------------------------------------------------------ e2m1 blocks --
def _pack(x):
    """fp32 [.., dh] -> codes uint8 [.., dh / 2] (the lower dim in the lower
    half of a byte), scales uint8 [.., dh / 32]: a block of 32 dims has the
    scale 2^(s - 127) that brings its largest magnitude to 4 .. 8, within
    2^-125 .. 2^125; values go to the nearest e2m1 number, ties to the even
    code, those above 6 to 6."""
    b = x.reshape(*x.shape[:-1], -1, 32)
    top = b.abs().amax(-1)
    e = torch.where(top > 0, torch.frexp(top).exponent - 3, -125).clamp(-125, 125)
    a = torch.ldexp(b, -e[..., None])
    sign = torch.signbit(a)
    a = a.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = (torch.round(a / step) * step).clamp(max=6.0)
    code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a * 0.5 + 4)).to(torch.uint8)
    code = (code | sign.to(torch.uint8) << 3).reshape(*x.shape[:-1], -1, 2)
    return code[..., 0] | code[..., 1] << 4, (e + 127).to(torch.uint8)


def _unpack(codes, scales, dtype=torch.float32):
    """The values that codes [.., dh / 2] and scales [.., dh / 32] stand for."""
    two = torch.tensor([[E2M1[i & 15], E2M1[i >> 4]] for i in range(256)], dtype=dtype, device=GPU)
    v = two[codes.int()].reshape(*codes.shape[:-1], -1, 32)
    return torch.ldexp(v, scales.int()[..., None] - 127).flatten(-2)


# ----------------------------------------------------------------- inputs --
def prepare(case, seed):
    g = torch.Generator(device=GPU)
    g.manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device=GPU, dtype=dt)

    def i32(a):
        return torch.tensor(a, dtype=torch.int32, device=GPU)

    s = {"case": case}
    new, held = _shape(case)
    b, hq, hkv, dh, page = (case[x] for x in ("batch", "q_heads", "kv_heads", "dh", "page"))
    if case["kind"] == "block":
        s["q"] = normal(b, hq, dh)
    else:
        s["cu"] = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        s["cu_gpu"] = i32(s["cu"])
        s["last"] = s["cu_gpu"][1:].long() - 1
        # one product gives the three: they are views of its output
        qkv = normal(int(s["cu"][-1]), hq + 2 * hkv, dh)
        s["q"], s["k_new"], s["v_new"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        half = case["turned"] // 2
        s["freq"] = (BASE ** (-torch.arange(half, dtype=torch.float64, device=GPU) / half)).float()
        s["drop"] = i32(new)
    max_pages = -(-max(held) // page)
    cap, pages = max_pages * page, b * max_pages + 3
    channel = torch.exp(0.5 * torch.randn((hkv, 1, dh), generator=g, device=GPU)).to(dt)
    if case["bits"] == 4:  # heads before the places of a page: a head's rows lie together
        k, v = (_pack((normal(pages, hkv, page, dh) * c).float()) for c in (channel, 1.0))
        s["k"], s["k_scale"] = (t.transpose(1, 2) for t in k)
        s["v"], s["v_scale"] = (t.transpose(1, 2) for t in v)
    else:
        s["k"] = normal(pages, page, hkv, dh) * channel.transpose(0, 1)
        s["v"] = normal(pages, page, hkv, dh)
    s["table"] = torch.randperm(pages, generator=g, device=GPU)[:b * max_pages] \
        .view(b, max_pages).int()
    s["len"] = i32(held)
    # a heavy-tailed weight: few tokens draw most of the attention
    s["weight"] = torch.exp(2 * torch.randn(b, cap, generator=g, device=GPU))
    slot = torch.arange(cap, device=GPU)
    if case["evicted"]:  # every other token has left, of those before the newest
        n = i32(new)[:, None]
        before = (s["len"][:, None] - n) * 2
        order = torch.rand(b, 2 * cap, generator=g, device=GPU)
        order = order.masked_fill(torch.arange(2 * cap, device=GPU) >= before, 2.0)
        pos = order.argsort(dim=1)[:, :cap]
        at = s["len"][:, None] - n
        s["pos"] = torch.where(slot >= at, before + slot - at, pos).int().contiguous()
        s["seen"] = (before + n)[:, 0].int().contiguous()
    else:
        s["seen"] = s["len"].clone()
        s["pos"] = slot.int().repeat(b, 1)
    if case["kind"] == "block":  # bounds of the pages as they were one token before
        s["lo"], s["hi"] = (torch.zeros((pages, hkv, dh), dtype=dt, device=GPU) for _ in range(2))
        _bounds(s, (s["len"] - 1).clamp(min=0), torch.zeros_like(s["len"]))
    return s


# ------------------------------------------------------------------- runs --
def run(s):
    kind = s["case"]["kind"]
    if kind == "rotary":
        return _rotary_own(s) if own else _rotary_plain(s)
    if kind == "four":
        return _four_own(s) if own else _four_plain(s)
    return _block_own(s) if own else _block_plain(s)


def _cache(s):
    """The handles that a program keeps for its cache, made at the first pass."""
    if "cache" not in s:
        from paper_2607_02612_amd import kernels
        rest = [s[x] for x in ("table", "len", "seen", "weight", "pos")]
        if s["case"]["bits"] == 4:
            s["cache"] = kernels.TokenCache4(s["k"], s["v"], s["k_scale"], s["v_scale"], *rest,
                                             dtype=DTYPES[s["case"]["dtype"]])
        else:
            s["cache"] = kernels.TokenCache(s["k"], s["v"], *rest)
        if s["case"]["kind"] == "block":
            s["bounds"] = kernels.PageBounds(s["cache"], s["lo"], s["hi"])
    return s["cache"]


def _append_own(s):
    from paper_2607_02612_amd import kernels
    c = s["case"]
    return kernels.cache_append_rotary(
        _cache(s), s["q"], s["k_new"], s["v_new"], s["freq"], cu=s["cu"] if c["new"] > 1 else None,
        interleaved=c["pairs"], drop=s["drop"], rotated_k=c.get("keys", False))


def _rotary_own(s):
    q, k = _append_own(s)
    return _rotary_out(s, q, k)


def _rotary_out(s, q, k):
    out = {"q": q, "cache_k": s["k"], "cache_v": s["v"], "weight": s["weight"], "pos": s["pos"],
           "len": s["len"], "seen": s["seen"]}
    return dict(out, k=k) if s["case"]["keys"] else out


def _four_own(s):
    from paper_2607_02612_amd import kernels
    c = s["case"]
    q, _ = _append_own(s)
    out = kernels.paged_attention(q[s["last"]] if c["new"] > 1 else q, _cache(s),
                                  window=c["window"] or None, sinks=c["sinks"])
    return {"q": q, "out": out, "weight": s["weight"], "pos": s["pos"], "len": s["len"],
            "seen": s["seen"]}


def _block_own(s):
    from paper_2607_02612_amd import kernels
    c = s["case"]
    cache = _cache(s)
    s["bounds"].update(1)
    out, chosen = kernels.block_attention(s["q"], cache, s["bounds"], c["blocks"], first=c["first"],
                                          recent=c["recent"])
    return {"out": out, "chosen": chosen, "lo": s["lo"], "hi": s["hi"]}


# ------------------------------------------------------------- plain form --
def _turn(x, angle, turned, pairs):
    """x [rows, heads, dh], angle [rows, 1, turned / 2]: dims in pairs (2j,
    2j + 1), or (j, j + turned / 2), turned; the others as they are."""
    cos, sin = torch.cos(angle).to(x.dtype), torch.sin(angle).to(x.dtype)
    t = x[..., :turned]
    a, b = (t[..., ::2], t[..., 1::2]) if pairs else t.chunk(2, -1)
    a, b = a * cos - b * sin, b * cos + a * sin
    t = torch.stack((a, b), -1).flatten(-2) if pairs else torch.cat((a, b), -1)
    return torch.cat((t, x[..., turned:]), -1)


def _append_plain(s):
    c = s["case"]
    cu = s["cu_gpu"].long()
    r = torch.arange(s["q"].shape[0], device=GPU)
    seq = torch.searchsorted(cu, r, right=True) - 1
    nth = r - cu[seq]
    slot = (s["len"] - s["drop"]).long()[seq] + nth
    pos = (s["seen"] - s["drop"]).long()[seq] + nth
    angle = (pos[:, None].double() * s["freq"].double())[:, None]
    dt = s["q"].dtype
    q = _turn(s["q"].float(), angle, c["turned"], c["pairs"]).to(dt)
    # (rounded to 4 bits, values next to a border have to fall on the same side)
    k = s["k_new"].double() if c["bits"] == 4 else s["k_new"].float()
    k = _turn(k, angle, c["turned"], c["pairs"]).float().to(dt)
    page = c["page"]
    to = s["table"][seq, slot // page].long(), slot % page
    if c["bits"] == 4:
        s["k"][to], s["k_scale"][to] = _pack(k.float())
        s["v"][to], s["v_scale"][to] = _pack(s["v_new"].float())
    else:
        s["k"][to], s["v"][to] = k, s["v_new"]
    s["weight"][seq, slot] = 0.0
    s["pos"][seq, slot] = pos.int()
    more = (cu[1:] - cu[:-1]).int() - s["drop"]
    s["len"] += more
    s["seen"] += more
    return q, k


def _rotary_plain(s):
    return _rotary_out(s, *_append_plain(s))


def _attend(q, k, v, hidden):
    """Softmax attention of q [B, H, G, dh] over k, v [B, H, S, dh]: (out,
    probabilities); keys where `hidden` have no part, a query that sees none
    gives zeros."""
    t = torch.matmul(q, k.transpose(-1, -2)).mul_(1.0 / math.sqrt(q.shape[-1]))
    t.masked_fill_(hidden, -math.inf)
    t -= t.amax(-1, keepdim=True).clamp_min(-3e38)
    t.exp_()
    t /= t.sum(-1, keepdim=True).clamp_min(1e-38)
    return torch.matmul(t, v), t


def _four_plain(s):
    c = s["case"]
    q, _ = _append_plain(s)
    b, hkv, dh = c["batch"], c["kv_heads"], c["dh"]
    table = s["table"].long()
    k, v = (_unpack(s[x][table], s[x + "_scale"][table]).reshape(b, -1, hkv, dh).transpose(1, 2)
            for x in "kv")
    slot = torch.arange(k.shape[2], device=GPU)
    hidden = slot >= s["len"][:, None]
    if c["window"]:
        hidden = hidden | ((s["pos"] >= c["sinks"]) & (s["pos"] < (s["seen"] - c["window"])[:, None]))
    out, p = _attend(q[s["last"]].float().view(b, hkv, -1, dh), k, v, hidden[:, None, None])
    s["weight"] += p.sum((1, 2)) / c["q_heads"]
    return {"q": q, "out": out.reshape(b, c["q_heads"], dh).to(q.dtype), "weight": s["weight"],
            "pos": s["pos"], "len": s["len"], "seen": s["seen"]}


def _bounds(s, length, start):
    """lo and hi of the pages of slots start .. length - 1: the least and the
    greatest of each dim over a page's tokens."""
    c = s["case"]
    page, slots = c["page"], s["table"].shape[1] * c["page"]
    p = torch.arange(s["table"].shape[1], device=GPU)
    b, p = ((p * page < length[:, None]) & ((p + 1) * page > start[:, None])).nonzero(as_tuple=True)
    at = s["table"][b, p].long()
    k = _unpack(s["k"][at], s["k_scale"][at]) if c["bits"] == 4 else s["k"][at].float()
    slot = torch.arange(slots, device=GPU).view(-1, page)[p]
    out = (slot >= length[b][:, None])[..., None, None]
    s["lo"][at] = k.masked_fill(out, math.inf).amin(1).to(s["lo"].dtype)
    s["hi"][at] = k.masked_fill(out, -math.inf).amax(1).to(s["hi"].dtype)


def _block_plain(s):
    c = s["case"]
    b, hkv, dh, page, blocks = (c[x] for x in ("batch", "kv_heads", "dh", "page", "blocks"))
    length = s["len"]
    _bounds(s, length, length - 1)
    # the most that a head's product with a key of the page can be, next to a border in 64 bits
    table = s["table"].long()
    lo, hi = (s[x][table].double().permute(0, 2, 3, 1).contiguous() for x in ("lo", "hi"))
    q = s["q"].double().view(b, hkv, -1, dh)
    score = (torch.matmul(q.clamp(min=0), hi) + torch.matmul(q.clamp(max=0), lo)).amax(2).float()
    p = torch.arange(table.shape[1], device=GPU)
    n = ((length + page - 1) // page)[:, None, None]
    score = score.masked_fill((p < c["first"]) | (p >= n - c["recent"]), math.inf)
    score = score.masked_fill(p >= n, -math.inf)
    chosen = score.sort(dim=-1, descending=True, stable=True).indices[..., :blocks]
    chosen = chosen.masked_fill(chosen >= n, table.shape[1]).sort(-1).values
    some = torch.minimum(chosen, n - 1)
    at = torch.gather(table[:, None].expand(-1, hkv, -1), 2, some)
    h = torch.arange(hkv, device=GPU)[None, :, None]
    if c["bits"] == 4:
        k, v = (_unpack(s[x].transpose(1, 2)[at, h], s[x + "_scale"].transpose(1, 2)[at, h])
                for x in "kv")
    else:
        k, v = (s[x].transpose(1, 2)[at, h].float() for x in "kv")
    slot = chosen[..., None] * page + torch.arange(page, device=GPU)
    hidden = (slot >= length[:, None, None, None]).flatten(2)
    out, _ = _attend(s["q"].float().view(b, hkv, -1, dh), k.flatten(2, 3), v.flatten(2, 3),
                     hidden[:, :, None])
    return {"out": out.reshape(b, c["q_heads"], dh).to(s["q"].dtype),
            "chosen": chosen.masked_fill(chosen >= n, -1).int(), "lo": s["lo"], "hi": s["hi"]}


# -------------------------------------------------------------- 64 bits --
def exact(case, seed):
    s = prepare(case, seed)
    return {"rotary": _rotary_exact, "four": _four_exact, "block": _block_exact}[case["kind"]](s)


def _turn64(x, pos, c):
    """The rotation as a product of complex numbers."""
    x = x.double()
    half = c["turned"] // 2
    d = torch.arange(half, device=GPU)
    first, second = (2 * d, 2 * d + 1) if c["pairs"] else (d, d + half)
    f = BASE ** (-d.double() / half)
    angle = pos.double()[:, None, None] * f.float().double()
    z = torch.complex(x[..., first], x[..., second]) * torch.polar(torch.ones_like(angle), angle)
    out = x.clone()
    out[..., first], out[..., second] = z.real, z.imag
    return out


def _nearest(x):
    """The values that blocks of 32 numbers of the last axis are held as."""
    x = x.double()
    b = x.reshape(*x.shape[:-1], -1, 32)
    top = b.abs().max(-1).values.cpu().numpy()
    with np.errstate(divide="ignore"):
        e = np.clip(np.floor(np.log2(top)) - 2, -125, 125)
    scale = torch.from_numpy(2.0 ** e).to(GPU)[..., None]
    grid = torch.tensor(E2M1[:8], dtype=torch.float64, device=GPU)
    far = (b.abs() / scale)[..., None] - grid
    # the nearest number; of two as near the one of the even code
    cost = far.abs() + torch.tensor([0, 1e-9] * 4, dtype=torch.float64, device=GPU)
    return (torch.sign(b) * grid[cost.argmin(-1)] * scale).reshape(x.shape)


def _appended(s):
    """(sequence, slot, position) of every new row, turned queries and keys."""
    new, held = _shape(s["case"])
    seen = s["seen"].tolist()
    at = [(b, held[b] - n + i, seen[b] - n + i) for b, n in enumerate(new) for i in range(n)]
    seq, slot, pos = (torch.tensor(x, device=GPU) for x in zip(*at))
    q, k = (_turn64(s[x], pos, s["case"]) for x in ("q", "k_new"))
    return seq, slot, pos, q, k


def _state64(s, seq, slot, pos):
    weight, where = s["weight"].double(), s["pos"].clone()
    weight[seq, slot] = 0.0
    where[seq, slot] = pos.int()
    return weight, where


def _rotary_exact(s):
    c = s["case"]
    seq, slot, pos, q, k = _appended(s)
    weight, where = _state64(s, seq, slot, pos)
    page = s["table"].long()[seq, torch.div(slot, c["page"], rounding_mode="floor")]
    place = slot % c["page"]
    ck, cv = s["k"].double(), s["v"].double()
    ck[page, place], cv[page, place] = k, s["v_new"].double()
    out = {"q": q, "cache_k": ck, "cache_v": cv, "weight": weight, "pos": where, "len": s["len"],
           "seen": s["seen"]}
    return dict(out, k=k) if c["keys"] else out


def _weights64(q, k, see):
    e = (q @ k.mT) / math.sqrt(q.shape[-1])
    e = torch.where(see, e, torch.full_like(e, -math.inf))
    top = e.max(-1, keepdim=True).values
    e = torch.exp(e - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = e.sum(-1, keepdim=True)
    return torch.where(total > 0, e / total, torch.zeros_like(e))


def _held(s, x, pages, h):
    """Rows of head h in `pages` in 64 bits."""
    if s["case"]["bits"] == 4:
        return _unpack(s[x][pages, :, h], s[x + "_scale"][pages, :, h], torch.float64).flatten(0, 1)
    return s[x][pages, :, h].double().flatten(0, 1)


def _four_exact(s):
    c = s["case"]
    seq, slot, pos, q, k = _appended(s)
    weight, where = _state64(s, seq, slot, pos)
    # rows are rounded to their type, then to 4 bits
    rows = _nearest(k.float().to(s["q"].dtype)), _nearest(s["v_new"])
    at = q.to(s["q"].dtype).double()  # the attention's queries are of their type too
    out = torch.zeros((c["batch"], c["q_heads"], c["dh"]), dtype=torch.float64, device=GPU)
    group = c["q_heads"] // c["kv_heads"]
    for b in range(c["batch"]):
        n, mine = int(s["len"][b]), seq == b
        pages = s["table"][b, :-(-n // c["page"])].long()
        see = torch.ones(n, dtype=torch.bool, device=GPU)
        if c["window"]:
            p = where[b, :n]
            see = (int(s["seen"][b]) - 1 - p < c["window"]) | (p < c["sinks"])
        for h in range(c["kv_heads"]):
            k, v = (_held(s, x, pages, h)[:n] for x in "kv")
            k[slot[mine]], v[slot[mine]] = rows[0][mine, h], rows[1][mine, h]
            heads = slice(h * group, (h + 1) * group)
            w = _weights64(at[int(s["last"][b]), heads], k, see)
            out[b, heads] = w @ v
            weight[b, :n] += w.sum(0) / c["q_heads"]
    return {"q": q, "out": out, "weight": weight, "pos": where, "len": s["len"], "seen": s["seen"]}


def _block_exact(s):
    c = s["case"]
    page, group = c["page"], c["q_heads"] // c["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=GPU)
    chosen = np.full((c["batch"], c["kv_heads"], c["blocks"]), -1, np.int32)
    lo, hi = s["lo"].double(), s["hi"].double()
    for b in range(c["batch"]):
        n = int(s["len"][b])
        np_ = -(-n // page)
        pages = s["table"][b, :np_].long()
        for h in range(c["kv_heads"]):
            k, v = (_held(s, x, pages, h)[:n] for x in "kv")
            rows = k[(np_ - 1) * page:]  # the page of the newest token
            lo[pages[-1], h], hi[pages[-1], h] = rows.min(0).values, rows.max(0).values
            heads = slice(h * group, (h + 1) * group)
            q = s["q"][b, heads].double()
            a, z = lo[pages, h], hi[pages, h]
            most = torch.maximum(q[:, None] * a, q[:, None] * z).sum(-1).max(0).values.float()
            most = most.cpu().numpy().astype(np.float64)
            most[:c["first"]] = np.inf
            most[max(0, np_ - c["recent"]):] = np.inf
            take = np.sort(np.lexsort((np.arange(np_), -most))[:c["blocks"]])
            chosen[b, h, :len(take)] = take
            see = torch.zeros(np_ * page, dtype=torch.bool, device=GPU)
            see.view(-1, page)[torch.from_numpy(take).to(GPU)] = True
            out[b, heads] = _weights64(q, k, see[:n]) @ v
    return {"out": out, "chosen": torch.from_numpy(chosen).to(GPU), "lo": lo, "hi": hi}


# ------------------------------------------------------------------- work --
def work(case):
    """Each input read once and each output written once; two operations per
    multiply-add of the products with visible keys and values."""
    size = 2 if case["dtype"] == "bf16" else 4
    heads = case["kv_heads"] * case["dh"]
    row = heads * case["bits"] // 8 + (heads // 32 if case["bits"] == 4 else 0)
    qrow = case["q_heads"] * case["dh"] * size
    new, held = _shape(case)
    rows = sum(new)
    # new rows of three kinds in, turned queries out, a cached key and value, weight and position
    total = rows * (qrow + 2 * heads * size + qrow + 2 * row + 8)
    pairs = 0
    if case["kind"] == "rotary":
        flops = rows * (case["q_heads"] + case["kv_heads"]) * case["turned"] * 3
        return {"bytes": total + (rows * heads * size if case["keys"] else 0), "flops": flops}
    if case["kind"] == "four":
        for n, m in zip(held, new):
            visible = n
            if case["window"]:
                visible = min(n, case["window"] + case["sinks"])
                # of an evicted cache every other token is left, but for the newest
                if case["evicted"]:
                    visible = min(n, m + -(-max(0, visible - m) // 2)) if visible > m else visible
            pairs += visible
            total += visible * (2 * row + 8) + (4 * n if case["window"] else 0)
        total += case["batch"] * qrow
        return {"bytes": total, "flops": 4 * pairs * case["q_heads"] * case["dh"]}
    flops = 0
    for n in held:
        np_ = -(-n // case["page"])
        tokens = n - max(0, np_ - case["blocks"]) * case["page"]
        # bounds of all pages but the newest, which is read and whose bounds are written
        total += np_ * 2 * heads * size + (n - (np_ - 1) * case["page"]) * row
        total += tokens * 2 * row + 2 * qrow + 4 * case["kv_heads"] * case["blocks"]
        flops += 4 * tokens * case["q_heads"] * case["dh"] + 2 * np_ * case["q_heads"] * case["dh"]
    return {"bytes": total, "flops": flops}

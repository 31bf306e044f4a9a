"""Host-side refusals of rotated appends, caches in 4 bits, page bounds and
block attention (CPU): the C entries check every argument before any device call
(the pointers here are never dereferenced)."""
import ctypes
from ctypes import byref

import pytest
import torch

from paper_2607_02612_amd import _native, kernels
from test_cache_checks import BAD_CACHES, P, _cache, _cu, _i64

BIG = 1 << 40


def _scales(**over):
    a = dict(k=P, v=P, k_strides=(64, 4, 2), v_strides=(64, 4, 2))
    a.update(over)
    return _native.FusionScales(*a.values())


def _rows(**over):
    a = dict(q=P, k=P, v=P, q_strides=(256, 64), k_strides=(128, 64), v_strides=(128, 64), q_out=P,
             k_out=None, freq=P, drop=None, heads=4, half=32, interleaved=0)
    a.update(over)
    return _native.FusionRotaryRows(*a.values())


def _calls(c, s):
    """Status of each call that takes a cache and scales."""
    lib = _native.lib()
    return [lib.fusion_cache_append_rotary(c, s, byref(_rows()), None, None),
            lib.fusion_page_bounds(c, s, P, P, 0, None),
            lib.fusion_block_attention(c, s, P, P, P, _i64(256, 64), 4, 4, 1, 1, P, P, P, BIG, None)]


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("bad", BAD_CACHES)
def test_every_call_refuses_a_bad_cache(bad, four):
    lib = _native.lib()
    if four and set(bad) & {"k_strides", "v_strides"}:
        bad = {x: tuple(v + 1 for v in st) for x, st in bad.items()}
    c = byref(_cache(**bad))
    s = byref(_scales()) if four else None
    assert _calls(c, s) == [-1, -1, -1]
    assert lib.fusion_block_attention_workspace_bytes(c, s, 4, 4) == 0
    if four:
        assert lib.fusion_cache4_attention(c, s, P, _i64(256, 64), 4, 0, 0, 1, P, P, BIG, None) == -1
        assert lib.fusion_cache4_evict(c, s, 8, 0, 0, P, P, BIG, None) == -1
        assert lib.fusion_cache4_attention_workspace_bytes(c, s, 4, 1) == 0
        assert lib.fusion_cache4_evict_workspace_bytes(c, s, 8) == 0


@pytest.mark.parametrize("bad", [dict(k=None), dict(v=None), dict(k_strides=(64, -4, 2)),
                                 dict(v_strides=(-1, 4, 2))])
def test_every_call_refuses_bad_scales(bad):
    lib, c, s = _native.lib(), byref(_cache()), byref(_scales(**bad))
    assert _calls(c, s) == [-1, -1, -1]
    assert lib.fusion_cache4_attention(c, s, P, _i64(256, 64), 4, 0, 0, 1, P, P, BIG, None) == -1
    assert lib.fusion_cache4_evict(c, s, 8, 0, 0, P, P, BIG, None) == -1


def test_four_bits_need_scales_and_whole_blocks():
    lib = _native.lib()
    c, s = byref(_cache()), byref(_scales())
    assert lib.fusion_cache4_attention(c, None, P, _i64(256, 64), 4, 0, 0, 1, P, P, BIG, None) == -1
    assert lib.fusion_cache4_evict(c, None, 8, 0, 0, P, P, BIG, None) == -1
    assert lib.fusion_cache4_attention_workspace_bytes(c, None, 4, 1) == 0
    assert lib.fusion_cache4_evict_workspace_bytes(c, None, 8) == 0
    for dh in (8, 40, 80, 120):
        assert _calls(byref(_cache(dh=dh)), s) == [-1, -1, -1]
    n = lib.fusion_cache4_attention_workspace_bytes(c, s, 4, 1)
    assert n > 0 and lib.fusion_cache4_attention(c, s, P, _i64(256, 64), 4, 0, 0, 1, P, P, n - 1, None) == -3
    n = lib.fusion_cache4_evict_workspace_bytes(c, s, 8)
    assert n > 0 and lib.fusion_cache4_evict(c, s, 8, 0, 0, P, P, n - 1, None) == -3


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(k=None), dict(v=None), dict(q_out=None), dict(freq=None), dict(heads=-1),
    dict(heads=4097), dict(half=-4), dict(half=30), dict(half=36), dict(half=1 << 30),
    dict(half=3 << 29), dict(half=2**31 - 4), dict(interleaved=2), dict(q=P + 8),
    dict(k=P + 4), dict(q_out=P + 2), dict(k_out=P + 8), dict(q_strides=(256, 60)),
    dict(k_strides=(-128, 64)), dict(v_strides=(128, 65))])
def test_append_rotary_refuses(bad):
    lib, c = _native.lib(), byref(_cache())
    assert lib.fusion_cache_append_rotary(c, None, byref(_rows(**bad)), None, None) == -1
    assert lib.fusion_last_error().decode() != ""


def test_append_rotary_offsets():
    lib, c = _native.lib(), byref(_cache())
    cu = lambda a: a.ctypes.data_as(ctypes.c_void_p)
    down, late, none = _cu(0, 2, 1), _cu(1, 2, 3), _cu(0, 0, 0)
    assert lib.fusion_cache_append_rotary(c, None, None, None, None) == -1
    assert lib.fusion_cache_append_rotary(c, None, byref(_rows()), cu(down), None) == -1
    assert lib.fusion_cache_append_rotary(c, None, byref(_rows()), cu(late), None) == -1
    assert lib.fusion_cache_append_rotary(c, None, byref(_rows(q=None, k=None)), cu(none), None) == 0


def test_block_calls_refuse_bad_arguments():
    lib, c = _native.lib(), byref(_cache())
    assert lib.fusion_page_bounds(c, None, None, P, 0, None) == -1
    assert lib.fusion_page_bounds(c, None, P, None, 0, None) == -1
    assert lib.fusion_page_bounds(c, None, P, P + 8, 0, None) == -1
    assert lib.fusion_page_bounds(c, None, P, P, -1, None) == -1
    n = lib.fusion_block_attention_workspace_bytes(c, None, 4, 4)
    assert n > 0
    for heads, blocks in ((3, 4), (0, 4), (4, 0), (4, (1 << 30) + 1)):
        assert lib.fusion_block_attention_workspace_bytes(c, None, heads, blocks) == 0
    ok = dict(lo=P, hi=P, q=P, strides=_i64(256, 64), heads=4, blocks=4, first=1, recent=1, out=P,
              chosen=P, ws=P, n=n)
    for bad, code in [
            (dict(lo=None), -1), (dict(hi=None), -1), (dict(lo=P + 8), -1), (dict(q=None), -1),
            (dict(strides=None), -1), (dict(strides=_i64(256, 63)), -1), (dict(heads=3), -1),
            (dict(blocks=0), -1), (dict(blocks=(1 << 30) + 1), -1), (dict(first=-1), -1),
            (dict(recent=0), -1), (dict(first=3, recent=2), -1), (dict(out=None), -1),
            (dict(out=P + 4), -1), (dict(chosen=None), -1), (dict(ws=None), -1), (dict(ws=P + 64), -1),
            (dict(n=n - 1), -3)]:
        assert lib.fusion_block_attention(c, None, *dict(ok, **bad).values(), None) == code, bad


def test_binding_refuses_host_tensors():
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    with pytest.raises(ValueError):
        kernels.TokenCache4(u8(8, 16, 2, 32), u8(8, 16, 2, 32), u8(8, 16, 2, 2), u8(8, 16, 2, 2), i32(2, 4),
                            i32(2), i32(2), torch.zeros(2, 64), i32(2, 64))
    t = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    fake = type("Cache", (), dict(dtype=torch.bfloat16, batch=2, kv_heads=2, dh=64))()
    with pytest.raises(ValueError):
        kernels.cache_append_rotary(fake, t, t, t, torch.rand(32))
    with pytest.raises(ValueError):
        kernels.block_attention(t, fake, None, 4)


@pytest.mark.parametrize("v", [float("inf"), float("nan"), 2.5, -1, "3", [1]])
def test_binding_refuses_what_is_no_count(v):
    t = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    fake = type("Cache", (), dict(dtype=torch.bfloat16, batch=2, kv_heads=2, dh=64))()
    bounds = kernels.PageBounds.__new__(kernels.PageBounds)
    bounds.cache = fake
    for args in ((v, 0, 1), (4, v, 1), (4, 0, v)):
        with pytest.raises(ValueError):
            kernels.block_attention(t, fake, bounds, *args)
    with pytest.raises(ValueError):
        bounds.update(v)


def test_what_is_written_lies_apart():
    t = torch.zeros(100)
    kernels._beside(t[10:20], t[:10], t[20:], t[20:].view(8, 10)[:, ::2], t[:0], t[15:15])
    for other in (t[19:], t[:11], t, t[15:16], t.view(10, 10)[:3, 0], t[12:14].expand(3, 2)):
        with pytest.raises(ValueError):
            kernels._beside(t[10:20], other)


def _on_the_host(monkeypatch):
    """A cache of host tensors in one buffer, for the checks that come before any call
    (those of the tensors' place left out)."""
    monkeypatch.setattr(kernels, "_need", lambda *a: None)
    monkeypatch.setattr(kernels, "_here", lambda *a: 0)
    shapes = {"k": ((6, 16, 2, 32), torch.uint8), "v": ((6, 16, 2, 32), torch.uint8),
              "k_scale": ((6, 16, 2, 2), torch.uint8), "v_scale": ((6, 16, 2, 2), torch.uint8),
              "table": ((2, 3), torch.int32), "length": ((2,), torch.int32), "seen": ((2,), torch.int32),
              "weight": ((2, 48), torch.float32), "pos": ((2, 48), torch.int32)}
    room = torch.zeros(1 << 16, dtype=torch.uint8)
    room = room[-room.data_ptr() % 16:]
    ts, at = {}, 0
    for name, (shape, dtype) in shapes.items():
        n = torch.Size(shape).numel() * dtype.itemsize
        ts[name] = room[at:at + n].view(dtype).view(shape)
        at += -(-n // 16) * 16 + 4096  # (apart, so that a tensor can begin beside one)
    c = type("Cache", (), dict(ts, dtype=torch.bfloat16, batch=2, kv_heads=2, dh=64, device=room.device))()
    c._spans = [(t.data_ptr(), t.data_ptr() + t.nbytes) for t in ts.values()]
    return c, ts


def _over(t, shape, dtype, end=True):
    """A tensor whose first 16 bytes hold the last one of another, or whose last 16
    (of fewer: all but 4) hold the first ones."""
    base, n = t.untyped_storage(), torch.Size(shape).numel() * dtype.itemsize
    room = torch.tensor([], dtype=torch.uint8).set_(base)
    at = (t.data_ptr() + t.nbytes - 1) // 16 * 16 if end else t.data_ptr() + (16 if n >= 16 else 4) - n
    at -= base.data_ptr()
    return None if at < 0 or at + n > len(room) else room[at:at + n].view(dtype).view(shape)


TENSORS = ["k", "v", "k_scale", "v_scale", "table", "length", "seen", "weight", "pos"]


@pytest.mark.parametrize("end", [True, False])
@pytest.mark.parametrize("name", TENSORS)
def test_page_bounds_lie_apart_from_the_cache(monkeypatch, name, end):
    c, ts = _on_the_host(monkeypatch)
    free = [torch.zeros(6, 2, 64, dtype=torch.bfloat16) for _ in range(2)]
    kernels.PageBounds(c, *free)
    t = _over(ts[name], (6, 2, 64), torch.bfloat16, end)
    if t is None:
        pytest.skip("nothing lies there")
    for lo, hi in ((t, free[0]), (free[0], t)):
        with pytest.raises(ValueError, match="overlap"):
            kernels.PageBounds(c, lo, hi)
    with pytest.raises(ValueError, match="overlap"):
        kernels.PageBounds(c, free[0], free[0])


@pytest.mark.parametrize("end", [True, False])
@pytest.mark.parametrize("name", TENSORS)
def test_block_attention_writes_apart_from_the_cache(monkeypatch, name, end):
    c, ts = _on_the_host(monkeypatch)
    bounds = kernels.PageBounds(c, *(torch.zeros(6, 2, 64, dtype=torch.bfloat16) for _ in range(2)))
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    t = _over(ts[name], (2, 4, 64), torch.bfloat16, end)
    if t is None:
        pytest.skip("nothing lies there")
    for out in (t, q, bounds.lo.view(-1)[256:].view(2, 4, 64), bounds.hi.view(-1)[:512].view(2, 4, 64)):
        with pytest.raises(ValueError, match="overlap"):
            kernels.block_attention(q, c, bounds, 2, out=out)


@pytest.mark.parametrize("end", [True, False])
@pytest.mark.parametrize("name", TENSORS)
def test_turned_queries_go_apart_from_the_cache(monkeypatch, name, end):
    c, ts = _on_the_host(monkeypatch)
    q, k, v = (torch.zeros(2, h, 64, dtype=torch.bfloat16) for h in (4, 2, 2))
    room = torch.zeros(1024, dtype=torch.bfloat16)
    freq, drop = room[:64].view(torch.float32), room[1020:].view(torch.int32)
    t = _over(ts[name], (2, 4, 64), torch.bfloat16, end)
    if t is None:
        pytest.skip("nothing lies there")
    for out in (t, q, room[:512].view(2, 4, 64), room[56:568].view(2, 4, 64), room[512:].view(2, 4, 64)):
        with pytest.raises(ValueError, match="overlap"):
            kernels.cache_append_rotary(c, q, k, v, freq, drop=drop, out=out)


# Bytes of each tensor of a cache (in 4 bits) and of the rows that join it: 2, of 4 or 2 heads
# of 64; 32 frequencies; 2 counts.
HELD = {"k": 8 * 16 * 64, "v": 8 * 16 * 64, "ks": 8 * 16 * 4, "vs": 8 * 16 * 4, "table": 2 * 4 * 4,
        "len": 8, "seen": 8, "weight": 2 * 64 * 4, "pos": 2 * 64 * 4}
ROWS = {"q": 1024, "k": 512, "v": 512, "q_out": 1024, "k_out": 512, "freq": 128, "drop": 8}


def _append(four, at):
    """Status and message of an append whose tensors lie at the given addresses (those of
    the rows with an r_ before their name), the others apart."""
    if torch.cuda.is_available():
        pytest.skip("a call that is not refused would run on these addresses")
    where = {n: (i + 1) << 20 for i, n in enumerate([*HELD, *("r_" + n for n in ROWS)])}
    where.update(at)
    st = {n: (16 * 64, 64, 32) if four else (16 * 128, 128, 64) for n in ("k_strides", "v_strides")}
    c = _cache(**{n: where[n] for n in HELD if n not in ("ks", "vs")}, **st)
    s = _scales(k=where["ks"], v=where["vs"], k_strides=(64, 4, 2), v_strides=(64, 4, 2)) if four else None
    r = _rows(**{n: where["r_" + n] for n in ROWS})
    rc = _native.lib().fusion_cache_append_rotary(byref(c), s and byref(s), byref(r), None, None)
    return rc, _native.lib().fusion_last_error().decode()


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("held", HELD)
@pytest.mark.parametrize("row", ROWS)
def test_appends_refuse_rows_that_overlap_the_cache(row, held, four):
    """From the first byte, and by the last 16 of either (calls without a fault, which would
    start a kernel, are in test_gpu_overlaps.py)."""
    if held in ("ks", "vs") and not four or held == "table" and not row.endswith("_out"):
        pytest.skip("not written")
    n = HELD[held] * (4 if not four and held in "kv" else 1)
    base = 1 << 28
    for at in (base, base + (n - 1) // 16 * 16, base + 16 - ROWS[row]):
        if row == "drop" and at != base:
            at = base + (4 if at > base else -4)  # (one count beside)
        elif row == "drop" and held in ("len", "seen"):
            continue  # drop may be these themselves
        rc, message = _append(four, {held: base, "r_" + row: at})
        assert rc == -1 and "overlap" in message, (hex(at), message)


def test_appends_refuse_outputs_that_overlap_rows():
    for out in ("q_out", "k_out"):
        for row in ROWS:
            if row == out:
                continue
            for at in (1 << 28, (1 << 28) + (ROWS[row] - 1) // 16 * 16, (1 << 28) + 16 - ROWS[out]):
                rc, message = _append(False, {"r_" + row: 1 << 28, "r_" + out: at})
                assert rc == -1 and "overlap" in message, (out, row, hex(at), message)


def test_appends_refuse_rows_whose_span_reaches_the_cache():
    """The second of two rows far apart, or a head, lies in the cache."""
    if torch.cuda.is_available():
        pytest.skip("a call that is not refused would run on these addresses")
    for strides in ((1 << 20, 64), (256, 1 << 20), (1 << 62, 64)):
        c, r = _cache(k=1 << 28, v=1 << 32, table=64, len=128, seen=192, weight=256, pos=1024), \
            _rows(q=(1 << 28) - (1 << 21), k=1 << 40, v=1 << 41, q_out=1 << 42, freq=1 << 43, q_strides=strides)
        assert _native.lib().fusion_cache_append_rotary(byref(c), None, byref(r), None, None) == -1
        assert "overlap" in _native.lib().fusion_last_error().decode()


@pytest.mark.parametrize("four", [False, True])
def test_bounds_and_blocks_refuse_overlaps(four):
    """Bounds, and the output, choice and workspace of block attention, over each other and
    each tensor that is read."""
    if torch.cuda.is_available():
        pytest.skip("a call that is not refused would run on these addresses")
    lib = _native.lib()
    st = {n: (16 * 64, 64, 32) if four else (16 * 128, 128, 64) for n in ("k_strides", "v_strides")}
    size = dict(HELD, lo=8 * 2 * 128, hi=8 * 2 * 128, q=1024, out=1024, chosen=2 * 2 * 4 * 4)
    if not four:
        size = dict(size, k=4 * size["k"], v=4 * size["v"])
        del size["ks"], size["vs"]

    def call(blocks, at):
        where = {n: (i + 1) << 24 for i, n in enumerate([*size, "ws"])}
        where.update(at)
        c = byref(_cache(**{n: where[n] for n in HELD if n not in ("ks", "vs")}, **st))
        s = byref(_scales(k=where["ks"], v=where["vs"], k_strides=(64, 4, 2), v_strides=(64, 4, 2))) if four else None
        if not blocks:
            rc = lib.fusion_page_bounds(c, s, where["lo"], where["hi"], 0, None)
        else:
            size["ws"] = lib.fusion_block_attention_workspace_bytes(c, s, 4, 4)
            rc = lib.fusion_block_attention(c, s, where["lo"], where["hi"], where["q"], _i64(256, 64), 4, 4, 1, 1,
                                            where["out"], where["chosen"], where["ws"], BIG, None)
        return rc, lib.fusion_last_error().decode()

    for blocks, written in ((False, ("lo", "hi")), (True, ("out", "chosen", "ws"))):
        call(blocks, {"lo": None})  # (a refusal: the workspace's size)
        read = [n for n in size if blocks or n not in ("q", "out", "chosen", "ws")]
        for w in written:
            for x in read:
                if x == w:
                    continue
                base, align = 1 << 40, 256 if "ws" in (w, x) else 16
                for at in (base, base + (size[x] - 1) // align * align, base + align - -(-size[w] // align) * align):
                    if at + size[w] <= base:
                        continue
                    rc, message = call(blocks, {x: base, w: at})
                    assert rc == -1 and "overlap" in message, (w, x, at - base, message)


@pytest.mark.parametrize("dh", [33, 48, 63, 65, 97, 0, -32])
def test_empty_caches_of_odd_widths_are_refused(monkeypatch, dh):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch, "zeros", lambda *a, **k: pytest.fail("memory was taken"))
    with pytest.raises(ValueError, match="multiple of 32"):
        kernels.TokenCache4.empty(1, 64, 2, dh)

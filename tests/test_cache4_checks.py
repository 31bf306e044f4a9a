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
    c._written = kernels._in_order([s for s, n in zip(c._spans, TENSORS) if n != "table"])
    c._size = 2
    c._c = _cache(len=c.length.data_ptr(), seen=c.seen.data_ptr())
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


@pytest.mark.parametrize("end", [True, False])
@pytest.mark.parametrize("name", TENSORS)
def test_rows_lie_apart_from_what_an_append_writes(monkeypatch, name, end):
    """(The table is read only; drop may be the lengths or the positions themselves.)"""
    c, ts = _on_the_host(monkeypatch)
    c._ready = lambda *a: None
    c._ref, c._scales = byref(c._c), None
    reached = []
    monkeypatch.setattr(kernels._native.lib(), "fusion_cache_append_rotary",
                        lambda *a: reached.append(a) or 0, raising=False)
    rows = [torch.zeros(2, h, 64, dtype=torch.bfloat16) for h in (4, 2, 2)]
    freq, drop = torch.zeros(32), torch.zeros(2, dtype=torch.int32)
    kernels.cache_append_rotary(c, *rows, freq, drop=drop)
    kernels.cache_append_rotary(c, *rows, freq, drop=c.length)
    kernels.cache_append_rotary(c, *rows, freq, drop=c.seen)
    kernels.cache_append_rotary(c, *(t[:0] for t in rows), freq, [0, 0, 0], drop=drop)
    assert len(reached) == 4
    for i in range(5):
        args = [*rows, freq, drop]
        shape = [2, (4, 2, 2)[i], 64] if i < 3 else args[i].shape
        t = _over(ts[name], shape, args[i].dtype, end)
        if t is None:
            continue
        args[i] = t
        if i == 4 and t.data_ptr() in (c.length.data_ptr(), c.seen.data_ptr()):
            continue
        if name == "table":
            kernels.cache_append_rotary(c, *args[:4], drop=args[4])
            continue
        with pytest.raises(ValueError, match="overlap"):
            kernels.cache_append_rotary(c, *args[:4], drop=args[4])
    # rows far apart, of which the second one is in the cache's values
    far = torch.tensor([], dtype=torch.bfloat16).set_(c.v.untyped_storage())
    at = (c.v.data_ptr() - far.data_ptr()) // 2 - 1024
    rows[0] = far.as_strided((2, 4, 64), (2048, 64, 1), at)
    with pytest.raises(ValueError, match="overlap"):
        kernels.cache_append_rotary(c, *rows, freq, drop=drop)
    rows[0] = far.as_strided((2, 4, 64), (512, 64, 1), at)
    kernels.cache_append_rotary(c, *rows, freq, drop=drop)


@pytest.mark.parametrize("dh", [33, 48, 63, 65, 97, 0, -32])
def test_empty_caches_of_odd_widths_are_refused(monkeypatch, dh):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch, "zeros", lambda *a, **k: pytest.fail("memory was taken"))
    with pytest.raises(ValueError, match="multiple of 32"):
        kernels.TokenCache4.empty(1, 64, 2, dh)

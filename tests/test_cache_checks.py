"""Host-side refusals of windowed attention and the token cache (CPU): the C
entries check every argument before any device call (the pointers here are
never dereferenced), and the binding refuses tensors it cannot pass on."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2607_02612_amd import _native, kernels

P = 4096  # a 256-byte aligned address


def _i64(*v):
    return (ctypes.c_int64 * len(v))(*v)


def _cu(*v):
    return np.array(v, np.int32)


def _window(**over):
    a = dict(precision=1, q=P, k=P, v=P, strides=_i64(256, 64, 128, 64, 128, 64), size=None,
             cu=_cu(0, 3, 7), batch=2, heads=4, kv_heads=2, dh=64, window=8, sinks=1, causal=1,
             out=P, stream=None)
    a.update(over)
    cu = a["cu"]
    a["cu"] = None if cu is None else cu.ctypes.data_as(ctypes.c_void_p)
    return _native.lib().fusion_window_attention(*a.values())


@pytest.mark.parametrize("bad", [
    dict(precision=2), dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(strides=None),
    dict(cu=None), dict(cu=_cu(1, 3, 7)), dict(cu=_cu(0, 5, 3)), dict(cu=_cu(0, 3, -1)),
    dict(cu=_cu(0, 3, (1 << 30) + 1)), dict(batch=0), dict(batch=65537), dict(heads=3), dict(heads=0),
    dict(kv_heads=0), dict(heads=8192), dict(dh=0), dict(dh=12), dict(dh=136), dict(window=-1),
    dict(sinks=-1), dict(causal=2), dict(q=P + 8), dict(out=P + 2),
    dict(strides=_i64(256, 64, 128, 64, 128, 60)), dict(strides=_i64(-256, 64, 128, 64, 128, 64)),
    dict(precision=0, strides=_i64(256, 64, 128, 64, 128, 66)),
])
def test_window_attention_refuses(bad):
    if bad.get("batch") == 65537:
        bad = dict(bad, cu=np.zeros(65538, np.int32))
    assert _window(**bad) == -1
    assert _native.lib().fusion_last_error().decode() != ""


def test_window_attention_without_rows_does_nothing():
    assert _window(cu=_cu(0, 0, 0)) == 0


def _cache(**over):
    a = dict(k=P, v=P, k_strides=(2048, 128, 64), v_strides=(2048, 128, 64), table=P, len=P, seen=P,
             weight=P, pos=P, precision=1, batch=2, pages=8, page_size=16, max_pages=4, kv_heads=2,
             dh=64)
    a.update(over)
    a["k_strides"], a["v_strides"] = _i64(*a["k_strides"]), _i64(*a["v_strides"])
    return _native.FusionCache(*a.values())


BAD_CACHES = [dict(k=None), dict(v=None), dict(table=None), dict(len=None), dict(seen=None),
              dict(weight=None), dict(pos=None), dict(precision=3), dict(batch=0),
              dict(batch=65537), dict(pages=0), dict(page_size=0), dict(max_pages=0),
              dict(page_size=1 << 20, max_pages=1 << 20), dict(kv_heads=0), dict(dh=4), dict(dh=136),
              dict(k=P + 8), dict(k_strides=(2048, 128, 60)), dict(v_strides=(2048, -128, 64))]


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_every_cache_call_refuses_a_bad_cache(bad):
    lib, c = _native.lib(), ctypes.byref(_cache(**bad))
    big = 1 << 40
    assert lib.fusion_cache_append(c, P, P, _i64(128, 64, 128, 64), None, None) == -1
    assert lib.fusion_paged_attention(c, P, _i64(256, 64), 4, 0, 0, 1, P, P, big, None) == -1
    assert lib.fusion_cache_evict(c, 8, 0, 0, P, P, big, None) == -1
    assert lib.fusion_paged_attention_workspace_bytes(c, 4, 1) == 0
    assert lib.fusion_cache_evict_workspace_bytes(c, 8) == 0


def test_cache_calls_refuse_bad_arguments():
    lib, c = _native.lib(), ctypes.byref(_cache())
    ok = _i64(128, 64, 128, 64)
    cu = lambda *v: _cu(*v).ctypes.data_as(ctypes.c_void_p)  # noqa: E731
    keep = _cu(0, 2, 1)
    assert lib.fusion_cache_append(None, P, P, ok, None, None) == -1
    for k, v, st, off in [(None, P, ok, None), (P, None, ok, None), (P, P, None, None),
                          (P + 8, P, ok, None), (P, P, _i64(128, 64, 128, 4), None),
                          (P, P, ok, keep.ctypes.data_as(ctypes.c_void_p))]:
        assert lib.fusion_cache_append(c, k, v, st, off, None) == -1
    zero = _cu(0, 0, 0)
    assert lib.fusion_cache_append(c, P, P, ok, zero.ctypes.data_as(ctypes.c_void_p), None) == 0

    need = lib.fusion_paged_attention_workspace_bytes(c, 4, 1)
    assert need >= lib.fusion_paged_attention_workspace_bytes(c, 4, 0) > 0
    assert lib.fusion_paged_attention_workspace_bytes(c, 3, 1) == 0
    q2 = _i64(256, 64)
    for q, st, heads, window, sinks, acc, out, ws, n, code in [
            (None, q2, 4, 0, 0, 1, P, P, need, -1), (P, None, 4, 0, 0, 1, P, P, need, -1),
            (P, q2, 3, 0, 0, 1, P, P, need, -1), (P, q2, 4, -1, 0, 1, P, P, need, -1),
            (P, q2, 4, 0, -1, 1, P, P, need, -1), (P, q2, 4, 0, 0, 2, P, P, need, -1),
            (P, q2, 4, 0, 0, 1, None, P, need, -1), (P + 4, q2, 4, 0, 0, 1, P, P, need, -1),
            (P, _i64(256, 63), 4, 0, 0, 1, P, P, need, -1), (P, q2, 4, 0, 0, 1, P, None, need, -1),
            (P, q2, 4, 0, 0, 1, P, P + 128, need, -1), (P, q2, 4, 0, 0, 1, P, P, need - 1, -3)]:
        assert lib.fusion_paged_attention(c, q, st, heads, window, sinks, acc, out, ws, n,
                                          None) == code

    need = lib.fusion_cache_evict_workspace_bytes(c, 8)
    assert need > 0 and lib.fusion_cache_evict_workspace_bytes(c, 0) == 0
    for budget, sinks, recent, src, ws, n, code in [
            (0, 0, 0, P, P, need, -1), ((1 << 30) + 1, 0, 0, P, P, need, -1),
            (8, -1, 0, P, P, need, -1), (8, 0, -1, P, P, need, -1), (8, 4, 5, P, P, need, -1),
            (8, 0, 0, None, P, need, -1), (8, 0, 0, P, None, need, -1),
            (8, 0, 0, P, P + 64, need, -1), (8, 0, 0, P, P, need - 1, -3)]:
        assert lib.fusion_cache_evict(c, budget, sinks, recent, src, ws, n, None) == code


@pytest.mark.parametrize("pages,page,maxp", [(1, 1, 1), (1 << 20, 27, 1000), (8, 1 << 30, 1)])
def test_workspaces_grow_with_the_capacity_only(pages, page, maxp):
    """4 bytes per head and slot for the scores and 8 per move, besides a part
    that goes by batch, heads and the chip alone."""
    lib, c = _native.lib(), ctypes.byref(_cache(pages=pages, page_size=page, max_pages=maxp))
    cap = page * maxp
    n0 = lib.fusion_paged_attention_workspace_bytes(c, 4, 0)
    n1 = lib.fusion_paged_attention_workspace_bytes(c, 4, 1)
    assert n1 - n0 <= 2 * 4 * (cap + 256) * 4 + 4096
    assert lib.fusion_cache_evict_workspace_bytes(c, 8) <= 2 * 8 * 8 + 1024


def test_binding_refuses_host_tensors_and_shapes():
    t = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    for q, k, v in [(t(4, 2, 64), t(4, 2, 64)[:, :, :32], t(4, 2, 64)), (t(4, 128), t(4, 2, 64), t(4, 2, 64)),
                    (t(4, 2, 64), None, t(4, 2, 64)), (t(4, 2, 64), t(4, 2, 64), t(4, 1, 64)),
                    (t(4, 2, 64).int(), t(4, 2, 64), t(4, 2, 64)),
                    (t(4, 64, 2).transpose(1, 2), t(4, 2, 64), t(4, 2, 64))]:
        with pytest.raises(ValueError):
            kernels.window_attention(q, k, v, [0, 4])
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError):  # host tensors
        kernels.TokenCache(t(8, 16, 2, 64), t(8, 16, 2, 64), i32(2, 4), i32(2), i32(2),
                           torch.zeros(2, 64), i32(2, 64))


def test_binding_refuses_tangents():
    """A dual tensor's tangent would be dropped in silence."""
    from torch.autograd import forward_ad
    t = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    fake = type("Cache", (), dict(dtype=torch.bfloat16, batch=4, kv_heads=2, dh=64))()
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(t, torch.ones_like(t))
        size = forward_ad.make_dual(torch.ones(4), torch.ones(4))
        for call in [lambda: kernels.window_attention(dual, t, t, [0, 4]),
                     lambda: kernels.window_attention(t, dual, t, [0, 4]),
                     lambda: kernels.window_attention(t, t, dual, [0, 4]),
                     lambda: kernels.cache_append(fake, dual, t),
                     lambda: kernels.cache_append(fake, t, dual),
                     lambda: kernels.paged_attention(dual, fake)]:
            with pytest.raises(ValueError, match="tangent"):
                call()
        with pytest.raises(ValueError, match="tangent"):
            kernels._no_grad(size, "size")
        kernels._no_grad(t, "q")  # without a tangent it passes
    kernels._no_grad(t, "q")


@pytest.mark.parametrize("budget,sinks,recent", [
    ((1 << 30) + 1, 0, 0), (1 << 31, 0, 0), (1 << 40, 4, 64), (1 << 30, 0, (1 << 30) + 1),
    (1 << 30, 1 << 31, 0), (1 << 30, 1 << 29, (1 << 29) + 1), (0, 0, 0), (8, 4, 5), (8.5, 0, 0)])
def test_binding_refuses_budgets(budget, sinks, recent):
    """A budget beyond the library's range is refused, not cut (the result
    would have another shape), nor are the counts that have to fit it."""
    with pytest.raises(ValueError):
        kernels.cache_evict(None, budget, sinks, recent)


@pytest.mark.parametrize("v", [float("inf"), -float("inf"), float("nan"), 2.5, -1, None, "3", [1]])
def test_binding_refuses_what_is_no_count(v):
    for budget, sinks, recent in ((v, 0, 0), (8, v, 0), (8, 0, v)):
        with pytest.raises(ValueError):
            kernels.cache_evict(None, budget, sinks, recent)
    t = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    fake = type("Cache", (), dict(dtype=torch.bfloat16, batch=2, kv_heads=2, dh=64))()
    if v is not None:  # (no window)
        with pytest.raises(ValueError, match="window"):
            kernels.paged_attention(t, fake, window=v)

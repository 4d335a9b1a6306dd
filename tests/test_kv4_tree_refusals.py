"""What the calls for drafted trees and sliding windows on the paged 4-bit KV cache refuse, without a GPU: every check comes before anything is
launched, so addresses that were never allocated do for the arguments."""

import ctypes

import pytest
import torch

from test_kv4_refusals import (ALIGN, BAD_CACHES, NULL, OK, SCALE, SHAPE, UNSUPPORTED, WORKSPACE, attention_args, b, cache, host_cache,   # noqa: F401
                               place)

I32 = (1 << 31) - 1


# ---- attention
def window_args(b, cache_over={}, window=100, sinks=4, **over):
    a = attention_args(b, cache_over, **over)
    i = len(a) - 5                                                 # causal, out, workspace, its bytes, stream
    return a[:i] + [window, sinks] + a[i + 1:]


def tree_args(b, cache_over={}, mask=place(18), words=2, window=0, sinks=0, **over):
    a = attention_args(b, cache_over, **over)
    i = len(a) - 5
    return a[:i] + [mask, words, window, sinks] + a[i + 1:]


COMMON = [(dict(cache=None), NULL), (dict(T=-1), SHAPE), (dict(T=1 << 28), SHAPE), (dict(B=-1), SHAPE), (dict(n_heads=0), SHAPE), (dict(n_heads=5), SHAPE),
          (dict(max_q=0), SHAPE), (dict(table_pages=0), SHAPE), (dict(table_pages=1 << 24), SHAPE), (dict(n_prefix=-1), SHAPE),
          (dict(row_stride=4 * 128 - 8), SHAPE), (dict(row_stride=4 * 128 + 2), SHAPE), (dict(scale=0.0), SCALE), (dict(scale=float("nan")), SCALE),
          (dict(q=None), NULL), (dict(cu_q=None), NULL), (dict(kv_len=None), NULL), (dict(table=None), NULL), (dict(out=None), NULL),
          (dict(n_prefix=3, prefix_k=place(14)), NULL), (dict(q=place(10) + 8), ALIGN), (dict(out=place(16) + 8), ALIGN), (dict(cu_q=place(11) + 2), ALIGN),
          (dict(ws=place(17) + 128), ALIGN), (dict(out=place(10)), UNSUPPORTED), (dict(ws=None), WORKSPACE), (dict(ws_bytes=0), WORKSPACE),
          (dict(window=-1), SHAPE), (dict(window=-I32 - 1), SHAPE), (dict(sinks=-1), SHAPE), (dict(sinks=-I32 - 1), SHAPE)]


@pytest.mark.parametrize("over,status", COMMON + [(dict(window=0), SHAPE)])
def test_window_attention(b, over, status):
    assert b.status_str(b.lib().pq_kv4_window_attention(*window_args(b, **over))) == status


@pytest.mark.parametrize("over,status", COMMON + [
    (dict(words=0), SHAPE), (dict(words=-1), SHAPE), (dict(words=9), SHAPE), (dict(words=I32), SHAPE), (dict(mask=None), NULL), (dict(mask=place(18) + 2), ALIGN),
    (dict(mask=place(16)), UNSUPPORTED), (dict(mask=place(16) - 36), UNSUPPORTED), (dict(mask=place(16) + 5 * 1024 - 4), UNSUPPORTED)])
def test_tree_attention(b, over, status):
    assert b.status_str(b.lib().pq_kv4_tree_attention(*tree_args(b, **over))) == status


@pytest.mark.parametrize("over,status", BAD_CACHES)
def test_caches(b, over, status):
    L = b.lib()
    assert b.status_str(L.pq_kv4_window_attention(*window_args(b, over))) == status
    assert b.status_str(L.pq_kv4_tree_attention(*tree_args(b, over))) == status
    assert b.status_str(L.pq_kv4_keep(*keep_args(b, [{}, over] if over.get("n_pages") is None else [over]))) == status


def test_workspaces(b):
    L = b.lib()
    c = cache(b)
    for name, args, least in (("pq_kv4_window_attention", window_args, 1), ("pq_kv4_tree_attention", tree_args, 0)):
        need = getattr(L, name + "_workspace_bytes")
        n = need(5, 2, 4, 3, 16, 100, 4, c)
        assert n > 0 and n % 256 == 0
        assert b.status_str(getattr(L, name)(*args(b, window=100, sinks=4, ws_bytes=n - 1))) == WORKSPACE
        for bad in ((0, 2, 4, 3, 16, 100, 4), (5, 0, 4, 3, 16, 100, 4), (5, 2, 3, 3, 16, 100, 4), (5, 2, 4, 0, 16, 100, 4), (5, 2, 4, 3, 0, 100, 4),
                    (5, 2, 4, 3, 16, least - 1, 4), (5, 2, 4, 3, 16, 100, -1), (5, 2, 4, 3, 1 << 24, 100, 4)):
            assert need(*bad, c) == 0, bad
        assert need(5, 2, 4, 3, 16, 100, 4, None) == 0
        # no more than without a window, and within the documented bound
        for T in (1, 7, 64, 300, 4096, 100000, 1 << 20):
            for B in (1, 3, 64, 1000):
                for heads, kv in ((1, 1), (32, 8), (64, 8)):
                    for most in (1, 4, 17, 100, 1 << 30, I32):
                        for window in (1, 100, 5000, I32):
                            for sinks in (0, 100, I32):
                                got = need(T, B, heads, most, 5000, window, sinks, cache(b, n_kv_heads=kv))
                                assert 0 < got <= (160 << 20) + 2 * (T * heads + 16 * B * kv), (T, B, heads, kv, most, window, sinks)


# ---- tree
def tree_plan_args(**over):
    a = dict(parents=place(1), cu_q=place(2), kv_len=place(3), B=3, T=7, words=2, offset=0, mask=place(4), positions=place(5), stream=None)
    assert set(over) <= set(a)
    a.update(over)
    return list(a.values())


@pytest.mark.parametrize("over,status", [
    (dict(B=-1), SHAPE), (dict(B=1 << 26), SHAPE), (dict(T=-1), SHAPE), (dict(T=1 << 30), SHAPE), (dict(words=0), SHAPE), (dict(words=9), SHAPE),
    (dict(offset=-1), SHAPE), (dict(parents=None), NULL), (dict(cu_q=None), NULL), (dict(kv_len=None), NULL), (dict(mask=None), NULL),
    (dict(positions=None), NULL), (dict(parents=place(1) + 2), ALIGN), (dict(mask=place(4) + 1), ALIGN), (dict(positions=place(5) + 2), ALIGN),
    (dict(cu_q=place(2) + 3), ALIGN), (dict(kv_len=place(3) + 2), ALIGN), (dict(mask=place(1)), UNSUPPORTED), (dict(mask=place(1) + 24), UNSUPPORTED),
    (dict(positions=place(1)), UNSUPPORTED), (dict(positions=place(3) + 8), UNSUPPORTED), (dict(mask=place(2) - 52), UNSUPPORTED),
    (dict(mask=place(5) - 52), UNSUPPORTED), (dict(T=0, parents=None, cu_q=None, mask=None, positions=None), OK)])
def test_tree(b, over, status):
    assert b.status_str(b.lib().pq_kv4_tree(*tree_plan_args(**over))) == status


# ---- accept
def accept_args(**over):
    a = dict(tokens=place(1), parents=place(2), chosen=place(3), cu_q=place(4), kv_len=place(5), B=3, T=7, words=2, depth=5, table=place(6), table_pages=10,
             page_size=64, free=place(7), n_free=50, taken=place(8), accepted=place(9), next_token=place(10), path=place(11), kv_len_out=place(12),
             from_slots=place(13), to_slots=place(14), taken_out=place(15), stream=None)
    assert set(over) <= set(a)
    a.update(over)
    return list(a.values())


@pytest.mark.parametrize("over,status", [
    (dict(B=-1), SHAPE), (dict(B=1 << 26), SHAPE), (dict(T=-1), SHAPE), (dict(T=1 << 30), SHAPE), (dict(words=0), SHAPE), (dict(words=9), SHAPE),
    (dict(depth=0), SHAPE), (dict(depth=65), SHAPE), (dict(depth=-3), SHAPE), (dict(table_pages=0), SHAPE), (dict(table_pages=1 << 24), SHAPE),
    (dict(page_size=8), SHAPE), (dict(page_size=48), SHAPE), (dict(n_free=-1), SHAPE)] + [
    ({n: None}, NULL) for n in ("tokens", "parents", "chosen", "cu_q", "kv_len", "table", "free", "taken", "accepted", "next_token", "path", "kv_len_out",
                                "from_slots", "to_slots", "taken_out")] + [
    (dict(tokens=place(1) + 2), ALIGN), (dict(free=place(7) + 1), ALIGN), (dict(path=place(11) + 2), ALIGN), (dict(from_slots=place(13) + 4), ALIGN),
    (dict(to_slots=place(14) + 4), ALIGN), (dict(taken_out=place(8)), UNSUPPORTED), (dict(kv_len_out=place(5)), UNSUPPORTED),
    (dict(accepted=place(5) + 8), UNSUPPORTED), (dict(next_token=place(3) + 24), UNSUPPORTED), (dict(path=place(6) + 116), UNSUPPORTED),
    (dict(free=place(6) + 76), UNSUPPORTED), (dict(from_slots=place(1) - 112), UNSUPPORTED), (dict(to_slots=place(8) - 112), UNSUPPORTED)])
def test_accept(b, over, status):
    assert b.status_str(b.lib().pq_kv4_accept(*accept_args(**over))) == status


# ---- keep
def keep_args(b, layers=({},), **over):
    a = dict(from_slots=place(6), to_slots=place(7), B=3, width=5, caches=(b.KV4Cache * max(len(layers), 1))(*(cache(b, **x) for x in layers)),
             n=len(layers), stream=None)
    assert set(over) <= set(a)
    a.update(over)
    return list(a.values())


@pytest.mark.parametrize("over,status", [
    (dict(B=-1), SHAPE), (dict(B=1 << 26), SHAPE), (dict(width=0), SHAPE), (dict(width=257), SHAPE), (dict(width=-1), SHAPE), (dict(n=-1), SHAPE),
    (dict(caches=None), NULL), (dict(from_slots=None), NULL), (dict(to_slots=None), NULL), (dict(from_slots=place(6) + 4), ALIGN),
    (dict(to_slots=place(7) + 2), ALIGN), (dict(B=0, from_slots=None, to_slots=None), OK), (dict(n=0, caches=None, from_slots=None), OK)])
def test_keep(b, over, status):
    assert b.status_str(b.lib().pq_kv4_keep(*keep_args(b, **over))) == status


def test_keep_wants_layers_of_one_kind(b):
    for other in (dict(n_pages=101), dict(n_kv_heads=4), dict(head_dim=64), dict(page_size=32), dict(group=32)):
        assert b.status_str(b.lib().pq_kv4_keep(*keep_args(b, [{}, other]))) == SHAPE
    assert b.status_str(b.lib().pq_kv4_keep(*keep_args(b, [dict(n_kv_heads=1 << 20)], B=1 << 10))) == SHAPE


def test_nothing_to_do(b):
    L = b.lib()
    none = dict(q=None, cu_q=None, kv_len=None, table=None, out=None, ws=None, ws_bytes=0)
    for zero in (dict(T=0), dict(B=0)):
        assert b.status_str(L.pq_kv4_window_attention(*window_args(b, **zero, **none))) == OK
        assert b.status_str(L.pq_kv4_tree_attention(*tree_args(b, mask=None, **zero, **none))) == OK
    assert b.status_str(L.pq_kv4_window_attention(*window_args(b, window=0, T=0, **none))) == SHAPE


# ---- the Python entry points
def test_python_wants_tensors_on_the_gpu(b):
    i, i64 = torch.zeros(2, dtype=torch.int32), torch.zeros((2, 3), dtype=torch.int64)
    table, q, ws = torch.zeros((2, 3), dtype=torch.int32), torch.zeros((2, 2 * 64)).half(), torch.zeros(4096, dtype=torch.uint8)
    cu = torch.zeros(3, dtype=torch.int32)
    for out, w in ((None, None), (q.clone(), ws)):
        with pytest.raises(TypeError):
            b.pq_kv4_window_attention(q, cu, i, table, *host_cache(), 0.1, 1, 5, out=out, workspace=w)
        with pytest.raises(TypeError):
            b.pq_kv4_tree_attention(q, cu, i, table, *host_cache(), 0.1, 1, table[:, :1].contiguous(), out=out, workspace=w)
    for outs in ({}, dict(mask=table, positions=i)):
        with pytest.raises(TypeError):
            b.pq_kv4_tree(i, cu, i, 1, **outs)
    for outs in ({}, dict(accepted=i, next_token=i, path=table, kv_len_out=i, from_slots=i64, to_slots=i64, taken_out=i)):
        with pytest.raises(TypeError):
            b.pq_kv4_accept(i, i, i, cu, i, table, 16, 1, 3, **outs)
    with pytest.raises(TypeError):
        b.KV4Layers([host_cache()])


def test_python_checks_shapes(b, monkeypatch):
    """On the CPU, with the checks of the device taken out of the way: the sizes' own checks, before the library is called."""
    b.lib()
    monkeypatch.setattr(b, "_here", lambda t, dtype, what: None)
    monkeypatch.setattr(b, "_rows", lambda t, what: None)
    monkeypatch.setattr(b, "_stream", lambda: None)
    monkeypatch.setattr(b, "_call", b._Declines)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)
    called = []
    real = b.lib()
    names = [n for n in b.SIGNATURES if n.startswith("pq_kv4")]
    monkeypatch.setattr(b, "lib", lambda: type("L", (), {**{n: staticmethod(lambda *a: called.append(a) or 0) for n in names},
                                                         "pq_status_str": real.pq_status_str}))
    i32 = lambda *n: torch.zeros(n, dtype=torch.int32)

    def refused(f, *a, error=ValueError, **k):
        with pytest.raises(error):
            f(*a, **k)

    refused(b.pq_kv4_tree, i32(5), i32(2), i32(2), 1)
    refused(b.pq_kv4_tree, i32(5), i32(3), i32(2), 2, mask=i32(5, 1))
    refused(b.pq_kv4_tree, i32(5), i32(3), i32(2), 2, positions=i32(4))
    accept = lambda *a, **k: refused(b.pq_kv4_accept, *a, **k)
    accept(i32(5), i32(4), i32(5), i32(3), i32(2), i32(2, 3), 16, 1, 3)
    accept(i32(5), i32(5), i32(6), i32(3), i32(2), i32(2, 3), 16, 1, 3)
    accept(i32(5), i32(5), i32(5), i32(2), i32(2), i32(2, 3), 16, 1, 3)
    accept(i32(5), i32(5), i32(5), i32(3), i32(2), i32(3, 3), 16, 1, 3)
    accept(i32(5), i32(5), i32(5), i32(3), i32(2), i32(6), 16, 1, 3)
    accept(i32(5), i32(5), i32(5), i32(3), i32(2), i32(2, 3), 16, 1, 3, free_pages=i32(4))
    accept(i32(5), i32(5), i32(5), i32(3), i32(2), i32(2, 3), 16, 1, 3, taken=i32(1))
    accept(i32(5), i32(5), i32(5), i32(3), i32(2), i32(2, 3), 16, 1, 3, free_pages=i32(4), taken=i32(0))
    for name, small in (("accepted", i32(1)), ("next_token", i32(1)), ("path", i32(5)), ("kv_len_out", i32(1)), ("taken_out", i32(0)),
                        ("from_slots", torch.zeros(5, dtype=torch.int64)), ("to_slots", torch.zeros(5, dtype=torch.int64))):
        accept(i32(5), i32(5), i32(5), i32(3), i32(2), i32(2, 3), 16, 1, 3, **{name: small})
    accept(i32(5), i32(5), i32(5), i32(3), i32(2), i32(2, 3), 16, 1, 0, error=b.PQError)

    codes, q = host_cache(), torch.zeros((2, 2 * 64)).half()
    refused(b.pq_kv4_tree_attention, q, i32(3), i32(2), i32(2, 3), *codes, 0.1, 1, i32(3, 1))
    refused(b.pq_kv4_tree_attention, q, i32(3), i32(2), i32(2, 3), *codes, 0.1, 1, i32(2))
    for f, more in ((b.pq_kv4_window_attention, (7,)), (b.pq_kv4_tree_attention, (i32(2, 1),))):
        refused(f, q, i32(2), i32(2), i32(2, 3), *codes, 0.1, 1, *more)
        refused(f, q, i32(3), i32(2), i32(1, 3), *codes, 0.1, 1, *more)
        refused(f, q[:, :100], i32(3), i32(2), i32(2, 3), *codes, 0.1, 1, *more)
        refused(f, q, i32(3), i32(2), i32(2, 3), *codes, 0.1, 1, *more, prefix_k=torch.zeros((1, 2, 64)).half())
    refused(b.KV4Layers, [])
    refused(b.KV4Layers, [codes, host_cache(pages=4)])
    refused(b.KV4Layers, [codes[:2] + (codes[2][:1], codes[3])])
    refused(b.KV4Layers, [codes, codes])                            # what one of them had moved, the other would move again
    refused(b.KV4Layers, [(codes[0], codes[0]) + codes[2:]])
    both, steps = torch.zeros((5, 2, 16, 32), dtype=torch.uint8), [torch.ones((3, 2, 16, 1)) for _ in range(4)]
    refused(b.KV4Layers, [codes, (both[:3], both[2:]) + codes[2:]])
    refused(b.KV4Layers, [codes[:2] + (steps[0], steps[1]), host_cache()[:2] + (steps[1], steps[2])], 64)
    assert b.KV4Layers([codes[:2] + (steps[0], steps[1]), host_cache()[:2] + (steps[2], steps[3])], 64).count == 2
    layers = b.KV4Layers([codes, host_cache()[:2] + codes[2:]])     # (static steps do not move)
    assert layers.count == 2 and layers.address == ctypes.addressof(layers.caches)
    slots = torch.zeros((2, 3), dtype=torch.int64)
    refused(b.pq_kv4_keep, slots, slots[:1], layers)
    refused(b.pq_kv4_keep, slots[0], slots[0], layers)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    refused(b.pq_kv4_keep, slots, slots, layers)
    assert all(len(a) in (8, 1) for a in called)                    # (sizes of a workspace at most)


def test_native_calls_decline_what_is_not_plain(b):
    i, table, q = torch.zeros(2, dtype=torch.int32), torch.zeros((2, 3), dtype=torch.int32), torch.zeros((2, 2 * 64)).half()
    slots, c = torch.zeros((2, 3), dtype=torch.int64), b._call
    assert c.kv4_tree() == c.kv4_accept() == c.kv4_keep() == c.kv4_window_attention() == c.kv4_tree_attention() == -1
    assert c.kv4_tree(i, i, i, 1, 0, table, i) == -1
    assert c.kv4_accept(i, i, i, i, i, table, 16, 1, 3, None, None, i, i, table, i, slots, slots, i) == -1
    assert c.kv4_keep(slots, slots, 1 << 32, 1, 0) == -1 and c.kv4_keep(slots, slots, 0, 1, 0) == -1
    ws = torch.zeros(64, dtype=torch.uint8)
    assert c.kv4_window_attention(q, i, i, table, *host_cache(), 0.1, 1, 0, None, None, 5, 0, q, ws) == -1
    assert c.kv4_tree_attention(q, i, i, table, *host_cache(), 0.1, 1, 0, None, None, table, 5, 0, q, ws) == -1

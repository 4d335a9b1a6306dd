"""What the calls on the paged 4-bit KV cache refuse, without a GPU: every check comes before anything is launched, so addresses that
were never allocated do for the arguments."""

import ctypes

import pytest
import torch

NULL, SHAPE, UNSUPPORTED, SCALE, ALIGN, WORKSPACE, OK = "PQ_ERR_NULL", "PQ_ERR_SHAPE", "PQ_ERR_UNSUPPORTED", "PQ_ERR_SCALE", "PQ_ERR_ALIGN", "PQ_ERR_WORKSPACE", "PQ_OK"
AT = 1 << 32                       # arguments' made-up addresses, 1 GiB apart


def place(i):
    return AT + (i << 30)


@pytest.fixture(scope="module")
def b():
    import paper_2410_05265_amd.binding as binding
    binding.lib()
    return binding


def cache(b, **over):
    c = dict(k_codes=place(1), v_codes=place(2), k_scale=place(3), v_scale=place(4), n_pages=100, n_kv_heads=2, head_dim=128, page_size=64, group=0)
    c.update(over)
    return b.KV4Cache(*c.values())


BAD_CACHES = [(dict(k_codes=None), NULL), (dict(v_codes=None), NULL), (dict(k_scale=None), NULL), (dict(v_scale=None), NULL),
              (dict(n_pages=0), SHAPE), (dict(n_pages=-1), SHAPE), (dict(n_pages=1 << 31), SHAPE), (dict(n_kv_heads=0), SHAPE),
              (dict(page_size=0), SHAPE), (dict(page_size=8), SHAPE), (dict(page_size=48), SHAPE), (dict(page_size=2048), SHAPE),
              (dict(page_size=-64), SHAPE), (dict(head_dim=32), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED),
              (dict(group=16), SHAPE), (dict(group=-1), SHAPE), (dict(group=256), SHAPE), (dict(group=128, head_dim=64), SHAPE),
              (dict(k_codes=place(1) + 8), ALIGN), (dict(v_codes=place(2) + 4), ALIGN), (dict(k_scale=place(3) + 2), ALIGN),
              (dict(group=64, v_scale=place(4) + 4), ALIGN)]


# ---- slots
def slots_args(**over):
    a = dict(kv_len=place(1), q_len=place(2), B=3, table=place(3), table_pages=10, free=place(4), n_free=50, taken=None, page_size=64, T=7,
             offset=0, cu_q=place(5), kv_len_out=place(6), positions=place(7), slots=place(8), taken_out=place(9), stream=None)
    assert set(over) <= set(a)
    a.update(over)
    return list(a.values())


@pytest.mark.parametrize("over,status", [
    (dict(B=-1), SHAPE), (dict(B=1 << 26), SHAPE), (dict(T=-1), SHAPE), (dict(T=1 << 31), SHAPE), (dict(table_pages=0), SHAPE),
    (dict(n_free=-1), SHAPE), (dict(offset=-1), SHAPE), (dict(page_size=0), SHAPE), (dict(page_size=24), SHAPE), (dict(page_size=2048), SHAPE),
    (dict(kv_len=None), NULL), (dict(q_len=None), NULL), (dict(table=None), NULL), (dict(free=None), NULL), (dict(cu_q=None), NULL),
    (dict(kv_len_out=None), NULL), (dict(positions=None), NULL), (dict(slots=None), NULL), (dict(taken_out=None), NULL),
    (dict(kv_len=place(1) + 2), ALIGN), (dict(table=place(3) + 1), ALIGN), (dict(taken=place(10) + 2), ALIGN), (dict(slots=place(8) + 4), ALIGN),
    (dict(kv_len_out=place(1)), UNSUPPORTED), (dict(kv_len_out=place(1) + 8), UNSUPPORTED), (dict(cu_q=place(2) - 4), UNSUPPORTED),
    (dict(positions=place(4) + 196), UNSUPPORTED), (dict(taken=place(9), taken_out=place(9)), UNSUPPORTED), (dict(table=place(1) - 116), UNSUPPORTED),
    (dict(slots=place(4) - 48), UNSUPPORTED)])
def test_slots(b, over, status):
    assert b.status_str(b.lib().pq_kv4_slots(*slots_args(**over))) == status


# ---- append
def append_args(b, cache_over={}, **over):
    a = dict(qkv=place(10), row_stride=8 * 128, T=5, n_heads=4, positions=place(11), slots=place(12), q_weight=place(13), k_weight=place(14),
             eps=1e-6, cos_sin=place(15), max_positions=64, rotary_dim=128, interleaved=0, rotate=1, clip=1.0, cache=cache(b, **cache_over),
             q_out=place(16), stream=None)
    assert set(over) <= set(a)
    a.update(over)
    return list(a.values())


@pytest.mark.parametrize("over,status", [
    (dict(cache=None), NULL), (dict(T=-1), SHAPE), (dict(T=1 << 25), SHAPE), (dict(n_heads=0), SHAPE), (dict(n_heads=3), SHAPE),
    (dict(n_heads=65534, row_stride=65538 * 128), SHAPE), (dict(T=1 << 24, n_heads=512, row_stride=516 * 128), SHAPE),
    (dict(row_stride=8 * 128 - 8), SHAPE), (dict(row_stride=8 * 128 + 4), SHAPE),
    (dict(max_positions=0), SHAPE), (dict(rotary_dim=0), SHAPE), (dict(rotary_dim=8), SHAPE), (dict(rotary_dim=24), SHAPE), (dict(rotary_dim=144), SHAPE),
    (dict(eps=-1e-6), SHAPE), (dict(eps=float("nan")), SHAPE), (dict(eps=float("inf")), SHAPE),
    (dict(clip=0.0), SCALE), (dict(clip=-0.5), SCALE), (dict(clip=1.5), SCALE), (dict(clip=float("nan")), SCALE),
    (dict(qkv=None), NULL), (dict(slots=None), NULL), (dict(q_out=None), NULL), (dict(positions=None), NULL),
    (dict(qkv=place(10) + 8), ALIGN), (dict(q_out=place(16) + 2), ALIGN), (dict(q_weight=place(13) + 8), ALIGN), (dict(k_weight=place(14) + 8), ALIGN),
    (dict(cos_sin=place(15) + 4), ALIGN), (dict(positions=place(11) + 2), ALIGN), (dict(slots=place(12) + 4), ALIGN),
    (dict(q_out=place(10)), UNSUPPORTED), (dict(q_out=place(10) + 5 * 2048 - 16), UNSUPPORTED)])
def test_append(b, over, status):
    assert b.status_str(b.lib().pq_kv4_append(*append_args(b, **over))) == status


# ---- attention
def attention_args(b, cache_over={}, **over):
    a = dict(q=place(10), row_stride=4 * 128, T=5, n_heads=4, cu_q=place(11), kv_len=place(12), B=2, max_q=3, table=place(13), table_pages=16,
             cache=cache(b, **cache_over), prefix_k=None, prefix_v=None, n_prefix=0, scale=0.1, causal=1, out=place(16), ws=place(17),
             ws_bytes=1 << 28, stream=None)
    assert set(over) <= set(a)
    a.update(over)
    return list(a.values())


def need(b, T=5, B=2, n_heads=4, max_q=3, table_pages=16, **cache_over):
    return b.lib().pq_kv4_attention_workspace_bytes(T, B, n_heads, max_q, table_pages, cache(b, **cache_over))


@pytest.mark.parametrize("over,status", [
    (dict(cache=None), NULL), (dict(T=-1), SHAPE), (dict(T=1 << 28), SHAPE), (dict(T=1 << 62), SHAPE), (dict(B=-1), SHAPE), (dict(B=1 << 20), SHAPE),
    (dict(n_heads=0), SHAPE), (dict(n_heads=5), SHAPE), (dict(max_q=0), SHAPE), (dict(table_pages=0), SHAPE), (dict(table_pages=1 << 24), SHAPE),
    (dict(n_prefix=-1), SHAPE), (dict(n_prefix=1025, prefix_k=place(14), prefix_v=place(15)), SHAPE),
    (dict(row_stride=4 * 128 - 8), SHAPE), (dict(row_stride=4 * 128 + 2), SHAPE),
    (dict(scale=0.0), SCALE), (dict(scale=-1.0), SCALE), (dict(scale=float("inf")), SCALE), (dict(scale=float("nan")), SCALE),
    (dict(q=None), NULL), (dict(cu_q=None), NULL), (dict(kv_len=None), NULL), (dict(table=None), NULL), (dict(out=None), NULL),
    (dict(n_prefix=3, prefix_k=place(14)), NULL), (dict(n_prefix=3, prefix_v=place(14)), NULL),
    (dict(q=place(10) + 8), ALIGN), (dict(out=place(16) + 8), ALIGN), (dict(cu_q=place(11) + 2), ALIGN), (dict(kv_len=place(12) + 1), ALIGN),
    (dict(table=place(13) + 2), ALIGN), (dict(n_prefix=3, prefix_k=place(14) + 8, prefix_v=place(15)), ALIGN), (dict(ws=place(17) + 128), ALIGN),
    (dict(out=place(10)), UNSUPPORTED), (dict(out=place(10) + 5 * 1024 - 16), UNSUPPORTED), (dict(ws=None), WORKSPACE), (dict(ws_bytes=0), WORKSPACE)])
def test_attention(b, over, status):
    assert b.status_str(b.lib().pq_kv4_attention(*attention_args(b, **over))) == status


def test_attention_workspace(b):
    n = need(b)
    assert n > 0 and n % 256 == 0
    assert b.status_str(b.lib().pq_kv4_attention(*attention_args(b, ws_bytes=n - 1))) == WORKSPACE
    for bad in (dict(T=0), dict(T=-1), dict(B=0), dict(n_heads=3), dict(max_q=0), dict(table_pages=0), dict(table_pages=1 << 24), dict(T=1 << 28),
                dict(B=1 << 20), dict(head_dim=96), dict(page_size=20), dict(group=7), dict(n_pages=0)):
        assert need(b, **bad) == 0, bad
    assert b.lib().pq_kv4_attention_workspace_bytes(5, 2, 4, 3, 16, None) == 0
    # the pointers and the kind of steps do not matter
    assert need(b, k_codes=None, v_codes=None, k_scale=None, v_scale=None) == n
    # the documented bound, over the range of sizes
    for T in (1, 7, 64, 300, 4096, 100000, 1 << 20):
        for B in (1, 3, 64, 1000):
            for heads, kv in ((1, 1), (8, 8), (32, 8), (64, 8), (48, 3)):
                for most in (1, 4, 17, 100, 1 << 30):
                    for pages in (1, 30, 5000):
                        for D in (64, 128):
                            got = need(b, T=T, B=B, n_heads=heads, max_q=most, table_pages=pages, n_kv_heads=kv, head_dim=D)
                            assert 0 < got <= (160 << 20) + 2 * (T * heads + 16 * B * kv), (T, B, heads, kv, most, pages, D)


@pytest.mark.parametrize("over,status", BAD_CACHES)
def test_caches(b, over, status):
    assert b.status_str(b.lib().pq_kv4_append(*append_args(b, over))) == status
    assert b.status_str(b.lib().pq_kv4_attention(*attention_args(b, over))) == status


def test_nothing_to_do(b):
    """No tokens: sizes and cache are checked, the rest may be absent."""
    L = b.lib()
    none = dict(qkv=None, positions=None, slots=None, q_weight=None, k_weight=None, cos_sin=None, q_out=None)
    assert b.status_str(L.pq_kv4_append(*append_args(b, T=0, **none))) == OK
    assert b.status_str(L.pq_kv4_append(*append_args(b, dict(page_size=20), T=0, **none))) == SHAPE
    none = dict(q=None, cu_q=None, kv_len=None, table=None, out=None, ws=None, ws_bytes=0)
    assert b.status_str(L.pq_kv4_attention(*attention_args(b, T=0, **none))) == OK
    assert b.status_str(L.pq_kv4_attention(*attention_args(b, B=0, **none))) == OK
    assert b.status_str(L.pq_kv4_attention(*attention_args(b, dict(k_codes=None), T=0, **none))) == NULL


# ---- the Python entry points
def host_cache(pages=3, heads=2, ps=16, D=64):
    codes = torch.zeros((pages, heads, ps, D // 2), dtype=torch.uint8)
    return codes, codes.clone(), torch.ones(heads), torch.ones(heads)


def test_python_wants_tensors_on_the_gpu(b):
    i = torch.zeros(2, dtype=torch.int32)
    table = torch.zeros((2, 3), dtype=torch.int32)
    with pytest.raises(TypeError):
        b.pq_kv4_slots(i, i, table, i, 16, 4)
    out = dict(cu_q=torch.zeros(3, dtype=torch.int32), kv_len_out=i.clone(), positions=torch.zeros(4, dtype=torch.int32),
               slots=torch.zeros(4, dtype=torch.int64), taken_out=i.clone())
    with pytest.raises(TypeError):
        b.pq_kv4_slots(i, i, table, i, 16, 4, **out)
    x, q = torch.zeros((2, 6 * 64)).half(), torch.zeros((2, 2 * 64)).half()
    slots = torch.zeros(2, dtype=torch.int64)
    for o in (None, q.clone()):
        with pytest.raises(TypeError):
            b.pq_kv4_append(x, 2, i, slots, *host_cache(), out=o)
    for o, w in ((None, None), (q.clone(), torch.zeros(4096, dtype=torch.uint8))):
        with pytest.raises(TypeError):
            b.pq_kv4_attention(q, torch.zeros(3, dtype=torch.int32), i, table, *host_cache(), 0.1, 1, out=o, workspace=w)


def test_native_calls_decline_what_is_not_plain(b):
    i, table = torch.zeros(2, dtype=torch.int32), torch.zeros((2, 3), dtype=torch.int32)
    x, q, slots = torch.zeros((2, 6 * 64)).half(), torch.zeros((2, 2 * 64)).half(), torch.zeros(2, dtype=torch.int64)
    assert b._call.kv4_slots() == -1 and b._call.kv4_append() == -1 and b._call.kv4_attention() == -1
    assert b._call.kv4_slots(i, i, table, i, 16, 2, None, 0, torch.zeros(3, dtype=torch.int32), i, i, slots, i) == -1
    assert b._call.kv4_append(x, 2, i, slots, *host_cache(), None, None, 1e-6, None, False, True, 0, 1.0, q) == -1
    assert b._call.kv4_attention(q, i, i, table, *host_cache(), 0.1, 1, 0, None, None, True, q, torch.zeros(64, dtype=torch.uint8)) == -1


def test_python_checks_shapes(b, monkeypatch):
    """On the CPU, with the checks of the device taken out of the way: the sizes' own checks, before the library is called."""
    b.lib()
    monkeypatch.setattr(b, "_here", lambda t, dtype, what: None)
    monkeypatch.setattr(b, "_rows", lambda t, what: None)
    monkeypatch.setattr(b, "_stream", lambda: None)
    called = []
    monkeypatch.setattr(b, "lib", lambda: type("L", (), {n: staticmethod(lambda *a: called.append(a) or 0) for n in (
        "pq_kv4_slots", "pq_kv4_append", "pq_kv4_attention", "pq_kv4_attention_workspace_bytes")}))
    i32 = lambda *n: torch.zeros(n, dtype=torch.int32)
    codes = host_cache()

    def refused(f, *a, **k):
        with pytest.raises(ValueError):
            f(*a, **k)

    refused(b.pq_kv4_slots, i32(2), i32(3), i32(2, 3), i32(5), 16, 4)
    refused(b.pq_kv4_slots, i32(2), i32(2), i32(3, 3), i32(5), 16, 4)
    refused(b.pq_kv4_slots, i32(2), i32(2), i32(6), i32(5), 16, 4)
    refused(b.pq_kv4_slots, i32(2), i32(2), i32(2, 3), i32(5), 16, 4, taken=i32(0))
    refused(b.pq_kv4_slots, i32(2), i32(2), i32(2, 3), i32(5), 16, 4, cu_q=i32(2))
    refused(b.pq_kv4_slots, i32(2), i32(2), i32(2, 3), i32(5), 16, 4, positions=i32(3))
    refused(b.pq_kv4_slots, i32(2), i32(2), i32(2, 3), i32(5), 16, 4, slots=torch.zeros(3, dtype=torch.int64))

    x, slots = torch.zeros((2, 6 * 64)).half(), torch.zeros(2, dtype=torch.int64)
    refused(b.pq_kv4_append, x, 3, i32(2), slots, *codes)                                          # heads do not fill the rows
    refused(b.pq_kv4_append, x, 2, i32(2), slots[:1], *codes)
    refused(b.pq_kv4_append, x, 2, i32(1), slots, *codes, cos_sin=torch.zeros((5, 64)))
    refused(b.pq_kv4_append, x, 2, i32(2), slots, *codes, cos_sin=torch.zeros(64))
    refused(b.pq_kv4_append, x, 2, i32(2), slots, *codes, q_weight=torch.zeros(32).half())
    refused(b.pq_kv4_append, x, 2, i32(2), slots, codes[0], codes[1][:2], *codes[2:])
    refused(b.pq_kv4_append, x, 2, i32(2), slots, codes[0][0], codes[1][0], *codes[2:])
    refused(b.pq_kv4_append, x, 2, i32(2), slots, *codes[:2], codes[2][:1], codes[3])
    refused(b.pq_kv4_append, x, 2, i32(2), slots, *codes, group=32)                                # static steps where dynamic ones belong

    q = torch.zeros((2, 2 * 64)).half()
    attend = lambda *a, **k: refused(b.pq_kv4_attention, *a, **k)
    attend(q, i32(2), i32(2), i32(2, 3), *codes, 0.1, 1)
    attend(q, i32(3), i32(2), i32(1, 3), *codes, 0.1, 1)
    attend(q[:, :100], i32(3), i32(2), i32(2, 3), *codes, 0.1, 1)
    attend(q, i32(3), i32(2), i32(2, 3), *codes, 0.1, 1, prefix_k=torch.zeros((1, 2, 64)).half())
    attend(q, i32(3), i32(2), i32(2, 3), *codes, 0.1, 1, prefix_k=torch.zeros((1, 2, 64)).half(), prefix_v=torch.zeros((1, 1, 64)).half())
    assert not called or all(len(a) == 6 for a in called)                                          # (sizes of a workspace at most)
    b.pq_kv4_append(x, 2, i32(2), slots, *codes)
    assert len(called[-1]) == 18

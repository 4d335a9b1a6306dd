"""Python's numbers have no end, the library's have 32 bits: what does not fit is refused or, where any number is allowed, stands for the largest.  No
GPU needed: the checks of the device are taken out of the way, and the library's calls are recorded."""

import sys

import pytest
import torch

from test_kv4_refusals import b, host_cache          # noqa: F401

MOST, WRAPS = (1 << 31) - 1, 1 << 32


def i32(*n):
    return torch.zeros(n, dtype=torch.int32)


def wide(rows, columns):
    return i32(rows, 1).expand(rows, columns)         # (no memory behind it)


@pytest.fixture
def calls(b, monkeypatch):                            # noqa: F811
    real, made = b.lib(), {}
    monkeypatch.setattr(b, "_here", lambda t, dtype, what: None)
    monkeypatch.setattr(b, "_rows", lambda t, what: None)
    monkeypatch.setattr(b, "_result", lambda t, n, what: None)
    monkeypatch.setattr(b, "_stream", lambda: None)
    monkeypatch.setattr(b, "_call", b._Declines)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)

    def record(name):
        def call(*a):
            made[name] = a
            return 0
        return staticmethod(call)
    monkeypatch.setattr(b, "lib", lambda: type("L", (), {**{n: record(n) for n in b.SIGNATURES if n.startswith("pq_kv4")},
                                                         "pq_status_str": real.pq_status_str}))
    return made


def attend(b, kind, *sight, max_q=1, table=None, group=0, **more):          # noqa: F811
    q, table = torch.zeros((2, 2 * 64)).half(), i32(2, 3) if table is None else table
    return getattr(b, "pq_kv4_" + kind)(q, i32(3), i32(2), table, *host_cache(), 0.1, max_q, *sight, group=group, **more)


@pytest.mark.parametrize("far", [MOST + 1, WRAPS, WRAPS + 16, WRAPS + MOST, sys.maxsize, 1 << 80])
def test_numbers_of_any_size_stand_for_the_largest(b, calls, far):          # noqa: F811
    attend(b, "window_attention", far, sinks=5)
    assert calls["pq_kv4_window_attention"][15:17] == (MOST, 5) and calls["pq_kv4_window_attention_workspace_bytes"][5:7] == (MOST, 5)
    attend(b, "window_attention", 7, sinks=far, max_q=far)
    assert calls["pq_kv4_window_attention"][15:17] == (7, MOST) and calls["pq_kv4_window_attention"][7] == MOST
    attend(b, "tree_attention", i32(2, 1), window=far, sinks=far)
    assert calls["pq_kv4_tree_attention"][15:19] == (calls["pq_kv4_tree_attention"][15], 1, MOST, MOST)
    attend(b, "attention", max_q=far)
    assert calls["pq_kv4_attention"][7] == MOST and calls["pq_kv4_attention_workspace_bytes"][3] == MOST
    codes = host_cache()[0]
    for name, more in (("attention", ()), ("window_attention", (far, far)), ("tree_attention", (far, far))):
        getattr(b, "pq_kv4_%s_workspace_bytes" % name)(5, 2, 2, far, 3, *more, codes)
        assert calls["pq_kv4_%s_workspace_bytes" % name][3:-1] == (MOST, 3) + (MOST,) * len(more)


@pytest.mark.parametrize("far", [MOST + 1, WRAPS + 1, WRAPS + 16, -MOST - 2, 1 - WRAPS, 1 << 80])
def test_numbers_past_32_bits_are_refused(b, calls, far):                   # noqa: F811
    def refused(f, *a, error=b.PQError, **k):
        calls.clear()
        with pytest.raises(error):
            f(*a, **k)
        assert not [n for n in calls if not n.endswith("_bytes")]

    refused(b.pq_kv4_tree, i32(5), i32(3), i32(2), far)
    refused(b.pq_kv4_tree, i32(5), i32(3), i32(2), 1, position_offset=far)
    accept = (i32(5), i32(5), i32(5), i32(3), i32(2))
    refused(b.pq_kv4_accept, *accept, i32(2, 3), far, 1, 3)
    refused(b.pq_kv4_accept, *accept, i32(2, 3), 16, far, 3)
    refused(b.pq_kv4_accept, *accept, i32(2, 3), 16, 1, far)
    slots = (i32(2), i32(2), i32(2, 3), i32(4))
    refused(b.pq_kv4_slots, *slots, far, 5)
    refused(b.pq_kv4_slots, *slots, 16, 5, position_offset=far)
    if far < 0:
        refused(attend, b, "window_attention", far)
        refused(attend, b, "window_attention", 7, sinks=far)
        refused(attend, b, "tree_attention", i32(2, 1), window=far)
        refused(attend, b, "attention", max_q=far)
        assert b.pq_kv4_window_attention_workspace_bytes(5, 2, 2, 1, 3, far, 4, host_cache()[0]) == 0
    else:
        refused(b.pq_kv4_accept, *accept, wide(2, far), 16, 1, 3) if far < 1 << 40 else None
    assert b.pq_kv4_attention_workspace_bytes(5, 2, 2, 1, far, host_cache()[0]) == 0
    assert b.pq_kv4_tree_attention_workspace_bytes(5, 2, far, 1, 3, 5, 4, host_cache()[0]) == 0


@pytest.mark.parametrize("columns", [MOST + 1, WRAPS + 3])
def test_sizes_of_tensors_past_32_bits_are_refused(b, calls, columns):      # noqa: F811
    for f in (lambda: attend(b, "attention", table=wide(2, columns), workspace=torch.zeros(1)),
              lambda: attend(b, "window_attention", 5, table=wide(2, columns), workspace=torch.zeros(1)),
              lambda: attend(b, "tree_attention", wide(2, columns)),
              lambda: b.pq_kv4_slots(i32(2), i32(2), wide(2, columns), i32(4), 16, 5),
              lambda: b.pq_kv4_keep(torch.zeros((2, 1), dtype=torch.int64).expand(2, columns), torch.zeros((2, 1), dtype=torch.int64).expand(2, columns),
                                    b.KV4Layers([host_cache()]))):
        calls.clear()
        with pytest.raises(b.PQError):
            f()
        assert not [n for n in calls if not n.endswith("_bytes")]
    none = torch.zeros((0, columns, 16, 32), dtype=torch.uint8)             # (a cache of no pages: sizes without memory)
    steps = torch.zeros(1).expand(columns)
    with pytest.raises(ValueError):
        b._kv4_cache(none, none, steps, steps, 0)
    with pytest.raises(ValueError):
        b.pq_kv4_attention_workspace_bytes(5, 2, 2, 1, 3, none)

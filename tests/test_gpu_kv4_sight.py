"""Attention over the paged 4-bit KV cache with a sliding window and for trees of drafted tokens, against a plain implementation in 64 bits
(kv4_tree_reference.py) within the bound that its roundings add up to."""

import numpy as np
import pytest
import torch

import kv4_reference as R
import kv4_tree_reference as TR
from pq_testlib import dev, host
from test_gpu_kv4 import KV, attention_case, pq, put                          # noqa: F401 (pq: a fixture)
from test_gpu_kv4_tree import grow_trees

pytestmark = pytest.mark.gpu
FAR = (1 << 31) - 1


def attend(pq, d, max_q, window=0, sinks=0, mask=None, out=None, ws=None):
    a = (d["q"], d["cu"], d["kv"], d["table"], d["kc"], d["vc"], d["ks"], d["vs"], d["scale"], max_q)
    more = dict(sinks=sinks, group=d["group"], prefix_k=d["pk"], prefix_v=d["pv"], out=out, workspace=ws)
    return (pq.pq_kv4_window_attention(*a, window, **more) if mask is None else pq.pq_kv4_tree_attention(*a, mask, window=window, **more))[0]


def within(c, got, window, sinks, mask=None):
    want, bound, real = TR.attention(c, window, sinks, mask)
    err = np.abs(got.astype(np.float64).reshape(want.shape) - want)
    worst = (err / np.maximum(bound, 1e-30))[real].max(initial=0.0)
    assert worst <= 1.0, "error is %.3g times its bound" % worst
    return real


def check(pq, c, window=0, sinks=0, mask=None, hints=None):
    d = put(c)
    m = None if mask is None else dev(mask)
    first = None
    for hint in hints or (int(np.diff(c["cu"]).max(initial=1)) or 1,):
        out = torch.full(c["q"].shape, 5.0, dtype=torch.float16, device="cuda")
        got = host(attend(pq, d, hint, window, sinks, m, out))
        real = within(c, got, window, sinks, mask)
        assert np.all(got[~real] == 5.0)                           # rows of no request are left as they were
        first = got if first is None else first
    return first


def masks(c, words, seed):
    """Of trees as pq_kv4_tree makes them."""
    T = len(c["q"])
    parents = grow_trees(np.random.default_rng(seed), np.diff(c["cu"]), max(T, int(c["cu"][-1])))[:T]
    return TR.tree(parents, c["cu"], c["kv"], T, words)[0]


SHAPES = [(64, 0), (64, 32), (64, 64), (128, 0), (128, 32), (128, 64), (128, 128)]


# ---------------------------------------------------------------------------------------------- windows
@pytest.mark.parametrize("D,group", SHAPES)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (31, 0), (32, 32), (33, 5), (100, 40), (127, 33), (FAR, 0), (200, FAR)])
def test_window_of_decoded_tokens(pq, D, group, window, sinks):
    check(pq, attention_case(KV, [1] * len(KV), 4, 2, D, window % 1000 + D, group), window, sinks)


@pytest.mark.parametrize("D,group", SHAPES)
@pytest.mark.parametrize("window,sinks", [(1, 0), (7, 3), (32, 0), (64, 64), (65, 70), (150, 1), (1 << 30, 4)])
def test_window_of_ragged_queries(pq, D, group, window, sinks):
    kv, q = [300, 40, 3, 77, 130, 16, 0, 9, 500], [5, 40, 9, 0, 130, 1, 2, 9, 70]  # q > kv: rows that see nothing
    check(pq, attention_case(kv, q, 4, 2, D, 11, group, 32, prefix=0), window, sinks)
    check(pq, attention_case(kv, q, 6, 1, D, 12, group, 16, prefix=2), window, sinks)


@pytest.mark.parametrize("D,group", [(128, 0), (128, 128), (64, 0), (64, 32)])
@pytest.mark.parametrize("q_len", [193, 256, 400])
@pytest.mark.parametrize("window,sinks", [(20, 0), (64, 4), (200, 100)])
def test_window_of_prompts(pq, D, group, q_len, window, sinks):
    check(pq, attention_case([q_len, q_len + 170], [q_len, q_len], 2, 2, D, q_len, group, 64, prefix=3), window, sinks)
    check(pq, attention_case([q_len + 300], [q_len], 2, 1, D, q_len, group, 16), window, sinks)


@pytest.mark.parametrize("group", [0, 128])
def test_window_of_long_histories(pq, group):
    """Many parts of one window, a window that starts far in, sinks that take several tiles; few rows and many."""
    check(pq, attention_case([30000, 7], [1, 1], 2, 1, 128, 41, group, 128, prefix=1), 12345, 100)
    check(pq, attention_case([9000], [60], 8, 1, 128, 42, group, 64), 5000, 4)
    check(pq, attention_case([9000, 4000], [60, 9], 8, 1, 128, 43, group, 64), 3000, 4)


@pytest.mark.parametrize("q_len", [1, 30, 120])
def test_pages_behind_the_window_may_be_gone(pq, q_len):
    for group in (0, 64):
        c = attention_case([700, 330], [q_len, q_len], 4, 2, 128, 21, group, 16)
        want = None
        for gone in (False, True):
            for b, n in enumerate((700, 330)):
                first = n - q_len + 1 - 90                         # the first token that the first row's window holds
                if gone:
                    c["table"][b, 2:first // 16] = [-1, 1 << 30, len(c["kc"]), -7][b:b + 1] * (first // 16 - 2)
            got = check(pq, c, 90, 20)
            assert want is None or np.array_equal(want.view(np.uint16), got.view(np.uint16))
            want = got


@pytest.mark.parametrize("q_len", [3, 60])
def test_pages_that_are_none(pq, q_len):
    c = attention_case([300, 170, 33], [q_len, q_len, 1], 4, 2, 128, 22, 128, 16)
    c["table"][0, 1], c["table"][0, 16], c["table"][1, 9], c["table"][1, 0], c["table"][2, :3] = -1, 1 << 30, len(c["kc"]), -3, -7
    check(pq, c, 80, 20)
    check(pq, c, 0, 0, masks(c, 2, 3))
    check(pq, c, 80, 20, masks(c, 2, 3))


@pytest.mark.parametrize("Hq,D,group", [(8, 128, 0), (8, 128, 32), (4, 64, 64)])
def test_a_window_that_hides_nothing_is_causal_attention(pq, Hq, D, group):
    for kv, q in (([900, 300, 40], [1, 5, 40]), ([700], [300]), ([400, 800], [100, 260])):
        c = attention_case(kv, q, Hq, 2, D, 5, group, 32, prefix=2)
        chain = TR.tree(np.concatenate([np.arange(m) - 1 for m in q]).astype(np.int32), c["cu"], c["kv"], len(c["q"]), 8)[0]
        want, bound, _ = R.attention(c["q"], c["cu"], c["kv"], c["table"], c["kc"], c["vc"], c["ks"], c["vs"], c["scale"], group, c["pk"], c["pv"])
        for got in (check(pq, c, FAR), check(pq, c, 0, 0, chain), check(pq, c, FAR, 0, chain)):
            assert np.all(np.abs(got.reshape(want.shape) - want) <= bound)


# ------------------------------------------------------------------------------------------------ trees
@pytest.mark.parametrize("D,group", SHAPES)
@pytest.mark.parametrize("words,q_lens", [(1, [26, 1, 32, 7, 0, 31]), (2, [64, 33, 5]), (3, [70, 96, 2]), (8, [256, 100])])
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 5)])
def test_trees(pq, D, group, words, q_lens, window, sinks):
    r = np.random.default_rng(words)
    kv = [m + int(x) for m, x in zip(q_lens, [0, 300, 33, 5, 17, 64])]              # the first without a history
    c = attention_case(kv, q_lens, 4, 2, D, words, group, 16, prefix=int(r.integers(0, 4)))
    check(pq, c, window, sinks, masks(c, words, words))


@pytest.mark.parametrize("Hq", [1, 5, 8])
@pytest.mark.parametrize("q_len", [1, 2, 16, 17, 40, 64])
def test_trees_of_all_sizes(pq, Hq, q_len):
    for group in (0, 32):
        c = attention_case([q_len + 95, q_len, q_len + 31], [q_len] * 3, Hq, 1, 128, q_len, group, 32)
        check(pq, c, 0, 0, masks(c, 2, q_len))
    c = attention_case([q_len + 700], [q_len], Hq, 1, 128, q_len, 0, 32)            # a single request
    check(pq, c, 0, 0, masks(c, 2, q_len))


@pytest.mark.parametrize("D,group", [(128, 0), (128, 128), (64, 32)])
@pytest.mark.parametrize("q_len", [20, 100])
def test_any_mask(pq, D, group, q_len):
    """Masks that no tree has: bits of nodes that are not there, nodes that do not see themselves or see later ones, rows that see nothing."""
    r = np.random.default_rng(q_len)
    for before in (0, 45):
        c = attention_case([q_len + before] * 3, [q_len] * 3, 8, 2, D, q_len, group, 16)
        mask = r.integers(-(1 << 31), 1 << 31, (len(c["q"]), 4)).astype(np.int32)
        mask[r.random(len(mask)) < 0.3] = 0
        got = check(pq, c, 0, 0, mask)
        assert before or not got[~mask.any(1)].any()
        check(pq, c, 30, 2, mask)
        check(pq, c, 1, 0, mask)


@pytest.mark.parametrize("group", [0, 128])
def test_trees_beside_prompts_and_idle_requests(pq, group):
    q = [20, 33, 0, 200, 1, 32]
    c = attention_case([100, 90, 40, 260, 7, 32], q, 4, 2, 128, 9, group, 32, prefix=1, q_rows=sum(q) + 5)
    mask = masks(c, 1, 9)
    check(pq, c, 0, 0, mask, hints=(1, 20, 33, 200, 5000))
    check(pq, c, 50, 3, mask, hints=(1, 200))


@pytest.mark.parametrize("T", [10, 40, 61])
def test_fewer_rows_than_new_tokens(pq, T):
    """Rows end with the call: what a request has below T is its tree, and what it sees is counted from the whole lengths."""
    for group in (0, 64):
        c = attention_case([150, 80, 64], [25, 30, 40], 4, 2, 128, T, group, 16)
        c["q"] = np.ascontiguousarray(c["q"][:T])
        check(pq, c, 0, 0, masks(c, 1, 1))
        check(pq, c, 40, 4)


def test_histories_past_the_table(pq):
    for q_len in (4, 70):
        c = attention_case([300, 150], [q_len, q_len], 4, 2, 128, 3, 0, 16)
        c["table"] = np.ascontiguousarray(c["table"][:, :11])
        check(pq, c, 0, 0, masks(c, 3, 1))
        check(pq, c, 100, 4)
        check(pq, c, 200, 20, masks(c, 3, 1))


def test_lengths_out_of_range(pq):
    c = attention_case([40, 64, 5], [1, 1, 1], 4, 2, 128, 22, ps=16, W=4)
    c["kv"][:] = [-3, 1 << 30, 5]
    c["table"][1] = [0, 1, 2, 3]
    check(pq, c, 20, 3)
    check(pq, c, 20, 3, np.ones((3, 1), np.int32))
    check(pq, c, 0, 0, np.ones((3, 1), np.int32))


@pytest.mark.parametrize("D,group", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)])
@pytest.mark.parametrize("q_len", [9, 30, 120])
@pytest.mark.parametrize("what", [np.inf, np.nan])
def test_steps_that_are_not_finite_stay_with_who_sees_them(pq, D, group, q_len, what):
    """Between the sinks and the window, in another branch, and behind a node."""
    n = q_len + 211
    c = attention_case([n, n], [q_len, q_len], 8, 2, D, 5, group, 16, prefix=1)
    mask = masks(c, 4, 6)
    for tree in (False, True):
        bad = dict(c, ks=c["ks"].copy(), vs=c["vs"].copy())
        dirty = np.zeros(len(c["q"]), bool)
        for b in range(2):
            for t in ([30, 60, 115] if not tree else [60, 211 + q_len // 3, 211 + q_len - 2]):
                for s in ("ks", "vs"):
                    bad[s][c["table"][b, t // 16], :, t % 16] = what
                for i in range(q_len):
                    bits = sum(int(w) << (32 * j) for j, w in enumerate(mask[b * q_len + i].view(np.uint32))) if tree else None
                    dirty[b * q_len + i] |= TR.seen_by(i, q_len, q_len, n, n, 100, 8, bits)[t]
        assert (~dirty).any()
        want, bound, _ = TR.attention(c, 100, 8, mask if tree else None)
        for hint in (1, q_len, 1000):
            got = host(attend(pq, put(bad), hint, 100, 8, dev(mask) if tree else None)).astype(np.float64).reshape(want.shape)
            assert np.all((np.abs(got - want) <= bound)[~dirty])


@pytest.mark.parametrize("group", [0, 32, 128])
def test_sharp_softmax(pq, group):
    c = attention_case([700, 400], [12, 60], 4, 2, 128, 31, group, 64, prefix=2, q_size=60.0)
    check(pq, c, 150, 40)
    check(pq, c, 0, 0, masks(c, 2, 1))


@pytest.mark.parametrize("q_len", [3, 40])
def test_very_many_requests(pq, q_len):
    """More than 512: the tile kernel looks its tiles up in a list."""
    r = np.random.default_rng(q_len)
    kv = r.integers(q_len, q_len + 60, 700)
    c = attention_case(kv, r.integers(0, q_len + 1, 700), 8, 1, 64, 42, 0, 16)
    mask = masks(c, 2, 2)
    check(pq, c, 24, 5, hints=(q_len,))
    check(pq, c, 24, 5, mask, hints=(q_len,))


def test_strided_queries_other_streams_and_two_at_once(pq):
    c = attention_case([150, 90], [24, 30], 4, 2, 128, 51, 0, 32, prefix=1)
    mask = masks(c, 1, 1)
    d = put(c)
    wide = torch.full((len(c["q"]), 4 * 128 + 40), float("nan"), dtype=torch.float16, device="cuda")
    wide[:, :512] = d["q"]
    d["q"] = wide[:, :512]
    m = dev(mask)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for i, s in enumerate(streams):
        with torch.cuda.stream(s):
            got.append(attend(pq, d, 30, 60, 4, m if i else None))
    torch.cuda.synchronize()
    within(c, host(got[0]), 60, 4)
    within(c, host(got[1]), 60, 4, mask)


@pytest.mark.parametrize("q_len", [8, 64])
def test_captured_calls_follow_their_inputs(pq, q_len):
    """Two graphs that share scratch memory, replayed while masks, lengths and tables change; every replay equals the eager call."""
    r = np.random.default_rng(q_len)
    B = 3
    c = attention_case([900, 500, 700], [q_len] * B, 8, 2, 128, 7, 128, 32)
    c["vs"] = np.nan_to_num(c["vs"], nan=0.25)
    c["ks"] = np.nan_to_num(c["ks"], nan=0.25)
    d = put(c)
    mask = dev(masks(c, 2, 0))
    size = max(f(len(c["q"]), B, 8, q_len, c["table"].shape[1], 200, 4, d["kc"]) for f in (
        pq.pq_kv4_window_attention_workspace_bytes, pq.pq_kv4_tree_attention_workspace_bytes))
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    outs = [torch.zeros_like(d["q"]) for _ in range(2)]
    graphs = []
    torch.cuda.synchronize()
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            attend(pq, d, q_len, 200, 4, mask if i else None, outs[i], ws)
        graphs.append(g)
    for n in range(6):
        mask.copy_(dev(masks(c, 2, n)))
        d["kv"].copy_(dev(r.integers(q_len, 900, B).astype(np.int32)))
        d["table"].copy_(dev(r.integers(0, len(c["kc"]), c["table"].shape).astype(np.int32)))
        d["q"].copy_(dev(r.standard_normal(c["q"].shape).astype(np.float16)))
        graphs[n % 2].replay()
        torch.cuda.synchronize()
        eager = attend(pq, d, q_len, 200, 4, mask if n % 2 else None, ws=ws)
        assert torch.equal(outs[n % 2], eager)
        within(dict(c, kv=host(d["kv"]), table=host(d["table"]), q=host(d["q"])), host(eager), 200, 4, host(mask) if n % 2 else None)


@pytest.mark.parametrize("q_len", [1, 70])
def test_native_and_ctypes_paths_agree(pq, monkeypatch, q_len):
    c = attention_case([300, 200], [q_len, q_len], 4, 2, 128, 3, 0, 16, prefix=1)
    c["scale"] = float(c["scale"])
    d, m = put(c), dev(masks(c, 3, 1))
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    for mask in (None, m):
        a, b = (torch.zeros_like(d["q"]) for _ in range(2))
        taken = []
        name = "kv4_window_attention" if mask is None else "kv4_tree_attention"
        native = getattr(pq._call, name)
        with monkeypatch.context() as patch:
            patch.setattr(pq, "_call", type("C", (), {name: staticmethod(lambda *x: taken.append(native(*x)) or taken[-1])}))
            attend(pq, d, q_len, 50, 3, mask, a, ws)
        assert taken == [0]
        with monkeypatch.context() as patch:
            patch.setattr(pq, "_call", pq._Declines)
            attend(pq, d, q_len, 50, 3, mask, b, ws)
        assert torch.equal(a, b)

"""Drafted trees on the paged 4-bit KV cache: masks and positions, what is accepted, and the move of codes, against plain implementations
(kv4_tree_reference.py); every value equal.  A server's steps with all calls together."""

import numpy as np
import pytest
import torch

import kv4_tree_reference as TR
from pq_testlib import dev, host
from test_gpu_kv4 import i32, pq, rope_table                                        # noqa: F401 (pq: a fixture)

pytestmark = pytest.mark.gpu


def step_case(q_lens, words, seed, ps=16, kv=200, T=None, extra=3, vocabulary=5):
    """Trees with all kinds of parents (recent ones mostly, a few that are none), tokens of a small vocabulary so that siblings share some."""
    r = np.random.default_rng(seed)
    B = len(q_lens)
    cu = np.concatenate([[0], np.cumsum(q_lens)]).astype(np.int32)
    T = int(cu[-1]) + 7 if T is None else T
    before = r.integers(0, kv + 1, B)
    c = dict(cu=cu, kv=(before + q_lens).astype(np.int32), T=T, words=words, ps=ps)
    parents = np.full(T, 7, np.int32)
    for b, m in enumerate(q_lens):
        for i in range(m):
            t = cu[b] + i
            if t < T:
                parents[t] = -1 if i == 0 else r.integers(max(0, i - 6), i)
                if i and r.random() < 0.06:
                    parents[t] = r.choice([-1, i, i + 3, -9, 1 << 30])
    c["parents"] = parents
    c["tokens"], c["chosen"] = (r.integers(0, vocabulary, T).astype(np.int32) for _ in range(2))
    need = -(-c["kv"] // ps)
    W = int(need.max(initial=0)) + extra
    n = int(need.sum())
    order = r.permutation(n + 9).astype(np.int32)
    c["table"] = np.full((B, W), -1, np.int32)
    at = 0
    for b in range(B):
        c["table"][b, :need[b]] = order[at:at + need[b]]
        at += need[b]
    c["free"], c["taken"] = order, n
    return c


def check_tree(pq, c, offset=0):
    mask, pos = pq.pq_kv4_tree(dev(c["parents"]), dev(c["cu"]), dev(c["kv"]), c["words"], offset)
    want = TR.tree(c["parents"], c["cu"], c["kv"], c["T"], c["words"], offset)
    assert np.array_equal(host(mask), want[0]) and np.array_equal(host(pos), want[1])


def check_accept(pq, c, depth, free=True):
    f, t = (dev(c["free"]), i32([c["taken"]])) if free else (None, None)
    got = pq.pq_kv4_accept(dev(c["tokens"]), dev(c["parents"]), dev(c["chosen"]), dev(c["cu"]), dev(c["kv"]), dev(c["table"]), c["ps"], c["words"],
                           depth, free_pages=f, taken=t)
    want = TR.accept(c["tokens"], c["parents"], c["chosen"], c["cu"], c["kv"], c["T"], c["table"], c["ps"], c["words"], depth,
                     c["free"] if free else np.zeros(0, np.int32), c["taken"] if free else 0)
    for name, g, w in zip(("accepted", "next_token", "path", "kv_len_out", "from", "to", "taken_out"), got, want):
        assert np.array_equal(host(g), w), name
    if free:
        assert np.array_equal(host(f), want[7])
    return want


SIZES = [([1], 1), ([0], 1), ([26], 1), ([32, 31, 33, 1, 0, 64], 1), ([63, 64, 65, 2], 2), ([96, 5, 90], 3), ([256, 255, 257, 128, 3], 8), ([1] * 300, 1),
         ([17] * 70, 1), ([2000, 3, 40], 2)]


@pytest.mark.parametrize("q_lens,words", SIZES)
def test_masks_and_positions(pq, q_lens, words):
    for seed in range(3):
        check_tree(pq, step_case(q_lens, words, seed), offset=3 * seed)


def test_masks_of_chains_and_of_roots(pq):
    for m, words in ((1, 1), (32, 1), (64, 2), (256, 8)):
        c = step_case([m, m], words, 1)
        c["parents"][:2 * m] = np.concatenate([np.arange(m), np.arange(m)]) - 1    # chains: the masks of causal attention
        check_tree(pq, c)
        c["parents"][:] = -1
        check_tree(pq, c)


@pytest.mark.parametrize("T", [0, 1, 30, 50, 70])
def test_fewer_rows_than_new_tokens(pq, T):
    """Rows end with the call: what a request has below T is its tree."""
    c = step_case([20, 45, 60], 2, T, T=T)
    if T:
        check_tree(pq, c)
    check_accept(pq, c, 6)


@pytest.mark.parametrize("q_lens,words", SIZES)
@pytest.mark.parametrize("depth", [1, 4, 30])
def test_what_is_accepted(pq, q_lens, words, depth):
    for seed in range(3):
        check_accept(pq, step_case(q_lens, words, seed, ps=16, vocabulary=2 + seed), depth)


def test_accepted_edges(pq):
    c = step_case([60] * 5, 2, 4, vocabulary=1)                                     # every choice fits: the way is as long as it can be
    for b in range(5):
        c["parents"][60 * b:60 * b + 60] = np.arange(60) - 1
    want = check_accept(pq, c, 64)
    assert list(want[0]) == [60] * 5 and (want[4] == -1).all()
    check_accept(pq, c, 7)
    c = step_case([40, 40, 40], 2, 5, ps=16, kv=90)                                 # pages that the list had run out of, and tokens past the table
    c["table"][:, 2:4] = -1
    check_accept(pq, c, 12)
    c["table"] = np.ascontiguousarray(c["table"][:, :3])
    check_accept(pq, c, 12)
    c = step_case([33, 50, 2], 2, 6, ps=16)
    check_accept(pq, c, 9, free=False)
    for taken in (0, 1, 3, -4, len(c["free"]) + 5):                                 # more come back than were given out; a list that was too short
        c["taken"] = taken
        check_accept(pq, c, 9)
    c = step_case([20, 20], 1, 7)
    c["kv"][:] = [5, -3]                                                            # fewer cached tokens than new ones
    check_accept(pq, c, 9)
    check_tree(pq, c)


def test_accepted_of_many_requests(pq):
    r = np.random.default_rng(0)
    check_accept(pq, step_case(r.integers(0, 40, 2500), 1, 8, kv=60), 8)


def test_no_requests(pq):
    none, table = i32([]), torch.zeros((0, 4), dtype=torch.int32, device="cuda")
    mask, pos = pq.pq_kv4_tree(i32([1, 2, 3]), i32([0]), none, 2)
    assert not host(mask).any() and not host(pos).any()
    got = pq.pq_kv4_accept(none, none, none, i32([0]), none, table, 16, 1, 4, free_pages=i32([1, 2, 3]), taken=i32([2]))
    assert host(got[6])[0] == 2 and got[2].shape == (0, 4)


# ------------------------------------------------------------------------------------------------ keep
def layers_case(L, pages, H, ps, D, group, seed):
    r = np.random.default_rng(seed)
    c = []
    for _ in range(L):
        codes = [r.integers(0, 256, (pages, H, ps, D // 2)).astype(np.uint8) for _ in range(2)]
        steps = [r.random((pages, H, ps, D // group) if group else H).astype(np.float32) for _ in range(2)]
        c.append(codes + steps)
    return c


def check_keep(pq, layers, src, dst, group):
    pages, _, ps, _ = layers[0][0].shape
    put = [[dev(a) for a in layer] for layer in layers]
    pq.pq_kv4_keep(dev(src), dev(dst), pq.KV4Layers(put, group))
    for layer, got in zip(layers, put):
        TR.keep(src, dst, layer if group else layer[:2], ps, pages)
        for a, g in zip(layer, got):
            assert np.array_equal(a.view(np.uint8), host(g).view(np.uint8))


@pytest.mark.parametrize("D,group", [(64, 0), (64, 32), (64, 64), (128, 0), (128, 32), (128, 64), (128, 128)])
@pytest.mark.parametrize("H,L,width", [(1, 1, 1), (2, 3, 5), (8, 2, 16), (3, 2, 70), (32, 1, 12), (5, 1, 256)])
def test_keep(pq, D, group, H, L, width):
    r = np.random.default_rng(width)
    B, ps = 4, 16
    each = -(-(3 * width + 20) // ps)
    order = r.permutation(B * each)
    src, dst = (np.full((B, width), -1, np.int64) for _ in range(2))
    for b in range(B):
        path = np.cumsum(r.integers(1, 4, width)) - 1
        path -= path[0]
        first = r.integers(0, ps)
        for k in range(r.integers(0, width + 1) if b else width):
            if path[k] != k:
                src[b, k], dst[b, k] = (order[b * each + x // ps] * ps + x % ps for x in (first + path[k], first + k))
    check_keep(pq, layers_case(L, B * each, H, ps, D, group, 3), src, dst, group)


def test_keep_entries_that_move_nothing(pq):
    src = np.array([[-1, 5, 5, 48, 1 << 40, 7, -(1 << 62)], [9, -1, 40, 30, 31, 47, 20]], np.int64)
    dst = np.array([[3, -1, 5, 6, 2, 48, 1], [8, 10, -7, 1 << 50, 30, 31, 48]], np.int64)
    for group in (0, 32):
        check_keep(pq, layers_case(2, 3, 2, 16, 64, group, 1), src, dst, group)


@pytest.mark.parametrize("L", [95, 96, 97, 200])
def test_keep_many_layers(pq, L):
    src, dst = np.array([[4, 6, 9]], np.int64), np.array([[3, 4, 5]], np.int64)
    check_keep(pq, layers_case(L, 1, 1, 16, 64, 0, 2), src, dst, 0)


def test_keep_nothing(pq):
    none = torch.empty((0, 3), dtype=torch.int64, device="cuda")
    pq.pq_kv4_keep(none, none, pq.KV4Layers([[dev(a) for a in layer] for layer in layers_case(1, 1, 1, 16, 64, 0, 0)]))


# ----------------------------------------------------------------------------------------- all together
def grow_trees(r, q_lens, T):
    parents = np.full(T, -1, np.int32)
    at = 0
    for m in q_lens:
        for i in range(1, m):
            parents[at + i] = r.integers(max(0, i - 4), i)
        at += m
    return parents


@pytest.mark.parametrize("D,group,window,sinks", [(128, 0, 0, 0), (64, 32, 24, 3), (128, 128, 0, 0)])
def test_speculative_steps_of_a_server(pq, D, group, window, sinks):
    """Prompts, then steps with drafted trees: slots, tree, append, attention, accept and keep.  Beside it a second cache gets only what was
    accepted, one chain after another: codes, steps, lengths and page counts have to be the same, and attention within its bound."""
    Hq, Hkv, ps, B, W, words, depth, L, P = 4, 2, 16, 3, 14, 1, 6, 2, 2
    r = np.random.default_rng(D + group)
    pages = B * W + 4

    def fresh_layer():
        codes = [torch.zeros((pages, Hkv, ps, D // 2), dtype=torch.uint8, device="cuda") for _ in range(2)]
        steps = [torch.zeros((pages, Hkv, ps, D // group), device="cuda") if group else torch.tensor([0.4, 0.5], device="cuda") for _ in range(2)]
        return codes + steps

    spec, plain = ([fresh_layer() for _ in range(L)] for _ in range(2))
    handle = pq.KV4Layers(spec, group)
    free, free2 = (dev(np.arange(pages, dtype=np.int32)) for _ in range(2))
    table, table2 = (dev(np.full((B, W), -1, np.int32)) for _ in range(2))
    kv, kv2, taken, taken2 = i32([0] * B), i32([0] * B), i32([0]), i32([0])
    cs = dev(rope_table(D))
    pk, pv = (dev(r.standard_normal((P, Hkv, D)).astype(np.float16)) for _ in range(2))
    for step, q_lens in enumerate([[40, 33, 70], [12, 9, 20], [30, 1, 17], [0, 25, 40], [32, 32, 32]]):
        T = sum(q_lens) + 4
        cu, kv_all, pos, slot, taken = pq.pq_kv4_slots(kv, i32(q_lens), table, free, ps, T, taken=taken, position_offset=P)
        parents = dev(grow_trees(r, q_lens, T))
        mask, pos = pq.pq_kv4_tree(parents, cu, kv_all, words, position_offset=P, positions=pos)
        qkv = [r.standard_normal((T, (Hq + 2 * Hkv) * D)).astype(np.float16) for _ in range(L)]
        for layer, x in zip(spec, qkv):
            q = pq.pq_kv4_append(dev(x), Hq, pos, slot, *layer, cos_sin=cs, group=group)
            out, _ = pq.pq_kv4_tree_attention(q, cu, kv_all, table, *layer, D ** -0.5, max(q_lens), mask, window=window, sinks=sinks, group=group,
                                              prefix_k=pk, prefix_v=pv)
            c = dict(zip(("kc", "vc", "ks", "vs"), map(host, layer)), q=host(q), cu=host(cu), kv=host(kv_all), table=host(table), scale=D ** -0.5,
                     group=group, pk=host(pk), pv=host(pv))
            want, bound, real = TR.attention(c, window, sinks, host(mask))
            assert np.all((np.abs(host(out).reshape(want.shape) - want) <= bound)[real])
        tokens, chosen = (dev(r.integers(0, 3, T).astype(np.int32)) for _ in range(2))
        args = [host(t) for t in (tokens, parents, chosen, cu, kv_all)]
        expected = TR.accept(*args, T, host(table), ps, words, depth, host(free), int(host(taken)[0]))
        acc, nxt, path, kv, src, dst, taken = pq.pq_kv4_accept(tokens, parents, chosen, cu, kv_all, table, ps, words, depth, free_pages=free, taken=taken)
        for g, w in zip((acc, nxt, path, kv, src, dst, taken, free), expected):
            assert np.array_equal(host(g), w)
        pq.pq_kv4_keep(src, dst, handle)

        # the same tokens as chains
        rows, lens = [], []
        for b, m in enumerate(q_lens):
            way = host(path)[b]
            way = way[way >= 0] if m <= 32 * words else np.arange(m)
            rows += [sum(q_lens[:b]) + i for i in way]
            lens.append(len(way))
        cu2, kv2, pos2, slot2, taken2 = pq.pq_kv4_slots(kv2, i32(lens), table2, free2, ps, len(rows), taken=taken2, position_offset=P)
        assert np.array_equal(host(kv2), host(kv)) and np.array_equal(host(taken2), host(taken))
        for layer, x in zip(plain, qkv):
            pq.pq_kv4_append(dev(np.ascontiguousarray(x[rows])), Hq, pos2, slot2, *layer, cos_sin=cs, group=group)
        for layer, layer2 in zip(spec, plain):
            for a, a2 in zip(layer, layer2) if group else zip(layer[:2], layer2[:2]):
                for b, n in enumerate(host(kv)):
                    t = np.arange(n)
                    one, two = (host(x)[host(tab)[b, t // ps], :, t % ps] for x, tab in ((a, table), (a2, table2)))
                    assert np.array_equal(one.view(np.uint8), two.view(np.uint8))


def test_captured_step_follows_its_inputs(pq):
    """tree, accept and keep captured once and replayed with other trees, choices and lengths, with eager calls between."""
    words, depth, ps, B, T, W, L = 2, 8, 16, 4, 200, 20, 3
    r = np.random.default_rng(5)
    layers = layers_case(L, B * W, 2, ps, 64, 32, 4)
    put = [[dev(a) for a in layer] for layer in layers]
    handle = pq.KV4Layers(put, 32)
    t = {n: i32(np.zeros(T)) for n in ("parents", "tokens", "chosen")}
    cu, kv = i32(np.zeros(B + 1)), i32(np.zeros(B))
    table, free, taken = dev(r.permutation(B * W).reshape(B, W).astype(np.int32)), i32(np.arange(B * W)), i32([B * W])
    mask, pos = pq.pq_kv4_tree(t["parents"], cu, kv, words)
    outs = dict(zip(("accepted", "next_token", "path", "kv_len_out", "from_slots", "to_slots", "taken_out"),
                    pq.pq_kv4_accept(t["tokens"], t["parents"], t["chosen"], cu, kv, table, ps, words, depth, free_pages=free, taken=taken)))

    def step():
        pq.pq_kv4_tree(t["parents"], cu, kv, words, mask=mask, positions=pos)
        pq.pq_kv4_accept(t["tokens"], t["parents"], t["chosen"], cu, kv, table, ps, words, depth, free_pages=free, taken=taken, **outs)
        pq.pq_kv4_keep(outs["from_slots"], outs["to_slots"], handle)

    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        step()
    for i in range(5):
        q_lens = r.integers(0, 66, B)
        c = step_case(q_lens, words, 100 + i, kv=200, T=T, vocabulary=2)
        for n in t:
            t[n].copy_(dev(c[n]))
        cu.copy_(dev(c["cu"]))
        kv.copy_(dev(c["kv"]))
        free.copy_(i32(np.arange(B * W)))
        before = host(free)
        g.replay()
        torch.cuda.synchronize()
        want = TR.tree(c["parents"], c["cu"], c["kv"], T, words)
        assert np.array_equal(host(mask), want[0]) and np.array_equal(host(pos), want[1])
        want = TR.accept(c["tokens"], c["parents"], c["chosen"], c["cu"], c["kv"], T, host(table), ps, words, depth, before, B * W)
        for w, n in zip(want, outs):
            assert np.array_equal(host(outs[n]), w), n
        assert np.array_equal(host(free), want[7])
        for layer, got in zip(layers, put):
            TR.keep(want[4], want[5], layer, ps, B * W)
            for a, x in zip(layer, got):
                assert np.array_equal(a.view(np.uint8), host(x).view(np.uint8))


def test_native_and_ctypes_paths_agree(pq, monkeypatch):
    c = step_case([20, 40, 33, 60], 2, 3, vocabulary=2)
    layers = layers_case(2, len(c["free"]), 2, 16, 64, 32, 4)
    got = []
    for native in (True, False):
        d = {n: dev(v) for n, v in c.items() if isinstance(v, np.ndarray)}
        put = [[dev(a) for a in layer] for layer in layers]
        handle = pq.KV4Layers(put, 32)
        B, T, depth = 4, c["T"], 9
        mask, pos = torch.empty((T, 2), dtype=torch.int32, device="cuda"), torch.empty(T, dtype=torch.int32, device="cuda")
        outs = [torch.empty(n, dtype=kind, device="cuda") for n, kind in ((B, torch.int32), (B, torch.int32), ((B, depth), torch.int32), (B, torch.int32),
                                                                        ((B, depth), torch.int64), ((B, depth), torch.int64), (1, torch.int32))]
        names = dict(zip(("accepted", "next_token", "path", "kv_len_out", "from_slots", "to_slots", "taken_out"), outs))
        taken, real = [], pq._call

        def through(name):
            f = getattr(real if native else pq._Declines, name)
            return staticmethod(lambda *x: taken.append(f(*x)) or taken[-1])
        with monkeypatch.context() as patch:
            patch.setattr(pq, "_call", type("C", (), {n: through(n) for n in ("kv4_tree", "kv4_accept", "kv4_keep")}))
            pq.pq_kv4_tree(d["parents"], d["cu"], d["kv"], 2, 5, mask=mask, positions=pos)
            pq.pq_kv4_accept(d["tokens"], d["parents"], d["chosen"], d["cu"], d["kv"], d["table"], 16, 2, depth, free_pages=d["free"],
                             taken=i32([c["taken"]]), **names)
            pq.pq_kv4_keep(outs[4], outs[5], handle)
        assert taken == [0 if native else -1] * 3
        got.append([host(t) for t in [mask, pos, d["free"]] + outs + [a for layer in put for a in layer]])
    assert all(np.array_equal(a.view(np.uint8), b.view(np.uint8)) for a, b in zip(*got))

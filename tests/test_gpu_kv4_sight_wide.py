"""Sliding windows, drafted trees and the way of accepted tokens at the ends of their ranges: many requests, many tiles of rows, caches past
2^32 bytes."""

import numpy as np
import pytest
import torch

import kv4_tree_reference as TR
from pq_testlib import dev, host
from test_gpu_kv4 import attention_case, pq, put                             # noqa: F401 (pq: a fixture)
from test_gpu_kv4_sight import attend, masks, within
from test_gpu_kv4_tree import layers_case

pytestmark = pytest.mark.gpu


def some(c, mask, which):
    """The case of some of its requests, and their rows."""
    rows = np.concatenate([np.arange(c["cu"][b], c["cu"][b + 1]) for b in which])
    cu = np.concatenate([[0], np.cumsum(np.diff(c["cu"])[which])]).astype(np.int32)
    part = dict(c, q=np.ascontiguousarray(c["q"][rows]), cu=cu, kv=c["kv"][which], table=c["table"][which])
    return part, None if mask is None else mask[rows], rows


@pytest.mark.parametrize("D,group", [(64, 0), (128, 128)])
@pytest.mark.parametrize("B,q_len", [(1500, 13), (2100, 9)])
def test_many_requests_with_many_rows(pq, D, group, B, q_len):
    """More than 1024 requests and 1024 tiles of rows: the plan takes several of each with every thread, some have few rows and some none."""
    r = np.random.default_rng(B)
    q = np.where(r.random(B) < 0.1, r.integers(0, q_len, B), q_len)
    kv = q + r.integers(0, 150, B)
    c = attention_case(kv, q, 16, 1, D, 3, group, 32, W=2200)                  # (a table this long asks for the tile kernel)
    d, mask, which = put(c), masks(c, 1, 4), np.sort(r.choice(B, 60, False))
    for window, sinks, m in ((30, 4, None), (0, 0, mask), (40, 2, mask)):
        got = host(attend(pq, d, 40, window, sinks, None if m is None else dev(m)))
        part, its, rows = some(c, m, which)
        within(part, got[rows], window, sinks, its)
        assert np.isfinite(got).all()


@pytest.mark.parametrize("D,Hq,Hkv", [(64, 16, 8), (128, 8, 2)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (70, 3), (1000, 0)])
def test_prompts_of_many_tiles(pq, D, Hq, Hkv, window, sinks):
    """Runs of many short tiles.  A row of a prompt sees what a token that is decoded there would."""
    kv, q = np.array([5200, 300, 2500]), np.array([5000, 290, 2500])
    c = attention_case(kv, q, Hq, Hkv, D, 8, 0, 64, prefix=1)
    got = host(attend(pq, put(c), 5000, window, sinks))
    assert np.isfinite(got).all()
    r = np.random.default_rng(9)
    rows = np.sort(np.concatenate([r.choice(c["cu"][-1], 60, False), c["cu"][:-1], c["cu"][1:] - 1]))
    rows = np.unique(rows)
    b = np.searchsorted(c["cu"], rows, "right") - 1
    one = dict(c, q=np.ascontiguousarray(c["q"][rows]), cu=np.arange(len(rows) + 1, dtype=np.int32), table=c["table"][b],
               kv=(kv[b] - q[b] + rows - c["cu"][b] + 1).astype(np.int32))
    within(one, got[rows], window, sinks)


@pytest.mark.parametrize("group", [0, 64])
def test_caches_past_32_bits(pq, group):
    """Pages whose places lie past 2^32 bytes: moved in, and read by both attention kernels, as in a small cache."""
    Hq, Hkv, D, ps = 4, 2, 128, 1024
    pages, n = 40000, 1500                                                     # 5.2 GB of keys, 5.2 of values
    small = layers_case(1, 4, Hkv, ps, D, group, 5)[0]
    shape = (pages, Hkv, ps)
    large = [torch.empty(shape + (D // 2,), dtype=torch.uint8, device="cuda") for _ in range(2)]
    large += [torch.empty(shape + (D // group,), device="cuda") for _ in range(2)] if group else [dev(s) for s in small[2:]]
    small = [dev(a) for a in small]
    far = torch.tensor([pages - 1, 33333, pages - 2, 36000], device="cuda")
    for a, b in zip(small, large):
        if a.dim() > 1:
            b[far] = a
    src, dst = np.array([[5, 1700, 4000, 2 * ps + 7]]), np.array([[3, 1600, 2000, 900]])
    pq.pq_kv4_keep(dev(src), dev(dst), pq.KV4Layers([small], group))
    place = host(far)
    pq.pq_kv4_keep(dev(place[src // ps] * ps + src % ps), dev(place[dst // ps] * ps + dst % ps), pq.KV4Layers([large], group))
    for a, b in zip(small, large):
        assert torch.equal(a, b[far] if a.dim() > 1 else b)
    r = np.random.default_rng(6)
    for q_len in (1, 6, 200):
        c = dict(kv=np.array([n, n + 300], np.int32), cu=np.array([0, q_len, 2 * q_len], np.int32),
                 q=r.standard_normal((2 * q_len, Hq * D)).astype(np.float16), table=np.array([[1, 0], [3, 2]], np.int32))
        m = dev(masks(c, 7, q_len))
        c = put(dict(c, group=group, scale=0.05, pk=None, pv=None))
        for args in ((400, 10), (0, 0, m), (400, 10, m)):
            both = [attend(pq, dict(c, table=t, kc=x[0], vc=x[1], ks=x[2], vs=x[3]), q_len, *args)
                    for t, x in ((c["table"], small), (far[c["table"].long()].int(), large))]
            assert torch.equal(*both) and both[0].isfinite().all() and both[0].any()


def test_keep_of_very_many_requests(pq):
    """More than the launch has workgroups: 70001 requests that each move one token."""
    B, ps = 70001, 16
    pages = -(-2 * B // ps)
    layer = [dev(a) for a in layers_case(1, pages, 3, ps, 64, 32, 7)[0]]
    slots = torch.arange(B, device="cuda")[:, None]
    want = [a.clone() for a in layer]
    for a in want:
        flat = a.transpose(1, 2).reshape(pages * ps, 3, -1).clone()
        flat[:2 * B:2] = flat[1:2 * B:2].clone()
        a.copy_(flat.reshape(pages, ps, 3, -1).transpose(1, 2))
    pq.pq_kv4_keep(2 * slots + 1, 2 * slots, pq.KV4Layers([layer], 32))
    for a, b in zip(want, layer):
        assert torch.equal(a, b)


@pytest.mark.parametrize("B", [1, 16, 24, 25, 48])
def test_accepted_of_few_and_of_more_requests(pq, B):
    """One workgroup does for few requests, two launches for more."""
    r = np.random.default_rng(B)
    q = r.integers(0, 65, B)
    q[0] = 64
    kv = (q + r.integers(0, 100, B)).astype(np.int32)
    cu = np.concatenate([[0], np.cumsum(q)]).astype(np.int32)
    T, ps, depth = int(cu[-1]), 16, 7
    table = r.permutation(B * 12).reshape(B, 12).astype(np.int32)
    table[r.random(table.shape) < 0.05] = -1
    parents = np.concatenate([np.maximum(np.arange(m) - r.integers(1, 4, m), -1) for m in q]).astype(np.int32)
    tokens, chosen = (r.integers(0, 3, T).astype(np.int32) for _ in range(2))
    free = r.integers(0, 999, 200).astype(np.int32)
    for taken in (0, 3, 150, 500):
        want = TR.accept(tokens, parents, chosen, cu, kv, T, table, ps, 2, depth, free, taken)
        f = dev(free)
        got = pq.pq_kv4_accept(dev(tokens), dev(parents), dev(chosen), dev(cu), dev(kv), dev(table), ps, 2, depth, free_pages=f,
                               taken=dev(np.array([taken], np.int32)))
        for g, w in zip((*got, f), want):
            assert np.array_equal(host(g), w)

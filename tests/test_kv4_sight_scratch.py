"""The documented bound of the scratch memory of the attentions with windows and trees, where their lists are longest: as many requests as a call
may have, with as many rows as the row kernel or the tile kernel takes at least, on one head; and at random sizes."""

import itertools
import random

import pytest

from test_kv4_refusals import b, cache          # noqa: F401


def bound(T, B, heads, kv):
    return (160 << 20) + 2 * (T * heads + 16 * B * kv) + 96 * B


def needs(b, T, B, heads, max_q, pages, window, sinks, c):                  # noqa: F811
    return [getattr(b.lib(), "pq_kv4_%s_attention_workspace_bytes" % kind)(T, B, heads, max_q, pages, window, sinks, c) for kind in ("window", "tree")]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads,kv", [(1, 1), (2, 1), (8, 1), (8, 8), (4, 2)])
def test_longest_lists(b, D, heads, kv):                                    # noqa: F811
    per, seen = heads // kv, 0
    c = cache(b, n_kv_heads=kv, head_dim=D)
    for B, rows in itertools.product(((1 << 21) // kv - 1, 1 << 20, 100000, 3000, 257, 256), (16, 96, 104, 105, 106, 112, 128, 129, 176, 192, 193, 208, 257)):
        T = min(B * rows // per, ((1 << 30) - 1) // heads)
        for pages, window, max_q in itertools.product((16, 200), (1, 500, (1 << 31) - 1), (1, rows // per, rows // per + 1, 1000)):
            for got in needs(b, T, B, heads, max(max_q, 1), pages, window, 4, c) if B * kv < 1 << 21 else ():
                assert 0 < got <= bound(T, B, heads, kv), (B, rows, pages, window, max_q)
                seen += got > (160 << 20) + 2 * (T * heads + 16 * B * kv)
    assert seen if heads == 1 else True                                     # (what the lists of requests are for)


def test_random_sizes(b):                                                   # noqa: F811
    rng = random.Random(5)
    some = lambda most: int(2 ** rng.uniform(0, most))
    for _ in range(4000):
        kv = some(5)
        heads, B = kv * some(5), some(21)
        B = max(1, min(B, ((1 << 21) - 1) // kv))
        T = max(1, min(some(30), ((1 << 30) - 1) // heads))
        for got in needs(b, T, B, heads, some(20), some(13), some(30), some(12), cache(b, n_kv_heads=kv, head_dim=rng.choice([64, 128]))):
            assert 0 < got <= bound(T, B, heads, kv), (T, B, heads, kv)

"""The lists of the masked tile kernel's plan at their borders: as many requests and tiles of rows as the planning workgroup has threads, and one
more, by the workgroup beside the row kernel's join (256 threads) and by the one that plans alone (1024), which takes several to a thread then."""

import numpy as np
import pytest

from test_gpu_kv4_sight import attend, attention_case, dev, host, masks, pq, put, within          # noqa: F401
from test_gpu_kv4_sight_wide import some

pytestmark = pytest.mark.gpu


def check_some(pq, c, max_q, window, sinks, mask, seed):                                          # noqa: F811
    got = host(attend(pq, put(c), max_q, window, sinks, None if mask is None else dev(mask)))
    assert np.isfinite(got).all()
    B = len(c["kv"])
    which = np.unique(np.concatenate([[0, B - 2, B - 1], np.random.default_rng(seed).choice(B, min(B, 30), False)]))
    part, its, rows = some(c, mask, which)
    within(part, got[rows], window, sinks, its)


@pytest.mark.parametrize("B,empty", [(255, 0), (256, 0), (257, 0), (256 + 40, 40), (257 + 40, 40)])
def test_requests_and_tiles_beside_the_join(pq, B, empty):                                        # noqa: F811
    r = np.random.default_rng(B)
    q = np.full(B, 13)
    q[r.choice(B, empty, False)] = 0
    c = attention_case(q + r.integers(0, 150, B), q, 16, 1, 64, 3, 0, 32, W=80)
    check_some(pq, c, 13, 0, 0, masks(c, 1, 4), B)
    check_some(pq, c, 13, 2000, 3, None, B)


@pytest.mark.parametrize("B", [1023, 1024, 1025, 1100])
def test_requests_and_tiles_of_a_plan_alone(pq, B):                                               # noqa: F811
    r = np.random.default_rng(B)
    c = attention_case(13 + r.integers(0, 20, B), [13] * B, 16, 1, 128, 5, 0, 16, W=2)
    c["kv"] = np.minimum(c["kv"], 32).astype(np.int32)
    check_some(pq, c, 13, 0, 0, masks(c, 1, 4), B)
    check_some(pq, c, 13, 9, 2, None, B)


@pytest.mark.parametrize("q_len", [32767, 32768, 32769, 33000])
def test_tiles_of_one_prompt(pq, q_len):                                                          # noqa: F811
    """1024 tiles of rows, and a few more.  A row of a prompt sees what a token that is decoded there would."""
    c = attention_case([q_len + 40], [q_len], 8, 1, 64, 7, 0, 64)
    for window, sinks in ((70, 3), (600, 0)):
        got = host(attend(pq, put(c), q_len, window, sinks))
        assert np.isfinite(got).all()
        rows = np.unique(np.concatenate([[0, 31, 32, q_len - 33, q_len - 2, q_len - 1], np.random.default_rng(q_len).choice(q_len, 40, False)]))
        n = np.zeros(len(rows), int)
        one = dict(c, q=np.ascontiguousarray(c["q"][rows]), cu=np.arange(len(rows) + 1, dtype=np.int32), table=c["table"][n], kv=(40 + rows + 1).astype(np.int32))
        within(one, got[rows], window, sinks)

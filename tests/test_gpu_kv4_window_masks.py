"""Chains that are deeper than the window, as trees whose masks leave out what stands a window or more above, and as chains: the same tokens are seen."""

import numpy as np
import pytest

import kv4_tree_reference as TR
from kv4_window_masks import within_window
from test_gpu_kv4_sight import attend, attention_case, dev, host, pq, put, within          # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,group", [(128, 0), (64, 0), (128, 32), (64, 64)])
@pytest.mark.parametrize("m,words", [(20, 1), (64, 2), (130, 8), (256, 8)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 0), (16, 5), (50, 130)])
def test_chains_deeper_than_the_window(pq, D, group, m, words, window, sinks):            # noqa: F811
    c = attention_case([m, m + 1, m + 100], [m] * 3, 4, 2, D, m, group, 16, prefix=1)
    parents = np.concatenate([np.arange(m, dtype=np.int32) - 1] * 3)
    mask, pos = TR.tree(parents, c["cu"], c["kv"], 3 * m, words, 1)
    d = put(c)
    got = host(attend(pq, d, m, window, sinks, dev(within_window(mask, pos, c["cu"], window, sinks, 1))))
    within(c, got, window, sinks)                                  # the sliding window's own results
    within(c, host(attend(pq, d, m, window, sinks)), window, sinks)

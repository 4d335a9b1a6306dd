"""What a node sees under a window, by the plain implementation: the stated formula with the nodes out of the mask that stand a window or more above
is the sliding window at the node's position, along its own branch."""

import numpy as np
import pytest

import kv4_tree_reference as TR
from kv4_window_masks import within_window


@pytest.mark.parametrize("window,sinks", [(1, 0), (2, 0), (5, 3), (16, 0), (16, 400), (64, 4), (1000, 7)])
@pytest.mark.parametrize("before", [0, 1, 40])
def test_trimmed_masks_are_sliding_windows(window, sinks, before):
    r = np.random.default_rng(window + before)
    for m, words in ((1, 1), (32, 1), (64, 2), (200, 8)):
        for chain in (True, False):
            parents = np.array([i - 1 if chain else r.integers(-1, i) if i else -1 for i in range(m)], np.int32)
            cu, kv = np.array([0, m]), np.array([before + m])
            mask, pos = TR.tree(parents, cu, kv, m, words, 3)
            trimmed = within_window(mask, pos, cu, window, sinks, 3)
            for i in range(m):
                branch, at = [], i
                while at >= 0:
                    branch.append(at)
                    at = int(parents[at])
                branch.reverse()                                   # its k-th node stands at before + k
                p = before + len(branch) - 1
                near = lambda t: t < sinks or t > p - window
                want = {t for t in range(before) if near(t)} | {before + n for k, n in enumerate(branch) if near(before + k)}
                bits = sum(int(w) << (32 * k) for k, w in enumerate(trimmed[i].view(np.uint32)))
                assert set(np.flatnonzero(TR.seen_by(i, m, m, before + m, before + m, window, sinks, bits))) == want

"""Masks of drafted trees whose branches may be deeper than the window: without the nodes that stand a window or more above a row's own."""

import numpy as np


def within_window(mask, positions, cu, window, sinks, offset=0):
    """mask int32 [T, words] and positions of pq_kv4_tree -> a mask of the nodes that a sliding window leaves."""
    bits, words = mask.view(np.uint32).copy(), mask.shape[1]
    for b in range(len(cu) - 1):
        lo, hi = int(cu[b]), min(int(cu[b + 1]), len(mask))
        if hi - lo > 32 * words:
            continue                                               # a prompt
        for t in range(lo, hi):
            for j in range(hi - lo):
                if positions[lo + j] <= positions[t] - window and positions[lo + j] - offset >= sinks:
                    bits[t, j // 32] &= np.uint32(~(1 << j % 32) & 0xFFFFFFFF)
    return bits.view(np.int32)

"""How pq_kv4_keep shares out heads, on the CPU: a wavefront counts the pieces of its heads' entries in 32 bits."""

import os

import pytest

from test_kv4_tree_launches import launches

pytestmark = pytest.mark.skipif(not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"), reason="no HIP headers")


@pytest.mark.parametrize("D,group", [(64, 0), (64, 32), (128, 0), (128, 32)])
@pytest.mark.parametrize("Hkv,B,L", [(8, 1, 32), (8, 48, 80), (1 << 22, 255, 9), (1 << 22, 34, 60), (1 << 21, 511, 5), (1 << 24, 1, 96), (1 << 24, 63, 40),
                                     ((1 << 30) - 1, 1, 1), ((1 << 29) - 1, 2, 96), (1, (1 << 26) - 1, 96)])
def test_pieces_of_a_wavefront_are_counted_in_32_bits(D, group, Hkv, B, L):
    (rc, _, events), = launches([dict(fn="keep", B=B, L=L, Hkv=Hkv, D=D, group=group, ps=16, width=256)])
    assert rc == 0 and len(events) == 1
    _, _, groups, _ = events[0]
    in_x = min(B, 1 << 16)
    assert groups % (in_x * L) == 0 and groups * 64 < 1 << 32
    heads = -(-Hkv // (groups // (in_x * L)))                                # of a wavefront, on average
    assert 2 * heads * 256 * (D // 32) < 1 << 31

"""Which plan the sizes of test_gpu_kv4_plan_lists.py take, read on the CPU: the one beside the row kernel's join, or the one that is made alone."""

import os

import pytest

from test_kv4_tree_launches import attention, kernels

pytestmark = pytest.mark.skipif(not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"), reason="no HIP headers")


def test_who_plans():
    beside = dict(Hq=16, Hkv=1, D=64, ps=32, W=80, max_q=13)
    alone = dict(Hq=16, Hkv=1, D=128, ps=16, W=2, max_q=13)
    for fn, window in (("tree_attention", 0), ("window_attention", 2000)):
        for B in (255, 256, 257, 297):
            took = kernels(attention(fn, B=B, T=13 * B, window=window, **beside))
            assert "join_masked" in took[1] and "_tiles<" in took[2] and len(took) == 4
    for fn, window in (("tree_attention", 0), ("window_attention", 9)):
        for B in (1023, 1025, 1100):
            assert kernels(attention(fn, B=B, T=13 * B, window=window, **alone))[0] == "k_kv4_attention_plan"
    for T in (32767, 32769, 33000):
        assert kernels(attention("window_attention", B=1, T=T, max_q=T, Hq=8, Hkv=1, D=64, W=520, window=70))[0] == "k_kv4_attention_plan"

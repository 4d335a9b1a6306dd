"""Windows and first tokens past 32 bits, through both call paths: they hide nothing, as the largest that fits."""

import sys

import pytest

from test_gpu_kv4_sight import attend, attention_case, dev, host, masks, pq, put          # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("far", [(1 << 31) - 1, 1 << 31, (1 << 32) + 16, sys.maxsize])
def test_far_windows_hide_nothing(pq, far):                                               # noqa: F811
    import torch
    c = attention_case([200, 90], [3, 5], 4, 2, 64, 3, 0, 16, prefix=2)
    d, m = put(c), dev(masks(c, 1, 1))
    whole = host(attend(pq, d, 5, 1 << 20))
    tree = host(attend(pq, d, 5, 0, 0, m))
    out, ws = torch.empty((8, 4 * 64), dtype=torch.float16, device="cuda"), torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    for more in ({}, dict(out=out, ws=ws)):
        assert (host(attend(pq, d, 5, far, **more)) == whole).all()
        assert (host(attend(pq, d, 5, 16, far, **more)) == whole).all()
        assert (host(attend(pq, d, 5, far, 0, m, **more)) == tree).all()
        assert (host(attend(pq, d, 5, 16, far, m, **more)) == tree).all()

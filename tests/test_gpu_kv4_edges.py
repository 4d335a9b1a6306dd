"""The calls on the paged 4-bit KV cache where a step does not fit its rows or its table, and where values are not finite."""

import numpy as np
import pytest

import kv4_reference as R
from pq_testlib import host
from test_gpu_kv4 import attention_case, call, pq, put                                          # noqa: F401 (pq: a fixture)

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ values that are not finite
@pytest.mark.parametrize("D,group", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)])
@pytest.mark.parametrize("q_lens", [[3, 9], [40, 47], [120, 70]])
@pytest.mark.parametrize("what", [np.inf, -np.inf, np.nan])
def test_steps_that_are_not_finite_stay_with_who_sees_them(pq, D, group, q_lens, what):
    """A token whose value or key was infinite has an infinite step: the queries in front of it do not see it."""
    c = attention_case([200, 133], q_lens, 8, 2, D, 5, group, 16, prefix=1)
    clean = np.zeros(len(c["q"]), bool)
    for b, (n, m) in enumerate(zip((200, 133), q_lens)):
        first = n - m // 2                                         # this token, and one further on
        for t in (first, min(first + 5, n - 1)):
            c["vs"][c["table"][b, t // 16], :, t % 16] = what
            c["ks"][c["table"][b, t // 16], :, t % 16] = what
        lo = int(c["cu"][b])
        clean[lo:lo + m] = n - (m - 1 - np.arange(m)) <= first     # sees the tokens before this one
    assert 0 < clean.sum() < len(clean)
    want, bound, _ = R.attention(c["q"], c["cu"], c["kv"], c["table"], c["kc"], c["vc"], c["ks"], c["vs"], c["scale"], group, c["pk"], c["pv"])
    for hint in (1, max(q_lens), 1000):
        got = host(call(pq, put(c), hint)).astype(np.float64).reshape(want.shape)
        assert np.all((np.abs(got - want) <= bound)[clean])

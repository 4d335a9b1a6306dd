"""Launches of the calls on the paged 4-bit KV cache with very many requests, on the CPU."""

from test_kv4_launches import launches, pytestmark                                   # noqa: F401 (pytestmark: no HIP headers, no test)


def test_slots_launch_grows_no_further_than_the_card():
    """Every workgroup sums the requests in front of its own: with one to every 16 requests that were B^2 / 32 of them, hours for the largest B."""
    calls = [dict(fn="slots", B=B, T=T, ps=16, W=10) for B in (0, 1, 16, 17, 1000, 1 << 15, (1 << 15) + 1, 100003, (1 << 26) - 1) for T in (0, 1 << 20)]
    for call, (rc, _, events) in zip(calls, launches(calls)):
        assert rc == 0 and len(events) == 1
        groups = events[0][2]
        assert 0 < groups <= 2048 and (groups >= -(-call["B"] // 16) or groups > 1024), (call, groups)

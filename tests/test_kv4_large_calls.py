"""Launches of the calls on the paged 4-bit KV cache with very many requests, on the CPU."""

from test_kv4_launches import launches, pytestmark                                   # noqa: F401 (pytestmark: no HIP headers, no test)


def test_slots_launch_grows_no_further_than_the_card():
    """Every workgroup sums the requests in front of its own: with one to every 16 requests that were B^2 / 32 of them, hours for the largest B."""
    calls = [dict(fn="slots", B=B, T=T, ps=16, W=10) for B in (0, 1, 16, 17, 1000, 1 << 15, (1 << 15) + 1, 100003, (1 << 26) - 1) for T in (0, 1 << 20)]
    for call, (rc, _, events) in zip(calls, launches(calls)):
        assert rc == 0 and len(events) == 1
        groups = events[0][2]
        assert 0 < groups <= 2048 and (groups >= -(-call["B"] // 16) or groups > 1024), (call, groups)


def tiles_and_parts(**over):
    """Tiles of rows that the kernel for many rows is launched for, and parts of a history."""
    c = dict(fn="attention", Hq=32, Hkv=8, D=128, group=0, ps=64, W=520)
    c.update(over)
    grid = {e[1].split("<")[0]: e[2] for e in launches([c])[0][2] if e[0] == "launch"}
    most = grid["k_kv4_attention_tiles"] // c["Hkv"]
    tiles = grid.get("k_kv4_attention_join_tiles", 4 * c["Hkv"] * most) // (4 * c["Hkv"])
    return tiles, most // tiles


def test_decoding_requests_beside_a_prompt_do_not_take_its_parts():
    """512 new tokens of one request (8 tiles of 256 rows a head) are cut into parts beside 31, 63 or 255 that decode as they are alone: the
    launch counts tiles of the rows that may come, not one more for every request."""
    assert tiles_and_parts(T=512, B=1, max_q=512) == (8, 4)
    for others, least in ((1, 4), (31, 4), (63, 3), (127, 3), (255, 2)):
        tiles, parts = tiles_and_parts(T=512 + others, B=1 + others, max_q=512)
        assert parts >= least and 8 <= tiles <= 24, (others, tiles, parts)


def test_every_tile_of_rows_has_a_workgroup():
    """Requests of any sizes never have more tiles than the launch, whatever stands beside them."""
    for per_kv, lens in ((4, [49] * 40), (4, [65] * 30 + [1] * 30), (1, [193] * 9), (1, [257] * 12 + [3]), (1, [192, 192]), (8, [33, 32]), (1, [513, 1])):
        tiles, _ = tiles_and_parts(T=sum(lens), B=len(lens), max_q=max(max(lens), 200), Hq=8 * per_kv)
        assert tiles >= sum(-(-n * per_kv // 256) for n in lens if n * per_kv > 192)


def test_many_requests_get_a_list_of_their_tiles():
    """Beyond 512 requests no workgroup of the kernel for many rows walks over all of them."""
    for B, listed in ((2, 0), (512, 0), (513, 1), ((1 << 21) // 8 - 1, 1)):
        (rc, need, events), = launches([dict(fn="attention", T=60 * B, B=B, Hq=32, Hkv=8, D=128, group=0, ps=64, W=4, max_q=60)])
        names = [e[1] for e in events if e[0] == "launch"]
        assert rc == 0 and names.count("k_kv4_attention_tile_starts") == listed
        assert not listed or names.index("k_kv4_attention_tile_starts") == 0 and need >= 4 * (B + 1)

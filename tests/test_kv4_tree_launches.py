"""Which launches the calls for drafted trees and sliding windows on the paged 4-bit KV cache make, on the CPU: the rules that choose a kernel, the
dynamic LDS that the runtime is asked for before a kernel wants it, and launches within the runtime's bounds at the largest documented sizes."""

import ctypes
import json
import os
import re
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, HERE)
import launch_log                                                                   # noqa: E402

pytestmark = pytest.mark.skipif(not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"), reason="no HIP headers")


def launches(calls):
    r = subprocess.run([sys.executable, os.path.abspath(__file__), launch_log._stand_in(), launch_log.LIB], input=json.dumps(calls),
                       capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stderr[-4000:]
    return [(rc, need, [tuple(e) for e in events]) for rc, need, events in json.loads(r.stdout)]


def kernels(call):
    rc, _, events = launches([call])[0]
    assert rc == 0
    return [e[1] for e in events if e[0] == "launch"]


def attention(fn, **over):
    c = dict(fn=fn, T=64, B=64, Hq=32, Hkv=8, D=128, group=0, ps=64, W=128, max_q=1, window=0 if fn == "tree_attention" else 4096, sinks=4, words=1)
    assert set(over) <= set(c)
    c.update(over)
    return c


def rows(D, G, dynamic, blocks, together="false"):
    return ["k_kv4_attention_rows<%d, %d, %s, %d, pq::kv4::Masked>" % (D, G, dynamic, blocks), "k_kv4_attention_join_masked<%d, %d, %s>" % (D, blocks, together)]


@pytest.mark.parametrize("fn", ["window_attention", "tree_attention"])
def test_attention_takes_the_kernels_of_its_kind(fn):
    tiles = "k_kv4_attention_tiles<%d, %d, %s, pq::kv4::Masked>"
    for D, group in ((64, 0), (64, 32), (64, 64), (128, 0), (128, 32), (128, 64), (128, 128)):
        shape = (D, group or D, "true" if group else "false")
        assert kernels(attention(fn, D=D, group=group)) == rows(*shape, 1)
        many = [tiles % shape, "k_kv4_attention_join_runs<%d, %d>" % shape[:2]]
        assert kernels(attention(fn, T=4096, B=1, max_q=4096, W=64, D=D, group=group)) == ["k_kv4_attention_plan"] + many
        assert kernels(attention(fn, T=4000, B=8, max_q=500, W=64, D=D, group=group)) == rows(*shape, 1) + many
        limit = {}
        for call in (attention(fn, D=D, group=group), attention(fn, T=320, max_q=5, D=D, group=group), attention(fn, T=4000, B=8, max_q=500, D=D, group=group)):
            for what, kernel, _, lds in launches([call])[0][2]:
                if what == "allow":
                    limit[kernel] = lds
                else:
                    assert lds <= 160 * 1024 and (lds <= 65536 or limit.get(kernel, 0) >= lds), kernel


def test_rules_count_what_rows_may_see():
    """Under a window the same table holds less to do."""
    assert kernels(attention("window_attention", T=320, max_q=5, window=(1 << 31) - 1)) == rows(128, 128, "false", 2)
    assert kernels(attention("window_attention", T=320, max_q=5, window=300)) == rows(128, 128, "false", 1)

    def takes_tiles(**over):
        return any("_tiles<" in k for k in kernels(attention(**over)))
    for fn in ("window_attention", "tree_attention"):
        assert takes_tiles(fn=fn, B=2, T=98, max_q=49, W=10)                        # more than 192 rows always do
    much, little = dict(B=64, T=64 * 40, W=100), dict(B=4, T=160, W=60)
    assert takes_tiles(fn="tree_attention", max_q=27, **much) and not takes_tiles(fn="tree_attention", max_q=26, **much)       # 108 and 104 rows
    assert not takes_tiles(fn="tree_attention", max_q=48, **little)
    assert not takes_tiles(fn="window_attention", max_q=40, window=100, **much)
    # requests of few rows beside a prompt: a kernel of their own, unless they see little
    many = dict(fn="window_attention", B=5, T=2004, max_q=2000, W=200)
    assert len(kernels(attention(window=1000, **many))) == 3 and len(kernels(attention(window=4000, **many))) == 4


def test_few_histories_are_joined_by_workgroups():
    for B, T, max_q, together in ((1, 1, 1, "true"), (1, 8, 8, "true"), (4, 4, 1, "true"), (1, 26, 26, "false"), (16, 16, 1, "false")):
        assert kernels(attention("tree_attention", B=B, T=T, max_q=max_q)) == rows(128, 128, "false", 1, together)


def test_small_calls():
    for B, T in ((1, 26), (300, 5000), ((1 << 26) - 1, 5), (7, (1 << 30) - 1)):
        (rc, _, events), = launches([dict(fn="tree", B=B, T=T, words=8)])
        assert rc == 0 and [e[1] for e in events] == ["k_kv4_tree"] and 0 < events[0][2] * 64 < 1 << 32
    for B in (0, 1, 300, (1 << 26) - 1):
        (rc, _, events), = launches([dict(fn="accept", B=B, T=100, words=8, depth=256, W=100, ps=16)])
        assert rc == 0 and events and all(0 < e[2] * 1024 < 1 << 32 for e in events)
    for L, n in ((1, 1), (96, 1), (97, 2), (300, 4)):
        for B in (1, 48, (1 << 26) - 1):
            (rc, _, events), = launches([dict(fn="keep", B=B, L=L, Hkv=8, D=128, group=128, ps=16, width=256)])
            assert rc == 0 and len(events) == n and all(0 < e[2] * 256 < 1 << 32 for e in events)


def test_largest_sizes_stay_within_a_launch():
    """A launch holds less than 2^32 threads in a dimension."""
    big = (1 << 30) - 1
    for fn in ("window_attention", "tree_attention"):
        calls = [attention(fn, T=big // 32, B=B, max_q=q, W=16384, window=w) for B in (1, 1000, (1 << 21) // 8 - 1) for q in (1, 1000, (1 << 31) - 1)
                 for w in (1, (1 << 31) - 1)]
        calls += [attention(fn, T=big, Hq=1, Hkv=1, B=B, max_q=q, W=16384, D=64) for B in (1, (1 << 21) - 1) for q in (1, 100, 1 << 30)]
        for call, (rc, need, events) in zip(calls, launches(calls)):
            assert rc == 0, call
            assert need <= (160 << 20) + 2 * (call["T"] * call["Hq"] + 16 * call["B"] * call["Hkv"])
            for what, kernel, grid, _ in events:
                threads = 512 if "_tiles<" in kernel and "join" not in kernel else 256
                masked = "join_masked" in kernel
                y = (16 if "true" in kernel else 4) * (2 if ", 2," in kernel else 1) if masked else 4 if "join" in kernel else 1
                assert what == "allow" or 0 < grid // y * threads < 1 << 32, (call, kernel, grid)


def _main():
    log = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
    log.launch_log.restype = ctypes.c_char_p
    L = ctypes.CDLL(sys.argv[2])
    i32, i64, f32, p, size = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t

    class Cache(ctypes.Structure):
        _fields_ = [("k_codes", p), ("v_codes", p), ("k_scale", p), ("v_scale", p), ("n_pages", i64), ("n_kv_heads", i32), ("head_dim", i32),
                    ("page_size", i32), ("group", i32)]

    at = lambda i: p((i + 1) << 42)                                                 # (far apart and never read)
    L.pq_kv4_window_attention_workspace_bytes.restype = L.pq_kv4_tree_attention_workspace_bytes.restype = size
    out = []
    for c in json.load(sys.stdin):
        log.launch_log_clear()
        need = 0
        if c["fn"] == "tree":
            rc = L.pq_kv4_tree(at(0), at(1), at(2), i32(c["B"]), i64(c["T"]), i32(c["words"]), i32(0), at(3), at(4), p(0))
        elif c["fn"] == "accept":
            rc = L.pq_kv4_accept(at(0), at(1), at(2), at(3), at(4), i32(c["B"]), i64(c["T"]), i32(c["words"]), i32(c["depth"]), at(5), i32(c["W"]), i32(c["ps"]),
                                 at(6), i32(50), at(7), at(8), at(9), at(10), at(11), at(12), at(13), at(14), p(0))
        elif c["fn"] == "keep":
            caches = (Cache * c["L"])(*((at(3 * i), at(3 * i + 1), at(3 * i + 2), at(3 * i + 2), 1000, c["Hkv"], c["D"], c["ps"], c["group"]) for i in range(c["L"])))
            rc = L.pq_kv4_keep(at(1000), at(1001), i32(c["B"]), i32(c["width"]), caches, i32(c["L"]), p(0))
        else:
            cache = Cache(at(0), at(1), at(2), at(3), 1000, c["Hkv"], c["D"], c["ps"], c["group"])
            f = getattr(L, "pq_kv4_" + c["fn"])
            need = getattr(L, "pq_kv4_" + c["fn"] + "_workspace_bytes")(i64(c["T"]), i32(c["B"]), i32(c["Hq"]), i32(c["max_q"]), i32(c["W"]), i32(c["window"]),
                                                                       i32(c["sinks"]), ctypes.byref(cache))
            sight = [i32(c["window"]), i32(c["sinks"])]
            if c["fn"] == "tree_attention":
                sight = [at(10), i32(c["words"])] + sight
            rc = f(at(4), i64(c["Hq"] * c["D"]), i64(c["T"]), i32(c["Hq"]), at(5), at(6), i32(c["B"]), i32(c["max_q"]), at(7), i32(c["W"]), ctypes.byref(cache),
                   p(0), p(0), i32(0), f32(0.1), *sight, at(8), at(9), size(need), p(0))
        events = []
        for line in log.launch_log().decode().splitlines():
            what, name, grid, lds = line.split("\t")
            events.append((what, re.search(r"(k_\w+(?:<[^(]*>)?)", name).group(1), int(grid), int(lds)))
        out.append((rc, need, events))
    json.dump(out, sys.stdout)


if __name__ == "__main__":
    _main()

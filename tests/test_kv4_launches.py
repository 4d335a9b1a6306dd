"""Which launches the calls on the paged 4-bit KV cache make, on the CPU: the rules that choose a kernel, the dynamic LDS that the runtime is
asked for before a kernel wants it, and launches within the runtime's bounds at the largest documented sizes."""

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


def attention(**over):
    c = dict(fn="attention", T=64, B=64, Hq=32, Hkv=8, D=128, group=0, ps=64, W=128, max_q=1)
    c.update(over)
    return c


def rows(D, G, dynamic, blocks):
    return ["k_kv4_attention_rows<%d, %d, %s, %d>" % (D, G, dynamic, blocks), "k_kv4_attention_join<%d, %d>" % (D, blocks)]


def test_attention_takes_what_its_rules_say():
    one, two = rows(128, 128, "false", 1), rows(128, 128, "false", 2)
    tiles = "k_kv4_attention_tiles<128, 128, false>"
    assert kernels(attention()) == one
    assert kernels(attention(T=256, max_q=4)) == one                                # 16 rows
    assert kernels(attention(T=320, max_q=5)) == two                                # more, and 160 units and more for every wavefront
    assert kernels(attention(T=40, B=8, max_q=5)) == one                            # little to read
    assert kernels(attention(T=60 * 48, B=60, max_q=48)) == two                         # 192 rows
    assert kernels(attention(T=64 * 49, max_q=49)) == [tiles] + two                 # more: the tile kernel for those that have them
    assert kernels(attention(T=400, B=8, max_q=300, W=1)) == [tiles] + one
    assert kernels(attention(T=4096, B=1, max_q=4096, W=64)) == [tiles]             # a single request
    assert kernels(attention(T=500, B=1, Hq=64, max_q=500, W=520)) == [tiles, "k_kv4_attention_join_tiles<128, 128>"]
    assert kernels(attention(T=320, max_q=5, group=32)) == rows(128, 32, "true", 1)
    assert kernels(attention(T=320, max_q=5, group=64)) == rows(128, 64, "true", 2)
    assert kernels(attention(T=320, max_q=5, group=128)) == rows(128, 128, "true", 2)
    assert kernels(attention(T=320, max_q=5, D=64, group=32)) == rows(64, 32, "true", 2)
    assert kernels(attention(D=64)) == rows(64, 64, "false", 1)


def test_one_request_is_cut_into_whole_rounds():
    def groups(**over):
        return [e[2] for e in launches([attention(B=1, **over)])[0][2] if e[0] == "launch" and "_tiles<" in e[1]][0]
    assert groups(T=500, Hq=64, max_q=500, W=516) == 256
    assert groups(T=64, max_q=64, W=2048) == 256
    assert groups(T=400, Hq=8, Hkv=1, max_q=400, W=313) == 13 * 19
    assert groups(T=4096, max_q=4096, W=64) == 512                                  # enough as it is


def test_append_takes_several_heads_where_there_are_many():
    def names(**over):
        return kernels(dict(dict(fn="append", T=64, Hq=32, Hkv=8, D=128, group=0, ps=64, rotate=1), **over))
    assert names() == ["k_kv4_append<7, 0, true, false>"]
    assert names(T=1024) == ["k_kv4_append<7, 0, true, false>"]                     # 12288 turns of a head
    assert names(T=1025) == ["k_kv4_append<7, 0, true, true>"]
    assert names(T=2049, D=64, group=32, rotate=0) == ["k_kv4_append<6, 5, false, true>"]
    assert names(T=0) == []


def test_every_kernel_is_allowed_its_dynamic_lds():
    calls = [attention(T=T, B=B, max_q=q, D=D, group=g) for T, B, q in ((64, 64, 1), (320, 64, 5), (4000, 8, 500)) for D, g in (
        (64, 0), (64, 32), (64, 64), (128, 0), (128, 32), (128, 64), (128, 128))]
    limit, used = {}, set()
    for rc, _, events in launches(calls):
        assert rc == 0
        for what, kernel, _, lds in events:
            if what == "allow":
                limit[kernel] = lds
            else:
                used.add(kernel)
                assert lds <= 160 * 1024 and (lds <= 65536 or limit.get(kernel, 0) >= lds), kernel
    assert sum(k.startswith("k_kv4_attention_rows") for k in used) == 13 and sum(k.startswith("k_kv4_attention_tiles") for k in used) == 7


def test_largest_sizes_stay_within_a_launch():
    """A launch holds less than 2^32 threads in a dimension; x is the only one that grows, y at most 65535."""
    big = (1 << 30) - 1
    calls = [attention(T=big // 32, B=B, max_q=q, W=16384) for B in (1, 1000, (1 << 21) // 8 - 1) for q in (1, 5, 1000, 1 << 30)]
    calls += [attention(T=big, Hq=1, Hkv=1, B=B, max_q=q, W=16384, D=64) for B in (1, (1 << 21) - 1) for q in (1, 100, 1 << 30)]
    calls += [attention(T=1 << 20, Hq=1023, Hkv=1, B=1, max_q=1 << 20, W=16384)]
    for call, (rc, need, events) in zip(calls, launches(calls)):
        assert rc == 0, call
        assert need <= (160 << 20) + 2 * (call["T"] * call["Hq"] + 16 * call["B"] * call["Hkv"])
        for what, kernel, grid, _ in events:
            threads = 512 if "_tiles<" in kernel and "join" not in kernel else 256
            grid_x = grid // (4 if "join_tiles" in kernel else 8 if kernel.startswith("k_kv4_attention_join<") and kernel.endswith("2>") else
                              4 if "join" in kernel else 1)
            assert what == "allow" or 0 < grid_x * threads < 1 << 32, (call, kernel, grid)
    T = (1 << 25) - 1
    calls = [dict(fn="append", T=T, Hq=Hq, Hkv=1, D=D, group=0, ps=16, rotate=1) for Hq in (1, 60) for D in (64, 128)]
    calls += [dict(fn="append", T=32, Hq=65000, Hkv=1, D=128, group=0, ps=16, rotate=1)]
    for call, (rc, _, events) in zip(calls, launches(calls)):
        assert rc == 0 and len(events) == 1, call
        assert 0 < -(-call["T"] // (512 // call["D"])) * 256 < 1 << 32
    calls = [dict(fn="slots", B=B, T=T, ps=16, W=10) for B in (0, 1, (1 << 26) - 1) for T in (0, 1, (1 << 31) - 1)]
    for call, (rc, _, events) in zip(calls, launches(calls)):
        assert rc == 0 and len(events) == 1 and 0 < events[0][2] * 256 < 1 << 32, call


def _main():
    log = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
    log.launch_log.restype = ctypes.c_char_p
    L = ctypes.CDLL(sys.argv[2])
    i32, i64, f32, p, size = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t

    class Cache(ctypes.Structure):
        _fields_ = [("k_codes", p), ("v_codes", p), ("k_scale", p), ("v_scale", p), ("n_pages", i64), ("n_kv_heads", i32), ("head_dim", i32),
                    ("page_size", i32), ("group", i32)]

    at = lambda i: p((i + 1) << 44)                                                 # (far apart and never read)
    L.pq_kv4_attention_workspace_bytes.restype = size
    out = []
    for c in json.load(sys.stdin):
        log.launch_log_clear()
        need = 0
        if c["fn"] == "slots":
            rc = L.pq_kv4_slots(at(0), at(1), i32(c["B"]), at(2), i32(c["W"]), at(3), i32(100), p(0), i32(c["ps"]), i64(c["T"]), i32(0), at(4), at(5),
                                at(6), at(7), at(8), p(0))
        else:
            cache = Cache(at(0), at(1), at(2), at(3), 1000, c["Hkv"], c["D"], c["ps"], c["group"])
            if c["fn"] == "append":
                rc = L.pq_kv4_append(at(4), i64((c["Hq"] + 2 * c["Hkv"]) * c["D"]), i64(c["T"]), i32(c["Hq"]), at(5), at(6), p(0), p(0), f32(0), p(0), i64(0),
                                     i32(0), i32(0), i32(c["rotate"]), f32(1), ctypes.byref(cache), at(7), p(0))
            else:
                need = L.pq_kv4_attention_workspace_bytes(i64(c["T"]), i32(c["B"]), i32(c["Hq"]), i32(c["max_q"]), i32(c["W"]), ctypes.byref(cache))
                rc = L.pq_kv4_attention(at(4), i64(c["Hq"] * c["D"]), i64(c["T"]), i32(c["Hq"]), at(5), at(6), i32(c["B"]), i32(c["max_q"]), at(7),
                                        i32(c["W"]), ctypes.byref(cache), p(0), p(0), i32(0), f32(0.1), i32(1), at(8), at(9), size(need), p(0))
        events = []
        for line in log.launch_log().decode().splitlines():
            what, name, grid, lds = line.split("\t")
            events.append((what, re.search(r"(k_\w+(?:<[^(]*>)?)", name).group(1), int(grid), int(lds)))
        out.append((rc, need, events))
    json.dump(out, sys.stdout)


if __name__ == "__main__":
    _main()

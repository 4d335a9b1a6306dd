"""The calls on the paged 4-bit KV cache at the ends of their ranges: many tokens, many requests, caches past 2^31 bytes, calls at the same
time, the native call path against the ctypes path."""

import numpy as np
import pytest
import torch

import kv4_reference as R
from pq_testlib import dev, host
from test_gpu_kv4 import append_case, attention_case, call, check_append, check_attention, check_slots, i32, lengths, put, pq, rope_table, within

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ many tokens
# (from 12288 wavefronts of one head on, a wavefront takes several heads)
@pytest.mark.parametrize("D,T", [(64, 2110), (128, 1061)])
@pytest.mark.parametrize("rd,interleaved,norm,group", [(None, False, False, 0), (0, False, True, 32), (48, False, False, 64), (32, True, True, 0),
                                                       (None, True, False, 32), (None, False, True, 64)])
def test_append_many_tokens(pq, D, T, rd, interleaved, norm, group):
    """Odd numbers of heads and tokens, each kind of position rotation, some tokens without a slot."""
    c = append_case(T, 33, 11, D, T + 1, group)                                    # 55 heads: the last wavefronts have fewer
    c["slots"][[0, 5, 6, 7, T - 1]] = -1
    c["slots"][40:60] = -1                                                         # whole wavefronts of them
    r = np.random.default_rng(1)
    w = tuple(r.uniform(0.5, 1.5, D).astype(np.float16) for _ in range(2)) if norm else None
    check_append(pq, c, 33, 11, D, group, norm=w, cos_sin=None if rd == 0 else rope_table(rd or D), interleaved=interleaved,
                 stride=55 * D + 8)


def test_append_many_borders(pq):
    """Every value's and every key's quotient lies on a border: all of a wavefront's heads take the 64-bit path."""
    r = np.random.default_rng(2)
    T, D = 1100, 128
    c = append_case(T, 24, 12, D, 9, 0)
    c["vs"][:], c["ks"][:] = 0.25, 0.125
    x = c["qkv"].reshape(T, 48, D)
    k = r.integers(-10, 10, (T, 12, D))
    x[:, 36:] = ((k + 0.5) * 0.25).astype(np.float16)
    x[:, 24:36] = ((k + 0.5) * 0.125).astype(np.float16)
    check_append(pq, c, 24, 12, D, rotate=False)


def test_append_no_norm_for_queries_or_keys(pq):
    c = append_case(20, 4, 2, 128, 12, 0)
    w = np.random.default_rng(1).uniform(0.5, 1.5, 128).astype(np.float16)
    check_append(pq, c, 4, 2, 128, norm=(w, None))
    check_append(pq, c, 4, 2, 128, norm=(None, w))


def test_append_same_slot_twice(pq):
    """Two tokens with one slot: every byte is one of theirs, and the other places stay."""
    c = append_case(9, 2, 2, 64, 5, 0)
    c["slots"][4] = c["slots"][7]
    both = []
    for drop in (4, 7):
        d = {k: v.copy() for k, v in c.items()}
        d["slots"][drop] = -1
        t = [dev(d[n]) for n in ("kc", "vc", "ks", "vs")]
        pq.pq_kv4_append(dev(d["qkv"]), 2, None, dev(d["slots"]), *t)
        both.append([host(x) for x in t[:2]])
    t = [dev(c[n]) for n in ("kc", "vc", "ks", "vs")]
    pq.pq_kv4_append(dev(c["qkv"]), 2, None, dev(c["slots"]), *t)
    for n in range(2):
        got = host(t[n])
        assert np.all((got == both[0][n]) | (got == both[1][n]))


# ------------------------------------------------------------------------------------------------ many requests
@pytest.mark.parametrize("B,q", [(3000, 3), (700, 60)])
def test_slots_many_requests(pq, B, q):
    kv, n = lengths(B, 300, q, B)
    check_slots(pq, kv, n, 24, 16, 8 * B, int(n.sum()) + 100, seed=B)


def test_slots_one_long_prompt(pq):
    check_slots(pq, np.array([3], np.int32), np.array([100000], np.int32), 7000, 16, 6900, 100100)


def test_attention_more_histories_than_workgroups(pq):
    """70001 requests of up to 64 tokens: the second kernel walks over more histories than its launch has workgroups."""
    B, D, ps = 70001, 64, 16
    r = np.random.default_rng(4)
    kv = r.integers(0, 65, B).astype(np.int32)
    pages = 5000
    table = r.integers(0, pages, (B, 4)).astype(np.int32)
    kc, vc = (r.integers(0, 256, (pages, 1, ps, D // 2)).astype(np.uint8) for _ in range(2))
    q = (1.5 * r.standard_normal((B, D))).astype(np.float16)
    ks, vs = np.array([0.3], np.float32), np.array([0.4], np.float32)
    cu = np.arange(B + 1, dtype=np.int32)
    got, _ = pq.pq_kv4_attention(dev(q), dev(cu), dev(kv), dev(table), dev(kc), dev(vc), dev(ks), dev(vs), D ** -0.5, 1)
    got = host(got).astype(np.float64)
    k, v = (torch.from_numpy(R.unpack(x).astype(np.float64))[:, 0] * float(s[0]) for x, s in ((kc, ks), (vc, vs)))
    for b0 in range(0, B, 10000):
        at = torch.from_numpy(table[b0:b0 + 10000].astype(np.int64))
        n = len(at)
        kk, vv = k[at].reshape(n, 64, D), v[at].reshape(n, 64, D)
        s = (kk * torch.from_numpy(q[b0:b0 + n].astype(np.float64))[:, None]).sum(-1) * float(np.float32(D ** -0.5))
        s[torch.arange(64)[None] >= torch.from_numpy(kv[b0:b0 + n])[:, None]] = -np.inf
        w = torch.nan_to_num(torch.softmax(s, -1))                                  # (no tokens: zeros)
        o, big = ((w[:, :, None] * x).sum(1).numpy() for x in (vv, vv.abs()))
        # As in kv4_reference: probabilities and their sum half a step of fp16 each, the result half a step; scores of at most 2^8 (1.5 * 5
        # deviations * 8 * 0.3 * 8, times D^-0.5 and a sum over 64) to 2^-24 * 3 D of the sum of their products' sizes.
        size = (kk.abs() * torch.from_numpy(np.abs(q[b0:b0 + n]).astype(np.float64))[:, None]).sum(-1).amax(1).numpy()[:, None] * D ** -0.5
        e = size * (3 * D + 16) * 2.0 ** -24
        bound = (2.0 ** -11 * 1.01 + 2 * e + 2.0 ** -20) * (big + np.abs(o)) + (64 + 256) / 32 * 2.0 ** -24 * 16 * 3.2 + 64 * 2.0 ** -30 * 3.2 + \
            2.0 ** -11 * np.abs(o) + 2.0 ** -25
        assert np.all(np.abs(got[b0:b0 + n] - o) <= bound)


@pytest.mark.parametrize("D,Hkv,group", [(128, 2, 0), (128, 2, 64), (64, 4, 32)])
def test_attention_streams_large_caches(pq, D, Hkv, group):
    """More than 64 MiB of codes in a call, which go past the caches: one token each of nine requests, one of them with more rows than a
    wavefront takes (its codes are read twice)."""
    c = attention_case([33500] * 8 + [5000], [1] * 8 + [20], Hkv, Hkv, D, 111, group, 128, prefix=2)
    d = put(c)
    assert sum(int(n) for n in c["kv"]) * Hkv * D > 64 << 20
    got = [host(call(pq, d, 20)) for _ in range(2)]
    assert np.array_equal(got[0], got[1])
    within(c, got[0])


# ------------------------------------------------------------------------------------------------ past 32 bits
@pytest.mark.parametrize("group", [0, 64])
def test_caches_past_32_bits(pq, group):
    """Pages whose places lie past 2^32 bytes (and steps past 2^32): appended, and read by both attention kernels, as in a small cache."""
    Hq, Hkv, D, ps, T = 4, 2, 128, 1024, 300
    pages = 40000                                                                  # 5.2 GB of keys, 5.2 of values; 1.3 GB of steps each
    r = np.random.default_rng(3)
    shape = (pages, Hkv, ps)
    kc, vc = (torch.empty(shape + (D // 2,), dtype=torch.uint8, device="cuda") for _ in range(2))
    small = [torch.zeros((2, Hkv, ps, D // 2), dtype=torch.uint8, device="cuda") for _ in range(2)]
    if group:
        ks, vs = (torch.empty(shape + (D // group,), device="cuda") for _ in range(2))
        small += [torch.zeros((2, Hkv, ps, D // group), device="cuda") for _ in range(2)]
    else:
        ks, vs = (dev(r.uniform(0.3, 0.6, Hkv).astype(np.float32)) for _ in range(2))
        small += [ks, vs]
    far = np.array([[pages - 1, 33333]], np.int32)
    qkv = dev(r.standard_normal((T, (Hq + 2 * Hkv) * D)).astype(np.float16))
    at = np.arange(T) + ps - 150                                                   # over the end of the first page
    table = i32(far)
    slots = dev((far[0][at // ps].astype(np.int64) * ps + at % ps))
    near = dev(((at // ps).astype(np.int64) * ps + at % ps))
    for p in (kc, vc) + ((ks, vs) if group else ()):
        p[far[0].tolist()] = 0
    got = pq.pq_kv4_append(qkv, Hq, None, slots, kc, vc, ks, vs, group=group)
    want = pq.pq_kv4_append(qkv, Hq, None, near, *small, group=group)
    assert torch.equal(got, want)
    for big, s in zip((kc, vc) + ((ks, vs) if group else ()), small):
        assert torch.equal(big[far[0].tolist()], s)
    for n in (1, T):
        cu, kv = i32([0, n]), i32([int(at[-1]) + 1])
        a, _ = pq.pq_kv4_attention(got[:n].contiguous(), cu, kv, table, kc, vc, ks, vs, D ** -0.5, n, group=group)
        b, _ = pq.pq_kv4_attention(got[:n].contiguous(), cu, kv, i32([[0, 1]]), *small, D ** -0.5, n, group=group)
        assert torch.equal(a, b) and bool(a.any())


# ------------------------------------------------------------------------------------------------ ways to call
def test_two_streams_at_once(pq):
    """Calls on two streams, each with its own scratch memory, while both read one cache."""
    c = attention_case([4000, 900, 300, 17], [1, 1, 1, 1], 8, 2, 128, 71, 0, 64, prefix=3)
    p = attention_case([500, 900], [300, 150], 8, 2, 128, 72, 0, 64)
    dc, dp = put(c), put(p)
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for _ in range(10):
        for s, d, most, o in zip(streams, (dc, dp), (1, 300), outs):
            with torch.cuda.stream(s):
                o.append(call(pq, d, most))
    torch.cuda.synchronize()
    for case, o in zip((c, p), outs):
        within(case, host(o[0]))
        assert all(torch.equal(o[0], x) for x in o)


def test_native_and_ctypes_paths_agree(pq, monkeypatch):
    """Every call, with all its outputs given (the native path) and with the native path taken away."""
    c = attention_case([70, 20, 0], [2, 5, 0], 4, 2, 128, 81, 64, 16, prefix=2)
    c["scale"] = float(c["scale"])                                                 # (the native path takes plain numbers only)
    d = put(c)
    a = append_case(7, 4, 2, 128, 6, 64)
    table, free = dev(np.full((2, 6), -1, np.int32)), i32([5, 3, 1, 0, 2])

    def run():
        out = []
        t = table.clone()
        o = [i32([0] * 3), i32([0] * 2), i32([0] * 9), dev(np.zeros(9, np.int64)), i32([0])]
        pq.pq_kv4_slots(i32([0, 17]), i32([4, 3]), t, free, 16, 9, taken=i32([1]), position_offset=2, cu_q=o[0], kv_len_out=o[1], positions=o[2],
                        slots=o[3], taken_out=o[4])
        out += [t] + o
        x = [dev(a[n]) for n in ("kc", "vc", "ks", "vs")]
        q = torch.full((7, 512), 3.0, dtype=torch.float16, device="cuda")
        pq.pq_kv4_append(dev(a["qkv"]), 4, dev(a["positions"]), dev(a["slots"]), *x, cos_sin=dev(rope_table(64)), interleaved=True, group=64,
                         clip=0.9, out=q)
        out += x + [q]
        ws = torch.empty(pq.pq_kv4_attention_workspace_bytes(7, 3, 4, 5, c["table"].shape[1], d["kc"]), dtype=torch.uint8, device="cuda")
        for causal in (True, False):
            y = torch.full((7, 512), 3.0, dtype=torch.float16, device="cuda")
            call(pq, d, 5, causal, out=y, ws=ws)
            out.append(y)
        return out

    taken = []
    native = pq._call

    def watched(name):
        def f(*x):
            taken.append((name, getattr(native, name)(*x)))
            return taken[-1][1]
        return staticmethod(f)

    monkeypatch.setattr(pq, "_call", type("Watch", (), {n: watched(n) for n in ("kv4_slots", "kv4_append", "kv4_attention")}))
    one = run()
    assert taken == [("kv4_slots", 0), ("kv4_append", 0), ("kv4_attention", 0), ("kv4_attention", 0)]
    monkeypatch.setattr(pq, "_call", type("Declines", (), {n: staticmethod(lambda *x: -1) for n in ("kv4_slots", "kv4_append", "kv4_attention")}))
    for x, y in zip(one, run()):
        assert torch.equal(x.view(torch.uint8) if x.dtype == torch.float32 else x, y.view(torch.uint8) if y.dtype == torch.float32 else y)


def test_refusals_reach_the_caller(pq, monkeypatch):
    c = attention_case([70, 20], [2, 5], 4, 2, 64, 82, 0, 16)
    d = put(c)
    out = torch.empty_like(d["q"])
    with pytest.raises(pq.PQError):                                                # scratch memory too small
        call(pq, d, 5, out=out, ws=torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(pq.PQError):                                                # the output over the queries
        call(pq, d, 5, out=d["q"], ws=torch.empty(1 << 24, dtype=torch.uint8, device="cuda"))
    with pytest.raises(pq.PQError):                                                # lengths updated in place
        n = i32([3, 4])
        pq.pq_kv4_slots(n, i32([1, 1]), d["table"], i32([0, 1]), 16, 2, kv_len_out=n)
    with pytest.raises((TypeError, ValueError)):
        pq.pq_kv4_attention(d["q"].float(), d["cu"], d["kv"], d["table"], d["kc"], d["vc"], d["ks"], d["vs"], 0.1, 5)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)                    # as if another device were the current one
    with pytest.raises(ValueError):
        call(pq, d, 5)


@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("q_len", [1, 30, 47, 48, 49, 130])
def test_one_request_and_any_hint(pq, group, q_len):
    """One request alone, and with a second one beside it (which may go to another kernel), whatever the caller says of its rows."""
    check_attention(pq, attention_case([333], [q_len], 8, 2, 128, q_len, group, 16, prefix=35), hints=(q_len, 1, 40, 1000))
    check_attention(pq, attention_case([100, 333], [3, q_len], 8, 2, 128, q_len + 1, group, 16), hints=(q_len, 1000))


# (a table of half a million tokens, as a server's may be: the kernel for few rows takes 32 of them at once)
@pytest.mark.parametrize("D,group", [(64, 0), (64, 32), (64, 64), (128, 0), (128, 32), (128, 64), (128, 128)])
@pytest.mark.parametrize("case", ["ragged", "prefix", "none", "sharp", "steps"])
def test_few_rows_under_a_long_table(pq, D, group, case):
    if case == "steps" and group == 0:
        pytest.skip("dynamic steps")
    c = attention_case([300, 133, 0, 64, 31, 1], [9, 48, 2, 20, 0, 1], 4, 1, D, 101, group, 64, W=8192, prefix=37 if case == "prefix" else 0,
                       q_size=40.0 if case == "sharp" else 1.5)
    if case == "none":
        c["table"][0, 1], c["table"][1, 0], c["table"][3, 0] = -1, 1 << 30, len(c["kc"])
    if case == "steps":
        r = np.random.default_rng(0)
        live = np.isfinite(c["vs"])
        c["vs"][live] = (10.0 ** r.uniform(-9, 3, live.sum())).astype(np.float32)
    first = check_attention(pq, c)
    assert np.array_equal(first, check_attention(pq, c))
    check_attention(pq, c, causal=False)


# (groups of 4 heads and more than 48 queries: the kernel for many rows)
@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_prompts_over_pages_that_are_none(pq, group, causal):
    c = attention_case([200, 170, 133], [100, 60, 70], 8, 2, 128, 91, group, 16)
    c["table"][0, 1], c["table"][0, 3], c["table"][0, 12], c["table"][1, 0], c["table"][2, :9] = -1, 1 << 30, len(c["kc"]), -7, -1
    spare = next(p for p in range(len(c["kc"])) if p not in c["table"])            # page 0 stands in for those that are none: NaN there too
    if group:
        for n in ("kc", "vc", "ks", "vs"):
            c[n][spare] = c[n][0]
        c["table"] = np.where(c["table"] == 0, spare, c["table"]).astype(np.int32)
        c["ks"][0] = c["vs"][0] = np.nan
    check_attention(pq, c, causal)


def test_prompts_of_lengths_out_of_range(pq):
    c = attention_case([60, 64, 5], [60, 64, 50], 8, 2, 128, 92, ps=16, W=4)
    c["kv"][:] = [-3, 1 << 30, 5]                                                  # more queries than tokens: the first see nothing
    c["table"][1] = [0, 1, 2, 3]
    check_attention(pq, c)


@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("D", [64, 128])
def test_prompts_with_a_sharp_softmax_and_long_tails(pq, group, D):
    if group > D:
        pytest.skip("a group is no longer than a head")
    check_attention(pq, attention_case([700, 400], [110, 50], 8, 2, D, 93, group, 64, prefix=2, q_size=60.0))
    check_attention(pq, attention_case([3000], [50], 8, 2, D, 94, group, 64, q_size=1e-3))


@pytest.mark.parametrize("D,group", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)])
@pytest.mark.parametrize("prefix", [0, 40])
def test_prompts_with_dynamic_steps_over_a_wide_range(pq, D, group, prefix):
    c = attention_case([400, 150], [60, 55], 8, 2, D, 95, group, 64, prefix=prefix)
    r = np.random.default_rng(0)
    live = np.isfinite(c["vs"])
    c["vs"][live] = (10.0 ** r.uniform(-9, 4, live.sum())).astype(np.float32)
    check_attention(pq, c)


@pytest.mark.parametrize("group", [0, 32, 128])
def test_one_prompt_in_parts(pq, group):
    """Histories in many parts, some of them empty: a table far longer than the history."""
    for n in (1, 63, 600, 2100):
        check_attention(pq, attention_case([n], [min(n, 60)], 4, 1, 128, n, group, 64, W=500, prefix=2), hints=(60,))


def test_sizes_of_one(pq):
    """One page, one token, one head; no request; no token."""
    c = attention_case([1], [1], 1, 1, 64, 83, 0, 16)
    check_attention(pq, c)
    c = attention_case([0, 0], [1, 2], 2, 1, 128, 84, 0, 16)
    assert not check_attention(pq, c).any()
    d = put(c)
    empty = torch.empty((0, 256), dtype=torch.float16, device="cuda")
    got, _ = pq.pq_kv4_attention(empty, i32([0, 0, 0]), i32([0, 0]), d["table"], d["kc"], d["vc"], d["ks"], d["vs"], 0.1, 1)
    assert got.shape == (0, 256)
    got, _ = pq.pq_kv4_attention(d["q"], i32([0]), i32([]), i32(np.zeros((0, 4), np.int32)), d["kc"], d["vc"], d["ks"], d["vs"], 0.1, 1)
    assert not host(got).any()

"""The three calls on the paged 4-bit KV cache against plain implementations in 64 bits (kv4_reference.py): whole numbers and codes
equal, attention within the bound that its roundings add up to."""

import numpy as np
import pytest
import torch

import kv4_reference as R
import oracle as O
from pq_testlib import dev, host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pq():
    import paper_2410_05265_amd.binding as b
    b.lib()
    return b


def i32(a):
    return dev(np.asarray(a, dtype=np.int32))


# ------------------------------------------------------------------------------------------------ slots
def lengths(B, kv, q, seed):
    r = np.random.default_rng(seed)
    return r.integers(0, kv + 1, B).astype(np.int32), r.integers(0, q + 1, B).astype(np.int32)


def check_slots(pq, kv, q, W, ps, n_free, T, taken=None, offset=0, seed=0):
    r = np.random.default_rng(seed + 1)
    B = len(kv)
    table = np.full((B, W), -1, np.int32)
    for b in range(B):
        n = min(W, -(-max(int(kv[b]), 0) // ps))
        table[b, :n] = r.integers(0, 100000, n)
    free = r.permutation(n_free).astype(np.int32)
    want = R.slots(kv, q, table, free, ps, T, 0 if taken is None else taken, offset)
    t = dev(table)
    got = pq.pq_kv4_slots(dev(kv), dev(q), t, dev(free), ps, T, taken=None if taken is None else i32([taken]), position_offset=offset)
    for w, g in zip(want[:5], (t,) + got[:4]):
        assert np.array_equal(w, host(g))
    assert int(host(got[4])[0]) == want[5]


@pytest.mark.parametrize("B", [1, 2, 15, 16, 17, 64, 255, 300])
@pytest.mark.parametrize("ps", [16, 64])
def test_slots(pq, B, ps):
    kv, q = lengths(B, 500, 40, B)
    check_slots(pq, kv, q, 40, ps, 4 * B + 600, -(-int(q.sum()) // 32) * 32 + 32, seed=B)


def test_slots_edges(pq):
    one = np.array([1], np.int32)
    check_slots(pq, 0 * one, one, 1, 16, 1, 1)                                     # the first token of the first request
    check_slots(pq, np.array([16, 15, 0, 31], np.int32), np.array([1, 1, 0, 1], np.int32), 2, 16, 5, 3)     # around a page's end
    check_slots(pq, np.array([5, -3, 7], np.int32), np.array([-1, 2, 3], np.int32), 4, 16, 4, 8)            # negative counts as none
    check_slots(pq, np.array([30, 20, 10], np.int32), np.array([10, 30, 50], np.int32), 3, 16, 2, 96)       # the list ends
    check_slots(pq, np.array([60, 40], np.int32), np.array([10, 30], np.int32), 4, 16, 9, 64)               # the table ends
    check_slots(pq, np.array([3, 200], np.int32), np.array([4, 1], np.int32), 4, 16, 9, 5, taken=7, offset=3)
    check_slots(pq, np.array([0, 3], np.int32), np.array([20, 20], np.int32), 4, 16, 9, 25)                 # more tokens than rows
    check_slots(pq, np.array([0], np.int32), np.array([20], np.int32), 4, 16, 0, 20)                        # no page left at all
    check_slots(pq, np.array([7], np.int32), np.array([100001], np.int32), 2000, 64, 3000, 100096)          # one long prompt
    check_slots(pq, np.zeros(3, np.int32), np.zeros(3, np.int32), 4, 16, 3, 40)                             # nothing new, all padding


def test_slots_without_requests(pq):
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    cu, kv, pos, slot, taken = pq.pq_kv4_slots(none, none, torch.empty((0, 3), dtype=torch.int32, device="cuda"), i32([4, 5]), 16, 7, taken=i32([1]))
    assert host(cu).tolist() == [0] and host(pos).tolist() == [0] * 7 and host(slot).tolist() == [-1] * 7 and host(taken).tolist() == [1]


def test_slots_call_after_call(pq):
    """Steps in a row use the list on; a request's slots never meet another's."""
    B, W, ps = 5, 6, 16
    free = np.random.default_rng(1).permutation(30).astype(np.int32)
    table, kv, taken = dev(np.full((B, W), -1, np.int32)), i32([0] * B), None
    seen = set()
    for step in range(20):
        q = np.array([(step + b) % 4 for b in range(B)], np.int32)
        T = int(q.sum())
        cu, kv, pos, slot, taken = pq.pq_kv4_slots(kv, dev(q), table, dev(free), ps, T, taken=taken)
        new = host(slot).tolist()
        assert min(new, default=0) >= 0 and not seen & set(new) and len(set(new)) == T
        seen |= set(new)
    assert int(host(taken)[0]) == sum(-(-int(n) // ps) for n in host(kv))


# ----------------------------------------------------------------------------------------------- append
def rope_table(rd, positions=2000):
    a = np.arange(positions)[:, None] * 10000.0 ** (-np.arange(0, rd, 2) / rd)
    return np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)


def append_case(T, Hq, Hkv, D, seed, group, ps=16, extra=3):
    r = np.random.default_rng(seed)
    c = dict(qkv=(r.standard_normal((T, (Hq + 2 * Hkv) * D)) * np.exp(0.5 * r.standard_normal((Hq + 2 * Hkv) * D))).astype(np.float16))
    pages = -(-T // ps) + extra
    c["slots"] = r.permutation(pages * ps)[:T].astype(np.int64)
    c["positions"] = r.integers(0, 2000, T).astype(np.int32)
    shape = (pages, Hkv, ps)
    for n in "kv":
        c[n + "c"] = r.integers(0, 256, shape + (D // 2,)).astype(np.uint8)
        c[n + "s"] = r.uniform(0.3, 1.5, shape + (D // group,) if group else (Hkv,)).astype(np.float32)
    return c


def check_append(pq, c, Hq, Hkv, D, group=0, norm=None, cos_sin=None, interleaved=False, rotate=True, clip=1.0, eps=1e-6, stride=None):
    T = len(c["slots"])
    x = c["qkv"].reshape(T, Hq + 2 * Hkv, D)
    qw, kw = norm if norm is not None else (None, None)
    z = {"q": R.turn(x[:, :Hq], qw, eps, cos_sin, c["positions"], interleaved, rotate),
         "k": R.turn(x[:, Hq:Hq + Hkv], kw, eps, cos_sin, c["positions"], interleaved, rotate), "v": x[:, Hq + Hkv:].astype(np.float64)}
    kc, vc, ks, vs = (dev(c[n]) for n in ("kc", "vc", "ks", "vs"))
    ps, pages = c["kc"].shape[2], c["kc"].shape[0]
    qkv = dev(c["qkv"])
    if stride:
        wide = torch.full((T, stride), 7.0, dtype=torch.float16, device="cuda")
        wide[:, :qkv.shape[1]] = qkv
        qkv = wide[:, :qkv.shape[1]]
    out = torch.full((T, Hq * D), 9.0, dtype=torch.float16, device="cuda")
    got = pq.pq_kv4_append(qkv, Hq, dev(c["positions"]), dev(c["slots"]), kc, vc, ks, vs, q_weight=None if qw is None else dev(qw),
                           k_weight=None if kw is None else dev(kw), eps=eps, cos_sin=None if cos_sin is None else dev(cos_sin),
                           interleaved=interleaved, rotate=rotate, group=group, clip=clip, out=out)
    live = (c["slots"] >= 0) & (c["slots"] < pages * ps)
    page, at = c["slots"][live] // ps, c["slots"][live] % ps
    q = host(got).astype(np.float64).reshape(T, Hq, D)
    # queries: 16 roundings of the vector's length in the fp32 path, one to fp16
    length = np.sqrt((z["q"] ** 2).sum(-1, keepdims=True))
    assert np.all((np.abs(q - z["q"]) <= 2.0 ** -20 * length + 2.0 ** -11 * np.abs(z["q"]) + 2.0 ** -25)[live])
    assert np.all(q[~live] == 9.0)
    for n, codes, scales in (("k", kc, ks), ("v", vc, vs)):
        want_c, want_s = c[n + "c"].copy(), c[n + "s"].copy()
        y = z[n][live]
        if group:
            step = R.steps_of(y, group, clip)
            stored = host(scales)[page, :, at]
            # Both sides round to fp32.  A key's channels come out of the fp32 path with at most 12 roundings of 2^-24 of the vector's length
            # (the norm's weight, two of the position rotation, seven butterflies, two of the multiplier), and the norm's factor, common to
            # all, with half of the 12 of its sum of squares, half of one for the mean, 2^-23 of the reciprocal root: 8.5 * 2^-24.  The
            # largest moves by no more than that, and the step by clip / 7 of it.
            off = 2.0 ** -23 * step
            if n == "k":
                off += clip / 7 * (12 * 2.0 ** -24 * np.sqrt((y ** 2).sum(-1, keepdims=True)) + 8.5 * 2.0 ** -24 * np.abs(y).max(-1, keepdims=True))
            assert np.all(np.abs(stored.astype(np.float64) - step) <= off)
            want_s[page, :, at] = stored
            step = np.repeat(stored, group, -1)
        else:
            step = c[n + "s"][None, :, None]
        want_c[page, :, at] = R.pack(R.codes_of(y, step))
        assert np.array_equal(host(codes), want_c)
        assert np.array_equal(host(scales), want_s)


@pytest.mark.parametrize("T", [1, 3, 4, 5, 33, 130])
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 2, 128), (1, 1, 64), (10, 2, 64), (32, 8, 128), (3, 3, 128)])
def test_append_static(pq, T, Hq, Hkv, D):
    check_append(pq, append_case(T, Hq, Hkv, D, T, 0), Hq, Hkv, D, cos_sin=rope_table(D))


@pytest.mark.parametrize("D,group", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)])
@pytest.mark.parametrize("rotate", [True, False])
@pytest.mark.parametrize("clip", [1.0, 0.875])
def test_append_dynamic(pq, D, group, rotate, clip):
    c = append_case(70, 4, 2, D, group, group)
    c["qkv"][5] = 0                                                # a token of zeros: step 1
    check_append(pq, c, 4, 2, D, group=group, rotate=rotate, clip=clip, cos_sin=rope_table(D), interleaved=True)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rd", [16, 32, 48, 64, 96, 128])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_position_rotation(pq, D, rd, interleaved):
    if rd > D:
        rd -= D
    check_append(pq, append_case(37, 4, 2, D, rd, 0), 4, 2, D, cos_sin=rope_table(rd), interleaved=interleaved)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rotate", [True, False])
def test_append_norm(pq, D, rotate):
    r = np.random.default_rng(D)
    w = tuple(np.exp(0.3 * r.standard_normal(D)).astype(np.float16) for _ in range(2))
    c = append_case(41, 4, 2, D, 5, 0)
    check_append(pq, c, 4, 2, D, norm=w, rotate=rotate, cos_sin=rope_table(D), eps=1e-5)
    check_append(pq, c, 4, 2, D, norm=(w[0], None), rotate=rotate)                 # only one of the two
    check_append(pq, c, 4, 2, D, norm=(None, w[1]), rotate=rotate)


def test_append_padding_slots_positions_and_strides(pq):
    c = append_case(50, 4, 2, 128, 3, 0)
    c["slots"][[0, 7, 8, 9, 10, 49]] = -1
    c["slots"][[20, 21]] = [c["kc"].shape[0] * 16, 1 << 40]                        # past the cache
    c["positions"][[30, 31]] = [-5, 10 ** 9]                                       # clamped to the table
    check_append(pq, c, 4, 2, 128, cos_sin=rope_table(128), stride=8 * 128 + 72)


def test_append_borders(pq):
    """Quotients on and next to the border between two codes, in values and in keys: decided as in 64 bits."""
    r = np.random.default_rng(2)
    T, Hkv, D = 64, 2, 128
    c = append_case(T, 2, Hkv, D, 9, 0)
    s = c["vs"].astype(np.float64)
    k = r.integers(-10, 10, (T, Hkv, D))
    c["qkv"].reshape(T, 6, D)[:, 4:] = ((k + 0.5) * s[None, :, None]).astype(np.float16)
    c["qkv"].reshape(T, 6, D)[:, 2:4] = ((k + 0.5) * c["ks"].astype(np.float64)[None, :, None]).astype(np.float16)
    check_append(pq, c, 2, Hkv, D, rotate=False)
    c["vs"][:], c["ks"][:] = 0.25, 0.125                                           # exact ties
    c["qkv"].reshape(T, 6, D)[:, 4:] = ((k + 0.5) * 0.25).astype(np.float16)
    c["qkv"].reshape(T, 6, D)[:, 2:4] = ((k + 0.5) * 0.125).astype(np.float16)
    check_append(pq, c, 2, Hkv, D, rotate=False)
    c = append_case(T, 2, Hkv, 64, 9, 0)                                           # 1 / sqrt(64) is exact: rotated sums tie as well
    c["ks"][:] = 0.5
    c["qkv"][:] = r.integers(-3, 4, c["qkv"].shape).astype(np.float16)
    check_append(pq, c, 2, Hkv, 64)


def test_append_large_and_small(pq):
    c = append_case(30, 2, 2, 128, 4, 128)
    c["qkv"][::3] *= np.float16(2.0 ** -12)
    c["qkv"][1::3] = (c["qkv"][1::3].astype(np.float32) * 3000).clip(-60000, 60000).astype(np.float16)
    # (queries of that size leave fp16's range behind the rotation: only the cache is looked at)
    kc, vc, ks, vs = (dev(c[n]) for n in ("kc", "vc", "ks", "vs"))
    pq.pq_kv4_append(dev(c["qkv"]), 2, dev(c["positions"]), dev(c["slots"]), kc, vc, ks, vs, group=128)
    z = R.turn(c["qkv"].reshape(30, 6, 128)[:, 2:4], None, 0, None, None, False, True)
    page, at = c["slots"] // 16, c["slots"] % 16
    assert np.array_equal(host(kc)[page, :, at], R.pack(R.codes_of(z, R.steps_of(z, 128, 1.0))))


def test_append_codes_are_those_of_the_contiguous_quantizer(pq):
    T, Hq, Hkv, D = 48, 4, 2, 128
    c = append_case(T, Hq, Hkv, D, 6, 0)
    kc, vc, ks, vs = (dev(c[n]) for n in ("kc", "vc", "ks", "vs"))
    pq.pq_kv4_append(dev(c["qkv"]), Hq, None, dev(c["slots"]), kc, vc, ks, vs)
    v = np.ascontiguousarray(c["qkv"][:, (Hq + Hkv) * D:])
    codes = host(pq.pq_rotate_quant_heads(dev(v), Hkv, False, vs)).reshape(T, Hkv, D // 2)
    assert np.array_equal(host(vc)[c["slots"] // 16, :, c["slots"] % 16], codes)


# -------------------------------------------------------------------------------------------- attention
def attention_case(kv, q_lens, Hq, Hkv, D, seed, group=0, ps=16, W=None, prefix=0, q_size=1.5, q_rows=None):
    """A cache whose every place that no request holds is filled with what must not be read."""
    r = np.random.default_rng(seed)
    B = len(kv)
    need = [-(-max(int(n), 0) // ps) for n in kv]
    W = W or max(max(need), 1)
    n_pages = sum(need) + 2
    order = r.permutation(n_pages).astype(np.int32)
    table = np.full((B, W), -1, np.int32)
    table[:, :] = np.where(r.random((B, W)) < 0.5, -1, n_pages + 5)                # unused entries: none, or out of range
    c = dict(kv=np.asarray(kv, np.int32), cu=np.concatenate([[0], np.cumsum(q_lens)]).astype(np.int32), group=group, scale=1 / np.sqrt(D))
    for n in "kv":
        c[n + "c"] = r.integers(0, 256, (n_pages, Hkv, ps, D // 2)).astype(np.uint8)
        c[n + "s"] = np.full((n_pages, Hkv, ps, D // group), np.nan, np.float32) if group else r.uniform(0.2, 0.6, Hkv).astype(np.float32)
    at = 0
    for b in range(B):
        pages = order[at:at + need[b]]
        at += need[b]
        table[b, :need[b]] = pages
        if group:
            for n in "kv":
                s = np.full((need[b] * ps, Hkv, D // group), np.nan, np.float32)
                s[:int(kv[b])] = r.uniform(0.05, 0.6, (int(kv[b]), Hkv, D // group))
                c[n + "s"][pages] = s.reshape(need[b], ps, Hkv, D // group).transpose(0, 2, 1, 3)
    c["table"] = table
    T = q_rows or int(c["cu"][-1])
    c["q"] = (q_size * r.standard_normal((T, Hq * D))).astype(np.float16)
    c["pk"], c["pv"] = (((2.0, 0.3)[i] * r.standard_normal((prefix, Hkv, D))).astype(np.float16) if prefix else None for i in range(2))
    return c


def put(c):
    return {k: (dev(v) if isinstance(v, np.ndarray) else v) for k, v in c.items()}


def call(pq, d, max_q, causal=True, out=None, ws=None):
    return pq.pq_kv4_attention(d["q"], d["cu"], d["kv"], d["table"], d["kc"], d["vc"], d["ks"], d["vs"], d["scale"], max_q, group=d["group"],
                               prefix_k=d["pk"], prefix_v=d["pv"], causal=causal, out=out, workspace=ws)[0]


def within(c, got, causal=True):
    want, bound, real = R.attention(c["q"], c["cu"], c["kv"], c["table"], c["kc"], c["vc"], c["ks"], c["vs"], c["scale"], c["group"], c["pk"],
                                    c["pv"], causal)
    got = got.astype(np.float64).reshape(want.shape)
    # fp16 ends at 65504, and what lies above 65520 = 65504 + half a step rounds to infinity
    past = np.isinf(got) & (np.sign(got) == np.sign(want)) & (np.abs(want) + bound >= 65520)
    err = np.abs(np.where(past, want, got) - want)
    worst = (err / np.maximum(bound, 1e-30))[real].max(initial=0.0)
    assert worst <= 1.0, "error is %.3g times its bound" % worst
    return real


def check_attention(pq, c, causal=True, hints=None):
    d = put(c)
    most = int(np.diff(c["cu"]).max(initial=1))
    first = None
    for hint in hints or (max(most, 1),):
        out = torch.full(c["q"].shape, 5.0, dtype=torch.float16, device="cuda")
        got = host(call(pq, d, hint, causal, out))
        real = within(c, got, causal)
        assert np.all(got[~real] == 5.0)                           # rows of no request are left as they were
        first = got if first is None else first
    return first


KV = [0, 1, 15, 16, 17, 31, 32, 33, 64, 127, 128, 129, 300]


@pytest.mark.parametrize("D,group", [(64, 0), (64, 32), (64, 64), (128, 0), (128, 32), (128, 64), (128, 128)])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 2), (5, 1), (8, 1)])
def test_decode(pq, D, group, Hq, Hkv):
    check_attention(pq, attention_case(KV, [1] * len(KV), Hq, Hkv, D, Hq + D, group))


@pytest.mark.parametrize("group", [0, 32, 128])
@pytest.mark.parametrize("ps", [16, 32, 64, 128, 1024])
@pytest.mark.parametrize("prefix", [0, 1, 3, 40])
def test_pages_and_prefix(pq, group, ps, prefix):
    check_attention(pq, attention_case([0, 5, 200, 1100], [1, 1, 2, 1], 4, 2, 128, ps + prefix, group, ps, prefix=prefix))


@pytest.mark.parametrize("D,group", [(64, 0), (64, 32), (128, 0), (128, 64), (128, 128)])
@pytest.mark.parametrize("causal", [True, False])
def test_ragged_queries(pq, D, group, causal):
    kv, q = [300, 40, 3, 77, 130, 16, 0, 9], [5, 40, 9, 0, 130, 1, 2, 9]           # q > kv: rows that see nothing
    check_attention(pq, attention_case(kv, q, 4, 2, D, 11, group, 32, prefix=0), causal)
    check_attention(pq, attention_case(kv, q, 6, 1, D, 12, group, 16, prefix=2), causal)


@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("Hq,Hkv", [(2, 2), (8, 2)])
@pytest.mark.parametrize("q_len", [17, 63, 64, 65, 200, 333])
def test_prompts(pq, group, Hq, Hkv, q_len):
    check_attention(pq, attention_case([q_len, q_len + 70], [q_len, q_len], Hq, Hkv, 128, q_len, group, 64, prefix=3))


@pytest.mark.parametrize("group", [0, 64])
def test_hint_of_the_most_queries_does_not_matter(pq, group):
    c = attention_case([90, 200, 33], [3, 120, 1], 4, 2, 128, 8, group, 32, prefix=1)
    check_attention(pq, c, hints=(1, 4, 17, 120, 4096))


@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("q_len", [1, 40])
def test_pages_that_are_none(pq, group, q_len):
    """Entries of the table outside the cache: their tokens are not seen, and nothing is read there."""
    c = attention_case([100, 70, 33], [q_len, min(q_len, 70), 1], 4, 2, 128, 21, group, 16)
    c["table"][0, 1], c["table"][0, 3], c["table"][1, 0], c["table"][2, :3] = -1, 1 << 30, len(c["kc"]), -7
    check_attention(pq, c)


def test_lengths_out_of_range(pq):
    c = attention_case([40, 64, 5], [1, 1, 1], 4, 2, 128, 22, ps=16, W=4)
    c["kv"][:] = [-3, 1 << 30, 5]
    c["table"][1] = [0, 1, 2, 3]
    check_attention(pq, c)


@pytest.mark.parametrize("group", [0, 32, 128])
def test_sharp_softmax_and_long_tails(pq, group):
    """Scores far apart (the reference moves often), and all alike (a long history of equal weights)."""
    c = attention_case([700, 400], [2, 1], 4, 2, 128, 31, group, 64, prefix=2, q_size=60.0)
    check_attention(pq, c)
    c = attention_case([5000], [1], 4, 2, 128, 32, group, 64, q_size=1e-3)
    check_attention(pq, c)


def test_dynamic_steps_over_a_wide_range(pq):
    c = attention_case([400, 150], [1, 3], 4, 2, 128, 33, 128, 64)
    r = np.random.default_rng(0)
    live = np.isfinite(c["vs"])
    c["vs"][live] = (10.0 ** r.uniform(-9, 4, live.sum())).astype(np.float32)
    check_attention(pq, c)


@pytest.mark.parametrize("group", [0, 128])
def test_long_history_of_few_requests(pq, group):
    c = attention_case([30000, 7], [1, 1], 2, 1, 128, 41, group, 128, prefix=1)
    check_attention(pq, c)


def test_many_requests(pq):
    r = np.random.default_rng(3)
    kv = r.integers(0, 90, 700)
    check_attention(pq, attention_case(kv, r.integers(0, 3, 700), 2, 1, 64, 42, 0, 16))


def test_strided_queries_and_other_streams(pq):
    c = attention_case([150, 60], [4, 30], 4, 2, 128, 51, 0, 32, prefix=1)
    d = put(c)
    wide = torch.full((len(c["q"]), 4 * 128 + 40), float("nan"), dtype=torch.float16, device="cuda")
    wide[:, :512] = d["q"]
    d["q"] = wide[:, :512]
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        got = call(pq, d, 30)
    torch.cuda.synchronize()
    within(c, host(got))


@pytest.mark.parametrize("q_len", [1, 50])
def test_results_are_reproducible_and_other_rows_stay(pq, q_len):
    c = attention_case([5000, 300, 900], [q_len] * 3, 8, 2, 128, 61, 0, 64, prefix=3, q_rows=3 * q_len + 9)
    d = put(c)
    a, b = (host(call(pq, d, q_len)).view(np.uint16) for _ in range(2))
    assert np.array_equal(a, b)
    check_attention(pq, c)


# ----------------------------------------------------------------------------------------- all together
@pytest.mark.parametrize("D,group,prefix", [(128, 0, 3), (64, 32, 0), (128, 128, 1)])
def test_steps_of_a_server(pq, D, group, prefix):
    """Prompts, then decoded tokens with requests that join and rest, padded steps: slots, append and attention on one cache."""
    Hq, Hkv, ps, B, W = 4, 2, 16, 4, 12
    r = np.random.default_rng(7)
    pages = B * W
    free = dev(r.permutation(pages).astype(np.int32))
    table, kv, taken = dev(np.full((B, W), -1, np.int32)), i32([0] * B), None
    shape = (pages, Hkv, ps)
    kc, vc = (torch.zeros(shape + (D // 2,), dtype=torch.uint8, device="cuda") for _ in range(2))
    if group:
        ks, vs = (torch.full(shape + (D // group,), float("nan"), device="cuda") for _ in range(2))
    else:
        ks, vs = (dev(r.uniform(0.3, 0.6, Hkv).astype(np.float32)) for _ in range(2))
    pk, pv = ((dev(r.standard_normal((prefix, Hkv, D)).astype(np.float16)) if prefix else None) for _ in range(2))
    cs = dev(rope_table(D))
    for q_len in ([50, 17, 0, 90], [1, 1, 33, 1], [1, 0, 1, 3], [1, 1, 1, 1], [0, 0, 0, 0], [2, 70, 1, 1]):
        T = sum(q_len) + 5
        cu, kv, pos, slot, taken = pq.pq_kv4_slots(kv, i32(q_len), table, free, ps, T, taken=taken, position_offset=prefix)
        qkv = dev((r.standard_normal((T, (Hq + 2 * Hkv) * D))).astype(np.float16))
        q = pq.pq_kv4_append(qkv, Hq, pos, slot, kc, vc, ks, vs, cos_sin=cs, group=group)
        out, _ = pq.pq_kv4_attention(q, cu, kv, table, kc, vc, ks, vs, D ** -0.5, max(max(q_len), 1), group=group, prefix_k=pk, prefix_v=pv)
        c = dict(q=host(q), cu=host(cu), kv=host(kv), table=host(table), kc=host(kc), vc=host(vc), ks=host(ks), vs=host(vs), scale=D ** -0.5,
                 group=group, pk=None if pk is None else host(pk), pv=None if pv is None else host(pv))
        real = within(c, host(out))
        assert real.sum() == sum(q_len) and not host(out)[~real].any()


@pytest.mark.parametrize("group", [0, 128])
def test_captured_steps_follow_the_lengths(pq, group):
    """A captured decode step (slots, append, attention), replayed while lengths, tables and tokens change underneath; a second graph
    shares the scratch memory."""
    Hq, Hkv, D, ps, B, W = 8, 2, 128, 16, 3, 64
    r = np.random.default_rng(17)
    pages = B * W
    free, table = dev(r.permutation(pages).astype(np.int32)), dev(np.full((B, W), -1, np.int32))
    kv, kv_out, q_len, taken, taken_out = i32([0] * B), i32([0] * B), i32([1] * B), i32([0]), i32([0])
    kc, vc = (torch.zeros((pages, Hkv, ps, D // 2), dtype=torch.uint8, device="cuda") for _ in range(2))
    if group:
        ks, vs = (torch.zeros((pages, Hkv, ps, 1), device="cuda") for _ in range(2))
    else:
        ks, vs = (dev(r.uniform(0.3, 0.6, Hkv).astype(np.float32)) for _ in range(2))
    T = 8
    qkv = torch.zeros((T, (Hq + 2 * Hkv) * D), dtype=torch.float16, device="cuda")
    ws = torch.empty(pq.pq_kv4_attention_workspace_bytes(T, B, Hq, 1, W, kc) + 256, dtype=torch.uint8, device="cuda")
    cu, pos, slot = i32([0] * (B + 1)), i32([0] * T), dev(np.zeros(T, np.int64))
    outs = [torch.zeros((T, Hq * D), dtype=torch.float16, device="cuda") for _ in range(2)]
    q = torch.zeros((T, Hq * D), dtype=torch.float16, device="cuda")

    def step(out):
        pq.pq_kv4_slots(kv, q_len, table, free, ps, T, taken=taken, cu_q=cu, kv_len_out=kv_out, positions=pos, slots=slot, taken_out=taken_out)
        pq.pq_kv4_append(qkv, Hq, pos, slot, kc, vc, ks, vs, group=group, out=q)
        pq.pq_kv4_attention(q, cu, kv_out, table, kc, vc, ks, vs, D ** -0.5, 1, group=group, out=out, workspace=ws)
        kv.copy_(kv_out)
        taken.copy_(taken_out)

    graphs = []
    for out in outs:
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            step(out)
        graphs.append(g)
    for i in range(12):
        qkv.copy_(dev(r.standard_normal(tuple(qkv.shape)).astype(np.float16)))
        if i == 5:                                                 # one request rests, another grows by two
            q_len.copy_(i32([0, 2, 1]))
        if i == 8:                                                 # a jump: as if long prompts had been taken over
            kv.copy_(i32([600, 3, 77]))
            table[:, :40] = dev(r.permutation(B * 40).reshape(B, 40).astype(np.int32))
            if group:
                ks.fill_(0.4)
                vs.fill_(0.3)
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        c = dict(q=host(q), cu=host(cu), kv=host(kv), table=host(table), kc=host(kc), vc=host(vc), ks=host(ks), vs=host(vs), scale=D ** -0.5,
                 group=group, pk=None, pv=None)
        within(c, host(outs[i % 2]))

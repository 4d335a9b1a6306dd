"""The calls on the paged 4-bit KV cache where a step does not fit its rows or its table, and where values are not finite."""

import numpy as np
import pytest
import torch

import kv4_reference as R
from pq_testlib import dev, host
from test_gpu_kv4 import append_case, attention_case, call, check_slots, i32, lengths, pq, put, rope_table   # noqa: F401 (pq: a fixture)

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


@pytest.mark.parametrize("D,rd", [(128, 64), (128, 96), (64, 16), (128, 0)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T", [40, 2400])                          # (a head to a wavefront, and several)
def test_append_infinities_stay_in_their_channel(pq, D, rd, interleaved, T):
    """Channels that do not turn are what they were, whatever their neighbours hold; some vectors take the 64-bit path."""
    Hq, Hkv = 22, 11
    c = append_case(T, Hq, Hkv, D, T + rd, 0)
    r = np.random.default_rng(rd)
    c["ks"][:], c["vs"][:] = 0.25, 0.125
    x = c["qkv"].reshape(T, Hq + 2 * Hkv, D)
    odd = r.random((T, Hq + 2 * Hkv)) < 0.5
    x[odd, rd + 1] = np.float16(0.375)                             # on a border of the keys' codes (1.5 steps) and of the values' (3)
    for what in (np.inf, -np.inf, np.nan):
        at = r.integers(rd, D, (T, Hq + 2 * Hkv))
        put_here = r.random((T, Hq + 2 * Hkv)) < 0.3
        t, h = np.nonzero(put_here)
        x[t, h, at[t, h]] = what
    assert np.isfinite(x[..., :rd]).all()
    z = R.turn(x[:, :Hq + Hkv], None, 0, rope_table(rd) if rd else None, c["positions"], interleaved, False)
    t = [dev(c[n]) for n in ("kc", "vc", "ks", "vs")]
    q = host(pq.pq_kv4_append(dev(c["qkv"]), Hq, dev(c["positions"]), dev(c["slots"]), *t, cos_sin=dev(rope_table(rd)) if rd else None,
                              interleaved=interleaved, rotate=False)).astype(np.float64).reshape(T, Hq, D)
    assert np.array_equal(q[..., rd:], z[:, :Hq, rd:], equal_nan=True)                   # as they came
    assert np.all(np.abs(q[..., :rd] - z[:, :Hq, :rd]) <= 2.0 ** -11 * np.abs(z[:, :Hq, :rd]) + 2.0 ** -20 * 64)   # (pairs no longer than 64)
    page, at = c["slots"] // 16, c["slots"] % 16
    for codes, y, step in ((t[0], z[:, Hq:], c["ks"]), (t[1], x[:, Hq + Hkv:].astype(np.float64), c["vs"])):
        number = ~np.isnan(y)                                      # (a NaN has no code)
        want = R.codes_of(np.where(number, y, 0), step[None, :, None])
        got = R.unpack(host(codes)[page, :, at])
        assert np.array_equal(got[number], want[number])


def test_append_norm_of_zeros_with_the_smallest_eps(pq):
    """x / sqrt(0 + eps) of zeros is zero for any eps above it, subnormal numbers among them."""
    T, Hq, Hkv, D = 20, 4, 2, 128
    c = append_case(T, Hq, Hkv, D, 3, 0)
    c["qkv"][::2] = 0
    w = np.ones(D, np.float16)
    x = c["qkv"].reshape(T, Hq + 2 * Hkv, D)
    for eps in (1e-38, 1e-40, 1.5e-45):
        t = [dev(c[n]) for n in ("kc", "vc", "ks", "vs")]
        q = host(pq.pq_kv4_append(dev(c["qkv"]), Hq, None, dev(c["slots"]), *t, q_weight=dev(w), k_weight=dev(w), eps=eps)).reshape(T, Hq, D)
        z = R.turn(x[:, :Hq + Hkv], w, eps, None, None, False, True)
        length = np.sqrt((z[:, :Hq] ** 2).sum(-1, keepdims=True))
        assert np.all(np.abs(q.astype(np.float64) - z[:, :Hq]) <= 2.0 ** -20 * length + 2.0 ** -11 * np.abs(z[:, :Hq]) + 2.0 ** -25)
        assert np.array_equal(R.unpack(host(t[0])[c["slots"] // 16, :, c["slots"] % 16]), R.codes_of(z[:, Hq:], c["ks"][None, :, None]))


# ------------------------------------------------------------------------------------------------ steps that are cut off
def check_cut(pq, c, T=None, W=None, hints=(1,), causal=True):
    """The first T rows of case c over the first W pages of its table, against the whole case whose table's other entries are none."""
    T, W = T or len(c["q"]), W or c["table"].shape[1]
    whole = dict(c, table=c["table"].copy())
    whole["table"][:, W:] = -1
    want, bound, real = R.attention(whole["q"], c["cu"], c["kv"], whole["table"], c["kc"], c["vc"], c["ks"], c["vs"], c["scale"], c["group"],
                                    c["pk"], c["pv"], causal)
    d = put(dict(c, q=c["q"][:T].copy(), table=c["table"][:, :W].copy()))
    for hint in hints:
        got = host(call(pq, d, hint, causal)).astype(np.float64).reshape(want[:T].shape)
        err = (np.abs(got - want[:T]) / np.maximum(bound[:T], 1e-30))[real[:T]]
        assert err.max(initial=0.0) <= 1.0, "hint %d: error is %.3g times its bound" % (hint, err.max())


def not_appended(c, T):
    """The tokens of rows from T on have never been written: their steps may be anything."""
    if not c["group"]:
        return c
    ps = c["kc"].shape[2]
    for b in range(len(c["kv"])):
        for t in range(max(T, int(c["cu"][b])), int(c["cu"][b + 1])):
            at = int(c["kv"][b]) - (int(c["cu"][b + 1]) - t)
            for n in ("ks", "vs"):
                c[n][c["table"][b, at // ps], :, at % ps] = (np.nan, np.inf)[t % 2]
    return c


@pytest.mark.parametrize("D,group", [(128, 0), (64, 0), (64, 32), (128, 32), (128, 128)])
@pytest.mark.parametrize("kv,q_lens,T", [([10], [10], 6), ([300], [200], 130), ([70, 90, 33], [20, 60, 5], 50), ([300, 200, 40], [150, 170, 9], 200),
                                         ([50, 60, 70], [1, 2, 3], 2), ([333, 333], [130, 200], 131)])
def test_fewer_rows_than_new_tokens(pq, D, group, kv, q_lens, T):
    """pq_kv4_slots gives lengths that count every new token; what the rows there are see does not depend on those that are not there."""
    c = not_appended(attention_case(kv, q_lens, 8, 2, D, T, group, 16, prefix=2), T)
    check_cut(pq, c, T, hints=(1, max(q_lens), 1000))


@pytest.mark.parametrize("D,group", [(128, 0), (64, 32), (128, 128)])
@pytest.mark.parametrize("kv,q_lens,W", [([100], [50], 4), ([100, 64, 65, 300], [50, 40, 3, 100], 4), ([500, 400], [200, 130], 20), ([90, 20], [1, 1], 2)])
@pytest.mark.parametrize("causal", [True, False])
def test_histories_past_the_table(pq, D, group, kv, q_lens, W, causal):
    """Tokens behind the table's pages are not seen; what the others see stays."""
    check_cut(pq, attention_case(kv, q_lens, 8, 2, D, W, group, 16), W=W, hints=(1, max(q_lens), 1000), causal=causal)


@pytest.mark.parametrize("group,T,W", [(0, 60, 12), (128, 60, 12), (0, 300, 5), (64, 200, 6), (0, 20, 4)])
def test_a_step_with_too_few_rows_or_pages(pq, group, T, W):
    """slots, append and attention: more new tokens than rows, more tokens than the table holds."""
    Hq, Hkv, D, ps, q_lens = 8, 2, 128, 16, [30, 100, 0, 70]
    r = np.random.default_rng(T)
    B, pages = len(q_lens), 60
    kv = np.array([5, 0, 20, 17], np.int32)
    shape = (pages, Hkv, ps)
    kc, vc = (r.integers(0, 256, shape + (D // 2,)).astype(np.uint8) for _ in range(2))
    ks, vs = (r.uniform(0.2, 0.6, shape + (D // group,) if group else (Hkv,)).astype(np.float32) for _ in range(2))
    table = np.full((B, W), -1, np.int32)
    order = r.permutation(pages).astype(np.int32)
    for b in range(B):
        table[b, :-(-int(kv[b]) // ps)] = order[2 * b:2 * b + -(-int(kv[b]) // ps)]
    t, kc, vc, ks, vs = dev(table), dev(kc), dev(vc), dev(ks), dev(vs)
    cu, kv_all, pos, slot, _ = pq.pq_kv4_slots(dev(kv), i32(q_lens), t, dev(order[2 * B:]), ps, T, position_offset=1)
    qkv = dev(r.standard_normal((T, (Hq + 2 * Hkv) * D)).astype(np.float16))
    q = torch.zeros((T, Hq * D), dtype=torch.float16, device="cuda")
    pq.pq_kv4_append(qkv, Hq, pos, slot, kc, vc, ks, vs, cos_sin=dev(rope_table(D)), group=group, out=q)
    out, _ = pq.pq_kv4_attention(q, cu, kv_all, t, kc, vc, ks, vs, D ** -0.5, max(q_lens), group=group)
    rows = max(T, sum(q_lens))
    whole = np.zeros((rows, Hq * D), np.float16)
    whole[:T] = host(q)
    wide = np.full((B, 40), -1, np.int32)
    wide[:, :W] = host(t)
    want, bound, real = R.attention(whole, host(cu), host(kv_all), wide, host(kc), host(vc), host(ks), host(vs), D ** -0.5, group)
    got = host(out).astype(np.float64).reshape(want[:T].shape)
    assert np.all((np.abs(got - want[:T]) <= bound[:T])[real[:T]])


# ------------------------------------------------------------------------------------------------ prefix tokens
@pytest.mark.parametrize("D,group", [(64, 0), (128, 0), (64, 32), (128, 128)])
@pytest.mark.parametrize("q_len", [1, 20, 60])
@pytest.mark.parametrize("B", [1, 2])
def test_prefix_values_far_smaller_than_the_steps(pq, D, group, q_len, B):
    """The prefix tokens have nearly all the weight, as attention sinks do, and values below 2 * 10^-4 of a step: the result's error goes by
    its own size, not by the steps'."""
    P = 5
    c = attention_case([3000, 700][:B], [q_len] * B, 4, 1, D, q_len, group, 64, prefix=P)
    r = np.random.default_rng(1)
    if group:
        live = np.isfinite(c["vs"])
        c["vs"][live] = 256.0
        c["ks"][live] = 1e-3
    else:
        c["vs"][:], c["ks"][:] = 256.0, 1e-3
    # Scores: queries and prefix keys have 1 in channel 0, scaled to 20 there; cached keys stay below 8e-3 * sum|q| * scale < 1.
    scale = float(np.float32(c["scale"]))
    c["q"] = (0.01 * r.standard_normal(c["q"].shape)).astype(np.float16)
    c["q"].reshape(len(c["q"]), 4, D)[:, :, 0] = 16.0
    c["pk"][:] = (0.01 * r.standard_normal(c["pk"].shape)).astype(np.float16)
    c["pk"][:, :, 0] = np.float16(2.5 / scale)                     # 40: the cached tokens' weight is e^-40 * 3000 at most
    c["pv"] = r.uniform(0.01, 0.05, c["pv"].shape).astype(np.float16)
    want, _, real = R.attention(c["q"], c["cu"], c["kv"], c["table"], c["kc"], c["vc"], c["ks"], c["vs"], c["scale"], group, c["pk"], c["pv"])
    got = host(call(pq, put(c), q_len)).astype(np.float64).reshape(want.shape)
    err = np.abs(got - want)[real]
    # Half a step of fp16 for each probability (static steps: they stand below the fraction too, so what counts is how far the values, 0.01 to
    # 0.05, lie apart), and for the result, which is below 2^-4; scores of 40 to 2^-20, the cached tokens e^-39 * 3000 * 8 * 256 < 2^-30.
    bound = (0.05 if group else 0.04) * 2.0 ** -11 * 1.01 + 2.0 ** -16 + 2 * 0.05 * 2.0 ** -20 + 2.0 ** -30
    assert err.max() <= bound


@pytest.mark.parametrize("q_len", [1, 60])
@pytest.mark.parametrize("prefix", [0, 3])
def test_ends_of_the_static_steps(pq, q_len, prefix):
    """Steps of 2^-64 and 2^64: codes, attention with all weights alike; scores up to 2^20, where one token has all the weight."""
    least, most = 2.0 ** -64, 2.0 ** 64
    a = append_case(30, 4, 2, 64, 1, 0)
    for step, want in ((least, lambda x: np.clip(np.sign(x) * 8, -8, 7)), (most, lambda x: 0 * x)):
        a["ks"][:] = a["vs"][:] = step
        t = [dev(a[n]) for n in ("kc", "vc", "ks", "vs")]
        pq.pq_kv4_append(dev(a["qkv"]), 4, None, dev(a["slots"]), *t, rotate=False)
        x = a["qkv"].astype(np.float64).reshape(30, 8, 64)
        for codes, y in ((t[0], x[:, 4:6]), (t[1], x[:, 6:])):
            assert np.array_equal(R.unpack(host(codes)[a["slots"] // 16, :, a["slots"] % 16]), want(y))
    c = attention_case([200, 90], [q_len, q_len], 8, 2, 64, 2, 0, 16, prefix=prefix)
    c["ks"][:] = least
    if prefix:
        c["pk"][:] = 0
    for step in (least, 2.0 ** 10):
        c["vs"][:] = step
        check_cut(pq, c, hints=(q_len,))
    # the largest score of the cached tokens decides: the next is further off than fp32 could mistake
    c["ks"][:], c["vs"][:] = 2.0 ** 14, 1.0
    got = host(call(pq, put(c), q_len)).reshape(-1, 8, 64)
    cu, table = c["cu"], c["table"]
    for b, n in enumerate((200, 90)):
        for h in range(2):
            k, v = (R.unpack(x[table[b, :-(-n // 16)], h]).reshape(-1, 64)[:n].astype(np.float64) for x in (c["kc"], c["vc"]))
            for i in range(q_len):
                for g in range(4 * h, 4 * h + 4):
                    s = (k @ c["q"][cu[b] + i, 64 * g:64 * g + 64].astype(np.float64))[:n - (q_len - 1 - i)]
                    assert np.abs(s).max() * 0.125 * 2 ** 14 < 2 ** 20
                    one, two = np.sort(s)[[-1, -2]]
                    if one - two > 2e-4 * np.abs(s).max() and (one > 1 or not prefix):   # (e^-50 and less for the others)
                        assert np.array_equal(got[cu[b] + i, g], v[np.argmax(s)])


# ------------------------------------------------------------------------------------------------ roundings of the weights
def check_result_is_rounded_once(pq, c, q_len):
    """Within half a step of fp16 of the exact result, and 2^-18 of the values (weights of 22 bits, twice; sums and scores in fp32)."""
    want, _, real = R.attention(c["q"], c["cu"], c["kv"], c["table"], c["kc"], c["vc"], c["ks"], c["vs"], c["scale"], c["group"], c["pk"], c["pv"])
    got = host(call(pq, put(c), q_len)).astype(np.float64).reshape(want.shape)
    # (a value is at most 8 * 0.6; sums with the codes' offset 15 + 8 of them, rounded a few times to 2^-24)
    assert np.all((np.abs(got - want) <= 2.0 ** -11 * np.abs(want) + 2.0 ** -18 * 8 * 0.6 + 2.0 ** -25)[real])


@pytest.mark.parametrize("D,group", [(64, 0), (64, 32), (64, 64), (128, 0), (128, 32), (128, 64), (128, 128)])
@pytest.mark.parametrize("prefix", [0, 3])
def test_short_histories_are_rounded_once(pq, D, group, prefix):
    """Histories of one tile: every weight is a large one.  Scores of a few units, off by 2^-20: 2^-19 of a value at most, in the bound above."""
    n = np.arange(1, 33)
    check_result_is_rounded_once(pq, attention_case(n, [1] * 32, 4, 2, D, 5, group, 16, prefix=prefix, q_size=0.2), 1)


@pytest.mark.parametrize("D,group", [(64, 0), (64, 32), (64, 64), (128, 0), (128, 32), (128, 64), (128, 128)])
@pytest.mark.parametrize("q_len", [1, 3])
def test_one_token_with_all_the_weight_is_rounded_once(pq, D, group, q_len):
    """Somewhere in a long history; the others have less than 2^-25 of a value together."""
    kv = [3000, 700, 61, 1500]
    c = attention_case(kv, [q_len] * 4, 4, 2, D, 6, group, 16, q_size=0.3)
    r = np.random.default_rng(8)
    q = c["q"].reshape(-1, 4, D)
    sign = np.where(r.random((4, 2, D)) < 0.5, -1.0, 1.0)          # of each request and key/value head
    for b, n in enumerate(kv):
        lo = int(c["cu"][b])
        for h in range(2):
            q[lo:lo + q_len, 2 * h:2 * h + 2] = np.abs(q[lo:lo + q_len, 2 * h:2 * h + 2]) * sign[b, h] + 2.0 * sign[b, h]
            t = int(r.integers(0, n - q_len))
            page = c["table"][b, t // 16]
            c["kc"][page, h, t % 16] = R.pack(7 * sign[b, h])
            if group:
                c["ks"][page, h, t % 16] = 0.6
            else:
                c["ks"][:] = 0.6
    check_result_is_rounded_once(pq, c, q_len)


# ------------------------------------------------------------------------------------------------ sums over long flat histories
@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("many", [False, True])
def test_means_over_long_histories(pq, group, many):
    """Weights all alike and without a rounding of their own (static steps: it stands above and below the fraction; dynamic ones: the weight is the
    step, of 11 bits, times a power of two), and no round numbers: the sums have to round.  The result is the mean of the values, 4.3 / sqrt(n) of
    a code: far below the offset of 8 that codes may have on their way, whose sums of up to 8 n codes, rounded to half of 2^-24, n / 16 times in a
    row at random, are off by 2^-25 * 8 n * sqrt(n / 16 / 3): 5 % of the result's own rounding (2^-12 of it) for n = 2000 tokens in a row, nine times
    it for 32768.  A denominator that is cut off instead of rounded, 2^-24 of it for each of n / 4 pairs of a lane, is 2^-24 * n / 8 too small: 2^-12 for
    n = 32768.  Right sums leave the result's rounding alone, plus next to nothing."""
    Hq, Hkv, D, ps, W = 32, 8, 128, 1024, 128
    r = np.random.default_rng(9)
    kc, vc = (R.pack(r.integers(-7, 8, (W, Hkv, ps, D))) for _ in range(2))
    shape = (W, Hkv, ps, 1) if group else (Hkv,)
    step = 0.5 * (1 + 683 / 1024)
    ks, vs = (np.full(shape, step, np.float32) for _ in range(2))
    kc[..., 0] = 0x33                                              # channels 0 and 1 of every key: 3
    if many:                                                       # one request of many rows
        B, kv, q_len = 1, np.array([W * ps - 5]), 1024
    else:                                                          # decoded tokens of many requests, over the same pages
        B, q_len = 192, 1
        kv = W * ps - 1 - 9 * np.arange(B)
    table = np.broadcast_to(r.permutation(W).astype(np.int32), (B, W)).copy()
    q = torch.zeros((B * q_len, Hq * D), dtype=torch.float16, device="cuda")
    if not group:
        q.view(-1, Hq, D)[:, :, 0] = 1.7
    out, _ = pq.pq_kv4_attention(q, i32(np.arange(B + 1) * q_len), i32(kv), dev(table), dev(kc), dev(vc), dev(ks), dev(vs), D ** -0.5, q_len, group=group)
    code = R.unpack(vc[table[0]].transpose(0, 2, 1, 3).reshape(W * ps, Hkv, D // 2)).astype(np.int64)
    total = np.cumsum(code, axis=0)
    n = (kv[:, None] - (q_len - 1 - np.arange(q_len))).reshape(-1)
    want = np.repeat(step * total[n - 1] / n[:, None, None], Hq // Hkv, axis=1)
    err = host(out).astype(np.float64).reshape(want.shape) - want
    rounding = want.astype(np.float16).astype(np.float64) - want
    assert np.sqrt((err ** 2).mean()) <= 1.05 * np.sqrt((rounding ** 2).mean())


# ------------------------------------------------------------------------------------------------ very many requests
@pytest.mark.parametrize("B,q,short", [(32768, 3, 0), (32769, 3, 0), (40001, 5, 20000), (100003, 4, 0), (131072, 2, 100000)])
def test_slots_of_more_requests_than_workgroups(pq, B, q, short):
    """A workgroup places several chunks of requests one after another; a list that ends among them."""
    kv, n = lengths(B, 60, q, B)
    check_slots(pq, kv, n, 5, 16, 2 * B - short, int(n.sum()) + 77, taken=3, offset=2, seed=B)


# ------------------------------------------------------------------------------------------------ prompts beside decoding requests
@pytest.mark.parametrize("D,group", [(64, 0), (128, 0), (128, 32)])
@pytest.mark.parametrize("q_lens", [[1] * 7 + [60] + [1] * 24, [49, 1, 65, 2, 1, 129, 48, 0, 1], [1] * 40 + [50, 49, 51]])
def test_prompts_beside_decoding_requests(pq, D, group, q_lens):
    """Requests of 4 heads a key/value head: more than 48 queries take the kernel for many rows, in parts, the others the one for few."""
    r = np.random.default_rng(len(q_lens))
    kv = [m + int(r.integers(0, 900 if m > 2 else 200)) for m in q_lens]
    check_cut(pq, attention_case(kv, q_lens, 4, 1, D, 3, group, 64, W=64, prefix=3), hints=(max(q_lens),))


@pytest.mark.parametrize("D,group", [(64, 0), (128, 64)])
def test_prompts_among_very_many_requests(pq, D, group):
    """More than 512 requests, whose tiles of rows the kernel for many rows looks up in a list: a few prompts, in parts, among others."""
    r = np.random.default_rng(5)
    q_lens = r.integers(0, 3, 600)
    q_lens[[0, 17, 18, 333, 599]] = [70, 49, 130, 48, 65]
    kv = q_lens + r.integers(0, 30, 600)
    kv[[17, 599]] += 700
    check_cut(pq, attention_case(kv, q_lens, 4, 1, D, 4, group, 16, W=128, prefix=1), hints=(130,))


@pytest.mark.parametrize("group", [0, 64])
def test_very_many_prompts(pq, group):
    """1300 requests of more rows than the kernel for few takes, some of none: bit for bit what they are 100 at a time."""
    B, D, ps, pages = 1300, 64, 16, 900
    r = np.random.default_rng(6)
    q_lens = np.where(r.random(B) < 0.1, 0, r.integers(49, 140, B))
    kv = q_lens + r.integers(0, 60, B)
    table = r.integers(0, pages, (B, 16)).astype(np.int32)
    kc, vc = (dev(r.integers(0, 256, (pages, 2, ps, D // 2)).astype(np.uint8)) for _ in range(2))
    ks, vs = (dev(r.uniform(0.2, 0.6, (pages, 2, ps, D // group) if group else 2).astype(np.float32)) for _ in range(2))
    cu = np.concatenate([[0], np.cumsum(q_lens)])
    q = dev((1.5 * r.standard_normal((cu[-1], 8 * D))).astype(np.float16))

    def part(lo, hi):
        return pq.pq_kv4_attention(q[cu[lo]:cu[hi]], i32(cu[lo:hi + 1] - cu[lo]), i32(kv[lo:hi]), dev(table[lo:hi]), kc, vc, ks, vs, D ** -0.5, 139,
                                   group=group)[0]

    whole = part(0, B)
    assert bool(whole.any(dim=1).all())
    assert torch.equal(whole, torch.cat([part(lo, lo + 100) for lo in range(0, B, 100)]))

"""Plain implementations, in 64 bits, of drafted trees and sliding windows on the paged 4-bit cache; attention's bound is that of
kv4_reference.py, whose roundings its kernels share."""

import numpy as np

import kv4_reference as R


def rows_of(cu, kv_len, b, T):
    """(first row, rows that exist, new tokens in all, cached tokens in front of them)."""
    begin, end = int(cu[b]), max(int(cu[b + 1]), int(cu[b]))
    lo, hi = min(begin, T), min(end, T)
    return lo, hi - lo, end - begin, max(int(kv_len[b]), 0) - (end - begin)


def tree(parents, cu, kv_len, T, words, offset=0):
    """(mask int32 [T, words], positions int32 [T]), node by node."""
    mask, pos = np.zeros((T, words), np.uint32), np.zeros(T, np.int32)
    for b in range(len(kv_len)):
        lo, m, _, before = rows_of(cu, kv_len, b, T)
        seen = []
        for i in range(m):
            if m > 32 * words:
                pos[lo + i] = offset + max(before, 0) + i
                continue
            p = int(parents[lo + i])
            seen.append((seen[p] if 0 <= p < i else 0) | 1 << i)
            pos[lo + i] = offset + max(before, 0) + bin(seen[i]).count("1") - 1
            for w in range(words):
                mask[lo + i, w] = seen[i] >> (32 * w) & 0xFFFFFFFF
    return mask.view(np.int32), pos


def accept(tokens, parents, chosen, cu, kv_len, T, table, ps, words, depth, free, taken):
    """(accepted, next_token, path, kv_len_out, from_slots, to_slots, taken_out, free), request by request."""
    B, W = table.shape
    acc, nxt, out = (np.zeros(B, np.int32) for _ in range(3))
    path = np.full((B, depth), -1, np.int32)
    src, dst = (np.full((B, depth), -1, np.int64) for _ in range(2))
    free = free.copy()
    top = min(max(taken, 0), len(free))
    back = 0
    for b in range(B):
        lo, m, _, before = rows_of(cu, kv_len, b, T)
        before = max(before, 0)
        way = [0] if 0 < m <= 32 * words else []
        while way and len(way) < depth:
            at = way[-1]
            fits = [i for i in range(at + 1, m) if parents[lo + i] == at and tokens[lo + i] == chosen[lo + at]]
            if not fits:
                break
            way.append(fits[0])
        acc[b] = len(way) if m <= 32 * words else m
        nxt[b] = -1 if m == 0 else chosen[lo + (way[-1] if way else m - 1)]
        out[b] = before + acc[b]
        path[b, :len(way)] = way

        def slot(t):
            page = table[b, t // ps] if t // ps < W else -1
            return page * ps + t % ps if page >= 0 else -1

        for k, node in enumerate(way):
            f, t = slot(before + node), slot(before + k)
            if node != k and f >= 0 and t >= 0:
                src[b, k], dst[b, k] = f, t
        for col in range(-(-int(out[b]) // ps), min(W, -(-max(int(kv_len[b]), 0) // ps))):
            if table[b, col] >= 0:
                if back < top:
                    free[top - 1 - back] = table[b, col]
                back += 1
    return acc, nxt, path, out, src, dst, np.array([max(top - back, 0)], np.int32), free


def keep(src, dst, arrays, ps, n_pages):
    """Moves in arrays [pages, heads, ps, ...], in place, entry after entry."""
    for f, t in zip(src.ravel(), dst.ravel()):
        if 0 <= f < n_pages * ps and 0 <= t < n_pages * ps:
            for a in arrays:
                a[t // ps, :, t % ps] = a[f // ps, :, f % ps]


def seen_by(i, m, total, kv, n, window, sinks, bits):
    """Which of n cached tokens row i of m sees; bits: its mask as a number, or None of a chain."""
    t, before = np.arange(n), kv - total
    window = window or 1 << 60
    if bits is None:
        p = before + i
        return (t <= p) & ((t < sinks) | (t > p - window))
    nodes = [j for j in range(m) if bits >> j & 1]
    seen = (t < before) & ((t < sinks) | (t >= before + len(nodes) - window))
    for j in nodes:
        if 0 <= before + j < n:
            seen[before + j] = True
    return seen


def attention(c, window=0, sinks=0, mask=None):
    """(out [T, Hq, D] fp64, bound of a right kernel's error, rows that belong to a request) of a case as attention_case makes them."""
    q, cu, kv_len, table, group, scale = c["q"], c["cu"], c["kv"], c["table"], c["group"], np.float64(np.float32(c["scale"]))
    n_pages, Hkv, ps, half = c["kc"].shape
    D, T = 2 * half, len(q)
    Hq = q.shape[1] // D
    per = Hq // Hkv
    out, bound, real = np.zeros((T, Hq, D)), np.zeros((T, Hq, D)), np.zeros(T, bool)
    P = 0 if c["pk"] is None else len(c["pk"])
    for b in range(len(kv_len)):
        lo, m, total, _ = rows_of(cu, kv_len, b, T)
        capacity = table.shape[1] * ps
        kv = max(int(kv_len[b]), 0)
        kv = capacity if kv >= 1 << 30 else kv
        n = min(kv, capacity)
        real[lo:lo + m] = True
        pages = table[b, :-(-n // ps)] if n else table[b, :0]
        good = (pages >= 0) & (pages < n_pages)
        at = np.where(good, pages, 0)
        there = np.repeat(good, ps)[:n]
        tree_of = mask is not None and m <= 32 * mask.shape[1]
        for h in range(Hkv):
            side = []
            for code, s, p in ((c["kc"], c["ks"], c["pk"]), (c["vc"], c["vs"], c["pv"])):
                x = R.unpack(code[at, h]).reshape(-1, D)[:n].astype(np.float64)
                step = np.repeat(s[at, h].reshape(-1, D // group)[:n], group, 1).astype(np.float64) if group else np.float64(s[h])
                x = np.where(there[:, None], x * np.where(np.isfinite(step), step, 0), 0)
                side.append(x if p is None else np.concatenate([p[:, h].astype(np.float64), x]))
            k, v = side
            biggest = np.abs(v).max(initial=0.0)
            for i in range(m):
                bits = sum(int(w) << (32 * j) for j, w in enumerate(mask[lo + i].view(np.uint32))) if tree_of else None
                seen = np.concatenate([np.ones(P, bool), there & seen_by(i, m, total, kv, n, window, sinks, bits)])
                if not seen.any():
                    continue
                ks, vs = k[seen], v[seen]
                for g in range(h * per, (h + 1) * per):
                    x = q[lo + i, g * D:(g + 1) * D].astype(np.float64)
                    s = (ks @ x) * scale
                    w = np.exp(s - s.max())
                    w /= w.sum()
                    o = w @ vs
                    out[lo + i, g] = o
                    # as in kv4_reference.attention, over the tokens that the row sees and those of its tiles that it does not
                    e = ((np.abs(ks) @ np.abs(x)).max() * 3 * D + 8 * np.abs(s).max()) * scale * 2.0 ** -24 + 8 * np.abs(s).max() * 2.0 ** -24
                    big = w @ np.abs(vs) + np.abs(o)
                    bound[lo + i, g] = ((2.0 ** -11 * 1.01 + 2 * e + 2.0 ** -20) * big + (P + n) * 2.0 ** -30 * biggest +
                                        (P + n + 256) / 32 * 2.0 ** -24 * 16 * biggest + 2.0 ** -11 * np.abs(o) + 2.0 ** -25)
    return out, bound, real

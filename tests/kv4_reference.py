"""Plain implementations, in 64 bits, of the three calls on the paged 4-bit cache, and the bounds that a right kernel keeps."""

import numpy as np

import oracle as O


def slots(kv_len, q_len, table, free, ps, T, taken=0, offset=0):
    """(table, cu_q, kv_len_out, positions, slots, taken_out), request by request."""
    table = table.copy()
    W = table.shape[1]
    cu, pos, slot = [0], np.zeros(T, np.int32), np.full(T, -1, np.int64)
    for b, (n, m) in enumerate(zip(kv_len, q_len)):
        n, m = max(int(n), 0), max(int(m), 0)
        for col in range(-(-n // ps), min(W, -(-(n + m) // ps))):
            table[b, col] = free[taken] if taken < len(free) else -1
            taken += 1
        for i in range(m):
            t, p = cu[-1] + i, n + i
            if t < T:
                page = table[b, p // ps] if p // ps < W else -1
                pos[t] = offset + p
                slot[t] = page * ps + p % ps if page >= 0 else -1
        cu.append(cu[-1] + m)
    return table, np.array(cu, np.int32), np.maximum(kv_len, 0) + np.maximum(q_len, 0), pos, slot, taken


def turn(x, weight, eps, cos_sin, positions, interleaved, rotate):
    """Head vectors [T, H, D] fp64: norm, position rotation, Hadamard rotation."""
    y = x.astype(np.float64)
    T, H, D = y.shape
    if weight is not None:
        y = y / np.sqrt((y ** 2).mean(-1, keepdims=True) + np.float64(np.float32(eps))) * weight.astype(np.float64)
    if cos_sin is not None:
        rd = cos_sin.shape[1]
        cs = cos_sin[np.clip(positions, 0, len(cos_sin) - 1)].astype(np.float64)[:, None]
        c, s = cs[..., :rd // 2], cs[..., rd // 2:]
        a, b = (slice(0, rd, 2), slice(1, rd, 2)) if interleaved else (slice(0, rd // 2), slice(rd // 2, rd))
        z = y.copy()
        z[..., a], z[..., b] = y[..., a] * c - y[..., b] * s, y[..., b] * c + y[..., a] * s
        y = z
    if rotate:
        y = O.rotate(y.reshape(T, H * D), D).reshape(T, H, D)
    return y


def steps_of(z, group, clip):
    """fp32 dynamic steps [T, H, D / group] of values [T, H, D]."""
    m = np.abs(z.reshape(z.shape[:2] + (-1, group))).max(-1)
    s = (np.float64(np.float32(clip)) * m / 7.0).astype(np.float32)
    return np.where(s > 0, s, np.float32(1))


def codes_of(z, step):
    return np.clip(np.rint(z / step.astype(np.float64)), -8, 7).astype(np.int8)


def unpack(codes):
    lo = (codes << 4).astype(np.uint8).view(np.int8) >> 4
    hi = codes.view(np.int8) >> 4
    return np.stack([lo, hi], -1).reshape(codes.shape[:-1] + (2 * codes.shape[-1],))


def pack(codes):
    c = codes.astype(np.int8).view(np.uint8)
    return ((c[..., 0::2] & 15) | (c[..., 1::2] << 4)).astype(np.uint8)


def attention(q, cu, kv_len, table, kc, vc, ks, vs, scale, group=0, pk=None, pv=None, causal=True):
    """(out [T, Hq, D] fp64, bound of a right kernel's error, rows that belong to a request)."""
    n_pages, Hkv, ps, half = kc.shape
    D = 2 * half
    T = q.shape[0]
    Hq = q.shape[1] // D
    per = Hq // Hkv
    out, bound, real = np.zeros((T, Hq, D)), np.zeros((T, Hq, D)), np.zeros(T, bool)
    for b in range(len(kv_len)):
        lo, hi = int(cu[b]), int(cu[b + 1])
        n = int(min(max(kv_len[b], 0), table.shape[1] * ps))
        real[lo:hi] = True
        pages = table[b, :-(-n // ps)] if n else table[b, :0]
        good = (pages >= 0) & (pages < n_pages)
        at = np.where(good, pages, 0)
        there = np.repeat(good, ps)[:n]
        for h in range(Hkv):
            side = []
            for c, s, p in ((kc, ks, pk), (vc, vs, pv)):
                code = unpack(c[at, h]).reshape(-1, D)[:n].astype(np.float64)
                step = np.repeat(s[at, h].reshape(-1, D // group)[:n], group, 1).astype(np.float64) if group else np.float64(s[h])
                x = np.where(there[:, None], code * np.where(np.isfinite(step), step, 0), 0)
                side.append(x if p is None else np.concatenate([p[:, h].astype(np.float64), x]))
            P = 0 if pk is None else len(pk)
            seen0 = np.concatenate([np.ones(P, bool), there])
            k, v = side
            biggest = np.abs(v).max(initial=0.0)
            for i in range(hi - lo):
                last = n - (hi - lo - 1 - i) if causal else n
                seen = seen0 & (np.arange(P + n) < P + max(last, 0))
                for g in range(h * per, (h + 1) * per):
                    if not seen.any():
                        continue
                    x = q[lo + i, g * D:(g + 1) * D].astype(np.float64)
                    s = (k[seen] @ x) * np.float64(np.float32(scale))
                    w = np.exp(s - s.max())
                    w /= w.sum()
                    o = w @ v[seen]
                    out[lo + i, g] = o
                    # Scores: fp32 sums of D products (with the offset's three times as large) and four roundings of the result.
                    e = ((np.abs(k[seen]) @ np.abs(x)).max() * 3 * D + 8 * np.abs(s).max()) * np.float64(np.float32(scale)) * 2.0 ** -24
                    e += 8 * np.abs(s).max() * 2.0 ** -24
                    # Probabilities: half a step of fp16, in numerator and denominator; those below 2^-20 of the largest half a step of the
                    # subnormal ones.  The sums with the offset: codes up to 15 in fp32, a rounding for every 32 tokens.
                    big = w @ np.abs(v[seen]) + np.abs(o)
                    bound[lo + i, g] = ((2.0 ** -11 * 1.01 + 2 * e + 2.0 ** -20) * big + (P + n) * 2.0 ** -30 * biggest +
                                        (P + n + 256) / 32 * 2.0 ** -24 * 16 * biggest + 2.0 ** -11 * np.abs(o) + 2.0 ** -25)
    return out, bound, real

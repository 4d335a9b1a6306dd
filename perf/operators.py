"""Serving on a paged KV cache of 4-bit codes: what is measured of its three operators.

  slots      pq_kv4_slots      block table, slots and positions of a step's new tokens from the requests' lengths
  append     pq_kv4_append     per-head norm, position rotation and Hadamard rotation of queries and keys, 4-bit codes of
                               keys and values written to their slots
  attention  pq_kv4_attention  attention over the cache, one token per request up to whole prompts

A page of the cache holds page_size tokens of every key/value head, [n_pages, n_kv_heads, page_size, head_dim / 2] bytes, two
codes per byte with the even channel in the low nibble.  Steps are static, one per head (group = 0), or dynamic, one per `group`
channels of a token.  Head counts are those of the Llama-2-7B, Llama-3-8B and Llama-3-70B blocks and generic ones beside them.

Fields of a case
  slots      B requests, W pages a request may hold, ps tokens of a page, max_kv cached tokens, max_q new ones
  append     T tokens, Hq and Hkv heads of D channels, group, norm, rope ("half", "pairs" or ""), rd channels that it turns,
             rotate (Hadamard), ps, spread (one token each of T requests, else prompts)
  attention  B requests of up to max_kv cached tokens, up to max_q of them new, Hq, Hkv, D, group, prefix (fp16 tokens in front),
             ps, fresh (prompts without history: all cached tokens are new)

Codes are whole numbers: the definition rounds the quotient in double precision, so the bytes of the cache have to be equal.
"""

from __future__ import annotations

import math
import random

import torch

own = False

_MAX_POSITION = 131072 + 64


def listed():
    return [
        # one step of a batch that decodes: the bookkeeping before every layer, all latency
        {"name": "slots_decode", "kind": "slots", "B": 64, "W": 128, "ps": 64, "max_kv": 8000, "max_q": 1},
        # a large server's step with prompts and decoded tokens together
        {"name": "slots_prompts", "kind": "slots", "B": 1500, "W": 512, "ps": 16, "max_kv": 6000, "max_q": 200},
        # one token each of a decode batch through an 8B block: latency and a few megabytes
        {"name": "append_decode_8b", "kind": "append", "T": 64, "Hq": 32, "Hkv": 8, "D": 128, "group": 0, "norm": False,
         "rope": "half", "rd": 128, "rotate": True, "ps": 64, "spread": True},
        # a long prompt of an 8B block, static steps: the ordinary prefill
        {"name": "append_prefill_8b", "kind": "append", "T": 8192, "Hq": 32, "Hkv": 8, "D": 128, "group": 0, "norm": False,
         "rope": "half", "rd": 128, "rotate": True, "ps": 64, "spread": False},
        # a prompt of an odd length through a 70B block with head norms and one step per token and head (group-wise dynamic)
        {"name": "append_dynamic_70b", "kind": "append", "T": 2111, "Hq": 64, "Hkv": 8, "D": 128, "group": 128, "norm": True,
         "rope": "half", "rd": 128, "rotate": True, "ps": 64, "spread": False},
        # one token of one request: what a chat waits for
        {"name": "decode_one", "kind": "attention", "B": 1, "max_q": 1, "max_kv": 1537, "Hq": 32, "Hkv": 8, "D": 128,
         "group": 0, "prefix": 3, "ps": 64, "fresh": False},
        # a ragged decode batch of an 8B block behind its prefix
        {"name": "decode_batch_8b", "kind": "attention", "B": 64, "max_q": 1, "max_kv": 8192, "Hq": 32, "Hkv": 8, "D": 128,
         "group": 0, "prefix": 3, "ps": 64, "fresh": False},
        # a 7B block: every query head has keys and values of its own
        {"name": "decode_mha_7b", "kind": "attention", "B": 24, "max_q": 1, "max_kv": 2300, "Hq": 32, "Hkv": 32, "D": 128,
         "group": 0, "prefix": 4, "ps": 16, "fresh": False},
        # few requests with long histories and dynamic steps: the work has to be split over each history
        {"name": "decode_long_70b", "kind": "attention", "B": 3, "max_q": 1, "max_kv": 131072, "Hq": 64, "Hkv": 8, "D": 128,
         "group": 128, "prefix": 1, "ps": 128, "fresh": False},
        # some drafted tokens of each request are verified at once; small heads, groups of half a head
        {"name": "verify_batch", "kind": "attention", "B": 16, "max_q": 5, "max_kv": 4001, "Hq": 32, "Hkv": 8, "D": 64,
         "group": 32, "prefix": 0, "ps": 32, "fresh": False},
        # a chunk of a long prompt: few rows of queries over a long history
        {"name": "chunk_70b", "kind": "attention", "B": 1, "max_q": 500, "max_kv": 33000, "Hq": 64, "Hkv": 8, "D": 128,
         "group": 0, "prefix": 1, "ps": 64, "fresh": False},
        # prompts of different lengths, causal: the matrix products bound it
        {"name": "prefill_8b", "kind": "attention", "B": 4, "max_q": 4096, "max_kv": 4096, "Hq": 32, "Hkv": 8, "D": 128,
         "group": 0, "prefix": 3, "ps": 64, "fresh": True},
    ]


def _log_between(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """A case of one of the three operators, sizes over their whole ranges."""
    kind = rng.choice(["slots", "append", "append", "attention", "attention", "attention", "attention"])
    ps = rng.choice([16, 32, 64, 128])
    if kind == "slots":
        max_kv, max_q = _log_between(rng, 1, 20000), _log_between(rng, 1, 300)
        return {"kind": kind, "B": _log_between(rng, 1, 1500), "W": -(-(max_kv + max_q) // ps) + rng.randrange(4), "ps": ps,
                "max_kv": max_kv, "max_q": max_q}
    D = rng.choice([64, 128, 128])
    Hkv = rng.choice([1, 2, 4, 8, 8, 16, 32])
    Hq = Hkv * rng.choice([g for g in (1, 2, 4, 5, 8) if Hkv * g <= 64])
    group = rng.choice([0, 0, 0] + [g for g in (32, 64, 128) if g <= D])
    if kind == "append":
        rope = rng.choice(["half", "half", "pairs", ""])
        longest = min(8192, 8192 * 48 * 128 // ((Hq + 2 * Hkv) * D))
        return {"kind": kind, "T": _log_between(rng, 1, longest), "Hq": Hq, "Hkv": Hkv, "D": D, "group": group,
                "norm": rng.random() < 0.4, "rope": rope, "rd": rng.choice([D, D, D // 2]) if rope else 0,
                "rotate": rng.random() < 0.8, "ps": ps, "spread": rng.random() < 0.4}
    while True:
        how = rng.choice(["decode", "decode", "verify", "chunk", "prompt"])
        B = _log_between(rng, 1, 128 if how in ("decode", "verify") else 8)
        max_kv = _log_between(rng, 1, 131072)
        max_q = {"decode": 1, "verify": rng.randint(2, 8), "chunk": _log_between(rng, 9, 2048), "prompt": max_kv}[how]
        # no more than the largest listed cases hold in their plain form, and no more work than the largest
        if max_q <= min(max_kv, 4096) and B * Hkv * max_kv * D <= 280e6 and B * Hq * max_q * max_kv <= 1e9:
            return {"kind": kind, "B": B, "max_q": max_q, "max_kv": max_kv, "Hq": Hq, "Hkv": Hkv, "D": D, "group": group,
                    "prefix": rng.choice([0, 1, 3, 4, 17]), "ps": ps, "fresh": how == "prompt"}


# ---------------------------------------------------------------------------------------------- inputs
def _lengths(case):
    """(cached tokens with the new ones, new tokens) of every request of an attention case: a function of the case alone."""
    r = random.Random("%(B)d %(max_q)d %(max_kv)d" % case)
    kv = [case["max_kv"]] + [r.randint(max(1, case["max_kv"] // 4), case["max_kv"]) for _ in range(case["B"] - 1)]
    if case["fresh"]:
        return kv, list(kv)
    q = [case["max_q"]] + [r.randint(max(1, case["max_q"] // 2), case["max_q"]) for _ in range(case["B"] - 1)]
    return kv, [min(a, b) for a, b in zip(q, kv)]


def _slot_lengths(case):
    """(cached tokens, new tokens) of every request of a slots case."""
    r = random.Random("%(B)d %(max_q)d %(max_kv)d %(ps)d" % case)
    return [r.randint(0, case["max_kv"]) for _ in range(case["B"])], [r.randint(1, case["max_q"]) for _ in range(case["B"])]


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _codes_of(x, step):
    """Packed codes [..., C / 2] of values [..., C] whose steps broadcast against them."""
    c = (x / step).round_().clamp_(-8, 7).to(torch.int8)
    return ((c[..., 0::2] & 15) | (c[..., 1::2] << 4)).view(torch.uint8)


def _cache(gen, pages, case):
    """Codes and steps of rotated keys (or values): near-normal channels, a size of its own for each head."""
    H, ps, D, group = case["Hkv"], case["ps"], case["D"], case["group"]
    size = torch.exp(0.3 * torch.randn((H,), generator=gen, device="cuda"))
    step = (size * 4.0 / 7.0).float()
    codes = torch.empty((pages, H, ps, D // 2), dtype=torch.uint8, device="cuda")
    steps = torch.empty((pages, H, ps, D // group), dtype=torch.float32, device="cuda") if group else step
    some = max(1, (1 << 26) // (H * ps * D))
    for p in range(0, pages, some):
        n = min(some, pages - p)
        x = torch.randn((n, H, ps, D), generator=gen, device="cuda") * size[:, None, None]
        if group:
            g = x.view(n, H, ps, D // group, group)
            s = (g.abs().amax(-1) / 7.0).float()
            steps[p:p + n] = s
            codes[p:p + n] = _codes_of(g, s[..., None]).reshape(n, H, ps, D // 2)
        else:
            codes[p:p + n] = _codes_of(x, step[:, None, None])
    return codes, steps


def _table(gen, kv, ps, W, extra):
    """A block table [B, W] (-1 where a request has no page) over shuffled pages, and how many pages there are."""
    need = [-(-n // ps) for n in kv]
    pages = sum(need) + extra
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    col = torch.arange(W, device="cuda")[None, :]
    n = _int32(need).long()
    at = n.cumsum(0)[:, None] - n[:, None] + col
    return torch.where(col < n[:, None], order[at.clamp(max=pages - 1)], -1).to(torch.int32).contiguous(), pages, order


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000003 * (seed + 1))
    return gen


def _slots_inputs(case, seed):
    gen = _generator(seed)
    kv, q = _slot_lengths(case)
    total = sum(q)
    need = sum(-(-(a + b) // case["ps"]) - -(-a // case["ps"]) for a, b in zip(kv, q))
    table, pages, order = _table(gen, kv, case["ps"], case["W"], need + 7)
    return {"kv_len": _int32(kv), "q_len": _int32(q), "table": table, "free": order[pages - need - 7:].contiguous(),
            "T": -(-total // 64) * 64}                             # a step's buffers are padded


def _rope_table(rd):
    """fp32 [positions, rd]: cosines, then sines; angles in double precision."""
    inv = 500000.0 ** (-torch.arange(0, rd, 2, dtype=torch.float64, device="cuda") / rd)
    a = torch.arange(_MAX_POSITION, dtype=torch.float64, device="cuda")[:, None] * inv
    return torch.cat([a.cos(), a.sin()], 1).float()


def _append_inputs(case, seed):
    gen = _generator(seed)
    T, Hq, Hkv, D, ps = (case[k] for k in ("T", "Hq", "Hkv", "D", "ps"))

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    heads = Hq + 2 * Hkv
    channel = torch.exp(0.5 * normal(heads * D))
    d = {"qkv": (normal(T, heads * D) * channel).half()}
    if case["norm"]:
        d["wq"], d["wk"] = (torch.exp(0.2 * normal(D)).half() for _ in range(2))
    if case["spread"]:
        pages = T + 3
        page = torch.randperm(pages, generator=gen, device="cuda")[:T]
        d["slots"] = page * ps + torch.randint(0, ps, (T,), generator=gen, device="cuda")
        d["positions"] = torch.randint(0, 131072, (T,), generator=gen, device="cuda").to(torch.int32)
    else:
        pages = -(-T // ps) + 3
        order = torch.randperm(pages, generator=gen, device="cuda")
        t = torch.arange(T, device="cuda")
        d["slots"] = order[t // ps] * ps + t % ps
        d["positions"] = (t + int(torch.randint(0, 1000, (1,), generator=gen, device="cuda"))).to(torch.int32)
    shape = (pages, Hkv, ps)
    for name in ("k", "v"):
        d[name + "_codes"] = torch.zeros(shape + (D // 2,), dtype=torch.uint8, device="cuda")
        # a static step is the calibrated extreme over 7; that of normed heads is smaller
        d[name + "_scale"] = (torch.zeros(shape + (D // case["group"],), device="cuda") if case["group"] else
                              ((1.0 if case["norm"] and name == "k" else 1.6) * 4.0 / 7.0 * torch.exp(0.2 * normal(Hkv))).float())
    d["cos_sin"] = _rope_table(case["rd"]) if case["rope"] else None
    return d


def _attention_inputs(case, seed):
    gen = _generator(seed)
    kv, q = _lengths(case)
    D = case["D"]
    table, pages, _ = _table(gen, kv, case["ps"], -(-case["max_kv"] // case["ps"]), 5)
    d = {"kv_len": _int32(kv), "q_len": _int32(q), "table": table, "T": sum(q)}
    d["k_codes"], d["k_scale"] = _cache(gen, pages, case)
    d["v_codes"], d["v_scale"] = _cache(gen, pages, case)
    d["q"] = (1.5 * torch.randn((d["T"], case["Hq"] * D), generator=gen, device="cuda")).half()
    d["cu_q"] = torch.cat([_int32([0]), d["q_len"].cumsum(0).to(torch.int32)])
    for name, size in (("pk", 2.0), ("pv", 0.1)):                 # prefix tokens draw attention and hold small values
        d[name] = (size * torch.randn((case["prefix"], case["Hkv"], D), generator=gen, device="cuda")).half() if case["prefix"] else None
    return d


def prepare(case, seed):
    s = {"case": dict(case)}
    if case["kind"] == "slots":
        s.update(_slots_inputs(case, seed))
        s["taken"] = _int32([0])
        T, B = s["T"], case["B"]
        s["outs"] = {"cu_q": torch.empty(B + 1, dtype=torch.int32, device="cuda"), "kv_len_out": torch.empty_like(s["kv_len"]),
                     "positions": torch.empty(T, dtype=torch.int32, device="cuda"), "slots": torch.empty(T, dtype=torch.int64, device="cuda"),
                     "taken_out": torch.empty(1, dtype=torch.int32, device="cuda")}
    elif case["kind"] == "append":
        s.update(_append_inputs(case, seed))
        s["out"] = torch.empty((case["T"], case["Hq"] * case["D"]), dtype=torch.float16, device="cuda")
    else:
        s.update(_attention_inputs(case, seed))
        s["out"] = torch.empty_like(s["q"])
        # scratch memory as large as any of these calls asks for, kept like a server keeps it
        s["ws"] = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------------------------------ plain forms
def _plain_slots(s):
    c = s["case"]
    ps, W, T = c["ps"], c["W"], s["T"]
    kv, q, table, free = s["kv_len"].long(), s["q_len"].long(), s["table"], s["free"]
    end = kv + q
    before, after = ((kv + ps - 1) // ps).clamp(max=W), ((end + ps - 1) // ps).clamp(max=W)
    need = after - before
    first = s["taken"][0].long() + need.cumsum(0) - need
    col = torch.arange(W, device="cuda")[None, :]
    at = first[:, None] + col - before[:, None]
    page = torch.where((at >= 0) & (at < free.numel()), free[at.clamp(0, free.numel() - 1)], -1)
    table.copy_(torch.where((col >= before[:, None]) & (col < after[:, None]), page, table))
    cu = torch.cat([q.new_zeros(1), q.cumsum(0)])
    t = torch.arange(T, device="cuda")
    b = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    real = b < c["B"]
    b = b.clamp(max=c["B"] - 1)
    at = kv[b] + t - cu[b]
    page = torch.where(at < W * ps, table[b, (at // ps).clamp(0, W - 1)], -1).long()
    slots = torch.where(real & (page >= 0), page * ps + at % ps, -1)
    positions = torch.where(real, at, 0).to(torch.int32)
    return {"table": table, "cu_q": cu.to(torch.int32), "kv_len_out": end.to(torch.int32), "positions": positions, "slots": slots,
            "taken_out": (s["taken"] + need.sum()).to(torch.int32)}


def _hadamard(D, dtype):
    i = torch.arange(D, device="cuda")
    bits = i[:, None] & i[None, :]
    odd = sum((bits >> k) & 1 for k in range(8)) & 1
    return (1 - 2 * odd).to(dtype)


def _plain_heads(x, weight, s, dtype):
    """Norm, position rotation and Hadamard rotation of head vectors [T, H, D], in `dtype`."""
    c = s["case"]
    y = x.to(dtype)
    if c["norm"]:
        y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + 1e-6) * weight.to(dtype)
    if c["rope"]:
        rd = c["rd"]
        cs = s["cos_sin"][s["positions"].long()].to(dtype)[:, None, :]
        cos, sin = cs[..., :rd // 2], cs[..., rd // 2:]
        turned, rest = y[..., :rd], y[..., rd:]
        if c["rope"] == "half":
            a, b = turned[..., :rd // 2], turned[..., rd // 2:]
            turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        else:
            a, b = turned[..., 0::2], turned[..., 1::2]
            turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        y = torch.cat([turned, rest], -1)
    if c["rotate"]:
        y = (y.reshape(-1, c["D"]) @ _hadamard(c["D"], dtype)).reshape(y.shape) / math.sqrt(c["D"])
    return y


def _plain_append(s):
    c = s["case"]
    T, Hq, Hkv, D, group, ps = (c[k] for k in ("T", "Hq", "Hkv", "D", "group", "ps"))
    x = s["qkv"].view(T, Hq + 2 * Hkv, D)
    out = _plain_heads(x[:, :Hq], s.get("wq"), s, torch.float32).half().reshape(T, Hq * D)
    # codes lie next to the borders of the rounding: 64 bits
    keys, values = _plain_heads(x[:, Hq:Hq + Hkv], s.get("wk"), s, torch.float64), x[:, Hq + Hkv:].double()
    page, at = s["slots"] // ps, s["slots"] % ps

    def write(y, codes, scale):
        if group:
            g = y.view(T, Hkv, D // group, group)
            step = (g.abs().amax(-1) / 7.0).float()
            step = torch.where(step > 0, step, torch.ones_like(step))
            scale[page, :, at] = step
            codes[page, :, at] = _codes_of(g, step.double()[..., None]).reshape(T, Hkv, D // 2)
        else:
            codes[page, :, at] = _codes_of(y, scale.double()[None, :, None])

    write(keys, s["k_codes"], s["k_scale"])
    write(values, s["v_codes"], s["v_scale"])
    return _append_outputs(s, out)


def _append_outputs(s, q):
    outs = {"q": q, "k_codes": s["k_codes"], "v_codes": s["v_codes"]}
    if s["case"]["group"]:
        outs["k_scale"], outs["v_scale"] = s["k_scale"], s["v_scale"]
    return outs


def _dense(codes, scale, table, case):
    """Keys or values [B, Hkv, W * ps, D] fp32 of the requests' pages."""
    at = table.long().clamp(min=0)
    p = codes[at].transpose(1, 2)                                  # [B, Hkv, W, ps, D / 2]
    c = torch.stack([((p << 4).view(torch.int8) >> 4), (p.view(torch.int8) >> 4)], -1).flatten(-2)
    if case["group"]:
        step = scale[at].transpose(1, 2)
        x = (c.unflatten(-1, (-1, case["group"])).float() * step[..., None]).flatten(-2)
    else:
        x = c.float() * scale[None, :, None, None, None]
    return x.flatten(2, 3).contiguous()


def _plain_attention(s):
    c = s["case"]
    B, Hq, Hkv, D, mq, T = c["B"], c["Hq"], c["Hkv"], c["D"], c["max_q"], s["T"]
    g = Hq // Hkv
    cu, q_len, kv_len = s["cu_q"].long(), s["q_len"].long(), s["kv_len"].long()
    keys, values = (_dense(s[n + "_codes"], s[n + "_scale"], s["table"], c) for n in ("k", "v"))
    L = keys.shape[2]
    i = torch.arange(mq, device="cuda")
    rows = (cu[:-1, None] + i).clamp(max=T - 1)
    q = s["q"][rows].float().view(B, mq, Hkv, g, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, mq * g, D)
    scores = q @ keys.transpose(2, 3).contiguous()
    seen = torch.arange(L, device="cuda") < (kv_len - q_len)[:, None, None] + 1 + i[None, :, None]      # [B, mq, L]
    scores = scores.view(B, Hkv, mq, g, L).masked_fill_(~seen[:, None, :, None], -math.inf).view(B, Hkv, mq * g, L)
    if c["prefix"]:
        front = q @ s["pk"].float().permute(1, 2, 0).contiguous()
        scores = torch.cat([front, scores], -1)
        values = torch.cat([s["pv"].float().transpose(0, 1)[None].expand(B, -1, -1, -1), values], 2)
    top = scores.amax(-1, keepdim=True).clamp_(min=-1e30)
    p = scores.sub_(top).mul_(1.0 / math.sqrt(D)).exp_()
    o = (p @ values) / p.sum(-1, keepdim=True)
    o = o.view(B, Hkv, mq, g, D).permute(0, 2, 1, 3, 4).reshape(B, mq, Hq * D)
    t = torch.arange(T, device="cuda")
    b = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    return o[b, t - cu[b]].half()


def run(s):
    kind = s["case"]["kind"]
    if not own:
        return {"slots": _plain_slots, "append": _plain_append, "attention": _plain_attention}[kind](s)
    import paper_2410_05265_amd.binding as pq
    c = s["case"]
    if kind == "slots":
        pq.pq_kv4_slots(s["kv_len"], s["q_len"], s["table"], s["free"], c["ps"], s["T"], taken=s["taken"], **s["outs"])
        return {"table": s["table"], **s["outs"]}
    if kind == "append":
        q = pq.pq_kv4_append(s["qkv"], c["Hq"], s["positions"], s["slots"], s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"],
                             q_weight=s.get("wq"), k_weight=s.get("wk"), eps=1e-6, cos_sin=s["cos_sin"],
                             interleaved=c["rope"] == "pairs", rotate=c["rotate"], group=c["group"], out=s["out"])
        return _append_outputs(s, q)
    return pq.pq_kv4_attention(s["q"], s["cu_q"], s["kv_len"], s["table"], s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"],
                               1.0 / math.sqrt(c["D"]), c["max_q"], group=c["group"], prefix_k=s["pk"], prefix_v=s["pv"],
                               out=s["out"], workspace=s["ws"])[0]


# ---------------------------------------------------------------------------------------- what is needed
def work(case):
    if case["kind"] == "slots":
        kv, q = _slot_lengths(case)
        new = sum(-(-(a + b) // case["ps"]) - -(-a // case["ps"]) for a, b in zip(kv, q))
        T = -(-sum(q) // 64) * 64
        return {"bytes": 16.0 * case["B"] + 8.0 * new + 12.0 * T, "flops": 0.0}
    Hq, Hkv, D, group = case["Hq"], case["Hkv"], case["D"], case["group"]
    stored = Hkv * (D + (8 * D // group if group else 0))          # bytes of a token's keys and values
    if case["kind"] == "append":
        T = case["T"]
        flops = T * (Hq + Hkv) * D * ((4 if case["norm"] else 0) + (3 if case["rope"] else 0) + (math.log2(D) if case["rotate"] else 0))
        return {"bytes": float(T * ((2 * Hq + 2 * Hkv) * D * 2 + stored + 12 + 4 * case["rd"])), "flops": float(flops)}
    kv, q = _lengths(case)
    pairs = sum(n * (m - n) + n * (n + 1) // 2 + n * case["prefix"] for m, n in zip(kv, q))
    return {"bytes": float(4 * sum(q) * Hq * D + sum(kv) * stored + 4 * case["prefix"] * Hkv * D), "flops": 4.0 * D * Hq * pairs}


# -------------------------------------------------------------------------------------- the 64-bit result
def _exact_slots(case, seed):
    """The definition, request by request, on the host."""
    d = _slots_inputs(case, seed)
    ps, W, T = case["ps"], case["W"], d["T"]
    kv, q = _slot_lengths(case)
    table, free = d["table"].cpu().tolist(), d["free"].cpu().tolist()
    taken, cu, positions, slots = 0, [0], [], []
    for b, (n, m) in enumerate(zip(kv, q)):
        for col in range(-(-n // ps), min(W, -(-(n + m) // ps))):
            table[b][col] = free[taken] if taken < len(free) else -1
            taken += 1
        for p in range(n, n + m):
            page = table[b][p // ps] if p // ps < W else -1
            positions.append(p)
            slots.append(page * ps + p % ps if page >= 0 else -1)
        cu.append(cu[-1] + m)
    pad = T - cu[-1]
    return {"table": _int32(table), "cu_q": _int32(cu), "kv_len_out": _int32([a + b for a, b in zip(kv, q)]),
            "positions": _int32(positions + [0] * pad), "slots": torch.tensor(slots + [-1] * pad, dtype=torch.int64, device="cuda"),
            "taken_out": _int32([taken])}


def _exact_append(case, seed):
    d = _append_inputs(case, seed)
    T, Hq, Hkv, D, group, ps, rd = (case[k] for k in ("T", "Hq", "Hkv", "D", "group", "ps", "rd"))
    y = d["qkv"].double().view(T, Hq + 2 * Hkv, D).clone()
    turned = slice(0, Hq + Hkv)                                    # queries and keys
    if case["norm"]:
        scale = (y[:, turned].pow(2).sum(-1, keepdim=True) / D + 1e-6).rsqrt()
        weight = torch.cat([d["wq"].double().expand(Hq, D), d["wk"].double().expand(Hkv, D)])
        y[:, turned] *= scale * weight
    if case["rope"]:
        cs = d["cos_sin"].double()[d["positions"].long()]
        angle = torch.complex(cs[:, :rd // 2], cs[:, rd // 2:])[:, None]
        first = slice(0, rd // 2) if case["rope"] == "half" else slice(0, rd, 2)
        second = slice(rd // 2, rd) if case["rope"] == "half" else slice(1, rd, 2)
        z = torch.complex(y[:, turned, first].contiguous(), y[:, turned, second].contiguous()) * angle
        y[:, turned, first], y[:, turned, second] = z.real, z.imag
    if case["rotate"]:
        z = y[:, turned].clone()
        h = 1
        while h < D:                                               # stage by stage
            pair = z.view(T, Hq + Hkv, D // (2 * h), 2, h)
            z = torch.stack([pair[..., 0, :] + pair[..., 1, :], pair[..., 0, :] - pair[..., 1, :]], -2).reshape(T, Hq + Hkv, D)
            h *= 2
        y[:, turned] = z * D ** -0.5
    outs = {"q": y[:, :Hq].reshape(T, Hq * D)}
    flat = torch.stack([d["slots"] // ps, d["slots"] % ps])
    for name, x in (("k", y[:, Hq:Hq + Hkv]), ("v", y[:, Hq + Hkv:])):
        if group:
            biggest = x.unflatten(-1, (D // group, group)).abs().amax(-1)
            step = torch.where(biggest > 0, biggest / 7.0, torch.ones_like(biggest)).float()
            d[name + "_scale"][flat[0], :, flat[1]] = step
            step = step.double().repeat_interleave(group, -1)
        else:
            step = d[name + "_scale"].double()[:, None].expand(Hkv, D)
        code = torch.clamp(torch.round(x / step), -8, 7).long() & 15
        d[name + "_codes"][flat[0], :, flat[1]] = (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8)
        outs[name + "_codes"] = d[name + "_codes"]
        if group:
            outs[name + "_scale"] = d[name + "_scale"].double()
    return outs


def _exact_attention(case, seed):
    d = _attention_inputs(case, seed)
    Hq, Hkv, D, P, ps, group = (case[k] for k in ("Hq", "Hkv", "D", "prefix", "ps", "group"))
    kv, q = _lengths(case)
    per = Hq // Hkv
    out = torch.zeros((d["T"], Hq, D), dtype=torch.float64, device="cuda")
    start = 0
    for b, (n, m) in enumerate(zip(kv, q)):
        pages = d["table"][b, :-(-n // ps)].long()
        for h in range(Hkv):
            side = []
            for name in ("k", "v"):
                raw = d[name + "_codes"][pages, h].reshape(-1, D // 2)[:n].long()
                code = torch.stack([raw % 16, raw // 16], -1).reshape(n, D)
                code = (code - 16 * (code > 7)).double()
                scale = d[name + "_scale"]
                step = scale[pages, h].reshape(-1, D // group)[:n].double().repeat_interleave(group, 1) if group else scale[h].double()
                side.append(torch.cat(([d["p" + name][:, h].double()] if P else []) + [code * step]))
            rows = max(1, (1 << 27) // (per * (n + P)))
            for r in range(0, m, rows):
                e = min(m, r + rows)
                x = d["q"][start + r:start + e].double().view(e - r, Hq, D)[:, h * per:(h + 1) * per].reshape(-1, D)
                w = x @ side[0].t().contiguous() / math.sqrt(D)
                last = torch.arange(r, e, device="cuda").repeat_interleave(per) + n - m + P
                w[torch.arange(n + P, device="cuda")[None] > last[:, None]] = -math.inf
                out[start + r:start + e, h * per:(h + 1) * per] = (torch.softmax(w, -1) @ side[1]).view(e - r, per, D)
        start += m
    return out.reshape(d["T"], Hq * D)


def exact(case, seed):
    return {"slots": _exact_slots, "append": _exact_append, "attention": _exact_attention}[case["kind"]](case, seed)

"""Drafted trees and sliding windows on the paged 4-bit KV cache: what is measured of five operators.

  tree        pq_kv4_tree              ancestor masks and positions of drafted tokens from their parents
  attention   pq_kv4_tree_attention    attention of the drafted tokens of each request over the cache and their own branch
              pq_kv4_window_attention  causal attention over the last `window` tokens and the first `sinks` ones
  accept      pq_kv4_accept            the branch that the model's own choices follow: its nodes, the next token, the slots its
                                       codes have to move between, and the pages of rejected tokens back on the free list
  keep        pq_kv4_keep              codes (and dynamic steps) of accepted tokens to their places, in all layers at once

A request's new tokens are its last ones in the cache.  Up to N = 32 * words of them are the nodes of a tree, in an order where
parents stand in front of their children, node 0 the token that the last step chose; more are a prompt (a chunk of one).  A page of
the cache holds page_size tokens of every key/value head, [n_pages, n_kv_heads, page_size, head_dim / 2] bytes, two codes per byte
with the even channel in the low nibble; steps are static, one per head (group = 0), or dynamic, one per `group` channels of a token.
Head counts are those of the Llama-2-7B, Llama-3-8B and Llama-3-70B blocks and generic ones beside them.

Fields of a case
  tree       B requests with up to `nodes` drafted tokens, `prompts` more with up to max_prompt new tokens, words, max_kv cached
             tokens in front of them
  accept     the same, and ps tokens of a page, depth (most nodes that are accepted)
  keep       B requests, width entries of a request, L layers, Hkv heads of D channels, group, ps
  attention  what = "tree": B requests of up to max_kv cached tokens, up to max_q of them drafted, of which the last `prompts` requests
             have up to max_prompt new tokens instead; what = "window": up to max_q new ones.  Hq, Hkv, D, group, prefix (fp16 tokens
             in front), ps, window (0: none), sinks, words, fresh (prompts without history: all cached tokens are new)

Masks, positions, slots and codes are whole numbers and have to be equal.
"""

from __future__ import annotations

import math
import random

import torch

own = False


def listed():
    return [
        # one chat with a small tree: all latency
        {"name": "tree_chat", "kind": "tree", "B": 1, "nodes": 26, "prompts": 0, "max_prompt": 0, "words": 1, "max_kv": 1900},
        # a server's step: drafted trees of many requests, some prompts beside them
        {"name": "tree_server", "kind": "tree", "B": 250, "nodes": 64, "prompts": 6, "max_prompt": 2000, "words": 2, "max_kv": 6000},
        # the walk through one chat's tree after the model has chosen
        {"name": "accept_chat", "kind": "accept", "B": 1, "nodes": 26, "prompts": 0, "max_prompt": 0, "words": 1, "max_kv": 1900, "ps": 64,
         "depth": 8},
        # the same for a server's step, small pages: some come back from nearly every request
        {"name": "accept_server", "kind": "accept", "B": 250, "nodes": 64, "prompts": 6, "max_prompt": 2000, "words": 2, "max_kv": 6000,
         "ps": 16, "depth": 12},
        # accepted tokens of one chat in the 32 layers of an 8B model
        {"name": "keep_chat_8b", "kind": "keep", "B": 1, "width": 8, "L": 32, "Hkv": 8, "D": 128, "group": 0, "ps": 64},
        # accepted tokens of a decode batch in 80 layers with one step per token and head
        {"name": "keep_batch_70b", "kind": "keep", "B": 48, "width": 12, "L": 80, "Hkv": 8, "D": 128, "group": 128, "ps": 16},
        # one chat's tree over its history
        {"name": "tree_one_8b", "kind": "attention", "what": "tree", "B": 1, "max_q": 26, "max_kv": 3001, "Hq": 32, "Hkv": 8, "D": 128,
         "group": 0, "prefix": 3, "ps": 64, "fresh": False, "window": 0, "sinks": 0, "words": 1, "prompts": 0, "max_prompt": 0},
        # a decode batch with large trees: 256 rows of every key/value head
        {"name": "tree_batch_8b", "kind": "attention", "what": "tree", "B": 32, "max_q": 64, "max_kv": 6001, "Hq": 32, "Hkv": 8, "D": 128,
         "group": 0, "prefix": 3, "ps": 64, "fresh": False, "window": 0, "sinks": 0, "words": 2, "prompts": 0, "max_prompt": 0},
        # small trees and a chunk of a prompt in one call, dynamic steps, a window
        {"name": "tree_beside_prompt", "kind": "attention", "what": "tree", "B": 9, "max_q": 20, "max_kv": 12000, "Hq": 64, "Hkv": 8,
         "D": 128, "group": 128, "prefix": 1, "ps": 32, "fresh": False, "window": 4096, "sinks": 5, "words": 1, "prompts": 1,
         "max_prompt": 300},
        # one token of one request in a long chat, of which it sees the last part
        {"name": "window_one_8b", "kind": "attention", "what": "window", "B": 1, "max_q": 1, "max_kv": 40001, "Hq": 32, "Hkv": 8, "D": 128,
         "group": 0, "prefix": 0, "ps": 64, "fresh": False, "window": 2048, "sinks": 4, "words": 0, "prompts": 0, "max_prompt": 0},
        # a ragged decode batch with a window
        {"name": "window_batch_8b", "kind": "attention", "what": "window", "B": 48, "max_q": 1, "max_kv": 20000, "Hq": 32, "Hkv": 8,
         "D": 128, "group": 0, "prefix": 3, "ps": 64, "fresh": False, "window": 4096, "sinks": 4, "words": 0, "prompts": 0, "max_prompt": 0},
        # prompts longer than the window: the matrix products bound it
        {"name": "window_prefill_8b", "kind": "attention", "what": "window", "B": 2, "max_q": 6000, "max_kv": 6000, "Hq": 32, "Hkv": 8,
         "D": 128, "group": 0, "prefix": 3, "ps": 64, "fresh": True, "window": 1024, "sinks": 4, "words": 0, "prompts": 0, "max_prompt": 0},
    ]


def _log_between(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """A case of one of the five operators, sizes over their whole ranges."""
    kind = rng.choice(["tree", "accept", "keep", "attention", "attention", "attention", "attention"])
    ps = rng.choice([16, 32, 64, 128])
    if kind in ("tree", "accept"):
        words = rng.choice([1, 1, 2, 2, 3, 4, 8])
        c = {"kind": kind, "B": _log_between(rng, 1, 300), "nodes": _log_between(rng, 1, 32 * words), "prompts": rng.choice([0, 0, 1, 5]),
             "max_prompt": 32 * words + _log_between(rng, 1, 3000), "words": words, "max_kv": _log_between(rng, 1, 8000)}
        return dict(c, ps=ps, depth=rng.randint(1, min(16, 32 * words))) if kind == "accept" else c
    D = rng.choice([64, 128, 128])
    Hkv = rng.choice([1, 2, 4, 8, 8, 16, 32])
    group = rng.choice([0, 0, 0] + [g for g in (32, 64, 128) if g <= D])
    if kind == "keep":
        while True:
            B, width, L = _log_between(rng, 1, 128), rng.randint(1, 16), _log_between(rng, 1, 80)
            if B * width * L * Hkv * D <= 48 * 12 * 80 * 8 * 128:
                return {"kind": kind, "B": B, "width": width, "L": L, "Hkv": Hkv, "D": D, "group": group, "ps": ps}
    Hq = Hkv * rng.choice([g for g in (1, 2, 4, 5, 8) if Hkv * g <= 64])
    c = {"kind": kind, "Hq": Hq, "Hkv": Hkv, "D": D, "group": group, "prefix": rng.choice([0, 1, 3, 4, 17]), "ps": ps, "prompts": 0,
         "max_prompt": 0, "words": 0}
    while True:
        what = rng.choice(["tree", "window"])
        how = rng.choice(["decode", "verify", "chunk", "prompt"]) if what == "window" else "tree"
        B = _log_between(rng, 1, 64 if how in ("decode", "verify", "tree") else 6)
        max_kv = _log_between(rng, 1, 60000)
        max_q = {"decode": 1, "verify": rng.randint(2, 8), "chunk": _log_between(rng, 9, 2048), "prompt": max_kv,
                 "tree": _log_between(rng, 1, 128)}[how]
        window = _log_between(rng, 1, 16000)
        more = {"window": window, "sinks": rng.choice([0, 1, 4, 5, 33, 100])}
        if what == "tree":
            more["words"] = -(-max_q // 32) + rng.choice([0, 0, 1])
            if rng.random() < 0.5:
                more.update(window=0, sinks=0)
            if B > 1 and rng.random() < 0.3:
                more.update(prompts=1, max_prompt=32 * more["words"] + rng.randint(1, 200))
        longest = max(max_q, more.get("max_prompt", 0))
        # no more than the largest listed cases hold in their plain form
        if max_q <= max_kv and longest <= 4096 and B * Hkv * max_kv * D <= 900e6 and B * Hq * longest * max_kv <= 1.2e9:
            return {**c, **more, "what": what, "B": B, "max_q": max_q, "max_kv": max_kv, "fresh": how == "prompt"}


# ---------------------------------------------------------------------------------------------- inputs
def _step_lengths(case):
    """(cached tokens without the new ones, new tokens) of every request of a step: a function of the case alone."""
    r = random.Random("%(B)d %(nodes)d %(prompts)d %(max_prompt)d %(max_kv)d" % case)
    q = [case["nodes"]] + [r.randint(max(1, case["nodes"] // 2), case["nodes"]) for _ in range(case["B"] - 1)]
    q += [r.randint(32 * case["words"] + 1, case["max_prompt"]) for _ in range(case["prompts"])]
    kv = [r.randint(0, case["max_kv"]) for _ in q]
    order = list(range(len(q)))
    r.shuffle(order)
    return [kv[i] for i in order], [q[i] for i in order]


def _lengths(case):
    """(cached tokens with the new ones, new tokens) of every request of an attention case."""
    r = random.Random("%(B)d %(max_q)d %(max_kv)d" % case)
    kv = [case["max_kv"]] + [r.randint(max(1, case["max_kv"] // 4), case["max_kv"]) for _ in range(case["B"] - 1)]
    if case["fresh"]:
        return kv, list(kv)
    q = [case["max_q"]] + [r.randint(max(1, case["max_q"] // 2), case["max_q"]) for _ in range(case["B"] - 1)]
    q = [min(a, b) for a, b in zip(q, kv)]
    for i in range(case["prompts"]):
        q[-1 - i] = r.randint(32 * case["words"] + 1, case["max_prompt"])
        kv[-1 - i] = max(kv[-1 - i], q[-1 - i])
    return kv, q


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
    """A block table [B, W] (-1 where a request has no page) over shuffled pages, how many pages there are, and their order."""
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


def _cu(q):
    q = _int32(q)
    return torch.cat([_int32([0]), q.cumsum(0).to(torch.int32)])


def _parents(gen, cu, T):
    """Parents int32 [T] within each request: recent tokens more often, so that branches grow; node 0 is the root."""
    t = torch.arange(T, device="cuda")
    b = torch.searchsorted(cu[1:].long().contiguous(), t, right=True)
    i = t - cu[b].long()
    u = torch.rand((T,), generator=gen, device="cuda").sqrt()
    return torch.where(i > 0, (i * u).long().clamp(max=i - 1), -1).to(torch.int32), b, i


def _step_inputs(case, seed):
    gen = _generator(seed)
    before, q = _step_lengths(case)
    T = -(-sum(q) // 64) * 64                                      # a step's buffers are padded
    total = sum(q)
    d = {"cu_q": _cu(q), "kv_len": _int32([a + b for a, b in zip(before, q)]), "T": T}
    parents, b, i = _parents(gen, d["cu_q"], total)
    d["parents"] = torch.cat([parents, torch.full((T - total,), -1, dtype=torch.int32, device="cuda")])
    if case["kind"] == "tree":
        return d
    ps = case["ps"]
    kv = [a + c for a, c in zip(before, q)]
    W = -(-max(kv) // ps) + 3
    d["table"], pages, order = _table(gen, kv, ps, W, 9)
    d["free"], d["taken"] = order.clone(), _int32([pages - 9])      # (taken: pages of the list that requests have)
    d["tokens"] = torch.randint(0, 300, (T,), generator=gen, device="cuda", dtype=torch.int32)
    chosen = torch.randint(0, 300, (T,), generator=gen, device="cuda", dtype=torch.int32)
    # three times in four what the model chooses is one of the drafted children (the last one)
    child = torch.full((T,), -1, dtype=torch.int64, device="cuda")
    at = torch.arange(total, device="cuda")
    has = parents >= 0
    child.scatter_reduce_(0, (d["cu_q"][b].long() + parents)[has], at[has], "amax")
    follows = (child >= 0) & (torch.rand((T,), generator=gen, device="cuda") < 0.75)
    d["chosen"] = torch.where(follows, d["tokens"][child.clamp(min=0)], chosen)
    return d


def _keep_inputs(case, seed):
    gen = _generator(seed)
    B, width, L, H, D, group, ps = (case[k] for k in ("B", "width", "L", "Hkv", "D", "group", "ps"))
    each = -(-4 * width // ps) + 1                                 # pages of a request's drafted tokens
    pages = B * each + 2
    order = torch.randperm(pages, generator=gen, device="cuda")[:B * each].view(B, each)
    first = torch.randint(0, ps, (B, 1), generator=gen, device="cuda")
    # accepted nodes: ascending, from the root on, some of them in a row; a request accepts 1 to width
    path = torch.randint(1, 4, (B, width), generator=gen, device="cuda").cumsum(1) - 1
    path = path - path[:, :1]
    k = torch.arange(width, device="cuda")[None]
    live = k < torch.randint(1, width + 1, (B, 1), generator=gen, device="cuda")

    def slot(i):
        at = first + i
        return order.gather(1, (at // ps).clamp(max=each - 1)) * ps + at % ps

    moved = live & (path != k)
    d = {"from": torch.where(moved, slot(path), -1).contiguous(), "to": torch.where(moved, slot(k.expand(B, -1)), -1).contiguous()}
    shape = (L, pages, H, ps)
    for name in ("k", "v"):
        d[name + "_codes"] = torch.randint(0, 256, shape + (D // 2,), generator=gen, device="cuda", dtype=torch.uint8)
        d[name + "_scale"] = torch.rand(shape + (D // group,) if group else (L, H), generator=gen, device="cuda") + 0.1
    return d


def _attention_inputs(case, seed):
    gen = _generator(seed)
    kv, q = _lengths(case)
    D, ps, tree = case["D"], case["ps"], case["what"] == "tree"
    table, pages, _ = _table(gen, kv, ps, -(-max(kv) // ps), 5)
    d = {"kv_len": _int32(kv), "q_len": _int32(q), "cu_q": _cu(q), "T": sum(q), "L": table.shape[1] * ps}
    if case["window"]:
        # a server takes pages back that no row sees any more
        col = torch.arange(table.shape[1], device="cuda")[None]
        gone = (d["kv_len"] - d["q_len"])[:, None] + (0 if tree else 1) - case["window"]
        table = torch.where((col * ps >= case["sinks"]) & ((col + 1) * ps <= gone), -1, table).to(torch.int32).contiguous()
    d["table"] = table
    d["k_codes"], d["k_scale"] = _cache(gen, pages, case)
    d["v_codes"], d["v_scale"] = _cache(gen, pages, case)
    d["q"] = (1.5 * torch.randn((d["T"], case["Hq"] * D), generator=gen, device="cuda")).half()
    for name, size in (("pk", 2.0), ("pv", 0.1)):                 # prefix tokens draw attention and hold small values
        d[name] = (size * torch.randn((case["prefix"], case["Hkv"], D), generator=gen, device="cuda")).half() if case["prefix"] else None
    if tree:
        parents, _, _ = _parents(gen, d["cu_q"], d["T"])
        d["mask"] = _plain_tree({"case": case, "parents": parents, "cu_q": d["cu_q"], "kv_len": d["kv_len"], "T": d["T"]})["mask"]
    return d


def prepare(case, seed):
    s = {"case": dict(case)}
    if case["kind"] == "tree":
        s.update(_step_inputs(case, seed))
        s["outs"] = {"mask": torch.empty((s["T"], case["words"]), dtype=torch.int32, device="cuda"),
                     "positions": torch.empty(s["T"], dtype=torch.int32, device="cuda")}
    elif case["kind"] == "accept":
        s.update(_step_inputs(case, seed))
        B, depth = s["kv_len"].numel(), case["depth"]
        s["outs"] = {n: torch.empty(shape, dtype=kind, device="cuda") for n, shape, kind in (
            ("accepted", B, torch.int32), ("next_token", B, torch.int32), ("path", (B, depth), torch.int32), ("kv_len_out", B, torch.int32),
            ("from_slots", (B, depth), torch.int64), ("to_slots", (B, depth), torch.int64), ("taken_out", 1, torch.int32))}
    elif case["kind"] == "keep":
        s.update(_keep_inputs(case, seed))
        if own:
            import paper_2410_05265_amd.binding as pq
            s["layers"] = pq.KV4Layers([tuple(s[n][i] for n in ("k_codes", "v_codes", "k_scale", "v_scale")) for i in range(case["L"])], case["group"])
    else:
        s.update(_attention_inputs(case, seed))
        s["out"] = torch.empty_like(s["q"])
        # scratch memory as large as any of these calls asks for, kept like a server keeps it
        s["ws"] = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------------------------------ plain forms
def _nodes(s, N):
    """Of every request's first N new tokens: row (clamped), whether it is a node of a tree, node number."""
    cu = s["cu_q"].long()
    i = torch.arange(N, device="cuda")[None]
    m = (cu[1:] - cu[:-1])[:, None]
    return (cu[:-1, None] + i).clamp(max=s["T"] - 1), (i < m) & (m <= N), i


def _reach(edges):
    """[B, N, N]: which nodes (columns) a node meets on its way up, itself among them; edges[b, i, parent of i]."""
    N = edges.shape[-1]
    return torch.matrix_power(torch.eye(N, dtype=torch.float64, device="cuda") + edges.double(), N) > 0


def _plain_tree(s):
    words = s["case"]["words"]
    N, T = 32 * words, s["T"]
    row, node, i = _nodes(s, N)
    up = s["parents"][row].long()
    edges = (node & (up >= 0) & (up < i))[..., None] & (up[..., None] == i[:, None])
    meets = _reach(edges) & node[..., None]
    bits = (meets.view(-1, N, words, 32).long() << torch.arange(32, device="cuda")).sum(-1).to(torch.int32)
    cu = s["cu_q"].long()
    t = torch.arange(T, device="cuda")
    b = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    real = b < cu.numel() - 1
    b = b.clamp(max=cu.numel() - 2)
    at = t - cu[b]
    is_tree = real & (cu[b + 1] - cu[b] <= N)
    deep = torch.where(is_tree, meets.sum(-1)[b, at.clamp(0, N - 1)] - 1, at)
    before = s["kv_len"].long()[b] - (cu[b + 1] - cu[b])
    return {"mask": torch.where(is_tree[:, None], bits[b, at.clamp(0, N - 1)], 0).to(torch.int32),
            "positions": torch.where(real, before + deep, 0).to(torch.int32)}


def _plain_accept(s):
    c = s["case"]
    N, T, ps, depth = 32 * c["words"], s["T"], c["ps"], c["depth"]
    table = s["table"].long()
    W = table.shape[1]
    row, node, i = _nodes(s, N)
    cu, kv = s["cu_q"].long(), s["kv_len"].long()
    m = cu[1:] - cu[:-1]
    before = kv - m
    up = s["parents"][row].long()
    asked = torch.gather(s["chosen"][row], 1, up.clamp(0, N - 1))
    fits = node & (up >= 0) & (up < i) & (s["tokens"][row] == asked)
    # of a parent's fitting children the lowest one
    same = (up[:, :, None] == up[:, None, :]) & fits[:, None, :] & (i[:, None] < i[..., None])
    edges = (fits & ~same.any(-1))[..., None] & (up[..., None] == i[:, None])
    meets = _reach(edges)
    taken = meets[..., 0] & node                                   # nodes whose way up ends at node 0
    deep = meets.sum(-1) - 1
    taken &= deep < depth
    count = taken.sum(-1)
    is_tree = m <= N
    path = torch.full((m.numel(), depth), -1, dtype=torch.int64, device="cuda")
    path = path.scatter_reduce(1, deep.clamp(max=depth - 1), torch.where(taken, i, -1), "amax")
    last = torch.where(is_tree, (torch.where(taken, i, -1)).amax(-1), m - 1)
    accepted = torch.where(is_tree, count, m)
    next_token = torch.where(m > 0, s["chosen"][(cu[:-1] + last.clamp(min=0)).clamp(max=T - 1)], -1)
    kv_out = before + accepted

    def slot(at):
        page = torch.gather(table, 1, (at // ps).clamp(0, W - 1))
        return torch.where((at // ps < W) & (page >= 0), page * ps + at % ps, -1)

    k = torch.arange(depth, device="cuda")[None]
    moved = (path >= 0) & (path != k)
    a, z = slot(before[:, None] + path.clamp(min=0)), slot(before[:, None] + k)
    moved &= (a >= 0) & (z >= 0)
    # pages behind what is kept go back, the first of them last
    col = torch.arange(W, device="cuda")[None]
    back = (col >= ((kv_out + ps - 1) // ps)[:, None]) & (col < ((kv + ps - 1) // ps)[:, None]) & (table >= 0)
    rank = back.flatten().cumsum(0).view_as(table) - 1
    top = s["taken"][0].long().clamp(max=s["free"].numel())
    at = torch.where(back & (rank < top), top - 1 - rank, s["free"].numel())
    free = torch.cat([s["free"], s["free"][:1]]).scatter(0, at.flatten(), table.to(torch.int32).flatten())[:-1]
    s["free"].copy_(free)
    return {"accepted": accepted.to(torch.int32), "next_token": next_token.to(torch.int32), "path": path.to(torch.int32),
            "kv_len_out": kv_out.to(torch.int32), "from_slots": torch.where(moved, a, -1), "to_slots": torch.where(moved, z, -1),
            "taken_out": (top - back.sum()).clamp(min=0).to(torch.int32).reshape(1), "free": s["free"]}


def _plain_keep(s):
    ps = s["case"]["ps"]
    live = (s["from"] >= 0).flatten()
    a, z = s["from"].flatten()[live], s["to"].flatten()[live]

    def move(x):
        x[:, z // ps, :, z % ps] = x[:, a // ps, :, a % ps]

    move(s["k_codes"])
    move(s["v_codes"])
    if s["case"]["group"]:
        move(s["k_scale"])
        move(s["v_scale"])
    return _keep_outputs(s)


def _keep_outputs(s):
    return {n: s[n] for n in (("k_codes", "v_codes", "k_scale", "v_scale") if s["case"]["group"] else ("k_codes", "v_codes"))}


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


def _plain_seen(s, mq):
    """[B, mq, L]: which cached tokens a request's rows see."""
    c = s["case"]
    cu, m, n = s["cu_q"].long(), s["q_len"].long(), s["kv_len"].long()
    t = torch.arange(s["L"], device="cuda")
    i = torch.arange(mq, device="cuda")
    before = (n - m)[:, None, None]
    rel = t - before                                               # [B, 1, L]: place among the new tokens
    ahead = (i + 1)[None, :, None].expand(m.numel(), -1, -1)       # new tokens that a row sees
    drafted = (rel >= 0) & (rel < ahead)
    if c["what"] == "tree":
        N = 32 * c["words"]
        rows = (cu[:-1, None] + i).clamp(max=s["T"] - 1)
        bits = ((s["mask"][rows].long()[..., None] >> torch.arange(32, device="cuda")) & 1).bool().flatten(-2)     # [B, mq, N]
        is_tree = (m <= N)[:, None, None]
        node = torch.gather(bits, 2, rel.clamp(0, N - 1).expand(-1, mq, -1)) & (rel >= 0) & (rel < m[:, None, None])
        drafted = torch.where(is_tree, node, drafted)
        ahead = torch.where(is_tree, bits.sum(-1, keepdim=True), ahead)
    history = rel < 0
    if c["window"]:
        near = (t < c["sinks"]) | (rel >= ahead - c["window"])
        history = history & near
        if c["what"] == "tree":
            drafted = drafted & (is_tree | near)
        else:
            drafted = drafted & near
    return history | drafted


def _plain_attention(s):
    c = s["case"]
    B, Hq, Hkv, D, T = c["B"], c["Hq"], c["Hkv"], c["D"], s["T"]
    mq, g = max(_lengths(c)[1]), c["Hq"] // c["Hkv"]
    cu = s["cu_q"].long()
    keys, values = (_dense(s[n + "_codes"], s[n + "_scale"], s["table"], c) for n in ("k", "v"))
    L = s["L"]
    rows = (cu[:-1, None] + torch.arange(mq, device="cuda")).clamp(max=T - 1)
    q = s["q"][rows].float().view(B, mq, Hkv, g, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, mq * g, D)
    scores = q @ keys.transpose(2, 3).contiguous()
    scores = scores.view(B, Hkv, mq, g, L).masked_fill_(~_plain_seen(s, mq)[:, None, :, None], -math.inf).view(B, Hkv, mq * g, L)
    if c["prefix"]:
        front = q @ s["pk"].float().permute(1, 2, 0).contiguous()
        scores = torch.cat([front, scores], -1)
        values = torch.cat([s["pv"].float().transpose(0, 1)[None].expand(B, -1, -1, -1), values], 2)
    top = scores.amax(-1, keepdim=True).clamp_(min=-1e30)
    p = scores.sub_(top).mul_(1.0 / math.sqrt(D)).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p @ values) / torch.where(total > 0, total, 1.0)
    o = o.view(B, Hkv, mq, g, D).permute(0, 2, 1, 3, 4).reshape(B, mq, Hq * D)
    t = torch.arange(T, device="cuda")
    b = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    return o[b, t - cu[b]].half()


def run(s):
    c = s["case"]
    kind = c["kind"]
    if not own:
        return {"tree": _plain_tree, "accept": _plain_accept, "keep": _plain_keep, "attention": _plain_attention}[kind](s)
    import paper_2410_05265_amd.binding as pq
    if kind == "tree":
        pq.pq_kv4_tree(s["parents"], s["cu_q"], s["kv_len"], c["words"], **s["outs"])
        return s["outs"]
    if kind == "accept":
        pq.pq_kv4_accept(s["tokens"], s["parents"], s["chosen"], s["cu_q"], s["kv_len"], s["table"], c["ps"], c["words"], c["depth"],
                         free_pages=s["free"], taken=s["taken"], **s["outs"])
        return {**s["outs"], "free": s["free"]}
    if kind == "keep":
        pq.pq_kv4_keep(s["from"], s["to"], s["layers"])
        return _keep_outputs(s)
    a = (s["q"], s["cu_q"], s["kv_len"], s["table"], s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"], 1.0 / math.sqrt(c["D"]))
    longest = max(c["max_q"], c["max_prompt"])
    if c["what"] == "tree":
        return pq.pq_kv4_tree_attention(*a, longest, s["mask"], window=c["window"], sinks=c["sinks"], group=c["group"], prefix_k=s["pk"],
                                        prefix_v=s["pv"], out=s["out"], workspace=s["ws"])[0]
    return pq.pq_kv4_window_attention(*a, longest, c["window"], sinks=c["sinks"], group=c["group"], prefix_k=s["pk"], prefix_v=s["pv"],
                                      out=s["out"], workspace=s["ws"])[0]


# ---------------------------------------------------------------------------------------- what is needed
def work(case):
    if case["kind"] in ("tree", "accept"):
        q = _step_lengths(case)[1]
        B, T = len(q), -(-sum(q) // 64) * 64
        if case["kind"] == "tree":
            return {"bytes": float(sum(q) * 4 + T * 4 * (case["words"] + 1) + 8 * B), "flops": 0.0}
        drafted = sum(m for m in q if m <= 32 * case["words"])
        return {"bytes": float(drafted * 12 + B * (20 + 20 * case["depth"])), "flops": 0.0}
    Hkv, D, group = case["Hkv"], case["D"], case["group"]
    stored = Hkv * (D + (8 * D // group if group else 0))          # bytes of a token's keys and values
    if case["kind"] == "keep":
        # a request accepts half of its entries on average, and all but the first few of those move
        return {"bytes": float(case["B"] * (16 * case["width"] + case["L"] * case["width"] * stored)), "flops": 0.0}
    Hq = case["Hq"]
    tokens = pairs = 0
    for n, m in zip(*_lengths(case)):
        before, window, sinks = n - m, case["window"] or n, min(case["sinks"], n)
        tree = case["what"] == "tree" and m <= 32 * case["words"]
        gone = max(0, before + 1 - window - sinks)                 # tokens that no row sees
        tokens += n - gone
        if tree:                                                   # (a node sees itself and its root at least)
            pairs += m * min(before, window + sinks) + 2 * m - 1
        else:
            pairs += sum(min(before + i + 1, window + sinks) for i in range(m))
        pairs += m * case["prefix"]
    q = sum(_lengths(case)[1])
    return {"bytes": float(4 * q * Hq * D + tokens * stored + 4 * case["prefix"] * Hkv * D), "flops": 4.0 * D * Hq * pairs}


# -------------------------------------------------------------------------------------- the 64-bit result
def _exact_tree(case, seed):
    """The definition, node by node, on the host."""
    d = _step_inputs(case, seed)
    before, q = _step_lengths(case)
    words, parents = case["words"], d["parents"].cpu().tolist()
    mask, positions, start = [], [], 0
    for n, m in zip(before, q):
        if m > 32 * words:
            mask += [0] * m
            positions += range(n, n + m)
        else:
            seen = []
            for i in range(m):
                p = parents[start + i]
                seen.append((1 << i) | (seen[p] if 0 <= p < i else 0))
            mask += seen
            positions += [n + bin(x).count("1") - 1 for x in seen]
        start += m
    pad = d["T"] - start
    parts = [[(x >> (32 * w)) & 0xFFFFFFFF for w in range(words)] for x in mask + [0] * pad]
    parts = [[x - (1 << 32) if x >> 31 else x for x in r] for r in parts]
    return {"mask": _int32(parts), "positions": _int32(positions + [0] * pad)}


def _exact_accept(case, seed):
    d = _step_inputs(case, seed)
    before, q = _step_lengths(case)
    N, ps, depth = 32 * case["words"], case["ps"], case["depth"]
    parents, tokens, chosen, table, free = (d[n].cpu().tolist() for n in ("parents", "tokens", "chosen", "table", "free"))
    top = min(int(d["taken"][0]), len(free))
    back, start = 0, 0
    outs = {n: [] for n in ("accepted", "next_token", "path", "kv_len_out", "from_slots", "to_slots")}
    for b, (n, m) in enumerate(zip(before, q)):
        path = [0] if m <= N else []
        while path and len(path) < depth:
            children = [i for i in range(path[-1] + 1, m) if parents[start + i] == path[-1] and tokens[start + i] == chosen[start + path[-1]]]
            if not children:
                break
            path.append(children[0])
        kept = len(path) if m <= N else m
        outs["accepted"].append(kept)
        outs["next_token"].append(chosen[start + (path[-1] if path else m - 1)])
        outs["path"].append(path + [-1] * (depth - len(path)))
        outs["kv_len_out"].append(n + kept)
        for name, side in (("from_slots", path), ("to_slots", range(len(path)))):
            row = [table[b][(n + x) // ps] * ps + (n + x) % ps if path[k] != k else -1 for k, x in enumerate(side)]
            outs[name].append(row + [-1] * (depth - len(row)))
        for col in range(-(-(n + kept) // ps), -(-(n + m) // ps)):
            if back < top:
                free[top - 1 - back] = table[b][col]
            back += 1
        start += m
    got = {n: torch.tensor(v, dtype=torch.int64 if n.endswith("slots") else torch.int32, device="cuda") for n, v in outs.items()}
    return {**got, "taken_out": _int32([max(0, top - back)]), "free": _int32(free)}


def _exact_keep(case, seed):
    d = _keep_inputs(case, seed)
    ps = case["ps"]
    for a, z in zip(d["from"].flatten().cpu().tolist(), d["to"].flatten().cpu().tolist()):
        if a >= 0:                                                 # (in a request's order, one after another)
            for name in ("k_codes", "v_codes") + (("k_scale", "v_scale") if case["group"] else ()):
                d[name][:, z // ps, :, z % ps] = d[name][:, a // ps, :, a % ps]
    return {n: d[n].double() if "scale" in n else d[n] for n in (("k_codes", "v_codes", "k_scale", "v_scale") if case["group"] else ("k_codes", "v_codes"))}


def _exact_attention(case, seed):
    d = _attention_inputs(case, seed)
    Hq, Hkv, D, P, ps, group = (case[k] for k in ("Hq", "Hkv", "D", "prefix", "ps", "group"))
    kv, q = _lengths(case)
    per, words = Hq // Hkv, case["words"]
    out = torch.zeros((d["T"], Hq, D), dtype=torch.float64, device="cuda")
    start = 0
    for b, (n, m) in enumerate(zip(kv, q)):
        window = case["window"] or 1 << 40
        t, i = torch.arange(n, device="cuda")[None], torch.arange(m, device="cuda")[:, None]
        where = n - m + i                                          # a row's position
        seen = t <= where
        if case["what"] == "tree" and m <= 32 * words:
            bits = (d["mask"][start:start + m].long() & 0xFFFFFFFF)[:, :, None] // (1 << torch.arange(32, device="cuda")) % 2
            bits = bits.reshape(m, 32 * words)[:, :m]
            where = n - m - 1 + bits.sum(1, keepdim=True)
            seen = torch.cat([((t < case["sinks"]) | (t > where - window))[:, :n - m].expand(m, -1), bits > 0], 1)
        else:
            seen = seen & ((t < case["sinks"]) | (t > where - window))
        pages = d["table"][b, :-(-n // ps)].long().clamp(min=0)
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
                w[:, P:].masked_fill_(~seen[r:e].repeat_interleave(per, 0), -math.inf)
                out[start + r:start + e, h * per:(h + 1) * per] = (torch.softmax(w, -1).nan_to_num(0.0) @ side[1]).view(e - r, per, D)
        start += m
    return out.reshape(d["T"], Hq * D)


def exact(case, seed):
    return {"tree": _exact_tree, "accept": _exact_accept, "keep": _exact_keep, "attention": _exact_attention}[case["kind"]](case, seed)

"""The operators of the attention half of a block-pruned decoder layer, as a serving program calls them between the projections:
norms of query and key heads with the position rotation and the append to a paged cache, attention over that cache with a
sliding window and first tokens that stay visible, and attention of a batch whose sequences share a long prefix.

Sizes are generic: heads of 64 to 128 values, groups of 1 to 16 query heads on a key head, pages of 16 to 128 tokens. The tokens
of a call lie one behind the other, sequence after sequence (`starts`); a sequence's new tokens are the last of its `lengths`
tokens. `listed()` has one token, batches of running answers, prompts of uneven length and long prompts."""
import math

import torch

own = False   # True: run() calls the library's operators; False: their plain form in 32 bits

BF16, F16 = "bf16", "f16"
TYPES = {BF16: torch.bfloat16, F16: torch.float16}
EPS = 1e-6
BASE = 10000.0


# ------------------------------------------------------------------ cases
def listed():
    def append(name, B, new, cached, Hq, Hkv, D, dt, page, rot, norm=True, interleaved=False, pad=0):
        return {"name": name, "op": "append", "B": B, "new_lo": new[0], "new_hi": new[1], "old_lo": cached[0], "old_hi": cached[1], "Hq": Hq,
                "Hkv": Hkv, "D": D, "dtype": dt, "page": page, "rot": rot, "norm": norm, "interleaved": interleaved, "pad": pad}

    def attend(name, B, new, cached, Hq, Hkv, D, dt, page, window=0, sinks=0, prefix=0):
        return {"name": name, "op": "prefix" if prefix else "attention", "B": B, "new_lo": new[0], "new_hi": new[1], "old_lo": cached[0],
                "old_hi": cached[1], "Hq": Hq, "Hkv": Hkv, "D": D, "dtype": dt, "page": page, "window": window, "sinks": sinks, "prefix": prefix}

    return [
        # one token of a running answer: latency only
        append("append_token", 1, (1, 1), (4000, 4000), 32, 8, 128, BF16, 64, 128),
        # prompts of uneven length on a small model: a part of each head is rotated, in neighbouring pairs, no norm; rows cut out of
        # a wider buffer (nothing 16-byte aligned)
        append("append_ragged", 13, (1, 235), (0, 900), 12, 4, 80, F16, 16, 32, norm=False, interleaved=True, pad=3),
        # a long prompt: bandwidth
        append("append_prompt", 1, (16384, 16384), (0, 0), 32, 8, 128, BF16, 64, 128),
        # one token of a running answer, sliding window with first tokens kept: latency
        attend("attention_token", 1, (1, 1), (6000, 6000), 32, 8, 128, BF16, 64, window=1024, sinks=4),
        # 64 running answers of uneven length: bandwidth of the cache
        attend("attention_batch", 64, (1, 1), (500, 8191), 32, 8, 128, BF16, 64),
        # three very long documents, one token each, eight query heads on a key head
        attend("attention_long", 3, (1, 1), (90001, 110001), 16, 2, 64, F16, 128),
        # prompts of uneven length on a small model with a short window, heads of 80 values
        attend("attention_ragged", 7, (1, 901), (0, 0), 12, 4, 80, F16, 16, window=300, sinks=5),
        # four long conversations get their next questions
        attend("attention_continue", 4, (100, 512), (9000, 15500), 32, 8, 128, BF16, 64),
        # a long prompt under a sliding window
        attend("attention_window", 1, (16384, 16384), (0, 0), 32, 8, 128, BF16, 64, window=4096, sinks=16),
        # a long prompt, every token sees all before it: the rate of the matrix products
        attend("attention_prompt", 1, (8192, 8192), (0, 0), 32, 8, 128, BF16, 64),
        # 64 answers to one long instruction
        attend("prefix_batch", 64, (1, 1), (1, 400), 32, 8, 128, BF16, 64, prefix=8192),
        # six answers to a short instruction that does not fill its last page, one query head on a key head
        attend("prefix_small", 6, (1, 1), (3, 40), 8, 8, 64, F16, 16, prefix=1001),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["append", "attention", "attention", "attention", "prefix"])
        Hkv, G = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2, 3, 4, 5, 8, 16])
        c = {"op": op, "Hq": Hkv * G, "Hkv": Hkv, "D": rng.choice([64, 80, 96, 128, 128]), "dtype": rng.choice([BF16, F16]),
             "page": rng.choice([16, 32, 64, 128]), "B": _log(rng, 1, 64)}
        if op == "append":
            new = _log(rng, 1, 16384 // c["B"])
            old = _log(rng, 1, 8192) - 1
            c.update(new_lo=rng.randint(1, new), new_hi=new, old_lo=rng.randint(0, old), old_hi=old, norm=rng.random() < 0.6,
                     interleaved=rng.random() < 0.4, pad=rng.choice([0, 0, 8, 1, 5]), rot=rng.choice([c["D"], c["D"], 32, c["D"] // 2]))
        else:
            running = op == "prefix" or rng.random() < 0.5      # a token a sequence, or prompts and their continuations
            old = _log(rng, 1, 512 if op == "prefix" else 65536 if running else 16384) - 1
            new = 1 if running else _log(rng, 2, 8192)
            if not running and rng.random() < 0.5:
                old = 0
            c.update(new_lo=rng.randint(1, new), new_hi=new, old_lo=rng.randint(0, old), old_hi=old,
                     window=rng.choice([0, 0, _log(rng, 16, 4096)]) if op == "attention" else 0, prefix=_log(rng, 100, 16384) if op == "prefix" else 0)
            c["sinks"] = rng.choice([0, 1, 4, 16, 130]) if c["window"] else 0
        if _fits(c):
            return c


def _fits(c):
    """No more work than the largest listed cases, and a plain form that fits the card."""
    new, length = _counts(c)
    if c["op"] == "append":
        return sum(new) * (c["Hq"] + 2 * c["Hkv"]) * c["D"] <= 16384 * 48 * 128
    scores = c["B"] * c["Hq"] * max(new) * max(length)
    return scores <= 1 << 32 and c["B"] * max(length) * c["Hkv"] * c["D"] <= 1 << 29 and sum(n * x for n, x in zip(new, length)) * c["Hq"] * c["D"] <= 1 << 37


def _counts(case):
    """New tokens and tokens in all of each sequence: spread evenly over the case's ranges, in mixed order."""
    B = case["B"]

    def spread(lo, hi, step):
        return [lo + (hi - lo) * ((step * b) % B) // max(1, B - 1) for b in range(B)] if B > 1 else [hi]

    step = next(s for s in (37, 29, 23, 1) if math.gcd(s, B) == 1)
    new = spread(case["new_lo"], case["new_hi"], step)
    old = spread(case["old_lo"], case["old_hi"], 1)
    return new, [n + o + case.get("prefix", 0) for n, o in zip(new, old)]


# ------------------------------------------------------------------ inputs
def _rand(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    B, Hq, Hkv, D, P, dt = case["B"], case["Hq"], case["Hkv"], case["D"], case["page"], TYPES[case["dtype"]]
    new, length = _counts(case)
    T, prefix = sum(new), case.get("prefix", 0)
    width = (max(length) + P - 1) // P
    # a server's pages: every sequence's lie scattered over the cache; those that a shared prefix fills are the same for all
    common = prefix // P
    need = [(n + P - 1) // P - common for n in length]
    pages = common + sum(need) + 3
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    at = torch.tensor([0] + need, device="cuda").cumsum(0)[:-1]
    place = torch.arange(width - common, device="cuda")
    rows = common + at[:, None] + place
    rows = torch.where(place < torch.tensor(need, device="cuda")[:, None], rows, torch.zeros_like(rows))
    table = torch.cat([order[:common].expand(B, common), order[rows]], 1).contiguous()
    # keys and values of earlier tokens, some channels off centre
    k = (_rand(g, pages, Hkv, P, D) + 0.5 * _rand(g, Hkv, 1, D)).to(dt)
    v = (_rand(g, pages, Hkv, P, D) + 0.5 * _rand(g, Hkv, 1, D)).to(dt)
    if prefix % P:     # the page that a prefix ends in holds copies of its last tokens in every sequence's own page
        last = table[:, common].long()
        k[last, :, :prefix % P] = k[last[:1], :, :prefix % P]
        v[last, :, :prefix % P] = v[last[:1], :, :prefix % P]
    d = {"k_cache": k, "v_cache": v, "table": table, "lengths": torch.tensor(length, dtype=torch.int32, device="cuda"),
         "starts": torch.tensor([0] + new, device="cuda").cumsum(0).to(torch.int32)}
    if case["op"] == "append":
        cols = (Hq + 2 * Hkv) * D
        buf = torch.zeros(T, cols + case["pad"], dtype=dt, device="cuda")
        buf[:, :cols] = (_rand(g, T, cols) * torch.exp(0.3 * _rand(g, T, 1))).to(dt)
        d["qkv"] = buf[:, :cols]
        angle = torch.arange(max(length), device="cuda", dtype=torch.float64)[:, None] * BASE ** (
            -torch.arange(0, case["rot"], 2, device="cuda", dtype=torch.float64) / case["rot"])
        d["rotation"] = torch.cat([angle.cos(), angle.sin()], 1).float()
        d["q_gamma"] = (1.0 + 0.2 * _rand(g, D)).to(dt) if case["norm"] else None
        d["k_gamma"] = (1.0 + 0.2 * _rand(g, D)).to(dt) if case["norm"] else None
    else:
        d["q"] = (1.5 * _rand(g, T, Hq, D)).to(dt)
    return {"case": case, "in": d, "most_new": max(new), "most": max(length), "ragged": max(new) > 1}


# ------------------------------------------------------------------ one pass
def _run_own(state):
    import paper_2407_19644_b200 as ubp
    c, d = state["case"], state["in"]
    starts = d["starts"] if state["ragged"] else None
    if c["op"] == "append":
        q = ubp.ubp_rotate_append(d["qkv"], c["Hq"], d["k_cache"], d["v_cache"], d["table"], d["lengths"], starts=starts, rotation=d["rotation"],
                                  interleaved=c["interleaved"], q_gamma=d["q_gamma"], k_gamma=d["k_gamma"], eps=EPS)
        return {"q": q, "k_cache": d["k_cache"], "v_cache": d["v_cache"]}
    if c["op"] == "prefix":
        return {"o": ubp.ubp_prefix_attention(d["q"], d["k_cache"], d["v_cache"], d["table"], d["lengths"], c["prefix"], starts=starts,
                                              max_new=state["most_new"])}
    return {"o": ubp.ubp_attention(d["q"], d["k_cache"], d["v_cache"], d["table"], d["lengths"], starts=starts, window=c["window"], sinks=c["sinks"],
                                   max_new=state["most_new"])}


def _tokens(d, T):
    """Sequence of each token, its place among the sequence's new tokens, and its position."""
    t = torch.arange(T, device="cuda")
    b = (t[:, None] >= d["starts"][None, 1:]).sum(1)
    i = t - d["starts"][b]
    return b, i, d["lengths"][b] - (d["starts"][b + 1] - d["starts"][b]) + i


def _plain_append(c, d):
    T, Hq, Hkv, D, r = d["qkv"].shape[0], c["Hq"], c["Hkv"], c["D"], c["rot"]
    b, _, at = _tokens(d, T)
    x = d["qkv"].float().view(T, Hq + 2 * Hkv, D)
    v, x = x[:, Hq + Hkv:], x[:, :Hq + Hkv]
    if c["norm"]:
        gamma = torch.cat([d["q_gamma"].float().expand(Hq, D), d["k_gamma"].float().expand(Hkv, D)])
        x = x * torch.rsqrt((x * x).mean(2, keepdim=True) + EPS) * gamma
    cos, sin = d["rotation"][at][:, None, :r // 2], d["rotation"][at][:, None, r // 2:]
    if c["interleaved"]:
        e, o = x[:, :, 0:r:2], x[:, :, 1:r:2]
        y = torch.cat([torch.stack([e * cos - o * sin, o * cos + e * sin], 3).flatten(2), x[:, :, r:]], 2)
    else:
        e, o = x[:, :, :r // 2], x[:, :, r // 2:r]
        y = torch.cat([e * cos - o * sin, o * cos + e * sin, x[:, :, r:]], 2)
    dt = TYPES[c["dtype"]]
    page, slot = d["table"][b, at // c["page"]].long(), at % c["page"]
    d["k_cache"][page, :, slot] = y[:, Hq:].to(dt)
    d["v_cache"][page, :, slot] = v.to(dt)
    return {"q": y[:, :Hq].to(dt), "k_cache": d["k_cache"], "v_cache": d["v_cache"]}


def _plain_attention(c, d, Q, L):
    """All sequences at once, queries padded to Q and tokens to L."""
    q = d["q"]
    T, Hq, D = q.shape
    B, Hkv, P = c["B"], c["Hkv"], c["page"]
    b, i, at = _tokens(d, T)
    x = torch.zeros(B, Q, Hq, D, device="cuda")
    x[b, i] = q.float() / math.sqrt(D)
    x = x.view(B, Q, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, Hq // Hkv * Q, D)
    k = d["k_cache"][d["table"].long()].float().permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, D)[:, :, :L]
    v = d["v_cache"][d["table"].long()].float().permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, D)[:, :, :L]
    j = torch.arange(L, device="cuda", dtype=torch.int32)
    place = torch.full((B, Q), -1, device="cuda", dtype=torch.int32)
    place[b, i] = at.to(torch.int32)
    hidden = j > place[:, :, None]
    if c["window"]:
        hidden |= (j <= place[:, :, None] - c["window"]) & (j >= c["sinks"])
    hidden |= (place < 0)[:, :, None] & (j > 0)          # (padding: any one token)
    hidden &= ~((place < 0)[:, :, None] & (j == 0))
    s = (x @ k.transpose(2, 3)).view(B, Hkv, Hq // Hkv, Q, L)
    s.masked_fill_(hidden[:, None, None], -math.inf)
    s -= s.amax(4, keepdim=True)
    s.exp_()
    o = s.view(B, Hkv, Hq // Hkv * Q, L) @ v / s.view(B, Hkv, Hq // Hkv * Q, L).sum(3, keepdim=True)
    o = o.view(B, Hkv, Hq // Hkv, Q, D).permute(0, 3, 1, 2, 4).reshape(B, Q, Hq, D)
    return {"o": o[b, i].to(q.dtype)}


def run(state):
    if own:
        return _run_own(state)
    c, d = state["case"], state["in"]
    return _plain_append(c, d) if c["op"] == "append" else _plain_attention(c, d, state["most_new"], state["most"])


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    new, length = _counts(case)
    T, Hq, Hkv, D = sum(new), case["Hq"], case["Hkv"], case["D"]
    tables = 4 * (2 * case["B"] + 1 + sum((n + case["page"] - 1) // case["page"] for n in length))
    if case["op"] == "append":     # rows in; queries, keys and values out; the rotation of the positions that occur
        n = T * (Hq + 2 * Hkv) * D
        positions = len(set(p for a, n_ in zip(new, length) for p in range(n_ - a, n_)))
        rotated = T * (Hq + Hkv)
        return {"bytes": 4 * n + 4 * case["rot"] * positions + 8 * case["B"] + (4 * D if case["norm"] else 0),
                "flops": 3.0 * rotated * case["rot"] + (4.0 * rotated * D if case["norm"] else 0.0)}
    W, S, prefix = case["window"], case["sinks"], case["prefix"]
    pairs, read = 0, prefix
    for a, n in zip(new, length):
        p = torch.arange(n - a, n, dtype=torch.float64)
        seen = p + 1 if not W else torch.minimum(p + 1, float(W) + torch.clamp(torch.minimum(p + 1 - W, torch.full_like(p, float(S))), min=0))
        pairs += int(seen.sum())
        first = max(0, n - a - W + 1) if W else 0                        # tokens of the cache that some query sees
        read += n - first + min(first, S) - prefix
    return {"bytes": 4 * T * Hq * D + 4 * read * Hkv * D + tables, "flops": 4.0 * pairs * Hq * D}


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    state = prepare(case, seed)
    d, new, length = state["in"], *_counts(case)
    Hq, Hkv, D, P = case["Hq"], case["Hkv"], case["D"], case["page"]
    first = [sum(new[:b]) for b in range(case["B"])]
    if case["op"] == "append":
        k, v, r = d["k_cache"].double(), d["v_cache"].double(), case["rot"]
        q = torch.empty(sum(new), Hq, D, dtype=torch.float64, device="cuda")
        for b, (t, a, n) in enumerate(zip(first, new, length)):
            x = d["qkv"][t:t + a].double().unflatten(1, (Hq + 2 * Hkv, D))
            p = torch.arange(n - a, n, device="cuda")
            turn = torch.polar(torch.ones_like(d["rotation"][p, :r // 2].double()), torch.atan2(d["rotation"][p, r // 2:].double(), d["rotation"][p, :r // 2].double()))
            turn = turn * torch.hypot(d["rotation"][p, r // 2:].double(), d["rotation"][p, :r // 2].double())
            heads = []
            for h in range(Hq + Hkv):
                u = x[:, h]
                if case["norm"]:
                    u = u / torch.sqrt(torch.linalg.vector_norm(u, dim=1, keepdim=True).square() / D + EPS) * (d["q_gamma"] if h < Hq else d["k_gamma"]).double()
                z = u[:, :r].unflatten(1, (r // 2, 2)) if case["interleaved"] else u[:, :r].unflatten(1, (2, r // 2)).transpose(1, 2)
                z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
                z = z.flatten(1) if case["interleaved"] else z.transpose(1, 2).flatten(1)
                heads.append(torch.cat([z, u[:, r:]], 1))
            q[t:t + a] = torch.stack(heads[:Hq], 1)
            page, slot = d["table"][b].long()[p // P], p % P
            k[page, :, slot] = torch.stack(heads[Hq:], 1)
            v[page, :, slot] = x[:, Hq + Hkv:]
        return {"q": q, "k_cache": k, "v_cache": v}
    W, S, G = case["window"], case["sinks"], Hq // Hkv
    o = torch.empty(d["q"].shape, dtype=torch.float64, device="cuda")
    for b, (t, a, n) in enumerate(zip(first, new, length)):
        pages = d["table"][b, :(n + P - 1) // P].long()
        k, v = (x[pages].transpose(0, 1).flatten(1, 2)[:, :n].double() for x in (d["k_cache"], d["v_cache"]))
        j = torch.arange(n, device="cuda")
        step = max(1, (1 << 28) // (n * G))
        for i in range(0, a, step):
            p = torch.arange(n - a + i, min(n, n - a + i + step), device="cuda")[:, None]
            seen = j <= p
            if W:
                seen &= (j > p - W) | (j < S)
            for h in range(Hkv):
                x = d["q"][t + i:t + i + len(p), h * G:(h + 1) * G].double().transpose(0, 1)
                s = torch.where(seen, torch.einsum("gid,jd->gij", x, k[h]) / math.sqrt(D), -math.inf)
                o[t + i:t + i + len(p), h * G:(h + 1) * G] = torch.einsum("gij,jd->gid", torch.softmax(s, 2), v[h]).transpose(0, 1)
    return {"o": o}

"""Attention as a decoder trains and serves it, and what keeps its cache small: the work a program hands to this library.

Every case is a dict of plain values.  ``op`` names the operator:

  triangle  online-softmax reducer over a triangular relation (causal attention of packed sequences of different lengths),
            grouped heads, optional mask of keys; forward, or forward + gradients
  shared    the same reducer over a paged cache whose sequences begin, group by group, with the same pages: a few new
            tokens per sequence
  weights   how much attention every cached position has received: the softmax weights of a chunk of new tokens, summed over
            its rows and the heads of a group, on top of what was there before
  evict     a cache is cut to a budget: the last positions stay and those with the largest weights, in their order, in other pages

``run`` computes the operators in plain torch operations, or, where ``own`` is true, through the library.
Inputs are made on the GPU from the seed alone.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # one short sequence of two heads in a training loop (the smallest step): launches and latency count
        {"name": "triangle_step_small", "op": "triangle", "segments": 1, "q": 65, "kv": 65, "ragged": False, "heads": 2, "kv_heads": 2,
         "D": 64, "dtype": "f16", "masked": False, "backward": True},
        # prompts of different lengths packed into one batch, before serving begins: forward only
        {"name": "triangle_prompts", "op": "triangle", "segments": 12, "q": 4096, "kv": 4096, "ragged": True, "heads": 32, "kv_heads": 8,
         "D": 128, "dtype": "bf16", "masked": False, "backward": False},
        # a training batch of ragged documents, padding masked
        {"name": "triangle_step_ragged", "op": "triangle", "segments": 16, "q": 1500, "kv": 1500, "ragged": True, "heads": 16, "kv_heads": 16,
         "D": 64, "dtype": "f16", "masked": True, "backward": True},
        # the largest training step: long sequences, grouped heads
        {"name": "triangle_step_large", "op": "triangle", "segments": 4, "q": 4096, "kv": 4096, "ragged": False, "heads": 16, "kv_heads": 4,
         "D": 128, "dtype": "bf16", "masked": False, "backward": True},
        # a handful of users on one short system prompt: latency counts
        {"name": "shared_tokens_short", "op": "shared", "groups": 1, "members": 4, "shared": 320, "q": 1, "kv": 77, "heads": 8, "kv_heads": 2,
         "D": 64, "dtype": "bf16", "page": 16},
        # next tokens of a batch of users whose caches begin with one long document
        {"name": "shared_tokens_batch", "op": "shared", "groups": 1, "members": 64, "shared": 8192, "q": 1, "kv": 1024, "heads": 32, "kv_heads": 8,
         "D": 128, "dtype": "bf16", "page": 32},
        # several samples of each of a few prompts, a few speculative tokens each
        {"name": "shared_samples", "op": "shared", "groups": 6, "members": 8, "shared": 16384, "q": 5, "kv": 333, "heads": 32, "kv_heads": 8,
         "D": 128, "dtype": "f16", "page": 64},
        # one new token's weights on a short cache: latency counts
        {"name": "weights_token_short", "op": "weights", "segments": 1, "q": 1, "kv": 777, "ragged": False, "heads": 8, "kv_heads": 2,
         "D": 64, "dtype": "bf16", "page": 16, "added": True},
        # new tokens of a batch of users: the bandwidth of the keys counts
        {"name": "weights_tokens_batch", "op": "weights", "segments": 64, "q": 1, "kv": 8192, "ragged": True, "heads": 32, "kv_heads": 8,
         "D": 128, "dtype": "bf16", "page": 32, "added": True},
        # a chunk of a long prompt: the exponentials count
        {"name": "weights_chunk", "op": "weights", "segments": 1, "q": 2048, "kv": 16384, "ragged": False, "heads": 32, "kv_heads": 8,
         "D": 128, "dtype": "f16", "page": 64, "added": False},
        # one user's cache is cut, many layers of a model one after the other: latency counts
        {"name": "evict_short", "op": "evict", "segments": 1, "kv": 777, "ragged": False, "kv_heads": 2, "D": 64, "dtype": "bf16", "page": 16,
         "keep": 256, "recent": 64},
        # a batch of users is cut to a quarter
        {"name": "evict_batch", "op": "evict", "segments": 64, "kv": 8192, "ragged": True, "kv_heads": 8, "D": 128, "dtype": "bf16", "page": 32,
         "keep": 2048, "recent": 256},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["triangle", "triangle", "shared", "shared", "weights", "weights", "evict"])
    kv_heads = rng.choice([1, 2, 3, 4, 8])
    heads = kv_heads * rng.choice([1, 2, 3, 4, 5, 8])
    D = rng.choice([32, 64, 64, 72, 96, 128, 128])
    c = {"op": op, "heads": heads, "kv_heads": kv_heads, "D": D, "dtype": rng.choice(["f16", "bf16"])}
    page = rng.choice([8, 16, 32, 48, 64, 128])
    while True:
        if op == "triangle":
            c |= {"segments": _log(rng, 1, 64), "q": _log(rng, 1, 4096), "ragged": rng.random() < 0.7, "masked": rng.random() < 0.3,
                  "backward": rng.random() < 0.6}
            c["kv"] = c["q"] if rng.random() < 0.7 else _log(rng, c["q"], 4096)     # the rows of a step may be the last of longer sequences
            if c["segments"] * c["q"] * c["kv"] * heads * D * (10 if c["backward"] else 4) <= 4 * 4096 * 4096 * 16 * 128 * 10:
                return c
        elif op == "shared":
            c |= {"groups": _log(rng, 1, 8), "members": _log(rng, 1, 64), "shared": _log(rng, 1, 16384) // page * page,
                  "q": rng.choice([1, 1, _log(rng, 2, 64)]), "kv": _log(rng, 1, 2048), "page": page}
            c["kv"] = max(c["kv"], c["q"])
            n = c["groups"] * c["members"]
            if n * c["q"] * (c["shared"] + c["kv"]) * heads * D <= 48 * 16384 * 8 * 32 * 128 and n * (c["shared"] + c["kv"]) * kv_heads * D <= 1 << 30:
                return c
        elif op == "weights":
            c |= {"segments": _log(rng, 1, 128), "q": rng.choice([1, 1, _log(rng, 2, 2048)]), "kv": _log(rng, 1, 65536), "ragged": rng.random() < 0.7,
                  "page": page, "added": rng.random() < 0.6}
            c["kv"] = max(c["kv"], c["q"])
            if c["segments"] * c["q"] * c["kv"] * heads * D <= 2048 * 16384 * 32 * 128 and c["segments"] * c["kv"] * kv_heads * D <= 1 << 28:
                return c
        else:
            kv = _log(rng, 1, 65536)
            keep = _log(rng, 1, kv)
            c = {"op": op, "segments": _log(rng, 1, 128), "kv": kv, "ragged": rng.random() < 0.7, "kv_heads": kv_heads, "D": D, "dtype": c["dtype"],
                 "page": page, "keep": keep, "recent": rng.randint(0, keep)}
            if c["segments"] * kv * kv_heads * D <= 1 << 28:
                return c


# ------------------------------------------------------------------------------------------------ inputs

def _lengths(n, longest, ragged, least, gen):
    """n lengths up to `longest`, spread evenly over its upper three quarters where ragged, in an order of their own."""
    low = max(least, longest // 4) if ragged else longest
    return longest - (longest - low) * torch.randperm(n, generator=gen) // max(n - 1, 1)


def _starts(lengths):
    s = torch.zeros(lengths.numel() + 1, dtype=torch.int64)
    s[1:] = torch.cumsum(lengths, 0)
    return s


def _rows(lengths):
    """The segment of every row, and its place in the segment."""
    seg = torch.repeat_interleave(torch.arange(lengths.numel()), lengths)
    return seg.to(DEV), (torch.arange(seg.numel()) - _starts(lengths)[seg]).to(DEV)


def _normal(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32) * scale).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    dt, D, hk = DTYPES[case["dtype"]], case["D"], case["kv_heads"]
    s = {"case": case, "scale": D ** -0.5}
    if case["op"] == "triangle":
        B, h = case["segments"], case["heads"]
        kl = _lengths(B, case["kv"], case["ragged"], 1, host)
        ql = torch.clamp(kl - (case["kv"] - case["q"]), min=1)
        s["q_start"], s["kv_start"] = (_starts(a).to(DEV, torch.int32) for a in (ql, kl))
        s["q_row"], s["kv_row"] = _rows(ql), _rows(kl)
        nq, nk = int(ql.sum()), int(kl.sum())
        s["q"] = _normal(gen, (nq, h, D), dt)
        kv = _normal(gen, (nk, 2, hk, D), dt)              # one projection gives keys and values
        s["key"], s["value"] = kv[:, 0], kv[:, 1]
        s["mask"] = torch.rand(nk, generator=gen, device=DEV) < 0.8 if case["masked"] else None
        s["grad_out"] = _normal(gen, (nq, h, D), dt, 0.1) if case["backward"] else None
        return s
    page = case["page"]
    if case["op"] == "shared":
        B, head = case["groups"] * case["members"], case["shared"] // page
        tail = _lengths(B, case["kv"], True, case["q"], host)
        kl, ql = case["shared"] + tail, torch.minimum(_lengths(B, case["q"], True, 1, host), tail)
        per = head + -(-case["kv"] // page)
        need = case["groups"] * head + B * (per - head)
        order = torch.randperm(need + 3, generator=gen, device=DEV)[:need].to(torch.int32)
        first = order[:case["groups"] * head].reshape(case["groups"], 1, head).expand(-1, case["members"], -1).reshape(B, head)
        s["table"] = torch.cat([first, order[case["groups"] * head:].reshape(B, per - head)], 1).contiguous()
        s["group_start"] = torch.arange(0, B + 1, case["members"], dtype=torch.int32, device=DEV)
        s["shared"] = torch.full((case["groups"],), case["shared"], dtype=torch.int32, device=DEV)
    else:
        B = case["segments"]
        kl = _lengths(B, case["kv"], case["ragged"], 1, host)
        ql = torch.minimum(_lengths(B, case.get("q", 1), case["ragged"], 1, host), kl)
        per = -(-case["kv"] // page)
        need = B * per
        # a cache in use: the pages of a sequence lie anywhere among those of the others
        s["table"] = torch.randperm(need + 3, generator=gen, device=DEV)[:need].to(torch.int32).reshape(B, per)
    s["kv_len"], s["q_start"], s["q_row"] = kl.to(DEV, torch.int32), _starts(ql).to(DEV, torch.int32), _rows(ql)
    s["key_pages"], s["value_pages"] = (_normal(gen, (need + 3, page, hk, D), dt) for _ in range(2))
    if case["op"] == "evict":
        # what attention leaves behind: a few positions with most of the weight, many with hardly any, some that no token has read
        w = torch.exp(3 * torch.randn((B, hk, per * page), generator=gen, device=DEV))
        s["weights"] = w * (torch.rand(w.shape, generator=gen, device=DEV) < 0.95)
        keep = -(-case["keep"] // page)
        s["to_table"] = torch.randperm(B * keep, generator=gen, device=DEV).to(torch.int32).reshape(B, keep)
        s["to_key"], s["to_value"] = (torch.zeros((B * keep, page, hk, D), dtype=dt, device=DEV) for _ in range(2))
        s["to_len"] = torch.zeros(B, dtype=torch.int32, device=DEV)
        return s
    s["q"] = _normal(gen, (int(ql.sum()), case["heads"], D), dt)
    if case["op"] == "weights":
        k, seen = _cached(s, "key_pages"), _seen(s)
        sc = _scores(_padded(s["q"], s["q_start"], case["q"])[0], k, s["scale"], seen[:, None, None], case["heads"], hk)
        s["lse"] = _unpad(torch.logsumexp(sc, -1), s["q_row"], case["heads"])      # the attention's own output
        s["weights"] = torch.zeros((B, hk, per * page), device=DEV)
        s["before"] = torch.exp(torch.randn(s["weights"].shape, generator=gen, device=DEV)) if case["added"] else None
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _padded(x, start, longest):
    """[segments, longest, ...] of the rows of x, and which of them exist."""
    at = torch.arange(longest, device=DEV)
    start = start.long()
    there = at[None] < (start[1:] - start[:-1])[:, None]
    return x[(start[:-1, None] + at[None]).clamp(max=max(x.shape[0] - 1, 0))], there


def _unpad(x, rows, heads):
    """[B, kv_heads, group, Lq, ...] back to [rows, heads, ...]."""
    x = x.flatten(1, 2).movedim(1, 2)
    return x[rows[0], rows[1]]


def _scores(q, key, scale, seen, heads, kv_heads):
    """[B, kv_heads, group, Lq, Lk]; -inf where a row does not read a key."""
    q = q.float().reshape(q.shape[0], q.shape[1], kv_heads, heads // kv_heads, q.shape[3])
    return (torch.einsum("bqhgd,bkhd->bhgqk", q, key.float()) * scale).masked_fill_(~seen, -math.inf)


def _softmax(sc):
    """The weights, in place, and the log of the masses."""
    top = sc.amax(-1, keepdim=True)
    top.masked_fill_(top == -math.inf, 0.0)
    sc.sub_(top).exp_()
    mass = sc.sum(-1, keepdim=True)
    sc.div_(mass.clamp(min=1e-30))
    return sc, (top + torch.log(mass))[..., 0]


def _cached(s, name):
    """[sequences, positions, kv_heads, D] of the cache."""
    return s[name][s["table"].long()].flatten(1, 2)


def _seen(s):
    """[sequences, new tokens, positions]: which positions a new token reads."""
    new = (s["q_start"][1:] - s["q_start"][:-1])[:, None]
    last = s["kv_len"][:, None] - new + torch.arange(s["case"]["q"], device=DEV)[None]
    at = torch.arange(s["table"].shape[1] * s["case"]["page"], device=DEV)
    return (at[None, None] <= last[:, :, None]) & (at[None, None] < s["kv_len"][:, None, None])


def _plain_triangle(s):
    c = s["case"]
    h, hk, D, dt = c["heads"], c["kv_heads"], c["D"], s["q"].dtype
    q, q_there = _padded(s["q"], s["q_start"], c["q"])
    k, there = _padded(s["key"], s["kv_start"], c["kv"])
    v, _ = _padded(s["value"], s["kv_start"], c["kv"])
    if s["mask"] is not None:
        there = there & _padded(s["mask"], s["kv_start"], c["kv"])[0]
    n, m = (s[x][1:] - s[x][:-1] for x in ("q_start", "kv_start"))
    last = (m - n)[:, None] + torch.arange(c["q"], device=DEV)[None]
    seen = there[:, None] & (torch.arange(c["kv"], device=DEV)[None, None] <= last[:, :, None])
    v = v.float()
    p, lse = _softmax(_scores(q, k, s["scale"], seen[:, None, None], h, hk))
    res = {"out": _unpad(torch.einsum("bhgqk,bkhd->bhgqd", p, v), s["q_row"], h).to(dt), "lse": _unpad(lse, s["q_row"], h)}
    if s["grad_out"] is None:
        return res
    g = _padded(s["grad_out"], s["q_start"], c["q"])[0]
    g = (g * q_there[:, :, None, None]).float().reshape(*g.shape[:2], hk, h // hk, D)
    q = q.float().reshape(g.shape)
    res["grad_value"] = torch.einsum("bhgqk,bqhgd->bkhd", p, g)
    ds = torch.einsum("bqhgd,bkhd->bhgqk", g, v)
    ds.sub_((ds * p).sum(-1, keepdim=True)).mul_(p).mul_(s["scale"])
    res["grad_q"] = _unpad(torch.einsum("bhgqk,bkhd->bhgqd", ds, k.float()), s["q_row"], h).to(dt)
    res["grad_key"] = torch.einsum("bhgqk,bqhgd->bkhd", ds, q)
    seg, place = s["kv_row"]
    for name in ("grad_key", "grad_value"):
        res[name] = res[name][seg, place].to(dt)
    return res


def _plain_shared(s):
    c = s["case"]
    h, hk = c["heads"], c["kv_heads"]
    q, _ = _padded(s["q"], s["q_start"], c["q"])
    p, lse = _softmax(_scores(q, _cached(s, "key_pages"), s["scale"], _seen(s)[:, None, None], h, hk))
    out = torch.einsum("bhgqk,bkhd->bhgqd", p, _cached(s, "value_pages").float())
    return {"out": _unpad(out, s["q_row"], h).to(s["q"].dtype), "lse": _unpad(lse, s["q_row"], h)}


def _plain_weights(s):
    c = s["case"]
    h, hk = c["heads"], c["kv_heads"]
    q, there = _padded(s["q"], s["q_start"], c["q"])
    lse = _padded(s["lse"], s["q_start"], c["q"])[0].masked_fill(~there[:, :, None], math.inf)
    sc = _scores(q, _cached(s, "key_pages"), s["scale"], _seen(s)[:, None, None], h, hk)
    sc.sub_(lse.movedim(1, 2).reshape(sc.shape[:-1])[..., None]).exp_()
    w = sc.sum((2, 3))
    if s["before"] is not None:
        w = s["before"] + w
    at = torch.arange(w.shape[2], device=DEV)
    return {"weights": torch.where(at[None, None] < s["kv_len"][:, None, None], w, s["weights"])}


def _plain_evict(s):
    c = s["case"]
    B, hk, page, keep = c["segments"], c["kv_heads"], c["page"], c["keep"]
    n = s["kv_len"].long()[:, None, None]
    at = torch.arange(s["weights"].shape[2], device=DEV)[None, None]
    rank = s["weights"].masked_fill(at >= n - c["recent"], math.inf).masked_fill(at >= n, -math.inf)
    first = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :keep]
    there = torch.arange(first.shape[2], device=DEV)[None, None] < n
    kept = torch.sort(first.masked_fill(~there, at.shape[2]), dim=-1).values
    there = kept < at.shape[2]
    kept = kept.masked_fill(~there, 0)
    seg, head = torch.arange(B, device=DEV)[:, None, None].expand_as(kept), torch.arange(hk, device=DEV)[None, :, None].expand_as(kept)
    place = torch.arange(kept.shape[2], device=DEV)[None, None].expand_as(kept)
    source = s["table"].long()[seg, kept // page] * page + kept % page
    target = s["to_table"].long()[seg, place // page] * page + place % page
    for name in ("key", "value"):
        s["to_" + name].flatten(0, 1)[target[there], head[there]] = s[name + "_pages"].flatten(0, 1)[source[there], head[there]]
    left = torch.zeros((B, hk, s["to_table"].shape[1] * page), device=DEV)
    left[..., :kept.shape[2]] = s["weights"].gather(2, kept).masked_fill(~there, 0.0)
    chosen = torch.full((B, hk, keep), -1, dtype=torch.int32, device=DEV)
    chosen[..., :kept.shape[2]] = kept.masked_fill(~there, -1).to(torch.int32)
    s["to_len"].copy_(s["kv_len"].clamp(max=keep))
    return {"key_pages": s["to_key"], "value_pages": s["to_value"], "kv_len": s["to_len"], "kept": chosen, "weights": left}


# ------------------------------------------------------------------------------------------------ through the library

def _own(s):
    from paper_2609_24802_b200 import api as T
    c = s["case"]
    if c["op"] == "triangle":
        g = T.TriangularRelation(s["q_start"], s["kv_start"], s["mask"])
        out, lse, _ = T.tiga_apply_triangular_attention(g, s["q"], s["key"], s["value"], s["scale"])
        res = {"out": out, "lse": lse}
        if s["grad_out"] is not None:
            res["grad_q"], res["grad_key"], res["grad_value"], _ = T.tiga_apply_triangular_attention_backward(
                g, s["q"], s["key"], s["value"], out, lse, s["grad_out"], s["scale"])
        return res
    cache = T.PagedCache(s["key_pages"], s["value_pages"], s["table"], s["kv_len"])
    if c["op"] == "shared":
        out, lse, _ = T.tiga_apply_shared_attention(cache, T.SharedPrefixes(s["group_start"], s["shared"]), s["q"], s["q_start"], s["scale"])
        return {"out": out, "lse": lse}
    if c["op"] == "weights":
        weights, _ = T.tiga_paged_attention_weights(cache, s["q"], s["q_start"], s["lse"], s["scale"], before=s["before"], weights=s["weights"])
        return {"weights": weights}
    to = T.PagedCache(s["to_key"], s["to_value"], s["to_table"], s["to_len"])
    kept, weights = T.tiga_paged_evict(cache, to, s["weights"], c["keep"], c["recent"])
    return {"key_pages": s["to_key"], "value_pages": s["to_value"], "kv_len": s["to_len"], "kept": kept, "weights": weights}


def run(state):
    if own:
        return _own(state)
    return {"triangle": _plain_triangle, "shared": _plain_shared, "weights": _plain_weights, "evict": _plain_evict}[state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------------ work, and 64 bits

def work(case):
    D, hk, h = case["D"], case["kv_heads"], case.get("heads", 0)
    if case["op"] == "shared":
        n, kv = case["groups"] * case["members"], case["kv"] * 0.625
        nq = n * max(1.0, case["q"] * 0.625)
        return {"bytes": int(4 * nq * h * D + 4 * nq * h + 4 * (case["groups"] * case["shared"] + n * kv) * hk * D),
                "flops": int(4 * nq * (case["shared"] + kv) * h * D)}
    B = case["segments"]
    part = 0.625 if case["ragged"] and B > 1 else 1.0       # mean length of a ragged batch over its longest
    nk = case["kv"] * part
    if case["op"] == "triangle":
        nq = max(1.0, nk - (case["kv"] - case["q"]))
        pairs = B * nq * (nk - (nq - 1) / 2) * (0.8 if case["masked"] else 1.0)
        flops, size = 4 * pairs * h * D, B * (4 * nq * h * D + 4 * nq * h + 4 * nk * hk * D)
        if case["backward"]:
            flops, size = 3.5 * flops, size + B * 4 * (nq * h + nk * hk) * D
        return {"bytes": int(size), "flops": int(flops)}
    if case["op"] == "weights":
        nq = max(1.0, case["q"] * part)
        return {"bytes": int(B * (nq * h * (2 * D + 4) + nk * hk * (2 * D + (8 if case["added"] else 4)))), "flops": int(2 * B * nq * max(1.0, nk - (nq - 1) / 2) * h * D)}
    kept = min(nk, case["keep"])
    return {"bytes": int(B * hk * (4 * nk + kept * (8 * D + 8))), "flops": int(B * hk * nk)}


def _exact_head(q, k, v, scale, seen, g=None):
    """One kv head of one sequence: q [n, group, D], k, v [m, D], seen [n, m]; everything in 64 bits."""
    x = (q @ k.T) * scale
    x = torch.where(seen[:, None], x, torch.full_like(x, -math.inf))
    lse = torch.logsumexp(x, -1)
    p = torch.exp(x - torch.where(lse == -math.inf, torch.zeros_like(lse), lse)[..., None])
    o = p @ v
    if g is None:
        return o, lse
    ds = p * (g @ v.T - (g * o).sum(-1, keepdim=True)) * scale
    return o, lse, ds @ k, torch.tensordot(ds, q, ([0, 1], [0, 1])), torch.tensordot(p, g, ([0, 1], [0, 1]))


def _exact_evict(s):
    c = s["case"]
    page, keep, hk = c["page"], c["keep"], c["kv_heads"]
    res = {"key_pages": s["to_key"].clone(), "value_pages": s["to_value"].clone(), "kv_len": s["kv_len"].clamp(max=keep)}
    kept = torch.full((c["segments"], hk, keep), -1, dtype=torch.int32, device=DEV)
    left = torch.zeros((c["segments"], hk, s["to_table"].shape[1] * page), dtype=torch.float64, device=DEV)
    for b, n in enumerate(s["kv_len"].tolist()):
        for i in range(hk):
            w = s["weights"][b, i, :n].double()
            old = max(n - c["recent"], 0)
            most = min(n, keep) - (n - old)
            if most < old:          # the largest weights; of equal ones at the border those that come first
                border = torch.topk(w[:old], most).values[-1] if most else math.inf
                chosen = w[:old] > border
                equal = (w[:old] == border).nonzero()[:, 0]
                chosen[equal[:most - int(chosen.sum())]] = True
            else:
                chosen = torch.ones(old, dtype=torch.bool, device=DEV)
            at = torch.cat([chosen.nonzero()[:, 0], torch.arange(old, n, device=DEV)])
            to = torch.arange(at.numel(), device=DEV)
            kept[b, i, :at.numel()], left[b, i, :at.numel()] = at.to(torch.int32), w[at]
            a, z = s["table"][b].long()[at // page], s["to_table"][b].long()[to // page]
            res["key_pages"][z, to % page, i], res["value_pages"][z, to % page, i] = s["key_pages"][a, at % page, i], s["value_pages"][a, at % page, i]
    return res | {"kept": kept, "weights": left}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "evict":
        return _exact_evict(s)
    h, hk, D = case["heads"], case["kv_heads"], case["D"]
    q = s["q"].double().reshape(-1, hk, h // hk, D)
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:3], dtype=torch.float64, device=DEV)
    qs = s["q_start"].tolist()
    if case["op"] == "triangle":
        ks = s["kv_start"].tolist()
        k, v = s["key"].double(), s["value"].double()
        res = {"out": out.view(-1, h, D), "lse": lse.view(-1, h)}
        if case["backward"]:
            g, gq, gk, gv = s["grad_out"].double().reshape(q.shape), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
            res |= {"grad_value": gv, "grad_q": gq.view(-1, h, D), "grad_key": gk}
        for b in range(case["segments"]):
            rows, keys, n, m = slice(qs[b], qs[b + 1]), slice(ks[b], ks[b + 1]), qs[b + 1] - qs[b], ks[b + 1] - ks[b]
            seen = torch.ones(n, m, dtype=torch.bool, device=DEV).tril(m - n)
            if s["mask"] is not None:
                seen = seen & s["mask"][keys][None]
            for i in range(hk):
                got = _exact_head(q[rows, i], k[keys, i], v[keys, i], s["scale"], seen, g[rows, i] if case["backward"] else None)
                out[rows, i], lse[rows, i] = got[:2]
                if case["backward"]:
                    gq[rows, i], gk[keys, i], gv[keys, i] = got[2:]
        return res
    w = s["weights"].double() if case["op"] == "weights" else None
    for b, m in enumerate(s["kv_len"].tolist()):
        rows, n = slice(qs[b], qs[b + 1]), qs[b + 1] - qs[b]
        seen = torch.ones(n, m, dtype=torch.bool, device=DEV).tril(m - n)
        for i in range(hk):
            k, v = (s[x][s["table"][b].long(), :, i].reshape(-1, D)[:m].double() for x in ("key_pages", "value_pages"))
            if w is None:
                out[rows, i], lse[rows, i] = _exact_head(q[rows, i], k, v, s["scale"], seen)
            else:
                x = torch.exp((q[rows, i] @ k.T) * s["scale"] - s["lse"].double().reshape(-1, hk, h // hk)[rows, i, :, None])
                w[b, i, :m] = (x * seen[:, None]).sum((0, 1)) + (s["before"][b, i, :m].double() if case["added"] else 0.0)
    return {"out": out.view(-1, h, D), "lse": lse.view(-1, h)} if w is None else {"weights": w}

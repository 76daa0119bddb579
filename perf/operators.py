"""Attention over relations that are not stored, and what feeds it: the work a program hands to this library.

Every case is a dict of plain values.  ``op`` names the operator:

  dense    online-softmax reducer over a block-diagonal dense relation (cross attention: the rows of a segment read all
           keys of that segment), grouped heads, optional mask of keys; forward, or forward + gradients
  paged    the same reducer over a triangular relation whose keys and values lie in the pages of a cache: a chunk of new
           tokens per sequence, down to single tokens
  rotary   rotary positions of queries and keys, forward + gradient
  append   keys (rotated on the way) and values of new tokens written into the pages of a cache

``run`` computes the operators in plain torch operations, or, where ``own`` is true, through the library.
Inputs are made on the GPU from the seed alone.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one short sequence of two heads in a training loop (the smallest step): launches and latency count
        {"name": "dense_step_small", "op": "dense", "segments": 1, "q": 65, "kv": 65, "ragged": False, "heads": 2, "kv_heads": 2,
         "D": 64, "dtype": "f16", "masked": False, "backward": True},
        # a few latent queries per graph that read all nodes of a padded batch of graphs: few rows, a long axis
        {"name": "dense_pool", "op": "dense", "segments": 32, "q": 64, "kv": 4096, "ragged": True, "heads": 8, "kv_heads": 8,
         "D": 64, "dtype": "bf16", "masked": True, "backward": False},
        # a decoder layer's cross attention in training, ragged targets and ragged encoder states
        {"name": "dense_step_ragged", "op": "dense", "segments": 16, "q": 1024, "kv": 1500, "ragged": True, "heads": 16, "kv_heads": 16,
         "D": 64, "dtype": "f16", "masked": False, "backward": True},
        # the largest training step: long targets and long encoder states, grouped heads (the largest case)
        {"name": "dense_step_large", "op": "dense", "segments": 4, "q": 4096, "kv": 4096, "ragged": False, "heads": 16, "kv_heads": 4,
         "D": 128, "dtype": "bf16", "masked": False, "backward": True},
        # one user's next token on a short cache: latency counts
        {"name": "paged_token_short", "op": "paged", "segments": 1, "q": 1, "kv": 777, "ragged": False, "heads": 8, "kv_heads": 2,
         "D": 64, "dtype": "bf16", "page": 16},
        # next tokens of a batch of users, ragged caches: the bandwidth of the cache counts
        {"name": "paged_tokens_batch", "op": "paged", "segments": 64, "q": 1, "kv": 8192, "ragged": True, "heads": 32, "kv_heads": 8,
         "D": 128, "dtype": "bf16", "page": 32},
        # one next token on a very long cache
        {"name": "paged_token_long", "op": "paged", "segments": 1, "q": 1, "kv": 262143, "ragged": False, "heads": 32, "kv_heads": 8,
         "D": 128, "dtype": "f16", "page": 64},
        # a chunk of a long prompt on what is cached of it: the products count
        {"name": "paged_chunk", "op": "paged", "segments": 1, "q": 2048, "kv": 16384, "ragged": False, "heads": 32, "kv_heads": 8,
         "D": 128, "dtype": "bf16", "page": 64},
        # queries and keys of a few tokens, part of the head, interleaved pairs
        {"name": "rotary_small", "op": "rotary", "tokens": 33, "far": 4096, "heads": 8, "kv_heads": 8, "D": 80, "turned": 32,
         "pairs": True, "scaled": False, "dtype": "f16"},
        # queries and keys of a training batch at positions of a long context, scaled frequencies
        {"name": "rotary_step", "op": "rotary", "tokens": 16384, "far": 1 << 20, "heads": 32, "kv_heads": 8, "D": 128, "turned": 128,
         "pairs": False, "scaled": True, "dtype": "bf16"},
        # the new tokens of a batch of users enter their caches
        {"name": "append_tokens", "op": "append", "segments": 64, "q": 1, "kv": 8192, "ragged": True, "kv_heads": 8, "D": 128,
         "turned": 128, "pairs": False, "dtype": "bf16", "page": 32},
        # chunks of long prompts enter their caches
        {"name": "append_chunks", "op": "append", "segments": 4, "q": 4096, "kv": 16384, "ragged": True, "kv_heads": 8, "D": 128,
         "turned": 64, "pairs": True, "dtype": "f16", "page": 64},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["dense", "dense", "paged", "paged", "rotary", "append"])
    kv_heads = rng.choice([1, 2, 3, 4, 8])
    heads = kv_heads * rng.choice([1, 2, 3, 4, 5, 8])
    D = rng.choice([32, 64, 64, 72, 96, 128, 128])
    dtype = rng.choice(["f16", "bf16"])
    while True:
        if op == "dense":
            c = {"op": op, "segments": _log(rng, 1, 64), "q": _log(rng, 1, 4096), "kv": _log(rng, 1, 4096), "ragged": rng.random() < 0.7,
                 "heads": heads, "kv_heads": kv_heads, "D": D, "dtype": dtype, "masked": rng.random() < 0.4, "backward": rng.random() < 0.6}
            if c["segments"] * c["q"] * c["kv"] * heads * D * (10 if c["backward"] else 4) <= 4 * 4096 * 4096 * 16 * 128 * 10:
                return c
        elif op == "paged":
            c = {"op": op, "segments": _log(rng, 1, 128), "q": rng.choice([1, 1, _log(rng, 2, 2048)]), "kv": _log(rng, 1, 131072),
                 "ragged": rng.random() < 0.7, "heads": heads, "kv_heads": kv_heads, "D": D, "dtype": dtype, "page": rng.choice([8, 16, 32, 48, 64, 128])}
            c["kv"] = max(c["kv"], c["q"])
            if c["segments"] * c["q"] * c["kv"] * heads * D <= 2048 * 16384 * 32 * 128 and c["segments"] * c["kv"] * kv_heads * D <= 1 << 28:
                return c
        elif op == "rotary":
            return {"op": op, "tokens": _log(rng, 1, 16384), "far": _log(rng, 16384, 1 << 22), "heads": heads, "kv_heads": kv_heads, "D": D,
                    "turned": rng.choice([D, D, D // 2]), "pairs": rng.random() < 0.5, "scaled": rng.random() < 0.5,
                    "dtype": rng.choice(["f16", "bf16", "f32"])}
        else:
            c = {"op": op, "segments": _log(rng, 1, 128), "q": rng.choice([1, _log(rng, 2, 4096)]), "kv": _log(rng, 1, 16384), "ragged": rng.random() < 0.7,
                 "kv_heads": kv_heads, "D": D, "turned": rng.choice([0, D, D // 2]), "pairs": rng.random() < 0.5, "dtype": dtype,
                 "page": rng.choice([8, 16, 32, 48, 64, 128])}
            c["kv"] = max(c["kv"], c["q"])
            if c["segments"] * c["kv"] * kv_heads * D <= 1 << 27:
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


def _frequencies(turned, scaled, base=10000.0, factor=8.0, length=8192.0, slow=1.0, fast=32.0):
    """Radians per position of every pair, in 64 bits.  Scaled: pairs that turn often over the original length stay, slow
    ones are interpolated, a ramp between."""
    f = base ** (-torch.arange(0, turned, 2, dtype=torch.float64) / turned)
    if not scaled:
        return f, 1.0
    keep = ((length * f / (2 * math.pi) - slow) / (fast - slow)).clamp(0, 1)
    return keep * f + (1 - keep) * f / factor, 0.1 * math.log(factor) + 1


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    D, hk = case["D"], case["kv_heads"]
    s = {"case": case}
    if case["op"] == "dense":
        B, h = case["segments"], case["heads"]
        ql, kl = _lengths(B, case["q"], case["ragged"], 1, host), _lengths(B, case["kv"], case["ragged"], 0, host)
        s["q_start"], s["kv_start"] = (_starts(a).to(DEV, torch.int32) for a in (ql, kl))
        s["q_row"], s["kv_row"] = _rows(ql), _rows(kl)
        nq, nk = int(ql.sum()), int(kl.sum())
        s["q"] = _normal(gen, (nq, h, D), dt)
        kv = _normal(gen, (nk, 2, hk, D), dt)              # one projection of the encoder's states gives both
        s["key"], s["value"] = kv[:, 0], kv[:, 1]
        s["mask"] = torch.rand(nk, generator=gen, device=DEV) < 0.8 if case["masked"] else None
        s["grad_out"] = _normal(gen, (nq, h, D), dt, 0.1) if case["backward"] else None
        s["scale"] = D ** -0.5
    elif case["op"] in ("paged", "append"):
        B, page = case["segments"], case["page"]
        kl = _lengths(B, case["kv"], case["ragged"], 1, host)
        ql = _lengths(B, case["q"], case["ragged"], 1, host)
        kl = torch.maximum(kl, ql)
        s["q_start"], s["kv_len"] = _starts(ql).to(DEV, torch.int32), kl.to(DEV, torch.int32)
        s["q_row"] = _rows(ql)
        per = -(-case["kv"] // page)
        need = B * per
        # a cache in use: the pages of a sequence lie anywhere among those of the others
        s["table"] = torch.randperm(need + 3, generator=gen, device=DEV)[:need].to(torch.int32).reshape(B, per)
        s["key_pages"] = _normal(gen, (need + 3, page, hk, D), dt)
        s["value_pages"] = _normal(gen, (need + 3, page, hk, D), dt)
        nq = int(ql.sum())
        if case["op"] == "paged":
            s["q"] = _normal(gen, (nq, case["heads"], D), dt)
            s["scale"] = D ** -0.5
        else:
            kv = _normal(gen, (nq, 2, hk, D), dt)
            s["key"], s["value"] = kv[:, 0], kv[:, 1]
            s["freq"], s["magnitude"] = _frequencies(case["turned"], False) if case["turned"] else (None, 1.0)
    else:
        n, h = case["tokens"], case["heads"]
        qkv = _normal(gen, (n, h + 2 * hk, D), dt)         # one projection gives queries, keys and values
        s["q"], s["key"] = qkv[:, :h], qkv[:, h:h + hk]
        s["grad_q"], s["grad_key"] = _normal(gen, (n, h, D), dt, 0.1), _normal(gen, (n, hk, D), dt, 0.1)
        s["positions"] = torch.randint(0, case["far"], (n,), generator=gen, device=DEV, dtype=torch.int32)
        s["freq"], s["magnitude"] = _frequencies(case["turned"], case["scaled"])
    if s.get("freq") is not None:
        s["freq"] = s["freq"].to(DEV)
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _padded(x, start, longest):
    """[segments, longest, ...] of the rows of x, and which of them exist."""
    at = torch.arange(longest, device=DEV)
    start = start.long()
    there = at[None] < (start[1:] - start[:-1])[:, None]
    return x[(start[:-1, None] + at[None]).clamp(max=max(x.shape[0] - 1, 0))], there


def _scores(q, key, scale, seen, heads, kv_heads):
    """softmax weights [B, kv_heads, group, Lq, Lk] and the log of the masses."""
    q = q.reshape(q.shape[0], q.shape[1], kv_heads, heads // kv_heads, q.shape[3])
    sc = torch.einsum("bqhgd,bkhd->bhgqk", q, key) * scale
    sc.masked_fill_(~seen, -math.inf)
    top = sc.amax(-1, keepdim=True)
    top.masked_fill_(top == -math.inf, 0.0)
    sc.sub_(top).exp_()
    mass = sc.sum(-1, keepdim=True)
    sc.div_(mass.clamp(min=1e-30))
    return sc, (top + torch.log(mass))[..., 0]


def _unpad(x, rows, heads):
    """[B, kv_heads, group, Lq, ...] back to [rows, heads, ...]."""
    x = x.flatten(1, 2).movedim(1, 2)
    return x[rows[0], rows[1]]


def _plain_dense(s):
    c = s["case"]
    h, hk, D, dt = c["heads"], c["kv_heads"], c["D"], s["q"].dtype
    q, _ = _padded(s["q"], s["q_start"], c["q"])
    k, there = _padded(s["key"], s["kv_start"], c["kv"])
    v, _ = _padded(s["value"], s["kv_start"], c["kv"])
    if s["mask"] is not None:
        there = there & _padded(s["mask"], s["kv_start"], c["kv"])[0]
    q, k, v = q.float(), k.float(), v.float()
    p, lse = _scores(q, k, s["scale"], there[:, None, None, None], h, hk)
    out = _unpad(torch.einsum("bhgqk,bkhd->bhgqd", p, v), s["q_row"], h)
    res = {"out": out.to(dt), "lse": _unpad(lse, s["q_row"], h)}
    if s["grad_out"] is None:
        return res
    g, q_there = _padded(s["grad_out"], s["q_start"], c["q"])
    g = (g * q_there[:, :, None, None]).float().reshape(*g.shape[:2], hk, h // hk, D)
    q = q.reshape(g.shape)
    res["grad_value"] = torch.einsum("bhgqk,bqhgd->bkhd", p, g)
    ds = torch.einsum("bqhgd,bkhd->bhgqk", g, v)
    ds.sub_((ds * p).sum(-1, keepdim=True)).mul_(p).mul_(s["scale"])
    res["grad_q"] = _unpad(torch.einsum("bhgqk,bkhd->bhgqd", ds, k), s["q_row"], h).to(dt)
    res["grad_key"] = torch.einsum("bhgqk,bqhgd->bkhd", ds, q)
    seg, place = s["kv_row"]
    for name in ("grad_key", "grad_value"):
        res[name] = res[name][seg, place].to(dt)
    return res


def _plain_paged(s):
    c = s["case"]
    h, hk, dt = c["heads"], c["kv_heads"], s["q"].dtype
    q, _ = _padded(s["q"], s["q_start"], c["q"])
    k, v = (s[n][s["table"].long()].flatten(1, 2).float() for n in ("key_pages", "value_pages"))
    new = (s["q_start"][1:] - s["q_start"][:-1])[:, None]
    last = s["kv_len"][:, None] - new + torch.arange(c["q"], device=DEV)[None]       # the last key that a row reads
    at = torch.arange(k.shape[1], device=DEV)
    seen = (at[None, None] <= last[:, :, None]) & (at[None, None] < s["kv_len"][:, None, None])
    p, lse = _scores(q.float(), k, s["scale"], seen[:, None, None], h, hk)
    return {"out": _unpad(torch.einsum("bhgqk,bkhd->bhgqd", p, v), s["q_row"], h).to(dt), "lse": _unpad(lse, s["q_row"], h)}


def _turn(x, angle, magnitude, pairs, inverse=False):
    """Rotary positions of x [n, heads, D] by angle [n, pairs of the head] (64 bits)."""
    r = 2 * angle.shape[1]
    cos = (magnitude * torch.cos(angle)).float()[:, None]
    sin = (magnitude * torch.sin(angle)).float()[:, None]
    if inverse:
        sin = -sin
    y = x.float()
    a, b = (y[..., 0:r:2], y[..., 1:r:2]) if pairs else (y[..., :r // 2], y[..., r // 2:r])
    a, b = a * cos - b * sin, a * sin + b * cos
    y = torch.cat([torch.stack([a, b], -1).flatten(-2) if pairs else torch.cat([a, b], -1), y[..., r:]], -1)
    return y.to(x.dtype)


def _plain_rotary(s):
    angle = s["positions"].double()[:, None] * s["freq"][None]
    m, pairs = s["magnitude"], s["case"]["pairs"]
    return {"q": _turn(s["q"], angle, m, pairs), "key": _turn(s["key"], angle, m, pairs),
            "grad_q": _turn(s["grad_q"], angle, m, pairs, True), "grad_key": _turn(s["grad_key"], angle, m, pairs, True)}


def _places(s):
    """Position of every new token in its sequence, and its slot in the cache."""
    seg, place = s["q_row"]
    new = s["q_start"][1:] - s["q_start"][:-1]
    pos = (s["kv_len"] - new).long()[seg] + place
    page = s["case"]["page"]
    return pos, s["table"].long()[seg, pos // page] * page + pos % page


def _plain_append(s):
    pos, slot = _places(s)
    key = s["key"]
    if s["freq"] is not None:
        key = _turn(key, pos.double()[:, None] * s["freq"][None], s["magnitude"], s["case"]["pairs"])
    s["key_pages"].flatten(0, 1)[slot] = key
    s["value_pages"].flatten(0, 1)[slot] = s["value"]
    return {"key_pages": s["key_pages"], "value_pages": s["value_pages"]}


# ------------------------------------------------------------------------------------------------ through the library

def _own(s):
    from paper_2609_24802_b200 import api as T
    c = s["case"]
    if c["op"] == "dense":
        g = T.DenseRelation(s["q_start"], s["kv_start"], s["mask"])
        out, lse, _ = T.tiga_apply_dense_attention(g, s["q"], s["key"], s["value"], s["scale"])
        res = {"out": out, "lse": lse}
        if s["grad_out"] is not None:
            res["grad_q"], res["grad_key"], res["grad_value"], _ = T.tiga_apply_dense_attention_backward(
                g, s["q"], s["key"], s["value"], out, lse, s["grad_out"], s["scale"])
        return res
    if c["op"] == "paged":
        cache = T.PagedCache(s["key_pages"], s["value_pages"], s["table"], s["kv_len"])
        out, lse, _ = T.tiga_apply_paged_attention(cache, s["q"], s["q_start"], s["scale"])
        return {"out": out, "lse": lse}
    rot = T.Rotary(s["freq"], pairs=c["pairs"], magnitude=s["magnitude"]) if s["freq"] is not None else None
    if c["op"] == "rotary":
        return {"q": T.tiga_apply_rotary(rot, s["q"], s["positions"]), "key": T.tiga_apply_rotary(rot, s["key"], s["positions"]),
                "grad_q": T.tiga_apply_rotary(rot, s["grad_q"], s["positions"], inverse=True),
                "grad_key": T.tiga_apply_rotary(rot, s["grad_key"], s["positions"], inverse=True)}
    cache = T.PagedCache(s["key_pages"], s["value_pages"], s["table"], s["kv_len"])
    T.tiga_paged_append(cache, s["key"], s["value"], s["q_start"], rotary=rot)
    return {"key_pages": s["key_pages"], "value_pages": s["value_pages"]}


def run(state):
    if own:
        return _own(state)
    return {"dense": _plain_dense, "paged": _plain_paged, "rotary": _plain_rotary, "append": _plain_append}[state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------------ work, and 64 bits

def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    D, hk, h = case["D"], case["kv_heads"], case.get("heads", 0)
    B = case.get("segments", 1)
    part = 0.625 if case.get("ragged") and B > 1 else 1.0       # mean length of a ragged batch over its longest
    if case["op"] == "dense":
        nq, nk, pairs = B * case["q"] * part, B * case["kv"] * part, B * case["q"] * case["kv"] * part * part
        if case["masked"]:
            pairs *= 0.8
        flops, size = 4 * pairs * h * D, 2 * nq * h * D * e + nq * h * 4 + 2 * nk * hk * D * e
        if case["backward"]:
            flops, size = 3.5 * flops, size + 2 * nq * h * D * e + 2 * nk * hk * D * e
        return {"bytes": int(size), "flops": int(flops)}
    if case["op"] == "paged":
        nq, nk = B * max(1, case["q"] * part if case["q"] > 1 else 1), B * case["kv"] * part
        pairs = nq * max(1.0, case["kv"] * part - (nq / B - 1) / 2)
        return {"bytes": int(2 * nq * h * D * e + nq * h * 4 + 2 * nk * hk * D * e), "flops": int(4 * pairs * h * D)}
    if case["op"] == "rotary":
        n = case["tokens"] * (h + hk)
        return {"bytes": int(2 * 2 * n * D * e), "flops": int(2 * 3 * n * case["turned"])}
    nq = B * max(1, case["q"] * part if case["q"] > 1 else 1)
    return {"bytes": int(2 * 2 * nq * hk * D * e), "flops": int(3 * nq * hk * case["turned"])}


def _exact_attention(q, k, v, scale, seen, g=None):
    """One head of one segment: q [n, D], k, v [m, D], seen [n, m]; everything in 64 bits."""
    x = (q @ k.T) * scale
    x = torch.where(seen, x, torch.full_like(x, -math.inf))
    lse = torch.logsumexp(x, -1)
    p = torch.exp(x - torch.where(lse == -math.inf, torch.zeros_like(lse), lse)[:, None])
    o = p @ v
    if g is None:
        return o, lse
    dp = g @ v.T
    ds = p * (dp - (g * o).sum(-1, keepdim=True)) * scale
    return o, lse, ds @ k, ds.T @ q, p.T @ g


def _exact_turn(x, pos, freq, m, pairs, sign):
    z = x.double().clone()
    for i in range(freq.numel()):
        a, b = (2 * i, 2 * i + 1) if pairs else (i, i + freq.numel())
        t = pos.double() * freq[i]
        c, s = m * torch.cos(t)[:, None], sign * m * torch.sin(t)[:, None]
        z[..., a], z[..., b] = x[..., a].double() * c - x[..., b].double() * s, x[..., a].double() * s + x[..., b].double() * c
    return z


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("dense", "paged"):
        h, hk = case["heads"], case["kv_heads"]
        if case["segments"] * h > 4096:
            return None
        q = s["q"].double()
        out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], dtype=torch.float64, device=DEV)
        qs = s["q_start"].tolist()
        if case["op"] == "paged":
            lens = s["kv_len"].tolist()
            for b in range(case["segments"]):
                rows, n = slice(qs[b], qs[b + 1]), qs[b + 1] - qs[b]
                pages = s["table"][b].long()
                seen = torch.arange(lens[b], device=DEV)[None] <= lens[b] - n + torch.arange(n, device=DEV)[:, None]
                for i in range(h):
                    k, v = (s[x][pages, :, i * hk // h].reshape(-1, case["D"])[:lens[b]].double() for x in ("key_pages", "value_pages"))
                    out[rows, i], lse[rows, i] = _exact_attention(q[rows, i], k, v, s["scale"], seen)
            return {"out": out, "lse": lse}
        ks = s["kv_start"].tolist()
        k, v = s["key"].double(), s["value"].double()
        res = {"out": out, "lse": lse}
        if case["backward"]:
            res |= {"grad_q": torch.zeros_like(q), "grad_value": torch.zeros_like(v), "grad_key": torch.zeros_like(k)}
        for b in range(case["segments"]):
            rows, keys = slice(qs[b], qs[b + 1]), slice(ks[b], ks[b + 1])
            seen = torch.ones(qs[b + 1] - qs[b], ks[b + 1] - ks[b], dtype=torch.bool, device=DEV)
            if s["mask"] is not None:
                seen &= s["mask"][keys][None]
            for i in range(h):
                j = i * hk // h
                got = _exact_attention(q[rows, i], k[keys, j], v[keys, j], s["scale"], seen, s["grad_out"][rows, i].double() if case["backward"] else None)
                out[rows, i], lse[rows, i] = got[:2]
                if case["backward"]:
                    res["grad_q"][rows, i] = got[2]
                    res["grad_key"][keys, j] += got[3]
                    res["grad_value"][keys, j] += got[4]
        return res if not case["backward"] else {n: res[n] for n in ("out", "lse", "grad_value", "grad_q", "grad_key")}
    pairs = case["pairs"]
    if case["op"] == "rotary":
        f, m, pos = s["freq"], s["magnitude"], s["positions"]
        return {"q": _exact_turn(s["q"], pos, f, m, pairs, 1), "key": _exact_turn(s["key"], pos, f, m, pairs, 1),
                "grad_q": _exact_turn(s["grad_q"], pos, f, m, pairs, -1), "grad_key": _exact_turn(s["grad_key"], pos, f, m, pairs, -1)}
    kp, vp = s["key_pages"].double(), s["value_pages"].double()
    qs, lens, page = s["q_start"].tolist(), s["kv_len"].tolist(), case["page"]
    for b in range(case["segments"]):
        n = qs[b + 1] - qs[b]
        pos = torch.arange(lens[b] - n, lens[b], device=DEV)
        key = s["key"][qs[b]:qs[b + 1]].double()
        if s["freq"] is not None:
            key = _exact_turn(s["key"][qs[b]:qs[b + 1]], pos, s["freq"], s["magnitude"], pairs, 1)
        at = s["table"][b].long()[pos // page]
        kp[at, pos % page], vp[at, pos % page] = key, s["value"][qs[b]:qs[b + 1]].double()
    return {"key_pages": kp, "value_pages": vp}

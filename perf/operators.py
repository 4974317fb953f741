"""Timed cases of the operators for several tokens per user: what is written into a key-value cache, and the partial
attention that reads it.

A case is a dict of plain values.  Every case has users, q_heads, kv_heads, head_dim, dtype, len_seed (lengths, tables and
positions belong to the case; the values come from prepare's seed) and

  entry "rotate"   rotary positions with several axes on a tensor of q_heads heads (queries, or queries and keys side by side):
                   tokens, axes, pairs (channel pairs that turn), adjacent (pairs (2j, 2j+1), else (j, j + pairs)), transposed (the
                   transposed map: the gradient)
  entry "append"   new tokens' keys (rotated on the way) and values into a cache, their queries rotated beside them:
                   new_lo..new_hi new tokens per user behind past_lo..past_hi tokens, layout, page, axes, pairs, adjacent
  entry "attend"   partial attention of each user's last new_lo..new_hi tokens over past_lo..past_hi tokens and themselves:
                   layout, page, out ("same": the inputs' type, "f32"), and what happens to the scores:
                   cap, slopes, causal, window, prefix (0 or the most tokens of a prefix that every query sees), documents (mean
                   length of the documents that the sequence is made of, 0: none)

  layout    "hnd" [user][head][capacity][d] | "nhd" [user][capacity][head][d] | "paged_hnd" [page][head][token][d] | "paged_nhd"
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
MOST_SCORES = 1.6e9      # of a drawn case: users * tokens * keys * query heads with every user as long as the longest
MOST_CACHE = 5.0e5       # tokens of a drawn case's caches
MOST_ROTATED = 1.0e6     # tokens * heads of a drawn rotation or append


def _rotate(name, tokens, heads, d, dtype, axes=3, pairs=0, adjacent=False, transposed=False, len_seed=1):
    return {"name": name, "entry": "rotate", "users": 1, "q_heads": heads, "kv_heads": 0, "head_dim": d, "dtype": dtype, "tokens": tokens,
            "axes": axes, "pairs": pairs or d // 2, "adjacent": adjacent, "transposed": transposed, "len_seed": len_seed}


def _append(name, users, heads, dtype, layout, new, past, page=0, axes=1, pairs=0, adjacent=False, len_seed=1):
    return {"name": name, "entry": "append", "users": users, "q_heads": heads[0], "kv_heads": heads[1], "head_dim": heads[2], "dtype": dtype,
            "layout": layout, "page": page, "new_lo": new[0], "new_hi": new[1], "past_lo": past[0], "past_hi": past[1], "axes": axes,
            "pairs": pairs or heads[2] // 2, "adjacent": adjacent, "len_seed": len_seed}


def _attend(name, users, heads, dtype, layout, new, past, page=0, out="same", cap=0.0, slopes=False, causal=True, window=0, prefix=0,
            documents=0, len_seed=1):
    return {"name": name, "entry": "attend", "users": users, "q_heads": heads[0], "kv_heads": heads[1], "head_dim": heads[2], "dtype": dtype,
            "layout": layout, "page": page, "new_lo": new[0], "new_hi": new[1], "past_lo": past[0], "past_hi": past[1], "out": out,
            "cap": cap, "slopes": slopes, "causal": causal, "window": window, "prefix": prefix, "documents": documents, "len_seed": len_seed}


def listed():
    b8, b70, b1, tiny = (32, 8, 128), (64, 8, 128), (32, 8, 64), (8, 8, 64)     # Llama-3-8B, Llama-3-70B and 1B-class attention shapes, fp32's
    return [
        # a prompt of a few words around one small image (16 x 16 patches): launches and latency only
        _rotate("rotate_image_bf16", 259, 32, 128, "bf16"),
        # a video's tokens (time, height, width), queries and keys of a layer side by side
        _rotate("rotate_video_bf16", 20240, 40, 128, "bf16"),
        # the gradient of a partial rotation with adjacent pairs, fp32
        _rotate("rotate_grad_f32", 5003, 24, 64, "f32", axes=2, pairs=24, adjacent=True, transposed=True),
        # a decode step's new tokens into token-major pages
        _append("append_step32_paged_bf16", 32, b8, "bf16", "paged_nhd", (1, 1), (512, 4096), page=16),
        # prompts of odd lengths, some of them with a cached beginning
        _append("append_prompts_f16", 8, b1, "f16", "hnd", (512, 4096), (0, 300), pairs=16, adjacent=True),
        # one user's single token, capped scores: latency
        _attend("token1_cap_bf16", 1, b8, "bf16", "hnd", (1, 1), (1531, 1531), out="f32", cap=50.0),
        # a decode step of the headline batch in token-major pages, bias by distance, partials for a merge
        _attend("tokens16_slopes_paged_bf16", 16, b8, "bf16", "paged_nhd", (1, 1), (512, 4096), page=16, out="f32", slopes=True),
        # a decode step over long prompts, capped scores
        _attend("tokens24_long_cap_f16", 24, b70, "f16", "hnd", (1, 1), (8192, 32768), cap=30.0),
        # six proposed tokens per user checked at once (speculative decoding), partials for a merge
        _attend("verify24_bf16", 24, b8, "bf16", "paged_hnd", (6, 6), (900, 8000), page=64, out="f32"),
        # prompts of odd lengths in one batch, capped scores
        _attend("prompts4_cap_bf16", 4, b8, "bf16", "hnd", (900, 4096), (0, 0), cap=50.0),
        # a chunk of a long prompt of packed documents behind what is cached already: the largest product
        _attend("chunk_documents_bf16", 1, b8, "bf16", "nhd", (8192, 8192), (8192, 8192), documents=9000),
        # fp32: two prompts whose first tokens see each other, windows behind them
        _attend("prefix_window_f32", 2, tiny, "f32", "hnd", (500, 1100), (0, 64), window=300, prefix=200),
    ]


def draw(rng):
    """Another case of the same ranges."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    heads = rng.choice([(8, 8, 64), (32, 8, 64), (32, 8, 128), (32, 8, 128), (64, 8, 128), (24, 24, 64), (14, 2, 64), (16, 1, 128)])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    seed = rng.randrange(1 << 30)
    entry = rng.choice(["rotate", "append", "attend", "attend", "attend"])
    axes = rng.choice([1, 2, 3])
    pairs = rng.choice([heads[2] // 2, heads[2] // 2, heads[2] // 4, 8])
    adjacent = rng.random() < 0.3
    layout = rng.choice(["hnd", "hnd", "nhd", "paged_hnd", "paged_nhd"])
    page = rng.choice([16, 32, 64, 128]) if layout.startswith("paged") else 0
    if entry == "rotate":
        tokens = log_int(1, MOST_ROTATED / heads[0])
        return dict(_rotate("", tokens, heads[0], heads[2], dtype, axes, pairs, adjacent, rng.random() < 0.3, seed))
    form = rng.choice(["token", "few", "prompt"])
    users = log_int(1, 64 if form == "prompt" else 256)
    if form == "token":
        new, past = (1, 1), log_int(1, 60000)
    elif form == "few":
        new, past = (rng.choice([0, 1, 2]), rng.randint(2, 12)), log_int(1, 20000)
    else:
        most = log_int(16, 6000)
        new, past = (max(1, most // rng.choice([1, 3, 10])), most), rng.choice([0, 0, log_int(1, 6000)])
    past = (past // rng.choice([1, 2, 8]), past)
    if entry == "append":
        past = (min(past[0], 4000), min(past[1], 4000))
        users = max(1, min(users, int(MOST_ROTATED / (heads[0] + 2 * heads[1]) / new[1]), int(MOST_CACHE / (new[1] + past[1]))))
        return _append("", users, heads, dtype, layout, new, past, page, axes, pairs, adjacent, seed)
    keys = new[1] + past[1]
    users = max(1, min(users, int(MOST_CACHE / keys), int(MOST_SCORES / (new[1] * keys * heads[0]))))
    causal = rng.random() < 0.8
    return _attend("", users, heads, dtype, layout, new, past, page, rng.choice(["same", "f32"]) if form != "prompt" else "same",
                   rng.choice([0.0, 0.0, 30.0, 50.0]), rng.random() < 0.3, causal, rng.choice([0, 0, 0, log_int(1, 2 * keys)]),
                   rng.choice([0, 0, 0, log_int(1, keys)]) if causal else 0, rng.choice([0, 0, 0, log_int(8, 2 * keys)]), seed)


def _lens(case):
    """New and held tokens per user (held: the new ones among them)."""
    r = np.random.default_rng([case["len_seed"], 7])
    n = case["users"]
    new = r.integers(case["new_lo"], case["new_hi"], n, endpoint=True)
    new[0] = max(1, new[0])      # (a call without any token is no work)
    return new.astype(np.int32), (new + r.integers(case["past_lo"], case["past_hi"], n, endpoint=True)).astype(np.int32)


def _positions(case, tokens):
    """[axes, tokens]: text runs (all axes alike) and frames or images between them (one axis per direction)."""
    r = np.random.default_rng([case["len_seed"], 13])
    at, out, axes = int(r.integers(0, 1000)), np.empty((3, tokens), np.int64), case["axes"]
    done = 0
    while done < tokens:
        h, w, t = (int(x) for x in r.integers(8, 40, 3))
        text = int(r.integers(1, 200))
        for grid in ((text,), (t, h, w)):
            n = min(tokens - done, int(np.prod(grid)))
            if len(grid) == 1:
                out[:, done:done + n] = at + np.arange(n)
            else:
                out[:, done:done + n] = at + np.stack([x.ravel() for x in np.indices(grid)])[:, :n]
            done, at = done + n, at + max(grid)
    return torch.from_numpy(out[:axes].astype(np.int32)).to(DEVICE)


def _pair_axis(case):
    """The axis of each pair: sections for time, height, width."""
    return np.array([j * case["axes"] // case["pairs"] for j in range(case["pairs"])], np.uint8)


def _inv_freq(case):
    return torch.pow(500000.0, -torch.arange(case["pairs"], dtype=torch.float64) / case["pairs"]).float().to(DEVICE)


def _slopes(case):
    n = case["q_heads"]
    return torch.pow(2.0, -8.0 * (torch.arange(n, dtype=torch.float64) + 1) / n).float().to(DEVICE)


def _masks(case):
    """Per user: the prefix's length (or None), and the ranges [lo, hi) of positions that each new token's document covers (or None)."""
    r = np.random.default_rng([case["len_seed"], 17])
    new, held = _lens(case)
    prefix = r.integers(0, case["prefix"], len(new), endpoint=True).astype(np.int32) if case["prefix"] else None
    ranges = None
    if case["documents"]:
        parts = []
        for n, l in zip(new, held):
            ends = np.cumsum(r.integers(1, 2 * case["documents"], 2 + 2 * int(l) // case["documents"] + 8, endpoint=True))
            ends = np.unique(np.append(ends[ends < l], l))
            which = np.searchsorted(ends, np.arange(l - n, l), side="right")
            parts.append(np.stack([np.concatenate([[0], ends])[which], ends[np.minimum(which, len(ends) - 1)]], 1))
        ranges = np.concatenate(parts).astype(np.int32).reshape(-1, 2)
    return prefix, ranges


def _cache(case, gen, held):
    """K and V storage (random), the block table (None unless paged), and what a view of it takes."""
    n, H, d, dt, page = case["users"], case["kv_heads"], case["head_dim"], DTYPES[case["dtype"]], case["page"]
    if page:
        pages = [-(-int(x) // page) for x in held]
        total, width = sum(pages) + 3, max(1, max(pages))
        order, at = np.random.default_rng([case["len_seed"], 19]).permutation(total).astype(np.int32), 0
        table = np.zeros((n, width), np.int32)
        for u, p in enumerate(pages):
            table[u, :p] = order[at:at + p]
            at += p
        table = torch.from_numpy(table).to(DEVICE)
        head_major = case["layout"] == "paged_hnd"
        shape = (total, H, page, d) if head_major else (total, page, H, d)
        strides = (d, page * d) if head_major else (H * d, d)
    else:
        cap, table = max(64, -(-int(held.max(initial=0)) // 64) * 64), None
        head_major = case["layout"] == "hnd"
        shape = (n, H, cap, d) if head_major else (n, cap, H, d)
        strides = (d, cap * d) if head_major else (H * d, d)
    k, v = (torch.randn(shape, generator=gen, device=DEVICE, dtype=dt) for _ in range(2))
    return {"k": k, "v": v, "table": table, "strides": strides, "head_major": head_major}


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    dt, Hq, H, d = DTYPES[case["dtype"]], case["q_heads"], case["kv_heads"], case["head_dim"]
    s = {"case": case}
    if case["entry"] == "rotate":
        s["x"] = torch.randn((case["tokens"], Hq, d), generator=gen, device=DEVICE, dtype=dt)
        tokens = case["tokens"]
    else:
        new, held = _lens(case)
        tokens = int(new.sum())
        s |= {"new": new, "held": held, "new_dev": torch.from_numpy(new).to(DEVICE).long(), "held_dev": torch.from_numpy(held).to(DEVICE).long()}
        s |= _cache(case, gen, held)
    if case["entry"] == "append":      # what a layer's projection leaves: the heads of q, k and v side by side
        s["qkv"] = torch.randn((tokens, Hq + 2 * H, d), generator=gen, device=DEVICE, dtype=dt)
    if case["entry"] == "attend":
        s["q"] = torch.randn((tokens, Hq, d), generator=gen, device=DEVICE, dtype=dt) * (3.0 if case["cap"] else 1.0)
        prefix, ranges = _masks(case)
        s["prefix"], s["prefix_dev"] = prefix, None if prefix is None else torch.from_numpy(prefix).to(DEVICE).long()
        s["ranges"] = None if ranges is None else torch.from_numpy(ranges).to(DEVICE)
        s["slopes"] = _slopes(case) if case["slopes"] else None
    else:
        s |= {"positions": _positions(case, tokens), "pair_axis": _pair_axis(case), "inv_freq": _inv_freq(case)}
        s["pair_axis_dev"] = torch.from_numpy(s["pair_axis"]).to(DEVICE).long()
    return s


# The plain forms

def _turn(s, x):
    """Rotary positions on x [tokens, heads, d], in 32 bits; angles, cosines and sines in 64."""
    case, P = s["case"], s["case"]["pairs"]
    angle = s["positions"][s["pair_axis_dev"]].t().double() * s["inv_freq"].double()
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if case.get("transposed"):
        sin = -sin
    f, y = x.float(), x.float()
    a, b = (f[..., 0:2 * P:2], f[..., 1:2 * P:2]) if case["adjacent"] else (f[..., :P], f[..., P:2 * P])
    first, second = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([first, second], -1).flatten(-2) if case["adjacent"] else torch.cat([first, second], -1)
    return torch.cat([turned, y[..., 2 * P:]], -1).to(x.dtype)


def _token_places(s):
    """For every new token: its user, and its place in the user's cache."""
    n = s["new_dev"]
    user = torch.repeat_interleave(torch.arange(len(n), device=DEVICE), n, output_size=int(s["new"].sum()))
    first = torch.cumsum(n, 0) - n
    return user, torch.arange(len(user), device=DEVICE) - first[user] + (s["held_dev"] - n)[user]


def _plain_append(s):
    case, Hq, H = s["case"], s["case"]["q_heads"], s["case"]["kv_heads"]
    turned = _turn(s, s["qkv"][:, :Hq + H])
    user, at = _token_places(s)
    if case["page"]:
        page, at = s["table"].long()[user, at // case["page"]], at % case["page"]
    else:
        page = user
    for cache, rows in ((s["k"], turned[:, Hq:]), (s["v"], s["qkv"][:, Hq + H:])):
        if s["head_major"]:
            cache[page, :, at] = rows
        else:
            cache[page, at] = rows
    return turned[:, :Hq].contiguous(), s["k"], s["v"]


def _padded_cache(s, cache):
    """[users, kv_heads, longest, d] in 32 bits."""
    case, longest = s["case"], int(s["held"].max())
    if case["page"]:
        x = cache[s["table"].long()]      # [users, pages, ...]
        x = x.transpose(1, 2).flatten(2, 3) if s["head_major"] else x.flatten(1, 2).transpose(1, 2)
    else:
        x = cache if s["head_major"] else cache.transpose(1, 2)
    x = x[:, :, :longest].float()
    return torch.where((torch.arange(longest, device=DEVICE) < s["held_dev"][:, None])[:, None, :, None], x, 0.0).contiguous()


def _plain_attend(s):
    case = s["case"]
    U, Hq, H, d = case["users"], case["q_heads"], case["kv_heads"], case["head_dim"]
    G, most, longest, dt = Hq // H, int(s["new"].max()), int(s["held"].max()), DTYPES[case["dtype"]]
    user, at = _token_places(s)
    row = at - (s["held_dev"] - s["new_dev"])[user]
    q = torch.zeros((U, most, Hq, d), device=DEVICE)
    q[user, row] = s["q"].float()
    q = q.view(U, most, H, G, d).permute(0, 2, 3, 1, 4).reshape(U, H, G * most, d).contiguous()
    k, v = _padded_cache(s, s["k"]), _padded_cache(s, s["v"])
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).view(U, H, G, most, longest)
    x *= 1.0 / math.sqrt(d)
    if case["cap"]:
        x = torch.tanh(x / case["cap"]) * case["cap"]
    key = torch.arange(longest, device=DEVICE)
    place = (s["held_dev"] - s["new_dev"])[:, None] + torch.arange(most, device=DEVICE)      # [users, most]
    apart = place[:, :, None] - key
    if case["slopes"]:
        x -= s["slopes"].view(H, G, 1, 1) * apart.abs()[:, None, None].float()
    seen = torch.ones_like(apart, dtype=torch.bool)
    if case["causal"]:
        seen &= apart >= 0
    if case["window"]:
        seen &= apart.abs() < case["window"]
    if s["prefix"] is not None:
        seen |= key < s["prefix_dev"][:, None, None]
    if s["ranges"] is not None:
        r = torch.zeros((U, most, 2), device=DEVICE, dtype=torch.int64)
        r[user, row] = s["ranges"].long()
        seen &= (key >= r[..., :1]) & (key < r[..., 1:])
    seen &= key < s["held_dev"][:, None, None]
    x.masked_fill_(~seen[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    x = (x - top).exp_()
    total = x.sum(-1, keepdim=True)
    a = torch.matmul(x.view(U, H, G * most, longest), v).view(U, H, G, most, d) / torch.where(total == 0, 1.0, total)
    lse = (total.log() + top)[..., 0]
    a = a.permute(0, 3, 1, 2, 4).reshape(U, most, Hq, d)[user, row]
    return a.to(torch.float32 if case["out"] == "f32" else dt), lse.permute(0, 3, 1, 2).reshape(U, most, Hq)[user, row].contiguous()


# The framework's calls

_context = None


def _ctx():
    """A serving process keeps one library context; views come and go."""
    global _context
    if _context is None:
        import paper_2409_19134_amd as spd
        _context = spd.Context(0)
    return _context


def _calls(s):
    """What a user's program keeps beside its tensors: a view of the cache, the rotation's or the scores' description, its result buffers."""
    import paper_2409_19134_amd as spd
    case, dt = s["case"], DTYPES[s["case"]["dtype"]]
    Hq, H, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    c = {"ctx": _ctx()}
    if case["entry"] != "rotate":
        c["shape"] = spd.make_shape(dt, Hq, H, d, 1.0 / math.sqrt(d))
        if case["page"]:
            c["view"] = spd.KVView(s["held"], *s["strides"], k_pool=s["k"], v_pool=s["v"], block_table=s["table"], block_size=case["page"],
                                   block_stride=H * case["page"] * d)
        else:
            c["view"] = spd.KVView(s["held"], *s["strides"], k=list(s["k"]), v=list(s["v"]))
    if case["entry"] == "attend":
        c["score"] = spd.Score(cap=case["cap"], slopes=s["slopes"], causal=case["causal"], window=case["window"], prefix=s["prefix"],
                               ranges=s["ranges"])
        c["out"] = torch.empty(s["q"].shape, device=DEVICE, dtype=torch.float32 if case["out"] == "f32" else dt)
        c["lse"] = torch.empty(s["q"].shape[:2], device=DEVICE)
    else:
        c["rope"] = spd.Rope(s["inv_freq"], n_axes=case["axes"], pair_axis=s["pair_axis"], adjacent=case["adjacent"])
        x = s["x"] if case["entry"] == "rotate" else s["qkv"][:, :Hq]
        c["y"] = torch.empty(x.shape, device=DEVICE, dtype=dt)
    return c


def run(s):
    case = s["case"]
    if own:
        if "calls" not in s:
            s["calls"] = _calls(s)
        c, Hq, H = s["calls"], case["q_heads"], case["kv_heads"]
        if case["entry"] == "rotate":
            return c["ctx"].spd_rotate(c["rope"], s["x"], s["positions"], c["y"], transposed=case["transposed"])
        if case["entry"] == "append":
            qkv = s["qkv"]
            c["ctx"].spd_append_tokens(c["shape"], c["view"], s["new"], qkv[:, Hq:Hq + H], qkv[:, Hq + H:], rope=c["rope"],
                                       positions=s["positions"], q=qkv[:, :Hq], q_out=c["y"])
            return c["y"], s["k"], s["v"]
        return c["ctx"].spd_partial_attn_tokens(c["shape"], s["q"], c["view"], s["new"], c["score"], c["out"], c["lse"])
    if case["entry"] == "rotate":
        return _turn(s, s["x"])
    return _plain_append(s) if case["entry"] == "append" else _plain_attend(s)


def _seen_pairs(case):
    """(query, key) pairs that the masks leave, and keys that any query of their user sees."""
    new, held = _lens(case)
    prefix, ranges = _masks(case)
    pairs = keys = at = 0
    for u, (n, l) in enumerate(zip(new.astype(np.int64), held.astype(np.int64))):
        q = np.arange(l - n, l)
        lo, hi = (ranges[at:at + n, 0], ranges[at:at + n, 1]) if ranges is not None else (np.zeros(n, np.int64), np.full(n, l))
        at += n
        a0 = np.maximum(lo, q - case["window"] + 1) if case["window"] else lo
        a1 = np.minimum(hi, q + 1 if case["causal"] else q + case["window"] if case["window"] else hi)
        b1 = np.minimum(hi, prefix[u]) if prefix is not None else lo
        a, b = np.maximum(a1 - a0, 0), np.maximum(b1 - lo, 0)
        both = np.maximum(np.minimum(a1, b1) - np.maximum(a0, lo), 0)
        pairs += int((a + b - both).sum())
        mark = np.zeros(int(l) + 1, np.int64)
        for i0, i1, size in ((a0, a1, a), (lo, b1, b)):
            np.add.at(mark, i0[size > 0], 1)
            np.add.at(mark, i1[size > 0], -1)
        keys += int((np.cumsum(mark) > 0).sum())
    return pairs, keys


def work(case):
    es, Hq, H, d = 4 if case["dtype"] == "f32" else 2, case["q_heads"], case["kv_heads"], case["head_dim"]
    if case["entry"] == "rotate":
        T, P = case["tokens"], case["pairs"]
        return {"bytes": 2 * T * Hq * d * es + T * case["axes"] * 4 + P * 4, "flops": 6 * T * Hq * P}
    tokens = int(_lens(case)[0].sum())
    if case["entry"] == "append":
        return {"bytes": 2 * tokens * (Hq + 2 * H) * d * es + tokens * case["axes"] * 4, "flops": 6 * tokens * (Hq + H) * case["pairs"]}
    pairs, keys = _seen_pairs(case)
    eo = 4 if case["out"] == "f32" else es
    return {"bytes": keys * 2 * H * d * es + tokens * Hq * (d * (es + eo) + 4), "flops": pairs * Hq * d * 4}


# From the definitions in 64 bits: token by token's angles as complex numbers, attention user by user and head by head

def _exact_turn(case, x, s):
    P = case["pairs"]
    z = torch.polar(torch.ones((), device=DEVICE, dtype=torch.float64),
                    s["inv_freq"].double()[None] * s["positions"].double().t()[:, s["pair_axis_dev"]])[:, None]
    y = x.double().clone()
    i, j = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if case["adjacent"] else (slice(0, P), slice(P, 2 * P))
    w = torch.complex(y[..., i], y[..., j]) * (z.conj() if case.get("transposed") else z)
    y[..., i], y[..., j] = w.real, w.imag
    return y


def _user_rows(case, s, cache, u):
    """A user's tokens [kv_heads, held, d] (a view where the storage allows it)."""
    n = int(s["held"][u])
    if not case["page"]:
        x = cache[u] if s["head_major"] else cache[u].transpose(0, 1)
        return x[:, :n]
    ids = s["table"][u, :-(-n // case["page"])].long()
    x = cache[ids]
    x = x.transpose(0, 1) if s["head_major"] else x.permute(2, 0, 1, 3)
    return x.reshape(case["kv_heads"], -1, case["head_dim"])[:, :n]


def exact(case, seed):
    s = prepare(case, seed)
    if case["entry"] == "rotate":
        return _exact_turn(case, s["x"], s)
    Hq, H, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    if case["entry"] == "append":
        if s["k"].numel() > 4e8:
            return None
        qkv = s["qkv"]
        k, v, at = s["k"].double(), s["v"].double(), 0
        rows_k = _exact_turn(case, qkv[:, Hq:Hq + H], s)
        for u, (n, l) in enumerate(zip(s["new"].tolist(), s["held"].tolist())):
            place = torch.arange(l - n, l, device=DEVICE)
            block = s["table"][u].long()[place // case["page"]] if case["page"] else torch.full_like(place, u)
            place = place % case["page"] if case["page"] else place
            for cache, rows in ((k, rows_k), (v, qkv[:, Hq + H:].double())):
                if s["head_major"]:
                    cache.transpose(1, 2).index_put_((block, place), rows[at:at + n])
                else:
                    cache.index_put_((block, place), rows[at:at + n])
            at += n
        return _exact_turn(case, qkv[:, :Hq], s), k, v
    G, at = Hq // H, 0
    a = torch.zeros(s["q"].shape, device=DEVICE, dtype=torch.float64)
    lse = torch.full(s["q"].shape[:2], -math.inf, device=DEVICE, dtype=torch.float64)
    for u, (n, l) in enumerate(zip(s["new"].tolist(), s["held"].tolist())):
        if n == 0:
            continue
        K, V = _user_rows(case, s, s["k"], u), _user_rows(case, s, s["v"], u)
        apart = torch.arange(l - n, l, device=DEVICE)[:, None] - torch.arange(l, device=DEVICE)[None]
        key = torch.arange(l, device=DEVICE)[None]
        hidden = torch.zeros((n, l), device=DEVICE, dtype=torch.bool)
        if case["causal"]:
            hidden |= apart < 0
        if case["window"]:
            hidden |= apart.abs() >= case["window"]
        if s["prefix"] is not None:
            hidden &= key >= int(s["prefix"][u])
        if s["ranges"] is not None:
            r = s["ranges"][at:at + n]
            hidden |= (key < r[:, :1]) | (key >= r[:, 1:])
        for h in range(Hq):
            x = s["q"][at:at + n, h].double() @ K[h // G].double().t().contiguous() / math.sqrt(d)
            if case["cap"]:
                x = case["cap"] * torch.tanh(x / case["cap"])
            if s["slopes"] is not None:
                x -= s["slopes"][h].double() * apart.abs().double()
            x[hidden] = -math.inf
            total = torch.logsumexp(x, 1)
            lse[at:at + n, h] = total
            a[at:at + n, h] = torch.nan_to_num(torch.exp(x - total[:, None]), nan=0.0) @ V[h // G].double()
        at += n
    return a, lse

"""Timed cases of the operators for trees of drafted tokens and for the caches they leave behind: the tree's sets of ancestors, the partial attention of
a tree's tokens over a cache, the tokens that are kept afterwards, and copies of pages for users that fork.

A case is a dict of plain values.  Every case has entry and len_seed (lengths, trees, tables, lists and places belong to the case; the values come from
prepare's seed) and

  entry "plan"    from every drafted token's parent the set of drafted tokens that it sees, its depth and its position: users, new_lo..new_hi tokens per
                  user, words (of 64 bits) of a set
  entry "attend"  partial attention of each user's new_lo..new_hi drafted tokens over past_lo..past_hi tokens, and (inside) over those drafted tokens that
                  lie on their branch, which are the last of the same cache; not inside: the cache is the other owner's and holds none of them:
                  users, q_heads, kv_heads, head_dim, dtype, layout, page, words, out ("same": the inputs' type, "f32"), and what happens to the scores:
                  cap, slopes, window, prefix (0 or the most tokens of a prefix that every query sees)
  entry "keep"    some of the last new_lo..new_hi tokens of every user's cache, moved together behind the past_lo..past_hi tokens in front of them, in
                  all layers: users, kv_heads, head_dim, dtype, layers, layout, page, keep_lo..keep_hi (how many; of new_lo..new_hi at most), sinks (that
                  many of them are the first ones, in place)
  entry "pages"   copies of pages in all layers' pools: kv_heads, head_dim, dtype, layers, layout, page, pairs, partial (only as many tokens of each page
                  as the fork holds there)

  layout    "hnd" [user][head][capacity][d] | "nhd" [user][capacity][head][d] | "paged_hnd" [page][head][token][d] | "paged_nhd"
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
MOST_SCORES = 3.8e8      # of a drawn case: users * tokens * keys * query heads with every user as long as the longest (fp32: a sixth)
MOST_CACHE = 1.5e5       # tokens of a drawn case's caches (fp32: half)
MOST_MOVED = 2.0e8       # bytes of a drawn case's caches or pages


def _plan(name, users, new, words, len_seed=1):
    return {"name": name, "entry": "plan", "users": users, "new_lo": new[0], "new_hi": new[1], "words": words, "len_seed": len_seed}


def _attend(name, users, heads, dtype, layout, new, past, words=1, page=0, out="same", inside=True, cap=0.0, slopes=False, window=0, prefix=0, len_seed=1):
    return {"name": name, "entry": "attend", "users": users, "q_heads": heads[0], "kv_heads": heads[1], "head_dim": heads[2], "dtype": dtype,
            "layout": layout, "page": page, "words": words, "new_lo": new[0], "new_hi": new[1], "past_lo": past[0], "past_hi": past[1], "out": out,
            "inside": inside, "cap": cap, "slopes": slopes, "window": window, "prefix": prefix, "len_seed": len_seed}


def _keep(name, users, heads, dtype, layers, layout, new, past, keep, sinks=0, page=0, len_seed=1):
    return {"name": name, "entry": "keep", "users": users, "kv_heads": heads[1], "head_dim": heads[2], "dtype": dtype, "layers": layers, "layout": layout,
            "page": page, "new_lo": new[0], "new_hi": new[1], "past_lo": past[0], "past_hi": past[1], "keep_lo": keep[0], "keep_hi": keep[1],
            "sinks": sinks, "len_seed": len_seed}


def _pages(name, heads, dtype, layers, layout, page, pairs, partial, len_seed=1):
    return {"name": name, "entry": "pages", "kv_heads": heads[1], "head_dim": heads[2], "dtype": dtype, "layers": layers, "layout": layout, "page": page,
            "pairs": pairs, "partial": partial, "len_seed": len_seed}


def listed():
    b8, b70, b1, tiny = (32, 8, 128), (64, 8, 128), (32, 8, 64), (8, 8, 64)     # Llama-3-8B, Llama-3-70B and 1B-class attention shapes, fp32's
    return [
        # one user's draft of a few tokens: latency only
        _plan("plan_user", 1, (13, 13), 1),
        # a large batch's wide trees
        _plan("plan_users256", 256, (100, 500), 8),
        # one user's small tree over a short cache, partials for a merge: latency
        _attend("tree1_bf16", 1, b8, "bf16", "hnd", (16, 16), (1531, 1531), out="f32"),
        # drafts of a few tokens each (at most 32 rows to a KV head) for a larger batch of a small model
        _attend("tree40_few_f16", 40, b1, "f16", "paged_nhd", (4, 8), (300, 3000), page=32, out="f32"),
        # the headline batch with trees of odd sizes in token-major pages, partials for a merge
        _attend("tree16_paged_bf16", 16, b8, "bf16", "paged_nhd", (10, 26), (512, 4096), page=16, out="f32"),
        # full trees over long caches, results in the model's type
        _attend("tree24_bf16", 24, b8, "bf16", "paged_hnd", (50, 64), (900, 8000), page=64),
        # large trees over long prompts, groups of eight query heads, capped scores: the largest product
        _attend("tree8_long_cap_f16", 8, b70, "f16", "hnd", (31, 48), (8192, 32768), cap=30.0),
        # fp32: windows and distance biases by depth, trees of more than one word
        _attend("tree3_window_slopes_f32", 3, tiny, "f32", "nhd", (5, 130), (200, 1100), words=3, out="f32", slopes=True, window=300),
        # after a step of checking: the accepted branch moves together, all layers of a small model in one call
        _keep("keep_step32_bf16", 32, b8, "bf16", 8, "paged_nhd", (20, 26), (100, 500), (1, 6), page=16),
        # a cache that has grown too long keeps its first tokens and some of the others
        _keep("keep_third_f16", 3, b1, "f16", 2, "hnd", (8000, 20000), (0, 0), (2500, 6500), sinks=4),
        # every user forks once: the pages that the copies go on writing
        _pages("pages_fork32_bf16", b8, "bf16", 8, "paged_nhd", 16, 32, True),
        # pages moved to the front of the pool, or a long prompt given to another user as a copy
        _pages("pages_move_f16", b1, "f16", 2, "paged_hnd", 64, 1000, False),
    ]


def draw(rng):
    """Another case of the same ranges."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    heads = rng.choice([(8, 8, 64), (32, 8, 64), (32, 8, 128), (32, 8, 128), (64, 8, 128), (24, 24, 64), (14, 2, 64), (16, 1, 128)])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    seed = rng.randrange(1 << 30)
    entry = rng.choice(["plan", "attend", "attend", "attend", "attend", "keep", "keep", "pages"])
    layout = rng.choice(["hnd", "nhd", "paged_hnd", "paged_nhd"])
    page = rng.choice([16, 32, 64, 128]) if layout.startswith("paged") else 0
    token_bytes = 2 * heads[1] * heads[2] * (4 if dtype == "f32" else 2)
    if entry == "plan":
        most = log_int(2, 512)
        return _plan("", log_int(1, 256), (max(1, most // rng.choice([1, 2, 5])), most), rng.randint(-(-most // 64), 8), seed)
    if entry == "attend":
        most = log_int(2, 200)
        new = (rng.choice([0, 1, most // 2, most]), most)
        past = rng.choice([0, log_int(1, 30000), log_int(100, 30000), log_int(100, 30000)])
        keys = past + most
        most_scores, most_cache = (MOST_SCORES / 6, MOST_CACHE / 2) if dtype == "f32" else (MOST_SCORES, MOST_CACHE)
        users = max(1, min(log_int(1, 128), int(most_cache / keys), int(most_scores / (most * keys * heads[0]))))
        return _attend("", users, heads, dtype, layout, new, (past // rng.choice([1, 2, 8]), past), rng.randint(-(-most // 64), 4), page,
                       rng.choice(["same", "f32"]), rng.random() < 0.75, rng.choice([0.0, 0.0, 0.0, 30.0, 50.0]), rng.random() < 0.25,
                       rng.choice([0, 0, 0, log_int(1, 2 * keys)]), rng.choice([0, 0, 0, log_int(1, keys)]), seed)
    layers = rng.choice([1, 2, 4, 8])
    if entry == "pages":
        layout, page = rng.choice(["paged_hnd", "paged_nhd"]), rng.choice([16, 32, 64, 128])
        pairs = max(1, min(log_int(1, 2000), int(MOST_MOVED / (2 * page * token_bytes * layers))))
        return _pages("", heads, dtype, layers, layout, page, pairs, rng.random() < 0.5, seed)
    if rng.random() < 0.5:      # after a step of checking
        new = rng.randint(2, 64)
        new, keep, sinks, past = (rng.choice([1, new]), new), (rng.choice([0, 1]), rng.randint(1, 8)), 0, (0, log_int(1, 300))
    else:
        new = log_int(64, 20000)
        new, keep, sinks, past = (new // rng.choice([1, 3]), new), (new // 8, new // 3), rng.choice([0, 4, 16]), (0, 0)
    users = max(1, min(log_int(1, 64), int(MOST_MOVED / ((new[1] + past[1]) * token_bytes * layers))))
    return _keep("", users, heads, dtype, layers, layout, new, past, keep, sinks, page, seed)


def _lens(case):
    """Drafted (or last) tokens of every user, and tokens that its cache holds."""
    r = np.random.default_rng([case["len_seed"], 7])
    n = case["users"]
    new = r.integers(case["new_lo"], case["new_hi"], n, endpoint=True)
    new[0] = max(1, new[0])      # (a call without any token is no work)
    if case["entry"] == "plan":
        return new.astype(np.int32), r.integers(0, 100000, n).astype(np.int32)
    held = r.integers(case["past_lo"], case["past_hi"], n, endpoint=True) + (new if case.get("inside", True) else 0)
    return new.astype(np.int32), held.astype(np.int32)


def _parents(case):
    """[T]: a token's parent among its user's drafted tokens, always an earlier one; -1: it follows the cache's last token.  Level by level, as a
    draft grows: children of the tokens about a third of the way back, some chains."""
    r = np.random.default_rng([case["len_seed"], 11])
    parts = []
    for n in _lens(case)[0].tolist():
        i = np.arange(n)
        parts.append(np.where(r.random(n) < 0.25, i - 1, r.integers(np.maximum(i // 3 - 2, -1), i, n)))
    return np.concatenate(parts).astype(np.int32)


def _tree(case):
    """Sets [T, words] and depths [T], token by token: a token sees what its parent sees, and itself."""
    parents, W, at = _parents(case).tolist(), case["words"], 0
    seen, depth = [], []
    for n in _lens(case)[0].tolist():
        for i in range(n):
            p = parents[at + i]
            seen.append((seen[at + p] if p >= 0 else 0) | 1 << i)
            depth.append(depth[at + p] + 1 if p >= 0 else 0)
        at += n
    words = np.array([[x >> 64 * w & (1 << 64) - 1 for w in range(W)] for x in seen], np.uint64).reshape(-1, W)
    return words.view(np.int64), np.array(depth, np.int32)


def _kept(case):
    """[T]: of every user's last tokens first the numbers of those that are kept, and how many these are.  A kept token is in place already or
    comes from behind them all, so that a second pass finds what the first one found."""
    r = np.random.default_rng([case["len_seed"], 23])
    lists, counts = [], []
    for n in _lens(case)[0].tolist():
        m = min(int(r.integers(case["keep_lo"], case["keep_hi"], endpoint=True)), n)
        stay = min(m, case["sinks"] or int(r.integers(0, m, endpoint=True)))
        m = min(m, stay + n // 2 - m // 2)
        far = np.sort(r.permutation(np.arange(m, n))[:m - stay])
        m = stay + len(far)
        lists.append(np.concatenate([np.arange(stay), far, np.full(n - m, -1)]))
        counts.append(m)
    return np.concatenate(lists).astype(np.int32), np.array(counts, np.int32)


def _caches(case, gen, held, layers):
    """Every layer's K and V storage (random), the block table (None unless paged), and what a view of them takes."""
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
    k, v = ([torch.randn(shape, generator=gen, device=DEVICE, dtype=dt) for _ in range(layers)] for _ in range(2))
    return {"k": k, "v": v, "table": table, "strides": strides, "head_major": head_major}


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    s = {"case": case}
    if case["entry"] == "pages":
        H, d, page, pairs = case["kv_heads"], case["head_dim"], case["page"], case["pairs"]
        r = np.random.default_rng([case["len_seed"], 29])
        total = 2 * pairs + 5
        order = r.permutation(total).astype(np.int32)
        s["pairs"] = torch.from_numpy(np.stack([order[:pairs], order[pairs:2 * pairs]], 1)).to(DEVICE).contiguous()
        tokens = r.integers(1, page, pairs, endpoint=True).astype(np.int32) if case["partial"] else np.full(pairs, page, np.int32)
        s["tokens"] = torch.from_numpy(tokens).to(DEVICE)
        s["head_major"] = case["layout"] == "paged_hnd"
        shape = (total, H, page, d) if s["head_major"] else (total, page, H, d)
        s["strides"] = (d, page * d) if s["head_major"] else (H * d, d)
        s["k"], s["v"] = ([torch.randn(shape, generator=gen, device=DEVICE, dtype=DTYPES[case["dtype"]]) for _ in range(case["layers"])] for _ in range(2))
        return s
    new, held = _lens(case)
    tokens = int(new.sum())
    s |= {"new": new, "held": held, "new_dev": torch.from_numpy(new).to(DEVICE).long(), "held_dev": torch.from_numpy(held).to(DEVICE).long()}
    if case["entry"] == "plan":      # (another seed's trees: another user's draft behind the same cache)
        shift = int(np.random.default_rng([case["len_seed"], int(seed)]).integers(0, 50000))
        s["parents"], s["held"] = torch.from_numpy(_parents(case)).to(DEVICE), held + np.int32(shift)
        s["held_dev"] = torch.from_numpy(s["held"]).to(DEVICE).long()
        return s
    s |= _caches(case, gen, held, case.get("layers", 1))
    if case["entry"] == "keep":
        keep, count = _kept(case)
        s["keep"], s["count"] = torch.from_numpy(keep).to(DEVICE), torch.from_numpy(count).to(DEVICE)
        return s
    seen, depth = _tree(case)
    s["seen"], s["depth"] = torch.from_numpy(seen).to(DEVICE), torch.from_numpy(depth).to(DEVICE)
    s["q"] = torch.randn((tokens, case["q_heads"], case["head_dim"]), generator=gen, device=DEVICE, dtype=DTYPES[case["dtype"]]) * (3.0 if case["cap"] else 1.0)
    r = np.random.default_rng([case["len_seed"], 17])
    s["prefix"] = r.integers(0, case["prefix"], case["users"], endpoint=True).astype(np.int32) if case["prefix"] else None
    s["prefix_dev"] = torch.from_numpy(s["prefix"]).to(DEVICE).long() if case["prefix"] else None
    n = case["q_heads"]
    s["slopes"] = torch.pow(2.0, -8.0 * (torch.arange(n, dtype=torch.float64) + 1) / n).float().to(DEVICE) if case["slopes"] else None
    return s


# The plain forms

def _rows(s):
    """For every token of the ragged list: its user, and its number among the user's."""
    n = s["new_dev"]
    user = torch.repeat_interleave(torch.arange(len(n), device=DEVICE), n, output_size=int(s["new"].sum()))
    return user, torch.arange(len(user), device=DEVICE) - (torch.cumsum(n, 0) - n)[user]


def _plain_plan(s):
    """Whom a token sees, by squaring: its parent's step taken once, twice, four times, ..."""
    W, most = s["case"]["words"], int(s["new"].max())
    user, row = _rows(s)
    reach = torch.zeros((len(s["new"]), most, most), device=DEVICE)
    has = s["parents"] >= 0
    reach[user[has], row[has], s["parents"].long()[has]] = 1.0
    reach += torch.eye(most, device=DEVICE)
    for _ in range(max(1, (most - 1).bit_length())):
        reach = (torch.matmul(reach, reach) > 0).float()
    mine = reach[user, row]
    depth = mine.sum(1).to(torch.int32) - 1
    bits = torch.zeros((len(user), 64 * W), device=DEVICE, dtype=torch.int64)
    bits[:, :most] = mine.long()
    seen = (bits.view(-1, W, 64) << torch.arange(64, device=DEVICE)).sum(2)
    return seen, depth, (s["held_dev"][user] + depth).to(torch.int32)


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
    if longest == 0:
        return (torch.zeros(s["q"].shape, device=DEVICE, dtype=torch.float32 if case["out"] == "f32" else dt),
                torch.full(s["q"].shape[:2], -math.inf, device=DEVICE))
    user, row = _rows(s)
    begin = s["held_dev"] - (s["new_dev"] if case["inside"] else 0)      # where the tree begins, as a position and as a place
    q = torch.zeros((U, most, Hq, d), device=DEVICE)
    q[user, row] = s["q"].float()
    q = q.view(U, most, H, G, d).permute(0, 2, 3, 1, 4).reshape(U, H, G * most, d).contiguous()
    k, v = _padded_cache(s, s["k"][0]), _padded_cache(s, s["v"][0])
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).view(U, H, G, most, longest)
    x *= 1.0 / math.sqrt(d)
    if case["cap"]:
        x = torch.tanh(x / case["cap"]) * case["cap"]
    depth = torch.zeros((U, most), device=DEVICE, dtype=torch.int64)
    depth[user, row] = s["depth"].long()
    key = torch.arange(longest, device=DEVICE)
    drafted = key - begin[:, None]      # [users, keys]: the drafted token that lies there, if not negative
    node = drafted.clamp(0, most - 1)
    place = torch.where(drafted >= 0, begin[:, None] + depth.gather(1, node), key) if case["inside"] else key.expand(U, longest)
    apart = (begin[:, None] + depth)[:, :, None] - place[:, None]      # [users, most, keys]
    if case["slopes"]:
        x -= s["slopes"].view(H, G, 1, 1) * apart.abs()[:, None, None].float()
    seen = torch.ones_like(apart, dtype=torch.bool)
    if case["window"]:
        seen &= apart.abs() < case["window"]
    if s["prefix"] is not None:
        seen |= (key < s["prefix_dev"][:, None, None]) & ((drafted < 0)[:, None] if case["inside"] else True)
    if case["inside"]:
        sets = torch.zeros((U, most, case["words"]), device=DEVICE, dtype=torch.int64)
        sets[user, row] = s["seen"]
        branch = (sets.gather(2, (node // 64)[:, None].expand(U, most, longest)) >> (node % 64)[:, None]) & 1
        seen &= (drafted < 0)[:, None] | (branch == 1)
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


def _plain_keep(s):
    """All kept rows are read before any is written."""
    case = s["case"]
    user, row = _rows(s)
    kept = torch.nonzero(row < s["count"][user])[:, 0]
    u, first = user[kept], (s["held_dev"] - s["new_dev"])[user[kept]]
    to, frm = first + row[kept], first + s["keep"].long()[kept]
    if case["page"]:
        B, table = case["page"], s["table"].long()
        pages, to, frm = (table[u, to // B], table[u, frm // B]), to % B, frm % B
    else:
        pages = (u, u)
    for cache in s["k"] + s["v"]:
        x = cache.transpose(1, 2) if s["head_major"] else cache
        x[pages[0], to] = x[pages[1], frm]
    return s["k"], s["v"]


def _plain_pages(s):
    case, pairs = s["case"], s["pairs"].long()
    moved = torch.arange(case["page"], device=DEVICE) < s["tokens"][:, None]
    which, at = torch.nonzero(moved, as_tuple=True)
    for pool in s["k"] + s["v"]:
        if not case["partial"]:
            pool[pairs[:, 1]] = pool[pairs[:, 0]]
            continue
        x = pool.transpose(1, 2) if s["head_major"] else pool
        x[pairs[which, 1], at] = x[pairs[which, 0], at]
    return s["k"], s["v"]


# The framework's calls

_context = None


def _ctx():
    """A serving process keeps one library context; views come and go."""
    global _context
    if _context is None:
        import paper_2409_19134_amd as spd
        _context = spd.Context(0)
    return _context


def _views(s, spd):
    case = s["case"]
    if case["page"]:
        table = s["table"] if "table" in s else None
        return [spd.KVView(s["held"] if "held" in s else [], *s["strides"], k_pool=k, v_pool=v, block_table=table, block_size=case["page"],
                           block_stride=case["kv_heads"] * case["page"] * case["head_dim"]) for k, v in zip(s["k"], s["v"])]
    return [spd.KVView(s["held"], *s["strides"], k=list(k), v=list(v)) for k, v in zip(s["k"], s["v"])]


def _calls(s):
    """What a user's program keeps beside its tensors: views of its layers' caches, the scores' description, its result buffers."""
    import paper_2409_19134_amd as spd
    case = s["case"]
    c = {"ctx": _ctx()}
    if case["entry"] == "plan":
        c["tree"] = spd.Tree(int(s["new"].sum()), case["words"], device=DEVICE)
        return c
    dt = DTYPES[case["dtype"]]
    c["shape"] = spd.make_shape(dt, case.get("q_heads", case["kv_heads"]), case["kv_heads"], case["head_dim"], 1.0 / math.sqrt(case["head_dim"]))
    c["views"] = _views(s, spd)
    if case["entry"] == "attend":
        c["tree"] = spd.Tree.of(s["seen"], s["depth"])
        c["score"] = spd.Score(cap=case["cap"], slopes=s["slopes"], window=case["window"], prefix=s["prefix"],
                               q_pos=None if case["inside"] else s["held"])
        c["out"] = torch.empty(s["q"].shape, device=DEVICE, dtype=torch.float32 if case["out"] == "f32" else dt)
        c["lse"] = torch.empty(s["q"].shape[:2], device=DEVICE)
    return c


def run(s):
    case = s["case"]
    if own:
        if "calls" not in s:
            s["calls"] = _calls(s)
        c = s["calls"]
        if case["entry"] == "plan":
            t = c["ctx"].spd_tree_plan(s["parents"], s["new"], first=s["held"], tree=c["tree"])
            return t.seen, t.depth, t.positions
        if case["entry"] == "attend":
            return c["ctx"].spd_partial_attn_tree(c["shape"], s["q"], c["views"][0], s["new"], c["tree"], c["score"], c["out"], c["lse"])
        if case["entry"] == "keep":
            c["ctx"].spd_keep_tokens(c["shape"], c["views"], s["new"], s["keep"], s["count"])
        else:
            c["ctx"].spd_copy_pages(c["shape"], c["views"], s["pairs"], s["tokens"] if case["partial"] else None)
        return s["k"], s["v"]
    if case["entry"] == "plan":
        return _plain_plan(s)
    return _plain_attend(s) if case["entry"] == "attend" else _plain_keep(s) if case["entry"] == "keep" else _plain_pages(s)


def _seen_pairs(case):
    """(query, key) pairs that the masks leave, and keys that any query of their user sees."""
    new, held = _lens(case)
    depth_all, seen_all = _tree(case)[1], _tree(case)[0]
    prefix = np.random.default_rng([case["len_seed"], 17]).integers(0, case["prefix"], case["users"], endpoint=True) if case["prefix"] else np.zeros(len(new), np.int64)
    pairs = keys = at = 0
    for n, l, pre in zip(new.tolist(), held.tolist(), prefix.tolist()):
        begin = l - n if case["inside"] else l
        depth = depth_all[at:at + n].astype(np.int64)
        lo = np.clip(begin + depth - case["window"] + 1, 0, begin) if case["window"] else np.zeros(n, np.int64)
        pre = min(pre, begin)
        pairs += int((begin - lo + np.minimum(lo, pre)).sum())
        keys += begin - max(0, int(lo.min(initial=begin)) - pre) if n else 0
        if case["inside"] and n:
            branch = np.minimum(depth + 1, case["window"] or n)
            pairs += int(branch.sum())
            keys += n
        at += n
    return pairs, keys


def work(case):
    if case["entry"] == "plan":
        n = _lens(case)[0].astype(np.int64)
        return {"bytes": int(n.sum()) * (4 + 8 * case["words"] + 8), "flops": 0}
    es, H, d = 4 if case["dtype"] == "f32" else 2, case["kv_heads"], case["head_dim"]
    if case["entry"] == "pages":
        tokens = case["pairs"] * case["page"]
        if case["partial"]:
            r = np.random.default_rng([case["len_seed"], 29])
            r.permutation(2 * case["pairs"] + 5)
            tokens = int(r.integers(1, case["page"], case["pairs"], endpoint=True).sum())
        return {"bytes": tokens * 2 * H * d * es * 2 * case["layers"], "flops": 0}
    if case["entry"] == "keep":
        keep, count = _kept(case)
        new, at, moved = _lens(case)[0], 0, 0
        for n, m in zip(new.tolist(), count.tolist()):
            moved += int((keep[at:at + m] != np.arange(m)).sum())
            at += n
        return {"bytes": moved * 2 * H * d * es * 2 * case["layers"] + 4 * int(count.sum()), "flops": 0}
    Hq, tokens = case["q_heads"], int(_lens(case)[0].sum())
    pairs, keys = _seen_pairs(case)
    eo = 4 if case["out"] == "f32" else es
    return {"bytes": keys * 2 * H * d * es + tokens * Hq * (d * (es + eo) + 4) + tokens * (8 * case["words"] + 4), "flops": pairs * Hq * d * 4}


# From the definitions, in 64 bits: attention user by user and head by head, branches walked from parent to parent; copies row by row on the host's lists

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


def _exact_attend(case, s):
    Hq, G, d, at = case["q_heads"], case["q_heads"] // case["kv_heads"], case["head_dim"], 0
    a = torch.zeros(s["q"].shape, device=DEVICE, dtype=torch.float64)
    lse = torch.full(s["q"].shape[:2], -math.inf, device=DEVICE, dtype=torch.float64)
    parents = _parents(case).tolist()
    for u, (n, l) in enumerate(zip(s["new"].tolist(), s["held"].tolist())):
        if n == 0 or l == 0:
            at += n
            continue
        begin = l - n if case["inside"] else l
        position, hidden = list(range(l)), np.zeros((n, l), bool)
        hidden[:, begin:] = True
        depth = []
        for i in range(n):
            j, steps = i, 0
            while j >= 0:
                if case["inside"]:
                    hidden[i, begin + j] = False
                j, steps = parents[at + j], steps + 1
            depth.append(steps - 1)
            if case["inside"]:
                position[begin + i] = begin + steps - 1
        apart = np.abs(begin + np.array(depth)[:, None] - np.array(position)[None])
        if case["window"]:
            hidden |= apart >= case["window"]
        if s["prefix"] is not None:
            hidden[:, :min(begin, int(s["prefix"][u]))] = False
        apart, hidden = torch.from_numpy(apart).to(DEVICE).double(), torch.from_numpy(hidden).to(DEVICE)
        K, V = _user_rows(case, s, s["k"][0], u), _user_rows(case, s, s["v"][0], u)
        for h in range(Hq):
            x = s["q"][at:at + n, h].double() @ K[h // G].double().t().contiguous() / math.sqrt(d)
            if case["cap"]:
                x = case["cap"] * torch.tanh(x / case["cap"])
            if s["slopes"] is not None:
                x -= s["slopes"][h].double() * apart
            x[hidden] = -math.inf
            total = torch.logsumexp(x, 1)
            lse[at:at + n, h] = total
            a[at:at + n, h] = torch.nan_to_num(torch.exp(x - total[:, None]), nan=0.0) @ V[h // G].double()
        at += n
    return a, lse


def exact(case, seed):
    if case["entry"] == "plan":      # whole numbers
        return None
    s = prepare(case, seed)
    if case["entry"] == "attend":
        return _exact_attend(case, s)
    if sum(x.numel() for x in s["k"]) > 1e9:
        return None
    out = [[x.double() for x in s[name]] for name in ("k", "v")]
    if case["entry"] == "pages":
        frm, to = s["pairs"].cpu().numpy().T
        for old, x in zip(s["k"] + s["v"], out[0] + out[1]):
            for i, n in enumerate(s["tokens"].tolist()):
                if s["head_major"]:
                    x[to[i], :, :n] = old[frm[i], :, :n].double()
                else:
                    x[to[i], :n] = old[frm[i], :n].double()
        return out
    keep, count = _kept(case)
    for old, x in zip(s["k"] + s["v"], out[0] + out[1]):
        at = 0
        for u, (n, l, m) in enumerate(zip(s["new"].tolist(), s["held"].tolist(), count.tolist())):
            rows = _user_rows(case, s, old, u)[:, torch.from_numpy(l - n + keep[at:at + m]).long().to(DEVICE)].double()
            at += n
            place = torch.arange(l - n, l - n + m, device=DEVICE)
            if case["page"]:
                block, place = s["table"][u].long()[place // case["page"]], place % case["page"]
                (x.transpose(1, 2) if s["head_major"] else x)[block, place] = rows.transpose(0, 1)
            elif s["head_major"]:
                x[u][:, place] = rows
            else:
                x[u][place] = rows.transpose(0, 1)
    return out

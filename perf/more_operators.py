"""The operators of a cache in use, as measurable cases: what a decoder does with a cache besides attending over all of it
with one token.

  tree    binding.tree_attention                  drafted tokens, each of which sees the cache and its ancestors among them
  weigh   binding.decode_attention_accumulate     one new query per sequence; each row's softmax weight is added to its sum
  evict   binding.cache_evict                     the rows of the largest sums stay, the holes are filled with rows from behind
  bounds  binding.block_bounds                    least and greatest value of each channel of the keys of each block
  sparse  block_bounds of the new token, binding.block_select, binding.decode_attention_blocks
                                                  a decoding step over the blocks whose keys can have the largest scores

Shapes are the head geometries, contexts and batches of the benchmark and the tests, and points between them.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ---------------------------------------------------------------- cases

def _tree(name, B, T, n, heads, dtype="bf16", page=0, cap=0.0, slopes=False, window=0, kept=False, ragged=False):
    """T drafted tokens, the last of up to n rows; kept: the cache's rows have positions of their own, four apart in the mean."""
    Hq, Hkv, d = heads
    return {"name": name, "op": "tree", "B": B, "T": min(T, n), "n": n, "Hq": Hq, "Hkv": Hkv, "d": d, "dtype": dtype, "page": page,
            "cap": cap, "slopes": slopes, "window": window, "kept": kept, "ragged": ragged}


def _weigh(name, B, n, heads, dtype="bf16", page=0, cap=0.0, slopes=False, window=0, kept=False, ragged=False):
    return {**_tree(name, B, 1, n, heads, dtype, page, cap, slopes, window, kept, ragged), "op": "weigh"}


def _evict(name, B, n, budget, heads, dtype="bf16", page=0, recent=0, first=0, ragged=False):
    """Caches of up to n rows, of which `budget` stay: the last `recent` positions and the first `first` ones in any case."""
    _, Hkv, d = heads
    return {"name": name, "op": "evict", "B": B, "n": n, "budget": budget, "Hkv": Hkv, "d": d, "dtype": dtype, "page": page,
            "recent": min(recent, budget), "first": min(first, budget - min(recent, budget)), "ragged": ragged}


def _bounds(name, B, n, new, block, heads, dtype="bf16", page=0, ragged=False):
    """The blocks that hold any of the last `new` rows (0: all blocks)."""
    _, Hkv, d = heads
    return {"name": name, "op": "bounds", "B": B, "n": n, "new": new, "block": block, "Hkv": Hkv, "d": d, "dtype": dtype,
            "page": page, "ragged": ragged}


def _sparse(name, B, n, block, most, heads, dtype="bf16", page=0, cap=0.0, first=1, recent=2, ragged=False):
    """`most` blocks of each KV head, the first and the last ones among them."""
    Hq, Hkv, d = heads
    recent = min(recent, most)
    return {"name": name, "op": "sparse", "B": B, "n": n, "block": block, "most": most, "Hq": Hq, "Hkv": Hkv, "d": d, "dtype": dtype,
            "page": page, "cap": cap, "first": min(first, most - recent), "recent": recent, "ragged": ragged}


def listed():
    return [
        # a few drafted tokens of a small model behind a short cache: nothing but latency
        _tree("tree-5-of-1k", 1, 5, 1001, (8, 8, 64)),
        # requests over compressed caches, biased by the kept rows' own positions
        _tree("tree-26-batch-kept", 8, 26, 5000, (28, 4, 128), dtype="fp16", slopes=True, kept=True, ragged=True),
        # a wide tree over the whole cache of a long request, in 16-slot pages
        _tree("tree-64-of-100k-paged", 1, 64, 100003, (32, 8, 128), page=16),
        # one request over a compressed cache: nothing but latency
        _weigh("weigh-2k", 1, 2049, (32, 8, 128), kept=True),
        # a batch of requests with capped scores
        _weigh("weigh-batch-paged", 32, 6001, (16, 4, 64), dtype="fp16", page=16, cap=50.0, ragged=True),
        # the rows' weights gathered over whole long caches
        _weigh("weigh-100k", 2, 100003, (32, 8, 128), ragged=True),
        # a step of decoding within a budget: one row too many in every head
        _evict("evict-one", 8, 2049, 2048, (32, 8, 128), page=16, recent=32, first=4),
        # whole prompts' caches, compressed by the weights that their rows have had
        _evict("evict-32k-to-2k", 4, 32768, 2048, (32, 8, 128), recent=32, first=4, ragged=True),
        # whole prompts, behind their append
        _bounds("bounds-prompts-32k", 2, 32768, 0, 16, (32, 8, 128)),
        # a chunk of a prompt
        _bounds("bounds-chunk-paged", 8, 9001, 300, 32, (16, 4, 64), dtype="fp16", page=48, ragged=True),
        # a step of one request with a medium context
        _sparse("sparse-8k", 1, 8192, 16, 64, (32, 8, 128)),
        # a step of long requests
        _sparse("sparse-batch-128k-paged", 4, 131072, 16, 128, (64, 8, 128), page=16, cap=30.0, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    heads = rng.choice([(8, 8, 64), (16, 4, 64), (64, 1, 64), (32, 8, 128), (32, 8, 128), (28, 4, 128), (64, 8, 128), (32, 32, 128)])
    Hq, Hkv, d = heads
    dtype, page, ragged = rng.choice(["bf16", "bf16", "fp16"]), rng.choice([0, 0, 1, 16, 48, 64, 256]), rng.random() < 0.5
    cap, slopes, kept = rng.choice([0.0, 0.0, 30.0, 50.0]), rng.random() < 0.3, rng.random() < 0.3
    window = _log_int(rng, 16, 8192) if rng.random() < 0.2 else 0
    op = rng.choice(["tree", "tree", "weigh", "evict", "bounds", "sparse"])
    n, B = _log_int(rng, 1, 200000), _log_int(rng, 1, 64)
    if op == "tree":
        T = _log_int(rng, 1, 256)
        n = max(T, min(n, 32 * 64 * 100003 // (Hq * T), 8 * 100003 * 128 // (Hkv * d)))
        B = max(1, min(B, 32 * 64 * 100003 // (Hq * T * n), 8 * 100003 * 128 // (n * Hkv * d)))
        c = _tree("", B, T, n, heads, dtype, page, cap, slopes, window, kept, ragged)
    elif op == "weigh":
        n = max(1, min(n, 2 * 100003 * 8 * 128 // (Hkv * d)))
        B = max(1, min(B, 2 * 100003 * 8 * 128 // (n * Hkv * d)))
        c = _weigh("", B, n, heads, dtype, page, cap, slopes, window, kept, ragged)
    elif op == "evict":
        B = max(1, min(B, 4 * 32768 * 8 * 128 // (n * Hkv * d)))
        n = max(2, min(n, 4 * 32768 * 8 * 128 // (B * Hkv * d)))
        budget = n - 1 if rng.random() < 0.4 else _log_int(rng, 1, n - 1)
        c = _evict("", B, n, min(budget, 8192), heads, dtype, page, rng.choice([0, 1, 32, 100]), rng.choice([0, 4]), ragged)
    elif op == "bounds":
        n = max(1, min(n, 2 * 32768 * 8 * 128 // (Hkv * d)))
        B = max(1, min(B, 2 * 32768 * 8 * 128 // (n * Hkv * d)))
        c = _bounds("", B, n, rng.choice([0, 1, _log_int(rng, 1, n)]), rng.choice([16, 32, 64, 128]), heads, dtype, page, ragged)
    else:
        n = max(1, min(n, 4 * 131072 * 8 * 128 // (Hkv * d)))
        B = max(1, min(B, 4 * 131072 * 8 * 128 // (n * Hkv * d)))
        block = rng.choice([16, 16, 32, 64, 128])
        most = _log_int(rng, 1, 4096 // block)
        B = max(1, min(B, 4 * 128 * 16 * 64 * 128 // (most * block * Hq * d)))
        c = _sparse("", B, n, block, most, heads, dtype, page, cap, rng.choice([0, 1, 4]), rng.choice([0, 1, 2]), ragged)
    del c["name"]
    return c


def _lengths(c, least=1):
    """Valid rows of the sequences: the longest, and the others evenly down to a quarter (prepare deals them out)."""
    n = c["n"]
    if not c["ragged"] or c["B"] == 1:
        return [n] * c["B"]
    return [max(least, round(n * (1 - 0.75 * i / (c["B"] - 1)))) for i in range(c["B"])]


# ---------------------------------------------------------------- inputs

def _dealt(values, gen):
    v = torch.tensor(values, dtype=torch.int32)
    return v[torch.randperm(len(values), generator=gen)].to(DEV)


def _bits(T, seed):
    """The ancestors of T drafted tokens, themselves included, in words of 32 bits: chains with side branches."""
    rng = random.Random(seed)
    rows = []
    for t in range(T):
        parent = rng.choice([t - 1, t - 1, rng.randrange(-1, t)]) if t else -1
        rows.append((rows[parent] if parent >= 0 else 0) | 1 << t)
    words = [[(r >> 32 * w & 0xFFFFFFFF) for w in range(-(-T // 32))] for r in rows]
    return [[w - (1 << 32) if w >> 31 else w for w in r] for r in words]


def prepare(case, seed):
    c, dt = case, TYPES[case["dtype"]]
    g, gc = torch.Generator(device=DEV).manual_seed(seed), torch.Generator().manual_seed(seed)
    B, Hkv, d, n, op = c["B"], c["Hkv"], c["d"], c["n"], c["op"]
    s = {"case": c, "positions": None, "q_pos": None}
    s["count"] = _dealt(_lengths(c, c.get("T", 1)), gc)
    if c["page"]:
        per = -(-n // c["page"])
        s["table"] = torch.randperm(B * per, generator=g, device=DEV).to(torch.int32).view(B, per)
        shape = (B * per, Hkv, c["page"], d)
    else:
        s["table"], shape = None, (B, Hkv, n, d)
    s["K"] = torch.randn(shape, generator=g, device=DEV, dtype=dt)
    s["V"] = torch.randn(shape, generator=g, device=DEV, dtype=dt) if op != "bounds" else None
    there = torch.arange(n, device=DEV) < s["count"][:, None]
    if c.get("kept") or op == "evict":  # the kept rows' positions
        gaps = torch.randint(1, 8, (B, Hkv, n), generator=g, device=DEV)
        s["positions"] = (gaps.cumsum(2) - 1).to(torch.int32).masked_fill_(~there[:, None], -1)
    if op in ("weigh", "evict"):
        # sums of softmax weights: few rows have most of it, the last ones have not had time to gather any, some have none
        w = torch.randn(B, Hkv, n, generator=g, device=DEV).mul_(2).exp_()
        w *= ((s["count"][:, None] - torch.arange(n, device=DEV)).clamp(min=0) / n)[:, None]
        s["weights"] = w * (torch.rand(B, Hkv, n, generator=g, device=DEV) > 0.05)
    if op == "evict":
        s["new_positions"], s["new_weights"] = torch.full_like(s["positions"], -1), torch.zeros_like(s["weights"])
        s["new_count"] = torch.zeros_like(s["count"])
        return s
    if op in ("bounds", "sparse"):
        s["new"] = torch.minimum(torch.full_like(s["count"], c["new"]), s["count"]) if c.get("new") else None
        s["bounds"] = torch.zeros(B, Hkv, -(-n // c["block"]), 2, d, device=DEV, dtype=dt)
        if op == "bounds":
            return s
        _plain_bounds(s)  # (as the steps before have left them)
        s["new"] = torch.ones_like(s["count"])
        s["blocks"] = torch.empty(B, Hkv, c["most"], device=DEV, dtype=torch.int32)
    # queries of neighbouring tokens point largely the same way, so that scores vary as they do in a trained model
    Hq, T = c["Hq"], c.get("T", 1)
    q = torch.randn(B, T, Hq, d, generator=g, device=DEV).mul_(0.9).add_(torch.randn(B, 1, Hq, d, generator=g, device=DEV)).to(dt)
    s["slopes"] = (2.0 ** (-8.0 * torch.arange(1, Hq + 1, device=DEV) / Hq)).float() if c.get("slopes") else None
    if op == "tree":
        s["q"] = q.transpose(1, 2)  # as the projection leaves them
        s["tree"] = torch.tensor([_bits(T, seed * 1000 + b) for b in range(B)], dtype=torch.int32, device=DEV)
        s["out"] = torch.empty(B, Hq, T, d, device=DEV, dtype=dt)
        s["lse"] = torch.empty(B, Hq, T, device=DEV)
        if c["kept"]:  # the drafted tokens' positions, which the append has written into their rows
            depth = _mask(s["tree"]).sum(2, dtype=torch.int32)
            past = (s["count"] - T).long()
            s["q_pos"] = s["positions"].masked_fill(torch.arange(n, device=DEV) >= past[:, None, None], -1).amax((1, 2))[:, None] + depth
            rows = past[:, None] + torch.arange(T, device=DEV)
            s["positions"].scatter_(2, rows[:, None].expand(B, Hkv, T), s["q_pos"][:, None].expand(B, Hkv, T))
        return s
    s["q"] = q[:, 0]
    if c.get("kept"):
        s["q_pos"] = s["positions"].amax((1, 2)) + 1
    s["out"] = torch.empty(B, Hq, d, device=DEV, dtype=dt)
    s["lse"] = torch.empty(B, Hq, device=DEV)
    return s


# ---------------------------------------------------------------- plain forms

def _rows(s, x, j):
    """Rows j [B or 1, Hkv or 1, m] of every sequence and head: [B, Hkv, m, d], from a compact cache or from pages."""
    c = s["case"]
    B, Hkv = c["B"], c["Hkv"]
    b, h = torch.arange(B, device=DEV)[:, None, None], torch.arange(Hkv, device=DEV)[None, :, None]
    if s["table"] is None:
        return x[b, h, j]
    return x[s["table"][b, j // c["page"]].long(), h, j % c["page"]]


def _mask(bits):
    """[B, T, T]: whether drafted token t sees u."""
    u = torch.arange(bits.shape[1], device=DEV)
    return (bits[:, :, u // 32] >> (u % 32) & 1).bool()


def _attention(q, K, V, seen, dist, c, slopes):
    """q [B,Hkv,G,T,d], K and V [B,Hkv,n,d], seen [B,Hkv,1,T,n]; (out [B,Hkv,G,T,d], lse [B,Hkv,G,T], weights [B,Hkv,G,T,n])"""
    B, Hkv, G, T, d = q.shape
    score = torch.matmul(q.reshape(B, Hkv, G * T, d), K.transpose(2, 3)).view(B, Hkv, G, T, -1).div_(math.sqrt(d))
    if c["cap"]:
        score.div_(c["cap"]).tanh_().mul_(c["cap"])
    if slopes is not None:
        score -= slopes.view(1, Hkv, G, 1, 1) * dist.abs().float()
    score.masked_fill_(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(top.masked_fill(top == -math.inf, 0)).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (top + total.log()).squeeze(-1)
    p /= total.masked_fill(total == 0, 1)
    return torch.matmul(p.view(B, Hkv, G * T, -1), V).view(B, Hkv, G, T, d), lse, p


def _plain_cache(s):
    """(K, V, seen, dist) of queries [B, T] over whole caches: [B,Hkv,1,T,n]."""
    c = s["case"]
    B, n, T = c["B"], c["n"], c["T"]
    j = torch.arange(n, device=DEV)
    there = j < s["count"][:, None]
    K, V = _rows(s, s["K"], j[None, None]).float(), _rows(s, s["V"], j[None, None]).float()
    V = V.masked_fill(~there[:, None, :, None], 0)
    past = s["count"][:, None].long() - T
    if c["op"] == "tree":
        sees = _mask(s["tree"])
        depth = sees.sum(2) - torch.diagonal(sees, 0, 1, 2).long()
        u = (j - past).clamp(0, T - 1)[:, None, :].expand(B, T, n)
        allowed = torch.where((j < past)[:, None], True, sees.gather(2, u)) & there[:, None]
        at = past + depth if s["q_pos"] is None else s["q_pos"].long()
        pos = torch.where(j < past, j, past + depth.gather(1, u[:, 0]))[:, None] if s["positions"] is None else s["positions"].long()
        upto = torch.where(j < past, 0, 2 ** 40)[:, None, None]  # (what a drafted token sees of the others its bits alone say)
    else:
        allowed, upto = there[:, None], 0
        at = s["count"][:, None].long() - 1 if s["q_pos"] is None else s["q_pos"][:, None].long()
        pos = j[None, None] if s["positions"] is None else s["positions"].long()
    dist = at[:, None, :, None] - pos[:, :, None]
    seen = allowed[:, None] & (pos >= 0)[:, :, None] & (dist >= -upto)
    if c["window"]:
        seen = seen & (dist < c["window"])
    return K, V, seen[:, :, None], dist[:, :, None]


def _plain_tree(s):
    c = s["case"]
    B, Hq, Hkv, d, T = (c[k] for k in ("B", "Hq", "Hkv", "d", "T"))
    q = s["q"].float().reshape(B, Hkv, Hq // Hkv, T, d)
    out, lse, _ = _attention(q, *_plain_cache(s), c, s["slopes"])
    s["out"].copy_(out.view(B, Hq, T, d))
    s["lse"].copy_(lse.view(B, Hq, T))
    return {"out": s["out"], "lse": s["lse"]}


def _plain_weigh(s):
    c = s["case"]
    B, Hq, Hkv, d = (c[k] for k in ("B", "Hq", "Hkv", "d"))
    q = s["q"].float().reshape(B, Hkv, Hq // Hkv, 1, d)
    out, lse, p = _attention(q, *_plain_cache(s), c, s["slopes"])
    s["weights"] += p.sum((2, 3))
    s["out"].copy_(out.view(B, Hq, d))
    s["lse"].copy_(lse.view(B, Hq))
    return {"out": s["out"], "lse": s["lse"], "weights": s["weights"]}


def _plain_evict(s):
    c = s["case"]
    B, Hkv, n, budget = c["B"], c["Hkv"], c["n"], c["budget"]
    j = torch.arange(n, device=DEV)
    count = s["count"].long()[:, None, None]
    pos = s["positions"]
    newest = pos.masked_fill(j >= count, -1).amax(2, keepdim=True)
    key = s["weights"].masked_fill((pos >= 0) & ((pos > newest - c["recent"]) | (pos < c["first"])), math.inf)
    key = key.masked_fill(j >= count, -math.inf)
    order = key.sort(dim=2, descending=True, stable=True).indices
    keep = torch.zeros(B, Hkv, n, dtype=torch.bool, device=DEV).scatter_(2, order[:, :, :budget], True) & (j < count)
    small = count <= budget
    keep = torch.where(small, j < count, keep)
    hole, late = ~keep & (j < budget) & (j < count), keep & (j >= budget) & ~small
    rank = late.cumsum(2) - 1
    b, g, src = late.nonzero(as_tuple=True)
    to = torch.zeros(B, Hkv, budget, dtype=torch.long, device=DEV)
    hb, hg, hj = hole.nonzero(as_tuple=True)
    to[hb, hg, (hole.cumsum(2) - 1)[hb, hg, hj]] = hj
    dst = to[b, g, rank[b, g, src]]
    new = count.clamp(max=budget)
    s["new_positions"].copy_(torch.where(j < new, pos, torch.where(j < count, -1, s["new_positions"])))
    s["new_weights"].copy_(torch.where(j < new, s["weights"], torch.where(j < count, 0.0, s["new_weights"])))
    s["new_positions"][b, g, dst], s["new_weights"][b, g, dst] = pos[b, g, src], s["weights"][b, g, src]
    s["new_count"].copy_(s["count"].clamp(max=budget))
    if s["table"] is None:
        s["K"][b, g, dst], s["V"][b, g, dst] = s["K"][b, g, src], s["V"][b, g, src]
    else:
        page = c["page"]
        at, frm = (s["table"][b, dst // page].long(), g, dst % page), (s["table"][b, src // page].long(), g, src % page)
        s["K"][at], s["V"][at] = s["K"][frm], s["V"][frm]
    return {"K": s["K"], "V": s["V"], "positions": s["new_positions"], "weights": s["new_weights"], "count": s["new_count"]}


def _plain_bounds(s):
    c = s["case"]
    B, Hkv, d, n, block = c["B"], c["Hkv"], c["d"], c["n"], c["block"]
    whole = s["new"] is None
    count = s["count"].long()
    first = torch.zeros_like(count) if whole else (count - s["new"]) // block
    most = -(-n // block) if whole else min(-(-n // block), ((c.get("new") or 1) + block - 2) // block + 1)
    at = first[:, None] + torch.arange(most, device=DEV)
    j = (at[:, :, None] * block + torch.arange(block, device=DEV)).view(B, 1, most * block)
    there = (j < count[:, None, None]).view(B, 1, most, block, 1)
    K = _rows(s, s["K"], j.clamp(max=n - 1)).view(B, Hkv, most, block, d)
    low, high = K.masked_fill(~there, math.inf).amin(3), K.masked_fill(~there, -math.inf).amax(3)
    b, k = (at * block < count[:, None]).nonzero(as_tuple=True)
    s["bounds"][b, :, at[b, k]] = torch.stack([low, high], 3)[b, :, k]
    return {"bounds": s["bounds"]}


def _plain_sparse(s):
    c = s["case"]
    B, Hq, Hkv, d, block, most = (c[k] for k in ("B", "Hq", "Hkv", "d", "block", "most"))
    _plain_bounds(s)
    q = s["q"].double().reshape(B, Hkv, Hq // Hkv, d)
    # which blocks are taken is decided in 64 bits, and rounded once
    score = torch.matmul(s["bounds"].double().flatten(3), torch.cat([q.clamp(max=0).sum(2), q.clamp(min=0).sum(2)], 2)[..., None])
    score = score.squeeze(-1).float()
    k = torch.arange(score.shape[2], device=DEV)
    blocks = ((s["count"] + block - 1) // block)[:, None, None]
    score = score.masked_fill((k < c["first"]) | (k >= blocks - c["recent"]), math.inf).masked_fill(k >= blocks, -math.inf)
    order = score.sort(dim=2, descending=True, stable=True).indices[:, :, :most]
    order = torch.where(torch.arange(order.shape[2], device=DEV) < blocks, order, len(k)).sort(dim=2).values
    s["blocks"].fill_(-1)
    s["blocks"][:, :, :order.shape[2]] = torch.where(order < len(k), order, -1)
    j = (s["blocks"].long()[..., None] * block + torch.arange(block, device=DEV)).flatten(2)
    seen = (j >= 0) & (j < s["count"][:, None, None])
    j = j.clamp(0, c["n"] - 1)
    K, V = _rows(s, s["K"], j).float(), _rows(s, s["V"], j).float().masked_fill(~seen[..., None], 0)
    out, lse, _ = _attention(q.float()[:, :, :, None], K, V, seen[:, :, None, None], None, c, None)
    s["out"].copy_(out.view(B, Hq, d))
    s["lse"].copy_(lse.view(B, Hq))
    return {"out": s["out"], "lse": s["lse"], "blocks": s["blocks"], "bounds": s["bounds"]}


# ---------------------------------------------------------------- one pass

def run(state):
    s = state
    c = s["case"]
    if not own:
        return {"tree": _plain_tree, "weigh": _plain_weigh, "evict": _plain_evict, "bounds": _plain_bounds, "sparse": _plain_sparse}[c["op"]](s)
    from paper_2406_02069_amd import binding
    if c["op"] == "tree":
        out, lse = binding.tree_attention(s["q"], s["K"], s["V"], s["count"], tree=s["tree"], block_table=s["table"], k_cap=c["n"],
                                          positions=s["positions"], q_pos=s["q_pos"], slopes=s["slopes"], cap=c["cap"],
                                          window=c["window"], out=s["out"], lse=s["lse"], want_lse=True)
        return {"out": out, "lse": lse}
    if c["op"] == "weigh":
        out, lse = binding.decode_attention_accumulate(s["q"], s["K"], s["V"], s["count"], s["weights"], block_table=s["table"],
                                                       k_cap=c["n"], positions=s["positions"], q_pos=s["q_pos"], slopes=s["slopes"],
                                                       cap=c["cap"], window=c["window"], out=s["out"], lse=s["lse"], want_lse=True)
        return {"out": out, "lse": lse, "weights": s["weights"]}
    if c["op"] == "evict":
        binding.cache_evict(s["K"], s["V"], s["count"], s["positions"], s["weights"], c["budget"], recent=c["recent"],
                            first=c["first"], block_table=s["table"], k_cap=c["n"], positions_out=s["new_positions"],
                            weights_out=s["new_weights"], count_out=s["new_count"])
        return {"K": s["K"], "V": s["V"], "positions": s["new_positions"], "weights": s["new_weights"], "count": s["new_count"]}
    binding.block_bounds(s["K"], s["count"], s["bounds"], c["block"], new_lens=s["new"], block_table=s["table"], k_cap=c["n"])
    if c["op"] == "bounds":
        return {"bounds": s["bounds"]}
    binding.block_select(s["q"], s["bounds"], s["count"], c["block"], c["most"], first=c["first"], recent=c["recent"], k_cap=c["n"],
                         blocks_out=s["blocks"])
    out, lse = binding.decode_attention_blocks(s["q"], s["K"], s["V"], s["count"], s["blocks"], c["block"], block_table=s["table"],
                                               k_cap=c["n"], cap=c["cap"], out=s["out"], lse=s["lse"], want_lse=True)
    return {"out": out, "lse": lse, "blocks": s["blocks"], "bounds": s["bounds"]}


# ---------------------------------------------------------------- accounting

def work(case):
    c = case
    B, Hkv, d, op = c["B"], c["Hkv"], c["d"], c["op"]
    lens = _lengths(c, c.get("T", 1))
    pages = 4 * sum(-(-n // c["page"]) for n in lens) if c["page"] else 0
    if op in ("tree", "weigh"):
        Hq, T = c["Hq"], c["T"]
        rows = [min(n, (c["window"] // 4 if c["kept"] else c["window"]) + T) if c["window"] else n for n in lens]
        row = d * 2 * 2 + (4 if c["kept"] else 0) + (8 if op == "weigh" else 0)
        given = 4 * T * (-(-T // 32) + (1 if c["kept"] else 0)) if op == "tree" else 0
        return {"bytes": sum(rows) * Hkv * row + B * (Hq * T * (d * 2 * 2 + 4) + given + 4) + pages, "flops": sum(rows) * T * Hq * d * 4}
    if op == "evict":
        moved = 0
        for n in lens:  # of the kept rows those behind the budget: the last ones, and their share of the others
            if n > c["budget"]:
                late = min(c["recent"], n - c["budget"])
                moved += late + max(0, c["budget"] - c["recent"] - c["first"]) * (n - c["budget"] - late) // n
        return {"bytes": sum(lens) * Hkv * 16 + moved * Hkv * d * 2 * 4 + 8 * B, "flops": sum(lens) * Hkv}
    touched = [n if op == "bounds" and not c["new"] else n - max(n - (c.get("new") or 1), 0) // c["block"] * c["block"] for n in lens]
    blocks = [-(-n // c["block"]) for n in touched]
    moved = (sum(touched) * Hkv * d * 2 + sum(blocks) * Hkv * d * 4 + 8 * B, 2 * sum(touched) * Hkv * d)
    if op == "bounds":
        return {"bytes": moved[0] + (4 * sum(-(-n // c["page"]) for n in touched) if c["page"] else 0), "flops": moved[1]}
    Hq, every = c["Hq"], [-(-n // c["block"]) for n in lens]
    rows = [min(n, c["most"] * c["block"]) for n in lens]
    read = sum(every) * Hkv * d * 4 + sum(rows) * Hkv * d * 4 + B * Hkv * c["most"] * 8
    return {"bytes": moved[0] + read + B * (Hq * (d * 2 * 2 + 4) + 4), "flops": moved[1] + sum(every) * Hkv * d * 4 + sum(rows) * Hq * d * 4}


# ---------------------------------------------------------------- 64 bits

def _cache_rows(s, x, b, g, n):
    if s["table"] is None:
        return x[b, g, :n]
    pages = s["table"][b, :-(-n // s["case"]["page"])].long()
    return x[pages, g].reshape(-1, x.shape[-1])[:n]


def _softmax64(q, K, V, seen, dist, c, slopes):
    """q [h, T, d], K and V [n, d], seen and dist [T, n]: (out, lse, weights)"""
    z = torch.matmul(q.double(), K.double().t()) * c["d"] ** -0.5
    if c["cap"]:
        z = torch.tanh(z / c["cap"]) * c["cap"]
    if slopes is not None:
        z = z - slopes.double()[:, None, None] * dist.abs()
    z = torch.where(seen, z, -math.inf)
    lse = torch.logsumexp(z, -1)
    p = torch.exp(z - lse.masked_fill(lse == -math.inf, 0)[..., None])
    return torch.matmul(p, V.double()), lse, p


def _exact_attention(c, s):
    B, Hq, Hkv, d, T, op = c["B"], c["Hq"], c["Hkv"], c["d"], c["T"], c["op"]
    G = Hq // Hkv
    out = torch.zeros(B, Hq, T, d, dtype=torch.float64, device=DEV)
    lse = torch.full((B, Hq, T), -math.inf, dtype=torch.float64, device=DEV)
    total = s["weights"].double() if op == "weigh" else None
    q = s["q"] if op == "tree" else s["q"][:, :, None]
    bits = s["tree"].tolist() if op == "tree" else None
    for b in range(B):
        n = int(s["count"][b])
        past = n - T
        if op == "tree":
            words = [sum((w & 0xFFFFFFFF) << 32 * i for i, w in enumerate(r)) for r in bits[b]]
            sees = torch.tensor([[r >> u & 1 for u in range(T)] for r in words], device=DEV) == 1
            steps = torch.tensor([bin(r & ~(1 << t)).count("1") for t, r in enumerate(words)], device=DEV)
            at = past + steps if s["q_pos"] is None else s["q_pos"][b].long()
            whole = torch.cat([torch.arange(past, device=DEV), past + steps])
        else:
            at = torch.tensor([n - 1], device=DEV) if s["q_pos"] is None else s["q_pos"][b:b + 1].long()
            whole = torch.arange(n, device=DEV)
        for g in range(Hkv):
            pos = whole if s["positions"] is None else s["positions"][b, g, :n].long()
            dist = at[:, None] - pos
            seen = (dist >= 0) & (pos >= 0)
            if op == "tree":
                seen[:, past:] = sees & (pos >= 0)[past:]
            if c["window"]:
                seen &= dist < c["window"]
            hs = slice(g * G, g * G + G)
            o, z, p = _softmax64(q[b, hs], _cache_rows(s, s["K"], b, g, n), _cache_rows(s, s["V"], b, g, n), seen, dist, c,
                                 None if s["slopes"] is None else s["slopes"][hs])
            out[b, hs], lse[b, hs] = o, z
            if op == "weigh":
                total[b, g, :n] += p.sum((0, 1))
    if op == "tree":
        return {"out": out, "lse": lse}
    return {"out": out[:, :, 0], "lse": lse[:, :, 0], "weights": total}


def _exact_evict(c, s):
    K, V, pos, w = s["K"].double(), s["V"].double(), s["new_positions"].clone(), s["new_weights"].double()
    for b in range(c["B"]):
        n, budget = int(s["count"][b]), c["budget"]
        for g in range(c["Hkv"]):
            p, x = s["positions"][b, g, :n].cpu().numpy(), s["weights"][b, g, :n].cpu().numpy()
            rows = list(range(n))
            if n > budget:
                last = p.max()
                safe = (p >= 0) & ((p > last - c["recent"]) | (p < c["first"]))
                ranked = sorted(rows, key=lambda r: (not safe[r], 0.0 if safe[r] else -x[r], r))
                stay = set(ranked[:budget])
                late = iter(sorted(r for r in stay if r >= budget))
                rows = [r if r in stay else next(late) for r in range(budget)]
            src = torch.tensor(rows, device=DEV)
            m = len(rows)
            pos[b, g, :m], w[b, g, :m] = s["positions"][b, g, src], s["weights"][b, g, src].double()
            pos[b, g, m:n], w[b, g, m:n] = -1, 0
            dst = torch.arange(m, device=DEV)
            if s["table"] is None:
                K[b, g, dst], V[b, g, dst] = s["K"][b, g, src].double(), s["V"][b, g, src].double()
            else:
                t, page = s["table"][b].long(), c["page"]
                K[t[dst // page], g, dst % page] = s["K"][t[src // page], g, src % page].double()
                V[t[dst // page], g, dst % page] = s["V"][t[src // page], g, src % page].double()
    return {"K": K, "V": V, "positions": pos, "weights": w, "count": s["count"].clamp(max=c["budget"])}


def exact(case, seed):
    c, s = case, prepare(case, seed)
    B, Hkv, d, op = c["B"], c["Hkv"], c["d"], c["op"]
    if op in ("tree", "weigh"):
        return _exact_attention(c, s)
    if op == "evict":
        return _exact_evict(c, s) if sum(_lengths(c)) * Hkv <= 2 * 10 ** 6 else None
    block = c["block"]
    bounds = s["bounds"].double()
    for b in range(B):
        n = int(s["count"][b])
        first = 0 if s["new"] is None else (n - int(s["new"][b])) // block
        if n * Hkv == 0:
            continue
        for g in range(Hkv):
            rows = _cache_rows(s, s["K"], b, g, n)[first * block:].double()
            whole = len(rows) // block
            parts = [rows[:whole * block].view(whole, block, d).aminmax(dim=1)] if whole else []
            if len(rows) % block:
                parts.append(rows[whole * block:][None].aminmax(dim=1))
            bounds[b, g, first:first + whole + (len(rows) % block > 0)] = torch.cat([torch.stack(tuple(x), 1) for x in parts])
    if op == "bounds":
        return {"bounds": bounds}
    Hq, most = c["Hq"], c["most"]
    G = Hq // Hkv
    out = torch.zeros(B, Hq, d, dtype=torch.float64, device=DEV)
    lse = torch.full((B, Hq), -math.inf, dtype=torch.float64, device=DEV)
    blocks = torch.full((B, Hkv, most), -1, dtype=torch.int32)
    for b in range(B):
        n = int(s["count"][b])
        have = -(-n // block)
        for g in range(Hkv):
            q = s["q"][b, g * G:g * G + G].double()
            score = sum(torch.maximum(q[h] * bounds[b, g, :have, 0], q[h] * bounds[b, g, :have, 1]).sum(1) for h in range(G))
            score = score.float().cpu().tolist()
            ranked = sorted(range(have), key=lambda k: (not (k < c["first"] or k >= have - c["recent"]), -score[k], k))
            forced = [k for k in range(have) if k < c["first"] or k >= have - c["recent"]]
            taken = sorted((sorted(forced) + [k for k in ranked if k not in set(forced)])[:most])
            blocks[b, g, :len(taken)] = torch.tensor(taken, dtype=torch.int32)
            j = (torch.tensor(taken, device=DEV)[:, None] * block + torch.arange(block, device=DEV)).view(-1)
            j = j[j < n]
            o, z, _ = _softmax64(q[:, None], _cache_rows(s, s["K"], b, g, n)[j], _cache_rows(s, s["V"], b, g, n)[j],
                                 torch.ones(1, len(j), dtype=torch.bool, device=DEV), None, c, None)
            out[b, g * G:g * G + G], lse[b, g * G:g * G + G] = o[:, 0], z[:, 0]
    return {"out": out, "lse": lse, "blocks": blocks.to(DEV), "bounds": bounds}

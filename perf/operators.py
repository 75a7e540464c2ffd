"""The operators around the compression step, as measurable cases: rotary positions with the append to a cache, the
attention of a prompt that hands its softmax denominators on, and the attention of one new token over a long cache.

  rotary   binding.rotary_append          rotated queries, rotated keys and values in the cache's rows (all layers do it,
                                          for a prompt as for each new token)
  prefill  binding.prefill_attention      a prompt's, or a chunk of a prompt's, attention under causal, window, document
                                          and prefix masks, with scores capped by a tanh and biased by distance
  decode   binding.decode_attention_long  one new query per sequence over a whole or a compressed cache

Shapes are the head geometries, contexts and batches of the benchmark and the tests, and points between them.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ---------------------------------------------------------------- cases

def _rotary(name, B, T, heads, dtype="bf16", rot=None, layout="half", scaling="none", k_cap=0, page=0, ragged=False,
            far=False):
    """T new tokens per sequence behind a cache's rows (k_cap 0: the cache is theirs alone); far: positions are given
    (those of a compressed cache lie behind its rows), otherwise they are the rows' numbers."""
    Hq, Hkv, d = heads
    return {"name": name, "op": "rotary", "B": B, "T": T, "Hq": Hq, "Hkv": Hkv, "d": d, "dtype": dtype, "rot": rot or d,
            "layout": layout, "scaling": scaling, "k_cap": max(k_cap, T), "page": page, "ragged": ragged, "far": far}


def _prefill(name, B, T, N, heads, dtype="bf16", cap=0.0, slopes=False, window=0, docs=0, prefix=False, ragged=False):
    """Queries of the last T of N positions (T == N: whole prompts)."""
    Hq, Hkv, d = heads
    return {"name": name, "op": "prefill", "B": B, "T": T, "N": N, "Hq": Hq, "Hkv": Hkv, "d": d, "dtype": dtype, "cap": cap,
            "slopes": slopes, "window": window, "docs": docs, "prefix": prefix, "ragged": ragged}


def _decode(name, B, n, heads, dtype="bf16", page=0, cap=0.0, slopes=False, window=0, kept=False, ragged=False):
    """kept: the cache's rows are a kept subset with positions of their own, four apart in the mean."""
    Hq, Hkv, d = heads
    return {"name": name, "op": "decode", "B": B, "n": n, "Hq": Hq, "Hkv": Hkv, "d": d, "dtype": dtype, "page": page,
            "cap": cap, "slopes": slopes, "window": window, "kept": kept, "ragged": ragged}


def listed():
    return [
        # one new token of one request behind a compressed cache: nothing but latency
        _rotary("rotary-token", 1, 1, (32, 8, 128), k_cap=2048, scaling="bands", far=True),
        # one new token of each of 64 requests, interleaved pairs in half of the head, 16-slot pages
        _rotary("rotary-batch-paged", 64, 1, (16, 4, 64), dtype="fp16", rot=32, layout="interleaved", k_cap=2500, page=16,
                ragged=True),
        # a batch of ragged prompts behind their projections
        _rotary("rotary-prompts-16k", 8, 16384, (32, 8, 128), scaling="ramp", ragged=True),
        # a small multi-head model with a short prompt
        _prefill("prefill-37", 1, 37, 37, (8, 8, 64)),
        # the benchmark's medium prompt
        _prefill("prefill-8k", 1, 8192, 8192, (32, 8, 128)),
        # packed documents with a prefix each that sees itself whole, capped scores
        _prefill("prefill-docs-12001", 2, 12001, 12001, (16, 4, 64), dtype="fp16", cap=50.0, docs=23, prefix=True),
        # a chunk of a long prompt, scores biased by distance: few query rows, many keys
        _prefill("prefill-chunk-300-of-50k", 1, 300, 50001, (28, 4, 128), slopes=True),
        # the benchmark's long prompt
        _prefill("prefill-32k", 1, 32768, 32768, (32, 8, 128)),
        # a short cache of a small model: nothing but latency
        _decode("decode-1k", 1, 1000, (8, 8, 64)),
        # the longest context of the tests, one request, whole cache in 16-slot pages
        _decode("decode-128k-paged", 1, 131072, (32, 8, 128), page=16),
        # requests over compressed caches: the bias goes by the kept rows' own positions
        _decode("decode-kept-batch", 16, 5000, (28, 4, 128), dtype="fp16", slopes=True, kept=True, ragged=True),
        # a batch of long requests of a large model, capped scores
        _decode("decode-batch-100k", 4, 100003, (64, 8, 128), page=64, cap=30.0, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    heads = rng.choice([(8, 8, 64), (16, 4, 64), (64, 1, 64), (32, 8, 128), (32, 8, 128), (28, 4, 128), (64, 8, 128), (32, 32, 128)])
    Hq, Hkv, d = heads
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    op = rng.choice(["rotary", "prefill", "decode"])
    if op == "rotary":
        most = 8 * 16384 * 40 * 128  # elements of the largest listed case
        if rng.random() < 0.5:
            B, T = _log_int(rng, 1, 256), 1
        else:
            T = _log_int(rng, 2, 100000)
            B = max(1, min(_log_int(rng, 1, 16), most // (T * (Hq + Hkv) * d)))
        T = max(1, min(T, most // (B * (Hq + Hkv) * d)))
        c = _rotary("", B, T, heads, dtype, rot=rng.choice([d, d, d // 2, 24]), layout=rng.choice(["half", "interleaved"]),
                    scaling=rng.choice(["none", "linear", "bands", "ramp"]), k_cap=T if T > 4096 else T + _log_int(rng, 16, 4096),
                    page=rng.choice([0, 0, 16, 48, 256]), ragged=rng.random() < 0.5, far=rng.random() < 0.4)
    elif op == "prefill":
        mask = rng.choice(["none", "none", "window", "docs", "prefix"])
        N = _log_int(rng, 1, 131072)
        T = N if rng.random() < 0.6 else _log_int(rng, 1, N)
        B = _log_int(rng, 1, 8)
        most = 32 * 32768 * 32768 * 128  # products of the largest listed case, without its mask
        most = most * 3 // 4 if T == N else most // 2  # (a chunk's queries see most keys, a prefix both ways)
        T = max(1, min(T, most // (Hq * N * d)))
        B = max(1, min(B, most // (Hq * T * N * d)))
        N = T if T > N // 2 else N
        c = _prefill("", B, T, N, heads, dtype, cap=rng.choice([0.0, 0.0, 30.0, 50.0]), slopes=rng.random() < 0.3,
                     window=_log_int(rng, 16, 8192) if mask == "window" else 0,
                     docs=_log_int(rng, 1, 64) if mask in ("docs", "prefix") else 0, prefix=mask == "prefix",
                     ragged=rng.random() < 0.5)
    else:
        most = 4 * 100003 * 8 * 128
        n = _log_int(rng, 1, 400000)
        B = _log_int(rng, 1, 64)
        n = max(1, min(n, most // (Hkv * d)))
        B = max(1, min(B, most // (n * Hkv * d)))
        c = _decode("", B, n, heads, dtype, page=rng.choice([0, 0, 1, 16, 48, 64, 256]), cap=rng.choice([0.0, 0.0, 30.0, 50.0]),
                    slopes=rng.random() < 0.3, window=_log_int(rng, 16, 8192) if rng.random() < 0.2 else 0,
                    kept=rng.random() < 0.3, ragged=rng.random() < 0.5)
    del c["name"]
    return c


def _lengths(c, most):
    """Valid lengths of the sequences: the longest, and the others evenly down to a quarter (prepare deals them out)."""
    if not c["ragged"] or c["B"] == 1:
        return [most] * c["B"]
    return [max(1, round(most * (1 - 0.75 * i / (c["B"] - 1)))) for i in range(c["B"])]


def _documents(c, n):
    """Lengths of the documents packed into n positions: in the ratio 1 : 2 : 3 : ..., the last takes the rest."""
    k = max(1, min(c["docs"], n))
    whole = k * (k + 1) // 2
    ends = [n * (i * (i + 1) // 2) // whole for i in range(1, k + 1)]
    return [b - a for a, b in zip([0] + ends[:-1], ends) if b > a]


# ---------------------------------------------------------------- inputs

def _inverse_frequencies(c):
    """Radians per position of each pair, in 64 bits.  "linear": positions divided by a factor of 8.  "bands": as they
    are where a wave is short against the trained context of 8192, divided by 8 where it is long, blended between.
    "ramp": divided by 16 where fewer than 1 turn fits into the trained context, as they are from 32 turns on, a ramp
    over the pairs' numbers between, and a magnitude that grows with the factor's logarithm."""
    rot, base, trained = c["rot"], 500000.0 if c["scaling"] == "bands" else 10000.0, 8192.0
    i = torch.arange(rot // 2, dtype=torch.float64, device=DEV)
    f = base ** (-2 * i / rot)
    if c["scaling"] == "linear":
        return f / 8, 1.0
    if c["scaling"] == "bands":
        blend = ((trained * f / (2 * math.pi) - 1) / (4 - 1)).clamp(0, 1)
        return (1 - blend) * f / 8 + blend * f, 1.0
    if c["scaling"] == "ramp":
        def at(turns):
            return rot * math.log(trained / (turns * 2 * math.pi)) / (2 * math.log(base))
        lo, hi = max(math.floor(at(32)), 0), min(math.ceil(at(1)), rot - 1)
        ramp = ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return f / 16 * ramp + f * (1 - ramp), 0.1 * math.log(16) + 1
    return f, 1.0


def _dealt(values, gen):
    v = torch.tensor(values, dtype=torch.int32)
    return v[torch.randperm(len(values), generator=gen)].to(DEV)


def _pool(c, rows, dt, g):
    """Pages in random order for `rows` rows of every sequence: (K pool, V pool, block table)."""
    per = -(-rows // c["page"])
    table = torch.randperm(c["B"] * per, generator=g, device=DEV).to(torch.int32).view(c["B"], per)
    shape = (c["B"] * per, c["Hkv"], c["page"], c["d"])
    return (torch.randn(shape, generator=g, device=DEV, dtype=dt), torch.randn(shape, generator=g, device=DEV, dtype=dt), table)


def prepare(case, seed):
    c, dt = case, TYPES[case["dtype"]]
    g, gc = torch.Generator(device=DEV).manual_seed(seed), torch.Generator().manual_seed(seed)
    B, Hq, Hkv, d = c["B"], c["Hq"], c["Hkv"], c["d"]
    s = {"case": c}
    if c["op"] == "rotary":
        T, cap = c["T"], c["k_cap"]
        # the projections' output [B, T, heads, d], as the model's matrix product leaves it
        x = torch.randn(B, T, Hq + 2 * Hkv, d, generator=g, device=DEV, dtype=dt).transpose(1, 2)
        s["q"], s["k"], s["v"] = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
        s["new"] = _dealt(_lengths(c, T), gc)
        old = _dealt([(cap - T) * (B - i) // B for i in range(B)], gc) if T < cap else torch.zeros_like(s["new"])
        s["count"] = s["new"] + old
        s["positions"] = None
        if c["far"]:
            s["positions"] = 29 * old[:, None] + torch.arange(T, device=DEV, dtype=torch.int32)
        s["inv_freq"], s["magnitude"] = _inverse_frequencies(c)
        if c["page"]:
            s["K"], s["V"], s["table"] = _pool(c, cap, dt, g)
        else:
            s["K"] = torch.randn(B, Hkv, cap, d, generator=g, device=DEV, dtype=dt)
            s["V"], s["table"] = torch.randn(B, Hkv, cap, d, generator=g, device=DEV, dtype=dt), None
        s["q_out"] = torch.zeros(B, Hq, T, d, device=DEV, dtype=dt)
        return s
    # queries of neighbouring tokens point largely the same way, so that scores vary as they do in a trained model
    base = torch.randn(B, Hq, 1, d, generator=g, device=DEV)
    s["slopes"] = (2.0 ** (-8.0 * torch.arange(1, Hq + 1, device=DEV) / Hq)).float() if c["slopes"] else None
    if c["op"] == "prefill":
        T, N = c["T"], c["N"]
        s["q"] = torch.randn(B, Hq, T, d, generator=g, device=DEV).mul_(0.9).add_(base).to(dt)
        s["K"] = torch.randn(B, Hkv, N, d, generator=g, device=DEV, dtype=dt)
        s["V"] = torch.randn(B, Hkv, N, d, generator=g, device=DEV, dtype=dt)
        s["K"][:, :, 0] *= 4  # an attention sink
        s["lens"] = _dealt(_lengths(c, N), gc) if c["ragged"] else None
        n = s["lens"].cpu() if c["ragged"] else torch.full((B,), N)
        s["start"] = (n - T).clamp(min=0).to(torch.int32).to(DEV) if T < N else None
        s["doc_start"] = s["prefix_end"] = None
        if c["docs"]:
            starts, ends = torch.zeros(B, N, dtype=torch.int32), torch.zeros(B, N, dtype=torch.int32)
            for b in range(B):
                lens = torch.tensor(_documents(c, int(n[b])))
                lens = lens[torch.randperm(len(lens), generator=gc)]
                first = lens.cumsum(0) - lens
                starts[b, :int(n[b])] = first.repeat_interleave(lens).int()
                ends[b, :int(n[b])] = (first + lens // 4).repeat_interleave(lens).int()
            s["doc_start"] = starts.to(DEV)
            s["prefix_end"] = ends.to(DEV) if c["prefix"] else None
        return s
    n = c["n"]
    s["q"] = torch.randn(B, Hq, d, generator=g, device=DEV).mul_(0.9).add_(base[:, :, 0]).to(dt)
    s["count"] = _dealt(_lengths(c, n), gc)
    if c["page"]:
        s["K"], s["V"], s["table"] = _pool(c, n, dt, g)
    else:
        s["K"] = torch.randn(B, Hkv, n, d, generator=g, device=DEV, dtype=dt)
        s["V"], s["table"] = torch.randn(B, Hkv, n, d, generator=g, device=DEV, dtype=dt), None
    s["positions"] = s["q_pos"] = None
    if c["kept"]:
        gaps = torch.randint(1, 8, (B, Hkv, n), generator=g, device=DEV)
        s["positions"] = (gaps.cumsum(2) - 1).to(torch.int32)
        s["positions"][(torch.arange(n, device=DEV) >= s["count"][:, None])[:, None].expand(B, Hkv, n)] = -1
        s["q_pos"] = s["positions"].amax((1, 2)) + 1
    s["out"] = torch.empty(B, Hq, d, device=DEV, dtype=dt)
    s["lse"] = torch.empty(B, Hq, device=DEV, dtype=torch.float32)
    return s


# ---------------------------------------------------------------- plain forms

def _rows(s, x, rows):
    """The first `rows` rows of every sequence: [B, Hkv, rows, d], from a compact cache or from pages."""
    if s["table"] is None:
        return x[:, :, :rows]
    page = x.shape[2]
    j = torch.arange(rows, device=DEV)
    return x[s["table"][:, j // page].long(), :, (j % page)].transpose(1, 2)


def _turned(x, cos, sin, layout):
    half = cos.shape[-1]
    x = x.float()
    if layout == "half":
        a, b, rest = x[..., :half], x[..., half:2 * half], x[..., 2 * half:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)
    a, b, rest = x[..., 0:2 * half:2], x[..., 1:2 * half:2], x[..., 2 * half:]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), rest], -1)


def _plain_rotary(s):
    c = s["case"]
    t = torch.arange(c["T"], device=DEV)
    row = (s["count"] - s["new"])[:, None] + t
    pos = row if s["positions"] is None else s["positions"]
    angle = pos.double()[:, None, :, None] * s["inv_freq"]
    cos, sin = (angle.cos() * s["magnitude"]).float(), (angle.sin() * s["magnitude"]).float()
    there = t < s["new"][:, None]
    q = _turned(s["q"], cos, sin, c["layout"]).to(s["q"].dtype)
    k = _turned(s["k"], cos, sin, c["layout"]).to(s["k"].dtype)
    s["q_out"].copy_(torch.where(there[:, None, :, None], q, s["q_out"]))
    b, t = there.nonzero(as_tuple=True)
    at = row[b, t].long()
    if s["table"] is None:
        s["K"][b, :, at], s["V"][b, :, at] = k[b, :, t], s["v"][b, :, t]
    else:
        page = s["table"][b, at // c["page"]].long()
        s["K"][page, :, at % c["page"]], s["V"][page, :, at % c["page"]] = k[b, :, t], s["v"][b, :, t]
    return {"q": s["q_out"], "K": s["K"], "V": s["V"]}


def _softmax_product(score, seen, V):
    """softmax over the seen keys times V, and the log of its denominator; nothing seen: zero and -inf."""
    score.masked_fill_(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = (score - top.masked_fill(top == -math.inf, 0)).exp_()
    total = p.sum(-1, keepdim=True)
    return torch.matmul(p, V) / total.masked_fill(total == 0, 1), (top + total.log()).squeeze(-1)


def _plain_prefill(s):
    c = s["case"]
    B, Hq, Hkv, d, T, N = (c[k] for k in ("B", "Hq", "Hkv", "d", "T", "N"))
    G = Hq // Hkv
    K, V = s["K"].float(), s["V"].float()
    n = torch.full((B,), N, device=DEV) if s["lens"] is None else s["lens"].long()
    there = torch.arange(N, device=DEV) < n[:, None]
    if s["lens"] is not None:
        V = V.masked_fill(~there[:, None, :, None], 0)
    out = torch.empty(B, Hq, T, d, device=DEV, dtype=s["q"].dtype)
    lse = torch.empty(B, Hq, T, device=DEV)
    first = torch.zeros(B, device=DEV, dtype=torch.long) if s["start"] is None else s["start"].long()
    step = max(1, min(T, 2 ** 30 // (B * Hq * N)))
    for t0 in range(0, T, step):  # as many query rows at a time as 4 GB of scores hold
        rows = min(step, T - t0)
        p = first[:, None] + torch.arange(t0, t0 + rows, device=DEV)
        valid = (p >= 0) & (p < n[:, None])
        at = p.clamp(0, N - 1)
        lo = torch.zeros_like(p) if s["doc_start"] is None else s["doc_start"].long().gather(1, at)
        if c["window"]:
            lo = torch.maximum(lo, p - c["window"] + 1)
        hi = p if s["prefix_end"] is None else torch.maximum(p, s["prefix_end"].long().gather(1, at) - 1)
        keys = max(1, min(N, N if s["prefix_end"] is not None or s["start"] is not None else t0 + rows))
        j = torch.arange(keys, device=DEV)
        seen = (j >= lo[..., None]) & (j <= hi[..., None]) & valid[..., None] & there[:, None, :keys]
        q = s["q"][:, :, t0:t0 + rows].float().reshape(B, Hkv, G * rows, d)
        score = torch.matmul(q, K[:, :, :keys].transpose(2, 3)).view(B, Hkv, G, rows, keys).div_(math.sqrt(d))
        if c["cap"]:
            score.div_(c["cap"]).tanh_().mul_(c["cap"])
        if s["slopes"] is not None:
            far = (p[..., None] - j).abs().float()
            score -= s["slopes"].view(1, Hkv, G, 1, 1) * far[:, None, None]
        o, z = _softmax_product(score.view(B, Hkv, G * rows, keys), seen[:, None, None].expand(B, 1, G, rows, keys).reshape(B, 1, G * rows, keys), V[:, :, :keys])
        out[:, :, t0:t0 + rows] = o.view(B, Hq, rows, d)
        lse[:, :, t0:t0 + rows] = z.view(B, Hq, rows)
    return {"out": out, "lse": lse}


def _plain_decode(s):
    c = s["case"]
    B, Hq, Hkv, d, n = (c[k] for k in ("B", "Hq", "Hkv", "d", "n"))
    G = Hq // Hkv
    K, V = _rows(s, s["K"], n).float(), _rows(s, s["V"], n).float()
    j = torch.arange(n, device=DEV)
    seen = (j < s["count"][:, None])[:, None]
    V = V.masked_fill(~seen[..., None], 0)
    pos = j.view(1, 1, n) if s["positions"] is None else s["positions"]
    at = (s["count"] - 1 if s["q_pos"] is None else s["q_pos"]).view(B, 1, 1)
    seen = seen & (pos >= 0) & (pos <= at)
    if c["window"]:
        seen = seen & (pos > at - c["window"])
    score = torch.matmul(s["q"].float().view(B, Hkv, G, d), K.transpose(2, 3)).div_(math.sqrt(d))
    if c["cap"]:
        score.div_(c["cap"]).tanh_().mul_(c["cap"])
    if s["slopes"] is not None:
        score -= s["slopes"].view(1, Hkv, G, 1) * (at - pos).float()[:, :, None]
    o, z = _softmax_product(score, seen[:, :, None].expand(score.shape), V)
    s["out"].copy_(o.view(B, Hq, d))
    s["lse"].copy_(z.view(B, Hq))
    return {"out": s["out"], "lse": s["lse"]}


# ---------------------------------------------------------------- one pass

def run(state):
    s = state
    c = s["case"]
    if not own:
        return {"rotary": _plain_rotary, "prefill": _plain_prefill, "decode": _plain_decode}[c["op"]](s)
    from paper_2406_02069_amd import binding
    if c["op"] == "rotary":
        binding.rotary_append(s["q"], s["k"], s["v"], s["inv_freq"], s["K"], s["V"], s["count"], layout=c["layout"],
                              magnitude=s["magnitude"], positions=s["positions"], new_lens=s["new"],
                              block_table=s["table"], k_cap=c["k_cap"], q_out=s["q_out"])
        return {"q": s["q_out"], "K": s["K"], "V": s["V"]}
    if c["op"] == "prefill":
        out, lse = binding.prefill_attention(s["q"], s["K"], s["V"], seq_lens=s["lens"], q_start=s["start"],
                                             doc_start=s["doc_start"], prefix_end=s["prefix_end"], slopes=s["slopes"],
                                             cap=c["cap"], window=c["window"], want_lse=True)
        return {"out": out, "lse": lse}
    out, lse = binding.decode_attention_long(s["q"], s["K"], s["V"], s["count"], block_table=s["table"], k_cap=c["n"],
                                             positions=s["positions"], q_pos=s["q_pos"], slopes=s["slopes"], cap=c["cap"],
                                             window=c["window"], out=s["out"], lse=s["lse"], want_lse=True)
    return {"out": out, "lse": lse}


# ---------------------------------------------------------------- accounting

def _pairs(c, n):
    """(query, key) pairs that the masks of one sequence leave, and the keys that some query of it sees."""
    p = torch.arange(max(n - c["T"], 0) if c["T"] < c["N"] else 0, n)
    p = p[:c["T"]]
    if len(p) == 0:
        return 0, 0
    lo, hi = torch.zeros_like(p), p.clone()
    if c["docs"]:
        lens = torch.tensor(_documents(c, n))
        first = (lens.cumsum(0) - lens).repeat_interleave(lens)
        lo = first[p]
        if c["prefix"]:
            hi = torch.maximum(hi, lo + (lens // 4).repeat_interleave(lens)[p] - 1)
    if c["window"]:
        lo = torch.maximum(lo, p - c["window"] + 1)
    return int((hi - lo + 1).sum()), int(hi.max() - lo.min() + 1)


def work(case):
    c = case
    B, Hq, Hkv, d = c["B"], c["Hq"], c["Hkv"], c["d"]
    if c["op"] == "rotary":
        tokens = sum(_lengths(c, c["T"]))
        moved = tokens * ((Hq + 2 * Hkv) * d * 2 * 2 + (4 if c["far"] else 0))
        return {"bytes": moved + c["rot"] // 2 * 8 + B * (8 + (4 if c["page"] else 0)), "flops": tokens * (Hq + Hkv) * c["rot"] * 3}
    if c["op"] == "prefill":
        found = [_pairs(c, n) for n in _lengths(c, c["N"])]
        pairs, keys = sum(f[0] for f in found), sum(f[1] for f in found)
        given = (4 if c["docs"] else 0) + (4 if c["prefix"] else 0)
        return {"bytes": B * c["T"] * (Hq * (d * 2 * 2 + 4) + given) + keys * Hkv * d * 2 * 2, "flops": pairs * Hq * d * 4}
    rows = _lengths(c, c["n"])
    if c["window"]:  # (kept rows lie four positions apart)
        rows = [min(n, c["window"] // 4 if c["kept"] else c["window"]) for n in rows]
    moved = sum(rows) * Hkv * (d * 2 * 2 + (4 if c["kept"] else 0)) + (sum(-(-n // c["page"]) * 4 for n in rows) if c["page"] else 0)
    return {"bytes": moved + B * (Hq * (d * 2 * 2 + 4) + 4), "flops": sum(rows) * Hq * d * 4}


# ---------------------------------------------------------------- 64 bits

def exact(case, seed):
    c, s = case, prepare(case, seed)
    B, Hq, Hkv, d = c["B"], c["Hq"], c["Hkv"], c["d"]
    G = Hq // Hkv
    if c["op"] == "rotary":
        q_out, K, V = s["q_out"].double(), s["K"].double(), s["V"].double()
        half = c["rot"] // 2
        for b in range(B):
            new = int(s["new"][b])
            at = int(s["count"][b]) - new + torch.arange(new, device=DEV)
            pos = at if s["positions"] is None else s["positions"][b, :new]
            turn = torch.polar(torch.full((new, half), float(s["magnitude"]), dtype=torch.float64, device=DEV),
                               pos.double()[:, None] * s["inv_freq"][None])

            def turned(x):
                x = x[:, :new].double()
                if c["layout"] == "half":
                    z = torch.complex(x[..., :half].contiguous(), x[..., half:2 * half].contiguous()) * turn
                    return torch.cat([z.real, z.imag, x[..., 2 * half:]], -1)
                z = torch.view_as_complex(x[..., :2 * half].reshape(x.shape[0], new, half, 2).contiguous()) * turn
                return torch.cat([torch.view_as_real(z).flatten(-2), x[..., 2 * half:]], -1)

            q_out[b, :, :new] = turned(s["q"][b])
            k, v = turned(s["k"][b]), s["v"][b, :, :new].double()
            if s["table"] is None:
                K[b, :, at], V[b, :, at] = k, v
            else:
                page = s["table"][b].long()[at // c["page"]]
                K[page, :, at % c["page"]], V[page, :, at % c["page"]] = k.transpose(0, 1), v.transpose(0, 1)
        return {"q": q_out, "K": K, "V": V}
    if c["op"] == "prefill":
        T, N = c["T"], c["N"]
        out = torch.zeros(B, Hq, T, d, dtype=torch.float64, device=DEV)
        lse = torch.full((B, Hq, T), -math.inf, dtype=torch.float64, device=DEV)
        for b in range(B):
            n = N if s["lens"] is None else int(s["lens"][b])
            first = 0 if s["start"] is None else int(s["start"][b])
            rows = max(0, min(T, n - first))
            for h in range(Hq):
                K, V = s["K"][b, h // G, :n].double(), s["V"][b, h // G, :n].double()
                step = max(1, 2 ** 28 // n)
                for t0 in range(0, rows, step):
                    t1 = min(rows, t0 + step)
                    pos = torch.arange(first + t0, first + t1, device=DEV)
                    dist = pos[:, None] - torch.arange(n, device=DEV)[None]
                    seen = dist >= 0
                    if s["prefix_end"] is not None:
                        seen |= torch.arange(n, device=DEV) < s["prefix_end"][b, pos][:, None]
                    if s["doc_start"] is not None:
                        seen &= torch.arange(n, device=DEV) >= s["doc_start"][b, pos][:, None]
                    if c["window"]:
                        seen &= dist < c["window"]
                    z = s["q"][b, h, t0:t1].double() @ K.t() * d ** -0.5
                    if c["cap"]:
                        z = torch.tanh(z / c["cap"]) * c["cap"]
                    if s["slopes"] is not None:
                        z = z - float(s["slopes"][h]) * dist.abs()
                    z = torch.where(seen, z, -math.inf)
                    total = torch.logsumexp(z, -1)
                    out[b, h, t0:t1] = torch.exp(z - total.masked_fill(total == -math.inf, 0)[:, None]) @ V
                    lse[b, h, t0:t1] = total
        return {"out": out, "lse": lse}
    out = torch.zeros(B, Hq, d, dtype=torch.float64, device=DEV)
    lse = torch.full((B, Hq), -math.inf, dtype=torch.float64, device=DEV)
    for b in range(B):
        n = int(s["count"][b])
        for g in range(Hkv):
            if s["table"] is None:
                K, V = s["K"][b, g, :n], s["V"][b, g, :n]
            else:
                pages = s["table"][b, :-(-n // c["page"])].long()
                K, V = s["K"][pages, g].reshape(-1, d)[:n], s["V"][pages, g].reshape(-1, d)[:n]
            at = n - 1 if s["q_pos"] is None else int(s["q_pos"][b])
            dist = at - (torch.arange(n, device=DEV) if s["positions"] is None else s["positions"][b, g, :n])
            z = s["q"][b, g * G:(g + 1) * G].double() @ K.double().t() * d ** -0.5
            if c["cap"]:
                z = torch.tanh(z / c["cap"]) * c["cap"]
            if s["slopes"] is not None:
                z = z - s["slopes"][g * G:(g + 1) * G].double()[:, None] * dist
            z = z.masked_fill(dist < 0, -math.inf)
            if c["window"]:
                z = z.masked_fill(dist >= c["window"], -math.inf)
            total = torch.logsumexp(z, -1)
            out[b, g * G:(g + 1) * G] = torch.exp(z - total.masked_fill(total == -math.inf, 0)[:, None]) @ V.double()
            lse[b, g * G:(g + 1) * G] = total
    return {"out": out, "lse": lse}

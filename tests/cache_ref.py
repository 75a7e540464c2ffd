"""Plain forms in 64 bits of the operators of a cache in use, for their tests: which rows a drafted token sees, weights with their
room, evictions row by row, bounds and selected blocks."""
import math

import torch

from tests import attention_bounds
from tests.attention_bounds import HALF_STEP

DEV = "cuda:0"
# Rounding of a weight for the product with V: to two numbers of the type (up to 32 query rows a KV head), else once.
TOKEN = {t: h * h for t, h in HALF_STEP.items()}
TOKEN_SMALL = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -38}
PROMPT = HALF_STEP
PROMPT_SMALL = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -33}


def paged(x, page, table, pages):
    """Rows [B,Hkv,n,d] in pools of `pages` pages through a table; what no row fills is NaN."""
    B, Hkv, n, d = x.shape
    pool = torch.full((pages, Hkv, page, d), math.nan, dtype=x.dtype, device=x.device)
    j = torch.arange(n, device=x.device)
    for b in range(B):
        at = table[b].long()[j // page]
        ok = (at >= 0) & (at < pages)
        pool[at[ok], :, (j % page)[ok]] = x[b].transpose(0, 1)[ok]
    return pool


def unpaged(pool, table, n):
    """Rows [B,Hkv,n,d] of pools."""
    j = torch.arange(n, device=pool.device)
    page = pool.shape[2]
    return torch.stack([pool[table[b].long()[j // page], :, j % page].transpose(0, 1) for b in range(table.shape[0])])


def make_cache(B, Hkv, n, d, dtype, page, g):
    """(K rows, V rows, K and V as a call takes them, table)"""
    K, V = (torch.randn(B, Hkv, n, d, generator=g, device=DEV).to(dtype) for _ in range(2))
    if not page:
        return K, V, K, V, None
    per = -(-n // page)
    table = torch.randperm(B * per + 2, generator=g, device=DEV)[:B * per].to(torch.int32).view(B, per).contiguous()
    return K, V, paged(K, page, table, B * per + 2), paged(V, page, table, B * per + 2), table


def random_tree(T, rng):
    """Parents of T drafted tokens."""
    return [rng.choice([t - 1, rng.randrange(-1, t)]) if t else -1 for t in range(T)]


def tree_rows(bits, T, new, count, k_cap, positions, q_pos, window):
    """(seen [T, k_cap], dist [T, k_cap]) of a sequence and KV head; bits: a set of drafted tokens for each t; positions [k_cap] and
    q_pos [T] as lists, or None."""
    past, n = max(count, 0) - new, min(max(count, 0), k_cap)
    depth = [len([u for u in bits[t] if u < new and u != t]) for t in range(T)]
    at = [past + depth[t] for t in range(T)] if q_pos is None else q_pos
    pos = list(positions) if positions is not None else [j if j < past else past + depth[min(j - past, T - 1)] for j in range(k_cap)]
    j, p, a = torch.arange(k_cap), torch.tensor(pos), torch.tensor(at)[:, None]
    sees = torch.zeros(T, k_cap, dtype=torch.bool)
    for t in range(min(new, T)):
        for u in bits[t]:
            if u < new and 0 <= past + u < k_cap:
                sees[t, past + u] = True
    seen = torch.where(j < past, p <= a, sees) & (j < n)
    if positions is not None:
        seen &= p >= 0
    if window:
        seen &= p > a - window
    seen[min(new, T):] = False
    return seen.to(DEV), (a - p).abs().to(DEV)


def infinite_sums(V, seen):
    """[T, d]: the sum of those values of V that are not finite and that a row sees (0: none)."""
    odd = torch.where(torch.isfinite(V.double()), 0.0, V.double())
    plus, minus, nan = (seen.double() @ (x.double()) > 0 for x in (odd == math.inf, odd == -math.inf, torch.isnan(odd)))
    return torch.where(nan | (plus & minus), math.nan, torch.where(plus, math.inf, torch.where(minus, -math.inf, 0.0)))


def check_rows(out, lse, q, K, V, seen, dist, scale, dtype, cap=0.0, slope=None, rows=1):
    """One head's outputs [T, d] and lse [T] against 64 bits; rows: query rows of the KV head, by which the weights are rounded."""
    odd = infinite_sums(V, seen)
    Vf = torch.where(torch.isfinite(V), V, 0)
    any_seen = seen.any(0)
    Kf, Vf = K.clone(), Vf.clone()
    Kf[~any_seen] = 0
    token = rows <= 32
    want = attention_bounds.attend(q, Kf, Vf, seen, dist, scale, dtype, cap, slope, (TOKEN if token else PROMPT)[dtype],
                                   (TOKEN_SMALL if token else PROMPT_SMALL)[dtype])
    special = odd != 0
    assert torch.equal(torch.isnan(out[special]), torch.isnan(odd[special]))
    fine = special & ~torch.isnan(odd)
    assert torch.equal(out[fine].double(), odd[fine])
    attention_bounds.check(torch.where(special, want[0].to(out.dtype), out), lse, *want)
    none = ~seen.any(1)
    assert not out[none].any()


def weights_of(q, K, seen, dist, scale, cap=0.0, slope=None):
    """(weights [n], room [n]) of query heads q [G, d] over one KV head: their sum of softmax weights in 64 bits, and how far it may be
    off.  A weight is exp(s - lse): the errors of a score and of the log-sum-exp as attention_bounds has them, the difference's
    rounding and the exponential; then G additions, and the smallest normal fp32 of each."""
    G, n = q.shape[0], K.shape[0]
    total, room = torch.zeros(n, dtype=torch.float64, device=DEV), torch.zeros(n, dtype=torch.float64, device=DEV)
    for h in range(G):
        sl = None if slope is None else float(slope[h])
        _, lse, _, lse_room = attention_bounds.attend(q[h][None], K, torch.zeros_like(K), seen[None], dist[None], scale, torch.bfloat16, cap, sl)
        if not bool(seen.any()):
            continue
        s = (q[h].double() @ K.double().t()) * scale
        err = (K.shape[1] + 2) * 2.0 ** -23 * (q[h].double().abs() @ K.double().abs().t()) * scale + 2.0 ** -23 * s.abs()
        if cap:
            y = s / cap
            s = cap * torch.tanh(y)
            err = torch.where(y.abs() < 0.359, err + 7 * 2.0 ** -24 * s.abs(), err + 2.0 ** -21 * cap)
        if sl is not None:
            s = s - sl * dist
            err = err + 2.0 ** -22 * abs(sl) * dist + 2.0 ** -24 * s.abs()
        w = torch.where(seen, torch.exp(s - lse), 0.0)
        total += w
        room += 1.01 * w * (err + lse_room + 2.0 ** -23 * (s - lse).abs() + 2.0 ** -21) + 2.0 ** -126 * seen
    return total, room + (G + 1) * 2.0 ** -24 * total


def evicted(pos, w, n, budget, recent, first):
    """Rows whose content is in rows 0 .. min(n, budget) - 1 after the eviction of one head: pos, w lists."""
    if n <= budget:
        return list(range(n))
    newest = max([p for p in pos[:n]] + [-1])

    def rank(r):
        p, x = pos[r], w[r]
        if p < 0:
            return (3, 0.0, r)
        if p < first or p > newest - recent:
            return (0, 0.0, r)
        return (2, 0.0, r) if math.isnan(x) else (1, -x, r)

    stay = set(sorted(range(n), key=rank)[:budget])
    late = iter(sorted(r for r in stay if r >= budget))
    return [r if r in stay else next(late) for r in range(budget)]


def bounds_of(K, n, block, absent=None):
    """[blocks, 2, d] of one head's rows K [k, d]."""
    d = K.shape[1]
    out = torch.zeros(-(-n // block), 2, d, dtype=K.dtype, device=K.device)
    for k in range(out.shape[0]):
        rows = torch.arange(k * block, min(n, (k + 1) * block), device=K.device)
        if absent is not None:
            rows = rows[~absent[rows]]
        if len(rows) == 0:
            continue
        x = K[rows].float()
        nan = torch.isnan(x).any(0)
        out[k, 0] = torch.where(nan, -math.inf, torch.nan_to_num(x, nan=0.0, posinf=math.inf, neginf=-math.inf).amin(0)).to(K.dtype)
        out[k, 1] = torch.where(nan, math.inf, torch.nan_to_num(x, nan=0.0, posinf=math.inf, neginf=-math.inf).amax(0)).to(K.dtype)
    return out


def block_scores(q, bounds):
    """fp32 [blocks] of query heads q [G, d] and bounds [blocks, 2, d]: in 64 bits, rounded once."""
    q, b = q.double()[:, None], bounds.double()[None]
    lo, hi = b[:, :, 0], b[:, :, 1]
    s = torch.where(q < 0, q * lo, q * hi)
    s = s.sum((0, 2)).float()
    return torch.where(torch.isnan(s), math.inf, s)


def blocks_taken(score, most, first, recent):
    """The listed blocks of one head, ascending, -1 behind."""
    have = len(score)
    s = score.tolist()
    rank = sorted(range(have), key=lambda k: (0 if k < first or k >= have - recent else 1, 0.0 if k < first or k >= have - recent else -s[k], k))
    taken = sorted(rank[:most])
    return taken + [-1] * (most - len(taken))

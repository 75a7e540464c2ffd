"""Plain attention in 64 bits for the tests of the kernels over whole caches, with what their tolerance is made of."""
import math

import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def attend(q, K, V, seen, dist, scale, cap=0.0, slope=None):
    """One head: q [n, d], K and V [m, d], seen [n, m] (bool), dist [n, m], slope a number or None.
    Returns (out [n, d], lse [n], room [n, d], lse_room [n]) in 64 bits: keys that are not seen count as absent."""
    q, K, V = q.double(), K.double(), V.double()
    any_seen = seen.any(0)
    K, V = K.clone(), V.clone()
    K[~any_seen], V[~any_seen] = 0, 0
    s = q @ K.t() * scale
    if cap:
        s = cap * torch.tanh(s / cap)
    if slope is not None:
        s = s - slope * dist.abs()
    s = s.masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - lse.masked_fill(torch.isinf(lse), 0)[:, None])
    out, spread = p @ V, p @ V.abs()
    # A score's error: d + 2 roundings of partial sums below sum |q k|, the tanh's 2^-22 cap, two roundings of the bias and
    # of the sum with it.  It weighs where the weight is above 2^-40.
    size = q.abs() @ K.abs().t() * scale * ((q.shape[1] + 2) * 2.0 ** -24) + cap * 2.0 ** -22
    if slope is not None:
        size = size + 2.0 ** -23 * (slope * dist.abs() + s.masked_fill(~seen, 0).abs())
    err = torch.where(p > 2.0 ** -40, size, torch.zeros_like(size)).amax(-1)
    return out, lse, (2 * err[:, None] + 2.0 ** -14) * spread, err + 2.0 ** -20 + 2.0 ** -22 * lse.abs().masked_fill(torch.isinf(lse), 0)


def check(got, got_lse, out, lse, room, lse_room, dtype, weights=0.0):
    """got against out: half a step of the type, and `room` for scores and sums in 32 bits (2^-14: chains of up to 1024
    additions); weights: relative rounding of the softmax weights times their spread, as `room` has it per 2^-14."""
    tol = HALF_STEP[dtype] * out.abs() + room * (1 + HALF_STEP[dtype]) + weights * room * 2.0 ** 14 + \
        (2.0 ** -25 if dtype == torch.float16 else 0.0)
    err = (got.double() - out).abs()
    assert bool((err <= tol).all()), (float((err - tol).max()), float(err.max()))
    if got_lse is not None:
        none = torch.isneginf(lse)
        assert torch.equal(torch.isneginf(got_lse.double()), none)
        assert bool(((got_lse.double() - lse).abs().masked_fill(none, 0) <= lse_room).all())

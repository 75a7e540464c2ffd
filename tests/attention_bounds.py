"""Plain attention in 64 bits, and how far a kernel in 32 bits with 16-bit operands may be from it, term by term.

A score's error e_j, in nats, is the relative error of its weight w_j (the softmax' value):
  products   d + 2 additions of a matrix instruction, which may cut off instead of rounding: 2^-23 each of sum |q k| scale
  scale      its own rounding and the product's: 2^-23 |s|
  cap        up to |s / cap| = 0.36 a polynomial: the fit 2^-24, six roundings of 2^-24 of the score; beyond it a sum and a
             reciprocal: 2^-21 cap
  bias       the slope's conversion, the distance, their product and the sum: 2^-22 slope |distance| + 2^-24 |s|
  exponent   rounding of the argument, 2^-24 of its distance from the largest score, and the exponential's 2^-22
Then, with spread = sum w |V|:
  out        sum w e (|V| + |out|), since what all weights share divides out; `weights` spread for weights that are rounded;
             `small` sum |V| where they have a least step (`small` in units of the largest weight: a row's sum is 1 at least);
             n / 8 + 64 additions and rescalings of 2^-23 in the sums of n keys; half a step of the result's type;
             2^-126 (sum |V| + 1): fp32 and bf16 have no normal numbers below that, and a weight or a result that is
             smaller may be taken as 0 (e^-120, a key 120 nats below the largest, is 2^-173, which fp32 does not hold at all)
  lse        sum w e, the same additions, 2^-22 of itself and of ln n
First-order terms are multiplied by 1.01 for the products of errors."""
import math

import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def attend(q, K, V, seen, dist, scale, dtype, cap=0.0, slope=None, weights=0.0, small=0.0):
    """One head: q [m, d], K and V [n, d], seen [m, n] (bool), dist [m, n] (query's position minus the key's), slope a number
    or None.  Returns (out [m, d], lse [m], room of out, room of lse) in 64 bits; rows that see nothing: 0 and -inf."""
    q, K, V = q.double(), K.double(), V.double()
    n, d = K.shape
    far = dist.abs().double()
    s = q @ K.t() * scale
    err = (d + 2) * 2.0 ** -23 * (q.abs() @ K.abs().t()) * scale + 2.0 ** -23 * s.abs()
    if cap:
        y = s / cap
        s = cap * torch.tanh(y)
        err = torch.where(y.abs() < 0.359, err + 7 * 2.0 ** -24 * s.abs(), err + 2.0 ** -21 * cap)
    if slope is not None:
        s = s - slope * far
        err = err + 2.0 ** -22 * abs(slope) * far + 2.0 ** -24 * s.abs()
    s = s.masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(s, -1)
    none = torch.isneginf(lse)
    base = lse.masked_fill(none, 0)[:, None]
    w = torch.exp(s - base)
    err = (err + 2.0 ** -24 * (s - base).abs() + 2.0 ** -22).masked_fill(~seen, 0)
    Vs = V.masked_fill(~seen.any(0)[:, None], 0)
    size = Vs.abs()
    out, spread = w @ Vs, w @ size
    we = w * err.clamp(max=1e300)
    chain = (n / 8 + 64) * 2.0 ** -23
    room = we @ size + we.sum(-1, keepdim=True) * out.abs() + weights * spread + small * (seen.double() @ size) + \
        chain * (spread + out.abs())
    room = 1.01 * room * (1 + HALF_STEP[dtype]) + HALF_STEP[dtype] * out.abs() + (2.0 ** -25 if dtype == torch.float16 else 0.0) + \
        2.0 ** -126 * (seen.double() @ size + 1)
    lse_room = 1.01 * (we.sum(-1) + chain + 2.0 ** -22 * (lse.masked_fill(none, 0).abs() + math.log(n) + 1))
    return out, lse, room, lse_room


def fits(got, got_lse, out, lse, room, lse_room):
    """(whether the outputs are within their room, whether the log-sum-exps are)"""
    fine = bool(((got.double() - out).abs() <= room).all())
    if got_lse is None:
        return fine, True
    none = torch.isneginf(lse)
    return fine, torch.equal(torch.isneginf(got_lse.double()), none) and \
        bool(((got_lse.double() - lse).abs().masked_fill(none, 0) <= lse_room).all())


def check(got, got_lse, out, lse, room, lse_room):
    assert bool((~torch.isnan(got)).all())
    worst = float(((got.double() - out).abs() / room).max())
    worst_lse = 0.0 if got_lse is None else float(((got_lse.double() - lse).abs().masked_fill(torch.isneginf(lse), 0) / lse_room).max())
    assert fits(got, got_lse, out, lse, room, lse_room) == (True, True), (worst, worst_lse)

"""The tolerances of tests/attention_bounds.py tell right results from wrong ones (no GPU)."""
import math

import pytest
import torch

from tests.attention_bounds import HALF_STEP, attend, fits

# (dtype, d, query rows = keys, cap, scale, slope, spread of the queries): what the GPU tests of these bounds run
CASES = [(torch.float16, 64, 3, 2.0, None, None, 1.0), (torch.float16, 64, 130, 2.0, None, None, 1.0), (torch.float16, 64, 130, 50.0, None, None, 1.0),
         (torch.float16, 64, 130, 5.0, 1.0, None, 1.0), (torch.float16, 64, 130, 1e-3, None, None, 1.0), (torch.float16, 64, 130, 1e6, None, None, 1.0),
         (torch.float16, 64, 3, 1e6, None, None, 1.0), (torch.bfloat16, 128, 150, 0.0, 5.0, None, 1.0), (torch.bfloat16, 128, 200, 0.0, None, 0.25, 1.5),
         (torch.bfloat16, 64, 333, 50.0, None, None, 1.5), (torch.float16, 128, 300, 30.0, None, 2.0 ** -5, 1.5), (torch.bfloat16, 128, 1000, 1e6, None, None, 1.5)]


@pytest.mark.parametrize("dtype,d,T,cap,scale,slope,wide", CASES)
def test_wrong_results_are_refused(dtype, d, T, cap, scale, slope, wide):
    g = torch.Generator().manual_seed(T + d)
    q, K, V = ((torch.randn(T, d, generator=g) * f).to(dtype) for f in (wide, 1.0, 1.0))
    dist = torch.arange(T)[:, None] - torch.arange(T)
    seen = dist >= 0
    out, lse, room, lse_room = attend(q, K, V, seen, dist, scale or d ** -0.5, dtype, cap, slope, weights=HALF_STEP[dtype])
    ok = lambda x, z=None: fits(x, lse if z is None else z, out, lse, room, lse_room)
    assert ok(out.to(dtype), lse.float()) == (True, True)
    assert not ok(torch.zeros_like(out))[0] and not ok(-out)[0] and not ok(V.double())[0]
    mean = torch.stack([V[:t + 1].double().mean(0) for t in range(T)])
    if cap != 1e-3:                                        # (there all scores are next to 0: the mean is what is right)
        assert not ok(mean)[0]
    assert not ok(out, lse + 2e-3 * (1 + lse.abs()))[1]
    assert not ok(out * (1 + 4 * HALF_STEP[dtype]) + 8 * HALF_STEP[dtype])[0]


def test_an_inexact_tanh_is_refused():
    # cap - 2 cap / (1 + e^(2 s / cap)) in 32 bits is off by 2^-23 cap: nothing at a cap of 50, a tenth of a nat at a million
    g = torch.Generator().manual_seed(3)
    T, d, cap = 130, 64, 1e6
    q, K, V = (torch.randn(T, d, generator=g).half() for _ in range(3))
    dist = torch.arange(T)[:, None] - torch.arange(T)
    seen = dist >= 0
    out, lse, room, lse_room = attend(q, K, V, seen, dist, d ** -0.5, torch.float16, cap, weights=2.0 ** -11)
    s = (q.double() @ K.double().t() * d ** -0.5).float()
    s = (cap - 2 * cap / (1 + torch.exp(2 * s / cap))).double().masked_fill(~seen, -math.inf)
    got = (torch.softmax(s, -1) @ V.double()).half()
    assert fits(got, torch.logsumexp(s, -1), out, lse, room, lse_room) == (False, False)


def test_rows_that_see_nothing():
    q, K, V = torch.ones(2, 64).half(), torch.ones(3, 64).half(), torch.ones(3, 64).half()
    seen = torch.tensor([[True, False, False], [False, False, False]])
    out, lse, room, lse_room = attend(q, K, V, seen, torch.zeros(2, 3), 0.125, torch.float16)
    assert not out[1].any() and bool(torch.isneginf(lse[1]))
    assert fits(out, lse, out, lse, room, lse_room) == (True, True)
    assert not fits(out, torch.zeros(2), out, lse, room, lse_room)[1]

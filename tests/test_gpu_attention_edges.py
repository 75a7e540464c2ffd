"""Attention where weights, values and scores lie far apart: prompt attention and attention of one token."""
import math

import pytest
import torch

from paper_2406_02069_amd import binding
from tests.attention_bounds import HALF_STEP, attend, check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _sink(B, Hq, Hkv, d, n, gap, size, dtype, at=0):
    """(q [B,Hq,d], K, V [1,Hkv,n,d]): all keys score 0, but for one that is `gap` nats above them and has no value (an
    attention sink); the others' values lie around `size`, so that what rounds all weights the same way does not average out."""
    g = torch.Generator(device=DEV).manual_seed(n + d)
    q, K = torch.zeros(B, Hq, d, dtype=dtype, device=DEV), torch.zeros(1, Hkv, n, d, dtype=dtype, device=DEV)
    q[..., 0], K[:, :, at, 0] = math.sqrt(d), gap                      # scale 1 / sqrt(d)
    V = (size * (1 + 0.25 * torch.randn(1, Hkv, n, d, generator=g, device=DEV))).to(dtype)
    V[:, :, at] = 0
    return q, K, V


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("B,Hq,Hkv,d,n", [(1, 8, 1, 64, 256), (1, 40, 1, 64, 256), (300, 68, 2, 64, 2000), (1, 16, 2, 64, 5000), (3, 64, 1, 64, 9001)])
@pytest.mark.parametrize("gap,size", [(9, 1.0), (12, 1.0), (15, 1.0), (18, 1.0), (18, 1000.0), (20, 1000.0)])
def test_one_token_weights_far_below_the_largest(B, Hq, Hkv, d, n, gap, size, dtype):
    # with 33 to 64 heads a group one wave has all of a range's keys, its largest weight among them.  A weight has two
    # roundings of the type, the second one 2^-25 at least in units of 2^-13 of the reference
    q, K, V = _sink(B, Hq, Hkv, d, n, gap, size, dtype, 5)
    count = torch.full((B,), n, dtype=torch.int32, device=DEV)
    out, lse = binding.decode_attention_long(q, K.expand(B, Hkv, n, d), V.expand(B, Hkv, n, d), count, want_lse=True)
    torch.cuda.synchronize()
    small = 2.0 ** -38 if dtype == torch.float16 else 0.0
    seen, dist = torch.ones(1, n, dtype=torch.bool, device=DEV), torch.zeros(1, n, device=DEV)
    for kv in range(Hkv):
        want = attend(q[0, 0][None], K[0, kv], V[0, kv], seen, dist, d ** -0.5, dtype, weights=HALF_STEP[dtype] ** 2, small=small)
        for b in {0, B - 1}:
            for h in range(kv * Hq // Hkv, (kv + 1) * Hq // Hkv):
                check(out[b, h][None], lse[b, h][None], *want)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d,T,n", [(64, 4, 300), (128, 40, 2000), (64, 9, 9001)])
@pytest.mark.parametrize("gap,size", [(9, 1.0), (12, 1.0), (15, 1.0), (18, 1.0), (18, 1000.0), (20, 1000.0)])
def test_prompt_weights_far_below_the_largest(d, T, n, gap, size, dtype):
    # a weight has one rounding of the type, 2^-25 at least in units of 2^-8 of the reference
    q, K, V = _sink(1, 2, 1, d, n, gap, size, dtype, 5)
    out, lse = binding.prefill_attention(q[:, :, None].expand(1, 2, T, d), K, V, q_start=torch.tensor([n - T], dtype=torch.int32, device=DEV),
                                         want_lse=True)
    torch.cuda.synchronize()
    dist = n - T + torch.arange(T, device=DEV)[:, None] - torch.arange(n, device=DEV)
    small = 2.0 ** -33 if dtype == torch.float16 else 0.0
    want = attend(q[0, :1].expand(T, d), K[0, 0], V[0, 0], dist >= 0, dist, d ** -0.5, dtype, weights=HALF_STEP[dtype], small=small)
    for h in range(2):
        check(out[0, h], lse[0, h], *want)

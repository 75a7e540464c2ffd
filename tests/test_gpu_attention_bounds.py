"""Prompt attention and attention of one token within the bounds that tests/attention_bounds.py derives term by term: at caps
near and far from the scores, scales, biases, windows and types."""
import pytest
import torch

from paper_2406_02069_amd import binding
from tests.attention_bounds import HALF_STEP, attend, check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# Rounding of a weight for the product with V: once to the type (prompt), to two numbers of the type (one token; what the
# first leaves is 2^-8 or 2^-11 of it, and is rounded by as much).
PROMPT = HALF_STEP
TOKEN = {t: h * h for t, h in HALF_STEP.items()}
# Half the type's last step, in units of the largest weight.
PROMPT_SMALL = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -33}
TOKEN_SMALL = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -38}


@pytest.mark.parametrize("dtype,Hq,Hkv,d,T,cap,scale,slope,wide,window", [
    (torch.float16, 4, 2, 64, 3, 2.0, None, None, 1.0, 0), (torch.float16, 4, 2, 64, 130, 2.0, None, None, 1.0, 0),
    (torch.float16, 4, 2, 64, 130, 50.0, None, None, 1.0, 0), (torch.float16, 4, 2, 64, 130, 5.0, 1.0, None, 1.0, 0),
    (torch.float16, 4, 2, 64, 130, 1e-3, None, None, 1.0, 0), (torch.float16, 4, 2, 64, 130, 1e6, None, None, 1.0, 0),
    (torch.float16, 4, 2, 64, 3, 1e6, None, None, 1.0, 0), (torch.bfloat16, 4, 2, 128, 150, 0.0, 5.0, None, 1.0, 0),
    (torch.bfloat16, 6, 2, 128, 200, 0.0, None, 0.25, 1.5, 0), (torch.bfloat16, 7, 1, 64, 333, 50.0, None, None, 1.5, 0),
    (torch.float16, 4, 4, 128, 300, 30.0, None, 2.0 ** -5, 1.5, 129), (torch.bfloat16, 2, 1, 128, 1000, 1e6, None, None, 1.5, 0),
    (torch.bfloat16, 1, 1, 64, 1, 0.0, None, None, 1.0, 0), (torch.float16, 2, 1, 128, 4000, 0.0, None, None, 1.5, 700)])
def test_prompt(dtype, Hq, Hkv, d, T, cap, scale, slope, wide, window):
    print("bounds prompt", dtype, Hq, Hkv, d, T, cap, scale, slope, wide, window, flush=True)
    g = torch.Generator(device=DEV).manual_seed(T + d)
    q = (torch.randn(1, Hq, T, d, generator=g, device=DEV) * wide).to(dtype)
    K, V = (torch.randn(1, Hkv, T, d, generator=g, device=DEV).to(dtype) for _ in range(2))
    sl = None if slope is None else torch.full((Hq,), slope, device=DEV)
    out, lse = binding.prefill_attention(q, K, V, cap=cap, scale=scale, slopes=sl, window=window, want_lse=True)
    torch.cuda.synchronize()
    dist = torch.arange(T, device=DEV)[:, None] - torch.arange(T, device=DEV)
    seen = (dist >= 0) & (dist < (window or T))
    for h in range(Hq):
        check(out[0, h], lse[0, h], *attend(q[0, h], K[0, h * Hkv // Hq], V[0, h * Hkv // Hq], seen, dist, scale or d ** -0.5, dtype, cap,
                                            slope, PROMPT[dtype], PROMPT_SMALL[dtype]))


@pytest.mark.parametrize("T,N,window,dtype", [(70, 9000, 0, torch.bfloat16), (33, 5000, 1500, torch.float16)])
def test_chunk_in_ranges(T, N, window, dtype):
    Hq, Hkv, d = 4, 2, 128
    g = torch.Generator(device=DEV).manual_seed(N)
    q = torch.randn(1, Hq, T, d, generator=g, device=DEV).to(dtype)
    K, V = (torch.randn(1, Hkv, N, d, generator=g, device=DEV).to(dtype) for _ in range(2))
    out, lse = binding.prefill_attention(q, K, V, q_start=torch.tensor([N - T], dtype=torch.int32, device=DEV), window=window, want_lse=True)
    torch.cuda.synchronize()
    dist = N - T + torch.arange(T, device=DEV)[:, None] - torch.arange(N, device=DEV)
    seen = (dist >= 0) & (dist < (window or N))
    for h in range(Hq):
        check(out[0, h], lse[0, h], *attend(q[0, h], K[0, h // 2], V[0, h // 2], seen, dist, d ** -0.5, dtype, 0.0, None, PROMPT[dtype], PROMPT_SMALL[dtype]))


@pytest.mark.parametrize("dtype,Hq,Hkv,d,n,cap,scale,slope,window", [
    (torch.float16, 4, 2, 64, 3, 2.0, None, None, 0), (torch.float16, 8, 2, 64, 1000, 1e6, None, None, 0),
    (torch.bfloat16, 8, 1, 128, 5000, 50.0, None, None, 0), (torch.bfloat16, 40, 1, 128, 700, 5.0, 1.0, None, 0),
    (torch.float16, 7, 1, 128, 3000, 1e-3, None, 0.25, 0), (torch.bfloat16, 8, 2, 128, 9000, 0.0, 3.0, None, 2500),
    (torch.bfloat16, 4, 4, 64, 1, 0.0, None, None, 0), (torch.float16, 33, 1, 128, 257, 30.0, None, 2.0 ** -5, 0)])
def test_one_token(dtype, Hq, Hkv, d, n, cap, scale, slope, window):
    print("bounds token", dtype, Hq, Hkv, d, n, cap, scale, slope, window, flush=True)
    g = torch.Generator(device=DEV).manual_seed(n + d)
    q = torch.randn(1, Hq, d, generator=g, device=DEV).to(dtype)
    K, V = (torch.randn(1, Hkv, n, d, generator=g, device=DEV).to(dtype) for _ in range(2))
    sl = None if slope is None else torch.full((Hq,), slope, device=DEV)
    out, lse = binding.decode_attention_long(q, K, V, torch.tensor([n], dtype=torch.int32, device=DEV), cap=cap, scale=scale, slopes=sl,
                                             window=window, want_lse=True)
    torch.cuda.synchronize()
    dist = (n - 1 - torch.arange(n, device=DEV))[None]
    seen = dist < (window or n)
    for h in range(Hq):
        kv = h * Hkv // Hq
        check(out[0, h][None], lse[0, h][None], *attend(q[0, h][None], K[0, kv], V[0, kv], seen, dist, scale or d ** -0.5, dtype, cap, slope,
                                                        TOKEN[dtype], TOKEN_SMALL[dtype]))

"""Attention of a prompt (pkv_prefill_attention) against plain attention in 64 bits, row by row."""
import math

import pytest
import torch

from paper_2406_02069_amd import binding
from tests.attention_ref import HALF_STEP, attend, check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _make(B, Hq, Hkv, d, T, N, dtype, seed, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    q = (torch.randn(B, Hq, T, d, generator=g, device=DEV) * scale).to(dtype)
    K = torch.randn(B, Hkv, N, d, generator=g, device=DEV).to(dtype)
    V = torch.randn(B, Hkv, N, d, generator=g, device=DEV).to(dtype)
    return q, K, V, g


def _seen(N, n, start, T, window=0, doc=None, pre=None):
    """(seen [T, N], distance [T, N]) of one sequence."""
    p = start + torch.arange(T, device=DEV)
    j = torch.arange(N, device=DEV)
    there = (p >= 0) & (p < n)
    at = p.clamp(0, N - 1)
    hi = p if pre is None else torch.maximum(p, pre[at].long() - 1)
    lo = torch.zeros_like(p) if doc is None else doc[at].long()
    if window:
        lo = torch.maximum(lo, p - window + 1)
    seen = (j >= lo[:, None]) & (j <= hi[:, None]) & there[:, None] & (j < n)
    return seen, p[:, None] - j


def _compare(out, lse, q, K, V, lens=None, start=None, doc=None, pre=None, slopes=None, cap=0.0, window=0, scale=None, heads=None):
    B, Hq, T, d = q.shape
    N, G = K.shape[2], Hq // K.shape[1]
    for b in range(B):
        n = N if lens is None else min(max(int(lens[b]), 0), N)
        s0 = 0 if start is None else int(start[b])
        for h in heads or range(Hq):
            for t0 in range(0, T, 2048):
                t1 = min(T, t0 + 2048)
                seen, dist = _seen(N, n, s0 + t0, t1 - t0, window, None if doc is None else doc[b], None if pre is None else pre[b])
                want = attend(q[b, h, t0:t1], K[b, h // G], V[b, h // G], seen, dist, d ** -0.5 if scale is None else scale, cap,
                              None if slopes is None else float(slopes[h]))
                check(out[b, h, t0:t1], None if lse is None else lse[b, h, t0:t1], *want, q.dtype, weights=HALF_STEP[q.dtype])
                none = ~seen.any(1)
                assert not out[b, h, t0:t1][none].any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("B,Hq,Hkv,d,T,cap,slopes,window", [
    (1, 1, 1, 64, 1, 0.0, False, 0), (2, 4, 2, 128, 1, 20.0, True, 0), (1, 8, 8, 64, 37, 0.0, False, 0), (3, 6, 2, 128, 64, 0.0, True, 0),
    (2, 4, 1, 128, 65, 0.0, False, 16), (1, 7, 1, 64, 333, 50.0, False, 0), (2, 32, 8, 128, 200, 0.0, False, 1),
    (1, 4, 4, 128, 1000, 30.0, True, 129), (1, 128, 1, 64, 19, 0.0, False, 0), (1, 2, 1, 128, 5001, 0.0, False, 0),
    (1, 2, 2, 64, 3000, 0.0, False, 700)])
def test_whole_prompts(B, Hq, Hkv, d, T, cap, slopes, window, dtype):
    print("prefill", B, Hq, Hkv, d, T, cap, slopes, window, dtype, flush=True)
    q, K, V, _ = _make(B, Hq, Hkv, d, T, T, dtype, T + d + Hq, 1.5)
    sl = 2.0 ** (-8.0 * torch.arange(1, Hq + 1, device=DEV) / Hq) if slopes else None
    out, lse = binding.prefill_attention(q, K, V, slopes=sl, cap=cap, window=window, want_lse=True)
    torch.cuda.synchronize()
    _compare(out, lse, q, K, V, slopes=sl, cap=cap, window=window)


@pytest.mark.parametrize("T,N,Hq,Hkv,d", [(1, 900, 8, 2, 128), (5, 64, 4, 4, 64), (130, 4000, 8, 2, 128), (32, 20000, 32, 8, 128),
                                          (64, 700, 6, 3, 64), (700, 1500, 4, 1, 128)])
def test_chunks_and_ragged_batches(T, N, Hq, Hkv, d):
    # query rows in front of, inside and behind the valid positions; K and V behind a sequence's end are never used
    B = 4
    print("prefill chunk", T, N, Hq, Hkv, d, flush=True)
    q, K, V, g = _make(B, Hq, Hkv, d, T, N, torch.bfloat16, N + T)
    lens = torch.tensor([N, max(N // 3, 1), 0, N + 50], dtype=torch.int32, device=DEV)
    start = torch.tensor([N - T, N // 3 - T // 2, 0, -(T // 2)], dtype=torch.int32, device=DEV)
    q[:, :, 0] *= 3
    for b in range(B):
        K[b, :, min(int(lens[b]), N):], V[b, :, min(int(lens[b]), N):] = math.nan, math.inf
    out, lse = binding.prefill_attention(q, K, V, seq_lens=lens, q_start=start, want_lse=True)
    torch.cuda.synchronize()
    assert not bool(torch.isnan(out).any())
    _compare(out, lse, q, K, V, lens, start)


@pytest.mark.parametrize("prefix,window,slopes,N,docs", [(False, 0, False, 1000, [1, 1, 63, 64, 65, 400, 406]), (True, 0, False, 777, [300, 5, 472]),
                                                        (True, 90, True, 1500, [700, 800]), (True, 0, True, 130, [130]),
                                                        (False, 33, False, 4100, [2000, 100, 2000])])
def test_documents_and_prefixes(prefix, window, slopes, N, docs):
    B, Hq, Hkv, d = 2, 8, 2, 128
    q, K, V, g = _make(B, Hq, Hkv, d, N, N, torch.float16, N)
    lens = torch.tensor([N, N - 50], dtype=torch.int32, device=DEV)
    first = torch.tensor(docs).cumsum(0) - torch.tensor(docs)
    doc = first.repeat_interleave(torch.tensor(docs)).int()
    doc = torch.stack([doc, doc.roll(7).clamp(max=N)]).to(DEV).contiguous()       # (the second: documents out of order, some rows empty)
    pre = torch.stack([(first + torch.tensor(docs) // 3).repeat_interleave(torch.tensor(docs)).int()] * 2).to(DEV) if prefix else None
    if prefix:
        pre[1, :9] = 2 ** 31 - 1
        pre[1, 9:20] = -2 ** 31
        pre = pre.contiguous()
    doc[0, N // 2], doc[0, N // 2 + 1] = N + 5, -3                                 # sees nothing; sees all before it
    sl = torch.linspace(0.02, 0.5, Hq, device=DEV) if slopes else None
    out, lse = binding.prefill_attention(q, K, V, seq_lens=lens, doc_start=doc, prefix_end=pre, window=window, slopes=sl, want_lse=True)
    torch.cuda.synchronize()
    _compare(out, lse, q, K, V, lens, None, doc, pre, sl, 0.0, window)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,window,d", [(200, 0, 128), (300, 40, 64), (65, 0, 64)])
def test_hidden_keys_may_hold_anything(T, window, d, dtype):
    # a NaN or an infinity in K or V has no influence on the rows that do not see its key; the others are as plain attention has them
    q, K, V, g = _make(1, 4, 2, d, T, T, dtype, T)
    bad = [T - 1, T // 2, T // 2 + 1, 3]
    V[0, 0, bad[0], 5], V[0, 0, bad[1], :] = math.inf, math.nan
    V[0, 1, bad[2], d - 1], V[0, 1, bad[3], 0] = -math.inf, math.nan
    K[0, 0, bad[2], 7], K[0, 1, bad[0]] = math.nan, math.inf
    out, lse = binding.prefill_attention(q, K, V, window=window, want_lse=True)
    torch.cuda.synchronize()
    seen, dist = _seen(T, T, 0, T, window)
    for h in range(4):
        Kh, Vh = K[0, h // 2].double(), V[0, h // 2].double()
        for t in range(T):
            at = seen[t].nonzero()[:, 0]
            s = q[0, h, t].double() @ Kh[at].t() * d ** -0.5
            want = torch.softmax(s, 0) @ Vh[at]
            fine = torch.isfinite(want)
            got = out[0, h, t].double()
            assert torch.equal(torch.isnan(want), torch.isnan(got)), (h, t)
            assert torch.equal(want[torch.isinf(want)], got[torch.isinf(want)]), (h, t)
            assert bool(((got - want)[fine].abs() <= 3 * HALF_STEP[dtype] * Vh[at][:, fine].abs().nan_to_num(0, 0, 0).amax(0)).all()), (h, t)


def test_strides_scale_and_large_scores():
    B, Hq, Hkv, d, T = 2, 4, 2, 128, 150
    g = torch.Generator(device=DEV).manual_seed(5)
    x = torch.randn(B, T, Hq + 2 * Hkv, d, generator=g, device=DEV).to(torch.bfloat16).transpose(1, 2)
    q, K, V = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    room = torch.full((B, T, Hq, d), 7.0, dtype=torch.bfloat16, device=DEV)
    out, lse = binding.prefill_attention(q, K, V, scale=5.0, want_lse=True, out=room.transpose(1, 2))
    torch.cuda.synchronize()
    _compare(out, lse, q, K, V, scale=5.0)


def test_longest_offsets():
    # keys behind 2^31 elements of K: the last rows of a sequence of rows that lie far apart
    N, d, st = 2100, 128, 1 << 20
    big = torch.empty(2, N * st, dtype=torch.bfloat16, device=DEV)
    K, V = (big[i].view(1, 1, N, st)[..., :d] for i in range(2))
    q, Kn, Vn, g = _make(1, 2, 1, d, 70, N, torch.bfloat16, 8)
    K.copy_(Kn)
    V.copy_(Vn)
    start = torch.tensor([N - 70], dtype=torch.int32, device=DEV)
    out, lse = binding.prefill_attention(q, K, V, q_start=start, want_lse=True)
    torch.cuda.synchronize()
    _compare(out, lse, q, Kn, Vn, start=start)


def test_same_bits_every_time_on_another_stream_and_from_a_graph():
    for T, N in ((90, 3000), (700, 700)):                                         # with and without ranges of keys
        q, K, V, g = _make(2, 8, 2, 128, T, N, torch.bfloat16, 7)
        lens, start = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([N, N - 33], [N - T, N - T - 33]))
        call = lambda **kw: binding.prefill_attention(q, K, V, seq_lens=lens, q_start=start, **kw)
        out, lse = call(want_lse=True)
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            again = call(want_lse=True)
        torch.cuda.synchronize()
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
        ws = torch.empty(1 << 26, dtype=torch.uint8, device=DEV)
        o, z = torch.empty_like(out), torch.empty_like(lse)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call(out=o, lse=z, workspace=ws)
        for step in range(3):
            q.copy_(torch.randn(q.shape, generator=g, device=DEV))
            start -= 1
            ws.fill_(255)
            graph.replay()
            torch.cuda.synchronize()
            out, lse = call(want_lse=True)
            torch.cuda.synchronize()
            assert torch.equal(o, out) and torch.equal(z, lse)


@pytest.mark.parametrize("window", [0, 4096])
def test_a_long_prompt(window):
    q, K, V, g = _make(1, 4, 1, 128, 20000, 20000, torch.bfloat16, 11)
    K[:, :, 0] *= 4
    out, lse = binding.prefill_attention(q, K, V, window=window, want_lse=True)
    torch.cuda.synchronize()
    _compare(out, lse, q, K, V, window=window, heads=[0, 3])


@pytest.mark.parametrize("cap,scale", [(2.0, None), (50.0, None), (5.0, 1.0), (1e-3, None), (1e6, None)])
def test_caps_near_and_far_from_the_scores(cap, scale):
    # scores far below the cap, at it and far beyond; few keys, so that the log-sum-exp is as small as the scores
    for T in (3, 130):
        q, K, V, _ = _make(1, 4, 2, 64, T, T, torch.float16, 21)
        out, lse = binding.prefill_attention(q, K, V, cap=cap, scale=scale, want_lse=True)
        torch.cuda.synchronize()
        _compare(out, lse, q, K, V, cap=cap, scale=scale)


def test_more_query_rows_than_keys_and_two_calls_at_once():
    B, Hq, Hkv, d, T, N = 2, 4, 2, 64, 300, 70
    q, K, V, _ = _make(B, Hq, Hkv, d, T, N, torch.bfloat16, 17)
    lens, start = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([70, 33], [-100, 0]))
    out, lse = binding.prefill_attention(q, K, V, seq_lens=lens, q_start=start, want_lse=True)
    torch.cuda.synchronize()
    _compare(out, lse, q, K, V, lens, start)
    q, K, V, _ = _make(1, 8, 2, 128, 60, 9000, torch.float16, 18)
    start = torch.tensor([8900], dtype=torch.int32, device=DEV)
    ws = [torch.empty(1 << 25, dtype=torch.uint8, device=DEV) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [None, None]
    for rep in range(6):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i] = binding.prefill_attention(q, K, V, q_start=start, window=1000 * i, want_lse=True, workspace=ws[i])
    torch.cuda.synchronize()
    for i in range(2):
        _compare(*got[i], q, K, V, start=start, window=1000 * i)


def test_values_of_every_size_and_masked_rows_of_the_lowest_value():
    # scores over the whole range of the type, some keys at its lowest value: rows whose scores are all far below zero
    T, d = 96, 64
    q, K, V, g = _make(1, 2, 1, d, T, T, torch.float16, 19)
    q[0, 0] *= 30
    K[0, 0, 40:60] = torch.finfo(torch.float16).min
    q[0, 1] = q[0, 1].abs()                                   # its scores with those keys: about -4e5 each
    V[0, 0, ::7] *= 1000
    out, lse = binding.prefill_attention(q, K, V, want_lse=True)
    torch.cuda.synchronize()
    _compare(out, lse, q, K, V)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("B,T,N,Hq,Hkv,d,window,prefix,cap,lens,start", [
    (3, 40, 9000, 8, 2, 128, 0, False, 0.0, [9000, 1600, 0], None),                        # one long, one short, one empty
    (5, 300, 7000, 12, 4, 64, 900, False, 30.0, [7000, 6999, 77, 300, 1], None),
    (2, 129, 6200, 2, 1, 64, 0, True, 0.0, [6200, 5000], None), (2, 129, 3000, 2, 1, 64, 0, True, 0.0, [3000, 2000], None),
    (4, 70, 6500, 8, 8, 128, 0, False, 0.0, [6500, 2000, 1800, 6400], [-30, 1990, 1800, -70]),   # rows before, behind, none at all
    (3, 1500, 7001, 4, 2, 128, 0, False, 0.0, [7001, 900, 4000], [5501, -700, 3900]),
    (64, 2, 6400, 4, 1, 64, 0, False, 0.0, None, None), (65, 2, 6400, 4, 1, 64, 0, False, 0.0, None, None)])
def test_ragged_sequences_in_ranges(B, T, N, Hq, Hkv, d, window, prefix, cap, lens, start, dtype):
    print("ragged", B, T, N, Hq, Hkv, d, window, prefix, cap, dtype, flush=True)
    q, K, V, g = _make(B, Hq, Hkv, d, T, N, dtype, N + T)
    if lens is None:
        lens = torch.randint(0, N + 1, (B,), generator=torch.Generator().manual_seed(B)).tolist()
    lens_t = torch.tensor(lens, dtype=torch.int32, device=DEV)
    start_t = torch.tensor([n - T for n in lens] if start is None else start, dtype=torch.int32, device=DEV)
    pre = None
    if prefix:
        pre = torch.zeros(B, N, dtype=torch.int32, device=DEV)
        pre[:, ::3] = N - 5
    for b in range(B):
        K[b, :, lens[b]:], V[b, :, lens[b]:] = math.nan, math.inf
    out, lse = binding.prefill_attention(q, K, V, seq_lens=lens_t, q_start=start_t, prefix_end=pre, window=window, cap=cap, want_lse=True)
    torch.cuda.synchronize()
    _compare(out, lse, q, K, V, lens_t, start_t, pre=pre, window=window, cap=cap)

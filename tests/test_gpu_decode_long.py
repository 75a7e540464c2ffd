"""Attention of one token over caches of any length (pkv_decode_attention_long) against plain attention in 64 bits."""
import math

import pytest
import torch

from paper_2406_02069_amd import binding
from tests.attention_ref import attend, check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _make(B, Hq, Hkv, d, k_cap, dtype, page, seed, scale=1.0):
    """(q, K, V as rows, K, V as the call takes them, table)"""
    g = torch.Generator(device=DEV).manual_seed(seed)
    q = (torch.randn(B, Hq, d, generator=g, device=DEV) * scale).to(dtype)
    K = torch.randn(B, Hkv, k_cap, d, generator=g, device=DEV).to(dtype)
    V = torch.randn(B, Hkv, k_cap, d, generator=g, device=DEV).to(dtype)
    if not page:
        return q, K, V, K, V, None
    per = -(-k_cap // page)
    table = torch.randperm(B * per + 2, generator=g, device=DEV)[:B * per].to(torch.int32).view(B, per).contiguous()
    Kp = torch.full((B * per + 2, Hkv, page, d), math.nan, dtype=dtype, device=DEV)   # what no table names is never used
    Vp = Kp.clone()
    j = torch.arange(k_cap, device=DEV)
    for b in range(B):
        at = table[b].long()[j // page]
        Kp[at, :, j % page], Vp[at, :, j % page] = K[b].transpose(0, 1), V[b].transpose(0, 1)
    return q, K, V, Kp, Vp, table


def _compare(out, lse, q, K, V, count, dtype, positions=None, q_pos=None, slopes=None, cap=0.0, window=0, scale=None, absent=None):
    B, Hq, d = q.shape
    Hkv, k_cap = K.shape[1], K.shape[2]
    G = Hq // Hkv
    j = torch.arange(k_cap, device=DEV)
    for b in range(B):
        n = min(max(int(count[b]), 0), k_cap)
        at = n - 1 if q_pos is None else int(q_pos[b])
        for g in range(Hkv):
            pos = j if positions is None else positions[b, g, :k_cap].long()
            seen = (j < n) & (pos >= 0) & (pos <= at)
            if window:
                seen = seen & (pos > at - window)
            if absent is not None:
                seen = seen & ~absent[b]
            for h in range(g * G, g * G + G):
                want = attend(q[b, h][None], K[b, g], V[b, g], seen[None], (at - pos)[None], d ** -0.5 if scale is None else scale,
                              cap, None if slopes is None else float(slopes[h]))
                check(out[b, h][None], None if lse is None else lse[b, h][None], *want, dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("B,Hq,Hkv,d,k_cap,page,cap,slopes,window", [
    (3, 8, 8, 64, 1, 0, 0.0, False, 0), (4, 8, 2, 128, 31, 0, 30.0, False, 0), (4, 28, 4, 128, 33, 16, 0.0, True, 0),
    (2, 64, 1, 64, 700, 48, 50.0, True, 100), (2, 34, 2, 128, 1025, 1, 0.0, False, 7), (1, 128, 1, 128, 513, 0, 0.0, False, 0),
    (1, 40, 1, 64, 300, 7, 0.0, False, 0), (5, 6, 2, 128, 5000, 256, 0.0, True, 0), (1, 32, 8, 128, 40001, 16, 0.0, False, 0),
    (1, 4, 2, 64, 140000, 64, 20.0, False, 0), (2, 16, 16, 128, 9000, 0, 0.0, False, 2500)])
def test_rows(B, Hq, Hkv, d, k_cap, page, cap, slopes, window, dtype):
    print("decode long", B, Hq, Hkv, d, k_cap, page, cap, slopes, window, dtype, flush=True)
    q, K, V, Kc, Vc, table = _make(B, Hq, Hkv, d, k_cap, dtype, page, k_cap + d, 1.5)
    count = torch.tensor([k_cap, k_cap // 2, 0, 1, k_cap + 9][:B], dtype=torch.int32, device=DEV)
    sl = 2.0 ** (-8.0 * torch.arange(1, Hq + 1, device=DEV) / Hq) if slopes else None
    out, lse = binding.decode_attention_long(q, Kc, Vc, count, block_table=table, k_cap=k_cap, slopes=sl, cap=cap, window=window,
                                             want_lse=True)
    torch.cuda.synchronize()
    _compare(out, lse, q, K, V, count, dtype, slopes=sl, cap=cap, window=window)
    if B > 2:
        assert not out[2].any() and bool(torch.isneginf(lse[2]).all())


@pytest.mark.parametrize("slopes,window,page", [(False, 0, 0), (True, 900, 16), (True, 0, 5), (False, 40, 0)])
def test_positions_of_kept_rows(slopes, window, page):
    B, Hq, Hkv, d, k_cap = 4, 12, 4, 128, 610
    q, K, V, Kc, Vc, table = _make(B, Hq, Hkv, d, k_cap, torch.bfloat16, page, 3)
    g = torch.Generator(device=DEV).manual_seed(9)
    room = torch.randint(1, 6, (B, Hkv, k_cap + 3), generator=g, device=DEV).cumsum(2).to(torch.int32) - 1
    count = torch.tensor([610, 200, 33, 5], dtype=torch.int32, device=DEV)
    room[1, :, 200:] = -1                                  # as idx_out has it behind the count
    room[0, :, 17] = -1                                    # a hole
    q_pos = torch.tensor([int(room.max()) + 3, 500, 20, -1], dtype=torch.int32, device=DEV)   # rows behind the query; none at all
    sl = torch.linspace(0.01, 0.3, Hq, device=DEV) if slopes else None
    out, lse = binding.decode_attention_long(q, Kc, Vc, count, block_table=table, k_cap=k_cap, positions=room, q_pos=q_pos, slopes=sl,
                                             window=window, want_lse=True)
    torch.cuda.synchronize()
    _compare(out, lse, q, K, V, count, torch.bfloat16, room, q_pos, sl, 0.0, window)
    assert not out[3].any() and bool(torch.isneginf(lse[3]).all())


def test_what_is_not_seen_may_hold_anything():
    B, Hq, Hkv, d, k_cap, page = 3, 8, 2, 128, 400, 16
    q, K, V, Kc, Vc, table = _make(B, Hq, Hkv, d, k_cap, torch.float16, page, 4)
    count = torch.tensor([390, 77, 16], dtype=torch.int32, device=DEV)
    pos = torch.arange(k_cap, device=DEV, dtype=torch.int32).expand(B, Hkv, k_cap).contiguous()
    pos[:, :, 5::9] = -1
    absent = torch.zeros(B, k_cap, dtype=torch.bool, device=DEV)
    table[0, 3], table[1, 1] = 10 ** 6, -4                 # pages that do not exist
    absent[0, 48:64] = True
    absent[1, 16:32] = True
    for b in range(B):                                     # everything that is not seen: infinities and NaN
        for j in range(k_cap):
            if j >= int(count[b]) or int(pos[b, 0, j]) < 0:
                page_at = int(table[b, j // page])
                if 0 <= page_at < Kc.shape[0]:
                    Kc[page_at, :, j % page] = math.nan if j % 2 else math.inf
                    Vc[page_at, :, j % page] = -math.inf if j % 3 else math.nan
    out, lse = binding.decode_attention_long(q, Kc, Vc, count, block_table=table, k_cap=k_cap, positions=pos, want_lse=True)
    torch.cuda.synchronize()
    _compare(out, lse, q, K, V, count, torch.float16, positions=pos, absent=absent)


def test_strides_scale_and_large_scores():
    B, Hq, Hkv, d, k_cap = 2, 8, 2, 64, 300
    g = torch.Generator(device=DEV).manual_seed(5)
    qkv = torch.randn(B, 3, Hq, d, generator=g, device=DEV).to(torch.bfloat16)
    q = qkv[:, 1]
    buf = torch.randn(2, B, k_cap + 5, Hkv, d + 8, generator=g, device=DEV).to(torch.bfloat16)
    K, V = buf[0, :, :k_cap, :, :d].transpose(1, 2), buf[1, :, :k_cap, :, :d].transpose(1, 2)
    count = torch.tensor([300, 299], dtype=torch.int32, device=DEV)
    out, lse = binding.decode_attention_long(q, K, V, count, scale=6.0, want_lse=True)       # scores of some hundreds
    torch.cuda.synchronize()
    _compare(out, lse, q, K, V, count, torch.bfloat16, scale=6.0)


def test_longest_offsets():
    # a pool of 2^32 elements and a little: the last page is used
    d, Hkv, page = 128, 8, 128
    pages = 2 ** 32 // (Hkv * page * d) + 1
    K = torch.empty(pages, Hkv, page, d, dtype=torch.bfloat16, device=DEV)
    V = torch.empty(pages, Hkv, page, d, dtype=torch.bfloat16, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(6)
    K[-1], V[-1] = (torch.randn(Hkv, page, d, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    q = torch.randn(1, 8, d, generator=g, device=DEV).to(torch.bfloat16)
    table, count = torch.tensor([[pages - 1]], dtype=torch.int32, device=DEV), torch.tensor([128], dtype=torch.int32, device=DEV)
    out, lse = binding.decode_attention_long(q, K, V, count, block_table=table, want_lse=True)
    torch.cuda.synchronize()
    _compare(out, lse, q, K[-1:], V[-1:], count, torch.bfloat16)


def test_same_bits_every_time_on_another_stream_and_from_a_graph():
    B, Hq, Hkv, d, k_cap = 2, 32, 8, 128, 6000
    q, K, V, Kc, Vc, table = _make(B, Hq, Hkv, d, k_cap, torch.bfloat16, 16, 7)
    count = torch.tensor([6000, 2222], dtype=torch.int32, device=DEV)
    out, lse = binding.decode_attention_long(q, Kc, Vc, count, block_table=table, k_cap=k_cap, want_lse=True)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        again = binding.decode_attention_long(q, Kc, Vc, count, block_table=table, k_cap=k_cap, want_lse=True)
    torch.cuda.synchronize()
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    ws = torch.empty(1 << 24, dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    o, z = torch.empty_like(out), torch.empty_like(lse)
    with torch.cuda.graph(graph, stream=side):
        binding.decode_attention_long(q, Kc, Vc, count, block_table=table, k_cap=k_cap, out=o, lse=z, workspace=ws)
    for step in range(3):
        q.copy_(torch.randn(q.shape, device=DEV))
        count.copy_(torch.tensor([6000 - 999 * step, 17 + step], dtype=torch.int32))
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        out, lse = binding.decode_attention_long(q, Kc, Vc, count, block_table=table, k_cap=k_cap, want_lse=True)
        torch.cuda.synchronize()
        assert torch.equal(o, out) and torch.equal(z, lse)


def test_agrees_with_the_attention_over_compressed_caches():
    B, Hq, Hkv, d, k_cap = 3, 16, 4, 128, 1500
    q, K, V, _, _, _ = _make(B, Hq, Hkv, d, k_cap, torch.bfloat16, 0, 8)
    count = torch.tensor([1500, 64, 900], dtype=torch.int32, device=DEV)
    out, lse = binding.decode_attention_long(q, K, V, count, want_lse=True)
    ref, ref_lse = binding.decode_attention(q, K, V, count, want_lse=True)
    torch.cuda.synchronize()
    # the other call's values are within 1e-4 of the exact ones, ours within half a step and 2^-13 of the values' size
    assert bool(((out.float() - ref).abs() <= 2.0 ** -8 * ref.abs() + 5e-4).all())
    torch.testing.assert_close(lse, ref_lse, rtol=1e-5, atol=1e-4)


@pytest.mark.parametrize("B,Hkv,G,d,k_cap,page,window", [(64, 1, 3, 64, 3000, 0, 0), (65, 2, 2, 64, 1200, 16, 0), (300, 1, 1, 64, 700, 0, 0),
                                                       (7, 8, 4, 128, 6000, 16, 1000), (40, 8, 1, 64, 900, 0, 0), (2, 1, 70, 128, 9000, 0, 0)])
def test_ragged_batches_of_all_sizes(B, Hkv, G, d, k_cap, page, window):
    # ranges by the sequences' lengths, equal numbers of ranges, and none: sequences of all lengths, empty ones among them
    print("ragged", B, Hkv, G, d, k_cap, page, window, flush=True)
    q, K, V, Kc, Vc, table = _make(B, Hkv * G, Hkv, d, k_cap, torch.bfloat16, page, B)
    g = torch.Generator().manual_seed(B)
    count = torch.randint(0, k_cap + 1, (B,), generator=g).to(torch.int32)
    count[::5] = torch.randint(0, 40, (len(count[::5]),), generator=g).to(torch.int32)
    count[B // 2] = k_cap
    count = count.to(DEV)
    out, lse = binding.decode_attention_long(q, Kc, Vc, count, block_table=table, k_cap=k_cap, window=window, want_lse=True)
    torch.cuda.synchronize()
    _compare(out, lse, q, K, V, count, torch.bfloat16, window=window)


def test_dimensions_of_one_element_may_have_any_stride():
    g = torch.Generator(device=DEV).manual_seed(12)
    x = torch.randn(3 * 64 + 5, generator=g, device=DEV).to(torch.bfloat16)
    q = x.as_strided((1, 1, 64), (7, 3, 1))
    K, V = x[64:].as_strided((1, 1, 1, 64), (1, 5, 9, 1)), x[128:].as_strided((1, 1, 1, 64), (11, 5, 2, 1))
    out, lse = binding.decode_attention_long(q, K, V, torch.ones(1, dtype=torch.int32, device=DEV), want_lse=True)
    torch.cuda.synchronize()
    assert torch.equal(out, V[:, :, 0])                      # one row: its value, whatever the score
    out4, _ = binding.prefill_attention(q[:, :, None], K, V)
    torch.cuda.synchronize()
    assert torch.equal(out4[:, :, 0], V[:, :, 0])


def test_two_calls_at_once_and_shared_pages():
    # two calls on two streams, each with its own workspace; sequences whose tables name the same pages (a shared beginning)
    B, Hq, Hkv, d, k_cap, page = 4, 32, 8, 128, 5000, 16
    q, K, V, Kc, Vc, table = _make(B, Hq, Hkv, d, k_cap, torch.bfloat16, page, 31)
    shared = 2000 // page
    table[1:, :shared] = table[0, :shared]
    K[1:, :, :shared * page], V[1:, :, :shared * page] = K[0, :, :shared * page], V[0, :, :shared * page]
    count = torch.tensor([5000, 4000, 2001, 1999], dtype=torch.int32, device=DEV)
    ws = [torch.empty(1 << 25, dtype=torch.uint8, device=DEV) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [None, None]
    for rep in range(8):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i] = binding.decode_attention_long(q, Kc, Vc, count, block_table=table, k_cap=k_cap, workspace=ws[i], want_lse=True,
                                                       window=300 * i)
    torch.cuda.synchronize()
    _compare(*got[0], q, K, V, count, torch.bfloat16)
    _compare(*got[1], q, K, V, count, torch.bfloat16, window=300)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("B,Hq,Hkv,d,k_cap,page", [(1, 8, 2, 128, 40, 0), (2, 6, 1, 64, 2000, 16), (1, 33, 1, 128, 1500, 0)])
def test_values_that_are_not_finite_in_seen_rows(B, Hq, Hkv, d, k_cap, page, dtype):
    # their columns are as a sum with positive weights has them, the others untouched
    print("not finite", B, Hq, Hkv, d, k_cap, page, dtype, flush=True)
    q, K, V, _, _, _ = _make(B, Hq, Hkv, d, k_cap, dtype, 0, 17)
    j = [k_cap - 1, k_cap // 2, 3, 20]
    V[0, 0, j[0], 0], V[0, 0, j[1], d - 1], V[0, 0, j[2], 9] = math.inf, -math.inf, math.nan
    V[0, 0, j[2], 33], V[0, 0, j[3], 33] = math.inf, -math.inf
    V[-1, -1, j[3], 40] = V[-1, -1, j[1], 40] = math.inf
    Kc, Vc, table = K, V, None
    if page:
        per = -(-k_cap // page)
        table = torch.arange(B * per, dtype=torch.int32, device=DEV).flip(0).view(B, per).contiguous()
        Kc, Vc = (torch.zeros(B * per, Hkv, page, d, dtype=dtype, device=DEV) for _ in range(2))
        rows = torch.arange(k_cap, device=DEV)
        for b in range(B):
            at = table[b].long()[rows // page]
            Kc[at, :, rows % page], Vc[at, :, rows % page] = K[b].transpose(0, 1), V[b].transpose(0, 1)
    count = torch.full((B,), k_cap, dtype=torch.int32, device=DEV)
    out, lse = binding.decode_attention_long(q, Kc, Vc, count, block_table=table, k_cap=k_cap, want_lse=True)
    torch.cuda.synchronize()
    odd = (~torch.isfinite(V)).any(2).repeat_interleave(Hq // Hkv, 1)                     # [B, Hq, d]
    want = V.double().masked_fill(torch.isfinite(V), 0).sum(2).repeat_interleave(Hq // Hkv, 1)
    assert torch.equal(out.double()[odd].nan_to_num(7, 8, 9), want[odd].nan_to_num(7, 8, 9))
    _compare(out.masked_fill(odd, 0), lse, q, K, V.masked_fill((~torch.isfinite(V)).any(2, keepdim=True), 0), count, dtype)


@pytest.mark.parametrize("B,Hkv,G,d,k_cap,page,longest", [(130, 8, 1, 64, 9000, 16, 9000), (256, 1, 4, 64, 6000, 0, 5999), (66, 1, 2, 128, 20000, 48, 20000),
                                                        (64, 32, 1, 64, 5000, 16, 5000), (34, 32, 2, 64, 4097, 0, 4097), (257, 2, 1, 64, 3000, 16, 3000)])
def test_one_long_sequence_among_many_short_ones(B, Hkv, G, d, k_cap, page, longest):
    print("one long", B, Hkv, G, d, k_cap, page, longest, flush=True)
    g = torch.Generator().manual_seed(B)
    count = torch.randint(0, 90, (B,), generator=g).to(torch.int32)
    count[[1, B // 2, B - 1]] = torch.tensor([700, longest, 33], dtype=torch.int32)
    count[::7] = 0
    count[B // 2] = longest
    gd = torch.Generator(device=DEV).manual_seed(B)
    q = torch.randn(B, Hkv * G, d, generator=gd, device=DEV).to(torch.bfloat16)
    rows = int(count.sum()) + B * max(page, 1)
    step = max(page, 1)
    K, V = (torch.randn(rows // step + 1, Hkv, step, d, generator=gd, device=DEV).to(torch.bfloat16) for _ in range(2))
    if page:
        need = -(-count // page)
        table = torch.full((B, -(-k_cap // page)), -1, dtype=torch.int32)
        at = 0
        for b in range(B):
            table[b, :int(need[b])] = torch.arange(at, at + int(need[b]), dtype=torch.int32)
            at += int(need[b])
        table = table.to(DEV)
        out, lse = binding.decode_attention_long(q, K, V, count.to(DEV), block_table=table, k_cap=k_cap, want_lse=True)
        per = lambda x, b: x[table[b, :max(1, int(need[b]))].clamp(0).long()].transpose(0, 1).reshape(Hkv, -1, d)
    else:
        Kc, Vc = (torch.randn(1, Hkv, k_cap, d, generator=gd, device=DEV).to(torch.bfloat16).expand(B, Hkv, k_cap, d) for _ in range(2))
        out, lse = binding.decode_attention_long(q, Kc, Vc, count.to(DEV), want_lse=True)
        per = lambda x, b: x[b]
        K, V = Kc, Vc
    torch.cuda.synchronize()
    for b in list(range(0, B, 5)) + [1, B // 2, B - 1]:
        _compare(out[b:b + 1], lse[b:b + 1], q[b:b + 1], per(K, b)[None], per(V, b)[None], count[b:b + 1], torch.bfloat16)

"""Attention of drafted tokens (pkv_tree_attention) against plain attention in 64 bits."""
import math
import random

import pytest
import torch

from paper_2406_02069_amd import binding
from tests.cache_ref import check_rows, make_cache, random_tree, tree_rows

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _bits(parents):
    sets = []
    for t, p in enumerate(parents):
        sets.append((sets[p] if p >= 0 else set()) | {t})
    return sets


def _compare(out, lse, q, K, V, count, new, bits, positions=None, q_pos=None, slopes=None, cap=0.0, window=0, scale=None, absent=None):
    """bits[b]: sets of drafted tokens; absent [B, k_cap]: rows on pages that do not exist."""
    B, Hq, T, d = q.shape
    Hkv, k_cap = K.shape[1], K.shape[2]
    G = Hq // Hkv
    for b in range(B):
        for g in range(Hkv):
            seen, dist = tree_rows(bits[b], T, int(new[b]), int(count[b]), k_cap, None if positions is None else positions[b, g, :k_cap].tolist(),
                                   None if q_pos is None else q_pos[b].tolist(), window)
            if absent is not None:
                seen &= ~absent[b]
            for h in range(g * G, g * G + G):
                check_rows(out[b, h], None if lse is None else lse[b, h], q[b, h], K[b, g], V[b, g], seen, dist,
                           d ** -0.5 if scale is None else scale, q.dtype, cap, None if slopes is None else float(slopes[h]), T * G)


def _inputs(B, Hq, Hkv, d, T, k_cap, page, dtype, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    q = torch.randn(B, Hq, T, d, generator=g, device=DEV).to(dtype)
    cache = make_cache(B, Hkv, k_cap, d, dtype, page, g)
    rng = random.Random(seed)
    parents = [random_tree(T, rng) for _ in range(B)]
    tree = torch.stack([binding.tree_bits(p, device=DEV) for p in parents])
    return q, cache, tree, [_bits(p) for p in parents]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("B,Hq,Hkv,d,T,k_cap,page,cap,slopes,window", [
    (3, 8, 8, 64, 1, 1, 0, 0.0, False, 0), (4, 8, 2, 128, 5, 37, 0, 30.0, False, 0), (4, 28, 4, 128, 7, 70, 16, 0.0, True, 0),
    (2, 16, 4, 64, 33, 700, 48, 50.0, True, 100), (2, 34, 2, 128, 26, 1025, 1, 0.0, False, 9), (1, 64, 1, 128, 3, 513, 0, 0.0, False, 0),
    (1, 8, 8, 64, 64, 300, 7, 0.0, False, 0), (5, 6, 2, 128, 16, 5000, 256, 0.0, True, 0), (1, 32, 8, 128, 64, 9001, 16, 0.0, False, 0),
    (2, 4, 2, 64, 256, 1500, 64, 20.0, False, 0), (1, 12, 2, 128, 100, 2100, 0, 0.0, True, 500), (2, 8, 2, 128, 16, 3000, 0, 0.0, False, 0),
    (1, 128, 1, 64, 40, 800, 16, 0.0, False, 0), (2, 2, 2, 128, 200, 6500, 0, 0.0, False, 0)])
def test_rows(B, Hq, Hkv, d, T, k_cap, page, cap, slopes, window, dtype):
    print("tree", B, Hq, Hkv, d, T, k_cap, page, cap, slopes, window, dtype, flush=True)
    q, (K, V, Kc, Vc, table), tree, bits = _inputs(B, Hq, Hkv, d, T, k_cap, page, dtype, k_cap + d)
    count = torch.tensor([k_cap, max(k_cap // 2, 1), T, k_cap + 4, T - 1][:B], dtype=torch.int32, device=DEV)  # all, half, no past, more, one dropped
    sl = 2.0 ** (-8.0 * torch.arange(1, Hq + 1, device=DEV) / Hq) if slopes else None
    out, lse = binding.tree_attention(q, Kc, Vc, count, tree=tree, block_table=table, k_cap=k_cap, slopes=sl, cap=cap, window=window,
                                      want_lse=True)
    torch.cuda.synchronize()
    _compare(out, lse, q, K, V, count, [T] * B, bits, slopes=sl, cap=cap, window=window)


@pytest.mark.parametrize("Hq,Hkv,T", [(8, 2, 9), (8, 2, 40), (2, 2, 100)])
@pytest.mark.parametrize("slopes,window,page", [(False, 0, 0), (True, 300, 16), (True, 0, 5), (False, 60, 0)])
def test_positions_of_kept_rows(Hq, Hkv, T, slopes, window, page):
    B, d, k_cap = 4, 128, 610
    q, (K, V, Kc, Vc, table), tree, bits = _inputs(B, Hq, Hkv, d, T, k_cap, page, torch.bfloat16, 3)
    g = torch.Generator(device=DEV).manual_seed(9)
    room = torch.randint(1, 6, (B, Hkv, k_cap + 3), generator=g, device=DEV).cumsum(2).to(torch.int32) - 1
    room[:, 1] = room[:, 1].flip(1) if Hkv > 1 else room[:, 1]     # in no order
    count = torch.tensor([610, 200, T, 500], dtype=torch.int32, device=DEV)
    new = torch.tensor([T, T - 3, T, 1], dtype=torch.int32, device=DEV)
    room[0, :, 17] = -1                                            # a hole
    depth = torch.tensor([[len(s) for s in bits[b]] for b in range(B)], device=DEV)
    q_pos = (torch.tensor([1900, 450, 30, 900], device=DEV)[:, None] + depth).to(torch.int32)   # rows behind the query among the past
    for b in range(B):
        at = int(count[b]) - int(new[b])
        room[b, :, at:at + int(new[b])] = q_pos[b, :int(new[b])]
    room[0, :, int(count[0]) - 2] = -1                             # a drafted token that is not there
    sl = torch.linspace(0.01, 0.3, Hq, device=DEV) if slopes else None
    out, lse = binding.tree_attention(q, Kc, Vc, count, tree=tree, new_lens=new, block_table=table, k_cap=k_cap, positions=room, q_pos=q_pos,
                                      slopes=sl, window=window, want_lse=True)
    torch.cuda.synchronize()
    _compare(out, lse, q, K, V, count, new, bits, room, q_pos, sl, 0.0, window)


@pytest.mark.parametrize("Hq,Hkv,d,T", [(8, 2, 128, 12), (4, 4, 64, 70), (16, 2, 128, 33)])
def test_masks_of_any_kind(Hq, Hkv, d, T):
    # bits that are no tree: rows that see nothing, rows that do not see themselves, tokens in front of others; fewer tokens than rows
    B, k_cap = 4, 400
    q, (K, V, Kc, Vc, _), _, _ = _inputs(B, Hq, Hkv, d, T, k_cap, 0, torch.float16, 5)
    g = torch.Generator().manual_seed(T)
    mask = torch.rand(B, T, T, generator=g) < 0.3
    mask[:, 3] = False
    words = (T + 31) // 32
    tree = torch.zeros(B, T, words, dtype=torch.int64)
    for u in range(T):
        tree[:, :, u // 32] |= mask[:, :, u].long() << (u % 32)
    tree = torch.where(tree >= 2 ** 31, tree - 2 ** 32, tree).to(torch.int32).to(DEV)
    bits = [[set(mask[b, t].nonzero()[:, 0].tolist()) for t in range(T)] for b in range(B)]
    count = torch.tensor([T, 400, T - 2, 0], dtype=torch.int32, device=DEV)
    new = torch.tensor([T + 5, T - 4, T, 3], dtype=torch.int32, device=DEV)     # (clamped to T)
    out, lse = binding.tree_attention(q, Kc, Vc, count, tree=tree, new_lens=new, window=50, want_lse=True)
    torch.cuda.synchronize()
    new = new.clamp(max=T)
    _compare(out, lse, q, K, V, count, new, bits, window=50)
    assert not out[0, :, 3].any() and bool(torch.isneginf(lse[0, :, 3]).all())     # nothing of the past, nothing drafted
    assert not out[1, :, T - 4:].any() and not out[3].any()


@pytest.mark.parametrize("Hq,Hkv,d,T,n", [(8, 2, 128, 8, 500), (4, 4, 64, 130, 3000), (16, 4, 128, 20, 2000)])
def test_without_a_tree_it_is_a_chunk_of_a_prompt(Hq, Hkv, d, T, n):
    q, (K, V, _, _, _), _, _ = _inputs(2, Hq, Hkv, d, T, n, 0, torch.bfloat16, 6)
    count = torch.tensor([n, n - 77], dtype=torch.int32, device=DEV)
    out, lse = binding.tree_attention(q, K, V, count, want_lse=True)
    torch.cuda.synchronize()
    chain = [[set(range(t + 1)) for t in range(T)]] * 2
    _compare(out, lse, q, K, V, count, [T] * 2, chain)
    ref, ref_lse = binding.prefill_attention(q, K, V, seq_lens=count, q_start=count - T, want_lse=True)
    torch.cuda.synchronize()
    # each within its bounds of the same values: two roundings of the result and of the weights, scores in 32 bits
    assert bool(((out.float() - ref.float()).abs() <= 2.0 ** -7 * ref.float().abs() + 2.0 ** -7).all())
    torch.testing.assert_close(lse, ref_lse, rtol=1e-5, atol=1e-4)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("Hq,Hkv,T,page,window", [(8, 2, 9, 16, 0), (8, 2, 33, 0, 120), (4, 4, 100, 16, 60)])
def test_values_that_are_not_finite(Hq, Hkv, T, page, window, dtype):
    # in rows that are hidden from some or all, in K and in V; pages that do not exist
    B, d, k_cap = 2, 64, 500
    q, (K, V, Kc, Vc, table), tree, bits = _inputs(B, Hq, Hkv, d, T, k_cap, page, dtype, 11)
    count, new = torch.tensor([500, 300], dtype=torch.int32, device=DEV), torch.tensor([T, T - 2], dtype=torch.int32, device=DEV)
    absent = torch.zeros(B, k_cap, dtype=torch.bool, device=DEV)
    K[1, :, 300:], V[1, :, 300:] = math.nan, math.inf               # behind the count
    for b, n in ((0, 500), (1, 300)):
        past = n - int(new[b])
        V[b, 0, past + 1, 3] = math.inf                            # seen by its descendants
        V[b, 0, past + 2, 3] = -math.inf
        V[b, -1, past + 4, 7] = math.nan
        V[b, :, past + 5, 9] = -math.inf
        V[b, -1, past - 70, 11] = math.inf                         # seen by all, or outside of their windows
        V[b, 0, past - 2, d - 1] = math.nan
    if page:
        from tests.cache_ref import paged
        table[0, 3], table[1, 2] = 10 ** 6, -4
        absent[0, 48:64] = absent[1, 32:48] = True
        Kc, Vc = paged(K, page, table, Kc.shape[0]), paged(V, page, table, Kc.shape[0])
    out, lse = binding.tree_attention(q, Kc if page else K, Vc if page else V, count, tree=tree, new_lens=new, block_table=table, k_cap=k_cap,
                                      window=window, want_lse=True)
    torch.cuda.synchronize()
    _compare(out, lse, q, K, V, count, new, bits, window=window, absent=absent)
    # keys that are not finite, hidden from some tokens: those do not notice
    K2 = K.clone()
    at = 500 - T + 1
    K2[0, :, at] = math.nan
    V2 = torch.where(torch.isfinite(V), V, 0)
    plain = torch.isfinite(K2).all(-1)
    Kt, Vt = (K2, V2) if not page else (paged(K2, page, table, Kc.shape[0]), paged(V2, page, table, Kc.shape[0]))
    out, lse = binding.tree_attention(q, Kt, Vt, count, tree=tree, new_lens=new, block_table=table, k_cap=k_cap, window=window, want_lse=True)
    torch.cuda.synchronize()
    assert not bool(plain[0, 0, at])
    for g in range(Hkv):
        seen, dist = tree_rows(bits[0], T, T, 500, k_cap, None, None, window)
        seen &= ~absent[0]
        blind = ~seen[:, at]
        for h in range(g * Hq // Hkv, (g + 1) * Hq // Hkv):
            K0 = torch.nan_to_num(K2[0, g])
            check_rows(out[0, h][blind], lse[0, h][blind], q[0, h][blind], K0, V2[0, g], seen[blind], dist[blind], d ** -0.5, dtype, rows=T * Hq // Hkv)
            assert bool(torch.isnan(out[0, h][~blind]).all())


def test_strides_scale_and_large_scores():
    B, Hq, Hkv, d, T, k_cap = 2, 8, 2, 64, 11, 300
    g = torch.Generator(device=DEV).manual_seed(5)
    q = torch.randn(B, T, Hq + 3, d + 8, generator=g, device=DEV).to(torch.bfloat16)[:, :, 2:2 + Hq, :d].transpose(1, 2)
    buf = torch.randn(2, B, k_cap + 5, Hkv, d + 8, generator=g, device=DEV).to(torch.bfloat16)
    K, V = buf[0, :, :k_cap, :, :d].transpose(1, 2), buf[1, :, :k_cap, :, :d].transpose(1, 2)
    count = torch.tensor([300, 299], dtype=torch.int32, device=DEV)
    out = torch.full((B, T, Hq, d + 16), 7.0, dtype=torch.bfloat16, device=DEV)
    o, lse = binding.tree_attention(q, K, V, count, scale=6.0, want_lse=True, out=out[..., :d].transpose(1, 2))   # scores of some hundreds
    torch.cuda.synchronize()
    _compare(o, lse, q, K, V, count, [T] * B, [[set(range(t + 1)) for t in range(T)]] * B, scale=6.0)
    assert bool((out[..., d:] == 7).all())


def test_longest_offsets():
    d, Hkv, page, T = 128, 8, 128, 3
    pages = 2 ** 32 // (Hkv * page * d) + 1
    K, V = (torch.empty(pages, Hkv, page, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    g = torch.Generator(device=DEV).manual_seed(6)
    K[-1], V[-1] = (torch.randn(Hkv, page, d, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    q = torch.randn(1, 8, T, d, generator=g, device=DEV).to(torch.bfloat16)
    table, count = torch.tensor([[pages - 1]], dtype=torch.int32, device=DEV), torch.tensor([128], dtype=torch.int32, device=DEV)
    out, lse = binding.tree_attention(q, K, V, count, block_table=table, want_lse=True)
    torch.cuda.synchronize()
    _compare(out, lse, q, K[-1:], V[-1:], count, [T], [[set(range(t + 1)) for t in range(T)]])


@pytest.mark.parametrize("Hq,Hkv,T", [(32, 8, 4), (32, 8, 40)])
def test_same_bits_every_time_on_another_stream_and_from_a_graph(Hq, Hkv, T):
    B, d, k_cap = 2, 128, 6000
    q, (K, V, Kc, Vc, table), tree, bits = _inputs(B, Hq, Hkv, d, T, k_cap, 16, torch.bfloat16, 7)
    count = torch.tensor([6000, 2222], dtype=torch.int32, device=DEV)
    call = lambda **kw: binding.tree_attention(q, Kc, Vc, count, tree=tree, block_table=table, k_cap=k_cap, want_lse=True, **kw)  # noqa: E731
    out, lse = call()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        again = call()
    torch.cuda.synchronize()
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    ws = torch.empty(1 << 26, dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    o, z = torch.empty_like(out), torch.empty_like(lse)
    with torch.cuda.graph(graph, stream=side):
        call(out=o, lse=z, workspace=ws)
    for step in range(3):
        q.copy_(torch.randn(q.shape, device=DEV))
        count.copy_(torch.tensor([6000 - 999 * step, 117 + step], dtype=torch.int32))
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        out, lse = call()
        torch.cuda.synchronize()
        assert torch.equal(o, out) and torch.equal(z, lse)


@pytest.mark.parametrize("B,Hkv,G,d,T,k_cap,page,window", [(64, 1, 3, 64, 6, 3000, 0, 0), (65, 2, 2, 64, 3, 1200, 16, 0), (300, 1, 1, 64, 2, 700, 0, 0),
                                                          (7, 8, 4, 128, 30, 6000, 16, 1000), (40, 8, 1, 64, 9, 900, 0, 0)])
def test_ragged_batches_of_all_sizes(B, Hkv, G, d, T, k_cap, page, window):
    print("ragged tree", B, Hkv, G, d, T, k_cap, page, window, flush=True)
    q, (K, V, Kc, Vc, table), tree, bits = _inputs(B, Hkv * G, Hkv, d, T, k_cap, page, torch.bfloat16, B)
    g = torch.Generator().manual_seed(B)
    count = torch.randint(0, k_cap + 1, (B,), generator=g).to(torch.int32)
    count[::5] = torch.randint(0, 40, (len(count[::5]),), generator=g).to(torch.int32)
    count[B // 2] = k_cap
    count = count.to(DEV)
    new = torch.randint(0, T + 1, (B,), generator=g).to(torch.int32).to(DEV)
    out, lse = binding.tree_attention(q, Kc, Vc, count, tree=tree, new_lens=new, block_table=table, k_cap=k_cap, window=window, want_lse=True)
    torch.cuda.synchronize()
    _compare(out, lse, q, K, V, count, new, bits, window=window)


@pytest.mark.parametrize("B,Hq,Hkv,d,T,k_cap,page,dtype", [(9, 6, 2, 128, 33, 1700, 16, torch.bfloat16), (70, 5, 1, 64, 9, 900, 0, torch.float16),
                                                           (3, 7, 1, 128, 59, 4000, 0, torch.float16), (66, 3, 1, 128, 13, 1300, 5, torch.bfloat16)])
def test_many_rows_of_ragged_ranges(B, Hq, Hkv, d, T, k_cap, page, dtype):
    # ranges of many rows, joined: sequences of none, one and many ranges, rows that are not there, infinities in some range's values,
    # and whatever the workspace held
    print("many rows", B, Hq, Hkv, d, T, k_cap, page, dtype, flush=True)
    q, (K, V, Kc, Vc, table), tree, bits = _inputs(B, Hq, Hkv, d, T, k_cap, page, dtype, B)
    count = torch.tensor([k_cap - (k_cap * i // 7) % k_cap for i in range(B)], dtype=torch.int32, device=DEV)
    count[1], count[2] = 0, T + 40
    new = torch.tensor([T - i % 4 for i in range(B)], dtype=torch.int32, device=DEV)
    V[0, 0, 5, 3], V[0, 0, k_cap // 2, 3], V[0, 0, k_cap - T - 9, d - 1], V[2, 0, 20, 6] = math.inf, math.inf, -math.inf, math.nan
    if page:
        from tests.cache_ref import paged
        Vc = paged(V, page, table, Vc.shape[0])
    for fill in (255, 0):
        ws = torch.full((1 << 28,), fill, dtype=torch.uint8, device=DEV)
        out, lse = binding.tree_attention(q, Kc, Vc if page else V, count, tree=tree, new_lens=new, block_table=table, k_cap=k_cap, want_lse=True, workspace=ws)
        torch.cuda.synchronize()
        few = list(range(min(B, 9))) + ([B - 1] if B > 9 else [])
        _compare(out[few], lse[few], q[few], K[few], V[few], count[few], new[few], [bits[b] for b in few])
        assert not out[1].any() and bool(torch.isposinf(out[0, :Hq // Hkv, 0, 3]).all()) and bool(torch.isneginf(out[0, :Hq // Hkv, 0, d - 1]).all())


def test_two_calls_at_once():
    B, Hq, Hkv, d, T, k_cap = 4, 32, 8, 128, 24, 5000
    q, (K, V, Kc, Vc, table), tree, bits = _inputs(B, Hq, Hkv, d, T, k_cap, 16, torch.bfloat16, 31)
    count = torch.tensor([5000, 4000, 2001, 1999], dtype=torch.int32, device=DEV)
    streams = [torch.cuda.Stream() for _ in range(2)]
    ws = [torch.empty(1 << 27, dtype=torch.uint8, device=DEV) for _ in range(2)]
    torch.cuda.synchronize()
    got = [None, None]
    for rep in range(6):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i] = binding.tree_attention(q, Kc, Vc, count, tree=tree, block_table=table, k_cap=k_cap, workspace=ws[i], want_lse=True,
                                                window=300 * i)
    torch.cuda.synchronize()
    _compare(*got[0], q, K, V, count, [T] * B, bits)
    _compare(*got[1], q, K, V, count, [T] * B, bits, window=300)

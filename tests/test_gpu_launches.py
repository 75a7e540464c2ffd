"""Calls on caches with much more room than rows: how many workgroups they start, and what they do where one sequence has most of the
work."""
import pytest
import torch

from paper_2406_02069_amd import binding
from tests import captured
from tests.cache_ref import make_cache
from tests.test_gpu_weigh_evict import _case, _check, _compare

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TURNS = 2 * 2048                                                   # workgroups of 256 that the device holds at a time, twice


def _room(B, Hkv, d, k_cap):
    """A cache that a call can be captured with: pools of one page, which no replay reads."""
    pool = torch.zeros(1, Hkv, 16, d, dtype=torch.bfloat16, device=DEV)
    table = torch.zeros(B, k_cap // 16, dtype=torch.int32, device=DEV)
    return pool, table, torch.zeros(B, dtype=torch.int32, device=DEV), torch.zeros(B, Hkv, k_cap, device=DEV)


@pytest.mark.parametrize("B,Hkv,k_cap,budget", [(64, 8, 16384, 2048), (1, 8, 131072, 65536), (4, 8, 32768, 2048), (1, 1, 4096, 2048)])
def test_eviction_starts_two_turns_of_workgroups_at_most(B, Hkv, k_cap, budget):
    pool, table, count, w = _room(B, Hkv, 64, k_cap)
    pos = torch.zeros(B, Hkv, k_cap, dtype=torch.int32, device=DEV)
    ws = torch.empty(1 << 26, dtype=torch.uint8, device=DEV)
    other, out = pool.clone(), torch.zeros_like(count)
    got = captured.launches(lambda: binding.cache_evict(pool, other, count, pos, w, budget, block_table=table, k_cap=k_cap, count_out=out, workspace=ws))
    assert got[0] == (B * Hkv, 1024) and len(got) == 2
    assert got[1][1] == 256 and got[1][0] <= TURNS


@pytest.mark.parametrize("B,Hkv,k_cap", [(64, 8, 16384), (256, 4, 8192), (2, 8, 400000), (1, 2, 2048)])
def test_weights_start_two_turns_of_workgroups_beside_the_join_at_most(B, Hkv, k_cap):
    pool, table, count, w = _room(B, Hkv, 64, k_cap)
    q = torch.zeros(B, Hkv, 64, dtype=torch.bfloat16, device=DEV)
    out = torch.zeros_like(q)
    desc = binding.DecodeLongDesc(B=B, Hq=Hkv, Hkv=Hkv, d=64, k_cap=k_cap, page_size=16, num_pages=1, max_pages=k_cap // 16)
    ws = torch.empty(binding.load().pkv_decode_accumulate_workspace_bytes(binding.ctypes.byref(desc)), dtype=torch.uint8, device=DEV)
    got = captured.launches(lambda: binding.decode_attention_accumulate(q, pool, pool, count, w, block_table=table, k_cap=k_cap, out=out, workspace=ws))
    assert len(got) == 2 and got[1][1] == 256 and got[1][0] <= TURNS + B * Hkv


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("page", [0, 16])
def test_eviction_of_one_sequence_among_many(page, in_place):
    # one evicted as a whole, some by a few rows or by one, others not at all
    print("one of many", page, in_place, flush=True)
    B, Hkv, d, k_cap, budget = 40, 4, 64, 8000, 3001
    K, V, Kc, Vc, table, pos, w, g = _case(B, Hkv, d, k_cap, page, torch.bfloat16, 40)
    K, V, Kc, Vc = K.clone(), V.clone(), Kc.clone(), Vc.clone()
    count = torch.tensor([budget - 5, budget, budget + 1, 17, budget + 70, 0, budget + 200, budget + 1] * 5, dtype=torch.int32, device=DEV)
    count[33] = k_cap
    po, wo = (pos.clone(), w.clone()) if in_place else (torch.full_like(pos, 7), torch.full_like(w, 0.5))
    before, src = (po.clone(), wo.clone()), (po, wo) if in_place else (pos, w)
    kw = {} if in_place else dict(positions_out=po, weights_out=wo)
    co = binding.cache_evict(Kc, Vc, count, *src, budget, recent=20, first=2, block_table=table, k_cap=k_cap, **kw)
    torch.cuda.synchronize()
    _check(K, V, Kc, Vc, table, pos, w, count, budget, 20, 2, (po, wo, co), before)


@pytest.mark.parametrize("B", [40, 300])
def test_weights_of_one_long_sequence_among_many(B):
    print("one long", B, flush=True)
    Hq, Hkv, d, k_cap = 4, 2, 64, 20000
    g = torch.Generator(device=DEV).manual_seed(B)
    q = torch.randn(B, Hq, d, generator=g, device=DEV).to(torch.bfloat16)
    K, V, Kc, Vc, table = make_cache(B, Hkv, k_cap, d, torch.bfloat16, 0, g)
    count = torch.randint(0, 2100, (B,), generator=g, device=DEV).to(torch.int32)
    count[7], count[B - 1] = k_cap, 1025
    weights = torch.rand(B, Hkv, k_cap, generator=g, device=DEV)
    before = weights.clone()
    out, lse = binding.decode_attention_accumulate(q, Kc, Vc, count, weights, want_lse=True)
    torch.cuda.synchronize()
    some = [0, 3, 7, 8, B - 1]
    _compare(out[some], lse[some], weights[some], before[some], q[some], K[some], V[some], count[some])
    behind = torch.arange(k_cap, device=DEV) >= count[:, None, None]
    assert torch.equal(weights[behind.expand_as(weights)], before[behind.expand_as(weights)])
    total = (weights - before).double().sum(2)                     # a head's weights add up to 1: before is below 1, each of its sums rounds by 2^-24
    room = 1e-4 + count.double()[:, None] * 2.0 ** -23
    assert bool(((total - Hq / Hkv * (count > 0)[:, None]).abs() <= room).all())

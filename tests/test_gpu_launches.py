"""Calls on caches with much more room than rows: how many workgroups they start, and what they do where one sequence has most of the
work."""
import pytest
import torch

from paper_2406_02069_amd import binding
from tests import captured
from tests.test_gpu_weigh_evict import _case, _check

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

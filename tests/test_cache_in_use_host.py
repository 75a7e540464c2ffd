"""Refusals of the calls for a cache in use before anything is launched, their workspace sizes, and a tree's bits (no GPU)."""
import ctypes
import math
import random

import pytest
import torch

from paper_2406_02069_amd import binding
from tests.cache_ref import random_tree

I, U, W = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED, binding.ERR_WORKSPACE
CACHE = dict(k_cap=8192, page_size=0, num_pages=0, max_pages=0)
C = dict(c_sb=8 * 8192 * 128, c_sh=8192 * 128, c_st=128)
BAD_CACHES = [dict(B=0), dict(Hkv=0), dict(k_cap=0), dict(page_size=-1), dict(c_st=129), dict(c_sh=-8),
              dict(page_size=16, num_pages=0, max_pages=512), dict(page_size=16, num_pages=1, max_pages=511)]
NOT_BUILT = [dict(d=96), dict(B=65536), dict(k_cap=2 ** 30 + 1), dict(page_size=2 ** 20, num_pages=2 ** 12, max_pages=1), dict(c_st=2 ** 30 + 8)]
BAD_SCORES = [dict(Hq=0), dict(Hq=30), dict(dtype=2), dict(scale=-1.0), dict(scale=math.nan), dict(cap=-0.5), dict(cap=math.inf),
              dict(q_sh=4), dict(q_sb=-8), dict(cap=1e-44), dict(cap=3e38), dict(scale=3e38)]


def _ref(d):
    return ctypes.byref(d)


# ---- drafted tokens ----

def _tree_desc(**kw):
    return binding.TreeDesc(**{**dict(B=1, Hq=32, Hkv=8, d=128, T=16, dtype=0, window=0, reserved=0, scale=0.0, cap=0.0, q_sb=16 * 32 * 128, q_sh=16 * 128,
                                      q_st=128, p_sb=8 * 8192, p_sh=8192, o_sb=16 * 32 * 128, o_sh=16 * 128, o_st=128), **CACHE, **C, **kw})


def _tree(desc, **kw):
    lib = binding.load()
    p = dict(q=0x1000, K=0x2000, V=0x3000, table=None, count=0x4000, new=None, tree=None, pos=None, qp=None, sl=None, out=0x5000, lse=None, ws=0x10000,
             n=lib.pkv_tree_workspace_bytes(_ref(desc)))
    p.update(kw)
    return lib.pkv_tree_attention(_ref(desc), *p.values(), None)


@pytest.mark.parametrize("kw", BAD_CACHES + BAD_SCORES + [dict(T=0), dict(window=-1), dict(reserved=1), dict(q_st=4), dict(o_sb=-8), dict(o_st=12), dict(p_sb=-1)])
def test_tree_descriptors_refused(kw):
    d = _tree_desc(**kw)
    assert binding.load().pkv_tree_workspace_bytes(_ref(d)) == 0
    assert _tree(d, table=0x6000, n=1 << 40) == I


@pytest.mark.parametrize("kw", NOT_BUILT + [dict(T=257), dict(Hq=129, Hkv=1), dict(B=4096, Hq=64, T=256), dict(Hq=2 ** 30, Hkv=2 ** 24)])
def test_tree_not_built(kw):
    assert _tree(_tree_desc(**kw), table=0x6000, n=1 << 40) == U


def test_tree_pointers_and_workspace_refused():
    good = _tree_desc()
    need = binding.load().pkv_tree_workspace_bytes(_ref(good))
    assert need > 0
    for kw in (dict(q=None), dict(K=None), dict(V=None), dict(count=None), dict(out=None), dict(q=0x1008), dict(K=0x2004), dict(out=0x5008),
               dict(count=0x4002), dict(new=0x7001), dict(tree=0x7002), dict(sl=0x7002), dict(lse=0x7003), dict(pos=0x7000), dict(qp=0x7000),
               dict(pos=0x7001, qp=0x7000)):
        assert _tree(good, **kw) == I, kw
    for kw in (dict(ws=None), dict(ws=0x10080), dict(n=need - 1)):
        assert _tree(good, **kw) == W
    assert _tree(_tree_desc(page_size=16, num_pages=600, max_pages=512)) == I        # no table


def test_bits_of_trees():
    rng = random.Random(4)
    for T in (1, 2, 31, 32, 33, 64, 100, 256):
        parents = random_tree(T, rng)
        bits = binding.tree_bits(parents)
        assert bits.shape == (T, (T + 31) // 32) and bits.dtype == torch.int32
        sets = []
        for t, p in enumerate(parents):
            sets.append((sets[p] if p >= 0 else set()) | {t})
            got = {u for u in range(32 * bits.shape[1]) if int(bits[t, u // 32]) >> (u % 32) & 1}
            assert got == sets[t]
    for bad in ([], [0], [-2], [-1, 1], [-1] * 257):
        with pytest.raises(binding.PkvError) as e:
            binding.tree_bits(bad)
        assert e.value.status == I
    lib = binding.load()
    two = (ctypes.c_int32 * 2)(-1, 0)
    assert lib.pkv_tree_bits(2, None, two) == I and lib.pkv_tree_bits(2, two, None) == I


# ---- weights that add up ----

def _long_desc(**kw):
    return binding.DecodeLongDesc(**{**dict(B=1, Hq=32, Hkv=8, d=128, dtype=0, window=0, scale=0.0, cap=0.0, q_sb=32 * 128, q_sh=128, p_sb=8 * 8192, p_sh=8192),
                                     **CACHE, **C, **kw})


def _weigh(desc, **kw):
    lib = binding.load()
    p = dict(q=0x1000, K=0x2000, V=0x3000, table=None, count=0x4000, pos=None, qp=None, sl=None, w=0x8000, w_sb=8 * 8192, w_sh=8192, out=0x5000, lse=None,
             ws=0x10000, n=lib.pkv_decode_accumulate_workspace_bytes(_ref(desc)))
    p.update(kw)
    return lib.pkv_decode_attention_accumulate(_ref(desc), *p.values(), None)


@pytest.mark.parametrize("kw", BAD_CACHES + BAD_SCORES + [dict(window=-1), dict(p_sh=-1)])
def test_weigh_descriptors_refused(kw):
    d = _long_desc(**kw)
    assert binding.load().pkv_decode_accumulate_workspace_bytes(_ref(d)) == 0
    assert _weigh(d, table=0x6000, n=1 << 40) == I


@pytest.mark.parametrize("kw", NOT_BUILT + [dict(Hq=129, Hkv=1), dict(B=65535, Hq=512, Hkv=512), dict(B=65535, Hq=129, Hkv=129)])
def test_weigh_not_built(kw):
    assert _weigh(_long_desc(**kw), table=0x6000, n=1 << 50) == U


def test_weigh_of_too_many_rows_refused():
    for kw in (dict(B=65535, Hkv=128, Hq=128, k_cap=2 ** 18 + 2 ** 11), dict(B=4096, Hkv=512, Hq=512, k_cap=2 ** 20)):
        assert _weigh(_long_desc(**kw), n=1 << 60) == U, kw
        assert binding.load().pkv_decode_accumulate_workspace_bytes(_ref(_long_desc(**kw))) == 0
    assert binding.load().pkv_decode_accumulate_workspace_bytes(_ref(_long_desc(B=4096, Hkv=512, Hq=512, k_cap=2 ** 20 - 1024))) > 0


def test_weigh_pointers_and_workspace_refused():
    good = _long_desc()
    need = binding.load().pkv_decode_accumulate_workspace_bytes(_ref(good))
    assert need >= 32 * 8192 * 4 + binding.load().pkv_decode_long_workspace_bytes(_ref(good))
    for kw in (dict(q=None), dict(K=None), dict(V=None), dict(count=None), dict(out=None), dict(w=None), dict(w=0x8002), dict(w_sb=-1), dict(w_sh=-4),
               dict(q=0x1008), dict(out=0x5008), dict(lse=0x7003)):
        assert _weigh(good, **kw) == I, kw
    for kw in (dict(ws=None), dict(ws=0x10080), dict(n=need - 1)):
        assert _weigh(good, **kw) == W
    assert _weigh(_long_desc(page_size=16, num_pages=600, max_pages=512)) == I


# ---- eviction ----

def _evict_desc(**kw):
    s = dict(p_sb=8 * 8192, p_sh=8192, w_sb=8 * 8192, w_sh=8192, po_sb=8 * 8192, po_sh=8192, wo_sb=8 * 8192, wo_sh=8192)
    return binding.EvictDesc(**{**dict(B=1, Hkv=8, d=128, budget=2048, recent=32, first=4), **CACHE, **C, **s, **kw})


def _evict(desc, **kw):
    lib = binding.load()
    p = dict(K=0x2000, V=0x3000, table=None, count=0x4000, pos=0x5000, w=0x6000, po=0x7000, wo=0x8000, co=0x9000, ws=0x10000,
             n=lib.pkv_evict_workspace_bytes(_ref(desc)))
    p.update(kw)
    return lib.pkv_cache_evict(_ref(desc), *p.values(), None)


@pytest.mark.parametrize("kw", BAD_CACHES + [dict(budget=0), dict(recent=-1), dict(first=-1), dict(recent=2045), dict(recent=2 ** 31 - 1, first=2 ** 31 - 1),
                                             dict(p_sb=-1), dict(w_sh=-1), dict(po_sh=-1), dict(wo_sb=-1)])
def test_evict_descriptors_refused(kw):
    d = _evict_desc(**kw)
    assert binding.load().pkv_evict_workspace_bytes(_ref(d)) == 0
    assert _evict(d, table=0x6000, n=1 << 40) == I


@pytest.mark.parametrize("kw", NOT_BUILT + [dict(B=65535, Hkv=65)])
def test_evict_not_built(kw):
    assert _evict(_evict_desc(**kw), table=0x6000, n=1 << 50) == U


def test_evict_pointers_and_workspace_refused():
    good = _evict_desc()
    need = binding.load().pkv_evict_workspace_bytes(_ref(good))
    assert need > 0
    for kw in (dict(K=None), dict(V=None), dict(count=None), dict(pos=None), dict(w=None), dict(po=None), dict(wo=None), dict(K=0x2008), dict(V=0x3004),
               dict(count=0x4002), dict(pos=0x5001), dict(w=0x6002), dict(po=0x7001), dict(wo=0x8003), dict(co=0x9002), dict(co=0x4000)):
        assert _evict(good, **kw) == I, kw
    assert _evict(_evict_desc(po_sh=8200), po=0x5000) == I             # in place, with other strides
    assert _evict(_evict_desc(wo_sh=8200), wo=0x6000) == I
    for kw in (dict(ws=None), dict(ws=0x10080), dict(n=need - 1)):
        assert _evict(good, **kw) == W
    assert _evict(_evict_desc(page_size=16, num_pages=600, max_pages=512)) == I
    assert binding.load().pkv_evict_workspace_bytes(_ref(_evict_desc(budget=9000))) > 0


# ---- blocks ----

def _block_desc(**kw):
    return binding.BlockDesc(**{**dict(B=1, Hq=32, Hkv=8, d=128, dtype=0, block=16, most=64, first=1, recent=2, reserved=0, scale=0.0, cap=0.0, q_sb=32 * 128,
                                       q_sh=128, b_sb=8 * 512 * 256, b_sh=512 * 256), **CACHE, **C, **kw})


def _bounds(desc, **kw):
    p = dict(K=0x2000, table=None, count=0x4000, new=None, b=0x5000)
    p.update(kw)
    return binding.load().pkv_block_bounds(_ref(desc), *p.values(), None)


def _select(desc, **kw):
    lib = binding.load()
    p = dict(q=0x1000, b=0x5000, count=0x4000, out=0x6000, sc=None, ws=0x10000, n=lib.pkv_block_select_workspace_bytes(_ref(desc)))
    p.update(kw)
    return lib.pkv_block_select(_ref(desc), *p.values(), None)


def _blocks(desc, **kw):
    lib = binding.load()
    p = dict(q=0x1000, K=0x2000, V=0x3000, table=None, count=0x4000, blocks=0x6000, out=0x5000, lse=None, ws=0x10000,
             n=lib.pkv_decode_blocks_workspace_bytes(_ref(desc)))
    p.update(kw)
    return lib.pkv_decode_attention_blocks(_ref(desc), *p.values(), None)


@pytest.mark.parametrize("kw", BAD_CACHES + [dict(block=0), dict(block=-16), dict(reserved=1), dict(b_sb=4), dict(b_sh=-8), dict(dtype=2)])
def test_bounds_descriptors_refused(kw):
    assert _bounds(_block_desc(**kw), table=0x6000) == I


@pytest.mark.parametrize("kw", [dict(B=0), dict(Hkv=0), dict(k_cap=0), dict(block=0), dict(reserved=1), dict(most=0), dict(first=-1), dict(recent=-1),
                                dict(first=60, recent=5), dict(first=2 ** 31 - 1, recent=2 ** 31 - 1), dict(b_sb=4), dict(b_sh=-8)] + BAD_SCORES[:9])
def test_select_descriptors_refused(kw):
    d = _block_desc(**kw)
    assert binding.load().pkv_block_select_workspace_bytes(_ref(d)) == 0
    assert _select(d, n=1 << 40) == I


@pytest.mark.parametrize("kw", BAD_CACHES + BAD_SCORES + [dict(block=0), dict(reserved=1), dict(most=0)])
def test_block_attention_descriptors_refused(kw):
    d = _block_desc(**kw)
    assert binding.load().pkv_decode_blocks_workspace_bytes(_ref(d)) == 0
    assert _blocks(d, table=0x6000, n=1 << 40) == I


def test_blocks_not_built():
    for kw in NOT_BUILT + [dict(block=8), dict(block=24), dict(block=512), dict(B=65535, Hkv=65, Hq=65)]:
        assert _bounds(_block_desc(**kw), table=0x6000) == U, kw
        assert _blocks(_block_desc(**kw), table=0x6000, n=1 << 50) == U, kw
    for kw in [dict(d=96), dict(B=65536), dict(k_cap=2 ** 30 + 1), dict(block=8), dict(Hq=129, Hkv=1), dict(B=65535, Hq=512, Hkv=512)]:
        assert _select(_block_desc(**kw), n=1 << 50) == U, kw
    assert _blocks(_block_desc(Hq=129, Hkv=1), n=1 << 50) == U
    assert _blocks(_block_desc(most=2 ** 27), n=1 << 50) == U


def test_block_pointers_and_workspaces_refused():
    good = _block_desc()
    lib = binding.load()
    for kw in (dict(K=None), dict(count=None), dict(b=None), dict(K=0x2008), dict(b=0x5004), dict(count=0x4001), dict(new=0x7002)):
        assert _bounds(good, **kw) == I, kw
    assert _bounds(_block_desc(page_size=16, num_pages=600, max_pages=512)) == I
    need = lib.pkv_block_select_workspace_bytes(_ref(good))
    assert need > 0
    for kw in (dict(q=None), dict(b=None), dict(count=None), dict(out=None), dict(q=0x1008), dict(b=0x5004), dict(out=0x6002), dict(sc=0x7002)):
        assert _select(good, **kw) == I, kw
    for kw in (dict(ws=None), dict(ws=0x10080), dict(n=need - 1)):
        assert _select(good, **kw) == W
    need = lib.pkv_decode_blocks_workspace_bytes(_ref(good))
    assert need > 0
    for kw in (dict(q=None), dict(K=None), dict(V=None), dict(count=None), dict(blocks=None), dict(out=None), dict(blocks=0x6002), dict(K=0x2008)):
        assert _blocks(good, **kw) == I, kw
    for kw in (dict(ws=None), dict(ws=0x10080), dict(n=need - 1)):
        assert _blocks(good, **kw) == W
    assert _blocks(_block_desc(page_size=16, num_pages=600, max_pages=512)) == I


def test_launches_of_too_many_threads_and_lists_past_32_bits_refused():
    many = dict(B=2048, Hkv=2048)                                       # 2^22 workgroups of 1024
    assert _evict(_evict_desc(**many), n=1 << 50) == U
    assert _bounds(_block_desc(**many)) == U
    assert _select(_block_desc(Hq=2048, **many), n=1 << 50) == U
    for most in (2 ** 30 + 1, 2 ** 31 - 1):
        assert _select(_block_desc(most=most), n=1 << 50) == U
        assert binding.load().pkv_block_select_workspace_bytes(_ref(_block_desc(most=most))) == 0


def test_places_written_twice_refused():
    for kw in (dict(po_sh=0), dict(wo_sh=8191), dict(B=2, po_sb=0), dict(B=2, wo_sb=8191), dict(c_st=0), dict(c_sh=0), dict(B=2, c_sb=0)):
        assert _evict(_evict_desc(**kw)) == I, kw
    for kw in (dict(w_sh=0), dict(w_sh=8191)):
        assert _weigh(_long_desc(), **kw) == I, kw
    assert _weigh(_long_desc(B=2), w_sb=0) == I
    for kw in (dict(b_sh=0), dict(b_sh=512 * 256 - 8), dict(B=2, b_sb=0)):
        assert _bounds(_block_desc(**kw)) == I, kw


def test_places_that_interleave_refused():
    # every stride large enough by itself, and two places in one all the same
    n, c = 8192, 8192 * 128
    for kw in (dict(B=2, po_sb=n, po_sh=n), dict(B=2, wo_sb=n, wo_sh=n), dict(B=2, wo_sb=4 * n, wo_sh=n), dict(B=2, c_sb=c, c_sh=c), dict(c_sh=128, c_st=128),
               dict(c_sh=128, c_st=7 * 128), dict(B=2, c_sb=128, c_sh=256, c_st=8 * 128), dict(B=2, po_sh=2 ** 61, po_sb=2 ** 61)):
        assert _evict(_evict_desc(**kw)) == I, kw
    for kw in (dict(w_sb=n, w_sh=n), dict(w_sb=7 * n, w_sh=n), dict(w_sb=n, w_sh=2 * n - 1)):
        assert _weigh(_long_desc(B=2, c_sb=8 * c), **kw) == I, kw
    for kw in (dict(b_sb=512 * 256, b_sh=512 * 256), dict(b_sb=7 * 512 * 256)):
        assert _bounds(_block_desc(B=2, **kw)) == I, kw
    for kw in (dict(o_sh=0), dict(o_st=0), dict(o_sh=120), dict(o_sh=128), dict(o_sh=15 * 128), dict(o_st=2048), dict(B=2, o_sb=0), dict(B=2, o_sb=31 * 2048)):
        assert _tree(_tree_desc(**kw)) == I, kw


def test_places_of_any_order_taken():
    # (as far as the workspace, which is not there)
    n, c = 8192, 8192 * 128
    for kw in (dict(B=2, po_sb=n, po_sh=2 * n, wo_sb=n + 5, wo_sh=2 * n + 77), dict(B=3, c_sb=128, c_sh=3 * 128, c_st=24 * 128), dict(c_sh=128, c_st=8 * 128),
               dict(c_sb=0), dict(Hkv=1, c_sh=0, po_sh=0), dict(k_cap=1, budget=1, recent=0, first=0, c_st=0), dict(B=2, po_sb=2 ** 62, wo_sb=2 ** 62)):
        assert _evict(_evict_desc(**kw), ws=None) == W, kw
    for kw in (dict(w_sb=n, w_sh=2 * n), dict(w_sb=8 * n, w_sh=n)):
        assert _weigh(_long_desc(B=2), ws=None, **kw) == W, kw
    for kw in (dict(o_st=32 * 128, o_sh=128), dict(o_sb=0), dict(T=2, Hq=256, Hkv=8, o_st=256 * 128, o_sh=128), dict(B=2, o_sb=128, o_sh=256, o_st=32 * 256)):
        assert _tree(_tree_desc(**kw), ws=None) == W, kw


def test_binding_refuses_tensors_that_do_not_fit():
    q, K = torch.zeros(1, 8, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 16, 64, dtype=torch.bfloat16)
    n, w, p = torch.zeros(1, dtype=torch.int32), torch.zeros(1, 2, 16), torch.zeros(1, 2, 16, dtype=torch.int32)
    for call in (lambda: binding.tree_attention(q[:, :, None], K, K, n), lambda: binding.tree_attention(q, K, K, n),
                 lambda: binding.decode_attention_accumulate(q, K, K, n, w), lambda: binding.cache_evict(K, K, n, p, w, 4),
                 lambda: binding.block_bounds(K, n, torch.zeros(1, 2, 1, 2, 64, dtype=torch.bfloat16), 16),
                 lambda: binding.block_select(q, torch.zeros(1, 2, 1, 2, 64, dtype=torch.bfloat16), n, 16, 1),
                 lambda: binding.decode_attention_blocks(q, K, K, n, p, 16)):
        with pytest.raises(ValueError):
            call()                                             # not on the GPU, or with other dimensions
    with pytest.raises(ValueError):
        binding._row_values(w, "weights", torch.float32, 1, 2, 17, 0)      # fewer rows than the cache
    with pytest.raises(ValueError):
        binding._bounds_of(torch.zeros(1, 2, 3, 2, 64), 1, 2, 4, 64, torch.float32, 0)

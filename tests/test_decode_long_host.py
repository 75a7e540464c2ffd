"""Refusals of pkv_decode_attention_long before anything is launched, and its workspace sizes (no GPU)."""
import ctypes
import math

import pytest
import torch

from paper_2406_02069_amd import binding

I, U, W = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED, binding.ERR_WORKSPACE


def _desc(**kw):
    base = dict(B=1, Hq=32, Hkv=8, d=128, k_cap=8192, page_size=0, num_pages=0, max_pages=0, dtype=0, window=0, scale=0.0, cap=0.0,
                q_sb=32 * 128, q_sh=128, c_sb=8 * 8192 * 128, c_sh=8192 * 128, c_st=128, p_sb=8 * 8192, p_sh=8192)
    base.update(kw)
    return binding.DecodeLongDesc(**base)


def _call(desc, **kw):
    lib = binding.load()
    p = dict(q=0x1000, K=0x2000, V=0x3000, table=None, count=0x4000, pos=None, qp=None, sl=None, out=0x5000, lse=None, ws=0x10000,
             n=lib.pkv_decode_long_workspace_bytes(ctypes.byref(desc)))
    p.update(kw)
    return lib.pkv_decode_attention_long(ctypes.byref(desc), *p.values(), None)


@pytest.mark.parametrize("kw", [dict(B=0), dict(Hq=0), dict(Hkv=0), dict(Hq=30), dict(k_cap=0), dict(page_size=-1), dict(dtype=2),
                                dict(window=-1), dict(scale=-1.0), dict(scale=math.nan), dict(cap=-0.5), dict(cap=math.inf),
                                dict(q_sh=4), dict(q_sb=-8), dict(c_st=129), dict(c_sh=-8), dict(p_sb=-1),
                                dict(page_size=16, num_pages=0, max_pages=512), dict(page_size=16, num_pages=1, max_pages=511)])
def test_descriptors_refused(kw):
    d = _desc(**kw)
    assert binding.load().pkv_decode_long_workspace_bytes(ctypes.byref(d)) == 0
    assert _call(d, table=0x6000, n=1 << 30) == I


def test_what_is_not_built():
    for kw in (dict(d=96), dict(Hq=129, Hkv=1), dict(B=65536), dict(k_cap=2 ** 30 + 1),
               dict(page_size=2 ** 20, num_pages=2 ** 12, max_pages=1)):
        assert _call(_desc(**kw), table=0x6000, n=1 << 40) == U


def test_pointers_and_workspace_refused():
    good = _desc()
    need = binding.load().pkv_decode_long_workspace_bytes(ctypes.byref(good))
    assert need > 0
    for kw in (dict(q=None), dict(K=None), dict(V=None), dict(count=None), dict(out=None), dict(q=0x1008), dict(K=0x2004),
               dict(out=0x5008), dict(count=0x4002), dict(pos=0x7001), dict(sl=0x7002), dict(lse=0x7003)):
        assert _call(good, **kw) == I
    for kw in (dict(ws=None), dict(ws=0x10080), dict(n=need - 1)):
        assert _call(good, **kw) == W
    assert _call(_desc(page_size=16, num_pages=600, max_pages=512)) == I        # no table
    assert binding.load().pkv_decode_long_workspace_bytes(ctypes.byref(_desc(k_cap=200))) == 0


def test_binding_refuses_tensors_that_do_not_fit():
    q, K = torch.zeros(1, 8, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 16, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        binding.decode_attention_long(q, K, K, torch.zeros(1, dtype=torch.int32))           # not on the GPU
    with pytest.raises(ValueError):
        binding.decode_attention_long(q.float(), K, K, torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError):
        binding._scale(0.0)


def test_factors_that_are_not_finite_and_wide_rows():
    assert _call(_desc(cap=1e-44)) == I                        # the quotient of scale and cap
    assert _call(_desc(cap=3e38)) == I                         # the cap in units of log2
    assert _call(_desc(scale=3e38)) == I
    assert _call(_desc(c_st=2 ** 30 + 8)) == U
    assert _call(_desc(B=65535, Hq=512, Hkv=512)) == U


def test_binding_refuses_a_workspace_elsewhere():
    with pytest.raises(ValueError):
        binding._workspace(torch.zeros(8, dtype=torch.uint8), 0)
    assert binding._workspace(None, 0) == (None, 0)

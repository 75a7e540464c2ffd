"""Refusals of pkv_prefill_attention before anything is launched, and its workspace sizes (no GPU)."""
import ctypes
import math

import pytest
import torch

from paper_2406_02069_amd import binding

I, U, W = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED, binding.ERR_WORKSPACE


def _desc(**kw):
    base = dict(B=1, Hq=32, Hkv=8, d=128, T=64, N=8192, dtype=0, window=0, scale=0.0, cap=0.0,
                q_sb=32 * 64 * 128, q_sh=64 * 128, q_st=128, kv_sb=8 * 8192 * 128, kv_sh=8192 * 128, kv_st=128,
                o_sb=32 * 64 * 128, o_sh=64 * 128, o_st=128)
    base.update(kw)
    return binding.PrefillDesc(**base)


def _need(d):
    return binding.load().pkv_prefill_workspace_bytes(ctypes.byref(d))


def _call(desc, **kw):
    p = dict(q=0x1000, K=0x2000, V=0x3000, lens=None, start=None, doc=None, pre=None, sl=None, out=0x5000, lse=None, ws=0x10000,
             n=_need(desc))
    p.update(kw)
    return binding.load().pkv_prefill_attention(ctypes.byref(desc), *p.values(), None)


@pytest.mark.parametrize("kw", [dict(B=0), dict(Hq=0), dict(Hkv=0), dict(Hq=30), dict(T=0), dict(N=0), dict(dtype=2), dict(dtype=-1),
                                dict(window=-1), dict(scale=-1.0), dict(scale=math.inf), dict(cap=-0.5), dict(cap=math.nan),
                                dict(q_st=4), dict(q_sb=-8), dict(kv_st=129), dict(kv_sh=-8), dict(o_st=1), dict(o_sb=12)])
def test_descriptors_refused(kw):
    assert _need(_desc(**kw)) == 0
    assert _call(_desc(**kw), n=1 << 40) == I


def test_what_is_not_built():
    for kw in (dict(d=96), dict(Hq=129, Hkv=1), dict(B=65536), dict(N=2 ** 30 + 1), dict(T=2 ** 30 + 1), dict(T=2 ** 30),
               dict(kv_st=2 ** 23 + 8), dict(Hkv=2 ** 20, Hq=2 ** 20, T=2 ** 22)):
        assert _call(_desc(**kw), n=1 << 60) == U, kw


def test_pointers_and_workspace_refused():
    good = _desc()
    need = _need(good)
    assert need > 0 and _need(_desc(T=8192)) == 0
    for kw in (dict(q=None), dict(K=None), dict(V=None), dict(out=None), dict(q=0x1008), dict(K=0x2004), dict(out=0x5008),
               dict(lens=0x4002), dict(start=0x7001), dict(doc=0x7002), dict(pre=0x7003), dict(sl=0x7002), dict(lse=0x7003)):
        assert _call(good, **kw) == I
    for kw in (dict(ws=None), dict(ws=0x10080), dict(n=need - 1)):
        assert _call(good, **kw) == W


def test_binding_refuses_tensors_that_do_not_fit():
    q, K = torch.zeros(1, 8, 4, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 16, 64, dtype=torch.bfloat16)
    for args in ((q, K, K), (q.float(), K, K), (q[0], K, K), (q.transpose(2, 3), K, K)):
        with pytest.raises(ValueError):
            binding.prefill_attention(*args)


def test_factors_that_are_not_finite():
    for kw in (dict(cap=1e-44), dict(cap=3e38), dict(scale=3e38)):
        assert _call(_desc(**kw)) == I

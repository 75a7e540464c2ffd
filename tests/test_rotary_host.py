"""Host side of the rotary positions: frequencies against their formulas, refusals before anything is launched (no GPU)."""
import ctypes
import math

import pytest
import torch

from paper_2406_02069_amd import binding

I, U = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED


@pytest.mark.parametrize("rot,base", [(2, 10000.0), (24, 10000.0), (64, 500000.0), (128, 1e6), (256, 2.0)])
def test_frequencies(rot, base):
    trained, low, high, factor = 4096.0, 1.0, 8.0, 5.0
    for name in binding.ROTARY_SCALINGS:
        got, m = binding.rotary_frequencies(rot, name, base, factor, trained, low, high)
        pair = lambda u: rot * math.log(trained / (2 * math.pi * u)) / (2 * math.log(base))
        lo, hi = max(math.floor(pair(high)), 0), min(math.ceil(pair(low)), rot - 1)
        for i in range(rot // 2):
            f = base ** (-2 * i / rot)
            if name == "linear":
                f = f / factor
            elif name == "bands":
                u = trained * f / (2 * math.pi)
                s = (u - low) / (high - low)
                f = f / factor if u <= low else f if u >= high else (1 - s) * f / factor + s * f
            elif name == "ramp":
                r = min(max((i - lo) / max(hi - lo, 0.001), 0), 1)
                f = f / factor * r + f * (1 - r)
            assert abs(got[i].item() - f) <= 1e-13 * f, (name, i)      # a few roundings in 64 bits
        assert m == pytest.approx(0.1 * math.log(factor) + 1 if name == "ramp" else 1.0, rel=1e-7)


@pytest.mark.parametrize("bad", [dict(rot=0), dict(rot=7), dict(rot=258), dict(base=1.0), dict(base=math.inf), dict(factor=0.5),
                                 dict(factor=math.nan), dict(trained=0.0), dict(low=0.0), dict(low=9.0), dict(high=math.inf)])
def test_frequencies_refuse(bad):
    args = dict(rot=64, scaling="bands", base=10000.0, factor=2.0, trained=4096.0, low=1.0, high=8.0)
    args.update(bad)
    with pytest.raises(binding.PkvError) as e:
        binding.rotary_frequencies(**args)
    assert e.value.status == I
    assert binding.load().pkv_rotary_frequencies(64, 4, 1e4, 1, 1, 1, 2, (ctypes.c_double * 32)(), ctypes.byref(ctypes.c_float())) == I
    assert binding.load().pkv_rotary_frequencies(64, 0, 1e4, 1, 1, 1, 2, None, ctypes.byref(ctypes.c_float())) == I


def _desc(**kw):
    base = dict(B=2, Hq=8, Hkv=2, d=128, T=4, rot=128, layout=0, dtype=0, k_cap=16, page_size=0, num_pages=0, max_pages=0,
                magnitude=1.0, reserved=0)
    for n, h in (("q", 8), ("k", 2), ("v", 2), ("o", 8)):
        base.update({n + "_sb": h * 512, n + "_sh": 512, n + "_st": 128})
    base.update(c_sb=2 * 16 * 128, c_sh=16 * 128, c_st=128, p_sb=32, p_sh=16)
    base.update(kw)
    return binding.RotaryDesc(**base)


def _call(desc, **kw):
    p = dict(q=0x1000, k=0x2000, v=0x3000, f=0x4000, pos=None, new=None, count=None, table=None, qo=0x5000, K=0x6000, V=0x7000,
             pc=None, dr=None)
    p.update(kw)
    return binding.load().pkv_rotary_append(ctypes.byref(desc), *p.values(), None)


@pytest.mark.parametrize("kw", [dict(B=0), dict(Hq=0), dict(Hkv=0), dict(T=0), dict(reserved=1), dict(layout=2), dict(layout=-1),
                                dict(dtype=2), dict(rot=0), dict(rot=130), dict(rot=7), dict(magnitude=math.nan), dict(k_cap=0),
                                dict(q_st=4), dict(o_sh=513), dict(k_sb=-8), dict(v_st=129), dict(c_st=64), dict(c_sb=1),
                                dict(page_size=-1), dict(page_size=4, num_pages=3, max_pages=4)])
def test_descriptors_refused(kw):
    assert _call(_desc(**kw)) == I


def test_what_is_not_built():
    assert _call(_desc(d=96, rot=96)) == U
    assert _call(_desc(rot=12)) == U
    assert _call(_desc(B=2 ** 16, T=2 ** 15)) == U
    assert _call(_desc(Hq=70000)) == U


@pytest.mark.parametrize("kw", [dict(q=None), dict(qo=None), dict(k=None), dict(V=None), dict(f=None), dict(q=0x1008), dict(K=0x6004),
                                dict(f=0x4004), dict(pos=0x8002), dict(count=0x8001), dict(dr=0x8002), dict(pc=0x8002),
                                dict(q=None, qo=None, k=None, v=None, K=None, V=None),
                                dict(k=None, v=None, K=None, V=None, pc=0x8000)])
def test_pointers_refused(kw):
    assert _call(_desc(), **kw) == I


def test_pages_without_a_table_or_too_few_entries():
    assert _call(_desc(page_size=4, num_pages=3, max_pages=4)) == I
    assert _call(_desc(page_size=4, num_pages=3, max_pages=3), table=0x9000) == I
    assert _call(_desc(page_size=4, num_pages=0, max_pages=4), table=0x9000) == I


def test_binding_refuses_tensors_that_do_not_fit():
    x = torch.zeros(1, 4, 2, 64, dtype=torch.bfloat16)
    f = torch.zeros(32, dtype=torch.float64)
    with pytest.raises(ValueError):
        binding.rotary_append(x, None, None, f)                       # not on the GPU
    with pytest.raises(ValueError):
        binding.rotary_append(None, None, None, f)
    with pytest.raises(ValueError):
        binding.rotary_append(x.float(), None, None, f)
    with pytest.raises(ValueError):
        binding.rotary_append(x, x, x, f)                             # no caches

"""Workspace sizes of prompt attention with and without lengths (no GPU)."""
import ctypes

import pytest

from paper_2406_02069_amd import binding
from tests.test_prefill_host import W, _call, _desc, _need


def _even(d):
    return binding.load().pkv_prefill_even_workspace_bytes(ctypes.byref(d))


@pytest.mark.parametrize("kw,even,any_", [
    (dict(B=8, Hq=8, Hkv=8, T=8192, N=8192), 0, 2 * 1536 * 128 * 130 * 4),        # even prompts need none, ragged ones slots
    (dict(B=2, T=2048, N=65536), 0, 2 * 1536 * 128 * 130 * 4),
    (dict(B=1, T=64, N=8192), None, None), (dict(B=4, T=64, N=3000), None, None)])  # one sequence, few keys: the same
def test_sizes(kw, even, any_):
    d = _desc(**kw)
    if any_ is None:
        assert 0 < _even(d) == _need(d)
    else:
        assert (_even(d), _need(d)) == (even, any_)


def test_what_a_call_asks_for():
    # (calls that are refused, so that nothing is launched)
    for kw in (dict(B=2, T=64, N=9000), dict(B=1, T=64, N=8192), dict(B=3, T=100, N=20000)):
        d = _desc(**kw)
        even, most = _even(d), _need(d)
        assert 0 < even <= most
        assert _call(d, n=even - 1) == W and _call(d, ws=None) == W
        if d.B > 1:
            ragged = most if most > even else None
            for lens, start in ((0x4000, None), (None, 0x4000)):
                assert _call(d, lens=lens, start=start, n=0) == W
                if ragged is not None:
                    assert _call(d, lens=lens, start=start, n=most - 1) == W
    d = _desc(B=8, Hq=8, Hkv=8, T=8192, N=8192)
    assert _call(d, lens=0x4000, n=_need(d) - 1) == W and _call(d, lens=0x4000, ws=None) == W


def test_invalid_descriptors_have_none():
    assert _even(_desc(B=0)) == _even(_desc(d=96)) == _even(_desc(T=0)) == 0


def test_descriptors_with_small_and_large_caps():
    # what is refused has no workspace: a cap, or a quotient with the scale, that is no fp32 number
    for cap in (1e-3, 1e-8, 1e-30, 1e-37, 1e6, 1e30):
        assert _need(_desc(cap=cap)) > 0, cap
    for cap in (1e-40, 3e38):
        assert _need(_desc(cap=cap)) == 0, cap

"""Frequencies of rotary positions: the definition, and what each scaling keeps and slows."""
import numpy as np
import pytest

from paper_2011_10680_amd.convert import rotary_turns


@pytest.mark.parametrize("dim", [2, 4, 20, 64, 128])
def test_definition(dim):
    t = rotary_turns(dim, base=500.0)
    assert t.dtype == np.float64 and t.shape == (dim // 2,)
    for f in range(dim // 2):
        assert t[f] * 2 * np.pi == pytest.approx(500.0 ** (-2 * f / dim), rel=1e-14)


def test_scalings():
    plain = rotary_turns(64)
    assert np.allclose(rotary_turns(64, scaling="linear", factor=4.0), plain / 4, rtol=1e-15)
    base = rotary_turns(64, scaling="base", factor=4.0)
    assert base[0] == plain[0] and base[-1] == pytest.approx(plain[-1] / 4, rel=1e-12) and (np.diff(base / plain) < 0).all()
    parts = rotary_turns(64, scaling="parts", factor=8.0, original=8192, low=1.0, high=32.0)
    often, seldom = plain * 8192 >= 32, plain * 8192 <= 1
    assert often.any() and seldom.any()
    assert np.array_equal(parts[often], plain[often]) and np.allclose(parts[seldom], plain[seldom] / 8, rtol=1e-15)
    between = ~often & ~seldom
    assert ((parts < plain) & (parts > plain / 8))[between].all()
    assert np.array_equal(rotary_turns(64, scaling="parts", factor=1.0, original=100), plain)


@pytest.mark.parametrize("kw", [dict(rotary_dim=0), dict(rotary_dim=7), dict(rotary_dim=8, base=0.0), dict(rotary_dim=8, factor=0.5), dict(rotary_dim=8, scaling="other"),
                                dict(rotary_dim=8, scaling="parts"), dict(rotary_dim=8, scaling="parts", original=100, low=4.0, high=2.0)])
def test_refusals(kw):
    with pytest.raises(ValueError):
        rotary_turns(**kw)

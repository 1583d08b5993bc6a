"""The 4-bit group quantiser on the host: every weight within half a step of its code, and the codes' packing."""
import numpy as np
import pytest

import lm_reference as ref
from paper_2011_10680_amd.convert import quantize_groups


@pytest.mark.parametrize("N,K,group", [(3, 64, 32), (5, 96, 64), (1, 130, 128), (4, 2, 32)])
@pytest.mark.parametrize("zero_points", [False, True])
def test_codes_stand_for_the_weights(N, K, group, zero_points):
    r = np.random.default_rng(K)
    W = r.normal(size=(N, K)) + (0.7 if zero_points else 0.0)
    w, s, z = quantize_groups(W, group, zero_points)
    assert w.shape == (N, K // 2) and s.shape == (N, -(-K // group)) and (z is None) == (not zero_points)
    q = ref.unpack(w, z, group)
    step = np.repeat(s, group, axis=1)[:, :K]
    # half a step; the largest magnitude of a symmetric group lies half a step past its code 7, a zero point moves a range by half a step
    assert (np.abs(q * step - W) <= (1.0 if zero_points else 0.5) * step * (1 + 1e-12)).all()
    if not zero_points:
        assert q.min() >= -7 and q.max() <= 7


def test_zeros_and_refusals():
    w, s, z = quantize_groups(np.zeros((2, 32)), 32)
    assert not w.any() and (s == 1).all() and z is None
    w, s, z = quantize_groups(np.zeros((2, 32)), 32, True)
    assert not ref.unpack(w, z, 32).any()
    for K, group in ((33, 32), (32, 48), (32, 0), (32, -32)):
        with pytest.raises(ValueError):
            quantize_groups(np.zeros((1, K)), group)

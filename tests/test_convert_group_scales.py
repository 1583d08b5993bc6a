"""The 4-bit group quantiser with its scales in the activations' type: codes belong to the scale that the operator is given."""
import numpy as np
import pytest
import torch

import lm_reference as ref
from paper_2011_10680_amd import BF16, F16, S8
from paper_2011_10680_amd.convert import quantize_groups

_TYPES = {F16: torch.float16, BF16: torch.bfloat16}


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("zero_points", [False, True])
def test_codes_are_the_nearest_for_the_rounded_scale(dtype, zero_points):
    r = np.random.default_rng(dtype)
    W = r.normal(size=(40, 224)) + (0.4 if zero_points else 0.0)
    w, s, z = quantize_groups(W, 64, zero_points, dtype)
    assert np.array_equal(torch.from_numpy(s).to(_TYPES[dtype]).double().numpy(), s)                 # what the type holds,
    exact = quantize_groups(W, 64, zero_points)[1]
    assert (np.abs(s - exact) <= (2.0 ** -11 if dtype == F16 else 2.0 ** -8) * exact).all()       # and near
    step = np.repeat(s, 64, axis=1)[:, :224]
    code = ref.unpack(w, z, 64)
    lo, hi = (-7, 7) if z is None else (-np.repeat(z.astype(int), 64, axis=1)[:, :224], 15 - np.repeat(z.astype(int), 64, axis=1)[:, :224])
    assert np.array_equal(code, np.clip(np.rint(W / step), lo, hi))
    # with codes of the scale in 64 bits some lie past half a step of the scale in use
    other = ref.unpack(quantize_groups(W, 64, zero_points)[0], z, 64)
    if dtype == BF16 and not zero_points:
        assert (np.abs(other * step - W)[np.abs(other) < 7] > 0.5001 * step[np.abs(other) < 7]).any()


@pytest.mark.parametrize("dtype,tiny,far", [(F16, 1e-9, 1e6), (BF16, 1e-41, None)])
def test_scales_at_the_ends_of_the_type(dtype, tiny, far):
    W = np.zeros((2, 64))
    W[0, 3] = tiny
    w, s, _ = quantize_groups(W, 32, False, dtype)
    assert s[0, 0] > 0 and (s[0, 1], s[1, 0]) == (1.0, 1.0)
    assert np.array_equal(torch.from_numpy(s).to(_TYPES[dtype]).double().numpy(), s)
    step = np.repeat(s, 32, axis=1)
    assert (np.abs(ref.unpack(w, None, 32) * step - W) <= 0.5 * step).all()
    if far is not None:
        with pytest.raises(ValueError):
            quantize_groups(np.full((1, 32), far), 32, False, dtype)


def test_other_types_are_refused():
    with pytest.raises(ValueError):
        quantize_groups(np.ones((1, 32)), 32, False, S8)

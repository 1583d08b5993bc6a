"""hawq_linear_w4 on the GPU within the bound that the interface states: 32-bit sums of |x| * 31 |s|."""
import pytest

import lm_reference as ref
import test_gpu_lm_linear as base

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def stated(monkeypatch):
    """The comparison of test_gpu_lm_linear allows 143 |x| |s| a weight, for a form of the sums that the kernel does not have."""
    monkeypatch.setattr(ref, "F32", ref.F32 * 31 / 143)


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("M,N,K,group", [(1, 1000, 2048, 128), (13, 200, 8192, 64), (64, 129, 1000, 32), (33, 100, 4096, 4096), (5, 49, 250, 96)])
def test_sums(M, N, K, group, dtype, zeros):
    base._run(M, N, K, group, dtype, zeros, True)


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_sums_of_activations_far_from_zero_mean(dtype, zeros):
    base._run(9, 200, 2048, 128, dtype, zeros, False, mean=4.0)
    base._run(20, 200, 4096, 32, dtype, zeros, False, mean=40.0)

"""hawq_adapters on the GPU: tiles of a whole prompt whose rows all have adapters of their own, and one place of the result that is its base's beside one that is not."""
import pytest

from test_gpu_lm_adapters import _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [17, 64, 100])
@pytest.mark.parametrize("in_place", [False, True])
def test_many_adapters_in_a_prompt(n, in_place):
    for i, dtype in enumerate(("f16", "bf16")):
        _run(4200, 40, 72, n, 24, dtype, adapter=[j * 37 % (n + 1) - 1 for j in range(4200)], in_place=in_place, y_pad=8 * i, seed=n)

"""The example's decoder on the GPU where a request, or the cache, has no more room."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def test_a_request_that_outgrows_its_table_is_an_error():
    from paper_2011_10680_amd import lm_example as ex
    r = np.random.default_rng(1)
    prompts = [r.integers(0, 512, size=n).tolist() for n in (30, 2)]
    answers, _, _ = ex.generate(ex.Decoder(2, most=64, seed=3), prompts, 12)
    assert [len(a) for a in answers] == [12, 12]
    with pytest.raises(RuntimeError, match="block table"):
        ex.generate(ex.Decoder(2, most=64, seed=3), prompts, 60, drafting=False)
    with pytest.raises(RuntimeError, match="block table"):
        ex.Decoder(1, most=64).prompts([[1] * 65])


def test_a_full_cache_is_an_error():
    from paper_2011_10680_amd import lm_example as ex
    with pytest.raises(RuntimeError, match="full"):
        ex.Decoder(2, config=dict(ex.CONFIG, pages=3)).prompts([[1] * 40, [2] * 30])

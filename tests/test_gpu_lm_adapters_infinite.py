"""hawq_adapters on the GPU where a sum of its second product is infinite or no number: as the formula has it."""
import numpy as np
import pytest

import lm_step_reference as ref

pytestmark = pytest.mark.gpu


def _run(x, a, b, ranks, scales, adapter, base, dtype, b_pad=0, y_pad=0, in_place=False):
    """(y, what the formula gives, its bound) of values that the type holds"""
    import torch
    import paper_2011_10680_amd as hawq
    dt = {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    (M, K), (n, most, _), N = x.shape, a.shape, b.shape[1]

    def held(v, pad=0):
        t = torch.full(v.shape[:-1] + (v.shape[-1] + pad,), float("nan"), dtype=dt, device="cuda")[..., :v.shape[-1]]
        t.copy_(torch.from_numpy(v.astype(np.float32)))
        return t
    x, a, b, base = held(x), held(a), held(b, b_pad), held(base, y_pad)
    with np.errstate(invalid="ignore"):
        want, bound = ref.adapters(*(t.double().cpu().numpy() for t in (x, a, b)), ranks, scales.astype(np.float32).astype(np.float64), adapter, base.double().cpu().numpy(), dtype)
    y = base if in_place else held(np.zeros((M, N)), y_pad)
    d = hawq.AdaptersDesc(M=M, N=N, K=K, n_adapters=n, max_rank=most, dtype=hawq.F16 if dtype == "f16" else hawq.BF16, x_stride=K, base_stride=N + y_pad, y_stride=N + y_pad,
                          a_adapter=most * K, a_row=K, b_adapter=N * (most + b_pad), b_row=most + b_pad)
    room = torch.full((hawq.hawq_adapters_workspace_bytes(d),), 0xFF, dtype=torch.uint8, device="cuda")
    hawq.hawq_adapters(d, x, a, b, torch.tensor(ranks, dtype=torch.int32, device="cuda"), torch.from_numpy(scales.astype(np.float32)).cuda(),
                       torch.tensor(adapter, dtype=torch.int32, device="cuda"), base, y, room)
    torch.cuda.synchronize()
    return y.double().cpu().numpy(), want, bound


def _same(got, want, bound):
    fine = np.isfinite(want)
    assert (np.isnan(got) == np.isnan(want)).all(), np.argwhere(np.isnan(got) != np.isnan(want))[:5].tolist()
    assert (got[np.isinf(want)] == want[np.isinf(want)]).all()
    assert (np.abs(got[fine] - want[fine]) <= bound[fine]).all()


@pytest.mark.parametrize("M", [1, 5, 40, 4100])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("in_place,b_pad,y_pad", [(False, 0, 0), (True, 0, 0), (False, 1, 0), (True, 0, 3)])
@pytest.mark.parametrize("most", [16, 200])
def test_infinities_in_the_second_matrix(M, dtype, in_place, b_pad, y_pad, most):
    """Inner sums that the type holds and ones that it does not, all above 0 but those of a row of zeros: the sign of an infinity is b's and the scale's."""
    r = np.random.default_rng(M + most)
    N, K = 72, 32
    x, a, b, base = r.uniform(0.5, 2, size=(M, K)), r.uniform(0.5, 2, size=(2, most, K)), r.normal(size=(2, N, most)), r.normal(size=(M, N))
    x[::3] = 0
    x[::3, 7] = 1                                     # (an element of a: nothing is left for the second part)
    x[1::5] = 0                                       # (0 times an infinity is no number)
    inf = np.inf
    b[0, 3, 2], b[0, 5, 0], b[1, 17, most - 9] = inf, -inf, inf
    b[0, 8, 1], b[0, 8, 4] = inf, inf
    b[0, 40, 1], b[0, 40, 6] = inf, -inf
    b[1, 71, :] = -inf
    b[:, 33, most - 3:] = inf                         # past the ranks
    y = _run(x, a, b, [most - 3, most - 5], np.array([0.5, -0.25]), [(i % 4 + 3) % 4 - 1 if i else 0 for i in range(M)], base, dtype, b_pad, y_pad, in_place)
    assert np.isinf(y[1]).any() and (M < 5 or np.isnan(y[1]).any())
    _same(*y)


@pytest.mark.parametrize("M", [3, 4100])
def test_inner_sums_between_the_largest_bfloat16_and_infinity(M):
    """3.4e38 is a number of 32 bits and rounds to infinity in bf16."""
    K, N, R = 16, 40, 8
    x, a, b = np.ones((M, K)), np.zeros((1, R, K)), np.full((1, N, R), 2.0 ** -120)
    a[0, 1, :2] = 3.3895e38, 1.0e36
    a[0, 2, :2] = -3.3895e38, -0.9e36
    _same(*_run(x, a, b, [R], np.ones(1), [0] * M, np.zeros((M, N)), "bf16"))
    b[0, 4, 1] = 2.0                                  # beyond 32 bits
    b[0, 5, 1:3] = 2.0                                # (the difference of two such is not: 2^102 or so)
    got, want, bound = _run(x, a, b, [R], np.ones(1), [0] * M, np.zeros((M, N)), "bf16")
    rest = [n for n in range(N) if n not in (4, 5)]
    _same(got[:, rest], want[:, rest], bound[:, rest])
    assert np.isposinf(got[:, 4]).all()

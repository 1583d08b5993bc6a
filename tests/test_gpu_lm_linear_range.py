"""hawq_linear_w4 on the GPU at the ends of bf16's range and with infinite scales: what the formula gives, term by term."""
import numpy as np
import pytest

import lm_reference as ref

pytestmark = pytest.mark.gpu


def _call(x, w, s, z, bias, group, dtype="bf16"):
    import torch
    import paper_2011_10680_amd as hawq
    dt, ht = (torch.float16, hawq.F16) if dtype == "f16" else (torch.bfloat16, hawq.BF16)
    M, K = x.shape
    N = w.shape[0]
    to = lambda a: torch.from_numpy(np.asarray(a, np.float32)).to(dt)  # noqa: E731
    x, s, bias = to(x), to(s), None if bias is None else to(bias)
    y = torch.full((M, N), 7.0, dtype=dt, device="cuda")
    d = hawq.LinearW4Desc(M=M, N=N, K=K, group=group, x_dtype=ht, w_dtype=hawq.S4 if z is None else hawq.U4, x_stride=K, y_stride=N)
    hawq.hawq_linear_w4(d, x.cuda(), torch.from_numpy(w).cuda(), s.cuda(), None if z is None else torch.from_numpy(z).cuda(), None if bias is None else bias.cuda(), y)
    f64 = lambda t: t.float().numpy().astype(np.float64)  # noqa: E731
    return f64(y.cpu()), f64(x), f64(s), None if bias is None else f64(bias)


def _formula(x, w, s, z, bias, group):
    """Every term on its own: an infinity times a 0 is NaN, wherever the 0 stands."""
    q = ref.unpack(w, z, group).astype(np.float64)
    spread = np.repeat(s, group, axis=1)[:, :q.shape[1]]
    with np.errstate(invalid="ignore"):
        y = np.stack([(row[None] * q * spread).sum(axis=1) for row in x])
        return y if bias is None else y + bias


def _compare(got, want, u, size):
    finite = np.isfinite(want)
    with np.errstate(invalid="ignore"):
        bound = u * np.abs(want) + 2.0 ** -40 * size
        same = np.where(finite, np.abs(got - want) <= bound, np.where(np.isnan(want), np.isnan(got), got == want))
    assert same.all(), (np.argwhere(~same)[:4], got[~same][:4], want[~same][:4])


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("M,K,group", [(1, 64, 32), (5, 352, 64), (33, 1000, 128)])
def test_products_past_the_range_whose_scaled_sums_are_inside(M, K, group, zeros):
    """Activations of 1e38 times codes leave 32 bits, times their scales they are back: one such value a row, or two that cancel in part."""
    r = np.random.default_rng(K)
    N, groups = 70, -(-K // group)
    w = r.integers(0, 256, size=(N, K // 2), dtype=np.uint8)
    z = r.integers(0, 16, size=(N, groups), dtype=np.uint8) if zeros else None
    s = r.uniform(2.0 ** -10, 2.0 ** -7, size=(N, groups))
    x = np.zeros((M, K))
    for m in range(M):
        at = r.choice(K, size=2, replace=False)
        x[m, at] = (3e38, 0) if m % 2 == 0 else (2e38, -2.5e38)
    got, x, s, _ = _call(x, w, s, z, None, group)
    want = _formula(x, w, s, z, None, group)
    assert np.isfinite(want).all()
    _compare(got, want, ref.ROUND["bf16"], np.abs(want))


@pytest.mark.parametrize("zeros", [False, True])
def test_infinite_scales_and_a_bias(zeros):
    r = np.random.default_rng(1)
    M, N, K, group = 6, 40, 256, 64
    w = r.integers(0, 256, size=(N, K // 2), dtype=np.uint8)
    z = r.integers(0, 16, size=(N, 4), dtype=np.uint8) if zeros else None
    s = r.uniform(0.01, 0.1, size=(N, 4))
    s[3, 1], s[7, 0], s[11, 3], s[12, 2] = np.inf, -np.inf, np.nan, 0.0
    s[5] = np.inf
    if zeros:
        z[5] = 4
    w[5] = 0x55                                                            # (no weight of this output is 0)
    x = np.abs(r.normal(size=(M, K))) + 0.5
    x[2, 70] = 0.0
    x[3, 5], x[4, 200] = np.inf, np.nan
    bias = r.normal(size=N)
    for dtype in ("f16", "bf16"):
        got, xr, sr, br = _call(x, w, s, z, bias, group, dtype)
        want = _formula(xr, w, sr, z, br, group)
        assert np.isposinf(want[0, 5]) and np.isnan(want[2, 5])
        size = np.where(np.isfinite(want), 2.0 ** 40 * (K + 100) * ref.F32 * 31 * (np.abs(np.where(np.isfinite(xr), xr, 0)).sum(axis=1)[:, None] * 0.1 + 10), 0)
        _compare(got, want, ref.ROUND[dtype], size)


@pytest.mark.parametrize("K", [256, 250])
@pytest.mark.parametrize("M", [1, 5, 40])
def test_one_row_of_x_for_all(M, K):
    """A stride of 0: every row of y is the first one's."""
    import torch
    import paper_2011_10680_amd as hawq
    g = torch.Generator(device="cuda").manual_seed(K)
    x = torch.randn((1, K), generator=g, device="cuda").half()
    w = torch.randint(0, 256, (70, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    s = torch.rand((70, 4), generator=g, device="cuda").half()
    y, want = torch.empty((2, M, 70), dtype=torch.float16, device="cuda")
    for out, rows in ((y, x.expand(M, K)), (want, x.repeat(M, 1))):
        d = hawq.LinearW4Desc(M=M, N=70, K=K, group=64, x_dtype=hawq.F16, w_dtype=hawq.S4, x_stride=0 if out is y else K, y_stride=70)
        hawq.hawq_linear_w4(d, rows, w, s, None, None, out)
    assert torch.equal(y, want)

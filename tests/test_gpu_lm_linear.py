"""hawq_linear_w4 on the GPU against the definition in 64 bits."""
import numpy as np
import pytest

import lm_reference as ref

pytestmark = pytest.mark.gpu


def _run(M, N, K, group, dtype, zeros, bias, x_pad=0, y_pad=0, w_at=0, x_at=0, mean=0.0, seed=0, stream=None):
    import torch
    import paper_2011_10680_amd as hawq
    dt = {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    r = np.random.default_rng(seed)
    groups = -(-K // group)
    rounded = lambda a: torch.from_numpy(a.astype(np.float32)).to(dt)  # noqa: E731
    x = rounded(r.normal(size=(M, K)) + mean)
    w = r.integers(0, 256, size=(N, K // 2), dtype=np.uint8)
    s = rounded(r.uniform(0.002, 0.01, size=(N, groups)) * np.where(r.random((N, groups)) < 0.1, -1, 1))
    z = r.integers(0, 16, size=(N, groups), dtype=np.uint8) if zeros else None
    b = rounded(r.normal(size=N)) if bias else None
    # operands with padding around them that must not be read into the result nor written over
    xw = torch.full((M * (K + x_pad) + x_at + 64,), float("nan"), dtype=dt, device="cuda")
    xd = xw[x_at:x_at + M * (K + x_pad)].view(M, K + x_pad)[:, :K]
    xd.copy_(x)
    ww = torch.full((w_at + w.size + 64,), 0x77, dtype=torch.uint8, device="cuda")
    wd = ww[w_at:w_at + w.size]
    wd.copy_(torch.from_numpy(w).reshape(-1))
    y = torch.full((M, N + y_pad), 7.0, dtype=dt, device="cuda")
    d = hawq.LinearW4Desc(M=M, N=N, K=K, group=group, x_dtype=hawq.F16 if dtype == "f16" else hawq.BF16, w_dtype=hawq.U4 if zeros else hawq.S4,
                          x_stride=K + x_pad, y_stride=N + y_pad)
    hawq.hawq_linear_w4(d, xd, wd, s.cuda(), None if z is None else torch.from_numpy(z).cuda(), None if b is None else b.cuda(), y, stream=stream)
    torch.cuda.synchronize()
    got = y.float().cpu().numpy().astype(np.float64)
    assert (got[:, N:] == 7.0).all()
    want, size = ref.linear(x.float().numpy().astype(np.float64), w, s.float().numpy(), z, None if b is None else b.float().numpy().astype(np.float64), group)
    u = ref.ROUND[dtype]
    # the kernel may sum x (q + 128): at most 143 for a weight, in sums of a group's products and then of the groups
    bound = u * np.abs(want) + (1 + u) * ref.F32 * (group + groups + 64) * 143 * size
    assert (np.abs(got[:, :N] - want) <= bound).all(), (M, N, K, float((np.abs(got[:, :N] - want) / bound).max()))
    norm = np.linalg.norm(want)
    assert np.linalg.norm(got[:, :N] - want) <= (u + 1e-4) * norm


@pytest.mark.parametrize("M", [1, 2, 7, 15, 16, 17, 33, 64, 65, 130])
@pytest.mark.parametrize("N,K,group,dtype,zeros", [(100, 256, 128, "bf16", True), (33, 2048, 32, "f16", False), (1000, 512, 64, "bf16", False)])
def test_rows(M, N, K, group, dtype, zeros):
    _run(M, N, K, group, dtype, zeros, M % 2 == 0, seed=M)


@pytest.mark.parametrize("K", [2, 30, 32, 34, 64, 72, 96, 120, 128, 160, 250, 1000, 1056, 4096, 8200])
@pytest.mark.parametrize("group", [32, 64, 96, 128, 8224])
def test_reductions(K, group):
    for i, (dtype, zeros) in enumerate((("f16", True), ("bf16", True), ("f16", False), ("bf16", False))):
        _run(3 + 5 * i, 49, K, group, dtype, zeros, i % 2 == 1, seed=K + i)


@pytest.mark.parametrize("N", [1, 5, 16, 63, 64, 129, 4097, 20000])
def test_outputs(N):
    _run(1, N, 384, 128, "f16", False, True, seed=N)
    _run(20, N, 96, 32, "bf16", True, False, y_pad=3, seed=N)


@pytest.mark.parametrize("M,N,K", [(3, 40, 20000), (20, 6200, 8320), (40, 12300, 4160), (64, 3100, 160), (50, 200, 1056)])
def test_more_groups_than_fit_at_once(M, N, K):
    _run(M, N, K, 32, "bf16", True, False, seed=K)
    _run(M, N, K, 32, "f16", False, True, seed=K)


def test_rows_far_apart():
    """Rows of x whose offsets leave 32 bits of elements inside a tile."""
    import torch
    import paper_2011_10680_amd as hawq
    stride, M, N, K = 1 << 28, 13, 48, 256
    x = torch.empty((M - 1) * stride + K, dtype=torch.float16, device="cuda").as_strided((M, K), (stride, 1))
    g = torch.Generator(device="cuda").manual_seed(1)
    near = torch.randn((M, K), generator=g, device="cuda").half()
    x.copy_(near)
    w = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    s = torch.rand((N, 2), generator=g, device="cuda").half()
    y, want = torch.empty((2, M, N), dtype=torch.float16, device="cuda")
    for a, out, step in ((x, y, stride), (near, want, K)):
        hawq.hawq_linear_w4(hawq.LinearW4Desc(M=M, N=N, K=K, group=128, x_dtype=hawq.F16, w_dtype=hawq.S4, x_stride=step, y_stride=N), a, w, s, None, None, out)
    torch.cuda.synchronize()
    assert torch.equal(y, want)


@pytest.mark.parametrize("x_pad,x_at,w_at", [(8, 0, 0), (5, 0, 0), (0, 1, 0), (3, 3, 1), (0, 0, 4), (0, 0, 2), (0, 8, 16)])
def test_strides_and_alignment(x_pad, x_at, w_at):
    for dtype in ("f16", "bf16"):
        _run(5, 70, 320, 64, dtype, True, True, x_pad=x_pad, x_at=x_at, w_at=w_at)
        _run(18, 70, 328, 64, dtype, False, True, x_pad=x_pad, x_at=x_at, w_at=w_at)


def test_activations_far_from_zero_mean():
    for dtype in ("f16", "bf16"):
        _run(9, 200, 2048, 128, dtype, True, False, mean=4.0)


def test_another_stream_and_repeatability():
    import torch
    import paper_2011_10680_amd as hawq
    side = torch.cuda.Stream()
    M, N, K = 6, 512, 1024
    g = torch.Generator(device="cuda").manual_seed(3)
    w = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    s = torch.rand((N, K // 64), generator=g, device="cuda").to(torch.float16)
    x0 = torch.randn((M, K), generator=g, device="cuda").to(torch.float16)
    d = hawq.LinearW4Desc(M=M, N=N, K=K, group=64, x_dtype=hawq.F16, w_dtype=hawq.S4, x_stride=K, y_stride=N)
    want = torch.empty((M, N), dtype=torch.float16, device="cuda")
    hawq.hawq_linear_w4(d, x0, w, s, None, None, want)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        x = torch.zeros((M, K), dtype=torch.float16, device="cuda")
        big = torch.randn((4096, 4096), device="cuda")
        for _ in range(4):
            big = big @ big * 1e-3
        x.copy_(x0)                                   # ready only after the work above
        y = torch.empty((M, N), dtype=torch.float16, device="cuda")
        hawq.hawq_linear_w4(d, x, w, s, None, None, y)
    side.synchronize()
    assert torch.equal(y, want)


def test_no_rows():
    import torch
    import paper_2011_10680_amd as hawq
    t = torch.full((64,), 5.0, dtype=torch.float16, device="cuda")
    d = hawq.LinearW4Desc(M=0, N=4, K=32, group=32, x_dtype=hawq.F16, w_dtype=hawq.S4, x_stride=32, y_stride=4)
    hawq.hawq_linear_w4(d, t, t, t, None, None, t)
    torch.cuda.synchronize()
    assert (t == 5).all()


@pytest.mark.parametrize("M,K,group", [(1, 2048, 128), (13, 1000, 64), (70, 352, 32)])
@pytest.mark.parametrize("zeros", [False, True])
def test_values_that_are_not_finite_or_near_the_end_of_the_range(M, K, group, zeros):
    """Each row holds one value besides zeros: an output is that value times one weight, or NaN where an infinity meets a 0."""
    import torch
    import paper_2011_10680_amd as hawq
    N, groups = 100, -(-K // group)
    r = np.random.default_rng(M)
    w = r.integers(0, 256, size=(N, K // 2), dtype=np.uint8)
    s = torch.from_numpy(r.uniform(0.01, 0.1, size=(N, groups)).astype(np.float32)).to(torch.bfloat16)
    z = r.integers(0, 16, size=(N, groups), dtype=np.uint8) if zeros else None
    at = r.integers(0, K, size=M)
    value = np.array([2e37, np.inf, -2e37, np.nan, -np.inf, 1.0, 0.0])[np.arange(M) % 7] if M > 1 else np.array([2e37])
    x = np.zeros((M, K), dtype=np.float32)
    x[np.arange(M), at] = value
    x = torch.from_numpy(x).to(torch.bfloat16)
    y = torch.full((M, N), 7.0, dtype=torch.bfloat16, device="cuda")
    d = hawq.LinearW4Desc(M=M, N=N, K=K, group=group, x_dtype=hawq.BF16, w_dtype=hawq.U4 if zeros else hawq.S4, x_stride=K, y_stride=N)
    hawq.hawq_linear_w4(d, x.cuda(), torch.from_numpy(w).cuda(), s.cuda(), None if z is None else torch.from_numpy(z).cuda(), None, y)
    got = y.cpu().double().numpy()
    weight = ref.unpack(w, z, group)
    xs = x.double().numpy()
    with np.errstate(invalid="ignore"):
        want = np.stack([xs[m, at[m]] * weight[:, at[m]] * s.double().numpy()[:, at[m] // group] for m in range(M)])
    finite = np.isfinite(want)
    assert (np.isnan(got) == np.isnan(want)).all()
    assert (got[np.isinf(want)] == want[np.isinf(want)]).all()
    # products of 8 significant bits by 5 and a scale of 8 are exact in 32 bits, and so is their difference
    assert (np.abs(got[finite] - want[finite]) <= (ref.ROUND["bf16"] + 4 * ref.F32) * np.abs(want)[finite]).all()

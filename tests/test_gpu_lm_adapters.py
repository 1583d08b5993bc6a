"""hawq_adapters on the GPU against the definition in 64 bits."""
import numpy as np
import pytest

import lm_step_reference as ref

pytestmark = pytest.mark.gpu


def _run(M, N, K, n, most, dtype, adapter=None, ranks=None, x_pad=0, y_pad=0, a_pad=0, b_pad=0, x_at=0, a_at=0, b_at=0, in_place=False, size=1.0, garbage=True, seed=0):
    import torch
    import paper_2011_10680_amd as hawq
    dt = {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    r = np.random.default_rng(seed)

    def held(values, shape, pad, at):
        """values [..., cols] as a slice of a wider tensor that holds no numbers elsewhere"""
        whole = torch.full((at + int(np.prod(shape[:-1])) * (shape[-1] + pad) + 64,), float("nan"), dtype=dt, device="cuda")
        t = whole[at:at + int(np.prod(shape[:-1])) * (shape[-1] + pad)].view(*shape[:-1], shape[-1] + pad)[..., :shape[-1]]
        t.copy_(torch.from_numpy(values.astype(np.float32)))
        return t
    ranks = np.asarray(ranks if ranks is not None else r.integers(1, most + 1, size=n), np.int32)
    adapter = np.asarray(adapter if adapter is not None else r.integers(-1, n, size=M), np.int32)
    a, b = r.normal(size=(n, most, K)) * size / K ** 0.5, r.normal(size=(n, N, most))
    if garbage:                                       # what lies past the ranks
        for i in range(n):
            a[i, max(0, ranks[i]):] = np.nan
            b[i, :, max(0, ranks[i]):] = np.inf
    x, a, b, base = held(r.normal(size=(M, K)), (M, K), x_pad, x_at), held(a, (n, most, K), a_pad, a_at), held(b, (n, N, most), b_pad, b_at), held(r.normal(size=(M, N)), (M, N), y_pad, 0)
    want, bound = ref.adapters(x.double().cpu().numpy(), a.double().cpu().numpy(), b.double().cpu().numpy(), ranks, np.arange(n, dtype=np.float32) * np.float32(0.3) + 0.5, adapter,
                               base.double().cpu().numpy(), dtype)
    out = torch.full((M + 1, N + y_pad), 7.0, dtype=dt, device="cuda")
    y = base if in_place else out[:M, :N]
    d = hawq.AdaptersDesc(M=M, N=N, K=K, n_adapters=n, max_rank=most, dtype=hawq.F16 if dtype == "f16" else hawq.BF16, x_stride=K + x_pad, base_stride=N + y_pad, y_stride=N + y_pad,
                          a_adapter=most * (K + a_pad), a_row=K + a_pad, b_adapter=N * (most + b_pad), b_row=most + b_pad)
    room = hawq.hawq_adapters_workspace_bytes(d)
    workspace = torch.full((room + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    hawq.hawq_adapters(d, x, a, b, torch.from_numpy(ranks).cuda(), (torch.arange(n) * np.float32(0.3) + 0.5).float().cuda(), torch.from_numpy(adapter).cuda(), base, y, workspace[:room])
    torch.cuda.synchronize()
    assert bool((workspace[room:] == 0xFF).all())
    if not in_place:
        assert bool((out[:, N:] == 7.0).all()) and bool((out[M] == 7.0).all())
    got = y.double().cpu().numpy()
    off = np.abs(got - want)
    assert (off <= bound).all(), (M, N, K, n, most, float((off - bound).max()), np.argwhere(~(off <= bound))[:3].tolist())


@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 63, 64, 65, 130, 257])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_rows(M, dtype):
    _run(M, 96, 128, 5, 16, dtype, seed=M)
    _run(M, 200, 320, 3, 64, dtype, seed=M + 1)


@pytest.mark.parametrize("most", [1, 2, 5, 8, 16, 17, 31, 32, 33, 64, 100, 128, 200])
def test_ranks(most):
    _run(37, 70, 96, 4, most, "bf16", seed=most)
    _run(5, 130, 260, 4, most, "f16", ranks=[0, most, -3, most + 7], adapter=[0, 1, 2, 3, 1], garbage=False, seed=most)
    _run(140, 48, 64, 2, most, "f16", adapter=[1] * 100 + [-1] * 3 + [0] * 37, seed=most)


@pytest.mark.parametrize("K", [1, 2, 7, 8, 31, 32, 33, 64, 100, 255, 256, 1000, 4096, 8200])
def test_inputs(K):
    _run(20, 33, K, 3, 16, "f16", seed=K)
    _run(3, 64, K, 2, 8, "bf16", seed=K)


@pytest.mark.parametrize("N", [1, 3, 8, 15, 16, 17, 64, 100, 255, 1001, 5000])
def test_outputs(N):
    _run(18, N, 64, 3, 16, "bf16", seed=N)
    _run(2, N, 128, 2, 24, "f16", in_place=True, seed=N)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("pads", [dict(), dict(x_pad=8, y_pad=8, a_pad=8, b_pad=8), dict(x_pad=3), dict(a_pad=1), dict(b_pad=1), dict(y_pad=5), dict(x_at=1), dict(a_at=3), dict(b_at=1),
                                  dict(x_at=8, a_at=8, b_at=8)])
def test_strides_alignment_and_place(pads, in_place):
    _run(33, 72, 160, 4, 16, "bf16", in_place=in_place, seed=3, **pads)
    _run(5, 40, 64, 2, 32, "f16", in_place=in_place, seed=4, **pads)


def test_many_adapters_in_any_order_and_none():
    _run(300, 64, 64, 200, 8, "bf16", seed=1)
    _run(64, 64, 64, 64, 4, "f16", adapter=list(range(63, -1, -1)), seed=2)
    _run(70, 40, 64, 3, 8, "bf16", adapter=[-1] * 70)
    _run(50, 40, 64, 3, 8, "bf16", adapter=[3, -2, 1 << 30, -(1 << 31), 2] * 10)
    _run(1000, 32, 64, 2, 16, "bf16", adapter=[(i // 3) % 3 - 1 for i in range(1000)])


@pytest.mark.parametrize("M,N,K,most", [(512, 300, 64, 64), (577, 33, 200, 8), (640, 1000, 72, 136), (1030, 64, 1000, 20), (4096, 300, 64, 64), (4097, 33, 200, 8), (4160, 100, 72, 136),
                                        (4300, 64, 1000, 20)])
def test_whole_prompts(M, N, K, most):
    """Requests' rows one behind the other, and in between one in no order."""
    for i, dtype in enumerate(("f16", "bf16")):
        runs = [(j * 7 // M) % 4 - 1 for j in range(M)]
        runs[200:260] = [(j * 5) % 4 - 1 for j in range(60)]
        _run(M, N, K, 3, most, dtype, adapter=runs, in_place=i == 1, x_pad=8 * i, seed=M)


def test_no_adapters_at_all():
    import torch
    import paper_2011_10680_amd as hawq
    base = torch.randn((5, 33), device="cuda").half()
    y = torch.zeros_like(base)
    d = hawq.AdaptersDesc(M=5, N=33, K=8, n_adapters=0, max_rank=4, dtype=hawq.F16, x_stride=8, base_stride=33, y_stride=33, a_adapter=0, a_row=8, b_adapter=0, b_row=4)
    ws = torch.empty(hawq.hawq_adapters_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    hawq.hawq_adapters(d, torch.zeros((5, 8), dtype=torch.float16, device="cuda"), None, None, None, None, torch.zeros(5, dtype=torch.int32, device="cuda"), base, y, ws)
    torch.cuda.synchronize()
    assert torch.equal(y, base)


def test_inner_sums_beyond_the_type():
    """h of 10^6 (above f16's range) with a small b, and of 10^-9 with a large one: neither is lost on the way."""
    import torch
    import paper_2011_10680_amd as hawq
    for dtype, dt in (("f16", torch.float16), ("bf16", torch.bfloat16)):
        for xs, bs in ((300.0, 2.0 ** -14), (2.0 ** -14, 300.0)):
            M, N, K, R = 18, 50, 256, 16
            g = torch.Generator().manual_seed(1)
            x, a = torch.randn((M, K), generator=g).mul(xs).to(dt), torch.randn((1, R, K), generator=g).mul(xs).to(dt)
            b, base = torch.randn((1, N, R), generator=g).mul(bs).to(dt), torch.zeros((M, N), dtype=dt)
            y = torch.empty((M, N), dtype=dt, device="cuda")
            d = hawq.AdaptersDesc(M=M, N=N, K=K, n_adapters=1, max_rank=R, dtype=hawq.F16 if dtype == "f16" else hawq.BF16, x_stride=K, base_stride=N, y_stride=N, a_adapter=R * K, a_row=K,
                                  b_adapter=N * R, b_row=R)
            ws = torch.empty(hawq.hawq_adapters_workspace_bytes(d), dtype=torch.uint8, device="cuda")
            hawq.hawq_adapters(d, x.cuda(), a.cuda(), b.cuda(), torch.tensor([R], dtype=torch.int32, device="cuda"), torch.ones(1, device="cuda"), torch.zeros(M, dtype=torch.int32, device="cuda"),
                               base.cuda(), y, ws)
            want, bound = ref.adapters(x.double().numpy(), a.double().numpy(), b.double().numpy(), [R], np.ones(1), np.zeros(M, int), base.double().numpy(), dtype)
            assert (np.abs(y.double().cpu().numpy() - want) <= bound).all(), (dtype, xs)


def test_values_that_are_not_numbers_stay_in_their_row():
    import torch
    import paper_2011_10680_amd as hawq
    M, N, K, R = 40, 33, 64, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    x, a, b = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((M, K), (2, R, K), (2, N, R)))
    base = torch.randn((M, N), generator=g, device="cuda").bfloat16()
    x[3, 5], x[20, 1], x[21, 2] = float("inf"), float("nan"), float("nan")
    adapter = torch.tensor([i % 2 for i in range(M)], dtype=torch.int32, device="cuda")
    adapter[21] = -1
    y = torch.empty_like(base)
    d = hawq.AdaptersDesc(M=M, N=N, K=K, n_adapters=2, max_rank=R, dtype=hawq.BF16, x_stride=K, base_stride=N, y_stride=N, a_adapter=R * K, a_row=K, b_adapter=N * R, b_row=R)
    ws = torch.empty(hawq.hawq_adapters_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    hawq.hawq_adapters(d, x, a, b, torch.tensor([R, R], dtype=torch.int32, device="cuda"), torch.ones(2, device="cuda"), adapter, base, y, ws)
    torch.cuda.synchronize()
    fine = torch.isfinite(y).all(dim=1)
    assert [i for i in range(M) if not fine[i]] == [3, 20] and torch.equal(y[21], base[21])
    assert not bool(torch.isfinite(y[20]).any())


def test_repeated_calls_give_the_same_bits():
    import torch
    import paper_2011_10680_amd as hawq
    M, N, K, R = 48, 512, 2048, 16
    g = torch.Generator(device="cuda").manual_seed(1)
    x, a, b, base = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((M, K), (4, R, K), (4, N, R), (M, N)))
    adapter = torch.randint(-1, 4, (M,), generator=g, device="cuda").int()
    ranks, scales = torch.full((4,), R, dtype=torch.int32, device="cuda"), torch.ones(4, device="cuda")
    d = hawq.AdaptersDesc(M=M, N=N, K=K, n_adapters=4, max_rank=R, dtype=hawq.BF16, x_stride=K, base_stride=N, y_stride=N, a_adapter=R * K, a_row=K, b_adapter=N * R, b_row=R)
    ys = []
    for fill in (0, 0xFF, 0x33):
        ws = torch.full((hawq.hawq_adapters_workspace_bytes(d),), fill, dtype=torch.uint8, device="cuda")
        y = torch.empty_like(base)
        hawq.hawq_adapters(d, x, a, b, ranks, scales, adapter, base, y, ws)
        ys.append(y)
    torch.cuda.synchronize()
    assert torch.equal(ys[0], ys[1]) and torch.equal(ys[0], ys[2])

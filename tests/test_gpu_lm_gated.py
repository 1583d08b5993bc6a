"""hawq_gated_w4 on the GPU against the definition in 64 bits."""
import numpy as np
import pytest

import lm_step_reference as ref

pytestmark = pytest.mark.gpu


def _run(M, N, K, group, dtype, zeros, bias, kind="silu", x_pad=0, y_pad=0, w_at=0, x_at=0, mean=0.0, prompt=None, seed=0):
    import torch
    import paper_2011_10680_amd as hawq
    dt = {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    r = np.random.default_rng(seed)
    groups = -(-K // group)
    rounded = lambda a: torch.from_numpy(a.astype(np.float32)).to(dt)  # noqa: E731
    x = rounded(r.normal(size=(M, K)) + mean)
    w = r.integers(0, 256, size=(2 * N, K // 2), dtype=np.uint8)
    s = rounded(r.uniform(0.1, 0.5, size=(2 * N, groups)) / K ** 0.5 * np.where(r.random((2 * N, groups)) < 0.1, -1, 1))
    z = r.integers(0, 16, size=(2 * N, groups), dtype=np.uint8) if zeros else None
    b = rounded(r.normal(size=2 * N)) if bias else None
    # operands with padding around them that must not be read into the result nor written over
    xw = torch.full((M * (K + x_pad) + x_at + 64,), float("nan"), dtype=dt, device="cuda")
    xd = xw[x_at:x_at + M * (K + x_pad)].view(M, K + x_pad)[:, :K]
    xd.copy_(x)
    ww = torch.full((w_at + w.size + 64,), 0x77, dtype=torch.uint8, device="cuda")
    wd = ww[w_at:w_at + w.size]
    wd.copy_(torch.from_numpy(w).reshape(-1))
    y = torch.full((M + 1, N + y_pad), 7.0, dtype=dt, device="cuda")
    d = hawq.GatedW4Desc(M=M, N=N, K=K, group=group, x_dtype=hawq.F16 if dtype == "f16" else hawq.BF16, w_dtype=hawq.U4 if zeros else hawq.S4,
                         activation={"silu": hawq.SILU, "gelu": hawq.GELU, "gelu_tanh": hawq.GELU_TANH, "relu": hawq.RELU}[kind], x_stride=K + x_pad, y_stride=N + y_pad)
    room = hawq.hawq_gated_w4_workspace_bytes(d)
    assert prompt is None or (room > 0) == prompt          # the kernel for whole prompts has a workspace
    workspace = torch.full((room + 256,), 0xFF, dtype=torch.uint8, device="cuda")      # (not-a-number in 32 bits)
    hawq.hawq_gated_w4(d, xd, wd, s.cuda(), None if z is None else torch.from_numpy(z).cuda(), None if b is None else b.cuda(), y, workspace[:room] if room else None)
    torch.cuda.synchronize()
    assert bool((workspace[room:] == 0xFF).all())
    got = y.double().cpu().numpy()
    assert (got[:, N:] == 7.0).all() and (got[M] == 7.0).all()
    want, bound = ref.gated(x.double().numpy(), w, s.double().numpy(), z, None if b is None else b.double().numpy(), group, kind, dtype)
    off = np.abs(got[:M, :N] - want)
    assert (off <= bound).all(), (M, N, K, float((off / bound).max()))
    # together far less than the bound of each: the type's rounding and a thousandth
    assert np.linalg.norm(off) <= (ref.ROUND[dtype] + 1e-3) * np.linalg.norm(want)


@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 33, 64, 65, 127, 128, 129, 200, 257])
@pytest.mark.parametrize("N,K,group,dtype,zeros", [(100, 256, 128, "bf16", True), (33, 1024, 32, "f16", False), (300, 512, 64, "bf16", False), (130, 384, 128, "f16", True)])
def test_rows(M, N, K, group, dtype, zeros):
    _run(M, N, K, group, dtype, zeros, M % 2 == 0, seed=M)


@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("M", [3, 150])
def test_activations(kind, M):
    for dtype in ("f16", "bf16"):
        _run(M, 90, 256, 64, dtype, True, True, kind, seed=1)
        _run(M, 40, 128, 32, dtype, False, False, kind, mean=3.0, seed=2)


@pytest.mark.parametrize("K", [2, 30, 32, 34, 64, 72, 96, 128, 160, 250, 1000, 1056])
@pytest.mark.parametrize("group", [32, 64, 96, 128, 8224])
def test_reductions(K, group):
    for i, (dtype, zeros) in enumerate((("f16", True), ("bf16", True), ("f16", False), ("bf16", False))):
        _run((3, 140, 18, 300)[i], 49, K, group, dtype, zeros, i % 2 == 1, seed=K + i)


@pytest.mark.parametrize("N", [1, 5, 16, 63, 64, 65, 129, 4097])
def test_outputs(N):
    _run(1, N, 384, 128, "f16", False, True, seed=N)
    _run(20, N, 96, 32, "bf16", True, False, y_pad=3, seed=N)
    _run(150, N, 128, 64, "bf16", True, False, y_pad=3, seed=N)


@pytest.mark.parametrize("x_pad,x_at,w_at", [(8, 0, 0), (5, 0, 0), (0, 1, 0), (3, 3, 1), (0, 0, 4), (0, 0, 2), (0, 8, 16)])
def test_strides_and_alignment(x_pad, x_at, w_at):
    for M in (5, 140):
        _run(M, 70, 320, 64, "f16", True, True, x_pad=x_pad, x_at=x_at, w_at=w_at)
        _run(M, 70, 328, 64, "bf16", False, True, x_pad=x_pad, x_at=x_at, w_at=w_at)


@pytest.mark.parametrize("M,N,K,group", [(400, 5000, 32, 32), (257, 5001, 64, 64), (200, 9000, 96, 32), (200, 5000, 128, 128), (400, 5000, 288, 96), (400, 3000, 352, 64), (1040, 2113, 160, 8224),
                                         (300, 3000, 512, 128), (529, 3001, 1056, 96), (800, 2000, 1120, 32), (257, 5000, 4160, 32), (257, 5000, 8320, 64), (257, 5100, 1024, 256)])
def test_whole_prompts(M, N, K, group):
    """Tiles that end inside, steps that end inside, more groups than are in LDS at once, rows past the last whole tile (1, 16, 17 of them)."""
    for i, dtype in enumerate(("bf16", "f16")):
        _run(M + 15 * i, N, K, group, dtype, i == 0, i == 1, x_pad=8 * i, y_pad=3 * i, w_at=16 * i, prompt=True, seed=K)


@pytest.mark.parametrize("kind", ["gelu", "gelu_tanh", "relu"])
def test_whole_prompts_activations(kind):
    _run(300, 3000, 512, 128, "f16", False, True, kind, prompt=True, seed=5)


@pytest.mark.parametrize("M,N,K", [(3, 40, 20000), (20, 6200, 4160), (300, 500, 4160)])
def test_many_groups(M, N, K):
    _run(M, N, K, 32, "bf16", True, False, seed=K)


@pytest.mark.parametrize("M,N,K", [(2, 40, 256), (140, 40, 256), (300, 5000, 512)])
def test_infinities_and_no_numbers(M, N, K):
    """An infinite input shows in its own row alone: as the formula has it, an infinity or no number."""
    import torch
    import paper_2011_10680_amd as hawq
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((M, K), generator=g, device="cuda").half()
    x[1, 5], x[M - 1, 7] = float("inf"), float("nan")
    w = torch.randint(0, 256, (2 * N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    s = torch.full((2 * N, K // 64), 0.01, dtype=torch.float16, device="cuda")
    y = torch.empty((M, N), dtype=torch.float16, device="cuda")
    d = hawq.GatedW4Desc(M=M, N=N, K=K, group=64, x_dtype=hawq.F16, w_dtype=hawq.S4, activation=hawq.SILU, x_stride=K, y_stride=N)
    ws = torch.empty(max(16, hawq.hawq_gated_w4_workspace_bytes(d)), dtype=torch.uint8, device="cuda")
    hawq.hawq_gated_w4(d, x, w, s, None, None, y, ws)
    q = torch.stack((w & 15, w >> 4), dim=2).reshape(2 * N, K).cpu().double()
    both = x.cpu().double() @ (torch.where(q >= 8, q - 16, q) * float(s[0, 0])).t()
    want = (both[:, :N] / (1 + torch.exp(-both[:, :N])) * both[:, N:]).numpy()
    got = y.double().cpu().numpy()
    fine = np.isfinite(want)
    assert fine[0].all() and not fine[1].any() and np.isnan(got[M - 1]).all()
    assert (np.isfinite(got) == fine).all() and (np.isnan(got) == np.isnan(want)).all()
    assert (got[~fine & ~np.isnan(want)] == want[~fine & ~np.isnan(want)]).all()


@pytest.mark.parametrize("M,N", [(1, 48), (200, 48), (300, 9000)])
def test_one_row_for_all(M, N):
    """x_stride 0: every row of y is the same."""
    import torch
    import paper_2011_10680_amd as hawq
    K = 128
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((1, K), generator=g, device="cuda").bfloat16()
    w = torch.randint(0, 256, (2 * N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    s = torch.rand((2 * N, 1), generator=g, device="cuda").bfloat16()
    out = []
    for rows in (M, 1):
        y = torch.empty((rows, N), dtype=torch.bfloat16, device="cuda")
        d = hawq.GatedW4Desc(M=rows, N=N, K=K, group=128, x_dtype=hawq.BF16, w_dtype=hawq.S4, activation=hawq.RELU, x_stride=0, y_stride=N)
        ws = torch.empty(max(16, hawq.hawq_gated_w4_workspace_bytes(d)), dtype=torch.uint8, device="cuda")
        hawq.hawq_gated_w4(d, x, w, s, None, None, y, ws)
        out.append(y.float())
    torch.cuda.synchronize()
    # the two may sum in another order: half a step of the type apart, and a thousandth of 1
    assert bool((out[0] == out[0][:1]).all()) and float((out[0][0] - out[1][0]).abs().max()) <= 2.0 ** -7 * float(out[1].abs().max()) + 1e-3

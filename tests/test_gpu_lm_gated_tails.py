"""hawq_gated_w4 on the GPU where the gate's activation is next to nothing and the second projection large: the product is still a number of the type."""
import numpy as np
import pytest

import lm_step_reference as ref

pytestmark = pytest.mark.gpu

# gates from 0 to where activations pass the smallest normal number of 32 bits (2^-126) and the smallest of all (2^-149), all of them numbers of bf16
GATES = {"silu": np.arange(-112, 0, 0.5), "gelu": np.arange(-16, 0, 0.0625), "gelu_tanh": np.arange(-12, 0, 0.0625)}


@pytest.mark.parametrize("kind", sorted(GATES))
@pytest.mark.parametrize("M,N,K,group", [(1, 600, 64, 32), (30, 600, 128, 128), (70, 1000, 68, 64), (300, 3000, 512, 128)])
def test_tails(kind, M, N, K, group):
    """Rows of zeros: both projections are their biases."""
    import torch
    import paper_2011_10680_amd as hawq
    r = np.random.default_rng(1)
    gates = np.concatenate((GATES[kind], -GATES[kind]))
    g, u = np.resize(gates, N), np.resize(2.0 ** np.arange(60, 110, 7), N) * r.choice([-1, 1], size=N)
    bias = torch.from_numpy(np.concatenate((g, u))).bfloat16()
    assert (bias.double().numpy() == np.concatenate((g, u))).all()
    d = hawq.GatedW4Desc(M=M, N=N, K=K, group=group, x_dtype=hawq.BF16, w_dtype=hawq.S4, activation={"silu": hawq.SILU, "gelu": hawq.GELU, "gelu_tanh": hawq.GELU_TANH}[kind],
                         x_stride=K, y_stride=N)
    room = hawq.hawq_gated_w4_workspace_bytes(d)
    assert (room > 0) == (M == 300)                    # the kernel for whole prompts has a workspace
    w = torch.from_numpy(r.integers(0, 256, size=(2 * N, K // 2), dtype=np.uint8)).cuda()
    scales = torch.ones((2 * N, -(-K // group)), dtype=torch.bfloat16, device="cuda")
    y = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    hawq.hawq_gated_w4(d, torch.zeros((M, K), dtype=torch.bfloat16, device="cuda"), w, scales, None, bias.cuda(), y, torch.empty(max(room, 16), dtype=torch.uint8, device="cuda"))
    got = y.double().cpu().numpy()
    a, units = ref.activation(g, kind)
    want, half = a * u, ref.ROUND["bf16"]
    # The activation is off by its 32-bit roundings, and below 2^-126 by half a step of 2^-149 (of gelu by one, times half the gate: 8 at most)
    off = (ref.F32 * units * np.abs(a) + (8 * 2.0 ** -149 if kind == "gelu" else 2.0 ** -150)) * np.abs(u)
    bound = half * np.abs(want) + (1 + half) * (off + ref.F32 * np.abs(want)) + ref.TINY["bf16"]
    bad = np.abs(got - want) > bound
    assert not bad.any(), [(g[n], a[n], got[m, n] / u[n]) for m, n in np.argwhere(bad)[:4]]


@pytest.mark.parametrize("kind", sorted(GATES))
def test_gates_without_end(kind):
    """The largest numbers and infinities: 0 or the gate itself, and no number where the formula multiplies an infinity by 0."""
    import torch
    import paper_2011_10680_amd as hawq
    inf = float("inf")
    g = [-200.0, -1e4, -1e20, -3e38, 200.0, 1e20, 3e38, inf, -inf, float("nan"), -0.0, 0.0]
    N, K = len(g), 32
    bias = torch.tensor(g + [1.0] * N).bfloat16()
    y = torch.empty((1, N), dtype=torch.bfloat16, device="cuda")
    d = hawq.GatedW4Desc(M=1, N=N, K=K, group=32, x_dtype=hawq.BF16, w_dtype=hawq.S4, activation={"silu": hawq.SILU, "gelu": hawq.GELU, "gelu_tanh": hawq.GELU_TANH}[kind], x_stride=K,
                         y_stride=N)
    hawq.hawq_gated_w4(d, torch.zeros((1, K), dtype=torch.bfloat16, device="cuda"), torch.zeros((2 * N, K // 2), dtype=torch.uint8, device="cuda"),
                       torch.ones((2 * N, 1), dtype=torch.bfloat16, device="cuda"), None, bias.cuda(), y)
    got = y[0].double().cpu().tolist()
    assert got[:4] == [0.0] * 4 and got[4:8] == bias.double().tolist()[4:8] and got[10:] == [0.0, 0.0]
    assert all(v != v for v in got[8:10])

"""hawq_gated_w4 on the GPU: how near its 32-bit sums come to those in 64 bits, for inputs with a mean, whose zero points' part is far larger than what
is left of it.  A bias takes all but the last bits of a sum away, so that the rounding of the result does not hide them."""
import numpy as np
import pytest

import lm_reference as lm

pytestmark = pytest.mark.gpu


def errors(M, N, K, group, zeros, mean, seed=0):
    """(how far the sums of the gate are off, what a rounding of them is measured by, their size)"""
    import torch
    import paper_2011_10680_amd as hawq
    g = torch.Generator(device="cuda").manual_seed(seed)
    groups = -(-K // group)
    x = (torch.randn((1, K), generator=g, device="cuda") + mean).half()
    w = torch.randint(0, 256, (2 * N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    s = ((0.1 + 0.4 * torch.rand((2 * N, groups), generator=g, device="cuda")) / (8 * K ** 0.5)).half()
    s[N:] = 0                                          # the second projection is its bias, 1
    z = torch.randint(4, 12, (2 * N, groups), generator=g, device="cuda", dtype=torch.uint8) if zeros else None
    total, size = torch.zeros(N, dtype=torch.float64, device="cuda"), torch.zeros(N, dtype=torch.float64, device="cuda")
    for i in range(groups):
        k = slice(i * group, min(K, (i + 1) * group))
        codes = w[:N, k.start // 2:k.stop // 2]
        q = torch.stack((codes & 15, codes >> 4), dim=2).reshape(N, -1).double()
        q = torch.where(q >= 8, q - 16, q) if z is None else q - z[:N, i:i + 1]
        total += (q * x[:, k].double()).sum(dim=1) * s[:N, i].double()
        size += x[0, k].double().abs().sum() * s[:N, i].double()
    nearest = total.half()
    below = torch.where(nearest.double() >= total, torch.nextafter(nearest, torch.full_like(nearest, -torch.inf)), nearest)
    bias = torch.cat((-below, torch.ones_like(below)))
    y = torch.empty((M, N), dtype=torch.float16, device="cuda")
    d = hawq.GatedW4Desc(M=M, N=N, K=K, group=group, x_dtype=hawq.F16, w_dtype=hawq.U4 if zeros else hawq.S4, activation=hawq.RELU, x_stride=0, y_stride=N)
    room = hawq.hawq_gated_w4_workspace_bytes(d)
    assert (room > 0) == (M > 200)                     # the kernel for whole prompts has a workspace
    hawq.hawq_gated_w4(d, x, w, s, z, bias, y, torch.empty(max(room, 16), dtype=torch.uint8, device="cuda"))
    left = total - below.double()
    off = (y.double() - left).abs() - lm.ROUND["f16"] * left - 2.0 ** -25
    return off.clamp(min=0).cpu().numpy(), size.cpu().numpy(), float(total.abs().mean())


@pytest.mark.parametrize("M", [1, 20, 640])
@pytest.mark.parametrize("K,group", [(512, 128), (4096, 128), (4096, 32), (8192, 64), (65536, 128), (65536, 32)])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("mean", [0.0, 3.0, 30.0])
def test_sums(M, K, group, zeros, mean):
    """A running sum is 31 |x| |s| at most (weights 16 to 31, and as much that is taken off).  It is rounded to 2^-24 of that, not in one direction, less than
    three times for each group and some more where waves' parts are added up, the sums of x and the bias: six times the root of that number is not reached by
    tens of thousands of outputs."""
    off, size, _ = errors(M, 3000, K, group, zeros, mean)
    assert (off <= 6 * (3 * (K // group) + 64) ** 0.5 * lm.F32 * 31 * size).all(), float((off / size).max() / lm.F32)

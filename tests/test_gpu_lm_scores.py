"""Attention on the GPU where scores are so large that a 32-bit float no longer tells neighbours apart: the largest ones share the weight."""
import numpy as np
import pytest

import lm_reference as ref
import test_gpu_lm_attention as base

pytestmark = pytest.mark.gpu

# Only one element of queries and keys is not 0: scores are 256 * k * 2^j, exact in 32 bits, and neighbours lie 64 * 2^j apart or are equal,
# so that weights are 1 over the number of equals or (from j = 0 on) less than e^-63.
_J = [0, 6, 10, 14, 16, 18, 20, 24, 30]


def _keys(r, n, sign):
    k = np.floor(r.uniform(100, 200, size=n) * 4) / 4
    k[r.random(n) < 0.3] = 210.25 if sign > 0 else 90.5                            # (many share the largest score)
    return sign * k


def _check(got, scores, v, seen, u):
    s = np.where(seen, scores[None], -np.inf)
    p = np.exp(s - s.max(axis=1, keepdims=True))
    p /= p.sum(axis=1, keepdims=True)
    want, size = p @ v, p @ np.abs(v)
    assert (np.abs(got - want) <= u * np.abs(want) + (1.01 * u + 2 * ref.F32 * (scores.size + 64)) * size + 2.0 ** -25).all(), (got[-1, :4], want[-1, :4])


@pytest.mark.parametrize("j", _J)
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("D", [64, 128, 20])
def test_prompts(j, sign, D):
    import torch
    import paper_2011_10680_amd as hawq
    n = 300
    for dtype in ("f16", "bf16"):
        dt, ht = base._types(dtype)
        r = np.random.default_rng(j)
        q, k = torch.zeros((2, n, 1, D), dtype=dt, device="cuda")
        q[:, 0, 0] = 256
        k[:, 0, 0] = torch.from_numpy(_keys(r, n, sign)).to(dt).cuda()
        v = torch.randn((n, 1, D), device="cuda").to(dt)
        y = torch.full_like(v, 7.0)
        d = hawq.AttnPromptDesc(n_seqs=1, total=n, q_heads=1, kv_heads=1, head_dim=D, dtype=ht, scale=2.0 ** j, **base._rows(q=q, k=k, v=v, y=y))
        hawq.hawq_attn_prompt(d, q, k, v, torch.tensor([0, n], dtype=torch.int32, device="cuda"), y)
        _check(base._f64(y)[:, 0], 256 * base._f64(k)[:, 0, 0] * 2.0 ** j, base._f64(v)[:, 0], np.tril(np.ones((n, n), bool)), ref.ROUND[dtype])

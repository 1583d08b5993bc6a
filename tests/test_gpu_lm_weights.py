"""Softmax weights in attention on the GPU where many small ones stand beside a large one."""
import math

import numpy as np
import pytest

import lm_reference as ref
import test_gpu_lm_attention as base

pytestmark = pytest.mark.gpu

# Weights are held in 16 bits before they meet the values, so many small ones count only as far as a half reaches: with weights up to 2^15
# the largest is at least 2^7, and each is off by no more than 2^-32 of it (half the step of the smallest halves) or by a half's rounding.
# Sums are of 32 bits, 16 keys at a time (the matrix instruction's, or the lanes' own).

def _sums(keys):
    return 2.0 ** -18 + 2 * ref.F32 * (keys / 16 + 64)


@pytest.mark.parametrize("gap", [12.0, 17.5, 18.0])
@pytest.mark.parametrize("D", [8, 128])
@pytest.mark.parametrize("others", [1, 0])
def test_prompt_many_small_weights_add_up(gap, D, others):
    """One key far above many: what the many add together (their values 1, the one's 0), and what they take from the one (0 and 1)."""
    import torch
    import paper_2011_10680_amd as hawq
    n, u = 40000, ref.ROUND["f16"]
    q, k = torch.zeros((2, n, 1, D), dtype=torch.float16, device="cuda")
    q[:, :, 0] = 1.0
    k[0, :, 0] = gap
    i = np.arange(n)
    many = i * math.exp(-gap)
    v = torch.full_like(k, others)
    v[0] = 1 - others
    y = torch.empty_like(q)
    d = hawq.AttnPromptDesc(n_seqs=1, total=n, q_heads=1, kv_heads=1, head_dim=D, dtype=hawq.F16, scale=1.0, **base._rows(q=q, k=k, v=v, y=y))
    hawq.hawq_attn_prompt(d, q, k, v, torch.tensor([0, n], dtype=torch.int32, device="cuda"), y)
    got = base._f64(y)[:, 0]
    want = (1 - others + others * many) / (1 + many)
    bound = others * 2.0 ** -32 * i + ((1 + others) * u + _sums(i)) * want + 2.0 ** -25
    assert (np.abs(got - want[:, None]) <= bound[:, None]).all(), (got[-1, 0], want[-1], bound[-1])


@pytest.mark.parametrize("cache", ["same", "s8"])
@pytest.mark.parametrize("gap", [12.0, 17.5])
@pytest.mark.parametrize("drafts", [1, 20])
@pytest.mark.parametrize("others", [1, 0])
def test_cached_many_small_weights_add_up(cache, gap, drafts, others):
    """The same over a cache, with so many requests and heads that each is left to a single workgroup: its waves take 32 keys in turn, and the
    first 32 of every wave hold one of the four keys above the rest.  Drafts see the cache alone."""
    import torch
    import paper_2011_10680_amd as hawq
    n, H, B, D, page, u = 20000, 64, 72, 64, 16, ref.ROUND["f16"]
    n_pages, s8 = n // page, cache == "s8"
    q = torch.zeros((B * drafts, H, D), dtype=torch.float16, device="cuda")
    q[:, :, 0] = 1.0
    k = torch.zeros_like(q)
    shape = (n_pages, page, H, D)
    kc, vc = torch.zeros((2,) + shape, dtype=torch.int8 if s8 else torch.float16, device="cuda")
    ks, vs = (torch.full(shape[:3], f, device="cuda") if s8 else None for f in (gap / 64, 2.0 ** -7))       # codes of 64: gap and 1/2
    half = 64 if s8 else 0.5
    for j in (0, 32, 64, 96):
        kc[j // page, j % page, :, 0] = 64 if s8 else gap
    cd = hawq.CacheDesc(n_pages=n_pages, page=page, kv_heads=H, head_dim=D, dtype=hawq.S8 if s8 else hawq.F16, page_stride=kc.stride(0), token_stride=kc.stride(1),
                        head_stride=kc.stride(2))
    y = torch.empty_like(q)
    d = hawq.AttnTreeDesc(cache=cd, n_seqs=B, total=B * drafts, max_drafts=drafts, max_cached=n, q_heads=H, dtype=hawq.F16, table_stride=n_pages, scale=1.0,
                          **base._rows(q=q, k=k, v=k, y=y))
    ws = torch.empty(max(16, hawq.hawq_attn_tree_workspace_bytes(d)), dtype=torch.uint8, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    table, starts, lens = torch.arange(n_pages, **i32).expand(B, n_pages).contiguous(), torch.arange(0, B * drafts + 1, drafts, **i32), torch.full((B,), n, **i32)
    mask = torch.zeros(B * drafts, dtype=torch.int64, device="cuda")
    many = (n - 4) * math.exp(-gap)
    vc.fill_(half * others)
    for j in (0, 32, 64, 96):
        vc[j // page, j % page] = half * (1 - others)
    hawq.hawq_attn_tree(d, q, k, k, starts, mask, kc, vc, ks, vs, table, lens, y, ws)
    got, want = base._f64(y), 0.5 * (4 * (1 - others) + others * many) / (4 + many)
    bound = others * 2.0 ** -32 * 0.5 * n / 4 + ((1 + others) * u + _sums(n / 4)) * want + 2.0 ** -25
    assert (np.abs(got - want) <= bound).all(), (got.min(), got.max(), want, bound)

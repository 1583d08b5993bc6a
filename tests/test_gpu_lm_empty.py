"""hawq_attn_tree on the GPU where no request can hold a cached token."""
import numpy as np
import pytest

import lm_reference as ref
import test_gpu_lm_attention as base
from test_gpu_lm_edges import _strict

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 20])
@pytest.mark.parametrize("n_pages,width,bound", [(0, 0, 0), (0, 5, 100), (3, 0, 100), (3, 5, 0)])
def test_no_cache_no_table_or_no_bound(D, n_pages, width, bound):
    """Empty tensors have no address: drafts then see one another, whatever the lengths say."""
    import torch
    import paper_2011_10680_amd as hawq
    H, KV, page, drafts = 4, 2, 16, [3, 40]
    total = sum(drafts)
    g = torch.Generator(device="cuda").manual_seed(D)
    q, k, v = (torch.randn((total, h, D), generator=g, device="cuda").half() for h in (H, KV, KV))
    y = torch.full_like(q, 7.0)
    kc = torch.full((n_pages, page, KV, D), float("nan"), dtype=torch.float16, device="cuda")
    table = torch.zeros((2, width), dtype=torch.int32, device="cuda")
    cd = hawq.CacheDesc(n_pages=n_pages, page=page, kv_heads=KV, head_dim=D, dtype=hawq.F16, page_stride=page * KV * D, token_stride=KV * D, head_stride=D)
    d = hawq.AttnTreeDesc(cache=cd, n_seqs=2, total=total, max_drafts=40, max_cached=bound, q_heads=H, dtype=hawq.F16, table_stride=width, scale=0.2,
                          **base._rows(q=q, k=k, v=v, y=y))
    assert hawq.hawq_attn_tree_workspace_bytes(d) == 0
    i32 = dict(dtype=torch.int32, device="cuda")
    hawq.hawq_attn_tree(d, q, k, v, torch.tensor([0, 3, 43], **i32), None, kc, kc, None, None, table, torch.tensor([50, 7], **i32), y, None)
    torch.cuda.synchronize()
    got, qn, kn, vn = (base._f64(t) for t in (y, q, k, v))
    for f, e in ((0, 3), (3, 43)):
        for h in range(H):
            want, size, top = ref.attend(qn[f:e, h], kn[f:e, h // 2], vn[f:e, h // 2], np.tril(np.ones((e - f, e - f), bool)), float(np.float32(0.2)))
            _strict(got[f:e, h], want, size, top, e - f, D, "f16", (f, h))

"""The language-model operators on the GPU with more rows than one launch along x holds (2^32 threads)."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,cache", [(8, "same"), (8, "s8"), (7, "same"), (7, "s8")])
def test_store_of_very_many_rows(D, cache):
    """Rows of 8 elements go in whole vectors, of 7 a wave each; their number (70 million) passes what either had in one launch."""
    import torch
    import paper_2011_10680_amd as hawq
    total, heads, page, s8 = 8750000, 8, 32, cache == "s8"
    g = torch.Generator(device="cuda").manual_seed(D)
    x = torch.randint(-127, 128, (total, heads, D), generator=g, device="cuda", dtype=torch.int8)
    x[:, :, 0] = 127                                                              # (an 8-bit row's scale is 127 * (1 / 127): its codes are its elements)
    k = x.half()
    n_pages = -(-total // page)
    kc, vc = torch.full((2, n_pages, page, heads, D), 5, dtype=torch.int8 if s8 else torch.float16, device="cuda")
    ks, vs = torch.full((2, n_pages, page, heads), 9.0, device="cuda") if s8 else (None, None)
    slots = torch.arange(total - 1, -1, -1, device="cuda")
    slots[::1000] = -1
    cd = hawq.CacheDesc(n_pages=n_pages, page=page, kv_heads=heads, head_dim=D, dtype=hawq.S8 if s8 else hawq.F16, page_stride=kc.stride(0), token_stride=kc.stride(1),
                        head_stride=kc.stride(2))
    d = hawq.CacheStoreDesc(cache=cd, total=total, dtype=hawq.F16, k_token=k.stride(0), k_head=k.stride(1), v_token=k.stride(0), v_head=k.stride(1))
    hawq.hawq_cache_store(d, k, k, slots, kc, vc, ks, vs)
    torch.cuda.synchronize()
    want = x.flip(0)
    kept = (slots >= 0).flip(0)[:, None, None]
    for c, f in ((kc, ks), (vc, vs)):
        c = c.view(-1, heads, D)
        assert torch.equal(c[:total], torch.where(kept, want, torch.full_like(want, 5)).to(c.dtype)) and bool((c[total:] == 5).all())
        if s8:
            f = f.view(-1, heads)
            one = torch.tensor(127.0, device="cuda") * (torch.tensor(1.0, device="cuda") / 127)
            assert torch.equal(f[:total], torch.where(kept[:, :, 0], one, torch.tensor(9.0, device="cuda")).expand(total, heads)) and bool((f[total:] == 9).all())


@pytest.mark.parametrize("n,heads,D", [(5000, 4096, 8), (135000, 512, 3)])
def test_prompts_of_very_many_rows(n, heads, D):
    """As many prompts of one token as make more than 2^32 threads: each gives its own value back."""
    import torch
    import paper_2011_10680_amd as hawq
    g = torch.Generator(device="cuda").manual_seed(D)
    q = torch.randn((1, 1, D), generator=g, device="cuda").half()
    v = torch.randn((n, heads, D), generator=g, device="cuda").half()
    y = torch.full((n + 1, heads, D), 7.0, dtype=torch.float16, device="cuda")
    starts = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    d = hawq.AttnPromptDesc(n_seqs=n, total=n, q_heads=heads, kv_heads=heads, head_dim=D, dtype=hawq.F16, scale=1.0, q_token=0, q_head=0, k_token=0, k_head=0,
                            v_token=v.stride(0), v_head=v.stride(1), y_token=y.stride(0), y_head=y.stride(1))
    hawq.hawq_attn_prompt(d, q, q, v, starts, y)
    torch.cuda.synchronize()
    assert torch.equal(y[:n], v) and bool((y[n] == 7).all())


@pytest.mark.parametrize("M,N,K", [(2200000, 3, 2), (1100000, 1, 32)])
def test_linear_layers_of_very_many_rows(M, N, K):
    """More than 65535 tiles of rows.  Codes of 1 and small whole numbers: sums of x times a power of two, exact."""
    import torch
    import paper_2011_10680_amd as hawq
    g = torch.Generator(device="cuda").manual_seed(M)
    x = torch.randint(-8, 9, (M, K), generator=g, device="cuda", dtype=torch.int8).half()
    w = torch.full((N, K // 2), 0x11, dtype=torch.uint8, device="cuda")
    scales = (2.0 ** -torch.arange(N, device="cuda")).half()[:, None].contiguous()
    bias = torch.arange(N, device="cuda").half()
    whole = torch.full((M + 1, N), 7.0, dtype=torch.float16, device="cuda")
    d = hawq.LinearW4Desc(M=M, N=N, K=K, group=32, x_dtype=hawq.F16, w_dtype=hawq.S4, x_stride=K, y_stride=N)
    hawq.hawq_linear_w4(d, x, w, scales, None, bias, whole)
    torch.cuda.synchronize()
    want = (x.float().sum(dim=1, keepdim=True) * scales.float().t() + bias.float()).half()
    assert torch.equal(whole[:M], want) and bool((whole[M] == 7).all())


def test_tree_of_very_many_requests_and_heads():
    """65535 requests of 257 heads: more than 2^32 threads of the matrix form.  A token that sees only itself, and a few with a cached one."""
    import torch
    import paper_2011_10680_amd as hawq
    n, heads, D = 65535, 257, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.zeros((1, 1, D), device="cuda").half()
    v = torch.randn((n, heads, D), generator=g, device="cuda").half()
    cache = torch.randn((1, 16, heads, D), generator=g, device="cuda").half()
    cached = torch.zeros(n, dtype=torch.int32, device="cuda")
    cached[-3:] = 1
    y = torch.full((n + 1, heads, D), 7.0, dtype=torch.float16, device="cuda")
    cd = hawq.CacheDesc(n_pages=1, page=16, kv_heads=heads, head_dim=D, dtype=hawq.F16, page_stride=cache.stride(0), token_stride=cache.stride(1), head_stride=cache.stride(2))
    d = hawq.AttnTreeDesc(cache=cd, n_seqs=n, total=n, max_drafts=1, max_cached=1, q_heads=heads, dtype=hawq.F16, table_stride=1, scale=1.0, q_token=0, q_head=0, k_token=0,
                          k_head=0, v_token=v.stride(0), v_head=v.stride(1), y_token=y.stride(0), y_head=y.stride(1))
    assert hawq.hawq_attn_tree_workspace_bytes(d) == 0
    hawq.hawq_attn_tree(d, q, q, v, torch.arange(n + 1, dtype=torch.int32, device="cuda"), None, cache, cache, None, None, torch.zeros((n, 1), dtype=torch.int32, device="cuda"),
                        cached, y, None)
    torch.cuda.synchronize()
    assert torch.equal(y[:n - 3], v[:n - 3]) and bool((y[n] == 7).all())
    want = (v[n - 3:].double() + cache[0, 0].double()) / 2
    # both weights are 1 (scores of 0) and the sum is exact in 32 bits: one rounding to a half
    assert torch.equal(y[n - 3:n], want.float().half())

"""A server's step on the GPU captured once -- plan, linear layer, store, attention over the cache -- and replayed with other inputs."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["f16", "s8"])
def test_replays_equal_eager_calls(cache):
    import torch
    import paper_2011_10680_amd as hawq
    n, H, KV, D, page, width, K = 3, 8, 2, 64, 16, 40, 256
    s8 = cache == "s8"
    g = torch.Generator(device="cuda").manual_seed(1)
    i32 = dict(dtype=torch.int32, device="cuda")
    w = torch.randint(0, 256, ((H + 2 * KV) * D, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    s = (0.01 * torch.rand((w.shape[0], K // 64), generator=g, device="cuda")).half()
    x, lens = torch.zeros((n, K), dtype=torch.float16, device="cuda"), torch.tensor([500, 33, 0], **i32)
    fresh, free = torch.ones(n, **i32), torch.arange(100, 100 + n, **i32)
    pages = torch.arange(3 * 32, **i32)

    def buffers():
        table = torch.full((n, width), -1, **i32)
        table[:, :32] = pages.view(3, 32)
        kv = torch.full((2, 128, page, KV, D), 1, dtype=torch.int8 if s8 else torch.float16, device="cuda")
        f = torch.full((2, 128, page, KV), 0.01, device="cuda") if s8 else (None, None)
        return dict(table=table, starts=torch.empty(n + 1, **i32), slots=torch.empty(n, dtype=torch.int64, device="cuda"), counts=torch.empty(2, **i32), k=kv[0], v=kv[1],
                    ks=f[0], vs=f[1], qkv=torch.empty((n, H + 2 * KV, D), dtype=torch.float16, device="cuda"), y=torch.empty((n, H, D), dtype=torch.float16, device="cuda"))
    eager, held = buffers(), buffers()
    cd = hawq.CacheDesc(n_pages=128, page=page, kv_heads=KV, head_dim=D, dtype=hawq.S8 if s8 else hawq.F16, page_stride=eager["k"].stride(0), token_stride=eager["k"].stride(1),
                        head_stride=eager["k"].stride(2))
    lin = hawq.LinearW4Desc(M=n, N=w.shape[0], K=K, group=64, x_dtype=hawq.F16, w_dtype=hawq.S4, x_stride=K, y_stride=w.shape[0])
    row = (H + 2 * KV) * D
    st = hawq.CacheStoreDesc(cache=cd, total=n, dtype=hawq.F16, k_token=row, k_head=D, v_token=row, v_head=D)
    tr = hawq.AttnTreeDesc(cache=cd, n_seqs=n, total=n, max_drafts=1, max_cached=width * page, q_heads=H, dtype=hawq.F16, table_stride=width, scale=0.1, q_token=row, q_head=D,
                           k_token=row, k_head=D, v_token=row, v_head=D, y_token=H * D, y_head=D)
    ws = torch.empty(max(16, hawq.hawq_attn_tree_workspace_bytes(tr)), dtype=torch.uint8, device="cuda")

    def step(b):
        hawq.hawq_cache_plan(lens, fresh, page, free, b["table"], b["starts"], b["slots"], b["counts"])
        hawq.hawq_linear_w4(lin, x, w, s, None, None, b["qkv"])
        q, k, v = b["qkv"][:, :H], b["qkv"][:, H:H + KV], b["qkv"][:, H + KV:]
        hawq.hawq_attn_tree(tr, q, k, v, b["starts"], None, b["k"], b["v"], b["ks"], b["vs"], b["table"], lens, b["y"], ws)
        hawq.hawq_cache_store(st, k, v, b["slots"], b["k"], b["v"], b["ks"], b["vs"])
    step(eager)
    step(held)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(held)
    for i in range(5):
        x.copy_(torch.randn((n, K), generator=g, device="cuda"))
        lens += 1
        step(eager)
        graph.replay()
        torch.cuda.synchronize()
        for name in eager:
            if eager[name] is not None:
                assert torch.equal(eager[name], held[name]), (i, name)
        assert bool((eager["slots"] >= 0).all()) and bool(torch.isfinite(eager["y"]).all()) and not bool((eager["y"] == 0).all())

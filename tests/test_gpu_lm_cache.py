"""hawq_cache_plan and hawq_cache_store on the GPU: whole numbers and stored values equal those of the plain walk."""
import numpy as np
import pytest

import lm_reference as ref

pytestmark = pytest.mark.gpu


def _plan(cached, fresh, page, width, n_free, n_slots, seed=0):
    import torch
    import paper_2011_10680_amd as hawq
    r = np.random.default_rng(seed)
    cached, fresh = np.array(cached, np.int32), np.array(fresh, np.int32)
    n = len(cached)
    table = r.integers(0, 1000, size=(n, width)).astype(np.int32)
    free = (2000 + r.permutation(n_free)).astype(np.int32)
    want = ref.plan(cached, fresh, page, free, table, n_slots)
    cu = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    t, starts = cu(table), torch.full((n + 1,), 9, dtype=torch.int32, device="cuda")
    slots, counts = torch.full((n_slots,), 9, dtype=torch.int64, device="cuda"), torch.full((2,), 9, dtype=torch.int32, device="cuda")
    for _ in range(2):                                    # a repeated call gives the same
        hawq.hawq_cache_plan(cu(cached), cu(fresh), page, cu(free), t, starts, slots, counts)
        torch.cuda.synchronize()
        for got, exp, what in zip((t, starts, slots, counts), want, ("table", "starts", "slots", "counts")):
            assert np.array_equal(got.cpu().numpy(), exp), (what, page, width, n_free, n_slots)


@pytest.mark.parametrize("n", [0, 1, 2, 63, 64, 65, 255, 256, 257, 700, 3000])
@pytest.mark.parametrize("page", [1, 16, 24])
def test_plan_requests(n, page):
    r = np.random.default_rng(n + page)
    cached, fresh = r.integers(0, 90, size=n), r.integers(0, 40, size=n)
    fresh[::3] = 0
    total = int(fresh.sum())
    _plan(cached, fresh, page, 130 // page + 1, 40 * n + 5, total + 77, seed=n)
    _plan(cached, fresh, page, 130 // page + 1, max(0, total // page // 2), total, seed=n)          # too few free pages


def test_plan_edges():
    _plan([0], [0], 16, 4, 3, 0)
    _plan([0], [1], 16, 4, 0, 5)                          # no free page at all
    _plan([5, 0, 16], [200, 3, 1], 16, 2, 30, 300)        # more tokens than the table's row has room for
    _plan([-4, 7], [3, -9], 16, 3, 30, 20)                # negative numbers count as none
    _plan([100, 1], [5, 5], 16, 3, 30, 20)                # already past the table
    _plan([3, 3], [50, 60], 16, 0, 30, 120)               # a table without room
    _plan([10, 20, 30], [40, 50, 60], 8, 20, 90, 70)      # fewer slots than tokens
    _plan([0, 1], [5000, 9000], 16, 600, 2000, 15000)     # one request over many workgroups
    _plan([2 ** 30, 7], [40, 7], 1 << 20, 3000, 4000, 100)


def _store(total, kv_heads, D, dtype, cache, page, layout="dense", heads_first=False, skip=0.3, change=None, seed=0, spare=0):
    import torch
    import paper_2011_10680_amd as hawq
    dt, ht = (torch.float16, hawq.F16) if dtype == "f16" else (torch.bfloat16, hawq.BF16)
    g = torch.Generator(device="cuda").manual_seed(seed)
    kv = []
    for _ in range(2):
        x = torch.randn((total, kv_heads, D), generator=g, device="cuda").to(dt)
        if layout == "odd":
            w = torch.zeros((total, kv_heads, D + 5), dtype=dt, device="cuda")
            w[:, :, 3:D + 3] = x
            x = w[:, :, 3:D + 3]
        elif layout == "heads":
            x = x.permute(1, 0, 2).contiguous().permute(1, 0, 2)
        kv.append(x)
    if change:
        change(*kv)
    used = total // page + 2
    n_pages = spare + used
    shape = (n_pages, page, kv_heads, D)
    s8 = cache == "s8"
    caches, scales = [], []
    for _ in range(2):
        stored = (n_pages, kv_heads, page, D) if heads_first else shape
        c = torch.full(stored, 7, dtype=torch.int8 if s8 else dt, device="cuda") if not spare else torch.empty(stored, dtype=torch.int8 if s8 else dt, device="cuda")
        c[spare:] = 7
        caches.append(c.permute(0, 2, 1, 3) if heads_first else c)
        scales.append(torch.full(shape[:3], 5.0, device="cuda") if s8 else None)
    r = np.random.default_rng(seed)
    slots = spare * page + r.permutation(used * page)[:total].astype(np.int64)
    gone = r.random(total) < skip
    slots[gone] = r.choice([-1, -7, n_pages * page, 2 ** 40], size=int(gone.sum()))
    cd = hawq.CacheDesc(n_pages=n_pages, page=page, kv_heads=kv_heads, head_dim=D, dtype=hawq.S8 if s8 else ht, page_stride=caches[0].stride(0),
                        token_stride=caches[0].stride(1), head_stride=caches[0].stride(2))
    strides = {"%s_%s" % (n, w): t.stride(i) for n, t in zip("kv", kv) for i, w in enumerate(("token", "head"))}
    hawq.hawq_cache_store(hawq.CacheStoreDesc(cache=cd, total=total, dtype=ht, **strides), kv[0], kv[1], torch.from_numpy(slots).cuda(), *caches, *scales)
    torch.cuda.synchronize()
    at = torch.from_numpy(np.where(gone, 0, slots - spare * page)[~gone])
    for x, c, f in zip(kv, caches, scales):
        got = c[spare:].cpu()
        rows = x.cpu()[torch.from_numpy(~gone)]
        want = torch.full_like(got, 7)
        if s8:
            q, s = ref.codes(rows.float().numpy())
            want[at // page, at % page] = torch.from_numpy(q)
            fw = torch.full(f[spare:].shape, 5.0)
            fw[at // page, at % page] = torch.from_numpy(s)
            assert np.array_equal(f[spare:].cpu().numpy(), fw.numpy(), equal_nan=True)
            assert torch.equal(got, want)
        else:
            want[at // page, at % page] = rows
            assert torch.equal(got.view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("cache", ["same", "s8"])
@pytest.mark.parametrize("D", [1, 8, 20, 64, 80, 128, 136, 256])
def test_store_head_dims(D, cache):
    for dtype in ("f16", "bf16"):
        _store(45, 3, D, dtype, cache, 16, seed=D)


@pytest.mark.parametrize("cache", ["same", "s8"])
@pytest.mark.parametrize("page", [1, 7, 16, 24, 100])
@pytest.mark.parametrize("layout", ["dense", "heads", "odd"])
def test_store_layouts(page, cache, layout):
    for heads_first in (False, True):
        _store(130, 2, 128, "bf16", cache, page, layout, heads_first, seed=page)
        _store(19, 4, 72, "f16", cache, page, layout, heads_first, seed=page)


@pytest.mark.parametrize("total", [0, 1, 2, 63, 1025, 5000])
def test_store_lengths(total):
    for cache in ("same", "s8"):
        _store(total, 8, 128, "bf16", cache, 32)
        _store(total, 1, 64, "f16", cache, 32, skip=1.0)


def test_store_rows_at_the_ends_of_the_range():
    def change(k, v):
        k[0] = 0
        k[1, 0, 0] = float("inf")
        k[2, 1, 3] = float("nan")
        k[3] = 65504.0
        k[4] = 6e-8
        k[5, :, 1:] = 0
        v[0] = -0.0
        v[6] = torch_max
        v[7, 1] = -float("inf")
    import torch
    for dtype, torch_max in (("f16", 65504.0), ("bf16", torch.finfo(torch.bfloat16).max)):
        for cache in ("same", "s8"):
            for D in (64, 20):
                _store(12, 2, D, dtype, cache, 16, skip=0.0, change=change)


def test_store_broadcast_rows():
    """Strides of 0: one row of keys and values for every head and token."""
    import torch
    import paper_2011_10680_amd as hawq
    x = torch.randn((1, 1, 64), device="cuda").half()
    k = x.expand(10, 3, 64)
    cache = torch.zeros((2, 8, 3, 64), dtype=torch.float16, device="cuda")
    cd = hawq.CacheDesc(n_pages=2, page=8, kv_heads=3, head_dim=64, dtype=hawq.F16, page_stride=cache.stride(0), token_stride=cache.stride(1), head_stride=cache.stride(2))
    d = hawq.CacheStoreDesc(cache=cd, total=10, dtype=hawq.F16, k_token=0, k_head=0, v_token=0, v_head=0)
    other = torch.zeros_like(cache)
    hawq.hawq_cache_store(d, k, k, torch.arange(3, 13, device="cuda"), cache, other, None, None)
    torch.cuda.synchronize()
    flat = cache.view(16, 3, 64)
    assert torch.equal(cache, other) and torch.equal(flat[3:13], k) and not flat[:3].any() and not flat[13:].any()


def test_store_offsets_past_32_bits():
    _store(100, 8, 128, "bf16", "same", 16, spare=140000)

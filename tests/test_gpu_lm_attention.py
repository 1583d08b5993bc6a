"""hawq_attn_prompt and hawq_attn_tree on the GPU against the definition in 64 bits."""
import numpy as np
import pytest

import lm_reference as ref

pytestmark = pytest.mark.gpu

_NAN = float("nan")


def _types(dtype):
    import torch
    import paper_2011_10680_amd as hawq
    return (torch.float16, hawq.F16) if dtype == "f16" else (torch.bfloat16, hawq.BF16)


def _f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def _rows(**tensors):
    return {"%s_%s" % (n, w): t.stride(i) for n, t in tensors.items() for i, w in enumerate(("token", "head"))}


def _tensor(g, n, heads, D, dt, layout):
    """[n, heads, D]: dense, heads outermost, or inside a wider tensor whose rows are not 16-byte aligned."""
    import torch
    x = torch.randn((n, heads, D), generator=g, device="cuda").to(dt)
    if layout == "heads":
        return x.permute(1, 0, 2).contiguous().permute(1, 0, 2)
    if layout == "odd":
        w = torch.full((n, heads, D + 3), _NAN, dtype=dt, device="cuda")
        w[:, :, 1:D + 1] = x
        return w[:, :, 1:D + 1]
    return x


def _compare(got, want, size, top, keys, D, dtype, what):
    bound = ref.attention_bound(want, size, top, keys, D, dtype)
    same = (np.abs(got - want) <= bound) | (np.isnan(got) & np.isnan(want)) | (got == want)
    assert same.all(), (what, np.argwhere(~same)[:4], got[~same][:4], want[~same][:4], bound[~same][:4])


def _prompt(lens, q_heads, kv_heads, D, dtype, layout="dense", scale=None, change=None, seed=0, before=0):
    import torch
    import paper_2011_10680_amd as hawq
    dt, ht = _types(dtype)
    g = torch.Generator(device="cuda").manual_seed(seed)
    total = sum(lens)
    q, k, v = (_tensor(g, total, h, D, dt, layout) for h in (q_heads, kv_heads, kv_heads))
    if change:
        change(q, k, v)
    y = _tensor(g, total, q_heads, D, dt, layout)
    y.fill_(7.0)
    starts = np.concatenate(([0], np.cumsum(lens))).astype(np.int32)
    scale = D ** -0.5 if scale is None else scale
    d = hawq.AttnPromptDesc(n_seqs=len(lens), total=total, q_heads=q_heads, kv_heads=kv_heads, head_dim=D, dtype=ht, scale=scale, **_rows(q=q, k=k, v=v, y=y))
    hawq.hawq_attn_prompt(d, q, k, v, torch.from_numpy(starts).cuda(), y)
    torch.cuda.synchronize()
    got, qn, kn, vn, scale = _f64(y), _f64(q), _f64(k), _f64(v), float(np.float32(scale))
    for b, n in enumerate(lens):
        at = slice(starts[b], starts[b] + n)
        for h in range(q_heads):
            hk = h // (q_heads // kv_heads)
            want, size, top = ref.attend(qn[at, h], kn[at, hk], vn[at, hk], np.tril(np.ones((n, n), bool)), scale)
            _compare(got[at, h], want, size, top, n, D, dtype, (lens, b, h))


@pytest.mark.parametrize("D", [1, 8, 17, 40, 64, 80, 96, 128, 136, 256])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_prompt_head_dims(D, dtype):
    _prompt([37, 1, 70], 4, 2, D, dtype, seed=D)


@pytest.mark.parametrize("lens", [[1], [2, 1, 1], [0, 5, 0, 0, 64, 0], [31, 32, 33], [63, 64, 65], [127, 128, 129], [255, 256, 257], [300, 3], [700], [1] * 130])
def test_prompt_lengths(lens):
    _prompt(lens, 2, 1, 64, "bf16", seed=len(lens))
    _prompt(lens, 2, 2, 128, "f16", seed=len(lens))


@pytest.mark.parametrize("q_heads,kv_heads", [(1, 1), (3, 3), (7, 1), (12, 4), (40, 8)])
def test_prompt_heads(q_heads, kv_heads):
    _prompt([90, 33], q_heads, kv_heads, 64, "f16")
    _prompt([20, 129], q_heads, kv_heads, 128, "bf16")


@pytest.mark.parametrize("layout", ["dense", "heads", "odd"])
def test_prompt_layouts(layout):
    _prompt([65, 140], 6, 2, 64, "bf16", layout)
    _prompt([65, 140], 6, 2, 72, "f16", layout)
    _prompt([140], 4, 2, 128, "f16", layout)


def test_prompt_large_scores_and_scale():
    def change(q, k, v):
        q *= 6
        k[::7] *= 4
    for D in (64, 128):
        _prompt([200, 77], 2, 1, D, "bf16", change=change)
        _prompt([200], 2, 1, D, "f16", scale=-0.3)
        _prompt([150], 2, 1, D, "f16", scale=0.0)


@pytest.mark.parametrize("D", [64, 128, 20])
@pytest.mark.parametrize("value", [float("inf"), -float("inf"), _NAN])
def test_prompt_what_comes_later_plays_no_part(D, value):
    """An infinity or a NaN in a key or a value reaches the rows from its own on and no row before it, nor another sequence."""
    def keys(q, k, v):
        k[50, 0, 3] = value
        k[100, 0] = value

    def values(q, k, v):
        v[50, 0, 3] = value
        v[133, 0] = value
    for dtype in ("f16", "bf16"):
        _prompt([90, 80], 2, 1, D, dtype, change=values)
        _prompt([90, 80], 2, 1, D, dtype, change=keys)


def test_prompt_rows_of_minus_infinity_are_zeros():
    def change(q, k, v):
        q.fill_(1.0)
        k[:9] = -float("inf")
    for D in (64, 128, 10):
        _prompt([40, 5], 1, 1, D, "bf16", change=change)


def test_prompt_rows_outside_every_sequence_stay():
    import torch
    import paper_2011_10680_amd as hawq
    for D in (64, 128, 24):
        q = torch.randn((50, 2, D), device="cuda").half()
        y = torch.full_like(q, 7.0)
        d = hawq.AttnPromptDesc(n_seqs=2, total=50, q_heads=2, kv_heads=2, head_dim=D, dtype=hawq.F16, scale=0.1, **_rows(q=q, k=q, v=q, y=y))
        hawq.hawq_attn_prompt(d, q, q, q, torch.tensor([3, 20, 41], dtype=torch.int32, device="cuda"), y)
        torch.cuda.synchronize()
        assert (y[:3] == 7).all() and (y[41:] == 7).all() and not (y[3:41] == 7).any()


def test_prompt_wrong_starts_stay_inside():
    """Starts that decrease or leave the rows: no access outside, the rows of sound sequences as ever."""
    import torch
    import paper_2011_10680_amd as hawq
    for D in (64, 128, 24):
        q = torch.randn((64, 1, D), device="cuda").half()
        y = torch.full_like(q, 7.0)
        d = hawq.AttnPromptDesc(n_seqs=3, total=64, q_heads=1, kv_heads=1, head_dim=D, dtype=hawq.F16, scale=0.1, **_rows(q=q, k=q, v=q, y=y))
        for starts in ([0, 30, 10, 1000], [-50, 20, 2000000000, 64], [0, 0, 0, 0]):
            hawq.hawq_attn_prompt(d, q, q, q, torch.tensor(starts, dtype=torch.int32, device="cuda"), y)
        torch.cuda.synchronize()


def _tree_masks(r, drafts):
    out = []
    for n in drafts:
        seen = []
        for t in range(n):
            p = int(r.integers(-1, t)) if t else -1
            seen.append((seen[p] if p >= 0 else 0) | 1 << t)
        out += seen
    return out


def _tree(cached, drafts, q_heads, kv_heads, D, dtype, cache="same", page=16, masks="tree", layout="dense", heads_first=False, change=None, seed=0, spare=0, scale=None,
          bad_page=False, max_drafts=None):
    import torch
    import paper_2011_10680_amd as hawq
    dt, ht = _types(dtype)
    g, r = torch.Generator(device="cuda").manual_seed(seed), np.random.default_rng(seed)
    total, s8 = sum(drafts), cache == "s8"
    q, k, v = (_tensor(g, total, h, D, dt, layout) for h in (q_heads, kv_heads, kv_heads))
    y = _tensor(g, total, q_heads, D, dt, layout)
    y.fill_(7.0)
    need = [-(-c // page) for c in cached]
    n_pages, width = sum(need) + 2 + spare, max(need) + 1
    table, at = np.full((len(cached), width), -5, np.int32), 0
    order = spare + r.permutation(n_pages - spare)
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    shape = (n_pages, page, kv_heads, D)
    stored = (n_pages, kv_heads, page, D) if heads_first else shape
    caches, scales, real = [], [], []
    for _ in range(2):
        if s8:
            c = torch.randint(-127, 128, stored, generator=g, device="cuda", dtype=torch.int8)
            f = torch.rand(shape[:3], generator=g, device="cuda") * 0.02 + 0.001
        else:
            c, f = (torch.randn(stored, generator=g, device="cuda").to(dt) if not spare else torch.empty(stored, dtype=dt, device="cuda")), None
        c = c.permute(0, 2, 1, 3) if heads_first else c
        if spare:
            c[spare:] = torch.randn((n_pages - spare,) + shape[1:], generator=g, device="cuda").to(dt)
        caches.append(c)
        scales.append(f)
    # whatever lies past a request's last token, or in pages that nobody holds, is not a number
    for b, c in enumerate(cached):
        if c % page and not s8:
            for t in caches:
                t[int(table[b, c // page]), c % page:] = _NAN
        elif c % page:
            for t in scales:
                t[int(table[b, c // page]), c % page:] = _NAN
    if change:
        change(q, k, v, caches, table)
    if bad_page:
        table[0, 0] = n_pages + 3
        table[0, 1] = -1
    m = {"tree": lambda: _tree_masks(r, drafts), "none": lambda: [0] * total, "all": lambda: [(1 << 64) - 1] * total, "chain": lambda: None}[masks]()
    md = None if m is None else torch.tensor([x - (1 << 64) if x >> 63 else x for x in m], dtype=torch.int64, device="cuda")
    if m is None:
        m = [(2 << t) - 1 for n in drafts for t in range(n)]
    starts = np.concatenate(([0], np.cumsum(drafts))).astype(np.int32)
    scale = D ** -0.5 if scale is None else scale
    cd = hawq.CacheDesc(n_pages=n_pages, page=page, kv_heads=kv_heads, head_dim=D, dtype=hawq.S8 if s8 else ht, page_stride=caches[0].stride(0),
                        token_stride=caches[0].stride(1), head_stride=caches[0].stride(2))
    d = hawq.AttnTreeDesc(cache=cd, n_seqs=len(cached), total=total, max_drafts=max_drafts or max(drafts), max_cached=max(cached), q_heads=q_heads, dtype=ht, table_stride=width,
                          scale=scale, **_rows(q=q, k=k, v=v, y=y))
    ws = torch.empty(max(16, hawq.hawq_attn_tree_workspace_bytes(d)), dtype=torch.uint8, device="cuda")
    ws.fill_(0xFF)                                        # (not a number, read as floats)
    cu = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    hawq.hawq_attn_tree(d, q, k, v, cu(starts), md, caches[0], caches[1], scales[0], scales[1], cu(table), cu(np.array(cached, np.int32)), y, ws)
    torch.cuda.synchronize()
    got, qn, kn, vn, scale = _f64(y), _f64(q), _f64(k), _f64(v), float(np.float32(scale))
    for b, (c, n) in enumerate(zip(cached, drafts)):
        rows = slice(starts[b], starts[b] + n)
        past, good = [], np.ones(c, bool)
        if bad_page and b == 0:
            good[:2 * page] = False
        pages = torch.from_numpy(np.clip(table[b, :need[b]], 0, n_pages - 1).astype(np.int64)).cuda()
        for t, f in zip(caches, scales):
            x = t[pages].float() if f is None else t[pages].float() * f[pages][..., None]
            past.append(x.reshape(-1, kv_heads, D)[:c].cpu().numpy().astype(np.float64))
        tree = np.array([[m[starts[b] + i] >> j & 1 for j in range(n)] for i in range(n)], bool).reshape(n, n)
        seen = np.concatenate((np.broadcast_to(good, (n, c)), tree), axis=1)
        for h in range(q_heads):
            hk = h // (q_heads // kv_heads)
            want, size, top = ref.attend(qn[rows, h], np.concatenate((past[0][:, hk], kn[rows, hk])), np.concatenate((past[1][:, hk], vn[rows, hk])), seen, scale)
            _compare(got[rows, h], want, size, top, c + n, D, dtype, (b, h))
    return y


@pytest.mark.parametrize("cache", ["same", "s8"])
@pytest.mark.parametrize("D", [1, 8, 20, 64, 80, 96, 128, 144, 256])
def test_tree_head_dims(D, cache):
    for dtype in ("f16", "bf16"):
        _tree([75, 0, 130], [5, 3, 1], 4, 2, D, dtype, cache, seed=D)


@pytest.mark.parametrize("cached", [[0], [1], [15, 16, 17], [31, 32, 33, 63, 64, 65], [500, 0, 3, 257], [1100], [2300, 4]])
@pytest.mark.parametrize("cache", ["same", "s8"])
def test_one_token(cached, cache):
    for dtype, D, heads in (("f16", 64, (8, 1)), ("bf16", 128, (8, 2)), ("f16", 128, (2, 2))):
        _tree(cached, [1] * len(cached), *heads, D, dtype, cache, masks="chain", seed=sum(cached))


@pytest.mark.parametrize("drafts", [[2], [7, 1, 16], [17, 31, 33], [64, 1, 63], [40]])
@pytest.mark.parametrize("q_heads,kv_heads", [(1, 1), (6, 2), (7, 1), (32, 2)])
def test_trees(drafts, q_heads, kv_heads):
    cached = [100, 0, 333][:len(drafts)]
    _tree(cached, drafts, q_heads, kv_heads, 128, "bf16", seed=len(drafts))
    _tree(cached, drafts, q_heads, kv_heads, 64, "f16", "s8", seed=len(drafts))


@pytest.mark.parametrize("page", [1, 7, 16, 24, 33, 64, 100, 256])
@pytest.mark.parametrize("heads_first", [False, True])
def test_tree_pages(page, heads_first):
    for cache in ("same", "s8"):
        _tree([210, 64, 5], [9, 2, 1], 4, 2, 128, "bf16", cache, page=page, heads_first=heads_first, seed=page)
        _tree([210, 64, 5], [1, 1, 1], 4, 2, 80, "f16", cache, page=page, heads_first=heads_first, seed=page)


@pytest.mark.parametrize("masks", ["chain", "none", "all"])
def test_tree_masks(masks):
    """`none` with an empty cache: rows that see nothing are zeros."""
    for cache in ("same", "s8"):
        for D in (64, 128, 24):
            _tree([0, 40, 0], [64, 20, 1], 4, 2, D, "bf16", cache, masks=masks)


@pytest.mark.parametrize("layout", ["heads", "odd"])
def test_tree_layouts(layout):
    for D in (64, 128, 72):
        _tree([90, 17], [11, 4], 6, 2, D, "f16", layout=layout)
        _tree([90, 17], [11, 4], 6, 2, D, "bf16", "s8", layout=layout)


@pytest.mark.parametrize("value", [float("inf"), -float("inf"), _NAN])
def test_tree_unseen_drafts_play_no_part(value):
    def keys(q, k, v, caches, table):
        k[3] = value
        k[9, 0, 5] = value

    def values(q, k, v, caches, table):
        v[3] = value
        v[9, 0, 5] = value
    for D in (64, 128, 20):
        for cache in ("same", "s8"):
            _tree([50, 20], [8, 7], 4, 2, D, "bf16", cache, change=keys, seed=5)
            _tree([50, 20], [8, 7], 4, 2, D, "f16", cache, change=values, seed=5)


@pytest.mark.parametrize("value", [float("inf"), _NAN])
def test_cached_values_that_are_not_numbers_stay_in_their_request(value):
    def change(q, k, v, caches, table):
        caches[1][int(table[0, 1]), 3, 0, 5] = value
    for D in (64, 128, 20):
        _tree([50, 70], [3, 2], 4, 2, D, "bf16", change=change)


@pytest.mark.parametrize("drafts", [[1, 2], [9, 20]])
@pytest.mark.parametrize("page", [16, 24])
def test_values_that_are_not_numbers_in_a_cache_that_is_shared_out(drafts, page):
    """A part of a long cache with a NaN or an infinity in it: its rows and elements, and only those."""
    def change(q, k, v, caches, table):
        caches[1][int(table[0, 100]), 3, 0, 5] = _NAN
        caches[1][int(table[1, 7]), 2, 1] = float("inf")
        v[1, 0, 9] = -float("inf")
    for D in (64, 128):
        _tree([3000, 4500], drafts, 8, 2, D, "bf16", page=page, change=change)


def test_many_requests():
    r = np.random.default_rng(9)
    cached = r.integers(0, 700, size=70).tolist()
    _tree(cached, [1] * 70, 2, 1, 64, "f16", masks="chain")
    _tree(cached, r.integers(1, 30, size=70).tolist(), 2, 1, 64, "bf16", "s8")
    _tree((r.integers(0, 3000, size=12)).tolist(), r.integers(1, 20, size=12).tolist(), 32, 4, 64, "bf16")


def test_tree_pages_outside_the_cache_are_not_seen():
    for D in (64, 20):
        for cache in ("same", "s8"):
            _tree([100, 40], [5, 2], 4, 2, D, "bf16", cache, bad_page=True)


def test_tree_more_room_for_drafts_than_there_are():
    _tree([30, 9], [5, 2], 4, 2, 128, "bf16", max_drafts=64)
    _tree([3000, 9], [1, 1], 4, 2, 128, "bf16", max_drafts=16)


def test_tree_large_scores():
    def change(q, k, v, caches, table):
        q *= 8
    for cache in ("same", "s8"):
        _tree([600, 90], [3, 9], 8, 2, 128, "bf16", cache, change=change)
        _tree([600, 90], [3, 1], 8, 2, 64, "f16", cache, change=change)


def test_tree_offsets_past_32_bits():
    """Pages whose elements lie past 2^31 (and bytes past 2^32)."""
    _tree([70, 33], [3, 1], 8, 8, 128, "bf16", page=16, spare=140000)
    _tree([70, 33], [3, 1], 8, 8, 128, "f16", page=24, spare=94000)


def test_tree_long_cache_is_the_same_on_every_run():
    import torch
    a, b = (_tree([9000], [2], 4, 1, 64, "f16") for _ in range(2))
    assert torch.equal(a, b)


def test_graph_replays():
    """Prompt and tree attention captured once, replayed with new inputs and eager work between: the same bits as eager calls."""
    import torch
    import paper_2011_10680_amd as hawq
    D, H = 128, 4
    q = torch.randn((40, H, D), device="cuda").half()
    out = [torch.empty_like(q) for _ in range(4)]
    starts = torch.tensor([0, 15, 40], dtype=torch.int32, device="cuda")
    cache = torch.randn((200, 16, H, D), device="cuda").half()
    table = torch.arange(200, dtype=torch.int32, device="cuda").reshape(2, 100)
    cached = torch.tensor([1500, 1599], dtype=torch.int32, device="cuda")
    dp = hawq.AttnPromptDesc(n_seqs=2, total=40, q_heads=H, kv_heads=H, head_dim=D, dtype=hawq.F16, scale=0.1, **_rows(q=q, k=q, v=q, y=q))
    cd = hawq.CacheDesc(n_pages=200, page=16, kv_heads=H, head_dim=D, dtype=hawq.F16, page_stride=cache.stride(0), token_stride=cache.stride(1), head_stride=cache.stride(2))
    dt = hawq.AttnTreeDesc(cache=cd, n_seqs=2, total=40, max_drafts=25, max_cached=1600, q_heads=H, dtype=hawq.F16, table_stride=100, scale=0.1, **_rows(q=q, k=q, v=q, y=q))
    ws = torch.empty(max(16, hawq.hawq_attn_tree_workspace_bytes(dt)), dtype=torch.uint8, device="cuda")

    def both(a, b):
        hawq.hawq_attn_prompt(dp, q, q, q, starts, a)
        hawq.hawq_attn_tree(dt, q, q, q, starts, None, cache, cache, None, None, table, cached, b, ws)
    both(out[0], out[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(out[2], out[3])
    for i in range(3):
        q.copy_(torch.randn_like(q))
        both(out[0], out[1])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], out[2]) and torch.equal(out[1], out[3]), i

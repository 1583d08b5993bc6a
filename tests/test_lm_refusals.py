"""The language-model operators' argument checks, on the host: a refused call has a code and enqueues nothing (there is no GPU to enqueue to)."""
import ctypes

import pytest

OK, NULL, SHAPE, DTYPE, RANGE, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3, 4, 6, 8
P = ctypes.c_void_p(4096)
ODD = ctypes.c_void_p(4097)
TWO = ctypes.c_void_p(4098)


@pytest.fixture(scope="module")
def lib():
    import paper_2011_10680_amd as hawq
    from paper_2011_10680_amd import build
    if build.is_stale():
        build.build()
    return hawq.load_library()


def _ref(cls, base, kw):
    return ctypes.byref(cls(**dict(base, **kw)))


def test_linear(lib):
    import paper_2011_10680_amd as hawq
    base = dict(M=1, N=16, K=64, group=32, x_dtype=hawq.F16, w_dtype=hawq.S4, x_stride=64, y_stride=16)

    def call(x=P, w=P, scales=P, zeros=None, bias=None, y=P, **kw):
        return lib.hawq_linear_w4(_ref(hawq.LinearW4Desc, base, kw), x, w, scales, zeros, bias, y, None)
    assert lib.hawq_linear_w4(None, P, P, P, None, None, P, None) == NULL
    assert call(M=0) == OK and call(M=0, x=None, y=None) == OK
    for name in ("x", "w", "scales", "y"):
        assert call(**{name: None}) == NULL, name
    for kw in (dict(M=-1), dict(N=0), dict(K=0), dict(K=63), dict(group=0), dict(group=48), dict(group=-32), dict(x_stride=63), dict(y_stride=15)):
        assert call(**kw) == SHAPE, kw
    for kw in (dict(x_dtype=hawq.S8), dict(x_dtype=9), dict(w_dtype=hawq.S8), dict(w_dtype=hawq.F16), dict(zeros=P)):
        assert call(**kw) == DTYPE, kw
    assert call(w_dtype=hawq.U4) == NULL
    for name in ("x", "scales", "bias", "y"):
        assert call(**{name: ODD}) == UNSUPPORTED, name


def test_prompt(lib):
    import paper_2011_10680_amd as hawq
    base = dict(n_seqs=2, total=10, q_heads=4, kv_heads=2, head_dim=64, dtype=hawq.BF16, scale=0.1, q_token=256, q_head=64, k_token=128, k_head=64, v_token=128, v_head=64,
                y_token=256, y_head=64)

    def call(q=P, k=P, v=P, starts=P, y=P, **kw):
        return lib.hawq_attn_prompt(_ref(hawq.AttnPromptDesc, base, kw), q, k, v, starts, y, None)
    assert lib.hawq_attn_prompt(None, P, P, P, P, P, None) == NULL
    assert call(n_seqs=0) == OK and call(total=0, q=None, y=None) == OK
    for name in ("q", "k", "v", "starts", "y"):
        assert call(**{name: None}) == NULL, name
    for kw in (dict(n_seqs=-1), dict(total=-1), dict(q_heads=0), dict(kv_heads=0), dict(kv_heads=3), dict(head_dim=0), dict(head_dim=257), dict(q_token=-1), dict(k_head=-8),
               dict(y_token=63), dict(y_head=63), dict(y_token=128), dict(v_token=1 << 41)):
        assert call(**kw) == SHAPE, kw
    for dt in (hawq.S8, hawq.S32, 7):
        assert call(dtype=dt) == DTYPE
    for s in (float("nan"), float("inf")):
        assert call(scale=s) == RANGE
    for kw in (dict(q=ODD), dict(y=ODD), dict(starts=TWO)):
        assert call(**kw) == UNSUPPORTED, kw


def _cache(hawq, **kw):
    return hawq.CacheDesc(**dict(dict(n_pages=50, page=16, kv_heads=2, head_dim=64, dtype=hawq.BF16, page_stride=2048, token_stride=128, head_stride=64), **kw))


def test_tree(lib):
    import paper_2011_10680_amd as hawq
    base = dict(n_seqs=2, total=10, max_drafts=5, max_cached=300, q_heads=4, dtype=hawq.BF16, table_stride=20, scale=0.1, q_token=256, q_head=64, k_token=128, k_head=64,
                v_token=128, v_head=64, y_token=256, y_head=64)
    names = ("q", "k", "v", "starts", "mask", "k_cache", "v_cache", "k_scales", "v_scales", "table", "cached", "y", "workspace")

    def call(bytes=1 << 40, cache=None, **kw):
        args = [kw.pop(n, None if n in ("mask", "k_scales", "v_scales") else P) for n in names]
        d = hawq.AttnTreeDesc(cache=_cache(hawq, **(cache or {})), **dict(base, **kw))
        return lib.hawq_attn_tree(ctypes.byref(d), *args, bytes, None)
    assert lib.hawq_attn_tree(None, *[P] * 13, 0, None) == NULL
    assert call(n_seqs=0) == OK and call(total=0, q=None, y=None) == OK
    for name in ("q", "k", "v", "starts", "k_cache", "v_cache", "table", "cached", "y"):
        assert call(**{name: None}) == NULL, name
    for kw in (dict(n_seqs=-1), dict(total=-1), dict(max_drafts=0), dict(max_drafts=65), dict(max_cached=-1), dict(q_heads=0), dict(q_heads=3), dict(table_stride=-1),
               dict(q_token=-1), dict(y_token=128), dict(cache=dict(n_pages=-1)), dict(cache=dict(page=0)), dict(cache=dict(kv_heads=0)), dict(cache=dict(head_dim=257)),
               dict(cache=dict(token_stride=64)), dict(cache=dict(page_stride=2047)), dict(cache=dict(head_stride=1))):
        assert call(**kw) == SHAPE, kw
    for kw in (dict(dtype=hawq.U8), dict(cache=dict(dtype=hawq.F16)), dict(cache=dict(dtype=hawq.U4)), dict(k_scales=P), dict(v_scales=P)):
        assert call(**kw) == DTYPE, kw
    assert call(scale=float("nan")) == RANGE
    assert call(cache=dict(dtype=hawq.S8)) == NULL and call(cache=dict(dtype=hawq.S8), k_scales=P) == NULL
    for kw in (dict(q=ODD), dict(k_cache=ODD), dict(starts=TWO), dict(table=TWO), dict(mask=ctypes.c_void_p(4100)), dict(cache=dict(dtype=hawq.S8), k_scales=TWO, v_scales=P)):
        assert call(**kw) == UNSUPPORTED, kw


def test_tree_workspace(lib):
    import paper_2011_10680_amd as hawq
    base = dict(n_seqs=1, total=1, max_drafts=1, max_cached=1 << 20, q_heads=4, dtype=hawq.BF16, table_stride=1 << 16, scale=0.1, q_token=256, q_head=64, k_token=128, k_head=64,
                v_token=128, v_head=64, y_token=256, y_head=64)
    assert hawq.hawq_attn_tree_workspace_bytes(hawq.AttnTreeDesc(cache=_cache(hawq), **dict(base, max_drafts=0))) == 0
    assert hawq.hawq_attn_tree_workspace_bytes(hawq.AttnTreeDesc(cache=_cache(hawq), **dict(base, max_cached=0))) == 0
    need = hawq.hawq_attn_tree_workspace_bytes(hawq.AttnTreeDesc(cache=_cache(hawq), **base))
    if need:
        d = hawq.AttnTreeDesc(cache=_cache(hawq), **base)
        args = [P, P, P, P, None, P, P, None, None, P, P, P]
        assert lib.hawq_attn_tree(ctypes.byref(d), *args, P, need - 1, None) == WORKSPACE
        assert lib.hawq_attn_tree(ctypes.byref(d), *args, None, need, None) == NULL
        assert lib.hawq_attn_tree(ctypes.byref(d), *args, ctypes.c_void_p(4104), need, None) == UNSUPPORTED


def test_plan(lib):
    def call(n=2, page=16, width=4, n_free=3, n_slots=9, **kw):
        names = ("cached", "fresh", "free", "table", "starts", "slots", "counts")
        return lib.hawq_cache_plan(n, page, width, n_free, n_slots, *[kw.get(k, P) for k in names], None)
    for name in ("cached", "fresh", "free", "table", "starts", "slots", "counts"):
        assert call(**{name: None}) == NULL, name
    for kw in (dict(n=-1), dict(page=0), dict(width=-1), dict(n_free=-1), dict(n_slots=-1)):
        assert call(**kw) == SHAPE, kw
    assert call(n_slots=1 << 31) == UNSUPPORTED
    assert call(table=TWO) == UNSUPPORTED and call(slots=ctypes.c_void_p(4100)) == UNSUPPORTED


def test_plan_of_more_table_entries_than_it_counts(lib):
    def call(n, width):
        return lib.hawq_cache_plan(n, 16, width, 3, 9, P, P, P, P, P, P, P, None)
    assert call(1 << 16, (1 << 14) + 1) == UNSUPPORTED
    assert call((1 << 30) + 1, 0) == UNSUPPORTED


def test_store(lib):
    import paper_2011_10680_amd as hawq
    base = dict(total=5, dtype=hawq.BF16, k_token=128, k_head=64, v_token=128, v_head=64)
    names = ("k", "v", "slots", "k_cache", "v_cache", "k_scales", "v_scales")

    def call(cache=None, **kw):
        args = [kw.pop(n, None if n.endswith("scales") else P) for n in names]
        return lib.hawq_cache_store(ctypes.byref(hawq.CacheStoreDesc(cache=_cache(hawq, **(cache or {})), **dict(base, **kw))), *args, None)
    assert lib.hawq_cache_store(None, *[P] * 8) == NULL
    assert call(total=0, k=None) == OK and call(cache=dict(n_pages=0)) == OK
    for name in ("k", "v", "slots", "k_cache", "v_cache"):
        assert call(**{name: None}) == NULL, name
    for kw in (dict(total=-1), dict(k_token=-1), dict(cache=dict(page=-1)), dict(cache=dict(token_stride=127)), dict(cache=dict(page_stride=100))):
        assert call(**kw) == SHAPE, kw
    for kw in (dict(dtype=hawq.S4), dict(cache=dict(dtype=hawq.F16)), dict(k_scales=P)):
        assert call(**kw) == DTYPE, kw
    assert call(cache=dict(dtype=hawq.S8)) == NULL
    for kw in (dict(k=ODD), dict(v_cache=ODD), dict(slots=ctypes.c_void_p(4100))):
        assert call(**kw) == UNSUPPORTED, kw

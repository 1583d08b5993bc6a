"""The language-model operators at the ends of what they take: values that are not finite where a row sees them, lengths and starts beyond what
a call says, bounds far above the lengths, paths that only certain sizes reach."""
import numpy as np
import pytest

import lm_reference as ref
import test_gpu_lm_attention as base

pytestmark = pytest.mark.gpu

_NAN, _INF = float("nan"), float("inf")


def _strict(got, want, size, top, keys, D, dtype, what, more=0.0):
    """Infinities and NaN have to be where the definition has them; the rest lies within the derived bound (and what a caller adds to it)."""
    finite = np.isfinite(want)
    with np.errstate(invalid="ignore"):
        bound = ref.attention_bound(np.where(finite, want, 0), np.where(np.isfinite(size), size, 0), top, keys, D, dtype) + more
        same = np.where(finite, np.abs(got - want) <= bound, np.where(np.isnan(want), np.isnan(got), got == want))
    assert same.all(), (what, np.argwhere(~same)[:4], got[~same][:4], want[~same][:4], bound[~same][:4])


@pytest.fixture
def strict(monkeypatch):
    monkeypatch.setattr(base, "_compare", _strict)


def test_the_strict_comparison_finds_what_differs():
    one, inf = np.ones((1, 1)), np.full((1, 1), _INF)
    for got, want in ((one, inf), (-inf, inf), (inf, one), (inf * 0, inf), (one, inf * 0)):
        with np.errstate(invalid="ignore"), pytest.raises(AssertionError):
            _strict(got, want, np.abs(want), 1.0, 1, 8, "f16", "")
    for both in (one, inf, -inf, np.full((1, 1), _NAN)):
        _strict(both, both, np.abs(both), 1.0, 1, 8, "f16", "")


@pytest.mark.parametrize("D", [64, 128, 20])
@pytest.mark.parametrize("value", [_INF, -_INF, _NAN])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_prompt_rows_that_see_values_that_are_not_finite(strict, D, value, dtype):
    def keys(q, k, v):
        k[50, 0, 3] = value
        k[100, 0] = value

    def values(q, k, v):
        v[50, 0, 3] = value
        v[133, 0] = value
        v[140, 0, 7] = -value
        v[150, 0, 7] = value
    base._prompt([90, 80], 2, 1, D, dtype, change=values)
    base._prompt([90, 80], 2, 1, D, dtype, change=keys)


@pytest.mark.parametrize("D", [64, 128, 20])
@pytest.mark.parametrize("value", [_INF, -_INF, _NAN])
@pytest.mark.parametrize("cache", ["same", "s8"])
def test_tree_rows_that_see_values_that_are_not_finite(strict, D, value, cache):
    def keys(q, k, v, caches, table):
        k[3] = value
        k[9, 0, 5] = value

    def values(q, k, v, caches, table):
        v[3] = value
        v[9, 0, 5] = value
        if cache == "same":
            caches[1][int(table[0, 1]), 3, 0, 5] = value
    for dtype in ("f16", "bf16"):
        base._tree([50, 20], [8, 7], 4, 2, D, dtype, cache, change=keys, seed=5)
        base._tree([50, 20], [8, 7], 4, 2, D, dtype, cache, change=values, seed=5)


@pytest.mark.parametrize("drafts", [[1, 2], [9, 20]])
@pytest.mark.parametrize("page", [16, 24])
def test_shared_out_caches_with_values_that_are_not_finite(strict, drafts, page):
    def change(q, k, v, caches, table):
        caches[1][int(table[0, 100]), 3, 0, 5] = _NAN
        caches[1][int(table[1, 7]), 2, 1] = _INF
        v[1, 0, 9] = -_INF
    for D in (64, 128):
        base._tree([3000, 4500], drafts, 8, 2, D, "bf16", page=page, change=change)


# ---- descriptors that say less, or more, than the device data ------------------------------------------------------------------

def _guarded(shape, dt, fill=7.0, margin=4096):
    """A tensor with the same fill before and behind it, and the whole."""
    import torch
    n = int(np.prod(shape))
    whole = torch.full((n + 2 * margin,), fill, dtype=dt, device="cuda")
    return whole, whole[margin:margin + n].view(shape)


def _check_guards(whole, n, margin=4096, fill=7.0):
    assert bool((whole[:margin] == fill).all()) and bool((whole[margin + n:] == fill).all())


_FORMS = {  # q_heads, kv_heads, head_dim, cached tokens
    "matrix": (4, 2, 64, [40, 300, 17]),
    "plain": (4, 2, 20, [40, 300, 17]),
    "shared out": (4, 2, 64, [1500, 3000, 70]),
    "listed": (32, 8, 64, [1500, 4500, 70]),
}


def _tree_as_described(form, starts, total, cached, max_cached, max_drafts, width=None, dtype="bf16", cache="same", page=16, seed=0, held=None):
    """hawq_attn_tree against its definition with every length clamped as the interface says; rows that no request has keep their fill.
    held: the tokens that the tables and caches really hold (default: cached)."""
    import torch
    import paper_2011_10680_amd as hawq
    q_heads, kv_heads, D, _ = _FORMS[form]
    dt, ht = base._types(dtype)
    g, r = torch.Generator(device="cuda").manual_seed(seed), np.random.default_rng(seed)
    n, s8 = len(cached), cache == "s8"
    q, k, v = (torch.randn((total, h, D), generator=g, device="cuda").to(dt) for h in (q_heads, kv_heads, kv_heads))
    whole, y = _guarded((total, q_heads, D), dt)
    need = [-(-c // page) for c in (held or cached)]
    width = max(need) if width is None else width
    n_pages = sum(need) + 1
    order, at = r.permutation(n_pages), 0
    table = np.full((n, width), n_pages + 9, np.int32)
    for b, c in enumerate(need):
        table[b, :min(c, width)] = order[at:at + c][:width]
        at += c
    shape = (n_pages, page, kv_heads, D)
    caches = [torch.randint(-127, 128, shape, generator=g, device="cuda", dtype=torch.int8) if s8 else torch.randn(shape, generator=g, device="cuda").to(dt) for _ in "kv"]
    scales = [torch.rand(shape[:3], generator=g, device="cuda") * 0.02 + 0.001 if s8 else None for _ in "kv"]
    cd = hawq.CacheDesc(n_pages=n_pages, page=page, kv_heads=kv_heads, head_dim=D, dtype=hawq.S8 if s8 else ht, page_stride=caches[0].stride(0),
                        token_stride=caches[0].stride(1), head_stride=caches[0].stride(2))
    d = hawq.AttnTreeDesc(cache=cd, n_seqs=n, total=total, max_drafts=max_drafts, max_cached=max_cached, q_heads=q_heads, dtype=ht, table_stride=width, scale=D ** -0.5,
                          **base._rows(q=q, k=k, v=v, y=y))
    size = hawq.hawq_attn_tree_workspace_bytes(d)
    ws_whole, ws = _guarded((max(16, -(-size // 4)),), torch.float32, fill=3.0)
    ws.fill_(_NAN)
    cu = lambda a: torch.from_numpy(np.asarray(a, np.int32)).cuda()  # noqa: E731
    hawq.hawq_attn_tree(d, q, k, v, cu(starts), None, caches[0], caches[1], scales[0], scales[1], cu(table), cu(cached), y, ws)
    torch.cuda.synchronize()
    _check_guards(whole, total * q_heads * D)
    _check_guards(ws_whole, ws.numel(), fill=3.0)
    got, qn, kn, vn = base._f64(y), base._f64(q), base._f64(k), base._f64(v)
    first = [min(max(s, 0), total) for s in starts[:-1]]
    last = [min(max(e, f), total) for f, e in zip(first, starts[1:])]
    rows = [range(f, f + min(e - f, max_drafts)) for f, e in zip(first, last)]
    owners = np.zeros(total, int)
    for x in rows:
        owners[list(x)] += 1
    assert (got[owners == 0] == 7.0).all()
    for b, x in enumerate(rows):
        if not len(x):
            continue
        c = min(max(cached[b], 0), max_cached, width * page)
        pages = table[b, np.arange(c) // page].astype(np.int64)
        seen_c = pages < n_pages
        at_page, place = torch.from_numpy(np.minimum(pages, n_pages - 1)).cuda(), torch.arange(c, device="cuda") % page
        past = [base._f64(t[at_page, place].float() * (1 if f is None else f[at_page, place][..., None])) for t, f in zip(caches, scales)]
        m = len(x)
        seen = np.concatenate((np.broadcast_to(seen_c, (m, c)), np.tril(np.ones((m, m), bool))), axis=1)
        alone = owners[list(x)] == 1
        for h in range(q_heads):
            hk = h // (q_heads // kv_heads)
            want, size_, top = ref.attend(qn[list(x), h], np.concatenate((past[0][:, hk], kn[list(x), hk])), np.concatenate((past[1][:, hk], vn[list(x), hk])), seen,
                                          float(np.float32(D ** -0.5)))
            _strict(got[list(x), h][alone], want[alone], size_[alone], top, c + m, D, dtype, (form, b, h))


@pytest.mark.parametrize("form", list(_FORMS))
@pytest.mark.parametrize("cache", ["same", "s8"])
def test_tree_lengths_beyond_the_bounds_are_clamped(form, cache):
    lens = _FORMS[form][3]
    starts = [0, 9, 9 + 20, 9 + 20 + 11]
    _tree_as_described(form, starts, 45, lens, max(lens), 20, cache=cache)                                       # as it should be, five rows left over
    _tree_as_described(form, starts, 45, [n + 5000 for n in lens], max(lens), 20, cache=cache, held=lens, width=max(-(-n // 16) for n in lens))
    _tree_as_described(form, starts, 45, [-5, lens[1], -(1 << 31)], max(lens), 20, cache=cache, held=lens)       # negative: none
    _tree_as_described(form, starts, 45, lens, max(lens) + 9000, 20, cache=cache)                                # a bound past the table
    _tree_as_described(form, starts, 45, [lens[0], (1 << 31) - 1, lens[2]], (1 << 30), 20, cache=cache, held=lens)   # more than the table has room for
    _tree_as_described(form, starts, 45, lens, max(lens) // 2, 20, cache=cache)                                  # a bound below the lengths
    _tree_as_described(form, starts, 45, lens, max(lens), 7, cache=cache)                                        # more drafts than there is room for


@pytest.mark.parametrize("form", list(_FORMS))
@pytest.mark.parametrize("starts", [[4, 9, 20, 33], [5, 30, 10, 400], [-3, 7, 7, 999], [1 << 30, -(1 << 31), (1 << 31) - 1, 12], [0, 0, 0, 0], [40, 30, 20, 10]])
def test_tree_wrong_starts_stay_inside(form, starts):
    """Rows of one request alone are as ever, rows of none keep their fill, whatever the starts are."""
    _tree_as_described(form, starts, 40, _FORMS[form][3], max(_FORMS[form][3]), 30)


@pytest.mark.parametrize("D", [64, 128, 24])
@pytest.mark.parametrize("starts,sound", [([0, 30, 10, 1000], [(0, 10)]), ([-50, 20, 2000000000, 64], [(0, 20), (20, 64)]), ([0, 0, 0, 0], []), ([3, 20, 20, 41], [(3, 20), (20, 41)]),
                                          ([64, 20, 10, 5], []), ([1 << 30, -(1 << 31), (1 << 31) - 1, 12], [])])
def test_prompt_wrong_starts_write_nothing_else(D, starts, sound):
    import torch
    import paper_2011_10680_amd as hawq
    total = 64
    g = torch.Generator(device="cuda").manual_seed(D)
    q = torch.randn((total, 2, D), generator=g, device="cuda").half()
    whole, y = _guarded((total, 2, D), torch.float16)
    d = hawq.AttnPromptDesc(n_seqs=3, total=total, q_heads=2, kv_heads=2, head_dim=D, dtype=hawq.F16, scale=0.1, **base._rows(q=q, k=q, v=q, y=y))
    hawq.hawq_attn_prompt(d, q, q, q, torch.tensor(starts, dtype=torch.int32, device="cuda"), y)
    torch.cuda.synchronize()
    _check_guards(whole, total * 2 * D)
    got, x = base._f64(y), base._f64(q)
    first = [min(max(s, 0), total) for s in starts[:-1]]
    held = np.zeros(total, bool)
    for f, e in zip(first, starts[1:]):
        held[f:min(max(e, f), total)] = True
    assert (got[~held] == 7).all()
    for f, e in sound:
        for h in range(2):
            want, size, top = ref.attend(x[f:e, h], x[f:e, h], x[f:e, h], np.tril(np.ones((e - f, e - f), bool)), float(np.float32(0.1)))
            _strict(got[f:e, h], want, size, top, e - f, D, "f16", (starts, f, h))


def test_listed_parts_over_an_8_bit_cache(strict):
    base._tree([1500, 4500, 70], [9, 20, 11], 32, 8, 128, "bf16", "s8")
    base._tree([1500, 4500, 70, 0, 9000], [9, 64, 11, 3, 1], 32, 8, 64, "f16", "s8", page=24)


@pytest.mark.parametrize("form", list(_FORMS))
@pytest.mark.parametrize("cache", ["same", "s8"])
def test_tree_with_a_bound_far_above_the_lengths(form, cache):
    lens = _FORMS[form][3]
    _tree_as_described(form, [0, 9, 29, 40], 45, lens, 100000, 20, cache=cache, width=6300)
    _tree_as_described(form, [0, 1, 2, 3], 3, lens, 1 << 20, 1, cache=cache, width=1 << 16)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_the_same_bits_on_every_run(dtype):
    """Prompts of several sequences, drafted trees that are listed and single tokens over shared-out caches: no order of workgroups shows."""
    import torch
    import paper_2011_10680_amd as hawq
    dt, ht = base._types(dtype)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((1700, 32 + 8 + 8, 128), generator=g, device="cuda").to(dt)
    q, k, v = x[:, :32], x[:, 32:40], x[:, 40:]
    cache = torch.randn((400, 16, 8, 128), generator=g, device="cuda").to(dt)
    codes = torch.randint(-127, 128, cache.shape, generator=g, device="cuda", dtype=torch.int8)
    scales = torch.rand(cache.shape[:3], generator=g, device="cuda") * 0.01
    i32 = dict(dtype=torch.int32, device="cuda")
    table, cached = torch.arange(400, **i32).reshape(2, 200).contiguous(), torch.tensor([3000, 1777], **i32)
    y = torch.empty((1700, 32, 128), dtype=dt, device="cuda")
    dp = hawq.AttnPromptDesc(n_seqs=3, total=1700, q_heads=32, kv_heads=8, head_dim=128, dtype=ht, scale=0.09, **base._rows(q=q, k=k, v=v, y=y))

    def tree(drafts, kc, s):
        cd = hawq.CacheDesc(n_pages=400, page=16, kv_heads=8, head_dim=128, dtype=ht if s is None else hawq.S8, page_stride=kc.stride(0), token_stride=kc.stride(1),
                            head_stride=kc.stride(2))
        d = hawq.AttnTreeDesc(cache=cd, n_seqs=2, total=2 * drafts, max_drafts=drafts, max_cached=3000, q_heads=32, dtype=ht, table_stride=200, scale=0.09,
                              **base._rows(q=q, k=k, v=v, y=y))
        ws = torch.empty(hawq.hawq_attn_tree_workspace_bytes(d), dtype=torch.uint8, device="cuda").fill_(int(torch.randint(0, 256, (1,))))
        hawq.hawq_attn_tree(d, q, k, v, torch.tensor([0, drafts, 2 * drafts], **i32), None, kc, kc, s, s, table, cached, y, ws)
    calls = [lambda: hawq.hawq_attn_prompt(dp, q, k, v, torch.tensor([0, 700, 701, 1700], **i32), y)]
    calls += [lambda n=n, kc=kc, s=s: tree(n, kc, s) for n in (1, 30) for kc, s in ((cache, None), (codes, scales))]
    for i, call in enumerate(calls):
        seen = []
        for _ in range(4):
            y.fill_(7.0)
            call()
            seen.append(y.clone())
        assert all(torch.equal(seen[0].view(torch.int16), s.view(torch.int16)) for s in seen[1:]), i

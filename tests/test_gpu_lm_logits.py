"""hawq_logits on the GPU against the definition in 64 bits."""
import numpy as np
import pytest

import lm_step_reference as ref

pytestmark = pytest.mark.gpu


def _run(drafts, V, past, dtype, biases=0, masks=0, pad=0, y_pad=0, at=0, y_at=0, in_place=False, use=("prompt", "starts", "drafts", "mask", "penalties"), rows="some", few=None, seed=0,
         behind=0, change=None):
    """drafts: rows of every request; past: their histories' lengths; few: tokens are of the first few ids; behind: rows past the last request."""
    import torch
    import paper_2011_10680_amd as hawq
    dt = {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    r = np.random.default_rng(seed)
    n, total = len(drafts), sum(drafts) + behind
    words = lambda shape: r.integers(-1, few or V + 1, size=shape).astype(np.int32)  # noqa: E731  (some outside the vocabulary)
    width = max(max(past), 1) + 3
    i = dict(past=words((n, width)), past_lens=np.array(past, np.int32), prompt_lens=r.integers(0, width, size=n).astype(np.int32),
             starts=np.concatenate(([0], np.cumsum(drafts))).astype(np.int32), drafts=words(total),
             mask=np.array([int(v) for v in r.integers(0, 1 << 63, size=total, dtype=np.int64)], np.int64),
             penalties=np.stack([r.choice([1.0, 1.3, 0.8], size=n), r.choice([0.0, 0.7, -0.2], size=n), r.choice([0.0, 0.3], size=n)], axis=1).astype(np.float32))
    counts = r.integers(0, biases + 1, size=n) if biases else np.zeros(n, int)
    m = int(counts.sum())
    i.update(bias_starts=np.concatenate(([0], np.cumsum(counts))).astype(np.int32), bias_ids=words(m), bias_values=r.normal(size=m).astype(np.float32) * 5)
    W = -(-V // 32) + (3 if masks else 0)
    i.update(allowed=r.integers(-2 ** 31, 2 ** 31, size=(max(masks, 1), W)).astype(np.int32), allowed_row=r.integers(-2, masks + 2, size=total).astype(np.int32))
    if masks > 1:
        i["allowed"][1] = 0                                          # a mask that leaves a row empty
    if change:
        change(i)
    if "prompt" not in use:
        i["prompt_lens"] = None
    for name in ("starts", "drafts", "mask", "penalties"):
        if name not in use:
            i[name] = None
    if rows != "some":
        i["allowed_row"] = None
    if not m:
        i["bias_starts"] = i["bias_ids"] = i["bias_values"] = None
    if not masks:
        i["allowed"] = i["allowed_row"] = None
    whole = torch.full((at + total * (V + pad) + 16,), float("nan"), dtype=dt, device="cuda")
    x = whole[at:at + total * (V + pad)].view(total, V + pad)[:, :V]
    x.copy_(torch.from_numpy(r.normal(size=(total, V)).astype(np.float32) * 4))
    x[0, V // 2] = float("-inf")
    held = x.double().cpu().numpy()
    out = torch.full((y_at + total * (V + y_pad) + 16,), 7.0, dtype=dt, device="cuda")
    y = x if in_place else out[y_at:y_at + total * (V + y_pad)].view(total, V + y_pad)[:, :V]
    d = hawq.LogitsDesc(n_seqs=n, total=total, vocab=V, dtype=hawq.F16 if dtype == "f16" else hawq.BF16, past_stride=width, n_bias=m, n_allowed=masks, allowed_stride=W,
                        x_stride=V + pad, y_stride=V + (pad if in_place else y_pad))
    c = {k: None if v is None else torch.from_numpy(np.ascontiguousarray(v)).cuda() for k, v in i.items()}
    hawq.hawq_logits(d, x, c["past"], c["past_lens"], c["prompt_lens"], c["starts"], c["drafts"], c["mask"], c["penalties"], c["bias_starts"], c["bias_ids"], c["bias_values"],
                     c["allowed"], c["allowed_row"], y)
    torch.cuda.synchronize()
    want, bound, written = ref.logits(held, i["past"], i["past_lens"], i["prompt_lens"], i["starts"], i["drafts"], i["mask"], i["penalties"], i["bias_starts"], i["bias_ids"],
                                      i["bias_values"], None if i["allowed"] is None else i["allowed"].view(np.uint32), i["allowed_row"], dtype)
    got = y.double().cpu().numpy()
    finite = np.isfinite(want)
    assert (got[written][~finite[written]] == want[written][~finite[written]]).all()
    off = np.where(finite, np.abs(got - np.where(finite, want, 0)), 0)[written]
    assert (off <= np.where(finite, bound, 0)[written]).all(), (drafts, V, float(off.max()))
    if in_place:
        assert int(torch.isnan(whole).sum()) == whole.numel() - total * V
        assert np.array_equal(got[~written], held[~written])
    else:
        assert (got[~written] == 7.0).all() and float(out[:y_at].sum()) == 7.0 * y_at and bool((out[y_at + total * (V + y_pad):] == 7.0).all())
        if y_pad:
            assert bool((out[y_at:y_at + total * (V + y_pad)].view(total, -1)[:, V:] == 7.0).all())


@pytest.mark.parametrize("V", [1, 2, 7, 31, 32, 33, 64, 100, 1000, 2048, 2049, 8191, 8192, 8193, 20001])
@pytest.mark.parametrize("in_place", [False, True])
def test_vocabularies(V, in_place):
    _run([1, 3], V, [5, 40], "f16", biases=4, masks=3, in_place=in_place, seed=V)
    _run([2], V, [30], "bf16", biases=0, masks=0, in_place=in_place, seed=V)
    _run([1], V, [0], "bf16", biases=9, masks=2, in_place=in_place, few=min(V, 5), seed=V)


@pytest.mark.parametrize("drafts", [[1], [1] * 9, [3, 1, 7], [64], [64, 1, 33], [0, 2, 0, 0, 5, 0], [70, 3]])
def test_requests(drafts):
    for i, use in enumerate((("prompt", "starts", "drafts", "mask", "penalties"), ("starts", "drafts", "penalties"), ("starts", "penalties"), ("prompt", "starts", "drafts"))):
        _run(drafts, 600, [13 * j % 50 for j in range(len(drafts))], "bf16" if i % 2 else "f16", biases=6, masks=4, use=use, few=40, seed=i)


@pytest.mark.parametrize("n", [63, 64, 65, 200, 4096, 4097, 5000])
def test_many_requests(n):
    """A row's request is found among all, empty ones and rows behind the last one too."""
    r = np.random.default_rng(n)
    _run(r.integers(0, 3, size=n).tolist() + [1], 40, r.integers(0, 6, size=n + 1).tolist(), "bf16", biases=1, masks=3, behind=2, few=40, seed=n)


def test_one_row_each_without_starts():
    for drafts in (True, False):
        _run([1] * 7, 900, [4, 0, 9, 100, 1, 2, 50], "f16", biases=3, masks=7, use=("prompt", "penalties") + (("drafts",) if drafts else ()), seed=1)
    _run([1] * 7, 900, [4, 0, 9, 100, 1, 2, 50], "f16", biases=3, masks=7, use=("prompt", "penalties"), rows="their own", seed=2)


@pytest.mark.parametrize("pad,y_pad,at,y_at,in_place", [(8, 8, 0, 0, False), (8, 0, 0, 0, False), (0, 3, 0, 0, False), (3, 0, 1, 0, False), (0, 0, 3, 5, False), (1, 1, 7, 7, False), (1, 0, 1, 0, True),
                                                        (24, 0, 8, 0, True), (5, 0, 0, 0, True), (2, 4, 2, 6, False)])
def test_strides_and_alignment(pad, y_pad, at, y_at, in_place):
    for V in (1000, 8199, 37):
        _run([2, 1, 4], V, [20, 300, 7], "bf16", biases=5, masks=4, pad=pad, y_pad=y_pad, at=at, y_at=y_at, in_place=in_place, few=V // 2, seed=V)


def test_rows_behind_the_last_request_stay():
    for in_place in (False, True):
        _run([2, 0, 1], 700, [9, 3, 4], "f16", biases=3, masks=3, behind=5, in_place=in_place, seed=3)


def test_long_history_of_few_tokens():
    """One token written 30000 times: counted, not saturated."""
    _run([1, 2], 300, [30000, 29999], "bf16", few=3, seed=1)
    _run([1], 9000, [70001], "f16", few=9000, seed=2)


def test_wrong_lengths_and_lists_are_bounded():
    def change(i):
        i["past_lens"][:] = [1 << 30, -5, 3]
        i["prompt_lens"][:] = [-7, 1 << 30, 0]
        i["allowed_row"][0] = -(1 << 31)
    # (the reference walks over the row's own length)
    def clamped(i):
        change(i)
        i["past_lens"][0] = i["past"].shape[1]
    _run([1, 1, 2], 500, [20, 20, 20], "f16", biases=3, masks=2, seed=4, change=clamped)
    import torch
    import paper_2011_10680_amd as hawq
    x = torch.randn((3, 500), device="cuda").half()
    y = torch.full_like(x, 7.0)
    i32 = dict(dtype=torch.int32, device="cuda")
    d = hawq.LogitsDesc(n_seqs=2, total=3, vocab=500, dtype=hawq.F16, past_stride=4, n_bias=2, n_allowed=1, allowed_stride=16, x_stride=500, y_stride=500)
    for starts in ([0, 9, 3], [-4, 1, 100], [5, 6, 7], [3, 2, 1]):
        for bias in ([0, 1 << 30, -1], [-9, 7, 9]):
            hawq.hawq_logits(d, x, torch.zeros((2, 4), **i32), torch.tensor([1 << 31 - 1, 4], **i32), torch.tensor([-1, 9], **i32), torch.tensor(starts, **i32),
                             torch.tensor([499, 500, -1], **i32), torch.full((3,), -1, dtype=torch.int64, device="cuda"), torch.ones((2, 3), device="cuda"), torch.tensor(bias, **i32),
                             torch.tensor([-1, 500], **i32), torch.ones(2, device="cuda"), torch.full((1, 16), -1, **i32), torch.tensor([7, 0, -1], **i32), y)
    torch.cuda.synchronize()


def test_the_same_token_twice_in_a_list_has_its_last_value():
    def change(i):
        i["bias_ids"][:] = 5
    _run([1, 2, 1], 700, [4, 4, 4], "f16", biases=40, few=9, seed=5, change=change)


@pytest.mark.parametrize("V", [30, 1000, 8193, 20001])
def test_long_lists_of_biases(V):
    """Lists longer than are searched for every token, with tokens listed more than once, and short ones beside them."""
    def change(i):
        n = i["bias_starts"]
        n[:] = np.concatenate(([0], np.sort(np.random.default_rng(1).integers(0, n[-1], size=len(n) - 2)), [n[-1]]))
    for in_place in (False, True):
        _run([2, 1, 3], V, [50, 3, 200], "f16", biases=3000, masks=3, in_place=in_place, pad=3, few=V + 1, seed=V, change=change)
        _run([1, 1], V, [5, 30], "bf16", biases=66, y_pad=5, seed=V)


def test_masked_values_whatever_they_hold():
    import torch
    import paper_2011_10680_amd as hawq
    V = 100
    for in_place in (False, True):
        x = torch.full((2, V), float("nan"), dtype=torch.bfloat16, device="cuda")
        x[:, 40:] = float("inf")
        x[:, 50] = 2.0
        bits = torch.zeros((1, 4), dtype=torch.int32, device="cuda")
        bits[0, 1] = 1 << (50 - 32)
        y = x if in_place else torch.empty_like(x)
        d = hawq.LogitsDesc(n_seqs=2, total=2, vocab=V, dtype=hawq.BF16, past_stride=0, n_bias=0, n_allowed=1, allowed_stride=4, x_stride=V, y_stride=V)
        hawq.hawq_logits(d, x, None, None, None, None, None, None, None, None, None, None, bits, torch.zeros(2, dtype=torch.int32, device="cuda"), y)
        torch.cuda.synchronize()
        assert float(y[0, 50]) == 2.0 and bool((y[:, :50] == float("-inf")).all()) and bool((y[:, 51:] == float("-inf")).all())


def test_one_row_of_logits_for_all():
    """x_stride 0: every request's own result from the same logits."""
    import torch
    import paper_2011_10680_amd as hawq
    x = torch.randn((1, 333), device="cuda").half()
    past = torch.arange(6, dtype=torch.int32, device="cuda").view(3, 2)
    y = torch.empty((3, 333), dtype=torch.float16, device="cuda")
    d = hawq.LogitsDesc(n_seqs=3, total=3, vocab=333, dtype=hawq.F16, past_stride=2, n_bias=0, n_allowed=0, allowed_stride=0, x_stride=0, y_stride=333)
    hawq.hawq_logits(d, x, past, torch.full((3,), 2, dtype=torch.int32, device="cuda"), None, None, None, None, torch.tensor([[1.0, 1.0, 0.5]] * 3, device="cuda"), None, None, None, None,
                     None, y)
    want = x.expand(3, -1).float().clone()
    for b in range(3):
        want[b, 2 * b:2 * b + 2] -= 1.5
    assert torch.equal(y, want.half())


@pytest.mark.parametrize("past", [2000, 2699, 2700, 5400, 5401, 9990, 10001, 15000])
@pytest.mark.parametrize("few", [None, 50])
def test_what_changes_in_place(past, few):
    """In place without masks only the tokens that occurred or are listed are touched, however many there are."""
    _run([1, 2], 20001, [past, past // 2], "bf16", biases=8, in_place=True, few=few, seed=past)
    _run([1, 2], 20001, [past, 10], "f16", biases=400, in_place=True, few=few, seed=past)


def test_many_logits():
    """Past 2^24 logits, with drafts, masks, short and long lists, and rows behind the last request."""
    _run([5] * 25 + [4], 131073, [40 * i for i in range(26)], "bf16", biases=60, masks=20, pad=3, behind=1, seed=1)
    _run([1] * 33, 600001, [1000] * 32 + [11000], "f16", biases=300, masks=5, in_place=True, few=3000, seed=2)


@pytest.mark.parametrize("seed", [1, 2])
def test_histories_of_neighbouring_hashes(seed):
    """Tokens whose product with the hash's factor has small upper bits: all begin their search in a few places beside one another."""
    V = 131072
    order = np.argsort((np.arange(V, dtype=np.uint64) * 2654435761 & 0xFFFFFFFF) >> 18, kind="stable").astype(np.int32)
    def change(i):
        i["past"][:] = order[np.random.default_rng(seed).integers(0, 9000, size=i["past"].shape)]
        i["past"][0, :9000] = order[:9000]
    _run([1, 1], V, [9900, 4000], "bf16", biases=20, in_place=True, seed=seed, change=change)

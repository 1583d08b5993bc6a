"""The operators of a language model served from 4-bit weights and a paged cache, as measurable cases.

A case is a dict of plain values.  `listed()` gives the fixed ones, `draw(rng)` one more of the same ranges; `prepare` makes what a
program holds before the call on the GPU, `run` is one pass: with `own` through the framework's entry points, without it in plain
torch operations in 32 bits.  `exact` is the definition in 64 bits, `work` the bytes and operations a pass cannot do without.

Kinds of case
  linear   activations of one to 64 tokens times 4-bit weights with a scale (and a zero point) per group (`hawq_linear_w4`)
  prompt   causal attention over whole prompts, packed one behind the other, grouped heads (`hawq_attn_prompt`)
  tree     attention of drafted tokens, or of one token, over a paged cache in 16 or 8 bits (`hawq_attn_tree`)
  plan     block tables, slots and sequence starts from the requests' lengths (`hawq_cache_plan`)
  store    new rows of keys and values to their slots of the cache, in 16 or 8 bits (`hawq_cache_store`)
Lengths are texts of integers joined by commas, one per sequence.
"""
import math
import random

import torch

own = False

_TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


# ---- cases ---------------------------------------------------------------------------------------------------------------

def _ints(text):
    return [int(v) for v in text.split(",")]


def _text(values):
    return ",".join(str(v) for v in values)


def _ragged(seed, n, most, least=1):
    """n lengths spread evenly from `least` to `most`, in a fixed shuffled order."""
    v = [least + (most - least) * i // max(1, n - 1) for i in range(n)]
    random.Random(seed).shuffle(v)
    return _text(v)


def listed():
    return [
        # the classifier's shape in 4 bits, for one token: a pure latency measurement
        dict(name="linear_1x1000x2048_f16", kind="linear", M=1, N=1000, K=2048, group=128, dtype="f16", zeros=False, bias=True, pad=0),
        # a wide layer for the thirteen tokens of a small draft tree: bound by the weights' bytes
        dict(name="linear_13x16384x8192_bf16", kind="linear", M=13, N=16384, K=8192, group=64, dtype="bf16", zeros=True, bias=False, pad=8),
        # a few short requests that arrive together, one of a single token: latency
        dict(name="prompt_short_f16", kind="prompt", lens="1,17,64,5,128,33", q_heads=16, kv_heads=16, head_dim=64, dtype="f16", fused=False),
        # an ordinary batch of prompts of very different lengths, q, k and v as slices of one projection's output
        dict(name="prompt_ragged_bf16", kind="prompt", lens=_ragged(1, 12, 2048), q_heads=32, kv_heads=8, head_dim=128, dtype="bf16", fused=True),
        # long documents: the matrix rate
        dict(name="prompt_long_bf16", kind="prompt", lens="8192,5000,8001", q_heads=32, kv_heads=8, head_dim=128, dtype="bf16", fused=True),
        # one user, one token, a short cache, one shared head of keys: latency
        dict(name="decode_one_f16", kind="tree", cached="611", drafts="1", q_heads=8, kv_heads=1, head_dim=64, dtype="f16", cache="f16", page=16, heads_first=False),
        # draft trees of many sizes over caches from empty to some thousands, pages that divide no tile
        dict(name="tree_ragged_bf16", kind="tree", cached="1500,0,4097,31,2048,777,1", drafts="13,25,1,8,40,13,64", q_heads=32, kv_heads=8, head_dim=128, dtype="bf16",
             cache="bf16", page=24, heads_first=True),
        # a batch in the midst of long answers, one token each, the cache in 8 bits: bound by the cache's bytes
        dict(name="decode_long_s8", kind="tree", cached=_ragged(2, 32, 16384, 500), drafts=_text([1] * 32), q_heads=32, kv_heads=8, head_dim=128, dtype="bf16", cache="s8",
             page=32, heads_first=False),
        # a few requests of some hundred tokens: latency
        dict(name="plan_few", kind="plan", n=5, page=16, cached=600, fresh=200, spare=64),
        # a large server's whole prefill wave
        dict(name="plan_many", kind="plan", n=2000, page=16, cached=2000, fresh=1000, spare=5000),
        # the accepted tokens of one step, the rejected ones' slots empty, into an 8-bit cache: latency
        dict(name="store_step_s8", kind="store", tokens=37, kv_heads=8, head_dim=128, dtype="bf16", cache="s8", page=16, n_pages=40, skip=0.3, heads_first=False, fused=True),
        # a prefill wave's keys and values
        dict(name="store_prompt_bf16", kind="store", tokens=20001, kv_heads=8, head_dim=128, dtype="bf16", cache="bf16", page=32, n_pages=1000, skip=0.0, heads_first=True,
             fused=True),
    ]


def _log_int(rng, lo, hi):
    """An integer in [lo, hi], spread evenly over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))


def _heads(rng):
    kv = rng.choice([1, 2, 4, 8])
    return kv * rng.choice([1, 1, 3, 4, 7, 8]), kv


def draw(rng):
    kind = rng.choice(["linear"] * 6 + ["prompt"] * 6 + ["tree"] * 7 + ["plan"] * 2 + ["store"] * 3)
    dtype = rng.choice(["f16", "bf16"])
    if kind == "linear":
        K = 32 * _log_int(rng, 8, 512) if rng.random() < 0.8 else 8 * _log_int(rng, 20, 1000)
        N = _log_int(rng, 100, min(32768, 16384 * 8192 // K))
        return dict(kind="linear", M=_log_int(rng, 1, 64), N=N, K=K, group=rng.choice([32, 64, 128]), dtype=dtype, zeros=rng.random() < 0.5, bias=rng.random() < 0.3,
                    pad=rng.choice([0, 0, 8, 24]))
    if kind == "prompt":
        q_heads, kv_heads = _heads(rng)
        head_dim = rng.choice([64, 80, 96, 128, 128])
        n, longest = _log_int(rng, 1, 48), _log_int(rng, 8, 8192)
        budget = 1.2e12 / (4 * 128 * q_heads)                     # no more scores than the largest listed case
        lens = [_log_int(rng, 1, longest) for _ in range(n - 1)] + [longest]
        while sum(v * v for v in lens) / 2 > budget or n * longest * longest * q_heads > 6.4e9:
            lens = lens[n // 2:] if n > 1 else [longest // 2]
            n, longest = len(lens), lens[-1]
        return dict(kind="prompt", lens=_text(lens), q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, dtype=dtype, fused=rng.random() < 0.5)
    if kind == "tree":
        q_heads, kv_heads = _heads(rng)
        head_dim = rng.choice([64, 80, 128, 128])
        n, longest = _log_int(rng, 1, 64), _log_int(rng, 4, 16384)
        n = max(1, min(n, 32 * 16384 * 8 // (longest * max(kv_heads, q_heads // 4))))
        cached = [longest] + [rng.choice([0, rng.randrange(longest + 1), rng.randrange(longest + 1), longest]) for _ in range(n - 1)]
        most = rng.choice([1, 1, 8, 24, 64])
        drafts = [rng.randrange(1, most + 1) for _ in range(n)]
        while sum(drafts) * longest * q_heads > 32 * 16384 * 32 * 4:  # what the plain form's scores take
            drafts = [max(1, d // 2) for d in drafts]
            if max(drafts) == 1:
                break
        return dict(kind="tree", cached=_text(cached), drafts=_text(drafts), q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, dtype=dtype,
                    cache=rng.choice([dtype, dtype, "s8"]), page=rng.choice([16, 32, 64, 24, 1 + rng.randrange(100)]), heads_first=rng.random() < 0.5)
    if kind == "plan":
        n, page = _log_int(rng, 1, 3000), rng.choice([1, 16, 32, 64, 24, 128])
        fresh = _log_int(rng, 1, max(1, min(2000, 1000000 // n)))
        return dict(kind="plan", n=n, page=page, cached=_log_int(rng, 1, 4000), fresh=fresh, spare=rng.choice([-3, 0, 100]))
    tokens = _log_int(rng, 1, 20000)
    page = rng.choice([16, 32, 64, 24, 1 + rng.randrange(100)])
    return dict(kind="store", tokens=tokens, kv_heads=rng.choice([1, 2, 4, 8]), head_dim=rng.choice([64, 80, 128, 128]), dtype=dtype, cache=rng.choice([dtype, "s8"]), page=page,
                n_pages=tokens * 5 // (4 * page) + 2, skip=rng.choice([0.0, 0.0, 0.3]), heads_first=rng.random() < 0.5, fused=rng.random() < 0.5)


# ---- what a program holds before the call --------------------------------------------------------------------------------

def _normal(g, shape, dtype):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _starts(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return at


def _qkv(g, total, q_heads, kv_heads, head_dim, dtype, fused):
    """Queries, keys and values of `total` tokens, [token, head, element]: three tensors, or slices of one projection's output."""
    if fused:
        x = _normal(g, (total, q_heads + 2 * kv_heads, head_dim), dtype)
        return x[:, :q_heads], x[:, q_heads:q_heads + kv_heads], x[:, q_heads + kv_heads:]
    return tuple(_normal(g, (total, h, head_dim), dtype) for h in (q_heads, kv_heads, kv_heads))


def _cache(g, case, n_pages):
    """Keys and values [page, token, head, element] with whatever an earlier use left in them, and the scales of an 8-bit cache."""
    shape = [n_pages, case["page"], case["kv_heads"], case["head_dim"]]
    stored = [shape[i] for i in (0, 2, 1, 3)] if case["heads_first"] else shape
    kv, scales = [], []
    for _ in range(2):
        if case["cache"] == "s8":
            t = torch.randint(-127, 128, stored, generator=g, device="cuda", dtype=torch.int8)
            scales.append(0.01 + 0.01 * torch.rand(shape[:3], generator=g, device="cuda"))
        else:
            t = _normal(g, stored, _TYPES[case["cache"]])
            scales.append(None)
        kv.append(t.permute(0, 2, 1, 3) if case["heads_first"] else t)
    return kv + scales


def _cache_desc(hawq, case, k_cache):
    return hawq.CacheDesc(n_pages=k_cache.shape[0], page=case["page"], kv_heads=case["kv_heads"], head_dim=case["head_dim"], dtype=_hawq_type(hawq, case["cache"]),
                          page_stride=k_cache.stride(0), token_stride=k_cache.stride(1), head_stride=k_cache.stride(2))


def _hawq_type(hawq, name):
    return {"f16": hawq.F16, "bf16": hawq.BF16, "s8": hawq.S8}[name]


def _row_strides(**tensors):
    return {"%s_%s" % (n, w): t.stride(i) for n, t in tensors.items() for i, w in enumerate(("token", "head"))}


def _tree_masks(seed, drafts):
    """Bit j of a drafted token's mask: it descends from (or is) drafted token j of its own request."""
    r, out = random.Random(seed), []
    for n in drafts:
        seen = []
        for t in range(n):
            parent = r.randrange(-1, t) if t else -1
            if t and r.random() < 0.5:
                parent = t - 1
            seen.append((seen[parent] if parent >= 0 else 0) | 1 << t)
        out += [m - (1 << 64) if m >> 63 else m for m in seen]
    return torch.tensor(out, dtype=torch.int64, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = {"case": case, "kind": case["kind"]}
    if own:
        import paper_2011_10680_amd as hawq
        s["hawq"] = hawq
    globals()["_prepare_" + case["kind"]](case, int(seed), g, s)
    return s


def _prepare_linear(case, seed, g, s):
    M, N, K, dt = case["M"], case["N"], case["K"], _TYPES[case["dtype"]]
    groups = -(-K // case["group"])
    x = _normal(g, (M, K + case["pad"]), dt)
    x[:, ::97] *= 8                                               # the outlying channels of a language model's activations
    s["x"] = x[:, :K]
    s["w"] = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    s["scales"] = (0.002 + 0.008 * torch.rand((N, groups), generator=g, device="cuda")).to(dt)
    s["zeros"] = torch.randint(4, 12, (N, groups), generator=g, device="cuda", dtype=torch.uint8) if case["zeros"] else None
    s["bias"] = _normal(g, (N,), dt) if case["bias"] else None
    s["y"] = torch.empty((M, N), dtype=dt, device="cuda")
    if "hawq" in s:
        h = s["hawq"]
        s["desc"] = h.LinearW4Desc(M=M, N=N, K=K, group=case["group"], x_dtype=_hawq_type(h, case["dtype"]), w_dtype=h.U4 if case["zeros"] else h.S4,
                                   x_stride=s["x"].stride(0), y_stride=N)


def _prepare_prompt(case, seed, g, s):
    lens, dt = _ints(case["lens"]), _TYPES[case["dtype"]]
    total = sum(lens)
    s["q"], s["k"], s["v"] = _qkv(g, total, case["q_heads"], case["kv_heads"], case["head_dim"], dt, case["fused"])
    s["starts"], s["longest"], s["scale"] = _int32(_starts(lens)), max(lens), case["head_dim"] ** -0.5
    s["y"] = torch.empty((total, case["q_heads"], case["head_dim"]), dtype=dt, device="cuda")
    if "hawq" in s:
        h = s["hawq"]
        s["desc"] = h.AttnPromptDesc(n_seqs=len(lens), total=total, q_heads=case["q_heads"], kv_heads=case["kv_heads"], head_dim=case["head_dim"],
                                     dtype=_hawq_type(h, case["dtype"]), scale=s["scale"], **_row_strides(q=s["q"], k=s["k"], v=s["v"], y=s["y"]))


def _prepare_tree(case, seed, g, s):
    cached, drafts, dt, page = _ints(case["cached"]), _ints(case["drafts"]), _TYPES[case["dtype"]], case["page"]
    total = sum(drafts)
    s["q"], s["k"], s["v"] = _qkv(g, total, case["q_heads"], case["kv_heads"], case["head_dim"], dt, True)
    need = [-(-n // page) for n in cached]
    width, n_pages = max(need) + 1, sum(need) + 3
    s["k_cache"], s["v_cache"], s["k_scales"], s["v_scales"] = _cache(g, case, n_pages)
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    held = torch.arange(width, device="cuda")[None] < _int32(need)[:, None]
    at = (torch.cumsum(_int32(need), 0) - _int32(need))[:, None] + torch.arange(width, device="cuda")[None]
    s["table"] = torch.where(held, order[at.clamp(max=n_pages - 1)], -1).to(torch.int32).contiguous()
    s["cached"], s["starts"], s["mask"] = _int32(cached), _int32(_starts(drafts)), _tree_masks(seed, drafts)
    s["longest"], s["most"], s["scale"] = max(cached), max(drafts), case["head_dim"] ** -0.5
    s["y"] = torch.empty((total, case["q_heads"], case["head_dim"]), dtype=dt, device="cuda")
    if "hawq" in s:
        h = s["hawq"]
        s["desc"] = h.AttnTreeDesc(cache=_cache_desc(h, case, s["k_cache"]), n_seqs=len(drafts), total=total, max_drafts=s["most"], max_cached=s["longest"],
                                   q_heads=case["q_heads"], dtype=_hawq_type(h, case["dtype"]), table_stride=width, scale=s["scale"],
                                   **_row_strides(q=s["q"], k=s["k"], v=s["v"], y=s["y"]))
        s["workspace"] = torch.empty(h.hawq_attn_tree_workspace_bytes(s["desc"]), dtype=torch.uint8, device="cuda")


def _prepare_plan(case, seed, g, s):
    n, page = case["n"], case["page"]
    r = random.Random(seed)
    cached, fresh = [r.randrange(case["cached"] + 1) for _ in range(n)], [r.randrange(case["fresh"] + 1) for _ in range(n)]
    have, want = [-(-c // page) for c in cached], [-(-(c + f) // page) for c, f in zip(cached, fresh)]
    n_free = max(1, sum(want) - sum(have) + case["spare"])
    order = torch.randperm(n_free + sum(have), generator=g, device="cuda").to(torch.int32)
    s["free"] = order[sum(have):].contiguous()
    width = -(-(case["cached"] + case["fresh"]) // page)
    at = torch.arange(width, device="cuda")[None]
    first = torch.cumsum(_int32(have), 0) - _int32(have)
    s["table"] = torch.where(at < _int32(have)[:, None], order[(first[:, None] + at).clamp(max=order.numel() - 1)], -1).to(torch.int32).contiguous()
    s["cached"], s["fresh"], s["page"] = _int32(cached), _int32(fresh), page
    s["n_slots"] = n * case["fresh"]
    s["starts"] = torch.empty(n + 1, dtype=torch.int32, device="cuda")
    s["slots"] = torch.empty(s["n_slots"], dtype=torch.int64, device="cuda")
    s["counts"] = torch.empty(2, dtype=torch.int32, device="cuda")


def _prepare_store(case, seed, g, s):
    total, dt = case["tokens"], _TYPES[case["dtype"]]
    _, s["k"], s["v"] = _qkv(g, total, 2 * case["kv_heads"], case["kv_heads"], case["head_dim"], dt, case["fused"])
    s["k_cache"], s["v_cache"], s["k_scales"], s["v_scales"] = _cache(g, case, case["n_pages"])
    slots = torch.randperm(case["n_pages"] * case["page"], generator=g, device="cuda")[:total]
    skipped = torch.rand(total, generator=g, device="cuda") < case["skip"]
    s["slots"] = torch.where(skipped, -1, slots)
    if "hawq" in s:
        h = s["hawq"]
        s["desc"] = h.CacheStoreDesc(cache=_cache_desc(h, case, s["k_cache"]), total=total, dtype=_hawq_type(h, case["dtype"]), **_row_strides(k=s["k"], v=s["v"]))


# ---- one pass ------------------------------------------------------------------------------------------------------------

def run(s):
    return globals()[("_own_" if own else "_plain_") + s["kind"]](s)


def _own_linear(s):
    s["hawq"].hawq_linear_w4(s["desc"], s["x"], s["w"], s["scales"], s["zeros"], s["bias"], s["y"])
    return s["y"]


def _own_prompt(s):
    s["hawq"].hawq_attn_prompt(s["desc"], s["q"], s["k"], s["v"], s["starts"], s["y"])
    return s["y"]


def _own_tree(s):
    s["hawq"].hawq_attn_tree(s["desc"], s["q"], s["k"], s["v"], s["starts"], s["mask"], s["k_cache"], s["v_cache"], s["k_scales"], s["v_scales"], s["table"], s["cached"],
                             s["y"], s["workspace"])
    return s["y"]


def _own_plan(s):
    s["hawq"].hawq_cache_plan(s["cached"], s["fresh"], s["page"], s["free"], s["table"], s["starts"], s["slots"], s["counts"])
    return {"table": s["table"], "starts": s["starts"], "slots": s["slots"], "counts": s["counts"]}


def _own_store(s):
    s["hawq"].hawq_cache_store(s["desc"], s["k"], s["v"], s["slots"], s["k_cache"], s["v_cache"], s["k_scales"], s["v_scales"])
    return _held(s)


def _held(s):
    """The cache's contents: an 8-bit cache's as the values they stand for."""
    if s["k_scales"] is None:
        return {"k": s["k_cache"], "v": s["v_cache"]}
    return {"k": s["k_cache"] * s["k_scales"][..., None], "v": s["v_cache"] * s["v_scales"][..., None]}


def _weights(s, dtype):
    """The 4-bit weights as the numbers they stand for, [N, K]."""
    c = s["case"]
    q = torch.stack((s["w"] & 15, s["w"] >> 4), dim=2).reshape(c["N"], c["K"]).to(dtype)
    spread = lambda t: t.to(dtype).repeat_interleave(c["group"], dim=1)[:, :c["K"]]  # noqa: E731
    q = torch.where(q >= 8, q - 16, q) if s["zeros"] is None else q - spread(s["zeros"])
    return q * spread(s["scales"])


def _plain_linear(s):
    y = s["x"].float() @ _weights(s, torch.float32).t()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    return y.to(s["x"].dtype)


def _softmax(scores, seen):
    """Over the last axis and what is seen of it; zeros where nothing is."""
    scores = scores.masked_fill(~seen, -math.inf)
    top = scores.amax(dim=-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(scores - top)
    return p / p.sum(dim=-1, keepdim=True).clamp(min=1e-38)


def _padded(x, starts, longest):
    """Packed rows [total, ...] as [sequence, longest, ...] in 32 bits; what lies past a sequence's end is some other row."""
    at = starts[:-1, None].long() + torch.arange(longest, device=x.device)[None]
    return x[at.clamp(max=x.shape[0] - 1)].float()


def _packed(y, starts, total):
    """The rows of [sequence, longest, ...] that are a sequence's own, one behind the other."""
    t = torch.arange(total, device=y.device)
    b = torch.searchsorted(starts[1:].long(), t, right=True)
    return y[b, t - starts.long()[b]]


def _grouped(q, kv_heads):
    """[sequence, row, q_heads, D] -> [sequence, kv_heads, heads of a group * rows, D]"""
    b, n, h, d = q.shape
    return q.reshape(b, n, kv_heads, h // kv_heads, d).permute(0, 2, 3, 1, 4).reshape(b, kv_heads, h // kv_heads * n, d)


def _ungrouped(y, n):
    b, kv, rows, d = y.shape
    return y.reshape(b, kv, rows // n, n, d).permute(0, 3, 1, 2, 4).reshape(b, n, kv * (rows // n), d)


def _plain_prompt(s):
    n, kv = s["longest"], s["case"]["kv_heads"]
    q, k, v = (_padded(s[x], s["starts"], n) for x in "qkv")
    scores = torch.matmul(_grouped(q, kv), k.permute(0, 2, 3, 1).contiguous()) * s["scale"]
    at = torch.arange(n, device=q.device)
    seen = (at[None] <= at[:, None]).repeat(scores.shape[2] // n, 1)
    y = torch.matmul(_softmax(scores, seen), v.permute(0, 2, 1, 3).contiguous())
    return _packed(_ungrouped(y, n), s["starts"], s["q"].shape[0]).to(s["q"].dtype)


def _plain_tree(s):
    n, L, kv, page = s["most"], s["longest"], s["case"]["kv_heads"], s["case"]["page"]
    at = torch.arange(L, device=s["q"].device)
    pages, within = s["table"].long().clamp(min=0)[:, at // page], (at % page)[None]
    old = [s[c][pages, within].float() if s[f] is None else s[c][pages, within].float() * s[f][pages, within][..., None]
           for c, f in (("k_cache", "k_scales"), ("v_cache", "v_scales"))]
    q, k, v = (_padded(s[x], s["starts"], n) for x in "qkv")
    k, v = torch.cat((old[0], k), dim=1), torch.cat((old[1], v), dim=1)
    scores = torch.matmul(_grouped(q, kv), k.permute(0, 2, 3, 1).contiguous()) * s["scale"]
    first = s["starts"].long()
    rows = (first[:-1, None] + torch.arange(n, device=q.device)[None]).clamp(max=s["q"].shape[0] - 1)
    tree = (s["mask"][rows][:, :, None] >> torch.arange(n, device=q.device)) & 1
    tree = (tree == 1) & (torch.arange(n, device=q.device) < (first[1:] - first[:-1])[:, None])[:, None]
    seen = torch.cat(((at < s["cached"][:, None])[:, None].expand(-1, n, -1), tree), dim=2)
    y = torch.matmul(_softmax(scores, seen.repeat(1, scores.shape[2] // n, 1)[:, None]), v.permute(0, 2, 1, 3).contiguous())
    return _packed(_ungrouped(y, n), s["starts"], s["q"].shape[0]).to(s["q"].dtype)


def _plain_plan(s):
    cached, fresh, free, page, width = s["cached"].long(), s["fresh"].long(), s["free"], s["page"], s["table"].shape[1]
    ends = torch.cumsum(fresh, 0)
    starts = torch.cat((ends.new_zeros(1), ends))
    have = (cached + page - 1) // page
    want = ((cached + fresh + page - 1) // page).clamp(max=width)
    taken = torch.cumsum((want - have).clamp(min=0), 0)
    p = torch.arange(width, device=free.device)[None]
    i = (taken - (want - have).clamp(min=0))[:, None] + p - have[:, None]
    given = torch.where(i < free.numel(), free[i.clamp(0, free.numel() - 1)], -1)
    table = torch.where((p >= have[:, None]) & (p < want[:, None]), given, s["table"]).to(torch.int32)
    t = torch.arange(s["n_slots"], device=free.device)
    b = torch.searchsorted(ends, t, right=True).clamp(max=cached.numel() - 1)
    at = cached[b] + t - starts[b]
    held = table[b, (at // page).clamp(max=width - 1)].long()
    slots = torch.where((t < ends[-1]) & (at // page < width) & (held >= 0), held * page + at % page, -1)
    return {"table": table, "starts": starts.to(torch.int32), "slots": slots, "counts": torch.stack((ends[-1], taken[-1])).to(torch.int32)}


def _plain_store(s):
    page, kept = s["case"]["page"], s["slots"] >= 0
    at = s["slots"][kept]
    for x, cache, scales in (("k", "k_cache", "k_scales"), ("v", "v_cache", "v_scales")):
        rows = s[x][kept].float()
        if s[scales] is not None:
            scale = rows.abs().amax(dim=-1) / 127
            s[scales][at // page, at % page] = scale
            rows = torch.where(scale[..., None] > 0, torch.round(rows / scale[..., None]), 0.0)
        s[cache][at // page, at % page] = rows.to(s[cache].dtype)
    return _held(s)


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------

def exact(case, seed):
    f = globals().get("_exact_" + case["kind"])
    if f is None:
        return None                                               # whole numbers: the plain form is exact
    s = {"case": case}
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    globals()["_prepare_" + case["kind"]](case, int(seed), g, s)
    return f(case, s)


def _exact_linear(case, s):
    x, codes, y = s["x"].double(), s["w"].to(torch.int64), torch.zeros((case["M"], case["N"]), dtype=torch.float64, device="cuda")
    for k0 in range(0, case["K"], case["group"]):
        k1, i = min(case["K"], k0 + case["group"]), k0 // case["group"]
        part = codes[:, k0 // 2:k1 // 2]
        even, odd = part % 16, part // 16
        if s["zeros"] is None:
            even, odd = (even + 8) % 16 - 8, (odd + 8) % 16 - 8
        else:
            even, odd = even - s["zeros"][:, i:i + 1].long(), odd - s["zeros"][:, i:i + 1].long()
        group = x[:, k0:k1:2] @ even.double().t() + x[:, k0 + 1:k1:2] @ odd.double().t()
        y += group * s["scales"][:, i].double()
    return y if s["bias"] is None else y + s["bias"].double()


def _attend(q, k, v, seen, scale):
    """One head: rows that see nothing are zeros."""
    e = (q @ k.t()) * scale
    e = torch.where(seen, e, torch.full_like(e, -math.inf))
    m = e.max(dim=1, keepdim=True).values
    p = torch.where(seen, torch.exp(e - torch.where(torch.isinf(m), torch.zeros_like(m), m)), torch.zeros_like(e))
    total = p.sum(dim=1, keepdim=True)
    return (p @ v) / torch.where(total > 0, total, torch.ones_like(total))


def _exact_prompt(case, s):
    q, k, v = (s[x].double() for x in "qkv")
    y, ratio, t0 = torch.empty_like(q), case["q_heads"] // case["kv_heads"], 0
    for n in _ints(case["lens"]):
        seen = torch.ones((n, n), dtype=torch.bool, device="cuda").tril()
        for h in range(case["q_heads"]):
            y[t0:t0 + n, h] = _attend(q[t0:t0 + n, h], k[t0:t0 + n, h // ratio], v[t0:t0 + n, h // ratio], seen, s["scale"])
        t0 += n
    return y


def _exact_tree(case, s):
    q, k, v = (s[x].double() for x in "qkv")
    y, ratio, t0, page = torch.empty_like(q), case["q_heads"] // case["kv_heads"], 0, case["page"]
    masks = s["mask"].tolist()
    for b, (length, n) in enumerate(zip(_ints(case["cached"]), _ints(case["drafts"]))):
        at = s["table"][b, :-(-length // page)].long()
        past = []
        for c, f in ((s["k_cache"], s["k_scales"]), (s["v_cache"], s["v_scales"])):
            rows = c[at].double()
            rows = rows if f is None else rows * f[at].double().unsqueeze(-1)
            past.append(rows.reshape(-1, case["kv_heads"], case["head_dim"])[:length])
        tree = torch.tensor([[masks[t0 + i] >> j & 1 for j in range(n)] for i in range(n)], device="cuda").bool()
        seen = torch.cat((torch.ones((n, length), dtype=torch.bool, device="cuda"), tree), dim=1)
        for h in range(case["q_heads"]):
            kv = h // ratio
            y[t0:t0 + n, h] = _attend(q[t0:t0 + n, h], torch.cat((past[0][:, kv], k[t0:t0 + n, kv])), torch.cat((past[1][:, kv], v[t0:t0 + n, kv])), seen, s["scale"])
        t0 += n
    return y


def _exact_store(case, s):
    out, page = {}, case["page"]
    kept = [(t, p) for t, p in enumerate(s["slots"].tolist()) if p >= 0]
    rows = torch.tensor([t for t, _ in kept], dtype=torch.long, device="cuda")
    at = torch.tensor([p for _, p in kept], dtype=torch.long, device="cuda")
    for x in "kv":
        c, f = s[x + "_cache"].double(), s[x + "_scales"]
        new = s[x][rows].double()
        if f is not None:
            c = c * f.double().unsqueeze(-1)
            step = new.abs().max(dim=-1, keepdim=True).values / 127
            new = torch.where(step > 0, torch.round(new / step) * step, new)
        c[torch.div(at, page, rounding_mode="floor"), at % page] = new
        out[x] = c
    return out


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        groups = -(-K // case["group"])
        return {"bytes": N * K // 2 + N * groups * (3 if case["zeros"] else 2) + 2 * M * (K + N) + (2 * N if case["bias"] else 0), "flops": 2 * M * N * K}
    if kind == "prompt":
        lens, D = _ints(case["lens"]), case["head_dim"]
        return {"bytes": 2 * sum(lens) * 2 * (case["q_heads"] + case["kv_heads"]) * D, "flops": 2 * D * case["q_heads"] * sum(n * (n + 1) for n in lens)}
    if kind == "tree":
        cached, drafts, D = _ints(case["cached"]), _ints(case["drafts"]), case["head_dim"]
        row = case["kv_heads"] * (D + 4 if case["cache"] == "s8" else 2 * D)
        return {"bytes": 2 * sum(cached) * row + sum(drafts) * (2 * 2 * D * (case["q_heads"] + case["kv_heads"]) + 8) + 4 * sum(-(-n // case["page"]) for n in cached),
                "flops": 4 * D * case["q_heads"] * sum(n * (length + (n + 1) / 2) for length, n in zip(cached, drafts))}
    if kind == "plan":
        n, fresh = case["n"], case["fresh"] * case["n"]
        return {"bytes": 12 * n + 8 * fresh + 8 * fresh // 2 // case["page"], "flops": 0}
    row = case["tokens"] * (1 - case["skip"]) * case["kv_heads"]
    return {"bytes": 8 * case["tokens"] + 2 * row * (case["head_dim"] * (3 if case["cache"] == "s8" else 4) + (4 if case["cache"] == "s8" else 0)), "flops": 0}

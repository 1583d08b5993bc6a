"""What a decoder's step needs beside its attention, cache and linear layers, as measurable cases.

A case is a dict of plain values.  `listed()` gives the fixed ones, `draw(rng)` one more of the same ranges; `prepare` makes what a
program holds before the call on the GPU, `run` is one pass: with `own` through the framework's entry points, without it in plain
torch operations in 32 bits.  `exact` is the definition in 64 bits, `work` the bytes and operations a pass cannot do without.

Kinds of case
  rotary     queries and keys of a batch of tokens turned by their positions (`hawq_rotary`)
  gated      both projections of a gated feed-forward block from 4-bit weights, the activation and the product (`hawq_gated_w4`)
  adapters   low-rank additions to a projection's output, another one for each row (`hawq_adapters`)
  logits     penalties for tokens that occurred, biases and grammar masks (`hawq_logits`)
Lists of numbers are texts of integers joined by commas.
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


def listed():
    return [
        # one user's next token, a small model: a pure latency measurement
        dict(name="rotary_one_f16", kind="rotary", tokens=1, q_heads=8, kv_heads=1, head_dim=64, rotary_dim=64, layout="halves", dtype="f16", far=611, factor=1, fused=True),
        # the drafts of a server's step in long contexts: a part of the head turned, neighbouring elements, frequencies scaled
        dict(name="rotary_part_bf16", kind="rotary", tokens=777, q_heads=32, kv_heads=8, head_dim=80, rotary_dim=32, layout="pairs", dtype="bf16", far=1000000, factor=8, fused=False),
        # a prefill wave, queries and keys as slices of one projection's output: bound by bytes
        dict(name="rotary_prompt_bf16", kind="rotary", tokens=20001, q_heads=32, kv_heads=8, head_dim=128, rotary_dim=128, layout="halves", dtype="bf16", far=8192, factor=1,
             fused=True),
        # one token through a small model's block: latency
        dict(name="gated_1x512x256_f16", kind="gated", M=1, N=512, K=256, group=64, dtype="f16", zeros=False, bias=False, activation="silu", pad=0),
        # the thirteen tokens of a small draft tree through a wide block: bound by the weights' bytes
        dict(name="gated_13x12288x4096_bf16", kind="gated", M=13, N=12288, K=4096, group=64, dtype="bf16", zeros=True, bias=False, activation="gelu", pad=8),
        # a prompt of two thousand tokens: the matrix rate
        dict(name="gated_2049x8192x4096_bf16", kind="gated", M=2049, N=8192, K=4096, group=128, dtype="bf16", zeros=True, bias=False, activation="silu", pad=0),
        # one request with an adapter of its own, a small model: latency
        dict(name="adapters_one_f16", kind="adapters", M=1, N=768, K=256, ranks="8,16,4,8", runs="2", dtype="f16", pad=0),
        # a step of 48 requests over twelve adapters and the plain model, in no order: bound by the adapters' bytes
        dict(name="adapters_step_bf16", kind="adapters", M=48, N=6144, K=4096, ranks="16,8,64,16,32,16,8,64,16,24,16,5", runs="mixed", dtype="bf16", pad=0),
        # prompts of seven requests packed one behind the other, one of them without an adapter
        dict(name="adapters_prompt_bf16", kind="adapters", M=5003, N=4096, K=4096, ranks="64,16,32,64", runs="0,2,1,-1,3,0,1", dtype="bf16", pad=64),
        # one user's next token: latency
        dict(name="logits_one_f16", kind="logits", drafts="1", vocab=32000, past="700", dtype="f16", biases=4, masks=1, pad=0),
        # draft trees of eight requests, some under a grammar, at most a few hundred tokens written
        dict(name="logits_drafts_bf16", kind="logits", drafts="13,25,1,8,40,13,64,7", vocab=64000, past="350,12,0,801,77,3000,5,9000", dtype="bf16", biases=50, masks=60, pad=64),
        # a large batch, one token each, an odd vocabulary, half of the requests under a grammar: bound by the logits' bytes
        dict(name="logits_batch_bf16", kind="logits", drafts=_text([1] * 256), vocab=128001, past=_text([16 * i for i in range(256)]), dtype="bf16", biases=20, masks=128, pad=0),
    ]


def _log_int(rng, lo, hi):
    """An integer in [lo, hi], spread evenly over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))


def draw(rng):
    kind = rng.choice(["rotary"] * 5 + ["gated"] * 7 + ["adapters"] * 6 + ["logits"] * 6)
    dtype = rng.choice(["f16", "bf16"])
    if kind == "rotary":
        kv, head_dim = rng.choice([1, 2, 4, 8]), rng.choice([64, 80, 96, 128, 128])
        return dict(kind="rotary", tokens=_log_int(rng, 1, 20000), q_heads=kv * rng.choice([1, 1, 2, 3, 4]), kv_heads=kv, head_dim=head_dim,
                    rotary_dim=rng.choice([head_dim, head_dim, head_dim // 2, 32, 20]), layout=rng.choice(["halves", "pairs"]), dtype=dtype, far=_log_int(rng, 100, 1000000),
                    factor=rng.choice([1, 1, 4, 32]), fused=rng.random() < 0.5)
    if kind == "gated":
        K = 32 * _log_int(rng, 4, 256) if rng.random() < 0.8 else 8 * _log_int(rng, 20, 1000)
        M = _log_int(rng, 1, 2049)
        N = _log_int(rng, 50, min(16384, 12288 * 4096 // K, 2049 * 8192 * 4096 // (M * K)))
        return dict(kind="gated", M=M, N=N, K=K, group=rng.choice([32, 64, 128]), dtype=dtype, zeros=rng.random() < 0.5, bias=rng.random() < 0.3,
                    activation=rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu"]), pad=rng.choice([0, 0, 8, 24]))
    if kind == "adapters":
        n, most = _log_int(rng, 1, 16), rng.choice([8, 16, 32, 64])
        M = _log_int(rng, 1, 5003)
        K, N = 8 * _log_int(rng, 8, 1024), 8 * _log_int(rng, 8, min(2048, 5003 * 512 // M)) - rng.choice([0, 0, 0, 3])
        runs = "mixed" if M <= 128 and rng.random() < 0.7 else _text([rng.randrange(-1, n) for _ in range(min(M, _log_int(rng, 1, 12)))])
        return dict(kind="adapters", M=M, N=N, K=K if M * K <= 5003 * 4096 else 4096, ranks=_text([rng.choice([most, most, 1 + rng.randrange(most)]) for _ in range(n)]),
                    runs=runs, dtype=dtype, pad=rng.choice([0, 0, 8, 64]))
    vocab = _log_int(rng, 1000, 128001) if rng.random() < 0.5 else 256 * _log_int(rng, 4, 500)
    n = _log_int(rng, 1, 256)
    most = rng.choice([1, 1, 8, 24])
    drafts = [rng.randrange(1, most + 1) for _ in range(n)]
    while sum(drafts) * vocab > 256 * 128001 * 3 // 4 and len(drafts) > 1:
        drafts = drafts[len(drafts) // 2:]
    longest = _log_int(rng, 1, 8000)
    return dict(kind="logits", drafts=_text(drafts), vocab=vocab, past=_text([rng.randrange(longest + 1) for _ in drafts]), dtype=dtype, biases=rng.choice([0, 5, 50]),
                masks=rng.choice([0, 0, 1, max(1, sum(drafts) // 2)]), pad=rng.choice([0, 0, 64, 3]))


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


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = {"case": case, "kind": case["kind"]}
    if own:
        import paper_2011_10680_amd as hawq
        s["hawq"] = hawq
        s["type"] = hawq.F16 if case["dtype"] == "f16" else hawq.BF16
    globals()["_prepare_" + case["kind"]](case, int(seed), g, s)
    return s


def _turns(case):
    """Revolutions a token, of every pair: frequencies that turn slower than once in the original context are divided by the factor, those that
    turn often stay, in between a mixture."""
    n, base, context = case["rotary_dim"] // 2, 10000.0, 8192.0
    f = [base ** (-i / n) / (2 * math.pi) for i in range(n)]
    share = [min(1.0, max(0.0, (v * context - 1) / 31)) for v in f]
    return [v * (m + (1 - m) / case["factor"]) for v, m in zip(f, share)]


def _prepare_rotary(case, seed, g, s):
    T, H, KV, D, dt = case["tokens"], case["q_heads"], case["kv_heads"], case["head_dim"], _TYPES[case["dtype"]]
    if case["fused"]:
        x = _normal(g, (T, H + 2 * KV, D), dt)
        s["q"], s["k"] = x[:, :H], x[:, H:H + KV]
    else:
        s["q"], s["k"] = _normal(g, (T, H, D), dt), _normal(g, (T, KV, D), dt)
    # several requests' tokens, each behind the other
    first = torch.randint(0, case["far"], (T,), generator=g, device="cuda")
    s["positions"] = (first[torch.arange(T, device="cuda") // 500 * 500] + torch.arange(T, device="cuda") % 500).to(torch.int32)
    s["turns"] = torch.tensor(_turns(case), dtype=torch.float64, device="cuda")
    s["scale"] = 1.0 if case["factor"] == 1 else 0.1 * math.log(case["factor"]) + 1.0
    s["yq"], s["yk"] = (torch.empty((T, h, D), dtype=dt, device="cuda") for h in (H, KV))
    if "hawq" in s:
        h = s["hawq"]
        s["desc"] = h.RotaryDesc(total=T, q_heads=H, kv_heads=KV, head_dim=D, rotary_dim=case["rotary_dim"], layout=h.ROTARY_HALVES if case["layout"] == "halves" else h.ROTARY_PAIRS,
                                 dtype=s["type"], scale=s["scale"],
                                 **{"%s_%s" % (n, w): s[n].stride(i) for n in ("q", "k", "yq", "yk") for i, w in enumerate(("token", "head"))})


def _prepare_gated(case, seed, g, s):
    M, N, K, dt = case["M"], case["N"], case["K"], _TYPES[case["dtype"]]
    groups = -(-K // case["group"])
    x = _normal(g, (M, K + case["pad"]), dt)
    x[:, ::97] *= 8                                               # the outlying channels of a language model's activations
    s["x"] = x[:, :K]
    s["w"] = torch.randint(0, 256, (2 * N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    size = (8 / K) ** 0.5 / 5                                     # projections of a few units
    s["scales"] = (size * (0.2 + 0.8 * torch.rand((2 * N, groups), generator=g, device="cuda"))).to(dt)
    s["zeros"] = torch.randint(4, 12, (2 * N, groups), generator=g, device="cuda", dtype=torch.uint8) if case["zeros"] else None
    s["bias"] = _normal(g, (2 * N,), dt) if case["bias"] else None
    s["y"] = torch.empty((M, N), dtype=dt, device="cuda")
    if "hawq" in s:
        h = s["hawq"]
        s["desc"] = h.GatedW4Desc(M=M, N=N, K=K, group=case["group"], x_dtype=s["type"], w_dtype=h.U4 if case["zeros"] else h.S4,
                                  activation={"silu": h.SILU, "gelu": h.GELU, "gelu_tanh": h.GELU_TANH, "relu": h.RELU}[case["activation"]], x_stride=s["x"].stride(0), y_stride=N)
        s["workspace"] = torch.empty(h.hawq_gated_w4_workspace_bytes(s["desc"]), dtype=torch.uint8, device="cuda")


def _prepare_adapters(case, seed, g, s):
    M, N, K, dt, ranks = case["M"], case["N"], case["K"], _TYPES[case["dtype"]], _ints(case["ranks"])
    n, most, r = len(ranks), max(ranks), random.Random(seed)
    s["x"] = _normal(g, (M, K + case["pad"]), dt)[:, :K]
    s["base"] = _normal(g, (M, N), dt)
    s["a"], s["b"] = _normal(g, (n, most, K), dt) * K ** -0.5, _normal(g, (n, N, most), dt)
    s["ranks"] = _int32(ranks)
    s["scales"] = torch.tensor([0.25 + r.random() for _ in ranks], dtype=torch.float32, device="cuda")
    if case["runs"] == "mixed":
        rows = [r.randrange(-1, n) for _ in range(M)]
    else:
        runs = _ints(case["runs"])
        ends = sorted(r.sample(range(1, M), len(runs) - 1)) + [M]
        rows = [a for a, begin, end in zip(runs, [0] + ends, ends) for _ in range(end - begin)]
    s["adapter"] = _int32(rows)
    s["y"] = torch.empty((M, N), dtype=dt, device="cuda")
    if "hawq" in s:
        h = s["hawq"]
        s["desc"] = h.AdaptersDesc(M=M, N=N, K=K, n_adapters=n, max_rank=most, dtype=s["type"], x_stride=s["x"].stride(0), base_stride=N, y_stride=N,
                                   a_adapter=s["a"].stride(0), a_row=s["a"].stride(1), b_adapter=s["b"].stride(0), b_row=s["b"].stride(1))
        s["workspace"] = torch.empty(h.hawq_adapters_workspace_bytes(s["desc"]), dtype=torch.uint8, device="cuda")


def _prepare_logits(case, seed, g, s):
    drafts, past, V, dt, r = _ints(case["drafts"]), _ints(case["past"]), case["vocab"], _TYPES[case["dtype"]], random.Random(seed)
    n, total = len(drafts), sum(drafts)
    words = lambda shape: (V * torch.rand(shape, generator=g, device="cuda") ** 3).to(torch.int32).clamp(max=V - 1)  # noqa: E731  (few words often)
    s["logits"] = (_normal(g, (total, V + case["pad"]), torch.float32) * 3).to(dt)[:, :V]
    s["past"], s["past_lens"] = words((n, max(past) + 64)), _int32(past)
    s["prompt_lens"] = _int32([v // 3 for v in past])
    s["starts"], s["drafts"] = _int32(_starts(drafts)), words((total,))
    masks = []
    for count in drafts:                                          # a tree of drafts: every token's ancestors and itself
        seen = []
        for t in range(count):
            parent = r.randrange(-1, t) if t and r.random() < 0.5 else t - 1
            seen.append((seen[parent] if parent >= 0 else 0) | 1 << t)
        masks += [m - (1 << 64) if m >> 63 else m for m in seen]
    s["mask"], s["most"] = torch.tensor(masks, dtype=torch.int64, device="cuda"), max(drafts)
    s["penalties"] = torch.tensor([[r.choice([1.0, 1.1, 1.3]), r.choice([0.0, 0.5]), r.choice([0.0, 0.25])] for _ in drafts], dtype=torch.float32, device="cuda")
    counts = [r.randrange(case["biases"] + 1) for _ in drafts]
    s["bias_starts"] = _int32(_starts(counts))
    s["bias_ids"] = _int32([i for count in counts for i in r.sample(range(V), count)])
    s["bias_values"] = torch.tensor([r.uniform(-10, 10) for _ in range(sum(counts))], dtype=torch.float32, device="cuda")
    W = -(-V // 32)
    s["allowed"] = torch.randint(-2 ** 31, 2 ** 31, (case["masks"], W), generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
    s["allowed"][::2, W // 8:] = 0                                # half of the grammars allow a small part of the vocabulary
    rows = list(range(case["masks"])) + [-1] * max(0, total - case["masks"])
    r.shuffle(rows)
    s["allowed_row"] = _int32(rows[:total])
    s["y"] = torch.empty((total, V), dtype=dt, device="cuda")
    if "hawq" in s:
        h = s["hawq"]
        s["desc"] = h.LogitsDesc(n_seqs=n, total=total, vocab=V, dtype=s["type"], past_stride=s["past"].stride(0), n_bias=sum(counts), n_allowed=case["masks"],
                                 allowed_stride=W, x_stride=s["logits"].stride(0), y_stride=V)


# ---- one pass ------------------------------------------------------------------------------------------------------------

def run(s):
    return globals()[("_own_" if own else "_plain_") + s["kind"]](s)


def _own_rotary(s):
    s["hawq"].hawq_rotary(s["desc"], s["q"], s["k"], s["positions"], s["turns"], s["yq"], s["yk"])
    return {"q": s["yq"], "k": s["yk"]}


def _own_gated(s):
    s["hawq"].hawq_gated_w4(s["desc"], s["x"], s["w"], s["scales"], s["zeros"], s["bias"], s["y"], s["workspace"])
    return s["y"]


def _own_adapters(s):
    s["hawq"].hawq_adapters(s["desc"], s["x"], s["a"], s["b"], s["ranks"], s["scales"], s["adapter"], s["base"], s["y"], s["workspace"])
    return s["y"]


def _own_logits(s):
    s["hawq"].hawq_logits(s["desc"], s["logits"], s["past"], s["past_lens"], s["prompt_lens"], s["starts"], s["drafts"], s["mask"], s["penalties"], s["bias_starts"],
                          s["bias_ids"], s["bias_values"], s["allowed"], s["allowed_row"], s["y"])
    return s["y"]


def _plain_rotary(s):
    R, scale = s["case"]["rotary_dim"], s["scale"]
    revolutions = s["positions"].double()[:, None] * s["turns"]                   # far positions: the angle in 64 bits
    angle = (revolutions - torch.floor(revolutions)) * (2 * math.pi)
    cos, sin = (torch.cos(angle) * scale).float()[:, None], (torch.sin(angle) * scale).float()[:, None]
    out = {}
    for name in "qk":
        x = s[name].float()
        if s["case"]["layout"] == "halves":
            a, b = x[..., :R // 2], x[..., R // 2:R]
            turned = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)
        else:
            a, b = x[..., 0:R:2], x[..., 1:R:2]
            turned = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=-1).flatten(-2)
        out[name] = torch.cat((turned, x[..., R:]), dim=-1).to(s[name].dtype)
    return out


def _weights(s):
    """The 4-bit weights as the numbers they stand for, [2 N, K]."""
    c = s["case"]
    q = torch.stack((s["w"] & 15, s["w"] >> 4), dim=2).reshape(2 * c["N"], c["K"]).float()
    spread = lambda t: t.float().repeat_interleave(c["group"], dim=1)[:, :c["K"]]  # noqa: E731
    q = torch.where(q >= 8, q - 16, q) if s["zeros"] is None else q - spread(s["zeros"])
    return q * spread(s["scales"])


def _activated(v, kind):
    if kind == "silu":
        return v / (1 + torch.exp(-v))
    if kind == "gelu":
        return 0.5 * v * (1 + torch.erf(v * 0.5 ** 0.5))
    if kind == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh((2 / math.pi) ** 0.5 * (v + 0.044715 * v * v * v)))
    return v.clamp(min=0)


def _plain_gated(s):
    both = s["x"].float() @ _weights(s).t()
    if s["bias"] is not None:
        both = both + s["bias"].float()
    gate, up = both[:, :s["case"]["N"]], both[:, s["case"]["N"]:]
    return (_activated(gate, s["case"]["activation"]) * up).to(s["x"].dtype)


def _plain_adapters(s):
    x, y = s["x"].float(), s["base"].float()
    at = torch.arange(s["a"].shape[1], device="cuda")
    for i in range(s["a"].shape[0]):
        h = (x @ s["a"][i].float().t()) * (at < s["ranks"][i])
        y = y + torch.where((s["adapter"] == i)[:, None], (h @ s["b"][i].float().t()) * s["scales"][i], 0.0)
    return y.to(s["x"].dtype)


def _plain_logits(s):
    V, total = s["case"]["vocab"], s["logits"].shape[0]
    n, longest = s["past"].shape
    at = torch.arange(longest, device="cuda")[None]
    ids = s["past"].long()
    held, written = at < s["past_lens"][:, None], (at < s["past_lens"][:, None]) & (at >= s["prompt_lens"][:, None])
    b = torch.searchsorted(s["starts"][1:].long(), torch.arange(total, device="cuda"), right=True)
    seen = torch.zeros((n, V), dtype=torch.float32, device="cuda").scatter_add_(1, ids, held.float())[b]
    count = torch.zeros((n, V), dtype=torch.float32, device="cuda").scatter_add_(1, ids, written.float())[b]
    j = torch.arange(s["most"], device="cuda")[None]
    first, size = s["starts"].long()[b][:, None], (s["starts"][1:] - s["starts"][:-1]).long()[b][:, None]
    ancestor = ((s["mask"][:, None] >> j & 1) == 1) & (j < size)
    tokens = s["drafts"].long()[(first + j).clamp(max=total - 1)]
    seen, count = seen.scatter_add_(1, tokens, ancestor.float()), count.scatter_add_(1, tokens, ancestor.float())
    x = s["logits"].float()
    r, presence, frequency = (s["penalties"][b, i][:, None] for i in range(3))
    x = torch.where(seen > 0, torch.where(x > 0, x / r, x * r), x)
    x = x - frequency * count - torch.where(count > 0, presence, 0.0)
    m = s["bias_ids"].numel()
    if m:
        request = torch.searchsorted(s["bias_starts"][1:].long(), torch.arange(m, device="cuda"), right=True)
        x = x + torch.zeros((n, V), dtype=torch.float32, device="cuda").index_put_((request, s["bias_ids"].long()), s["bias_values"], accumulate=True)[b]
    if s["allowed"].shape[0]:
        token = torch.arange(V, device="cuda")
        word = s["allowed"][s["allowed_row"].long().clamp(min=0)][:, token // 32]
        x = torch.where(((word >> (token % 32) & 1) == 1) | (s["allowed_row"] < 0)[:, None], x, -math.inf)
    return x.to(s["logits"].dtype)


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------

def exact(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = {"case": case}
    globals()["_prepare_" + case["kind"]](case, int(seed), g, s)
    return globals()["_exact_" + case["kind"]](case, s)


def _exact_rotary(case, s):
    # a pair as a complex number, times one of the angle
    a = torch.remainder(s["positions"].double().unsqueeze(1) * s["turns"], 1.0) * (2 * math.pi)
    turn = torch.polar(torch.full_like(a, s["scale"]), a).unsqueeze(1)
    half, out = case["rotary_dim"] // 2, {}
    for name in "qk":
        y = s[name].double().clone()
        i = torch.arange(half, device="cuda")
        re, im = (i, i + half) if case["layout"] == "halves" else (2 * i, 2 * i + 1)
        z = torch.complex(y[..., re], y[..., im]) * turn
        y[..., re], y[..., im] = z.real, z.imag
        out[name] = y
    return out


def _exact_gated(case, s):
    x, codes, N = s["x"].double(), s["w"].to(torch.int16), case["N"]
    both = torch.zeros((case["M"], 2 * N), dtype=torch.float64, device="cuda")
    for i, k0 in enumerate(range(0, case["K"], case["group"])):
        k1 = min(case["K"], k0 + case["group"])
        part = codes[:, k0 // 2:k1 // 2]
        even, odd = part % 16, part // 16
        if s["zeros"] is None:
            even, odd = (even + 8) % 16 - 8, (odd + 8) % 16 - 8
        else:
            even, odd = even - s["zeros"][:, i:i + 1].short(), odd - s["zeros"][:, i:i + 1].short()
        both += (x[:, k0:k1:2] @ even.double().t() + x[:, k0 + 1:k1:2] @ odd.double().t()) * s["scales"][:, i].double()
    if s["bias"] is not None:
        both += s["bias"].double()
    g, u = both[:, :N], both[:, N:]
    if case["activation"] == "silu":
        return g * torch.sigmoid(g) * u
    if case["activation"] == "gelu":
        return g * torch.special.ndtr(g) * u
    if case["activation"] == "gelu_tanh":
        return g * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)) * u    # (1 + tanh v) / 2 is the logistic function of 2 v
    return torch.relu(g) * u


def _exact_adapters(case, s):
    y, rows = s["base"].double().clone(), s["adapter"].tolist()
    for a, rank in enumerate(_ints(case["ranks"])):
        at = torch.tensor([m for m, v in enumerate(rows) if v == a], dtype=torch.long, device="cuda")
        if len(at):
            h = s["x"].double()[at] @ s["a"][a, :rank].double().t()
            y[at] += float(s["scales"][a]) * (h @ s["b"][a, :, :rank].double().t())
    return y


def _exact_logits(case, s):
    V, y, t = case["vocab"], s["logits"].double().clone(), 0
    masks, rows, bias = s["mask"].tolist(), s["allowed_row"].tolist(), s["bias_starts"].tolist()
    past_lens, prompt_lens, penalties = s["past_lens"].tolist(), s["prompt_lens"].tolist(), s["penalties"].double()
    for b, n in enumerate(_ints(case["drafts"])):
        past, first = s["past"][b].long(), t
        r, presence, frequency = (float(v) for v in penalties[b])
        for i in range(n):
            mine = s["drafts"][[first + j for j in range(n) if masks[t] >> j & 1]].long()
            count = torch.bincount(torch.cat((past[prompt_lens[b]:past_lens[b]], mine)), minlength=V).double()
            occurred = torch.bincount(torch.cat((past[:past_lens[b]], mine)), minlength=V) > 0
            row = y[t]
            row = torch.where(occurred & (row > 0), row / r, torch.where(occurred, row * r, row)) - frequency * count - presence * (count > 0)
            row[s["bias_ids"][bias[b]:bias[b + 1]].long()] += s["bias_values"][bias[b]:bias[b + 1]].double()
            if rows[t] >= 0:
                bits = torch.stack([s["allowed"][rows[t]] >> i & 1 for i in range(32)], dim=1).flatten()[:V]
                row[bits == 0] = -math.inf
            y[t] = row
            t += 1
    return y


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "rotary":
        rows = case["tokens"] * (case["q_heads"] + case["kv_heads"])
        return {"bytes": 4 * rows * case["head_dim"] + 4 * case["tokens"] + 4 * case["rotary_dim"], "flops": 3 * rows * case["rotary_dim"]}
    if kind == "gated":
        M, N, K = case["M"], case["N"], case["K"]
        groups = -(-K // case["group"])
        return {"bytes": N * K + 2 * N * groups * (3 if case["zeros"] else 2) + 2 * M * (K + N) + (4 * N if case["bias"] else 0), "flops": 4 * M * N * K}
    if kind == "adapters":
        M, N, K, ranks = case["M"], case["N"], case["K"], _ints(case["ranks"])
        used = range(len(ranks)) if case["runs"] == "mixed" else sorted(set(_ints(case["runs"])) - {-1})
        used = list(used)[:M]
        mean = sum(ranks[a] for a in used) / max(1, len(used))
        return {"bytes": 2 * M * (K + 2 * N) + 2 * (K + N) * sum(ranks[a] for a in used), "flops": int(2 * M * mean * (K + N))}
    rows, V = sum(_ints(case["drafts"])), case["vocab"]
    return {"bytes": 4 * rows * V + 4 * sum(_ints(case["past"])) + min(case["masks"], rows) * V // 8, "flops": 0}

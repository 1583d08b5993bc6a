"""A decoder's whole step in the library on the GPU: the example with rotary positions, the fused gate, adapters and rules against a plain forward
in 64 bits; the operators captured in one graph; on streams of their own."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _plain_logits(model, tokens, request):
    """The model's formulas over one sequence in 64 bits, with the weights that the nibbles stand for."""
    import torch
    from paper_2011_10680_amd.convert import rotary_turns
    c = model.config
    D, H, KV = c["head_dim"], c["q_heads"], c["kv_heads"]
    norm = lambda x: x * torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + 1e-6)  # noqa: E731
    x = model.embedding[torch.tensor(tokens, device="cuda")].double().cpu()
    n = len(tokens)
    a = 2 * np.pi * torch.arange(n, dtype=torch.float64)[:, None] * torch.from_numpy(rotary_turns(D))
    turn = torch.polar(torch.ones_like(a), a)[:, None]

    def turned(v):
        z = torch.complex(v[..., :D // 2].contiguous(), v[..., D // 2:].contiguous()) * turn
        return torch.cat((z.real, z.imag), dim=-1)
    i = int(model.adapter[request])
    for layer, ad in zip(model.layers, model.adapters):
        w = {k: v.real().double().cpu() for k, v in layer.items()}
        qkv = norm(x) @ w["qkv"].t()
        if i >= 0:
            r = int(ad.ranks[i])
            qkv = qkv + 0.5 * (norm(x) @ ad.a[i, :r].double().cpu().t()) @ ad.b[i, :, :r].double().cpu().t()
        qkv = qkv.view(n, H + 2 * KV, D)
        q, k, v = turned(qkv[:, :H]), turned(qkv[:, H:H + KV]), qkv[:, H + KV:]
        y = torch.empty(n, H, D, dtype=torch.float64)
        for h in range(H):
            s = q[:, h] @ k[:, h // (H // KV)].t() * D ** -0.5
            s = s.masked_fill(torch.ones(n, n).triu(1).bool(), float("-inf"))
            y[:, h] = torch.softmax(s, dim=1) @ v[:, h // (H // KV)]
        x = x + y.reshape(n, -1) @ w["out"].t()
        gate, up = (norm(x) @ w["up"].t()).chunk(2, dim=1)
        x = x + (torch.nn.functional.silu(gate) * up) @ w["down"].t()
    return norm(x) @ model.head.real().double().cpu().t()


# A token passes some twenty roundings to the activations' type (norms, projections, attention, residuals), each an independent relative error of at most
# u of its tensor, and two more a layer for the adapters' sum and the turned queries and keys: together under 24 u of the logits' norm
@pytest.mark.parametrize("dtype,far", [("f16", 24 * 2.0 ** -11), ("bf16", 24 * 2.0 ** -8)])
def test_prompt_and_tree_logits(dtype, far):
    import torch
    from paper_2011_10680_amd import lm_example as ex
    r = np.random.default_rng(3)
    prompts = [r.integers(0, 512, size=n).tolist() for n in (40, 1, 17)]
    model = ex.Decoder(3, dtype=torch.float16 if dtype == "f16" else torch.bfloat16, seed=4, whole=True, adapters=[1, -1, 0])
    got = model.prompts(prompts).double().cpu()
    # a chain, a tree with two branches, one token
    drafts = [r.integers(0, 512, size=n).tolist() for n in (2, 5, 1)]
    masks, paths = [[1, 3], [1, 3, 5, 11, 21], [1]], [[[0], [0, 1]], [[0], [0, 1], [0, 2], [0, 1, 3], [0, 2, 4]], [[0]]]
    after = model.check(drafts, masks).double().cpu()
    first = at = 0
    for b, p in enumerate(prompts):
        want = _plain_logits(model, p, b)
        assert float((got[first:first + len(p)] - want).norm() / want.norm()) <= far
        first += len(p)
        for path in paths[b]:
            want = _plain_logits(model, p + [drafts[b][j] for j in path], b)[-1]
            assert float((after[at] - want).norm() / want.norm()) <= far, (b, path)
            at += 1


def _ruled(logits, tokens, n_prompt, penalties, biases, allowed):
    """The rules for one row, by the definition."""
    r, presence, frequency = penalties
    row = logits.clone()
    for v in set(tokens):
        row[v] = row[v] / r if row[v] > 0 else row[v] * r
    for v in set(tokens[n_prompt:]):
        row[v] -= frequency * tokens[n_prompt:].count(v) + presence
    for v, add in biases.items():
        row[v] += add
    keep = row[allowed].clone()
    row[:] = float("-inf")
    row[allowed] = keep
    return row


def test_drafting_under_rules_writes_what_single_tokens_write():
    """The drafted answer is the single-token answer up to the first place where two ruled logits lie within rounding of one another."""
    import torch
    from paper_2011_10680_amd import lm_example as ex
    r = np.random.default_rng(5)
    prompts = [r.integers(0, 512, size=n).tolist() for n in (9, 30, 2)]
    penalties, biases, allowed = (1.25, 0.5, 0.25), {4: -50.0, 8: 3.0, 16: 2.0}, list(range(0, 512, 4))

    def make():
        return ex.Decoder(3, dtype=torch.float16, seed=6, whole=True, adapters=[0, 2, -1], rules=ex.Rules(3, 512, penalties, biases, allowed))
    plain, _, _ = ex.generate(make(), prompts, 24, drafting=False)
    drafted, _, _ = ex.generate(make(), prompts, 24)
    model = make()
    far = 24 * 2.0 ** -11
    for b, (p, x, y) in enumerate(zip(prompts, plain, drafted)):
        assert all(t % 4 == 0 and t != 4 for t in x + y)
        # the first written tokens are the ruled best of the plain forward, as far as rounding tells
        seen = list(p)
        for t in x[:6]:
            logits = _plain_logits(model, seen, b)[-1]
            row = _ruled(logits, seen, len(p), penalties, biases, allowed)
            assert float(row.max() - row[t]) <= 2 * penalties[0] * far * float(logits.norm())
            seen.append(t)
        if x == y:
            continue
        i = next(i for i, (s, t) in enumerate(zip(x, y)) if s != t)
        logits = _plain_logits(model, p + x[:i], b)[-1]
        row = _ruled(logits, p + x[:i], len(p), penalties, biases, allowed)
        assert abs(float(row[x[i]] - row[y[i]])) <= 2 * penalties[0] * far * float(logits.norm()), i


def _step(hawq, dtype, M, g):
    """Buffers of one step of M requests, and the calls over them."""
    import torch
    H, KV, D, K, V = 4, 2, 64, 256, 1000
    F = 512 if M < 500 else 3000                  # (the kernel for whole prompts)
    t = {torch.float16: hawq.F16, torch.bfloat16: hawq.BF16}[dtype]
    n = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)  # noqa: E731
    i32 = dict(dtype=torch.int32, device="cuda")
    w = torch.randint(0, 256, (2 * F, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    held = dict(w=w, s=(0.02 * torch.rand((2 * F, K // 64), generator=g, device="cuda")).to(dtype), a=n(3, 8, K), b=n(3, (H + 2 * KV) * D, 8), ranks=torch.tensor([8, 3, 5], **i32),
                scales=torch.ones(3, device="cuda"), turns=torch.from_numpy(10000.0 ** (-np.arange(D // 2) / (D // 2)) / 6.28).cuda(),
                penalties=torch.tensor([[1.2, 0.1, 0.2]] * M, device="cuda"), none=torch.zeros(M + 1, **i32))
    inputs = dict(x=n(M, K), adapter=torch.zeros(M, **i32), positions=torch.zeros(M, **i32), logits=n(M, V), past=torch.zeros((M, 50), **i32), lens=torch.zeros(M, **i32))
    row = (H + 2 * KV) * D

    def buffers():
        gd = hawq.GatedW4Desc(M=M, N=F, K=K, group=64, x_dtype=t, w_dtype=hawq.S4, activation=hawq.SILU, x_stride=K, y_stride=F)
        ad = hawq.AdaptersDesc(M=M, N=row, K=K, n_adapters=3, max_rank=8, dtype=t, x_stride=K, base_stride=row, y_stride=row, a_adapter=8 * K, a_row=K, b_adapter=8 * row, b_row=8)
        assert (hawq.hawq_gated_w4_workspace_bytes(gd) > 0) == (M >= 500)
        return dict(gd=gd, ad=ad, rd=hawq.RotaryDesc(total=M, q_heads=H, kv_heads=KV, head_dim=D, rotary_dim=D, layout=hawq.ROTARY_PAIRS, dtype=t, scale=1.0, q_token=row, q_head=D,
                                                     k_token=row, k_head=D, yq_token=row, yq_head=D, yk_token=row, yk_head=D),
                    ld=hawq.LogitsDesc(n_seqs=M, total=M, vocab=V, dtype=t, past_stride=50, n_bias=0, n_allowed=0, allowed_stride=0, x_stride=V, y_stride=V),
                    base=torch.ones((M, row), dtype=dtype, device="cuda"), qkv=torch.empty((M, row), dtype=dtype, device="cuda"), h=torch.empty((M, F), dtype=dtype, device="cuda"),
                    y=torch.empty((M, V), dtype=dtype, device="cuda"), ws=torch.empty(max(16, hawq.hawq_adapters_workspace_bytes(ad)), dtype=torch.uint8, device="cuda"),
                    gws=torch.empty(max(16, hawq.hawq_gated_w4_workspace_bytes(gd)), dtype=torch.uint8, device="cuda"))

    def run(b):
        hawq.hawq_adapters(b["ad"], inputs["x"], held["a"], held["b"], held["ranks"], held["scales"], inputs["adapter"], b["base"], b["qkv"], b["ws"])
        qkv = b["qkv"].view(M, H + 2 * KV, D)
        hawq.hawq_rotary(b["rd"], qkv[:, :H], qkv[:, H:H + KV], inputs["positions"], held["turns"], qkv[:, :H], qkv[:, H:H + KV])
        hawq.hawq_gated_w4(b["gd"], inputs["x"], held["w"], held["s"], None, None, b["h"], b["gws"])
        hawq.hawq_logits(b["ld"], inputs["logits"], inputs["past"], inputs["lens"], None, None, None, None, held["penalties"], None, None, None, None, None, b["y"])

    def change():
        for name in ("x", "logits"):
            inputs[name].copy_(torch.randn(inputs[name].shape, generator=g, device="cuda"))
        inputs["adapter"].copy_(torch.randint(-1, 3, (M,), generator=g, device="cuda"))
        inputs["positions"].copy_(torch.randint(0, 100000, (M,), generator=g, device="cuda"))
        inputs["past"].copy_(torch.randint(0, V, (M, 50), generator=g, device="cuda"))
        inputs["lens"].copy_(torch.randint(0, 51, (M,), generator=g, device="cuda"))
    return buffers, run, change


@pytest.mark.parametrize("M", [3, 600])
def test_replays_equal_eager_calls(M):
    """One graph of all four, replayed with other inputs; two graphs that share their workspaces in turn."""
    import torch
    import paper_2011_10680_amd as hawq
    g = torch.Generator(device="cuda").manual_seed(1)
    buffers, run, change = _step(hawq, torch.bfloat16, M, g)
    eager, held, other = buffers(), buffers(), buffers()
    other["ws"], other["gws"] = held["ws"], held["gws"]
    for b in (eager, held, other):
        run(b)
    torch.cuda.synchronize()
    graphs = []
    for b in (held, other):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run(b)
        graphs.append(graph)
    for i in range(4):
        change()
        run(eager)
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for name in ("qkv", "h", "y"):
            assert torch.equal(eager[name], held[name]) and torch.equal(eager[name], other[name]), (i, name)


def test_other_streams():
    """Two streams at once, each with its own buffers, on inputs that the stream itself makes."""
    import torch
    import paper_2011_10680_amd as hawq
    g = torch.Generator(device="cuda").manual_seed(2)
    sides = []
    for M in (40, 700):
        buffers, run, change = _step(hawq, torch.float16, M, g)
        change()
        want, got = buffers(), buffers()
        run(want)
        sides.append((run, want, got, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(3):
        for run, want, got, stream in sides:
            with torch.cuda.stream(stream):
                for name in ("qkv", "h", "y"):
                    got[name].fill_(9)
                run(got)
    torch.cuda.synchronize()
    for run, want, got, _ in sides:
        for name in ("qkv", "h", "y"):
            assert torch.equal(want[name], got[name]), name


def test_command_runs(capsys, monkeypatch):
    from paper_2011_10680_amd import lm_example as ex
    monkeypatch.setattr("sys.argv", ["lm_example", "--whole", "--tokens", "5"])
    ex.main()
    lines = capsys.readouterr().out.splitlines()
    assert len(lines) == 5
    for line in lines[:4]:
        answer = [int(t) for t in line.split("-> [")[1].rstrip("]").split(",")]
        assert len(answer) == 5 and all(t % 2 == 0 and t != 7 for t in answer)

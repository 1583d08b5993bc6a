"""The language-model operators together: a small decoder with 4-bit weights and a paged cache answers a few prompts.

Prompts of different lengths are taken in one packed batch (`hawq_linear_w4`, `hawq_attn_prompt`), their keys and values go to pages
of the cache (`hawq_cache_plan`, `hawq_cache_store`).  Then every step drafts a small tree of continuations for each request, checks
all of them in one pass (`hawq_attn_tree`) and keeps the longest branch that the model itself would have written, so that the answer is
that of decoding token by token.  The model is random: norms, gates and residuals are plain torch.

With `whole` the rest of a step runs in the library too: positions (`hawq_rotary`), the feed-forward's gate (`hawq_gated_w4`), adapters of the
requests' own (`hawq_adapters`), and rules for the answers (`hawq_logits`), which see a drafted token's own branch.

    python -m paper_2011_10680_amd.lm_example [--cache s8] [--tokens 24] [--whole]
"""
import argparse

import numpy as np
import torch

from . import (BF16, F16, ROTARY_HALVES, S4, S8, SILU, U4, AdaptersDesc, AttnPromptDesc, AttnTreeDesc, CacheDesc, CacheStoreDesc, GatedW4Desc, LinearW4Desc, LogitsDesc,
               RotaryDesc, hawq_adapters, hawq_adapters_workspace_bytes, hawq_attn_prompt, hawq_attn_tree, hawq_attn_tree_workspace_bytes, hawq_cache_plan, hawq_cache_store,
               hawq_gated_w4, hawq_gated_w4_workspace_bytes, hawq_linear_w4, hawq_logits, hawq_rotary)
from .convert import quantize_groups, rotary_turns

CONFIG = dict(layers=2, width=256, hidden=512, q_heads=8, kv_heads=2, head_dim=64, vocab=512, group=64, page=16, pages=256)
_HAWQ = {torch.float16: F16, torch.bfloat16: BF16}


def _strides(**tensors):
    return {"%s_%s" % (n, w): t.stride(i) for n, t in tensors.items() for i, w in enumerate(("token", "head"))}


class Linear:
    """A weight matrix as the framework holds it: nibbles, scales and, where asked for, zero points."""

    def __init__(self, weight, group, dtype, zero_points):
        w, s, z = quantize_groups(weight, group, zero_points, _HAWQ[dtype])
        self.N, self.K, self.group, self.dtype = weight.shape[0], weight.shape[1], group, dtype
        self.w, self.scales = torch.from_numpy(w).cuda(), torch.from_numpy(s).to(dtype).cuda()
        self.zeros = None if z is None else torch.from_numpy(z).cuda()

    def __call__(self, x):
        y = torch.empty((x.shape[0], self.N), dtype=self.dtype, device=x.device)
        d = LinearW4Desc(M=x.shape[0], N=self.N, K=self.K, group=self.group, x_dtype=_HAWQ[self.dtype], w_dtype=S4 if self.zeros is None else U4,
                         x_stride=x.stride(0), y_stride=self.N)
        hawq_linear_w4(d, x, self.w, self.scales, self.zeros, None, y)
        return y

    def gated(self, x):
        """silu of the first half of the outputs times the second half."""
        N = self.N // 2
        y = torch.empty((x.shape[0], N), dtype=self.dtype, device=x.device)
        d = GatedW4Desc(M=x.shape[0], N=N, K=self.K, group=self.group, x_dtype=_HAWQ[self.dtype], w_dtype=S4 if self.zeros is None else U4, activation=SILU,
                        x_stride=x.stride(0), y_stride=N)
        room = torch.empty(hawq_gated_w4_workspace_bytes(d), dtype=torch.uint8, device=x.device)
        hawq_gated_w4(d, x, self.w, self.scales, self.zeros, None, y, room)
        return y

    def real(self):
        """The matrix that the nibbles stand for, for checks."""
        q = torch.stack((self.w & 15, self.w >> 4), dim=2).reshape(self.N, self.K).float()
        spread = lambda t: t.float().repeat_interleave(self.group, dim=1)[:, :self.K]  # noqa: E731
        q = torch.where(q >= 8, q - 16, q) if self.zeros is None else q - spread(self.zeros)
        return q * spread(self.scales)


class Adapters:
    """Low-rank additions to one projection, of different ranks: a [adapter, rank, inputs], b [adapter, outputs, rank]."""

    def __init__(self, r, ranks, N, K, dtype):
        most = max(ranks)
        self.a = torch.from_numpy(r.normal(size=(len(ranks), most, K)) / K ** 0.5).to(dtype).cuda()
        self.b = torch.from_numpy(r.normal(size=(len(ranks), N, most)) / most ** 0.5).to(dtype).cuda()
        self.ranks, self.scales = torch.tensor(ranks, dtype=torch.int32, device="cuda"), torch.full((len(ranks),), 0.5, device="cuda")

    def add(self, x, y, adapter):
        """y += what the rows' adapters make of x."""
        n, most, K = self.a.shape
        d = AdaptersDesc(M=x.shape[0], N=y.shape[1], K=K, n_adapters=n, max_rank=most, dtype=_HAWQ[x.dtype], x_stride=x.stride(0), base_stride=y.stride(0), y_stride=y.stride(0),
                         a_adapter=self.a.stride(0), a_row=self.a.stride(1), b_adapter=self.b.stride(0), b_row=self.b.stride(1))
        room = torch.empty(hawq_adapters_workspace_bytes(d), dtype=torch.uint8, device=x.device)
        hawq_adapters(d, x, self.a, self.b, self.ranks, self.scales, adapter, y, y, room)


class Rules:
    """What the answers of n requests obey: (repetition, presence, frequency), a bias for some tokens, and the tokens allowed at all (None: all)."""

    def __init__(self, n, vocab, penalties=(1.0, 0.0, 0.0), biases=None, allowed=None):
        biases = biases or {}
        self.penalties = torch.tensor([penalties] * n, dtype=torch.float32, device="cuda")
        self.starts = torch.arange(n + 1, dtype=torch.int32, device="cuda") * len(biases)
        self.ids = torch.tensor(list(biases) * n, dtype=torch.int32, device="cuda")
        self.values = torch.tensor(list(biases.values()) * n, dtype=torch.float32, device="cuda")
        bits = np.zeros((1, -(-vocab // 32)), np.uint32)
        for v in allowed if allowed is not None else ():
            bits[0, v // 32] |= np.uint32(1 << v % 32)
        self.allowed = None if allowed is None else torch.from_numpy(bits.view(np.int32)).cuda()

    def apply(self, logits, past, past_lens, prompt_lens, starts=None, drafts=None, mask=None):
        """In place; one row for each request, or rows packed by starts, each behind its own branch of the drafts."""
        rows = None if self.allowed is None else torch.zeros(logits.shape[0], dtype=torch.int32, device=logits.device)
        d = LogitsDesc(n_seqs=past.shape[0], total=logits.shape[0], vocab=logits.shape[1], dtype=_HAWQ[logits.dtype], past_stride=past.stride(0), n_bias=self.ids.numel(),
                       n_allowed=0 if rows is None else 1, allowed_stride=0 if rows is None else self.allowed.stride(0), x_stride=logits.stride(0), y_stride=logits.stride(0))
        hawq_logits(d, logits, past, past_lens, prompt_lens, starts, drafts, mask, self.penalties, self.starts, self.ids, self.values, self.allowed, rows, logits)


def _norm(x):
    f = x.float()
    return (f * torch.rsqrt(f.square().mean(dim=-1, keepdim=True) + 1e-6)).to(x.dtype)


class Decoder:
    """The model, its cache, and the requests that hold pages of it."""

    def __init__(self, n_requests, dtype=torch.bfloat16, cache="same", seed=0, config=CONFIG, most=1024, whole=False, adapters=None, rules=None):
        """whole: positions are rotary and the gate is the library's.  adapters: each request's own (0, 1 or 2; -1: none).  rules: Rules of the answers."""
        c = self.config = dict(config)
        self.dtype, self.n = dtype, n_requests
        r = np.random.default_rng(seed)
        D, H, KV = c["head_dim"], c["q_heads"], c["kv_heads"]
        make = lambda n, k, z=False: Linear(r.normal(size=(n, k)) / k ** 0.5, c["group"], dtype, z)  # noqa: E731
        self.layers = [dict(qkv=make((H + 2 * KV) * D, c["width"]), out=make(c["width"], H * D, True), up=make(2 * c["hidden"], c["width"]), down=make(c["width"], c["hidden"], True))
                       for _ in range(c["layers"])]
        self.embedding = torch.from_numpy(r.normal(size=(c["vocab"], c["width"]))).to(dtype).cuda()
        self.head = make(c["vocab"], c["width"])
        s8 = cache == "s8"
        shape = (c["pages"], c["page"], KV, D)
        self.caches = [tuple(torch.zeros(shape, dtype=torch.int8 if s8 else dtype, device="cuda") for _ in "kv") +
                       (tuple(torch.zeros(shape[:3], device="cuda") for _ in "kv") if s8 else (None, None)) for _ in range(c["layers"])]
        k = self.caches[0][0]
        self.cache_desc = CacheDesc(n_pages=c["pages"], page=c["page"], kv_heads=KV, head_dim=D, dtype=S8 if s8 else _HAWQ[dtype], page_stride=k.stride(0),
                                    token_stride=k.stride(1), head_stride=k.stride(2))
        self.free = torch.arange(c["pages"], dtype=torch.int32, device="cuda")
        self.table = torch.full((n_requests, -(-most // c["page"])), -1, dtype=torch.int32, device="cuda")
        self.cached = torch.zeros(n_requests, dtype=torch.int32, device="cuda")
        self.lengths = [0] * n_requests                               # the same on the host
        self.whole, self.rules = whole, rules
        self.turns = torch.from_numpy(rotary_turns(D)).cuda()
        self.adapters = None
        if adapters is not None:
            self.adapter = torch.tensor(adapters, dtype=torch.int32, device="cuda")
            self.adapters = [Adapters(r, (4, 16, 8), (H + 2 * KV) * D, c["width"], dtype) for _ in range(c["layers"])]
        self.past = torch.zeros((n_requests, self.table.shape[1] * c["page"]), dtype=torch.int32, device="cuda")      # the cached tokens themselves
        self.prompt_lens = torch.zeros(n_requests, dtype=torch.int32, device="cuda")

    def _room(self, fresh):
        """Slots for `fresh[b]` more tokens of every request; their pages leave the free list."""
        if max(n + f for n, f in zip(self.lengths, fresh)) > self.table.shape[1] * self.config["page"]:
            raise RuntimeError("a request has outgrown its row of the block table")
        fresh_d = torch.tensor(fresh, dtype=torch.int32, device="cuda")
        starts = torch.empty(self.n + 1, dtype=torch.int32, device="cuda")
        slots, counts = torch.empty(sum(fresh), dtype=torch.int64, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
        hawq_cache_plan(self.cached, fresh_d, self.config["page"], self.free, self.table, starts, slots, counts)
        taken = int(counts[1])
        if taken > self.free.numel():
            raise RuntimeError("the cache is full")
        self.free = self.free[taken:].clone()
        return starts, slots, fresh_d

    def _grow(self, fresh, fresh_d):
        self.cached += fresh_d
        self.lengths = [n + f for n, f in zip(self.lengths, fresh)]

    def _store(self, layer, k, v, slots):
        d = CacheStoreDesc(cache=self.cache_desc, total=k.shape[0], dtype=_HAWQ[self.dtype], **_strides(k=k, v=v))
        hawq_cache_store(d, k, v, slots, *self.caches[layer])

    def _turn(self, q, k, positions):
        """Queries and keys in place."""
        c = self.config
        d = RotaryDesc(total=q.shape[0], q_heads=c["q_heads"], kv_heads=c["kv_heads"], head_dim=c["head_dim"], rotary_dim=c["head_dim"], layout=ROTARY_HALVES, dtype=_HAWQ[self.dtype],
                       scale=1.0, **_strides(q=q, k=k, yq=q, yk=k))
        hawq_rotary(d, q, k, positions, self.turns, q, k)

    def _forward(self, tokens, attend, positions, requests):
        """Logits of packed tokens at their positions in their requests; attend(layer, q, k, v, y) fills y."""
        c, x = self.config, self.embedding[tokens]
        D, H, KV = c["head_dim"], c["q_heads"], c["kv_heads"]
        for i, layer in enumerate(self.layers):
            inner = _norm(x)
            qkv = layer["qkv"](inner)
            if self.adapters is not None:
                self.adapters[i].add(inner, qkv, self.adapter[requests])
            qkv = qkv.view(-1, H + 2 * KV, D)
            if self.whole:
                self._turn(qkv[:, :H], qkv[:, H:H + KV], positions)
            y = torch.empty((qkv.shape[0], H, D), dtype=self.dtype, device="cuda")
            attend(i, qkv[:, :H], qkv[:, H:H + KV], qkv[:, H + KV:], y)
            x = x + layer["out"](y.view(-1, H * D))
            if self.whole:
                x = x + layer["down"](layer["up"].gated(_norm(x)))
                continue
            gate, up = layer["up"](_norm(x)).chunk(2, dim=1)
            x = x + layer["down"]((torch.nn.functional.silu(gate.float()) * up.float()).to(self.dtype))
        return self.head(_norm(x))

    def prompts(self, prompts):
        """Takes the requests' prompts; the logits of all their tokens, packed."""
        c, lens = self.config, [len(p) for p in prompts]
        starts, slots, fresh = self._room(lens)

        def attend(i, q, k, v, y):
            d = AttnPromptDesc(n_seqs=self.n, total=q.shape[0], q_heads=c["q_heads"], kv_heads=c["kv_heads"], head_dim=c["head_dim"], dtype=_HAWQ[self.dtype],
                               scale=c["head_dim"] ** -0.5, **_strides(q=q, k=k, v=v, y=y))
            hawq_attn_prompt(d, q, k, v, starts, y)
            self._store(i, k, v, slots)
        positions = torch.tensor([t for n in lens for t in range(n)], dtype=torch.int32, device="cuda")
        logits = self._forward(torch.tensor([t for p in prompts for t in p], device="cuda"), attend, positions, self._requests(lens))
        for b, p in enumerate(prompts):
            self.past[b, :len(p)] = torch.tensor(p, dtype=torch.int32)
        self.prompt_lens.copy_(fresh)
        self._grow(lens, fresh)
        return logits

    def _requests(self, lens):
        return torch.tensor([b for b, n in enumerate(lens) for _ in range(n)], device="cuda")

    def first(self, logits):
        """Logits of the prompts' last tokens by the rules; logits: what `prompts` gave."""
        ends = torch.cumsum(self.prompt_lens.long(), 0) - 1
        rows = logits[ends]
        if self.rules is not None:
            self.rules.apply(rows, self.past, self.cached, self.prompt_lens)
        return rows

    def check(self, drafts, masks):
        """Logits of drafted tokens (one list for each request, every token's mask over its own list); they are not stored yet."""
        c, lens = self.config, [len(d) for d in drafts]
        total = sum(lens)
        starts = torch.tensor(np.concatenate(([0], np.cumsum(lens))), dtype=torch.int32, device="cuda")
        mask = torch.tensor([m - (1 << 64) if m >> 63 else m for request in masks for m in request], dtype=torch.int64, device="cuda")
        self.drafted, self.workspace = [], None

        def attend(i, q, k, v, y):
            d = AttnTreeDesc(cache=self.cache_desc, n_seqs=self.n, total=total, max_drafts=max(lens), max_cached=max(self.lengths), q_heads=c["q_heads"], dtype=_HAWQ[self.dtype],
                             table_stride=self.table.shape[1], scale=c["head_dim"] ** -0.5, **_strides(q=q, k=k, v=v, y=y))
            if self.workspace is None:
                self.workspace = torch.empty(hawq_attn_tree_workspace_bytes(d), dtype=torch.uint8, device="cuda")
            hawq_attn_tree(d, q, k, v, starts, mask, *self.caches[i], self.table, self.cached, y, self.workspace)
            self.drafted.append((k, v))
        tokens = torch.tensor([t for d in drafts for t in d], device="cuda")
        # a drafted token lies as many tokens behind the cache as it has ancestors
        depth = torch.tensor([bin(m).count("1") - 1 for request in masks for m in request], dtype=torch.int32, device="cuda")
        requests = self._requests(lens)
        logits = self._forward(tokens, attend, self.cached[requests] + depth, requests)
        self.tokens = tokens.to(torch.int32)
        if self.rules is not None:
            self.rules.apply(logits, self.past, self.cached, self.prompt_lens, starts, self.tokens, mask)
        return logits

    def keep(self, lens, kept):
        """Stores what was kept of the last check's drafts: kept[b] are rows of request b, in order."""
        _, slots, fresh = self._room([len(k) for k in kept])
        first = np.concatenate(([0], np.cumsum(lens)))
        rows = [int(first[b]) + i for b, k in enumerate(kept) for i in k]
        at = torch.full((int(first[-1]),), -1, dtype=torch.int64, device="cuda")
        at[torch.tensor(rows, device="cuda")] = slots
        for i, (k, v) in enumerate(self.drafted):
            self._store(i, k, v, at)
        for b, k in enumerate(kept):
            self.past[b, self.lengths[b]:self.lengths[b] + len(k)] = self.tokens[[int(first[b]) + i for i in k]]
        self._grow([len(k) for k in kept], fresh)


def _draft(last, memory, width=2, depth=3):
    """A tree of guesses from what followed each token before: (tokens, parents, masks); the first token is `last` itself."""
    tokens, parents, masks, level = [last], [-1], [1], [0]
    for _ in range(depth):
        deeper = []
        for p in level:
            for t in memory.get(tokens[p], ())[-width:]:
                tokens.append(t)
                parents.append(p)
                masks.append(masks[p] | 1 << len(tokens) - 1)
                deeper.append(len(tokens) - 1)
        level = deeper
    return tokens, parents, masks


def generate(model, prompts, n_tokens, drafting=True):
    """Greedy answers of n_tokens each, the number of passes that they took, and the tokens written in all (requests that drafted well are ahead)."""
    out = [[int(t)] for t in model.first(model.prompts(prompts)).argmax(dim=1)]
    memory, passes = [{} for _ in prompts], 0
    for m, p in zip(memory, prompts):
        for a, b in zip(p, p[1:]):
            m.setdefault(a, []).append(b)
    while min(len(o) for o in out) < n_tokens:
        trees = [_draft(o[-1], m if drafting else {}) for o, m in zip(out, memory)]
        best = model.check([t[0] for t in trees], [t[2] for t in trees]).argmax(dim=1).tolist()
        passes += 1
        kept, first = [], 0
        for o, m, (tokens, parents, _) in zip(out, memory, trees):
            path, at = [0], 0
            while True:
                said = best[first + at]
                m.setdefault(tokens[at], []).append(said)
                o.append(said)
                at = next((i for i, p in enumerate(parents) if p == at and tokens[i] == said), None)
                if at is None:
                    break
                path.append(at)
            kept.append(path)
            first += len(tokens)
        model.keep([len(t[0]) for t in trees], kept)
    return [o[:n_tokens] for o in out], passes, sum(len(o) for o in out)


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--cache", choices=("same", "s8"), default="same")
    ap.add_argument("--tokens", type=int, default=24)
    ap.add_argument("--whole", action="store_true", help="rotary positions, the fused gate, adapters and rules for the answers")
    a = ap.parse_args()
    r = np.random.default_rng(1)
    prompts = [r.integers(0, CONFIG["vocab"], size=n).tolist() for n in (5, 37, 1, 18)]
    more = dict(whole=True, adapters=[0, 2, -1, 1], rules=Rules(len(prompts), CONFIG["vocab"], (1.3, 0.5, 0.2), {7: -100.0}, range(0, CONFIG["vocab"], 2))) if a.whole else {}
    answers, passes, written = generate(Decoder(len(prompts), cache=a.cache, **more), prompts, a.tokens)
    for p, o in zip(prompts, answers):
        print("%d tokens -> %s" % (len(p), o))
    print("%d passes after the prompts, %.2f tokens of a request in a pass" % (passes, (written / len(prompts) - 1) / passes))


if __name__ == "__main__":
    main()

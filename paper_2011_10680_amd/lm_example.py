"""The language-model operators together: a small decoder with 4-bit weights and a paged cache answers a few prompts.

Prompts of different lengths are taken in one packed batch (`hawq_linear_w4`, `hawq_attn_prompt`), their keys and values go to pages
of the cache (`hawq_cache_plan`, `hawq_cache_store`).  Then every step drafts a small tree of continuations for each request, checks
all of them in one pass (`hawq_attn_tree`) and keeps the longest branch that the model itself would have written, so that the answer is
that of decoding token by token.  The model is random: norms, gates and residuals are plain torch.

    python -m paper_2011_10680_amd.lm_example [--cache s8] [--tokens 24]
"""
import argparse

import numpy as np
import torch

from . import (BF16, F16, S4, S8, U4, AttnPromptDesc, AttnTreeDesc, CacheDesc, CacheStoreDesc, LinearW4Desc, hawq_attn_prompt, hawq_attn_tree,
               hawq_attn_tree_workspace_bytes, hawq_cache_plan, hawq_cache_store, hawq_linear_w4)
from .convert import quantize_groups

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

    def real(self):
        """The matrix that the nibbles stand for, for checks."""
        q = torch.stack((self.w & 15, self.w >> 4), dim=2).reshape(self.N, self.K).float()
        spread = lambda t: t.float().repeat_interleave(self.group, dim=1)[:, :self.K]  # noqa: E731
        q = torch.where(q >= 8, q - 16, q) if self.zeros is None else q - spread(self.zeros)
        return q * spread(self.scales)


def _norm(x):
    f = x.float()
    return (f * torch.rsqrt(f.square().mean(dim=-1, keepdim=True) + 1e-6)).to(x.dtype)


class Decoder:
    """The model, its cache, and the requests that hold pages of it."""

    def __init__(self, n_requests, dtype=torch.bfloat16, cache="same", seed=0, config=CONFIG, most=1024):
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

    def _forward(self, tokens, attend):
        """Logits of packed tokens; attend(layer, q, k, v, y) fills y."""
        c, x = self.config, self.embedding[tokens]
        D, H, KV = c["head_dim"], c["q_heads"], c["kv_heads"]
        for i, layer in enumerate(self.layers):
            qkv = layer["qkv"](_norm(x)).view(-1, H + 2 * KV, D)
            y = torch.empty((qkv.shape[0], H, D), dtype=self.dtype, device="cuda")
            attend(i, qkv[:, :H], qkv[:, H:H + KV], qkv[:, H + KV:], y)
            x = x + layer["out"](y.view(-1, H * D))
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
        logits = self._forward(torch.tensor([t for p in prompts for t in p], device="cuda"), attend)
        self._grow(lens, fresh)
        return logits

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
        return self._forward(torch.tensor([t for d in drafts for t in d], device="cuda"), attend)

    def keep(self, lens, kept):
        """Stores what was kept of the last check's drafts: kept[b] are rows of request b, in order."""
        _, slots, fresh = self._room([len(k) for k in kept])
        first = np.concatenate(([0], np.cumsum(lens)))
        rows = [int(first[b]) + i for b, k in enumerate(kept) for i in k]
        at = torch.full((int(first[-1]),), -1, dtype=torch.int64, device="cuda")
        at[torch.tensor(rows, device="cuda")] = slots
        for i, (k, v) in enumerate(self.drafted):
            self._store(i, k, v, at)
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
    ends = np.cumsum([len(p) for p in prompts]) - 1
    out = [[int(t)] for t in model.prompts(prompts)[torch.from_numpy(ends).cuda()].argmax(dim=1)]
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
    a = ap.parse_args()
    r = np.random.default_rng(1)
    prompts = [r.integers(0, CONFIG["vocab"], size=n).tolist() for n in (5, 37, 1, 18)]
    answers, passes, written = generate(Decoder(len(prompts), cache=a.cache), prompts, a.tokens)
    for p, o in zip(prompts, answers):
        print("%d tokens -> %s" % (len(p), o))
    print("%d passes after the prompts, %.2f tokens of a request in a pass" % (passes, (written / len(prompts) - 1) / passes))


if __name__ == "__main__":
    main()

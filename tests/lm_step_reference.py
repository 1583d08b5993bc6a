"""Plain 64-bit definitions of rotary positions, gated projections, adapters and logits processing (numpy), and bounds of a computed
result's distance from them: the stored type's rounding, half a step, and the 32-bit errors of what is computed on the way."""
import math

import numpy as np

import lm_reference as lm

ROUND, F32 = lm.ROUND, lm.F32
# half a step of the smallest values of the type
TINY = {"f16": 2.0 ** -25, "bf16": 2.0 ** -134}


def rotary(x, positions, turns, layout, scale):
    """x [total, heads, D] -> (turned, |scale| (|a| + |b|) of every element's pair, 0 for elements that are not turned)"""
    R = 2 * len(turns)
    r = positions.astype(np.longdouble)[:, None] * turns.astype(np.longdouble)
    a = 2 * np.longdouble(math.pi) * (r - np.rint(r))
    c, s = np.cos(a).astype(np.float64)[:, None], np.sin(a).astype(np.float64)[:, None]
    i, j = (np.arange(R // 2), np.arange(R // 2) + R // 2) if layout == "halves" else (np.arange(0, R, 2), np.arange(1, R, 2))
    y, size = x.copy(), np.zeros_like(x)
    y[..., i] = scale * (x[..., i] * c - x[..., j] * s)
    y[..., j] = scale * (x[..., j] * c + x[..., i] * s)
    size[..., i] = size[..., j] = abs(scale) * (np.abs(x[..., i]) + np.abs(x[..., j]))
    return y, size


def rotary_bound(y, size, positions, turns, dtype):
    """The revolutions' product is off by 2^-53 of itself, its fraction (under 1/2) by 2^-25 in 32 bits, together times 2 pi; sine and cosine by
    two units in the last place (2^-23), four roundings of 2^-24 follow (the scale, two products, the sum)."""
    u = ROUND[dtype]
    most = float(np.max(np.abs(positions.astype(np.float64)), initial=0)) * float(np.max(np.abs(turns), initial=0))
    off = 2 * math.pi * (most * 2.0 ** -53 + 2.0 ** -25) + 2.0 ** -23 + 4 * F32
    return np.where(size > 0, u * np.abs(y) + (1 + u) * off * size + TINY[dtype], 0)


def activation(g, kind):
    """(act(g), what 32-bit rounding of the argument of its exponential does, relative to it)"""
    if kind == "silu":
        with np.errstate(over="ignore"):
            return g / (1 + np.exp(-g)), np.full_like(g, 8.0)
    if kind == "gelu":
        # the tail's relative slope at t = g / sqrt 2 is 2 t^2 + 1 at most
        return np.array([0.5 * v * math.erfc(-v / math.sqrt(2)) for v in g.ravel()]).reshape(g.shape), 16 + 4 * g * g
    if kind == "gelu_tanh":
        t = 2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)
        with np.errstate(over="ignore"):
            return g / (1 + np.exp(-t)), 16 + 8 * np.abs(t)
    return np.maximum(g, 0), np.full_like(g, 1.0)


def gated(x, w, scales, zeros, bias, group, kind, dtype):
    """(y, bound)"""
    both, size = lm.linear(x, w, scales, zeros, bias, group)
    N = both.shape[1] // 2
    # as of hawq_linear_w4: the kernel may sum x (q + 128), at most 143 for a weight
    err = F32 * (group + scales.shape[1] + 64) * 143 * size
    g, u, ge, ue = both[:, :N], both[:, N:], err[:, :N], err[:, N:]
    a, units = activation(g, kind)
    y = a * u
    r = ROUND[dtype]
    # no activation is steeper than 1.13
    ae = 1.13 * ge + F32 * units * (np.abs(a) + 1.13 * ge) + 2.0 ** -126
    return y, r * np.abs(y) + (1 + r) * (ae * (np.abs(u) + ue) + np.abs(a) * ue + F32 * np.abs(y)) + TINY[dtype]


def adapters(x, a, b, ranks, scales, adapter, base, dtype):
    """(y, bound)"""
    y, bound = base.copy(), np.zeros_like(base)
    u = ROUND[dtype]
    for m in range(len(x)):
        i = adapter[m]
        if not 0 <= i < len(a):
            continue
        r = min(max(int(ranks[i]), 0), a.shape[1])
        if r == 0:
            continue
        h, hs = a[i, :r] @ x[m], np.abs(a[i, :r]) @ np.abs(x[m])
        add = scales[i] * (b[i, :, :r] @ h)
        # inner sums of K terms in 32 bits, then two parts of the type: 2^-17 of the sum, and in f16 2^-24 of the row's largest
        he = F32 * (x.shape[1] + 8) * hs
        he = he + 2.0 ** -17 * (np.abs(h) + he) + (2.0 ** -24 * np.max(np.abs(h) + he) if dtype == "f16" else 0)
        total = np.abs(b[i, :, :r]) @ (np.abs(h) + he)
        err = abs(scales[i]) * (np.abs(b[i, :, :r]) @ he + F32 * (2 * r + 8) * total) + 2 * F32 * (np.abs(base[m]) + np.abs(add))
        y[m] = base[m] + add
        bound[m] = u * np.abs(y[m]) + (1 + u) * err + TINY[dtype]
    return y, bound


def logits(x, past, past_lens, prompt_lens, starts, drafts, mask, penalties, bias_starts, bias_ids, bias_values, allowed, allowed_row, dtype):
    """(y, bound, written): None where an argument is not given; rows outside every request are not written."""
    V, u = x.shape[1], ROUND[dtype]
    y, bound, written = x.copy(), np.zeros_like(x), np.zeros(len(x), bool)
    n = len(starts) - 1 if starts is not None else len(x)
    inside = lambda t: 0 <= t < V  # noqa: E731
    for b in range(n):
        first, end = (starts[b], starts[b + 1]) if starts is not None else (b, b + 1)
        for t in range(first, end):
            occurred, count, bias = set(), {}, {}
            if penalties is not None:
                if past is not None:
                    for i, v in enumerate(past[b][:max(0, past_lens[b])]):
                        if inside(v):
                            occurred.add(int(v))
                            if prompt_lens is None or i >= prompt_lens[b]:
                                count[int(v)] = count.get(int(v), 0) + 1
                if drafts is not None:
                    for j in range(end - first):
                        if (int(mask[t]) >> j & 1 if j < 64 else 0) if mask is not None else first + j <= t:
                            v = int(drafts[first + j])
                            if inside(v):
                                occurred.add(v)
                                count[v] = count.get(v, 0) + 1
            if bias_starts is not None:
                for i in range(bias_starts[b], bias_starts[b + 1]):
                    if inside(bias_ids[i]):
                        bias[int(bias_ids[i])] = float(bias_values[i])
            row, size = x[t].copy(), np.abs(x[t])
            r, presence, frequency = (float(v) for v in penalties[b]) if penalties is not None else (1.0, 0.0, 0.0)
            for v in occurred:
                row[v] = row[v] / r if row[v] > 0 else row[v] * r
                size[v] = max(size[v], abs(row[v]))
            for v, c in count.items():
                row[v] -= frequency * c + presence
                size[v] += abs(frequency) * c + abs(presence)
            for v, add in bias.items():
                row[v] += add
                size[v] += abs(add)
            m = -1 if allowed is None else t if allowed_row is None else allowed_row[t]
            if allowed is not None and 0 <= m < len(allowed):
                bits = (allowed[m][np.arange(V) // 32].astype(np.int64) >> (np.arange(V) % 32)) & 1
                row[bits == 0] = -np.inf
            y[t], written[t] = row, True
            changed = np.zeros(V, bool)
            changed[sorted(occurred | set(count) | set(bias))] = True
            # each of the six operations by 2^-24 of no more than `size`; what nothing touches is as it was
            with np.errstate(invalid="ignore"):
                bound[t] = np.where(changed, u * np.abs(row) + (1 + u) * 6 * F32 * size + TINY[dtype], 0)
    return y, bound, written

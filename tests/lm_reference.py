"""Plain 64-bit definitions of the language-model operators (numpy), with the sums of magnitudes that bound a computed result's
distance from them."""
import numpy as np

# unit roundoff of the stored types: 11 and 8 significant bits, to nearest
ROUND = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}
F32 = 2.0 ** -24


def unpack(w, zeros, group):
    """[N, K/2] bytes -> [N, K] integers less their zero point."""
    q = np.stack((w & 15, w >> 4), axis=2).reshape(w.shape[0], -1).astype(np.int64)
    if zeros is None:
        return np.where(q >= 8, q - 16, q)
    return q - np.repeat(zeros.astype(np.int64), group, axis=1)[:, :q.shape[1]]


def linear(x, w, scales, zeros, bias, group):
    """(y, |x| |s| summed over k: what a rounding of any partial sum is measured by)"""
    q = unpack(w, zeros, group).astype(np.float64)
    s = np.repeat(scales.astype(np.float64), group, axis=1)[:, :q.shape[1]]
    y = x @ (q * s).T
    size = np.abs(x) @ np.abs(s).T
    return (y, size) if bias is None else (y + bias, size + np.abs(bias))


def attend(q, k, v, seen, scale):
    """One head.  q [n, D], k, v [m, D], seen [n, m].  (y, sum p |v|, largest sum |q||k| * scale): a value that is not seen plays
    no part, whatever it is; a row that sees nothing, or nothing above -infinity, is zeros."""
    n, D = q.shape
    y, size, top = np.zeros((n, D)), np.zeros((n, D)), 0.0
    for i in range(n):
        at = np.nonzero(seen[i])[0]
        if not len(at):
            continue
        with np.errstate(invalid="ignore", over="ignore"):
            s = (k[at] @ q[i]) * scale
            m = s.max()
            if m == -np.inf:
                continue
            p = np.exp(s - m)
            p /= p.sum()
            y[i] = (p[:, None] * v[at]).sum(axis=0)
            size[i] = (p[:, None] * np.abs(v[at])).sum(axis=0)
            top = max(top, float(np.nanmax(np.where(np.isfinite(s), np.abs(k[at]) @ np.abs(q[i]) * abs(scale), 0))))
    return y, size, top


def attention_bound(y, size, top, keys, head_dim, dtype):
    """Elementwise: the result's own rounding, the probabilities' rounding to the same type (twice where a running maximum moves:
    the sum of the weights is of unrounded ones), and the 32-bit errors of scores (through the exponential) and sums."""
    u = ROUND[dtype]
    f32 = 4 * F32 * (head_dim + 8) * max(1.0, top) + 4 * F32 * (keys + 64)
    # halves below 2^-14 keep 2^-25 of the largest probability, absolutely
    tiny = 2.0 ** -24 * keys * np.max(np.where(np.isfinite(size), size, 0), initial=0.0) if dtype == "f16" else 0.0
    return u * np.abs(y) + (1.01 * u + f32) * size + tiny + 1e-30


def plan(cached, fresh, page, free, table, n_slots):
    """Walks over the requests one by one."""
    table, starts, slots, taken = table.copy(), [0], np.full(n_slots, -1, np.int64), 0
    for b, (c, f) in enumerate(zip(np.maximum(cached, 0), np.maximum(fresh, 0))):
        for p in range(-(-int(c) // page), min(-(-int(c + f) // page), table.shape[1])):
            table[b, p] = free[taken] if taken < len(free) else -1
            taken += 1
        for t in range(int(f)):
            at = int(c) + t
            held = int(table[b, at // page]) if at // page < table.shape[1] else -1
            if starts[-1] + t < n_slots:
                slots[starts[-1] + t] = held * page + at % page if held >= 0 else -1
        starts.append(starts[-1] + int(f))
    return table, np.array(starts, np.int32), slots, np.array([starts[-1], taken], np.int32)


def codes(rows):
    """(codes, scales) of rows [..., D] in an 8-bit cache, computed in 32 bits as the interface says."""
    rows = rows.astype(np.float32)
    good = np.isfinite(rows).all(axis=-1)
    with np.errstate(invalid="ignore", divide="ignore"):
        scale = (np.abs(rows).max(axis=-1) * (np.float32(1) / np.float32(127))).astype(np.float32)
        q = np.rint(rows / scale[..., None]).astype(np.float32)
    scale = np.where(good, scale, np.float32("nan"))
    q = np.where((scale > 0)[..., None], np.clip(q, -127, 127), 0)
    return q.astype(np.int8), scale

"""CPU oracle of the operators of a decode step of many requests (TEST INFRASTRUCTURE ONLY).

Plain float64 definitions: attention of one token over a shared prefix and a sequence's own tokens, low-rank adapters by row, and log
probabilities with entropy, ranks and most likely tokens.  Shares no code with the HIP path.
"""
import numpy as np

from oracle import paged


def group_prefix(b, group_cu, prefix_lens):
    """(first sequence, tokens) of the prefix that sequence b shares; (b, 0) if it shares none."""
    for g, n in enumerate(prefix_lens):
        if group_cu[g] <= b < group_cu[g + 1]:
            return group_cu[g], max(int(n), 0)
    return b, 0


def shared_attention(q, read, lens, group_cu, prefix_lens):
    """q [B, H, D] float64; read(b, t) -> (k [Hkv, D], v [Hkv, D]) float64 of what sequence b's table names for position t, or None.  Returns
    per sequence (out, spread, keys seen): paged.attention's of its last token."""
    result = []
    for b, L in enumerate(lens):
        first, P = group_prefix(b, group_cu, prefix_lens)
        rows = [read(first if t < P else b, t) for t in range(max(L, 0))]
        rows = [r for r in rows if r is not None]
        if not rows:
            zero = np.zeros(q.shape[1:])
            result.append((zero, zero, np.zeros((0, 1, q.shape[2]))))
            continue
        k, v = np.stack([r[0] for r in rows]), np.stack([r[1] for r in rows])
        out, spread = paged.attention(q[b:b + 1], k, v, [len(rows) - 1])
        result.append((out[0], spread[0], k))
    return result


def lora(base, x, a, b, row_adapter, scales=None):
    """(out, bound): base + s (x A^T) B^T per row, and what FP32 sums and the pairs of the middle product may be off by beside the result's rounding."""
    base, x, a, b = (np.asarray(t).astype(np.float64) for t in (base, x, a, b))
    out, off = base.copy(), np.zeros_like(base)
    K, r = x.shape[1], a.shape[1]
    for m, n in enumerate(row_adapter):
        if not 0 <= n < a.shape[0]:
            continue
        s = 1.0 if scales is None else float(scales[n])
        with np.errstate(invalid="ignore"):
            h, size = a[n] @ x[m], np.abs(a[n]) @ np.abs(x[m])
            e = (K + 4) * 2.0 ** -24 * size + 2.0 ** -22 * np.abs(h) + 2.0 ** -39 * np.abs(h).max()
            out[m] += s * (b[n] @ h)
            off[m] = abs(s) * (np.abs(b[n]) @ (e + (2 * r + 8) * 2.0 ** -24 * np.abs(h)))
    return out, off + 2.0 ** -23 * (np.abs(base) + np.abs(out))


def in_order(x):
    """Indices of x in descending order, equal ones by index."""
    return np.lexsort((np.arange(len(x)), -x))


def logprobs(x, token, top):
    """(logprob, rank, entropy, ids, their logprobs, mean distance to the largest) of one row of logits; NaN, 0 and -1 where nothing is defined."""
    x = np.asarray(x).astype(np.float64) + 0.0
    nan = float("nan")
    if np.isnan(x).any() or not np.isfinite(x.max()):
        return nan, 0, nan, np.full(top, -1), np.full(top, nan), 0.0
    with np.errstate(divide="ignore", invalid="ignore"):
        d = x - x.max()
        e = np.exp(d)
        total = e.sum()
        logp = d - np.log(total)
        dist = float(np.where(e > 0, -e * np.where(e > 0, d, 0.0), 0.0).sum() / total)
        entropy = np.log(total) + dist
    order = in_order(x)
    known = 0 <= token < len(x)
    rank = int(np.nonzero(order == token)[0][0]) + 1 if known else 0
    return logp[token] if known else nan, rank, entropy, order[:top], logp[order[:top]], dist

"""CPU oracle of the operators around the paged KV4 cache (TEST INFRASTRUCTURE ONLY).

Plain float64 definitions: norm and rotation of heads, attention of ragged batches through a sliding window with first tokens that
stay visible, and the page arithmetic of a block table.  The quantizer is oracle/kv4.py's.  Shares no code with the HIP path.
"""
import numpy as np

from oracle import kv4

PAGE = 64


def turn_heads(x_fp16, gamma_fp16, eps, angles, positions, interleaved):
    """x_fp16 [M, heads, D], one position per row -> the same in FP16: x gamma / sqrt(mean(x^2) + eps) where gamma is given, then the
    rotation by angles [rows, rot] float32 (cosines, sines; None: none), in float64, converted to float32 and that to
    float16."""
    y = np.asarray(x_fp16, dtype=np.float16).astype(np.float64)
    if gamma_fp16 is not None:
        y = y / np.sqrt((y * y).mean(axis=-1, keepdims=True) + eps) * np.asarray(gamma_fp16, dtype=np.float16).astype(np.float64)
    if angles is not None:
        rot = angles.shape[1]
        row = angles[np.clip(positions, 0, angles.shape[0] - 1)].astype(np.float64)[:, None, :]
        c, s = row[..., :rot // 2], row[..., rot // 2:]
        a_at, b_at = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
        a, b = y[..., a_at].copy(), y[..., b_at].copy()
        y[..., a_at], y[..., b_at] = a * c - b * s, b * c + a * s
    if gamma_fp16 is None and angles is None:
        return np.asarray(x_fp16, dtype=np.float16)
    with np.errstate(over="ignore"):
        return y.astype(np.float32).astype(np.float16)


def rows_of(cu, starts, M):
    """(sequence, position) of each of M rows; sequence -1 where a row belongs to none."""
    seq, pos = np.full(M, -1), np.zeros(M, dtype=np.int64)
    for b in range(len(cu) - 1):
        for row in range(max(cu[b], 0), min(cu[b + 1], M)):
            seq[row], pos[row] = b, (0 if starts is None else starts[b]) + row - cu[b]
    return seq, pos


def place(table, pages, b, t):
    """(page, token in it) of position t of sequence b, or None."""
    if not 0 <= t < PAGE * table.shape[1]:
        return None
    page = int(table[b, t // PAGE])
    return (page, t % PAGE) if 0 <= page < pages else None


def visible(p, t, window, sinks):
    return t <= p and (window == 0 or t > p - window or t < sinks)


def attention(q, k, v, positions, window=0, sinks=0, held=None):
    """q [n, H, D] at `positions` [n] over k, v [t, Hkv, D] float64; held [t]: tokens that exist.  Returns (out, spread): float64
    [n, H, D], and the same sum over |v|, which bounds what rounding the weights can do."""
    n, H, D = q.shape
    r = H // k.shape[1]
    out, spread = np.zeros((n, H, D)), np.zeros((n, H, D))
    t = np.arange(k.shape[0])
    for i in range(n):
        see = (t <= positions[i]) & ((window == 0) | (t > positions[i] - window) | (t < sinks))
        if held is not None:
            see &= held
        if not see.any():
            continue
        for h in range(H):
            s = k[see, h // r] @ q[i, h] / np.sqrt(float(D))
            p = np.exp(s - s.max())
            p /= p.sum()
            out[i, h], spread[i, h] = p @ v[see, h // r], p @ np.abs(v[see, h // r])
    return out, spread


def quantized(x_fp16):
    """What the cache holds for FP16 vectors: float64."""
    return kv4.kv4_dequantize(*kv4.kv4_quantize(x_fp16))

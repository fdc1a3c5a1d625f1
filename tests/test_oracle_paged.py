"""The paged oracle against numbers worked out by hand, and against the contiguous oracle."""
import numpy as np
import pytest

from oracle import kv4, paged


def test_rotation_by_hand():
    x = np.zeros((1, 1, 4), dtype=np.float16)
    x[0, 0] = [1, 2, 3, 4]
    quarter = np.array([[0, 1, 1, 0]], dtype=np.float32)             # pair 0 by a quarter turn, pair 1 not at all: cos, cos, sin, sin
    assert paged.turn_heads(x, None, 0.0, quarter, np.array([0]), False)[0, 0].tolist() == [-3, 2, 1, 4]      # (1, 3) -> (-3, 1)
    assert paged.turn_heads(x, None, 0.0, quarter, np.array([0]), True)[0, 0].tolist() == [-2, 1, 3, 4]       # (1, 2) -> (-2, 1)
    assert paged.turn_heads(x, None, 0.0, quarter, np.array([7]), True)[0, 0].tolist() == [-2, 1, 3, 4]       # past the table: its last row
    g = np.array([2, 1, 1, 1], dtype=np.float16)
    y = paged.turn_heads(x, g, 0.5, None, np.array([0]), False)[0, 0]
    assert np.allclose(y, np.array([2, 2, 3, 4]) / np.sqrt(7.5 + 0.5), rtol=2 ** -11)


def test_rows_and_places():
    seq, pos = paged.rows_of([1, 3, 3, 4], [10, 5, 0], 6)
    assert seq.tolist() == [-1, 0, 0, 2, -1, -1] and pos.tolist() == [0, 10, 11, 0, 0, 0]
    table = np.array([[4, -1, 9]])
    assert paged.place(table, 5, 0, 63) == (4, 63) and paged.place(table, 5, 0, 64) is None
    assert paged.place(table, 5, 0, 128) is None and paged.place(table, 5, 0, 192) is None and paged.place(table, 5, 0, -1) is None


@pytest.mark.parametrize("window,sinks", [(0, 0), (5, 0), (5, 2), (1, 0), (40, 3)])
def test_attention_against_the_contiguous_oracle(window, sinks):
    rng = np.random.default_rng(3)
    L, H, Hkv, D = 23, 4, 2, 16
    k, v, q = (rng.standard_normal(s).astype(np.float16) for s in ((1, Hkv, L, D), (1, Hkv, L, D), (1, H, D)))
    kq, vq = kv4.kv4_quantize(k), kv4.kv4_quantize(v)
    out, spread = paged.attention(q.astype(np.float64), kv4.kv4_dequantize(*kq)[0].swapaxes(0, 1), kv4.kv4_dequantize(*vq)[0].swapaxes(0, 1),
                                  [L - 1], window, sinks)
    see = [t for t in range(L) if paged.visible(L - 1, t, window, sinks)]
    pick = lambda x: tuple(a[:, :, see] for a in x)                  # noqa: E731  (the visible tokens alone, seen whole)
    assert np.allclose(out, kv4.attention_decode(q, *pick(kq), *pick(vq), [len(see)]), atol=1e-12)
    assert (spread >= np.abs(out) - 1e-12).all()
    none, _ = paged.attention(q.astype(np.float64), kv4.kv4_dequantize(*kq)[0].swapaxes(0, 1), kv4.kv4_dequantize(*vq)[0].swapaxes(0, 1), [-1], window, sinks)
    assert not none.any()

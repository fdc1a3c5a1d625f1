"""The paged KV4 cache and prompt attention on the GPU against the float64 oracle.

Queries and keys after norm and rotation, codes, scales and zeros are bit-exact.  Attention is bounded term by term:
    |got - ref| <= 2^-11 |ref|                      the result's rounding to FP16
                 + 2^-11 sum_t p_t |v_t|            every softmax weight's (decode: weight times value scale's), half a step each
                 + (2 e + 2^-20) sum_t p_t |v_t|    errors e of the scores, in weights and in their sum; exp2 and FP32 sums
                 + n 2^-25 max|v|                   weights below FP16's normal numbers; the largest weight is at least 1
  with e = 130 2^-24 max_t sum_d |q_d k_td| / sqrt(128), the FP32 sum of 128 products in any order.
"""
import numpy as np
import pytest
import torch

from oracle import kv4, paged
from paper_2405_04532_amd import api, workloads as wl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
D, PAGE = 128, 64


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _heads(rows, heads, seed, stream=3, gain=8.0):
    """[rows, heads, 128] FP16 on the GPU, two large channels in every head."""
    k, v = wl.make_kv(1, heads, rows, D, seed, DEV, gain=gain)
    return (k if stream == 3 else v)[0].transpose(0, 1).contiguous()


def _tables(totals, width, seed, spare=2):
    """Pages of the sequences in any order; -1 behind them."""
    need = [-(-t // PAGE) for t in totals]
    pages = sum(need) + spare
    perm = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table, at = torch.full((len(totals), width), -1, dtype=torch.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n]
        at += n
    return table.to(DEV), pages


def _codes(pool, table, pages, Hkv, B, width):
    """Codes, scales and zeros of every place of a table of valid pages, through the contiguous cache's own unpacking."""
    page = pool.view(pages, Hkv, 8704)[table.long().clamp(min=0)]          # [B, width, Hkv, 8704]
    return [t.cpu().numpy() for t in api.kv4_unpack(page.transpose(1, 2).contiguous().view(-1), B, Hkv, width * PAGE)]


def _same(a, b):
    a, b = (x.cpu().numpy() if torch.is_tensor(x) else x for x in (a, b))
    nan = np.isnan(a) & np.isnan(b)
    return bool(((a.view(np.uint16) == b.view(np.uint16)) | nan).all())


# ------------------------------------------------------------------------------------------------------------------
# Norm, rotation, append
# ------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("H,Hkv,rot,near,norm,new,starts", [
    (4, 2, 128, False, False, [1, 1, 1], [0, 63, 64]),
    (4, 4, 128, True, True, [5, 0, 67, 1], [2, 9, 61, 127]),
    (7, 1, 64, False, True, [130], [0]),
    (3, 3, 64, True, False, [3, 2], [7, 100]),
    (2, 1, 96, False, False, [9, 40], [1, 30]),
    (5, 1, 16, False, True, [4, 4, 4, 4], [0, 1, 2, 3]),
    (4, 2, 0, False, False, [33, 1], [0, 64]),
    (4, 2, 0, False, True, [12], [50]),
    (2, 2, 128, False, False, [1] * 70, list(range(70))),
    (8, 8, 128, False, True, [300, 1, 17], [0, 200, 40])])
def test_append(H, Hkv, rot, near, norm, new, starts):
    B, M = len(new), sum(new)
    width = max((s + n + PAGE - 1) // PAGE for s, n in zip(starts, new)) + 1
    table, pages = _tables([width * PAGE] * B, width, 5)
    qkv = torch.cat((_heads(M, H, 11), _heads(M, Hkv, 12), _heads(M, Hkv, 13, 4)), dim=1)       # a fused projection: strided slices
    q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    v[0, 0], k[M // 2, 0] = 0, 0                            # vectors of zeros
    angles = api.rope_angles(width * PAGE, rot, device=DEV) if rot else None
    gq = (1 + 0.1 * _heads(1, 1, 14)[0, 0]) if norm else None
    gk = (1 + 0.1 * _heads(1, 1, 15)[0, 0]) if norm else None
    cu = np.concatenate(([0], np.cumsum(new)))
    pool = api.kv4_new_pool(pages, Hkv, DEV)
    pool += 7
    before = _codes(pool, table, pages, Hkv, B, width)
    qo, ko = api.qk_rope_kv4_append(q, k, v, pool, table, _ints(cu), _ints(starts), angles, gq, gk, 1e-5, near, want_k=True)
    seq, pos = paged.rows_of(cu, starts, M)
    host = lambda t: None if t is None else t.cpu().numpy()                # noqa: E731
    want_q = paged.turn_heads(host(q), host(gq), 1e-5, host(angles), pos, near)
    want_k = paged.turn_heads(host(k), host(gk), 1e-5, host(angles), pos, near)
    assert _same(qo, want_q) and _same(ko, want_k)
    # what the pages hold: the new tokens' numbers, and what was there everywhere else
    after = _codes(pool, table, pages, Hkv, B, width)
    want = [x.copy() for x in before]
    for x, at in ((want_k, 0), (host(v), 3)):
        c, s, z = kv4.kv4_quantize(x)
        want[at][seq, :, pos], want[at + 1][seq, :, pos], want[at + 2][seq, :, pos] = c, s, z
    for got, exp in zip(after, want):
        assert _same(got, exp) if got.dtype == np.float16 else np.array_equal(got, exp)
    # and back: dequantized, rounded once
    gk_, gv_ = api.kv4_paged_gather(pool, table, _ints(cu), _ints(starts), M, Hkv)
    assert _same(gk_, paged.quantized(want_k).astype(np.float16)) and _same(gv_, paged.quantized(host(v)).astype(np.float16))
    # in place, into the projection itself
    pool2 = api.kv4_new_pool(pages, Hkv, DEV)
    a, b = api.qk_rope_kv4_append(q, k, v, pool2, table, _ints(cu), _ints(starts), angles, gq, gk, 1e-5, near, q_out=q, k_out=k)
    assert a.data_ptr() == q.data_ptr() and b.data_ptr() == k.data_ptr()
    assert _same(q.contiguous(), want_q) and _same(k.contiguous(), want_k) and _same(v.contiguous(), host(v))
    assert _same(api.kv4_paged_gather(pool2, table, _ints(cu), _ints(starts), M, Hkv)[0], gk_)


def test_append_drops_what_has_no_place_and_leaves_other_rows():
    """Positions before and behind the table, pages that are none, rows of no sequence, an empty batch of rows."""
    Hkv, width, pages = 2, 2, 3
    table = _ints([[2, -1], [7, 0], [1, 1 << 30]])
    cu, starts = [1, 9, 75, 77], [-3, 60, 126]                             # rows 0 and 77, 78 belong to none
    M = 79
    k, v, q = _heads(M, Hkv, 21), _heads(M, Hkv, 22, 4), _heads(M, 3, 23)
    angles = api.rope_angles(100, device=DEV)                              # positions past it take its last row
    pool = torch.full((pages * Hkv * 8704,), 9, dtype=torch.uint8, device=DEV)
    qo, ko = torch.full_like(q, 5.0), torch.full_like(k, 6.0)
    api.qk_rope_kv4_append(q, k, v, pool, table, _ints(cu), _ints(starts), angles, q_out=qo, k_out=ko)
    seq, pos = paged.rows_of(cu, starts, M)
    live = seq >= 0
    ang = angles.cpu().numpy()
    want_k = paged.turn_heads(k.cpu().numpy(), None, 0, ang, pos, False)
    assert _same(qo[live], paged.turn_heads(q.cpu().numpy(), None, 0, ang, pos, False)[live]) and _same(ko[live], want_k[live])
    assert bool((qo[~live] == 5).all()) and bool((ko[~live] == 6).all())
    want = np.full((pages, Hkv, 64, 128), -1)
    expect = {}
    for row in np.flatnonzero(live):
        at = paged.place(table.cpu().numpy(), pages, seq[row], pos[row])
        if at:
            expect[at] = row
    got = _codes(pool, torch.arange(pages, device=DEV)[:, None], pages, Hkv, pages, 1)
    kc, vc = kv4.kv4_quantize(want_k)[0], kv4.kv4_quantize(v.cpu().numpy())[0]
    blank = _codes(torch.full_like(pool, 9), torch.arange(pages, device=DEV)[:, None], pages, Hkv, pages, 1)
    for page in range(pages):
        for t in range(64):
            row = expect.get((page, t))
            assert np.array_equal(got[0][page, :, t], blank[0][page, :, t] if row is None else kc[row]), (page, t)
            assert np.array_equal(got[3][page, :, t], blank[3][page, :, t] if row is None else vc[row]), (page, t)
    assert len(expect) == 5 + 62 and want.size
    # read back: zeros where there is no page, other rows as they were
    gk, gv = torch.full((M, Hkv, D), 3.0, dtype=torch.float16, device=DEV), torch.full((M, Hkv, D), 4.0, dtype=torch.float16, device=DEV)
    api.kv4_paged_gather(pool, table, _ints(cu), _ints(starts), M, Hkv, gk, gv)
    on = np.array([i in expect.values() for i in range(M)])
    assert bool((gk[~live] == 3).all()) and bool((gv[~live] == 4).all())
    assert not gk[torch.from_numpy(live & ~on).to(DEV)].any() and not gv[torch.from_numpy(live & ~on).to(DEV)].any()
    assert _same(gk[torch.from_numpy(on).to(DEV)], paged.quantized(want_k[on]).astype(np.float16))
    # no rows at all
    none = torch.empty((0, Hkv, D), dtype=torch.float16, device=DEV)
    api.kv4_paged_append(pool, none, none, table, _ints([0, 0, 0, 0]))
    assert api.kv4_paged_gather(pool, table, _ints([0, 0, 0, 0]), None, 0, Hkv)[0].shape == (0, Hkv, D)


def test_append_rounding():
    """Results at and next to midpoints of FP16 numbers, subnormal and overflowing ones, infinities and NaN: the float64 evaluation
    by way of float32."""
    M, H = 64, 4
    g = torch.Generator().manual_seed(8)
    x = (torch.randn(M, H, D, generator=g) * torch.exp2(torch.randint(-24, 16, (M, H, 1), generator=g).float())).half()
    x[0, 0, 0], x[1, 1, 3], x[2, 2, 2] = float("inf"), float("nan"), -float("inf")
    x[3] = torch.arange(512).view(4, 128).half() / 512 * 2.0 ** -14
    angles = torch.zeros(M, D)
    angles[:, :64] = 1.0                                                   # no turn: numbers come back as they are
    angles[1::3, :64], angles[1::3, 64:] = 0.5, 0.5                        # sums at midpoints
    angles[2::3] = torch.rand(angles[2::3].shape, generator=g) * 3 - 1
    angles[5, :64] = 1.0 + 2.0 ** -11                                      # beside midpoints of odd numbers
    angles[8, :64] = 1.0 + 2.0 ** -11 + 2.0 ** -23
    angles[11, :64] = 1.0 + 2.0 ** -11 - 2.0 ** -23
    for near in (False, True):
        kv = torch.zeros(M, 1, D, dtype=torch.float16, device=DEV)
        pool, table = api.kv4_new_pool(1, 1, DEV), _ints([[0]])
        qo, _ = api.qk_rope_kv4_append(x.to(DEV), kv, kv, pool, table, _ints([0, M]), None, angles.to(DEV), interleaved=near)
        with np.errstate(invalid="ignore"):
            want = paged.turn_heads(x.numpy(), None, 0, angles.numpy(), np.arange(M), near)
        assert _same(qo, want)
        # the same behind a norm; heads of zeros without an eps are 0 / 0
        x[4] = 0
        gamma = (1 + torch.randn(D, generator=g)).half()
        for eps in (0.0, 1e-5, 3e4):
            qo, _ = api.qk_rope_kv4_append(x.to(DEV), kv, kv, pool, table, _ints([0, M]), None, angles.to(DEV), q_gamma=gamma.to(DEV), eps=eps, interleaved=near)
            with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
                want = paged.turn_heads(x.numpy(), gamma.numpy(), eps, angles.numpy(), np.arange(M), near)
            # bit for bit, but that in a head with an infinity 1 / sqrt is 0: the products are zeros whose sign goes by their order
            endless = np.isinf(x.numpy().astype(np.float32)).any(axis=-1)
            assert _same(qo.cpu().numpy()[~endless], want[~endless]) and np.array_equal(qo.cpu().numpy()[endless], want[endless], equal_nan=True)


@pytest.mark.parametrize("B", [1, 63, 64, 65, 130, 5000])
def test_append_and_gather_of_many_sequences(B):
    """Up to 64 sequences are looked up by the lanes of a wave, more by a search; empty ones among them, the same token count at both ends."""
    new = [(3 * b) % 4 for b in range(B - 1)] + [2]
    starts = [(17 * b) % 70 for b in range(B)]
    cu = np.concatenate(([0], np.cumsum(new)))
    M = int(cu[-1])
    table, pages = _tables([128] * B, 2, 9)
    q, k, v = _heads(M, 2, 61), _heads(M, 1, 62), _heads(M, 1, 63, 4)
    angles = api.rope_angles(80, device=DEV)
    pool = api.kv4_new_pool(pages, 1, DEV)
    qo, ko = api.qk_rope_kv4_append(q, k, v, pool, table, _ints(cu), _ints(starts), angles, want_k=True)
    seq, pos = paged.rows_of(cu, starts, M)
    want_k = paged.turn_heads(k.cpu().numpy(), None, 0, angles.cpu().numpy(), pos, False)
    assert _same(qo, paged.turn_heads(q.cpu().numpy(), None, 0, angles.cpu().numpy(), pos, False)) and _same(ko, want_k)
    gk, gv = api.kv4_paged_gather(pool, table, _ints(cu), _ints(starts), M, 1)
    assert _same(gk, paged.quantized(want_k).astype(np.float16)) and _same(gv, paged.quantized(v.cpu().numpy()).astype(np.float16))


# ------------------------------------------------------------------------------------------------------------------
# Decode attention
# ------------------------------------------------------------------------------------------------------------------
def _bound(q, k, ref, spread, n):
    r = q.shape[1] // k.shape[1]
    e = 0.0
    for h in range(q.shape[1]):
        if k.shape[0] and q.shape[0]:
            e = max(e, float((np.abs(k[:, h // r]) @ np.abs(q[:, h]).T).max()))
    e *= 130 * 2.0 ** -24 / np.sqrt(128.0)
    return 2.0 ** -11 * np.abs(ref) + (2.0 ** -11 + 2 * e + 2.0 ** -20) * spread, e


def _filled(lens, Hkv, width, seed, spare=2):
    """A pool with these sequences' tokens, and its dequantized keys and values."""
    table, pages = _tables(lens, width, seed, spare)
    M = sum(lens)
    k, v = _heads(max(M, 1), Hkv, seed), _heads(max(M, 1), Hkv, seed + 1, 4)
    cu = np.concatenate(([0], np.cumsum(lens)))
    pool = torch.full((pages * Hkv * 8704,), 0xFF, dtype=torch.uint8, device=DEV)      # NaN parameters where nothing is written
    api.kv4_paged_append(pool, k[:M].contiguous(), v[:M].contiguous(), table, _ints(cu))
    return pool, table, pages, cu, paged.quantized(k[:M].cpu().numpy()), paged.quantized(v[:M].cpu().numpy())


def _check_decode(out, q, kh, vh, cu, lens, window, sinks, held=None):
    got, qd = out.cpu().numpy().astype(np.float64), q.cpu().numpy().astype(np.float64)
    for b, L in enumerate(lens):
        k, v = kh[cu[b]:cu[b] + L], vh[cu[b]:cu[b] + L]
        ref, spread = paged.attention(qd[b:b + 1], k, v, [L - 1], window, sinks, None if held is None else held[b][:L])
        tol, _ = _bound(qd[b:b + 1], k, ref, spread, L)
        tol = tol + L * 15 * 2.0 ** -25 + 2.0 ** -25
        assert (np.abs(got[b] - ref[0]) <= tol[0]).all(), (b, L, float(np.abs(got[b] - ref[0]).max()))
        if L == 0:
            assert not got[b].any()


@pytest.mark.parametrize("H,Hkv", [(4, 4), (8, 2), (7, 1), (16, 1), (9, 1)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (50, 0), (33, 4), (64, 70), (500, 3)])
def test_decode(H, Hkv, window, sinks):
    lens = [0, 1, 5, 31, 32, 33, 63, 64, 65, 130, 200, 257]
    width = 6
    pool, table, pages, cu, kh, vh = _filled(lens, Hkv, width, 31 + H)
    q = wl.make_queries(len(lens), H, D, 33, DEV)
    out = api.kv4_paged_attention_decode(q, pool, table, _ints(lens), Hkv, window=window, sinks=sinks)
    _check_decode(out, q, kh, vh, cu, lens, window, sinks)


@pytest.mark.parametrize("B,H,Hkv,lens,window,sinks", [
    (1, 4, 1, [4097], 0, 0), (1, 16, 1, [3000], 0, 0), (2, 8, 2, [2049, 1], 0, 0), (3, 4, 4, [900, 0, 511], 0, 0), (2, 4, 2, [5000, 130], 2000, 4),
    (1, 8, 1, [4200], 700, 100), (5, 6, 2, [64, 1500, 257, 1024, 3], 0, 0)])
def test_decode_shared_by_workgroups(B, H, Hkv, lens, window, sinks):
    """Long sequences with few heads, in a workspace that other calls use in turn; the same bits every time, and in a graph."""
    width = max(-(-n // PAGE) for n in lens) + 1
    pool, table, pages, cu, kh, vh = _filled(lens, Hkv, width, 51)
    q = wl.make_queries(B, H, D, 53, DEV)
    need = api.kv4_paged_attention_workspace_bytes(B, H, Hkv, width, window, sinks)
    assert need > api.GEMM_COUNTER_BYTES
    ws = api.new_workspace(need, DEV)
    ws[api.GEMM_COUNTER_BYTES:] = 0xFF                                     # only the counters have to be zero
    seq = _ints(lens)
    out = api.kv4_paged_attention_decode(q, pool, table, seq, Hkv, window, sinks, workspace=ws)
    _check_decode(out, q, kh, vh, cu, lens, window, sinks)
    for _ in range(5):
        again = api.kv4_paged_attention_decode(q, pool, table, seq, Hkv, window, sinks, workspace=ws)
        assert _same(again, out)
    assert not ws[:api.GEMM_COUNTER_BYTES].any()
    alone = api.kv4_paged_attention_decode(q, pool, table, seq, Hkv, window, sinks)
    _check_decode(alone, q, kh, vh, cu, lens, window, sinks)
    # two captured graphs that take turns in one workspace, with shorter sequences in the second
    short = _ints([max(n // 2, 0) for n in lens])
    outs, graphs = [torch.zeros_like(out), torch.zeros_like(out)], []
    side = torch.cuda.Stream()
    for o, s in zip(outs, (seq, short)):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            api.kv4_paged_attention_decode(q, pool, table, s, Hkv, window, sinks, out=o, workspace=ws)
        graphs.append(graph)
    want = [out, api.kv4_paged_attention_decode(q, pool, table, short, Hkv, window, sinks, workspace=ws)]
    for _ in range(3):
        for o in outs:
            o.zero_()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        assert _same(outs[0], want[0]) and _same(outs[1], want[1])
    with pytest.raises(api.QoqError):
        api.kv4_paged_attention_decode(q, pool, table, seq, Hkv, window, sinks, workspace=ws[:need - 16])


def test_decode_many_splits_of_garbage_lengths_and_pages():
    """Lengths past the table and below zero, pages that are none, in the middle and all of them."""
    B, H, Hkv, width = 4, 4, 2, 40
    full = width * PAGE
    pool, table, pages, cu, kh, vh = _filled([full, 700, 640, 100], Hkv, width, 61)
    holes = table.clone()
    holes[1, 3] = pages
    holes[1, 7] = -5
    holes[2] = 1 << 30
    held = [np.ones(full, dtype=bool) for _ in range(B)]
    held[1][3 * 64:4 * 64] = held[1][7 * 64:8 * 64] = False
    held[2][:] = False
    q = wl.make_queries(B, H, D, 63, DEV)
    ws = api.new_workspace(api.kv4_paged_attention_workspace_bytes(B, H, Hkv, width), DEV)
    for room in (None, ws):
        out = api.kv4_paged_attention_decode(q, pool, holes, _ints([1 << 30, 700, 640, -9]), Hkv, workspace=room)
        _check_decode(out, q, kh, vh, cu, [full, 700, 640, 0], 0, 0, held)
        assert not out[2:].any()


def test_decode_window_does_not_need_the_pages_in_front_of_it():
    """Pages between the sinks and the window are given away: their entries are gone, their bytes are NaN."""
    L, H, Hkv = 1000, 4, 1
    pool, table, pages, cu, kh, vh = _filled([L], Hkv, 16, 71)
    q = wl.make_queries(1, H, D, 73, DEV)
    want = api.kv4_paged_attention_decode(q, pool, table, _ints([L]), Hkv, window=200, sinks=4)
    gone = table.clone()
    gone[0, 1:(L - 200) // 64] = -1
    pool.view(pages, -1)[table[0, 1:(L - 200) // 64].long()] = 0xFF
    assert _same(api.kv4_paged_attention_decode(q, pool, gone, _ints([L]), Hkv, window=200, sinks=4), want)
    _check_decode(want, q, kh, vh, cu, [L], 200, 4)


def test_decode_strided_queries_and_a_large_batch():
    B, H, Hkv = 150, 4, 2
    lens = [(37 * i) % 140 for i in range(B)]
    pool, table, pages, cu, kh, vh = _filled(lens, Hkv, 3, 81)
    fused = wl.make_queries(B, H + 3, D, 83, DEV)
    q = fused[:, 1:1 + H]
    out = api.kv4_paged_attention_decode(q, pool, table, _ints(lens), Hkv)
    _check_decode(out, q, kh, vh, cu, lens, 0, 0)


# ------------------------------------------------------------------------------------------------------------------
# Prompt attention
# ------------------------------------------------------------------------------------------------------------------
def _prompts(new, held, H, Hkv, seed, behind=0):
    total = [n + h for n, h in zip(new, held)]
    M, Mk = sum(new) + behind, sum(total) + behind
    q = _heads(max(M, 1), H, seed, 4)[:M].contiguous()
    k, v = _heads(max(Mk, 1), Hkv, seed + 1)[:Mk].contiguous(), _heads(max(Mk, 1), Hkv, seed + 2, 4)[:Mk].contiguous()
    return q, k, v, np.concatenate(([0], np.cumsum(new))), np.concatenate(([0], np.cumsum(total)))


def _check_prefill(out, q, k, v, cu_q, cu_k, window, sinks, rows=None):
    got, qd, kd, vd = (t.cpu().numpy().astype(np.float64) for t in (out, q, k, v))
    for b in range(len(cu_q) - 1):
        n, m = cu_q[b + 1] - cu_q[b], cu_k[b + 1] - cu_k[b]
        pick = np.arange(n) if rows is None or n <= rows else np.unique(np.concatenate((np.arange(4), np.linspace(0, n - 1, rows).astype(int), np.arange(n - 4, n))))
        kb, vb = kd[cu_k[b]:cu_k[b + 1]], vd[cu_k[b]:cu_k[b + 1]]
        qb = qd[cu_q[b]:cu_q[b + 1]][pick]
        ref, spread = paged.attention(qb, kb, vb, m - n + pick, window, sinks)
        tol, _ = _bound(qb, kb, ref, spread, m)
        tol = tol + m * 2.0 ** -25 * (np.abs(vb).max() if m else 0) + 2.0 ** -25
        have = got[cu_q[b]:cu_q[b + 1]][pick]
        assert (np.abs(have - ref) <= tol).all(), (b, float((np.abs(have - ref) - tol).max()))
        blind = m - n + pick < 0
        assert not have[blind].any()


@pytest.mark.parametrize("H,Hkv", [(2, 2), (4, 1), (7, 1), (6, 2), (40, 1), (64, 1)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (40, 0), (100, 5), (64, 70)])
def test_prefill(H, Hkv, window, sinks):
    new, held = [1, 0, 33, 64, 130, 3], [0, 5, 0, 1, 70, 200]
    q, k, v, cu_q, cu_k = _prompts(new, held, H, Hkv, 91 + H)
    out = api.attention_prefill(q, k, v, _ints(cu_q), _ints(cu_k), window=window, sinks=sinks)
    _check_prefill(out, q, k, v, cu_q, cu_k, window, sinks)


@pytest.mark.parametrize("new,held,H,Hkv,window,sinks", [([700], [0], 4, 4, 0, 0), ([515, 260], [300, 0], 8, 2, 0, 0), ([300], [1500], 4, 1, 256, 4),
                                                         ([1], [2000], 8, 2, 0, 0), ([3, 1, 2], [1999, 900, 64], 8, 1, 0, 0), ([2], [3500], 4, 4, 1500, 64),
                                                         ([1], [6000], 4, 1, 0, 0), ([40, 1, 0, 9], [100, 5000, 70, 0], 7, 1, 0, 0), ([65], [2000], 2, 1, 900, 130)])
def test_prefill_longer(new, held, H, Hkv, window, sinks):
    q, k, v, cu_q, cu_k = _prompts(new, held, H, Hkv, 95)
    need = api.attention_prefill_workspace_bytes(len(q), len(k), len(new), H, Hkv, window, sinks)
    ws = api.new_workspace(need, DEV)
    out = api.attention_prefill(q, k, v, _ints(cu_q), _ints(cu_k), window=window, sinks=sinks)
    _check_prefill(out, q, k, v, cu_q, cu_k, window, sinks, rows=40)
    shared = api.attention_prefill(q, k, v, _ints(cu_q), _ints(cu_k), window=window, sinks=sinks, workspace=ws)
    _check_prefill(shared, q, k, v, cu_q, cu_k, window, sinks, rows=40)
    for _ in range(3):
        assert _same(api.attention_prefill(q, k, v, _ints(cu_q), _ints(cu_k), window=window, sinks=sinks, workspace=ws), shared)
    assert not ws[:api.GEMM_COUNTER_BYTES].any()
    if need:                                               # contents behind the counters are irrelevant; a smaller one is refused
        ws[api.GEMM_COUNTER_BYTES:] = 0xFF
        assert _same(api.attention_prefill(q, k, v, _ints(cu_q), _ints(cu_k), window=window, sinks=sinks, workspace=ws), shared)
        with pytest.raises(api.QoqError):
            api.attention_prefill(q, k, v, _ints(cu_q), _ints(cu_k), window=window, sinks=sinks, workspace=ws[:need - 16])


def test_prefill_more_queries_than_tokens_and_rows_of_no_sequence():
    """Queries in front of a sequence's first token see nothing; rows behind the last sequence stay as they were."""
    H, Hkv = 4, 2
    q, k, v, _, _ = _prompts([80], [80], H, Hkv, 97)
    cu_q, cu_k = [2, 40, 60, 75], [0, 10, 10, 90]                          # 38 queries of 10 tokens, 20 of none, 15 of 80
    out = torch.full((80, H, D), 9.0, dtype=torch.float16, device=DEV)
    api.attention_prefill(q, k, v, _ints(cu_q), _ints(cu_k), out=out)
    _check_prefill(out, q, k, v, cu_q, cu_k, 0, 0)
    assert bool((out[:2] == 9).all()) and bool((out[75:] == 9).all()) and not out[40:60].any()
    out.fill_(9.0)
    api.attention_prefill(q, k, v, _ints([0, 200]), _ints([-4, 500]), out=out)      # bounds past the rows: the nearest ones
    _check_prefill(out, q, k, v, [0, 80], [0, 160], 0, 0)
    none = torch.empty((0, Hkv, D), dtype=torch.float16, device=DEV)
    assert not api.attention_prefill(q, none, none, _ints([0, 80]), _ints([0, 0])).any()


@pytest.mark.parametrize("B", [1, 64, 65, 200])
def test_prefill_of_many_sequences(B):
    """More sequences than the lanes of a wave, empty ones among them; queries in front of the first row of the first sequence."""
    new, held = [(5 * b) % 4 for b in range(B - 1)] + [3], [(11 * b) % 90 for b in range(B)]
    q, k, v, cu_q, cu_k = _prompts(new, held, 4, 2, 113)
    ws = api.new_workspace(api.attention_prefill_workspace_bytes(len(q), len(k), B, 4, 2), DEV)
    for room in (None, ws):
        out = api.attention_prefill(q, k, v, _ints(cu_q), _ints(cu_k), window=40, sinks=2, workspace=room)
        _check_prefill(out, q, k, v, cu_q, cu_k, 40, 2)


def test_prefill_strided_slices():
    H, Hkv, M = 8, 2, 150
    qkv = torch.cat((_heads(M, H, 101, 4), _heads(M, Hkv, 102), _heads(M, Hkv, 103, 4)), dim=1)
    q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    cu = [0, 90, M]
    out = api.attention_prefill(q, k, v, _ints(cu), _ints(cu))
    assert _same(out, api.attention_prefill(q.contiguous(), k.contiguous(), v.contiguous(), _ints(cu), _ints(cu)))
    _check_prefill(out, q, k, v, cu, cu, 0, 0)


@pytest.mark.parametrize("window,sinks", [(0, 0), (30, 2)])
def test_prefill_infinities_and_nan_reach_only_the_queries_that_see_them(window, sinks):
    """Values and keys that are not finite at some tokens: earlier queries, and later ones whose window has passed, are as without: within the
    bound above of the same float64 result.  (Rows that share a tile with such a value are summed in another order than without it,
    so their bits may differ; the bound holds for any order.)"""
    H, Hkv, T = 2, 1, 200
    q, k, v, cu, _ = _prompts([T], [0], H, Hkv, 105)
    clean = api.attention_prefill(q, k, v, _ints(cu), _ints(cu), window=window, sinks=sinks)
    spots = {70: (3, float("inf")), 71: (4, float("nan")), 100: (5, -float("inf")), 101: (3, -float("inf")), 130: (5, -float("inf"))}
    v2 = v.clone()
    for t, (d, x) in spots.items():
        v2[t, 0, d] = x
    got = api.attention_prefill(q, k, v2, _ints(cu), _ints(cu), window=window, sinks=sinks).cpu().numpy().astype(np.float64)
    clean = clean.cpu().numpy()
    kd, vd, qd = (x.cpu().numpy().astype(np.float64) for x in (k, v, q))
    ref, spread = paged.attention(qd, kd, vd, np.arange(T), window, sinks)
    tol, _ = _bound(qd, kd, ref, spread, T)
    tol = tol + T * 2.0 ** -25 * np.abs(vd).max() + 2.0 ** -25
    assert (np.abs(clean - ref) <= tol).all()
    for i in range(T):
        for d in (2, 3, 4, 5):
            seen = [x for t, (dd, x) in spots.items() if dd == d and paged.visible(i, t, window, sinks)]
            if not seen:
                assert (np.abs(got[i, :, d] - ref[i, :, d]) <= tol[i, :, d]).all(), (i, d)
            elif any(np.isnan(seen)) or len(set(seen)) > 1:
                assert np.isnan(got[i, :, d]).all(), (i, d)
            else:                                                          # (a weight may be zero: NaN)
                ok = (got[i, :, d] == seen[0]) | np.isnan(got[i, :, d])
                assert ok.all(), (i, d)
    k2 = k.clone()
    k2[150] = float("nan")
    got = api.attention_prefill(q, k2, v, _ints(cu), _ints(cu), window=window, sinks=sinks).cpu().numpy()
    for i in range(T):
        if paged.visible(i, 150, window, sinks):
            assert np.isnan(got[i]).all()
        else:
            assert (np.abs(got[i].astype(np.float64) - ref[i]) <= tol[i]).all()


def test_prefill_values_that_are_not_finite_where_workgroups_share_keys():
    """The rows next to such values are done again by the workgroup that joins the others' sums."""
    H, Hkv, T = 2, 1, 900
    q, k, v, cu, _ = _prompts([T], [0], H, Hkv, 109)
    ws = api.new_workspace(api.attention_prefill_workspace_bytes(T, T, 1, H, Hkv), DEV)
    assert ws.numel() > api.GEMM_COUNTER_BYTES
    v2 = v.clone()
    v2[130, 0, 7], v2[700, 0, 8] = float("inf"), float("nan")
    got = api.attention_prefill(q, k, v2, _ints(cu), _ints(cu), workspace=ws).cpu().numpy().astype(np.float64)
    kd, vd, qd = (x.cpu().numpy().astype(np.float64) for x in (k, v, q))
    ref, spread = paged.attention(qd, kd, vd, np.arange(T))
    tol, _ = _bound(qd, kd, ref, spread, T)
    tol = tol + T * 2.0 ** -25 * np.abs(vd).max() + 2.0 ** -25
    hit = np.zeros(got.shape, dtype=bool)
    hit[130:, :, 7], hit[700:, :, 8] = True, True
    assert (np.abs(got - ref) <= tol)[~hit].all() and not np.isfinite(got[hit]).any()
    assert np.isnan(got[700:, :, 8]).all()
    assert _same(api.attention_prefill(q, k, v2, _ints(cu), _ints(cu), workspace=ws), got.astype(np.float16))
    assert not ws[:api.GEMM_COUNTER_BYTES].any()


def test_scores_of_any_size():
    """Scores far below zero for every token, and differences that leave one token alone."""
    H, Hkv, T = 2, 1, 100
    q, k, v, cu, _ = _prompts([T], [0], H, Hkv, 107)
    for scale in (3000.0, -3000.0):
        qs = torch.ones_like(q) * 50
        ks = (torch.sign(torch.ones_like(k)) * scale + k).half()
        out = api.attention_prefill(qs, ks, v, _ints(cu), _ints(cu))
        assert bool(torch.isfinite(out).all())
        got, kd, vd = out.cpu().numpy().astype(np.float64), ks.cpu().numpy().astype(np.float64), v.cpu().numpy().astype(np.float64)
        ref, spread = paged.attention(qs.cpu().numpy().astype(np.float64), kd, vd, np.arange(T))
        e = 130 * 2.0 ** -24 * 50 * 3100 * 128 / np.sqrt(128.0)             # scores of 1.7e6: FP32 holds them to about 0.1
        tol = 2.0 ** -11 * np.abs(ref) + (2.0 ** -11 + 2 * (np.exp(e) - 1)) * spread + T * 2.0 ** -25 * np.abs(vd).max()
        assert (np.abs(got - ref) <= tol).all()


# ------------------------------------------------------------------------------------------------------------------
# Together, as a serving program runs them
# ------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("H,Hkv,window,sinks", [(4, 4, 0, 0), (8, 2, 90, 4)])
def test_prompt_continued_prompt_and_generation(H, Hkv, window, sinks):
    """Two prompts, one of them in two parts (the second behind what the cache holds), then tokens one at a time."""
    B, width, eps = 2, 5, 1e-6
    lens, parts, steps = [150, 90], [[100, 90], [50, 0]], 3
    total = [n + steps for n in lens]
    table, pages = _tables([width * PAGE] * B, width, 7)
    qkv = [torch.cat((_heads(n, H, 200 + b), _heads(n, Hkv, 210 + b), _heads(n, Hkv, 220 + b, 4)), dim=1) for b, n in enumerate(total)]
    gq, gk = 1 + 0.1 * _heads(1, 1, 231)[0, 0], 1 + 0.1 * _heads(1, 1, 232)[0, 0]
    angles = api.rope_angles(width * PAGE, device=DEV)
    pool = api.kv4_new_pool(pages, Hkv, DEV)
    ws = api.new_workspace(max(api.kv4_paged_attention_workspace_bytes(B, H, Hkv, width, window, sinks),
                               api.attention_prefill_workspace_bytes(400, 400, B, H, Hkv, window, sinks)), DEV)
    turned = []
    for b, n in enumerate(total):
        x, pos = qkv[b].cpu().numpy(), np.arange(n)
        ang = angles.cpu().numpy()
        turned.append((paged.turn_heads(x[:, :H], gq.cpu().numpy(), eps, ang, pos, False), paged.turn_heads(x[:, H:H + Hkv], gk.cpu().numpy(), eps, ang, pos, False), x[:, H + Hkv:]))
    done = [0, 0]
    for part in parts:
        M = sum(part)
        cu, starts = np.concatenate(([0], np.cumsum(part))), list(done)
        rows = torch.cat([qkv[b][done[b]:done[b] + part[b]] for b in range(B)])
        q, k = api.qk_rope_kv4_append(rows[:, :H], rows[:, H:H + Hkv], rows[:, H + Hkv:], pool, table, _ints(cu), _ints(starts), angles, gq, gk, eps,
                                      want_k=True)
        if any(done):                                                      # keys and values of everything so far, out of the cache
            have = [done[b] + part[b] if part[b] else 0 for b in range(B)]
            cu_k = np.concatenate(([0], np.cumsum(have)))
            kk, vv = api.kv4_paged_gather(pool, table, _ints(cu_k), None, sum(have), Hkv)
            kd = [paged.quantized(turned[b][1][:have[b]]).astype(np.float16) for b in range(B)]
            vd = [paged.quantized(turned[b][2][:have[b]]).astype(np.float16) for b in range(B)]
            assert _same(kk, np.concatenate(kd)) and _same(vv, np.concatenate(vd))
        else:
            cu_k, kk, vv = cu, k, rows[:, H + Hkv:]
        out = api.attention_prefill(q, kk, vv, _ints(cu), _ints(cu_k), window, sinks, workspace=ws)
        assert _same(q, np.concatenate([turned[b][0][done[b]:done[b] + part[b]] for b in range(B)]))
        _check_prefill(out, q, kk, vv, cu, cu_k, window, sinks)
        done = [d + p for d, p in zip(done, part)]
        assert out.shape[0] == M
    cu = list(range(B + 1))
    for _ in range(steps):
        rows = torch.stack([qkv[b][done[b]] for b in range(B)])
        q, _ = api.qk_rope_kv4_append(rows[:, :H], rows[:, H:H + Hkv], rows[:, H + Hkv:], pool, table, _ints(cu), _ints(done), angles, gq, gk, eps)
        done = [d + 1 for d in done]
        out = api.kv4_paged_attention_decode(q, pool, table, _ints(done), Hkv, window, sinks, workspace=ws)
        kh = np.concatenate([paged.quantized(turned[b][1][:done[b]]) for b in range(B)])
        vh = np.concatenate([paged.quantized(turned[b][2][:done[b]]) for b in range(B)])
        _check_decode(out, q, kh, vh, np.concatenate(([0], np.cumsum(done))), done, window, sinks)


def test_pages_and_contiguous_cache_agree():
    """The same tokens in both caches: the same codes, and attention within the rounding of its weights."""
    B, H, Hkv, S = 3, 8, 2, 130
    k, v = wl.make_kv(B, Hkv, S, D, 41, DEV)
    q = wl.make_queries(B, H, D, 41, DEV)
    rows = lambda x: x.transpose(1, 2).contiguous()                        # noqa: E731
    cache = api.kv4_new_cache(B, Hkv, S, DEV)
    api.kv4_append(cache, rows(k), rows(v), _ints([0] * B), S)
    table, pages = _tables([S] * B, 3, 43)
    pool = api.kv4_new_pool(pages, Hkv, DEV)
    api.kv4_paged_append(pool, rows(k).view(B * S, Hkv, D), rows(v).view(B * S, Hkv, D), table, _ints([0, S, 2 * S, 3 * S]))
    a = api.kv4_unpack(cache, B, Hkv, S)
    b = _codes(pool, table, pages, Hkv, B, 3)
    for x, y in zip(a, b):
        assert np.array_equal(x.cpu().numpy().view(np.uint8), np.ascontiguousarray(y[:, :, :S]).view(np.uint8))
    lens = _ints([S, 64, 1])
    one, two = api.kv4_attention_decode(q, cache, lens, Hkv, S), api.kv4_paged_attention_decode(q, pool, table, lens, Hkv)
    assert torch.allclose(one.float(), two.float(), rtol=2e-3, atol=2e-3)


def test_another_stream_and_refusals_of_the_binding():
    H, Hkv, T = 4, 2, 70
    q, k, v, cu, _ = _prompts([T], [0], H, Hkv, 111)
    pool, table = api.kv4_new_pool(2, Hkv, DEV), _ints([[1, 0]])
    want = api.attention_prefill(q, k, v, _ints(cu), _ints(cu))
    c = _ints(cu)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = api.attention_prefill(q, k, v, c, c)
        api.kv4_paged_append(pool, k, v, table, c)
        gk, _ = api.kv4_paged_gather(pool, table, c, None, T, Hkv)
    side.synchronize()
    assert _same(got, want) and _same(gk, paged.quantized(k.cpu().numpy()).astype(np.float16))
    for bad in (dict(q=q.float()), dict(q=q.cpu()), dict(k=k[:, :, ::2]), dict(k=k[:-1]), dict(cu_k=c[:1]), dict(cu_q=c.long()), dict(out=q[:, :2]),
                dict(q=q.transpose(0, 1)), dict(workspace=torch.zeros(8)), dict(q=None), dict(window="x")):
        with pytest.raises((TypeError, ValueError, api.QoqError)):
            api.attention_prefill(**{**dict(q=q, k=k, v=v, cu_q=c, cu_k=c), **bad})
    for bad in (dict(pool=pool.float()), dict(block_table=table[0]), dict(block_table=table.repeat(2, 1)), dict(angles=torch.zeros(4, 120, device=DEV)),
                dict(q_gamma=torch.zeros(64, dtype=torch.float16, device=DEV)), dict(starts=_ints([0, 0])), dict(v=v[:, :1]), dict(q_out=q[:3]),
                dict(pool=pool[:8704]), dict(eps=-1.0), dict(q=None, q_out=q)):
        with pytest.raises((TypeError, ValueError, api.QoqError)):
            api.qk_rope_kv4_append(**{**dict(q=q, k=k, v=v, pool=pool, block_table=table, cu=c, starts=None, angles=None), **bad})
    lens = _ints([T])
    for bad in (dict(q=q), dict(seq_lens=_ints([1, 2])), dict(Hkv=3), dict(Hkv=0), dict(window=-1), dict(block_table=table.long()), dict(out=q[:2])):
        with pytest.raises((TypeError, ValueError, api.QoqError)):
            api.kv4_paged_attention_decode(**{**dict(q=q[:1], pool=pool, block_table=table, seq_lens=lens, Hkv=Hkv), **bad})
    for bad in (dict(rows=-1), dict(Hkv=0), dict(k_out=k[:5]), dict(cu=c.long()), dict(starts=_ints([0, 0]))):
        with pytest.raises((TypeError, ValueError, api.QoqError)):
            api.kv4_paged_gather(**{**dict(pool=pool, block_table=table, cu=c, starts=None, rows=T, Hkv=Hkv), **bad})


# ------------------------------------------------------------------------------------------------------------------
# Graphs, streams, far offsets
# ------------------------------------------------------------------------------------------------------------------
def test_a_graph_of_a_prompt_and_a_token():
    """Append, gather, a long prompt's and a few rows' attention and a decode step in one graph with one workspace, replayed with
    other inputs in the same tensors and eager calls in the same workspace between; every replay against the eager calls."""
    H, Hkv, window, sinks = 8, 2, 0, 0
    held, new, width = 4100, 512, 73
    total = held + new
    pool, table, pages, cu, _, _ = _filled([total], Hkv, width, 301)
    angles = api.rope_angles(width * PAGE, device=DEV)
    cu_new, cu_few, cu_all, starts, lens = _ints([0, new]), _ints([0, 20]), _ints([0, total]), _ints([held]), _ints([total])
    needs = [api.attention_prefill_workspace_bytes(m, total, 1, H, Hkv) for m in (new, 20)] + [api.kv4_paged_attention_workspace_bytes(1, H, Hkv, width)]
    assert min(needs) > api.GEMM_COUNTER_BYTES                             # all three share keys between workgroups
    ws = api.new_workspace(max(needs), DEV)
    x = torch.empty((new, H + 2 * Hkv, D), dtype=torch.float16, device=DEV)
    q, k = torch.empty((new, H, D), dtype=torch.float16, device=DEV), torch.empty((total, Hkv, D), dtype=torch.float16, device=DEV)
    v, outs = torch.empty_like(k), [torch.empty((m, H, D), dtype=torch.float16, device=DEV) for m in (new, 20, 1)]

    def step():
        api.qk_rope_kv4_append(x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:], pool, table, cu_new, starts, angles, q_out=q)
        api.kv4_paged_gather(pool, table, cu_all, None, total, Hkv, k, v)
        api.attention_prefill(q, k, v, cu_new, cu_all, window, sinks, out=outs[0], workspace=ws)
        api.attention_prefill(q[-20:], k, v, cu_few, cu_all, window, sinks, out=outs[1], workspace=ws)
        api.kv4_paged_attention_decode(q[-1:], pool, table, lens, Hkv, window, sinks, out=outs[2], workspace=ws)

    fill = lambda seed: x.copy_(torch.cat((_heads(new, H, seed), _heads(new, Hkv, seed + 1), _heads(new, Hkv, seed + 2, 4)), dim=1))      # noqa: E731
    want = []
    for seed in (310, 320, 330):
        fill(seed)
        step()
        want.append([t.clone() for t in (q, k, v, *outs)])
    _check_prefill(outs[0], q, k, v, [0, new], [0, total], window, sinks, rows=20)
    _check_prefill(outs[1], q[-20:], k, v, [0, 20], [0, total], window, sinks)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for i in (0, 1, 2, 1, 0):
        fill((310, 320, 330)[i])
        for t in (q, k, v, *outs):
            t.fill_(7.0)
        graph.replay()
        for have, exp in zip((q, k, v, *outs), want[i]):
            assert _same(have, exp)
        torch.cuda.synchronize()
        few = api.attention_prefill(q[:3], k, v, _ints([0, 3]), cu_all, window, sinks, workspace=ws)
        _check_prefill(few, q[:3], k, v, [0, 3], [0, total], window, sinks)
    assert not ws[:api.GEMM_COUNTER_BYTES].any()


def test_two_streams_at_once():
    """Calls that overlap in time, each with a workspace of its own, on the same cache."""
    H, Hkv, lens = 8, 2, [3000, 1700]
    width = 48
    pool, table, pages, cu, kh, vh = _filled(lens, Hkv, width, 341)
    k, v = (torch.from_numpy(t.astype(np.float16)).to(DEV) for t in (kh, vh))
    seq, cu_k, cu_q = _ints(lens), _ints(cu), _ints([0, 9, 12])
    q, few = wl.make_queries(2, H, D, 343, DEV), _heads(12, H, 344, 4)
    sizes = [api.kv4_paged_attention_workspace_bytes(2, H, Hkv, width), api.attention_prefill_workspace_bytes(12, sum(lens), 2, H, Hkv)]
    assert min(sizes) > 0
    streams, spaces = [torch.cuda.Stream() for _ in range(2)], [api.new_workspace(max(sizes), DEV) for _ in range(2)]
    want = (api.kv4_paged_attention_decode(q, pool, table, seq, Hkv, workspace=spaces[0]), api.attention_prefill(few, k, v, cu_q, cu_k, workspace=spaces[0]))
    _check_decode(want[0], q, kh, vh, cu, lens, 0, 0)
    _check_prefill(want[1], few, k, v, [0, 9, 12], cu, 0, 0)
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for stream, ws, kept in zip(streams, spaces, got):
            with torch.cuda.stream(stream):
                kept.append((api.kv4_paged_attention_decode(q, pool, table, seq, Hkv, workspace=ws), api.attention_prefill(few, k, v, cu_q, cu_k, workspace=ws)))
    torch.cuda.synchronize()
    for a, b in got[0] + got[1]:
        assert _same(a, want[0]) and _same(b, want[1])


def test_pages_shared_by_sequences():
    """Sequences with a common beginning name the same pages; a sequence may name a page more than once."""
    H, Hkv, width = 8, 2, 6
    pool, table, pages, cu, kh, vh = _filled([256, 100], Hkv, width, 351)
    t = table.clone()
    t[1, 2:4] = table[1, :2]                                               # 128 tokens of the first, then the second's 100
    t[1, :2] = table[0, :2]
    t[0, 4] = t[0, 1]                                                      # and the first goes on with its own second page
    lens = [320, 228]
    q = wl.make_queries(2, H, D, 353, DEV)
    pick = np.concatenate((np.arange(256), np.arange(64, 128), np.arange(128), 256 + np.arange(100)))
    out = api.kv4_paged_attention_decode(q, pool, t, _ints(lens), Hkv)
    _check_decode(out, q, kh[pick], vh[pick], [0, 320, 548], lens, 0, 0)
    gk, gv = api.kv4_paged_gather(pool, t, _ints([0, 320, 548]), None, 548, Hkv)
    assert _same(gk, kh[pick].astype(np.float16)) and _same(gv, vh[pick].astype(np.float16))


def test_pages_past_four_gigabytes():
    """The last pages of a pool of more than 2^32 bytes hold, return and serve what the first ones of a small pool do."""
    H, Hkv, lens = 8, 8, [200, 65]
    small, table, pages, cu, kh, vh = _filled(lens, Hkv, 4, 361)
    many = (1 << 32) // (Hkv * 8704) + 100
    far = torch.where(table >= 0, many - 1 - table, table)
    pool = torch.empty(many * Hkv * 8704, dtype=torch.uint8, device=DEV)
    M = sum(lens)
    q, k, v = _heads(M, H, 363, 4), _heads(M, Hkv, 364), _heads(M, Hkv, 365, 4)
    angles = api.rope_angles(256, device=DEV)
    got, one = [], wl.make_queries(2, H, D, 366, DEV)
    for p, t in ((small, table), (pool, far)):
        turned, _ = api.qk_rope_kv4_append(q, k, v, p, t, _ints(cu), None, angles)
        got.append((turned, *api.kv4_paged_gather(p, t, _ints(cu), None, M, Hkv), api.kv4_paged_attention_decode(one, p, t, _ints(lens), Hkv)))
    for a, b in zip(*got):
        assert _same(a, b)


def test_rows_past_four_gigabytes():
    """The last rows of tensors of more than 2^32 bytes, and rows that lie the largest stride apart."""
    H, Hkv, n = 8, 2, 600
    q, k, v, _, _ = _prompts([n], [0], H, Hkv, 371)
    want = api.attention_prefill(q, k, v, _ints([0, n]), _ints([0, n]))
    M = (1 << 32) // (H * D * 2) + 1000
    big_q, out = torch.empty((M, H, D), dtype=torch.float16, device=DEV), torch.empty((M, H, D), dtype=torch.float16, device=DEV)
    big_q[-n:] = q
    out[0], out[-n - 1] = 3.0, 4.0
    api.attention_prefill(big_q, k, v, _ints([M - n, M]), _ints([0, n]), out=out)
    # (a grid for so many rows takes 128 of them to a workgroup: other tiles, the same bound)
    _check_prefill(out[-n:], q, k, v, [0, n], [0, n], 0, 0, rows=40)
    assert bool((out[0] == 3).all()) and bool((out[-n - 1] == 4).all())
    angles = api.rope_angles(n, device=DEV)
    pool, table = api.kv4_new_pool(10, Hkv, DEV), _ints([[2, 0, 1, 9, 8, 7, 4, 3, 6, 5]])
    turned, _ = api.qk_rope_kv4_append(q, k, v, pool, table, _ints([0, n]), None, angles)
    kv = torch.zeros((M, 2 * Hkv, D), dtype=torch.float16, device=DEV)
    kv[-n:, :Hkv], kv[-n:, Hkv:] = k, v
    other = torch.zeros_like(pool)
    api.qk_rope_kv4_append(big_q, kv[:, :Hkv], kv[:, Hkv:], other, table, _ints([M - n, M]), None, angles, q_out=big_q)
    assert _same(big_q[-n:], turned)
    gk, gv = (t.view(-1)[:M * Hkv * D].view(M, Hkv, D) for t in (out, kv))
    api.kv4_paged_gather(other, table, _ints([M - n, M]), None, M, Hkv, gk, gv)
    ek, ev = api.kv4_paged_gather(pool, table, _ints([0, n]), None, n, Hkv)
    assert _same(gk[-n:], ek) and _same(gv[-n:], ev)
    del big_q, out, kv, gk, gv
    wide = torch.empty((n, 1 << 22), dtype=torch.float16, device=DEV)
    qs, ks, vs = wide[:, :H * D].view(n, H, D), wide[:, H * D:(H + Hkv) * D].view(n, Hkv, D), wide[:, -Hkv * D:].view(n, Hkv, D)
    qs.copy_(q), ks.copy_(k), vs.copy_(v)
    assert _same(api.attention_prefill(qs, ks, vs, _ints([0, n]), _ints([0, n])), want)
    many = _heads(n, 64, 373, 4)                                           # 128 rows to a workgroup
    assert _same(api.attention_prefill(many, ks, vs, _ints([0, n]), _ints([0, n])), api.attention_prefill(many, k, v, _ints([0, n]), _ints([0, n])))
    pool.zero_()
    assert _same(api.qk_rope_kv4_append(qs, ks, vs, pool, table, _ints([0, n]), None, angles)[0], turned)
    assert _same(api.kv4_paged_gather(pool, table, _ints([0, n]), None, n, Hkv)[0], ek)


def test_longest_sequence():
    """2^24 tokens, the most a table of 262144 pages holds, all in one page named again and again: each of its 64 tokens has the same
    weight as alone.  Each of 256 waves adds up 2^16 of them: 2^16 roundings of 2^-24 at most for the products, 2^13 for the weights, of
    which a lane has 4 of a chunk's 32, all relative to the sums of magnitudes."""
    H, Hkv, width = 4, 1, 1 << 18
    pool, table, pages, cu, kh, vh = _filled([64], Hkv, 1, 381)
    long = table[:, :1].repeat(1, width).contiguous()
    q = wl.make_queries(1, H, D, 383, DEV)
    ref, spread = paged.attention(q.cpu().numpy().astype(np.float64), kh, vh, [63])
    tol, _ = _bound(q.cpu().numpy().astype(np.float64), kh, ref, spread, 64)
    tol = tol + (2.0 ** 16 + 2.0 ** 13) * 2.0 ** -24 * spread + 64 * 15 * 2.0 ** -25 + 2.0 ** -25
    ws = api.new_workspace(api.kv4_paged_attention_workspace_bytes(1, H, Hkv, width), DEV)
    for length in (1 << 24, (1 << 31) - 1):                                # (more than the table holds: as many as it does)
        out = api.kv4_paged_attention_decode(q, pool, long, _ints([length]), Hkv, workspace=ws)
        assert (np.abs(out.cpu().numpy().astype(np.float64) - ref) <= tol).all()
    # through a window, behind the first tokens: the page's last 40 and first 5 tokens
    out = api.kv4_paged_attention_decode(q, pool, long, _ints([1 << 24]), Hkv, window=40, sinks=5, workspace=ws)
    see = np.array([t >= 24 or t < 5 for t in range(64)])
    ref, spread = paged.attention(q.cpu().numpy().astype(np.float64), kh, vh, [63], held=see)
    tol, _ = _bound(q.cpu().numpy().astype(np.float64), kh, ref, spread, 64)
    assert (np.abs(out.cpu().numpy().astype(np.float64) - ref) <= tol + 64 * 15 * 2.0 ** -25 + 2.0 ** -25).all()
    # the last token appended by its position
    k, v = _heads(1, Hkv, 385), _heads(1, Hkv, 386, 4)
    api.kv4_paged_append(pool, k, v, long, _ints([0, 1]), _ints([(1 << 24) - 1]))
    gk, gv = api.kv4_paged_gather(pool, long, _ints([0, 2]), _ints([(1 << 24) - 1]), 2, Hkv)
    assert _same(gk[:1], paged.quantized(k.cpu().numpy()).astype(np.float16)) and not gk[1].any() and not gv[1].any()


def test_prompt_attention_behind_millions_of_tokens():
    """Keys of more than 2^32 bytes: three queries behind 2^24 - 5 tokens, whose keys are zero but for some at both ends and at
    2^32 bytes; zero keys have one weight and zero values, so that the result has a plain form."""
    n = (1 << 24) - 2
    k, v = torch.zeros((n, 1, D), dtype=torch.float16, device=DEV), torch.zeros((n, 1, D), dtype=torch.float16, device=DEV)
    at = np.concatenate((np.arange(5), (1 << 24) // 2 + np.arange(-4, 5), (1 << 24) - 300 + np.arange(6), np.arange(n - 6, n)))
    some_k, some_v = _heads(len(at), 1, 391), _heads(len(at), 1, 392, 4)
    q = (_heads(3, 2, 393, 4) * 4).contiguous()
    k[torch.from_numpy(at).to(DEV)], v[torch.from_numpy(at).to(DEV)] = some_k, some_v
    kd, vd, qd = (t.cpu().numpy().astype(np.float64) for t in (some_k, some_v, q))
    ws = api.new_workspace(api.attention_prefill_workspace_bytes(3, n, 1, 2, 1), DEV)
    for space in (ws, None):
        got = api.attention_prefill(q, k, v, _ints([0, 3]), _ints([0, n]), workspace=space).cpu().numpy().astype(np.float64)
        for i in range(3):
            see = at <= n - 3 + i
            for h in range(2):
                s = kd[see, 0] @ qd[i, h] / np.sqrt(D)
                top = max(s.max(), 0.0)
                p = np.exp(s - top)
                total = p.sum() + (n - 2 + i - see.sum()) * np.exp(-top)
                ref, spread = p @ vd[see, 0] / total, p @ np.abs(vd[see, 0]) / total
                e = 130 * 2.0 ** -24 * float((np.abs(kd[:, 0]) @ np.abs(qd[i, h])).max()) / np.sqrt(D)
                # the zero keys' weights are one number, whose rounding does not average out: 2^-11 of it, or below FP16's normal numbers
                # 2^-25 of the largest weight; and without a workspace a lane adds up its share of 2^17 tiles in four sums, two
                # additions each: 2^18 half steps of 2^-24
                loss = n * 2.0 ** -25 / total + 2.0 ** 18 * 2.0 ** -24
                tol = 2 * 2.0 ** -11 * np.abs(ref) + (2.0 ** -11 + 2 * e + 2.0 ** -20 + loss) * spread + len(at) * 2.0 ** -25 * np.abs(vd).max()
                assert (np.abs(got[i, h] - ref) <= tol).all(), (i, h)


@pytest.mark.parametrize("B", [4096, 4097, 4160, 4161, 262208, 262209, 266304, 266305])
def test_every_sequence_of_a_large_batch_is_found(B):
    """One token per sequence, and so many sequences that 64 lanes look for one in two or three rounds, on both sides of where the last
    round's candidates fill a wave: every sequence's codes, cached numbers and attention (one key, weight 1: its value's bits)."""
    pages, width = -(-B // PAGE), 1
    table = (torch.arange(B, dtype=torch.int32, device=DEV) // PAGE)[:, None].contiguous()      # 64 sequences to a page, each at its own place
    starts = torch.arange(B, dtype=torch.int32, device=DEV) % PAGE
    cu = torch.arange(B + 1, dtype=torch.int32, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(B)
    q, k, v = (torch.randn((B, 1, D), generator=g, device=DEV, dtype=torch.float16) for _ in range(3))
    pool = api.kv4_new_pool(pages, 1, DEV)
    qo, ko = torch.full_like(q, 9.0), torch.full_like(k, 9.0)
    angles = torch.cat((torch.ones(PAGE, 64), torch.zeros(PAGE, 64)), dim=1).to(DEV)             # no turn
    api.qk_rope_kv4_append(q, k, v, pool, table, cu, starts, angles, q_out=qo, k_out=ko)
    assert torch.equal(qo, q) and torch.equal(ko, k)
    # the same tokens as one sequence's prompt: the pages of the pool in their order
    alone = api.kv4_new_pool(pages, 1, DEV)
    order = torch.arange(pages, dtype=torch.int32, device=DEV)[None]
    api.kv4_paged_append(alone, k, v, order, _ints([0, B]))
    assert torch.equal(pool, alone)
    gk, gv = torch.full_like(k, 9.0), torch.full_like(v, 9.0)
    api.kv4_paged_gather(pool, table, cu, starts, B, 1, gk, gv)
    ek, ev = api.kv4_paged_gather(alone, order, _ints([0, B]), None, B, 1)
    assert torch.equal(gk, ek) and torch.equal(gv, ev)
    out = torch.full_like(q, 9.0)
    api.attention_prefill(q, k, v, cu, cu, out=out)
    assert torch.equal(out, v)


@pytest.mark.parametrize("B", [4097, 4160])
def test_prefill_of_thousands_of_ragged_sequences(B):
    """Lengths from none to six, some behind cached tokens, and outputs that no sequence owns left as they were."""
    new, held = [(5 * b) % 7 for b in range(B)], [(11 * b) % 9 for b in range(B)]
    q, k, v, cu_q, cu_k = _prompts(new, held, 4, 2, 117, behind=3)
    out = torch.full_like(q, 9.0)
    api.attention_prefill(q, k, v, _ints(cu_q), _ints(cu_k), window=5, sinks=1, out=out)
    assert bool((out[-3:] == 9).all())
    _check_prefill(out, q, k, v, cu_q, cu_k, 5, 1)


def _chosen(lens, k, v, width, seed):
    """A pool with these keys and values: [tokens, Hkv, 128] FP16 of the sequences one after the other."""
    table, pages = _tables(lens, width, seed)
    cu = np.concatenate(([0], np.cumsum(lens)))
    pool = torch.full((pages * k.shape[1] * 8704,), 0xFF, dtype=torch.uint8, device=DEV)
    api.kv4_paged_append(pool, k, v, table, _ints(cu))
    return pool, table, cu, paged.quantized(k.cpu().numpy()), paged.quantized(v.cpu().numpy())


@pytest.mark.parametrize("H,Hkv", [(2, 2), (8, 1), (16, 1)])
@pytest.mark.parametrize("ahead", [2.8, 8.3, 10.4, 17.0])
@pytest.mark.parametrize("size,first", [(0.1, 1.0), (2.0 ** -10, 1.0), (2.0 ** -13, 1.0), (2.0 ** -16, 1.0), (1.0, 2.0 ** -9), (2.0 ** -8, 2.0 ** 9), (1.5e4, 1.0)])
def test_decode_of_light_tokens(H, Hkv, ahead, size, first):
    """A first token whose score is `ahead` above those of a long flat tail (natural logarithm), values of `size`, the first token's
    `first` times that: the light tokens' weights times the scale of their values, however small, keep their share.
    A product of weight and scale is rounded to FP16 as a multiple of a power of two: half a step is 2^-11 of it or, below FP16's normal numbers,
    2^-25 of that power, which lies 2^14 below the largest weight times the largest scale, or lower (scales below 2^-15 count as
    that).  So n tokens of codes up to 15 lose 15 n 2^-39 max(scale, 2^-15) at most, against weights whose sum is at least the largest of them."""
    L, width, lens = 3000, 48, [3000, 700, 65]
    n = sum(lens)
    g = torch.Generator().manual_seed(int(ahead * 10) + H)
    base = torch.randn(1, Hkv, D, generator=g)
    q = (base.repeat_interleave(H // Hkv, 1) * (1 + 0.05 * torch.randn(len(lens), H, 1, generator=g))).half()
    k = 0.02 * torch.randn(n, Hkv, D, generator=g)
    v = (size * torch.randn(n, Hkv, D, generator=g)).clamp(-6e4, 6e4)       # (FP16 numbers)
    cu = np.concatenate(([0], np.cumsum(lens)))
    for at in cu[:-1]:
        k[at] = base[0] * (ahead * np.sqrt(D) / (base[0] ** 2).sum(-1, keepdim=True))
        v[at] = v[at] * first
    pool, table, cu, kh, vh = _chosen(lens, k.half().to(DEV), v.half().to(DEV), width, 51)
    scale = float(kv4.kv4_quantize(v.half().numpy())[1].astype(np.float64).max())
    ws = api.new_workspace(api.kv4_paged_attention_workspace_bytes(3, H, Hkv, width), DEV)
    for window, sinks, room in ((0, 0, ws), (0, 0, None), (600, 4, None)):
        got = api.kv4_paged_attention_decode(q.to(DEV), pool, table, _ints(lens), Hkv, window, sinks, workspace=room).cpu().numpy().astype(np.float64)
        for b, n_b in enumerate(lens):
            kb, vb, qb = kh[cu[b]:cu[b] + n_b], vh[cu[b]:cu[b] + n_b], q[b:b + 1].numpy().astype(np.float64)
            ref, spread = paged.attention(qb, kb, vb, [n_b - 1], window, sinks)
            tol, _ = _bound(qb, kb, ref, spread, n_b)
            tol = tol[0] + 15 * n_b * 2.0 ** -39 * max(scale, 2.0 ** -15) + 2.0 ** -25
            assert (np.abs(got[b] - ref[0]) <= tol).all(), (b, window, float((np.abs(got[b] - ref[0]) / tol).max()))


def test_decode_of_values_of_every_size():
    """Values whose sizes change from token to token over all of FP16, up to its largest numbers: nothing overflows on the way."""
    H, Hkv, lens, width = 8, 1, [2000, 33], 32
    g = torch.Generator().manual_seed(77)
    n = sum(lens)
    q, k = torch.randn(2, H, D, generator=g).half(), torch.randn(n, Hkv, D, generator=g).half()
    v = (torch.randn(n, Hkv, D, generator=g).clamp(-1.9, 1.9) * torch.exp2(torch.randint(-20, 16, (n, Hkv, 1), generator=g).float())).half()
    pool, table, cu, kh, vh = _chosen(lens, k.to(DEV), v.to(DEV), width, 53)
    assert bool(torch.isfinite(v).all()) and float(v.abs().max()) > 6e4
    scale = float(kv4.kv4_quantize(v.numpy())[1].astype(np.float64).max())
    ws = api.new_workspace(api.kv4_paged_attention_workspace_bytes(2, H, Hkv, width), DEV)
    for room in (ws, None):
        got = api.kv4_paged_attention_decode(q.to(DEV), pool, table, _ints(lens), Hkv, workspace=room).cpu().numpy().astype(np.float64)
        for b, n_b in enumerate(lens):
            kb, vb, qb = kh[cu[b]:cu[b] + n_b], vh[cu[b]:cu[b] + n_b], q[b:b + 1].numpy().astype(np.float64)
            ref, spread = paged.attention(qb, kb, vb, [n_b - 1])
            tol, _ = _bound(qb, kb, ref, spread, n_b)
            assert (np.abs(got[b] - ref[0]) <= tol[0] + 15 * n_b * 2.0 ** -39 * scale + 2.0 ** -25).all(), b


@pytest.mark.parametrize("H,Hkv,new,held", [(2, 1, 5, 6000), (4, 1, 700, 5300), (2, 2, 40, 0)])
@pytest.mark.parametrize("ahead", [9.0, 12.5, 17.0])
def test_prefill_of_light_tokens(H, Hkv, new, held, ahead):
    """A first token whose score is `ahead` above those of all others (natural logarithm), which are alike, and whose values are zero: the others' weights
    keep their share.  A weight is off by 2^-11 of itself or, below FP16's normal numbers, by 2^-25 where the largest of the row is at least
    2^7: n 2^-32 max|v|."""
    T = new + held
    g = torch.Generator().manual_seed(int(10 * ahead))
    base = torch.randn(1, Hkv, D, generator=g)
    q = (base.repeat_interleave(H // Hkv, 1) * (1 + 0.02 * torch.randn(new, H, 1, generator=g))).half().to(DEV)
    k, v = torch.zeros(T, Hkv, D, dtype=torch.float16, device=DEV), torch.randn(T, Hkv, D, generator=g).abs().half().to(DEV)
    k[0] = (base[0] * (ahead * np.sqrt(D) / (base[0] ** 2).sum(-1, keepdim=True))).half().to(DEV)
    v[0] = 0
    cu_q, cu_k = [0, new], [0, T]
    ws = api.new_workspace(api.attention_prefill_workspace_bytes(new, T, 1, H, Hkv), DEV)
    pick = np.unique(np.concatenate((np.arange(min(new, 5)), np.linspace(0, new - 1, 20).astype(int))))
    qd, kd, vd = (t.cpu().numpy().astype(np.float64) for t in (q, k, v))
    ref, spread = paged.attention(qd[pick], kd, vd, held + pick)
    tol, _ = _bound(qd[pick], kd, ref, spread, T)
    tol = tol + T * 2.0 ** -32 * vd.max() + 2.0 ** -25
    for room in (ws, None):
        got = api.attention_prefill(q, k, v, _ints(cu_q), _ints(cu_k), workspace=room).cpu().numpy().astype(np.float64)[pick]
        assert (np.abs(got - ref) <= tol).all(), float((np.abs(got - ref) / tol).max())


def test_prefill_of_a_million_light_tokens():
    """Tokens whose weights are below FP16's normal numbers and make up a fifth of the sum: what the products take and what the weights' sum
    takes are the same numbers.  The tokens are alike, so their roundings do not average out: 2^-25 of at least 2^7 each, and a lane
    adds up its 2^13 tiles with the workspace, 2^15 without, in four sums of two additions a tile."""
    n, ahead = 1 << 20, 15.3
    g = torch.Generator().manual_seed(5)
    q = torch.randn(1, 1, D, generator=g).half().to(DEV)
    k, v = torch.zeros(n, 1, D, dtype=torch.float16, device=DEV), torch.full((n, 1, D), 0.5, dtype=torch.float16, device=DEV)
    k[0], v[0] = q[0] * (ahead * np.sqrt(D) / float((q.float() ** 2).sum())), 0
    score = float((q.double() * k[0].double()).sum()) / np.sqrt(D)
    tail = (n - 1) * np.exp(-score)
    ref = 0.5 * tail / (1 + tail)
    assert 0.1 < tail < 0.4
    ws = api.new_workspace(api.attention_prefill_workspace_bytes(1, n, 1, 1, 1), DEV)
    e = 130 * 2.0 ** -24 * float((q.double().abs() * k[0].double().abs()).sum()) / np.sqrt(D)
    for room, tiles in ((ws, 1 << 13), (None, 1 << 15)):
        got = api.attention_prefill(q, k, v, _ints([0, 1]), _ints([0, n]), workspace=room).double().cpu().numpy()
        tol = 2.0 ** -11 * ref + (2 * 2.0 ** -11 + 2 * e + 2.0 ** -20 + 2 * tiles * 2.0 ** -24) * ref + n * 2.0 ** -32 * 0.5
        assert (np.abs(got - ref) <= tol).all(), (float(np.abs(got - ref).max()), tol)


@pytest.mark.parametrize("new,held", [(40, 0), (5, 4000), (700, 4100)])
def test_prefill_of_queries_whose_scores_are_all_minus_infinity(new, held):
    """Keys with an infinity that a query turns into a score of minus infinity have no weight; where it sees nothing else, the softmax is
    0 / 0 and its row NaN, and not that of a query that sees nothing."""
    H, Hkv, T = 2, 1, new + held
    q, k, v, _, _ = _prompts([new], [held], H, Hkv, 121)
    q[:, :, 3] = torch.where(torch.arange(new, device=DEV)[:, None] % 2 == 0, -1.0, 1.0)
    some = 7                                                               # queries up to this one see nothing but such keys
    k[:held + some + 1, 0, 3] = float("inf")
    ws = api.new_workspace(api.attention_prefill_workspace_bytes(new, T, 1, H, Hkv), DEV)
    for window, sinks in ((0, 0), (5, 2)):
        for room in (ws, None):
            got = api.attention_prefill(q, k, v, _ints([0, new]), _ints([0, T]), window=window, sinks=sinks, workspace=room).cpu().numpy()
            # (even rows: minus infinity; odd ones: infinity, NaN as soon as one is seen)
            assert np.isnan(got[:min(some + 1, new)]).all(), (window, room is None)
    qs, ks = q.clone(), k.clone()
    qs[:, :, 3], cu_q, cu_k = -1.0, [0, 3, new], [0, 0, T]                 # and three queries of a sequence without tokens
    out = api.attention_prefill(qs, ks, v, _ints(cu_q), _ints(cu_k))
    assert not out[:3].any() and bool(torch.isnan(out[3:3 + max(some + 1 - 3, 0)]).all())


@pytest.mark.parametrize("near", [False, True])
def test_infinities_outside_the_turned_part_stay_where_they_are(near):
    """A norm divides a head with an infinity by infinity: NaN there and, among the elements that are not turned, zeros beside it."""
    M, H, rot = 5, 2, 32
    q, kv = _heads(M, H, 25), torch.zeros(M, 1, D, dtype=torch.float16, device=DEV)
    q[1, 0, 70], q[2, 1, 101], q[3, 0, 5], q[3, 1, 32] = float("inf"), -float("inf"), float("inf"), float("inf")
    gamma, angles = 1 + 0.1 * _heads(1, 1, 26)[0, 0], api.rope_angles(M, rot, device=DEV)
    pool, table = api.kv4_new_pool(1, 1, DEV), _ints([[0]])
    for g in (gamma, None):
        out, _ = api.qk_rope_kv4_append(q, kv, kv, pool, table, _ints([0, M]), None, angles, q_gamma=g, interleaved=near)
        with np.errstate(invalid="ignore"):
            want = paged.turn_heads(q.cpu().numpy(), None if g is None else g.cpu().numpy(), 1e-6, angles.cpu().numpy(), np.arange(M), near)
        assert np.array_equal(out.cpu().numpy(), want, equal_nan=True)


@pytest.mark.parametrize("empty", [62, 63, 64, 65, 300])
def test_long_runs_of_empty_sequences(empty):
    """More sequences without rows between two neighbouring rows than a wave has lanes; in front of the first row and behind the last."""
    new = [0] * empty + [1] + [0] * empty + [1, 1] + [0] * (2 * empty) + [2, 0, 1] + [0] * empty + [9] + [0] * empty
    B, M = len(new), sum(new)
    starts, held = [(17 * b) % 50 for b in range(B)], [(5 * b) % 3 for b in range(B)]
    cu = np.concatenate(([0], np.cumsum(new)))
    table, pages = _tables([64] * B, 1, 9)
    q, k, v = _heads(M, 4, 131), _heads(M, 2, 132), _heads(M, 2, 133, 4)
    angles = api.rope_angles(64, device=DEV)
    pool = api.kv4_new_pool(pages, 2, DEV)
    qo, ko = api.qk_rope_kv4_append(q, k, v, pool, table, _ints(cu), _ints(starts), angles, want_k=True)
    seq, pos = paged.rows_of(cu, starts, M)
    want_k = paged.turn_heads(k.cpu().numpy(), None, 0, angles.cpu().numpy(), pos, False)
    assert _same(qo, paged.turn_heads(q.cpu().numpy(), None, 0, angles.cpu().numpy(), pos, False)) and _same(ko, want_k)
    gk, gv = api.kv4_paged_gather(pool, table, _ints(cu), _ints(starts), M, 2)
    assert _same(gk, paged.quantized(want_k).astype(np.float16)) and _same(gv, paged.quantized(v.cpu().numpy()).astype(np.float16))
    q, k, v, cu_q, cu_k = _prompts(new, held, 4, 2, 135)
    _check_prefill(api.attention_prefill(q, k, v, _ints(cu_q), _ints(cu_k)), q, k, v, cu_q, cu_k, 0, 0)


@pytest.mark.parametrize("H,Hkv", [(2, 2), (8, 1), (16, 1)])
@pytest.mark.parametrize("size", [300.0, 1000.0, 2000.0, 2400.0, 3300.0, 4100.0, 9000.0, 30000.0])
def test_decode_of_the_largest_scores(H, Hkv, size):
    """Scores up to 10^10, far past where FP32 holds their units: one token ahead of all others is alone in the result, and tokens of
    one score share it evenly.  (Equal scores are the same sums and so the same numbers; a product and the result are rounded.)"""
    lens, width = [40, 333, 1500, 64], 24
    g = torch.Generator().manual_seed(int(size) + H)
    n, sign = sum(lens), torch.where(torch.rand(Hkv, D, generator=g) < 0.5, -1.0, 1.0)
    q = (size * sign).repeat_interleave(H // Hkv, 0)[None].repeat(4, 1, 1)
    k = (-size * sign)[None].repeat(n, 1, 1)
    v = torch.randn(n, Hkv, D, generator=g) * torch.exp2(3 * torch.rand(n, Hkv, 1, generator=g))
    cu = np.concatenate(([0], np.cumsum(lens)))
    ahead = [39, 7, 1000, None]                                            # in each sequence; in the last one all are alike
    for b, t in enumerate(ahead):
        if t is not None:
            k[cu[b] + t] *= -1
    pool, table, cu, _, vh = _chosen(lens, k.half().to(DEV), v.half().to(DEV), width, 57)
    ws = api.new_workspace(api.kv4_paged_attention_workspace_bytes(4, H, Hkv, width), DEV)
    for room in (ws, None):
        got = api.kv4_paged_attention_decode(q.half().to(DEV), pool, table, _ints(lens), Hkv, workspace=room).cpu().numpy().astype(np.float64)
        for b, t in enumerate(ahead):
            vb = np.repeat(vh[cu[b]:cu[b + 1]], H // Hkv, axis=1)
            ref, spread = (vb[t], np.abs(vb[t])) if t is not None else (vb.mean(axis=0), np.abs(vb).mean(axis=0))
            assert (np.abs(got[b] - ref) <= 2.0 ** -11 * np.abs(ref) + (2.0 ** -11 + 2.0 ** -20) * spread + 2.0 ** -25).all(), b


@pytest.mark.parametrize("H,Hkv,T", [(2, 1, 100), (8, 2, 900), (4, 4, 1300)])
@pytest.mark.parametrize("size", [300.0, 1000.0, 2000.0, 2400.0, 3300.0, 4100.0, 9000.0, 30000.0])
def test_prefill_of_the_largest_scores(H, Hkv, T, size):
    """The same of prompts: queries in front of a token that is ahead see tokens of one score, those behind it that token alone."""
    g = torch.Generator().manual_seed(int(size) + T)
    sign = torch.where(torch.rand(Hkv, D, generator=g) < 0.5, -1.0, 1.0)
    q = (size * sign).repeat_interleave(H // Hkv, 0)[None].repeat(T, 1, 1).half().to(DEV)
    k, at = (-size * sign)[None].repeat(T, 1, 1), T // 2 + 3
    k[at] *= -1
    v = (torch.randn(T, Hkv, D, generator=g) * torch.exp2(3 * torch.rand(T, Hkv, 1, generator=g))).half().to(DEV)
    vd = v.cpu().numpy().astype(np.float64)
    steps = np.arange(1, T + 1)[:, None, None]
    ref, spread = np.cumsum(vd, axis=0) / steps, np.cumsum(np.abs(vd), axis=0) / steps
    ref[at:], spread[at:] = vd[at], np.abs(vd[at])
    ref, spread = np.repeat(ref, H // Hkv, axis=1), np.repeat(spread, H // Hkv, axis=1)
    ws = api.new_workspace(api.attention_prefill_workspace_bytes(T, T, 1, H, Hkv), DEV)
    for room in (ws, None):
        got = api.attention_prefill(q, k.half().to(DEV), v, _ints([0, T]), _ints([0, T]), workspace=room).cpu().numpy().astype(np.float64)
        assert (np.abs(got - ref) <= 2.0 ** -11 * np.abs(ref) + (2.0 ** -11 + 2.0 ** -20) * spread + 2.0 ** -25).all()

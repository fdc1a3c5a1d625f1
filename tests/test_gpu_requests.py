"""Shared-prefix decode attention, adapters of many requests and log probabilities on the GPU against the float64 oracle.

Attention is bounded term by term as in tests/test_gpu_paged.py, with FP32 sums of any order over the tokens:
    |got - ref| <= 2^-11 |ref|                                     the result's rounding to FP16
                 + (2^-11 + 2 e + 2^-20 + (L + 160) 2^-24) sum_t p_t |v_t|   weight times scale rounded, scores, exp2, FP32 sums over tokens and parts
                 + 15 L 2^-25 + 2^-25                              the lightest tokens; FP16's smallest step
Adapters: FP32 sums of K and of 2 r products in any order, the middle product as pairs (oracle.requests.lora), and the result's rounding.
Log probabilities: each e^(x - r) is off by 2^-23 (the instruction) and its argument's rounding, ln 2 times 2^-24 of at most 1.45 |x - max| + 8, which
  weighted by p gives  dT = 2^-23 + 2^-24 (1.1 E|x - max| + 6) + chain 2^-24  with a chain of additions of at most V / 64 + 100; logprob is off by dT + 2^-24
  of itself, the entropy by dT (2 + 2 (1.45 E|x - max| + 8)) + 2^-24 of itself.
"""
import numpy as np
import pytest
import torch

from oracle import paged, requests
from paper_2405_04532_amd import api, workloads as wl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
D, PAGE = 128, 64


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _heads(rows, heads, seed, values=False, gain=8.0):
    return wl.make_kv(1, heads, rows, D, seed, DEV, gain=gain)[int(values)][0].transpose(0, 1).contiguous()


def _same(a, b):
    return bool(((a.view(torch.int16) == b.view(torch.int16)) | (a.isnan() & b.isnan())).all()) if a.dtype == torch.float16 else bool(
        ((a == b) | (a.isnan() & b.isnan())).all())


# ------------------------------------------------------------------------------------------------------------------
# Shared prefixes
# ------------------------------------------------------------------------------------------------------------------
class _Batch:
    """Sequences with their own copies of nothing: whole pages of a prefix are shared, the page in which it ends is the first member's."""

    def __init__(self, groups, lens, Hkv, seed, width=None, spare=2, values=None):
        # groups: (first, behind the last, prefix); lens: tokens of every sequence in all
        self.lens, self.Hkv, self.B = lens, Hkv, len(lens)
        self.cu = [g[0] for g in groups] + [groups[-1][1]] if groups else [0]
        self.prefix = [g[2] for g in groups]
        first = {b: (a, p) for a, e, p in groups for b in range(a, e)}
        reach = [max(n, first.get(b, (b, 0))[1] if first.get(b, (b, 0))[0] == b else 0) for b, n in enumerate(lens)]
        self.width = width or max(1, max(-(-max([n] + [p for _, _, p in groups]) // PAGE) for n in reach))
        need = []                                                              # pages of each sequence that are its own
        for b, n in enumerate(reach):
            a, p = first.get(b, (b, 0))
            need.append(-(-n // PAGE) - (0 if a == b else min(p, n) // PAGE))
        self.pages = sum(need) + spare
        perm = torch.randperm(self.pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
        table, at = torch.full((self.B, self.width), -1, dtype=torch.int32), 0
        for b, n in enumerate(reach):
            a, p = first.get(b, (b, 0))
            skip = 0 if a == b else min(p, n) // PAGE
            table[b, :skip] = table[a, :skip]
            table[b, skip:skip + need[b]] = perm[at:at + need[b]]
            at += need[b]
        # rows written: the first member all that it reaches, the others what lies behind the prefix
        starts = [0 if first.get(b, (b, 0))[0] == b else min(first[b][1], n) for b, n in enumerate(lens)]
        rows = [max(n - s, 0) for n, s in zip(reach, starts)]
        cu = np.concatenate(([0], np.cumsum(rows)))
        M = int(cu[-1])
        k, v = _heads(max(M, 1), Hkv, seed), _heads(max(M, 1), Hkv, seed + 1, True)
        v = values(v) if values else v
        self.table = table.to(DEV)
        self.pool = torch.full((self.pages * Hkv * 8704,), 0xFF, dtype=torch.uint8, device=DEV)    # NaN parameters where nothing is written
        api.kv4_paged_append(self.pool, k[:M].contiguous(), v[:M].contiguous(), self.table, _ints(cu.tolist()), _ints(starts))
        kq, vq = paged.quantized(k.cpu().numpy()), paged.quantized(v.cpu().numpy())
        held = {}                                                              # (page, token) -> row
        for b in range(self.B):
            for i in range(rows[b]):
                held[paged.place(table.numpy(), self.pages, b, starts[b] + i)] = int(cu[b]) + i
        self.rows = lambda t, b, pos: held.get(paged.place(t, self.pages, b, pos))
        self.read = lambda b, t: (lambda row: None if row is None else (kq[row], vq[row]))(self.rows(self.table_np, b, t))
        self.table_np = table.numpy()

    def call(self, q, lens=None, groups=True, **kw):
        cu, prefix = (self.cu, self.prefix) if groups else ([0], [])
        return api.kv4_shared_attention_decode(q, self.pool, self.table, _ints(self.lens if lens is None else lens), _ints(cu),
                                               _ints(prefix) if prefix else torch.empty(0, dtype=torch.int32, device=DEV), self.Hkv, **kw)

    def check(self, out, q, lens=None, cu=None, prefix=None):
        got, qd = out.cpu().numpy().astype(np.float64), q.cpu().numpy().astype(np.float64)
        ref = requests.shared_attention(qd, self.read, self.lens if lens is None else lens, self.cu if cu is None else cu, self.prefix if prefix is None else prefix)
        for b, (want, spread, k) in enumerate(ref):
            L, r = len(k), q.shape[1] // self.Hkv
            e = max([float((np.abs(k[:, h // r]) @ np.abs(qd[b, h])).max()) for h in range(q.shape[1])] if L else [0.0]) * 130 * 2.0 ** -24 / np.sqrt(128.0)
            tol = 2.0 ** -11 * np.abs(want) + (2.0 ** -11 + 2 * e + 2.0 ** -20 + (L + 160) * 2.0 ** -24) * spread + 15 * L * 2.0 ** -25 + 2.0 ** -25
            assert (np.abs(got[b] - want) <= tol).all(), (b, L, float((np.abs(got[b] - want) / tol).max()))
            if L == 0:
                assert not got[b].any()


@pytest.mark.parametrize("H,Hkv", [(4, 4), (8, 2), (7, 1), (16, 1), (9, 1), (6, 2)])
@pytest.mark.parametrize("prefix", [1, 31, 32, 33, 63, 64, 65, 100, 192, 250])
def test_shared(H, Hkv, prefix):
    lens = [prefix + n for n in (1, 5, 0, 31, 64, 200)] + [0, prefix // 2, prefix + 40]
    s = _Batch([(0, len(lens), prefix)], lens, Hkv, 31 + H)
    q = wl.make_queries(len(lens), H, D, 33, DEV)
    s.check(s.call(q), q)


@pytest.mark.parametrize("H,Hkv,groups,lens", [
    (4, 2, [(0, 3, 70), (3, 4, 130), (4, 9, 0), (9, 12, 64)], [80, 70, 200, 131, 5, 64, 65, 1, 0, 65, 100, 64]),     # a group of one, one without a prefix
    (8, 8, [(2, 5, 90), (5, 6, 33)], [17, 130, 100, 91, 90, 40, 300, 1]),                                             # sequences in front and behind
    (3, 1, [(0, 70, 129)], [129 + i for i in range(70)]),                                                             # more columns than a tile, heads that do not divide it
    (16, 1, [(0, 33, 65), (33, 40, 66)], [65 + (i * 7) % 50 for i in range(40)]),
    (2, 2, [], [100, 0, 65]),                                                                                         # no groups at all
    (2, 1, [(i, i + 1, i) for i in range(150)], [i + 3 for i in range(150)])])                                        # more groups than lanes
def test_shared_groups(H, Hkv, groups, lens):
    s = _Batch(groups, lens, Hkv, 41)
    q = wl.make_queries(len(lens), H, D, 43, DEV)
    s.check(s.call(q), q)


@pytest.mark.parametrize("B,H,Hkv,prefix,own", [(3, 4, 1, 4100, 700), (40, 8, 2, 1500, 40), (2, 16, 1, 3000, 1), (12, 8, 8, 900, 300)])
def test_shared_by_workgroups(B, H, Hkv, prefix, own):
    """Long prefixes cut over workgroups, in a workspace of any contents; the same bits every time, in graphs too, and within the bound of
    the call that reads every sequence by itself."""
    lens = [prefix + own - i * own // (2 * B) for i in range(B)]
    s = _Batch([(0, B, prefix)], lens, Hkv, 51)
    q = wl.make_queries(B, H, D, 53, DEV)
    need = api.kv4_shared_attention_workspace_bytes(B, H, Hkv, s.width, 1)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV)
    out = s.call(q, workspace=ws)
    pick = sorted({0, 1, B // 2, B - 1})
    got, want = out.cpu().numpy().astype(np.float64), requests.shared_attention(q.cpu().numpy().astype(np.float64)[pick],
                                                                                lambda i, t: s.read(pick[i], t) if t >= prefix else s.read(0, t),
                                                                                [lens[b] for b in pick], [0], [])
    for i, b in enumerate(pick):
        ref, spread, k = want[i]
        e = max(float((np.abs(k[:, h // (H // Hkv)]) @ np.abs(q[b, h].cpu().numpy().astype(np.float64))).max()) for h in range(H)) * 130 * 2.0 ** -24 / np.sqrt(128.0)
        tol = 2.0 ** -11 * np.abs(ref) + (2.0 ** -11 + 2 * e + 2.0 ** -20 + (len(k) + 160) * 2.0 ** -24) * spread + 15 * len(k) * 2.0 ** -25 + 2.0 ** -25
        assert (np.abs(got[b] - ref) <= tol).all(), (b, float((np.abs(got[b] - ref) / tol).max()))
    for _ in range(3):
        assert _same(s.call(q, workspace=ws), out)
    assert _same(s.call(q), out)
    # two captured graphs that take turns in one workspace, with shorter sequences in the second
    outs, graphs, short = [torch.zeros_like(out), torch.zeros_like(out)], [], [n // 2 for n in lens]
    cu, pl, seqs = _ints(s.cu), _ints(s.prefix), [_ints(lens), _ints(short)]
    want = [out, s.call(q, lens=short, workspace=ws)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for o, seq in zip(outs, seqs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            api.kv4_shared_attention_decode(q, s.pool, s.table, seq, cu, pl, Hkv, out=o, workspace=ws)
        graphs.append(graph)
    for _ in range(3):
        for o in outs:
            o.zero_()
        for graph in graphs:
            graph.replay()
        assert _same(s.call(q, workspace=ws), out)
        torch.cuda.synchronize()
        assert _same(outs[0], want[0]) and _same(outs[1], want[1])
    with pytest.raises(api.QoqError):
        s.call(q, workspace=ws[:need - 16])


def _check_some(s, out, q, lens, pick, bounds):
    """The bound of _Batch.check for some of the sequences; bounds: (first, behind the last, prefix) of the groups."""
    H, R = q.shape[1], q.shape[1] // s.Hkv
    of = {b: (a, p) for a, e, p in bounds for b in range(a, e)}
    qd, got = q.cpu().numpy().astype(np.float64), out.cpu().numpy().astype(np.float64)
    read = lambda i, t: s.read(of.get(pick[i], (pick[i], 0))[0] if t < of.get(pick[i], (0, 0))[1] else pick[i], t)
    for i, (ref, spread, k) in enumerate(requests.shared_attention(qd[pick], read, [lens[b] for b in pick], [0], [])):
        b = pick[i]
        e = max([float((np.abs(k[:, h // R]) @ np.abs(qd[b, h])).max()) for h in range(H)] if len(k) else [0.0]) * 130 * 2.0 ** -24 / np.sqrt(128.0)
        tol = 2.0 ** -11 * np.abs(ref) + (2.0 ** -11 + 2 * e + 2.0 ** -20 + (len(k) + 160) * 2.0 ** -24) * spread + 15 * len(k) * 2.0 ** -25 + 2.0 ** -25
        assert (np.abs(got[b] - ref) <= tol).all(), (b, float((np.abs(got[b] - ref) / tol).max()))


@pytest.mark.parametrize("H,Hkv,groups,B", [
    (32, 2, [(0, 256, 2176)], 256), (32, 2, [(0, 256, 2177)], 256), (32, 2, [(0, 255, 2300)], 256),     # 34, 35 and 36 pages for 64 tiles of 128 columns
    (9, 1, [(1, 600, 3361)], 601), (9, 1, [(1, 600, 3700)], 601),                                       # heads that do not divide a tile
    (32, 8, [(2, 120, 2500), (120, 121, 100), (121, 290, 2943), (290, 299, 0)], 300)])
def test_shared_of_many_sequences_behind_long_prefixes(H, Hkv, groups, B):
    of = {b: p for a, e, p in groups for b in range(a, e)}
    lens = [of.get(b, 0) + (b * 7) % 90 for b in range(B)]
    for a, e, p in groups:                                                   # members without tokens, with one, and that end inside the prefix or with it
        for b, n in zip(range(a + 1, e), (0, 1, p // 2, p // 2 + 1, p - 1, p)):
            lens[b] = max(n, 0)
    s = _Batch(groups, lens, Hkv, 141)
    q = wl.make_queries(B, H, D, 143, DEV)
    pick = sorted({0, B - 1} | {b for a, e, _ in groups for b in (a, a + 1, a + 2, a + 3, a + 5, a + 6, (a + e) // 2, e - 1) if b < e})
    out = s.call(q)
    _check_some(s, out, q, lens, pick, groups)
    for _ in range(3):
        assert _same(s.call(q), out)


@pytest.mark.parametrize("B,H,Hkv,groups", [
    (300, 16, 4, []), (7, 9, 1, []), (40, 32, 32, []),                       # no groups: one launch
    (400, 12, 4, [(0, 400, 300)]), (130, 8, 8, [(3, 60, 129), (60, 61, 70), (61, 125, 500)]),
    (1100, 16, 1, [(i * 10, i * 10 + 9, 40 + i) for i in range(110)]),       # more groups than lanes
    (520, 32, 2, [(0, 510, 2300)])])                                         # heads of a KV head in parts that differ
def test_shared_of_sequences_that_fill_the_chip(B, H, Hkv, groups):
    of = {b: p for a, e, p in groups for b in range(a, e)}
    lens = [of.get(b, 0) + (b * 5) % 70 for b in range(B)]
    for a, e, p in groups:
        for b, n in zip(range(a + 1, min(e, a + 6)), (0, 1, p // 2, p - 1, p)):
            lens[b] = max(n, 0)
    s = _Batch(groups, lens, Hkv, 161)
    q = wl.make_queries(B, H, D, 163, DEV)
    pick = sorted({0, 1, B - 1} | {b for a, e, _ in groups[::9] for b in (a, a + 1, a + 2, a + 3, a + 5, (a + e) // 2, e - 1) if b < e})
    ws = torch.full((api.kv4_shared_attention_workspace_bytes(B, H, Hkv, s.width, len(groups)),), 0xFF, dtype=torch.uint8, device=DEV)
    out = s.call(q, workspace=ws)
    _check_some(s, out, q, lens, pick, groups)
    for _ in range(3):
        assert _same(s.call(q), out)


@pytest.mark.parametrize("B,H,Hkv,prefix", [(256, 32, 2, 2300), (5, 8, 2, 300), (300, 16, 4, 130)])
@pytest.mark.parametrize("size", [2.0 ** -16, 2.0 ** -8, 1.0, 2.0 ** 7, 2.0 ** 14])
@pytest.mark.parametrize("heavy", [False, True])
def test_shared_values_of_any_size(B, H, Hkv, prefix, size, heavy):
    """Values up to `size`; heavy: every 50th token's 256 times the others'.  A product of weight and scale is off by 2^-33 of the largest scale at most where that
    is more than 2^-11 of itself, and a value is at most 15 scales and the weights' sum at least one: L 2^-33 15 s, with 15 s the range of the largest value
    and zero or the least, at most twice its size (of a half's subnormal steps one more, 15 2^-24 / 2)."""
    def values(v):
        v = v.float() / v.abs().max().float() * size
        if heavy:
            v[torch.arange(len(v), device=DEV) % 50 != 7] /= 256
        return v.half()
    groups = [(0, B, prefix)]
    lens = [prefix + (b * 3) % 40 if b % 5 else prefix - b for b in range(B)]
    s = _Batch(groups, lens, Hkv, 181, values=values)
    q = wl.make_queries(B, H, D, 183, DEV)
    out = s.call(q)
    pick = [0, 1, B // 2, B - 1]
    qd, got = q.cpu().numpy().astype(np.float64), out.cpu().numpy().astype(np.float64)
    read = lambda i, t: s.read(0 if t < prefix else pick[i], t)
    for i, (ref, spread, k) in enumerate(requests.shared_attention(qd[pick], read, [lens[b] for b in pick], [0], [])):
        b, L = pick[i], len(k)
        e = max([float((np.abs(k[:, h // (H // Hkv)]) @ np.abs(qd[b, h])).max()) for h in range(H)] if L else [0.0]) * 130 * 2.0 ** -24 / np.sqrt(128.0)
        tol = 2.0 ** -11 * np.abs(ref) + (2.0 ** -11 + 2 * e + 2.0 ** -20 + (L + 160) * 2.0 ** -24) * spread + L * 2.0 ** -33 * 2 * size + 2.0 ** -25
        assert (np.abs(got[b] - ref) <= tol).all(), (b, float((np.abs(got[b] - ref) / tol).max()))


@pytest.mark.parametrize("B,H,Hkv,prefix,cu", [(256, 32, 2, 2300, [0, 256, 0, 256, 3, 256]), (1200, 8, 1, 700, [9, 1100, 5, 1200, 0, 1 << 30]),
                                               (6, 8, 2, 200, [0, 6, 0, 6, 0, 6, 0, 6]), (300, 32, 4, 130, [0, 300] * 50)])
def test_shared_groups_that_overlap_touch_nothing_else(B, H, Hkv, prefix, cu):
    """Their results are unspecified, but nothing outside them and the workspace is written, and a call of proper groups is as it was."""
    s = _Batch([(0, B, prefix)], [prefix + b % 9 for b in range(B)], Hkv, 171)
    q = wl.make_queries(B, H, D, 173, DEV)
    want = s.call(q)
    need = api.kv4_shared_attention_workspace_bytes(B, H, Hkv, s.width, len(cu) - 1)
    held, ws = torch.full((B + 2, H, D), 7.0, dtype=torch.float16, device=DEV), torch.full((need + 4096,), 0x55, dtype=torch.uint8, device=DEV)
    before = s.pool.clone()
    api.kv4_shared_attention_decode(q, s.pool, s.table, _ints(s.lens), _ints(cu), _ints([prefix] * (len(cu) - 1)), Hkv, out=held[1:-1], workspace=ws[:need])
    torch.cuda.synchronize()
    assert (held[0] == 7).all() and (held[-1] == 7).all() and (ws[need:] == 0x55).all() and torch.equal(s.pool, before)
    assert _same(s.call(q), want)


def test_shared_many_sequences_limits_and_a_graph_of_other_lengths():
    """One captured call whose prefix grows and shrinks on the device past what changes how the waves share it; what lies behind a sequence's
    length, an infinity or pages that hold none of its tokens, is not in its result."""
    H, Hkv, B, prefix = 32, 2, 256, 2300
    groups = [(0, B, prefix)]
    lens = [prefix + b % 30 if b % 3 else prefix - 3 - b for b in range(B)]
    s = _Batch(groups, lens, Hkv, 151)
    q = wl.make_queries(B, H, D, 153, DEV)
    pick = [0, 1, 2, 3, 90, 129, 255]
    clean = s.call(q)
    _check_some(s, clean, q, lens, pick, groups)
    cu, pl, seq, out = _ints(s.cu), _ints([prefix]), _ints(lens), torch.zeros_like(clean)
    ws = torch.full((api.kv4_shared_attention_workspace_bytes(B, H, Hkv, s.width, 1),), 0xFF, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        api.kv4_shared_attention_decode(q, s.pool, s.table, seq, cu, pl, Hkv, out=out, workspace=ws)
    for tokens in (prefix, 640, 2177, 1, 2176, 0, prefix):
        # behind a shorter prefix the sequences' own pages hold the rest of it, but in the page in which it ends: lengths end with it
        now = [min(n, tokens) if n >= tokens else n for n in lens] if tokens != prefix else lens
        pl.copy_(_ints([tokens])), seq.copy_(_ints(now)), out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        _check_some(s, out, q, now, pick, [(0, B, tokens)])
        assert _same(api.kv4_shared_attention_decode(q, s.pool, s.table, seq, cu, pl, Hkv), out)
    # all sequences end in front of the prefix's last pages, which are none
    short = [min(n, 2200 - b) for b, n in enumerate(lens)]
    table = s.table.clone()
    table[:, 35:] = -1
    got = api.kv4_shared_attention_decode(q, s.pool, table, _ints(short), cu, pl, Hkv)
    _check_some(s, got, q, short, pick, groups)
    # an infinity among the prefix's last tokens
    bad = torch.full((1, Hkv, D), float("inf"), dtype=torch.float16, device=DEV)
    api.kv4_paged_append(s.pool, bad, bad, s.table[:1].contiguous(), _ints([0, 1]), _ints([prefix - 2]))
    got, sees = s.call(q), torch.tensor([n > prefix - 2 for n in lens], device=DEV)
    assert _same(got[~sees], clean[~sees]) and got[sees].isnan().all()


def test_shared_agrees_with_the_call_without_groups():
    """Prefixes of whole pages, which every member's table names: both calls read the same tokens."""
    H, Hkv, lens = 8, 2, [300, 257, 256, 400, 70]
    s = _Batch([(0, 4, 256)], lens, Hkv, 61)
    q = wl.make_queries(5, H, D, 63, DEV)
    whole = api.kv4_paged_attention_decode(q, s.pool, s.table, _ints(lens), Hkv)
    s.check(whole, q)
    s.check(s.call(q), q)
    s.check(s.call(q, groups=False), q, cu=[0], prefix=[])


def test_shared_garbage_lengths_pages_and_groups():
    H, Hkv = 4, 2
    s = _Batch([(0, 3, 128)], [256, 190, 160, 130], Hkv, 71, width=5)
    q = wl.make_queries(4, H, D, 73, DEV)
    lens = _ints([1 << 30, -5, 160, 130])                                   # past the table and below zero
    s.table[0, 1], s.table[2, 2] = -7, s.pages                              # pages that are none: in the prefix, and behind it
    s.table_np = s.table.cpu().numpy()
    out = api.kv4_shared_attention_decode(q, s.pool, s.table, lens, _ints([0, 3]), _ints([128]), Hkv)
    s.check(out, q, lens=[320, 0, 160, 130])
    # lengths of prefixes past the table and below zero
    out = api.kv4_shared_attention_decode(q, s.pool, s.table, _ints([200, 190, 160, 130]), _ints([0, 1, 4]), _ints([-3, 1 << 30]), Hkv)
    s.check(out, q, lens=[200, 190, 160, 130], cu=[0, 1, 4], prefix=[0, 320])
    # bounds outside the batch: the nearest ones
    out = api.kv4_shared_attention_decode(q, s.pool, s.table, _ints([200, 190, 160, 130]), _ints([-4, 1 << 30]), _ints([64]), Hkv)
    s.check(out, q, lens=[200, 190, 160, 130], cu=[0, 4], prefix=[64])


def test_shared_values_that_are_not_finite_reach_the_sequences_that_see_them():
    """An infinity among the prefix's last tokens (its scale is one, its values 0 times that): not in the results of members that end in front of it."""
    H, Hkv, prefix = 4, 2, 100
    lens = [130, 90, 99, 100, 7, 97]
    s = _Batch([(0, 6, prefix)], lens, Hkv, 81)
    q = wl.make_queries(6, H, D, 83, DEV)
    clean = s.call(q)
    s.check(clean, q)
    bad = torch.full((1, Hkv, D), float("inf"), dtype=torch.float16, device=DEV)
    api.kv4_paged_append(s.pool, bad, bad, s.table[:1].contiguous(), _ints([0, 1]), _ints([98]))
    out = s.call(q)
    sees = torch.tensor([n > 98 for n in lens])
    assert _same(out[~sees.to(DEV)], clean[~sees.to(DEV)])
    assert out[sees.to(DEV)].isnan().all()


def test_shared_strided_queries_another_stream_and_refusals():
    H, Hkv, B = 8, 2, 21
    s = _Batch([(0, B, 130)], [131 + 3 * i for i in range(B)], Hkv, 91)
    qkv = _heads(B, H + 2 * Hkv, 92)
    q = qkv[:, :H]
    want = s.call(q.contiguous())
    assert _same(s.call(q), want)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = s.call(q)
    side.synchronize()
    assert _same(got, want)
    out = torch.empty_like(want)
    assert s.call(q, out=out) is out or _same(out, want)
    assert _same(out, want)
    cu, prefix, lens = _ints(s.cu), _ints(s.prefix), _ints(s.lens)
    with pytest.raises(ValueError):
        api.kv4_shared_attention_decode(q, s.pool, s.table, lens, cu, _ints([1, 2]), Hkv)
    with pytest.raises(ValueError):
        api.kv4_shared_attention_decode(q, s.pool, s.table, lens[:3].contiguous(), cu, prefix, Hkv)
    with pytest.raises(TypeError):
        api.kv4_shared_attention_decode(q, s.pool, s.table, lens, cu.long(), prefix, Hkv)
    with pytest.raises(api.QoqError):
        api.kv4_shared_attention_decode(q[:, :7], s.pool, s.table, lens, cu, prefix, Hkv)


def test_shared_two_streams_at_once():
    H, Hkv = 8, 2
    s = _Batch([(0, 9, 700)], [705 + 5 * i for i in range(9)], Hkv, 101)
    q = wl.make_queries(9, H, D, 103, DEV)
    want = s.call(q)
    streams, spaces = [torch.cuda.Stream() for _ in range(2)], [torch.empty(api.kv4_shared_attention_workspace_bytes(9, H, Hkv, s.width, 1), dtype=torch.uint8, device=DEV) for _ in range(2)]
    cu, prefix, lens = _ints(s.cu), _ints(s.prefix), _ints(s.lens)
    torch.cuda.synchronize()
    got = []
    for _ in range(20):
        for stream, ws in zip(streams, spaces):
            with torch.cuda.stream(stream):
                got.append(api.kv4_shared_attention_decode(q, s.pool, s.table, lens, cu, prefix, Hkv, workspace=ws))
    torch.cuda.synchronize()
    assert all(_same(g, want) for g in got)


def test_shared_pages_past_four_gigabytes():
    Hkv, pages = 8, 70000                                                   # 4.87 GB
    pool = torch.empty(pages * Hkv * 8704, dtype=torch.uint8, device=DEV)
    table = _ints([[69999, 65000], [69999, 12]])
    k, v = _heads(100, Hkv, 111), _heads(100, Hkv, 112, True)
    api.kv4_paged_append(pool, k[:90].contiguous(), v[:90].contiguous(), table[:1].contiguous(), _ints([0, 90]))
    api.kv4_paged_append(pool, k[90:].contiguous(), v[90:].contiguous(), table[1:].contiguous(), _ints([0, 10]), _ints([64]))
    q = wl.make_queries(2, 8, D, 113, DEV)
    out = api.kv4_shared_attention_decode(q, pool, table, _ints([90, 74]), _ints([0, 2]), _ints([64]), Hkv)
    want = api.kv4_paged_attention_decode(q, pool, table, _ints([90, 74]), Hkv)
    assert (out.float() - want.float()).abs().max() <= 4 * 2.0 ** -11 * want.float().abs().max() + 1e-4


def _shared_pool(B, Hkv, prefix, own, seed):
    """Sequences of prefix (whole pages) + own tokens, keys with a channel (5) that no token has at zero."""
    width, first = -(-(prefix + own) // PAGE), prefix // PAGE
    n_own, M = width - first, prefix + B * own
    table = torch.empty((B, width), dtype=torch.int32)
    table[:, :first] = torch.arange(first)
    table[:, first:] = first + torch.arange(B * n_own).view(B, n_own)
    table = table.to(DEV)
    k, v = _heads(M, Hkv, seed), _heads(M, Hkv, seed + 1, True)
    k[..., 5] = k.abs().amax(-1).clamp(min=1.0)
    pool = torch.full(((first + B * n_own) * Hkv * 8704,), 0xFF, dtype=torch.uint8, device=DEV)
    starts = [0] + [prefix] * (B - 1)
    cu = [0] + [prefix + (b + 1) * own for b in range(B)]
    api.kv4_paged_append(pool, k, v, table, _ints(cu), _ints(starts))
    return pool, table


@pytest.mark.parametrize("B,H,Hkv,prefix,own", [(6, 8, 2, 192, 50), (3, 16, 1, 4096, 300), (300, 32, 4, 128, 40), (256, 32, 2, 2304, 30)])
def test_shared_queries_whose_scores_are_all_minus_infinity(B, H, Hkv, prefix, own):
    """A softmax of nothing but minus infinity is none: NaN, as in prompt attention, in that query's row alone; a sequence without tokens, or
    whose pages are none, has a zero row whatever its query is.  With and without groups, and in the call that has none."""
    pool, table = _shared_pool(B, Hkv, prefix, own, 201)
    lens = [prefix + own - b % 7 for b in range(B)]
    lens[1], lens[2] = prefix - 3, 0                                        # inside the prefix; nothing
    q = wl.make_queries(B, H, D, 203, DEV)
    bad = q.clone()
    hit = torch.zeros((B, H), dtype=torch.bool, device=DEV)
    for b, h in ((0, 0), (0, H - 1), (1, 1), (2, 0), (B - 1, 2), (B // 2, H // 2)):
        bad[b, h, 5] = -float("inf")
        hit[b, h] = lens[b] > 0
    cu, pl, ln = _ints([0, B]), _ints([prefix]), _ints(lens)
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    ws = api.new_workspace(api.kv4_paged_attention_workspace_bytes(B, H, Hkv, table.shape[1]), DEV)
    for call in (lambda t: api.kv4_shared_attention_decode(t, pool, table, ln, cu, pl, Hkv),
                 lambda t: api.kv4_shared_attention_decode(t, pool, table, ln, _ints([0]), none, Hkv),
                 lambda t: api.kv4_paged_attention_decode(t, pool, table, ln, Hkv), lambda t: api.kv4_paged_attention_decode(t, pool, table, ln, Hkv, workspace=ws)):
        clean, out = call(q), call(bad)
        assert torch.isfinite(clean).all() and out[hit].isnan().all() and _same(out[~hit], clean[~hit])
        assert not out[2].any()
    gone = table.clone()
    gone[0], gone[B - 1] = -1, 1 << 30
    keep = [b for b in range(B) if b not in (0, B - 1)]
    out, clean = (api.kv4_shared_attention_decode(t, pool, gone, ln, _ints([0]), none, Hkv) for t in (bad, q))
    assert not out[[0, B - 1]].any() and out[hit & (torch.arange(B, device=DEV) % (B - 1) > 0)[:, None]].isnan().all()
    assert _same(out[keep][~hit[keep]], clean[keep][~hit[keep]])


@pytest.mark.parametrize("B,H,Hkv", [(5, 8, 2), (40, 16, 1)])
def test_shared_of_more_groups_than_sequences(B, H, Hkv):
    """Most groups hold no sequence: in front of, between and behind those that do."""
    G, prefix = 2000, 130
    held = [(0, 2, prefix), (2, 3, 70), (3, B, 200)]
    lens = [next(p for a, e, p in held if a <= b < e) + 3 + b for b in range(B)]
    s = _Batch(held, lens, Hkv, 211)
    cu, pl = [0] * 700 + [2] * 300 + [3] * 500 + [B] * (G + 1 - 1500), [5] * G
    pl[699], pl[999], pl[1499] = prefix, 70, 200                            # the last group that begins in front of each bound holds what lies there
    q = wl.make_queries(B, H, D, 213, DEV)
    out = api.kv4_shared_attention_decode(q, s.pool, s.table, _ints(lens), _ints(cu), _ints(pl), Hkv)
    s.check(out, q)
    assert _same(out, s.call(q)) or (out.float() - s.call(q).float()).abs().max() < 1e-2


def test_shared_of_long_prefixes_in_more_groups_than_lanes():
    """70 groups of 128 columns a KV head behind 5 or 6 pages: the units of work of groups 64 and up are counted behind those of the first 64."""
    H, Hkv, n, G = 128, 8, 8, 70
    B = n * G
    groups = [(g * n, g * n + n, (0 if g == 30 else 321 + g % 64)) for g in range(G)]
    units = sum(Hkv * -(-p // PAGE) for _, _, p in groups)
    assert n * (H // Hkv) == 128 and units >= 2250 + 500                    # no column of a tile of 128 is empty: the form of many columns
    lens = [groups[b // n][2] + 1 + (b * 5) % 20 for b in range(B)]
    for g in (0, 63, 64, 69):
        a, p = groups[g][0], groups[g][2]
        lens[a + 1], lens[a + 2], lens[a + 3] = 0, p // 2, p
    s = _Batch(groups, lens, Hkv, 221)
    q = wl.make_queries(B, H, D, 223, DEV)
    out = s.call(q)
    _check_some(s, out, q, lens, [g * n + i for g in (0, 63, 64, 69) for i in (0, 1, 2, 3, 7)] + [30 * n, 31 * n, 65 * n + 4], groups)
    for _ in range(3):
        assert _same(s.call(q), out)
    # bounds that descend: nothing else is touched, and the next call is as it was
    need = api.kv4_shared_attention_workspace_bytes(B, H, Hkv, s.width, G)
    for cu in ([B - g * n for g in range(G + 1)], [(0 if g % 2 else B) for g in range(G + 1)], [(g * 37 % 71) * n for g in range(G + 1)]):
        held, ws = torch.full((B + 2, H, D), 7.0, dtype=torch.float16, device=DEV), torch.full((need + 4096,), 0x55, dtype=torch.uint8, device=DEV)
        before = s.pool.clone()
        api.kv4_shared_attention_decode(q, s.pool, s.table, _ints(s.lens), _ints(cu), _ints(s.prefix), Hkv, out=held[1:-1], workspace=ws[:need])
        torch.cuda.synchronize()
        assert (held[0] == 7).all() and (held[-1] == 7).all() and (ws[need:] == 0x55).all() and torch.equal(s.pool, before)
    assert _same(s.call(q), out)


# ------------------------------------------------------------------------------------------------------------------
# Adapters
# ------------------------------------------------------------------------------------------------------------------
def _half(seed, *shape, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * scale).half()


def _lora_inputs(M, N, K, rank, adapters, seed):
    x = _half(seed, M, K)
    x[:, ::97] *= 20.0
    return (_half(seed + 1, M, N), x, _half(seed + 2, adapters, rank, K, scale=K ** -0.5), _half(seed + 3, adapters, N, rank, scale=0.1),
            torch.rand(adapters, generator=torch.Generator().manual_seed(seed)).add(0.5).to(DEV))


def _check_lora(out, base, x, a, b, rows, scales, pick=None):
    pick = list(range(len(rows))) if pick is None else pick
    used = sorted({rows[m] for m in pick if 0 <= rows[m] < a.shape[0]}) or [0]
    at = {n: i for i, n in enumerate(used)}
    f = lambda t: t.cpu().numpy().astype(np.float64)      # noqa: E731
    ref, off = requests.lora(f(base[pick]), f(x[pick]), f(a[used]), f(b[used]), [at.get(rows[m], -1) for m in pick], None if scales is None else f(scales[used]))
    got = f(out[pick])
    with np.errstate(invalid="ignore"):                                     # (what is not finite in the definition is the same here)
        tol = 2.0 ** -11 * np.abs(ref) + off + 2.0 ** -25
        assert ((np.abs(got - ref) <= tol) | (got == ref) & np.isinf(ref) | np.isnan(got) & np.isnan(ref)).all(), float(np.nanmax(np.abs(got - ref) / tol))


@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 64, 130])
@pytest.mark.parametrize("N,K,rank", [(8, 8, 8), (64, 128, 16), (200, 776, 24), (72, 264, 32), (136, 1000, 40), (1032, 4096, 64)])
def test_lora(M, N, K, rank):
    adapters = 5
    base, x, a, b, scales = _lora_inputs(M, N, K, rank, adapters, M + N)
    rows = [(m * 7 + 3) % 6 for m in range(M)]                              # 5: none
    plan = api.lora_plan(_ints(rows), adapters)
    out = api.lora_add(base, x, a, b, plan, scales=scales)
    _check_lora(out, base, x, a, b, rows, scales)


@pytest.mark.parametrize("M,N,K,rank,adapters", [(513, 72, 136, 8, 3), (700, 264, 520, 16, 2), (1100, 520, 264, 64, 9), (600, 200, 2056, 40, 1), (520, 136, 72, 72, 2),
                                                 (640, 136, 200, 200, 600), (30, 264, 136, 512, 4), (5, 136, 264, 104, 4096), (1030, 72, 88, 128, 40)])
def test_lora_tiles_of_64_rows_and_large_ranks(M, N, K, rank, adapters):
    base, x, a, b, scales = _lora_inputs(M, N, K, rank, adapters, 7 * M)
    rows = [(m * m // 50) % (adapters + 2) - 1 for m in range(M)]
    plan = api.lora_plan(_ints(rows), adapters)
    pick = list(range(0, M, 13)) + [M - 1]
    out = api.lora_add(base, x, a, b, plan, scales=scales)
    _check_lora(out, base, x, a, b, rows, scales, pick)
    none = [m for m in range(M) if not 0 <= rows[m] < adapters]
    if none:
        assert _same(out[none], base[none])
    again = api.lora_add(base, x, a, b, api.lora_plan(_ints(rows), adapters), scales=scales)
    assert _same(out, again)                                               # whatever the order in a tile


@pytest.mark.parametrize("M", [33, 600])
def test_lora_in_place_strided_and_without_scales(M):
    """Onto slices of a fused projection's output, from a slice of wider activations; what lies beside is left alone."""
    N, K, rank, adapters = 192, 256, 16, 3
    _, x, a, b, _ = _lora_inputs(M, N, K, rank, adapters, 5)
    wide_x, fused = _half(11, M, K + 24), _half(12, M, 3 * N)
    wide_x[:, 8:8 + K] = x
    rows = [m % 4 for m in range(M)]
    plan = api.lora_plan(_ints(rows), adapters)
    keep = fused.clone()
    out = api.lora_add(fused[:, N:2 * N], wide_x[:, 8:8 + K], a, b, plan, out=fused[:, N:2 * N])
    assert out.data_ptr() == fused[:, N:2 * N].data_ptr()
    _check_lora(fused[:, N:2 * N], keep[:, N:2 * N], x, a, b, rows, None, list(range(0, M, 7)))
    assert _same(fused[:, :N], keep[:, :N]) and _same(fused[:, 2 * N:], keep[:, 2 * N:])
    assert _same(fused[3::4, N:2 * N], keep[3::4, N:2 * N])
    apart = torch.full((M, N + 8), 7.0, dtype=torch.float16, device=DEV)
    api.lora_add(keep[:, N:2 * N], x, a, b, plan, out=apart[:, :N])
    assert _same(apart[:, :N], fused[:, N:2 * N]) and (apart[:, N:] == 7.0).all()


def test_lora_of_no_rows_and_of_rows_without_adapters():
    base, x, a, b, scales = _lora_inputs(40, 64, 64, 8, 2, 3)
    empty = torch.empty(0, dtype=torch.int32, device=DEV)
    assert api.lora_add(base[:0], x[:0], a, b, api.lora_plan(empty, 2)).shape == (0, 64)
    for value in (-1, 2, 1 << 30, -(1 << 31)):
        assert _same(api.lora_add(base, x, a, b, api.lora_plan(_ints([value] * 40), 2), scales=scales), base)


def test_lora_plan_of_another_batch_writes_nothing():
    base, x, a, b, _ = _lora_inputs(40, 64, 64, 8, 2, 3)
    for plan in (api.lora_plan(_ints([0] * 41), 2), api.lora_plan(_ints([0] * 40), 3), torch.zeros(1000, dtype=torch.int32, device=DEV),
                 torch.full((1000,), 40, dtype=torch.int32, device=DEV)):
        out = torch.full_like(base, 7.0)
        api.lora_add(base, x, a, b, plan, out=out)
        assert (out == 7.0).all()


@pytest.mark.parametrize("M", [20, 530])
def test_lora_infinities_and_large_numbers(M):
    """What is not finite stays in its row; middle products past FP16's range count in full."""
    N, K, rank = 72, 136, 16
    base, x, a, b, scales = _lora_inputs(M, N, K, rank, 2, 9)
    rows = [m % 2 for m in range(M)]
    plan = api.lora_plan(_ints(rows), 2)
    clean = api.lora_add(base, x, a, b, plan, scales=scales)
    bad = x.clone()
    bad[3, 5], bad[8, 0] = float("nan"), float("inf")
    out = api.lora_add(base, bad, a, b, plan, scales=scales)
    others = [m for m in range(M) if m not in (3, 8)]
    assert _same(out[others], clean[others]) and out[3].isnan().all() and not torch.isfinite(out[8]).any()
    big = (x.float() * 1000.0).half()
    small = (b.float() / 4096.0).half()
    _check_lora(api.lora_add(base, big, (a.float() * 200.0).half(), small, plan, scales=scales), base, big, (a.float() * 200.0).half(), small, rows, scales, others[::5])
    tiny = (x.float() / 60000.0).half()
    _check_lora(api.lora_add(base, tiny, a, b, plan, scales=scales), base, tiny, a, b, rows, scales, others[::5])


@pytest.mark.parametrize("M,rank", [(20, 8), (20, 16), (37, 24), (37, 32), (37, 48), (37, 64), (20, 136), (300, 32), (530, 8), (530, 40), (530, 64), (600, 200)])
def test_lora_infinities_and_nan_in_b(M, rank):
    """Of a channel whose B holds an infinity, a row's result is the infinity that the definition gives (NaN where 0 or both signs meet it), also
    where x A^T is far below the row's other ranks; the other channels are untouched, in place as well."""
    N, K, inf = 200, 264, float("inf")
    base, x, a, b, scales = _lora_inputs(M, N, K, rank, 2, 900 + rank)
    x[5] = 0
    a[0, 0] *= 500.0
    a[0, 1] = 0
    a[0, 1, 0] = 2.0 ** -24                                                 # 2^-24 x beside some 10^4
    x[::2, 0] = x[::2, 0].clamp(min=2.0 ** -8, max=2.0 ** -6)
    rows = [m % 3 for m in range(M)]
    plan = api.lora_plan(_ints(rows), 2)
    clean = api.lora_add(base, x, a, b, plan, scales=scales)
    b[0, 3, 1], b[0, 70, rank - 1], b[0, 131, 0], b[1, 131, 5] = inf, -inf, inf, -inf
    b[1, 199, 0] = float("nan")
    b[1, 64, 2], b[1, 64, 3], b[0, 65, 4], b[0, 65, rank // 2] = inf, -inf, inf, inf
    out = api.lora_add(base, x, a, b, plan, scales=scales)
    f = lambda t: t.cpu().numpy().astype(np.float64)      # noqa: E731
    with np.errstate(invalid="ignore"):
        ref, _ = requests.lora(f(base), f(x), f(a), f(b), [n if n < 2 else -1 for n in rows], f(scales))
    got, was, bad = f(out), f(clean), ~np.isfinite(ref)
    assert np.isinf(ref).any() and np.isnan(ref).any() and bad.sum() > 6 * M // 4
    assert ((got == ref) | (np.isnan(got) & np.isnan(ref)))[bad].all(), np.argwhere(bad & ~((got == ref) | (np.isnan(got) & np.isnan(ref))))[:5]
    assert (got == was)[~bad].all()
    api.lora_add(base, x, a, b, plan, scales=scales, out=base)
    assert _same(base, out)


@pytest.mark.parametrize("M,rank", [(16, 8), (16, 72), (520, 8), (520, 64)])
@pytest.mark.parametrize("largest", [1.0, 1.0009765625, 1.9990234375])
def test_lora_small_middle_products_beside_large_ones(M, rank, largest):
    """Middle products of c 2^-41 beside one of `largest`, each brought to its own channel 2^39 times: off by 2^-22 of itself or 2^-39 of the largest,
    and the result's rounding (each is a single product, so nothing else is rounded)."""
    base = torch.zeros((M, 64), dtype=torch.float16, device=DEV)
    x, a, b = torch.zeros((M, 8), device=DEV), torch.zeros((1, rank, 8), device=DEV), torch.zeros((1, 64, rank), device=DEV)
    x[:, 0], x[:, 1] = largest, 2.0 ** -20
    a[0, 0, 0] = 1.0
    c = torch.zeros(64, device=DEV)
    for n in range(1, min(rank, 64)):
        c[n] = n % 15 + 1
        a[0, n, 1], b[0, n, n] = float(c[n]) * 2.0 ** -21, 1.0
    out = api.lora_add(base, x.half(), a.half(), b.half(), api.lora_plan(_ints([0] * M), 1), scales=torch.tensor([2.0 ** 39], device=DEV))
    want = c.double() / 4
    tol = 2.0 ** -22 * want + largest + 2.0 ** -11 * (want + largest)
    assert ((out.double() - want).abs() <= tol).all(), float(((out.double() - want).abs() / tol).max())


def test_lora_graph_with_its_plan_and_streams():
    """Plan and two projections in one graph, replayed with other adapters and activations in the same tensors; overlapping calls."""
    M, K, rank, adapters = 48, 512, 16, 6
    base, x, a, b, scales = _lora_inputs(M, 320, K, rank, adapters, 21)
    base2, x2, a2, b2, _ = _lora_inputs(M, 128, 320, rank, adapters, 22)
    need = max(api.lora_workspace_bytes(M, 320, K, rank, adapters), api.lora_workspace_bytes(M, 128, 320, rank, adapters))
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV)
    row = _ints([m % 7 for m in range(M)])
    plan, outs = api.lora_plan(row, adapters), [torch.empty_like(base), torch.empty_like(base2)]

    def step():
        api.lora_plan(row, adapters, out=plan)
        api.lora_add(base, x, a, b, plan, scales=scales, out=outs[0], workspace=ws)
        api.lora_add(base2, outs[0], a2, b2, plan, scales=scales, out=outs[1], workspace=ws)

    def fill(i):
        row.copy_(_ints([(m * (i + 1)) % 7 for m in range(M)]))
        x.copy_(_half(30 + i, M, K))

    want = []
    for i in range(3):
        fill(i)
        step()
        want.append([o.clone() for o in outs])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for i in (0, 1, 2, 1, 0):
        fill(i)
        for o in outs:
            o.fill_(7.0)
        graph.replay()
        assert _same(outs[0], want[i][0]) and _same(outs[1], want[i][1])
        torch.cuda.synchronize()
        api.lora_add(base, x, a, b, plan, workspace=ws)
    fill(0)
    api.lora_plan(row, adapters, out=plan)
    torch.cuda.synchronize()
    streams, spaces, got = [torch.cuda.Stream() for _ in range(2)], [api.new_workspace(need, DEV) for _ in range(2)], []
    torch.cuda.synchronize()
    for _ in range(20):
        for stream, space in zip(streams, spaces):
            with torch.cuda.stream(stream):
                got.append(api.lora_add(base, x, a, b, plan, scales=scales, workspace=space))
    torch.cuda.synchronize()
    assert all(_same(g, want[0][0]) for g in got)


@pytest.mark.parametrize("M,N,K,rank,adapters", [(20, 264, 4096, 8, 3), (37, 136, 4096, 64, 5), (300, 200, 2056, 32, 20), (7, 72, 1000, 200, 2), (9, 64, 8, 136, 2), (700, 136, 1032, 40, 4)])
def test_lora_workspace_of_any_contents_and_graphs_that_share_it(M, N, K, rank, adapters):
    """Sums joined by the second product and by a launch between, for few rows and many, one chunk of ranks and several."""
    base, x, a, b, scales = _lora_inputs(M, N, K, rank, adapters, 300 + M)
    rows = [(m * 5) % (adapters + 1) for m in range(M)]
    plan = api.lora_plan(_ints(rows), adapters)
    need = api.lora_workspace_bytes(M, N, K, rank, adapters)
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device=DEV)
    out = api.lora_add(base, x, a, b, plan, scales=scales, workspace=ws[:need])
    _check_lora(out, base, x, a, b, rows, scales, list(range(0, M, 11)) + [M - 1])
    assert (ws[need:] == 0xFF).all()
    half = torch.zeros_like(out)
    other = api.lora_add(half, x, a, b, plan)                               # another base, without scales
    outs, graphs = [torch.empty_like(out), torch.empty_like(out)], []
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for o, args in zip(outs, ((base, scales), (half, None))):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            api.lora_add(args[0], x, a, b, plan, scales=args[1], out=o, workspace=ws[:need])
        graphs.append(graph)
    for _ in range(3):
        ws.fill_(0xFF)
        for o, graph in zip(outs, graphs):
            o.fill_(7.0)
            graph.replay()
        torch.cuda.synchronize()
        assert _same(outs[0], out) and _same(outs[1], other)
        assert _same(api.lora_add(base, x, a, b, plan, scales=scales), out)
    with pytest.raises(api.QoqError):
        api.lora_add(base, x, a, b, plan, workspace=ws[:need - 16])


def test_calls_on_nothing():
    got = api.token_logprobs(torch.empty((0, 100), dtype=torch.float16, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV), top=5)
    assert [tuple(t.shape) for t in got] == [(0,), (0,), (0,), (0, 5), (0, 5)]
    with pytest.raises(api.QoqError):
        api.token_logprobs(torch.zeros((2, 4), dtype=torch.float16, device=DEV), top=5)
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    out = api.kv4_shared_attention_decode(torch.empty((0, 8, D), dtype=torch.float16, device=DEV), torch.zeros(2 * 2 * 8704, dtype=torch.uint8, device=DEV),
                                          torch.empty((0, 3), dtype=torch.int32, device=DEV), none, _ints([0]), none, 2)
    assert out.shape == (0, 8, D)


def test_lora_binding_refuses():
    base, x, a, b, scales = _lora_inputs(8, 64, 64, 8, 2, 3)
    plan = api.lora_plan(_ints([0] * 8), 2)
    for args in ((base, x[:7], a, b, plan), (base, x, a[:1], b, plan), (base, x, a, b[:, :32].contiguous(), plan), (base, x, a[:, :, :32].contiguous(), b, plan)):
        with pytest.raises(ValueError):
            api.lora_add(*args)
    with pytest.raises(TypeError):
        api.lora_add(base.float(), x, a, b, plan)
    with pytest.raises(ValueError):
        api.lora_add(base, x, a, b, plan, scales=scales[:1].contiguous())
    with pytest.raises(ValueError):
        api.lora_add(base.t().contiguous().t(), x, a, b, plan)
    with pytest.raises(api.QoqError):
        api.lora_add(base, x, a, b, plan[:20].contiguous())
    with pytest.raises(api.QoqError):
        api.lora_plan(_ints([0] * 8), 0)


# ------------------------------------------------------------------------------------------------------------------
# Log probabilities
# ------------------------------------------------------------------------------------------------------------------
def _check_logprobs(got, x, tokens, top, rows=None):
    lp, rank, ent, ids, tops = (None if t is None else t.cpu().numpy() for t in got)
    xs = x.detach().cpu().float().numpy()
    V = xs.shape[1]
    for m in range(xs.shape[0]) if rows is None else rows:
        wlp, wrank, went, wids, wtops, dist = requests.logprobs(xs[m], -1 if tokens is None else int(tokens[m]), top)
        dT = 2.0 ** -23 + 2.0 ** -24 * (1.1 * dist + 6) + (V / 64 + 100) * 2.0 ** -24

        def near(a, b, tol):
            a, b = np.asarray(a, dtype=np.float64), np.asarray(b, dtype=np.float64)
            with np.errstate(invalid="ignore"):
                return ((a == b) | (np.isnan(a) & np.isnan(b)) | (np.abs(a - b) <= tol)).all()

        if tokens is not None:
            assert near(lp[m], wlp, dT + 2.0 ** -24 * abs(wlp)), (m, lp[m], wlp)
            assert rank[m] == wrank, (m, rank[m], wrank)
        assert near(ent[m], went, dT * (2 + 2 * (1.45 * dist + 8)) + 2.0 ** -24 * abs(went)), (m, ent[m], went)
        if top:
            assert list(ids[m]) == list(wids), (m, ids[m], wids)
            with np.errstate(invalid="ignore"):
                assert near(tops[m], wtops, dT + 2.0 ** -24 * np.abs(wtops)), (m, tops[m], wtops)


def _logits(M, V, seed, dtype, spread=2.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn((M, V), generator=g, device=DEV) * spread
    x.scatter_add_(1, torch.randint(0, V, (M, 6), generator=g, device=DEV), torch.rand((M, 6), generator=g, device=DEV) * 14.0)
    return x.to(dtype)


def _workspace(x, top):
    return api.new_workspace(api.token_logprobs_workspace_bytes(x.shape[0], x.shape[1], top, x.dtype), DEV)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 31, 63, 100, 255, 257, 1000, 2047, 2048, 2049, 4099, 16385, 32000, 50257])
@pytest.mark.parametrize("top", [0, 1, 5, 32])
def test_logprobs(dtype, V, top):
    M, top = 5, min(top, V)
    x = _logits(M, V, V, dtype)
    tokens = [0, V - 1, int(x[2].float().argmax()), V // 2, V // 3]
    for ws in (None, _workspace(x, top)):
        _check_logprobs(api.token_logprobs(x, _ints(tokens), top, workspace=ws), x, tokens, top)
    _check_logprobs(api.token_logprobs(x, None, top), x, None, top)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("top", [0, 20])
def test_logprobs_strides_and_unaligned_rows(dtype, top):
    """Rows at any element, of any distance; what lies in front and behind does not count."""
    V = 4099
    wide = _logits(9, V + 1037, 3, dtype)
    wide[:, :5], wide[:, 5 + V:] = float("nan"), float("inf")
    for first in (5,):
        x = wide[:, first:first + V]
        tokens = [0, 1, V - 1, 17, 2000, -1, V, 3, 4000]
        for ws in (None, _workspace(x, top)):
            _check_logprobs(api.token_logprobs(x, _ints(tokens), top, workspace=ws), x, tokens, top)
    flat = _logits(1, 12 * 37 + 8, 4, dtype)[0]
    for shift in range(8):
        x = flat[shift:shift + 12 * 37].view(12, 37)
        tokens = list(range(0, 36, 3))
        _check_logprobs(api.token_logprobs(x, _ints(tokens), min(top, 37)), x, tokens, min(top, 37))


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("V", [300, 5003, 40000])
def test_logprobs_of_equal_logits_masks_and_extremes(dtype, shared, V):
    top, low = 20, torch.finfo(dtype).min
    x = torch.zeros((14, V), dtype=dtype, device=DEV)
    x[1] = 3.0
    x[2] = low                                                              # a mask of the type's lowest value everywhere: a uniform row
    x[3] = low
    x[3, V - 2] = 1.0
    x[4] = -float("inf")
    x[4, V // 2] = -5.0                                                     # one token allowed
    x[5] = -float("inf")
    x[5, 7::9] = torch.randn(len(range(7, V, 9)), device=DEV).to(dtype)
    x[6] = torch.arange(V, device=DEV) % 3                                  # many equal ones
    x[7] = -(torch.arange(V, device=DEV) % 2).to(dtype) * 0.0               # zeros of both signs
    x[8] = torch.finfo(dtype).max
    x[9, ::2] = low
    x[10] = torch.linspace(-30, 30, V, device=DEV).to(dtype)
    x[11] = torch.linspace(30, -30, V, device=DEV).to(dtype)
    x[12] = torch.randint(-3, 3, (V,), device=DEV).to(dtype)
    x[13, V // 3] = torch.finfo(dtype).max
    tokens = [V - 1, 5, V // 2, V - 2, 3, 16, V - 1, 1, 0, 1, V // 2, V // 2, V - 1, V // 3]
    ws = _workspace(x, top) if shared else None
    _check_logprobs(api.token_logprobs(x, _ints(tokens), top, workspace=ws), x, tokens, top)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_logprobs_of_rows_without_an_answer(dtype):
    V = 9001
    x = _logits(8, V, 5, dtype)
    x[0, 17], x[1, V - 1], x[2], x[3, 0], x[4, 100], x[4, 200] = float("nan"), float("inf"), -float("inf"), float("nan"), float("inf"), float("nan")
    x[5] = float("nan")
    tokens = [17, 0, 4, V - 1, 100, 1, V - 1, 0]
    for top in (0, 7):
        for ws in (None, _workspace(x, top)):
            _check_logprobs(api.token_logprobs(x, _ints(tokens), top, workspace=ws), x, tokens, top)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("shared", [False, True])
def test_logprobs_of_large_tokens_at_one_distance(dtype, shared):
    """The largest logits all at places that one lane reads, more than can be ranked at once."""
    V, top = 1 << 20, 32
    x = torch.randn((2, V), device=DEV).clamp(-4, 4).to(dtype)
    vec = 16 * 8 // torch.finfo(dtype).bits
    at = (torch.arange(0, V, 256 * vec, device=DEV)[:, None] + torch.arange(vec, device=DEV)).flatten()
    x[0, at] = (torch.rand(at.numel(), device=DEV) * 4 + 8).to(dtype)
    x[1, at] = 9.0
    tokens = [int(at[-1]), int(at[3000])]
    ws = _workspace(x, top) if shared else None
    _check_logprobs(api.token_logprobs(x, _ints(tokens), top, workspace=ws), x, tokens, top)


def test_logprobs_many_rows_and_the_longest():
    x = _logits(3000, 515, 7, torch.float16)
    tokens = [(m * 31) % 515 for m in range(3000)]
    _check_logprobs(api.token_logprobs(x, _ints(tokens), 3, workspace=_workspace(x, 3)), x, tokens, 3, range(0, 3000, 37))
    x = _logits(1, 1 << 24, 8, torch.float16)
    for ws in (None, _workspace(x, 32)):
        _check_logprobs(api.token_logprobs(x, _ints([12345678]), 32, workspace=ws), x, [12345678], 32)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("M,V", [(2, 1 << 24), (3, 1 << 20), (2, 300001), (1100, 128256)])
def test_logprobs_of_long_rows_of_near_equal_logits(dtype, M, V):
    """A workgroup to a row, whose sums are of many terms alike, above the reference that the first ones set: the bound has no term that grows with V
    (8 additions of FP32 within a vector, 32 of vectors, 64 of those, and 28 at most across lanes and waves, 132 in all; the others in FP64)."""
    g = torch.Generator(device=DEV).manual_seed(V)
    x = torch.empty((M, V), dtype=dtype, device=DEV)
    for m in range(M):
        x[m] = (torch.rand(V, generator=g, device=DEV) * 1.4 + 1.3).to(dtype) if m % 2 == 0 else 2.6875 + 0.0625 * (m % 3 - 1)
    x[:, :256 * 32] = 0
    tokens = _ints([V - 1 - m for m in range(M)])
    lp, _, ent, ids, tops = api.token_logprobs(x, tokens, top=1)
    for m in range(M):
        d = x[m].double()
        d = d - d.max()
        e = d.exp()
        lse = float(e.sum().log())
        dist = float((e * -d).sum() / e.sum())
        dT = 2.0 ** -23 + 2.0 ** -24 * (1.1 * dist + 6) + 132 * 2.0 ** -24
        want = float(d[V - 1 - m]) - lse
        assert abs(float(lp[m]) - want) <= dT + 2.0 ** -24 * abs(want), (m, float(lp[m]) - want, dT)
        assert abs(float(tops[m, 0]) + lse) <= dT + 2.0 ** -24 * lse, (m, float(tops[m, 0]) + lse, dT)
        assert abs(float(ent[m]) - (lse + dist)) <= dT * (2 + 2 * (1.45 * dist + 8)) + 2.0 ** -24 * (lse + dist), (m, float(ent[m]) - lse - dist)


def test_logprobs_past_four_gigabytes():
    V = 70001
    x = torch.zeros((32000, V), dtype=torch.float16, device=DEV)            # 4.5 GB: 2.24e9 elements
    rows = [0, 15338, 31999]
    for m in rows:
        x[m] = _logits(1, V, m, torch.float16)[0]
    tokens = torch.full((32000,), 5, dtype=torch.int32, device=DEV)
    got = api.token_logprobs(x, tokens, 4)
    pick = torch.tensor(rows, device=DEV)
    _check_logprobs([t[pick] for t in got], x[pick], [5, 5, 5], 4)
    assert (got[1][1:100] == 6).all() and (got[3][1:100] == torch.arange(4, device=DEV)).all()


def test_logprobs_same_bits_in_graphs_and_on_streams():
    x, y = _logits(7, 32000, 11, torch.float16), _logits(7, 32000, 12, torch.float16)
    tokens, top = _ints([5, 100, 31999, 0, 7, 8, 9]), 20
    ws = _workspace(x, top).fill_(0xFF)
    want = [[t.clone() for t in api.token_logprobs(z, tokens, top, workspace=ws)] for z in (x, y)]
    for _ in range(5):
        assert all(_same(a, b) for a, b in zip(api.token_logprobs(x, tokens, top, workspace=ws), want[0]))
    here = x.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        outs = api.token_logprobs(here, tokens, top, workspace=ws)
    for i in (1, 0, 1, 0):
        here.copy_((x, y)[i])
        for o in outs:
            o.fill_(3)
        graph.replay()
        assert all(_same(a, b) for a, b in zip(outs, want[i]))
        torch.cuda.synchronize()
        api.token_logprobs(y[:3], tokens[:3].contiguous(), 2, workspace=ws)
    streams, spaces, got = [torch.cuda.Stream() for _ in range(2)], [_workspace(x, top) for _ in range(2)], []
    torch.cuda.synchronize()
    for _ in range(20):
        for stream, space in zip(streams, spaces):
            with torch.cuda.stream(stream):
                got.append(api.token_logprobs(x, tokens, top, workspace=space))
    torch.cuda.synchronize()
    assert all(_same(a, b) for g in got for a, b in zip(g, want[0]))
    with pytest.raises(api.QoqError):
        api.token_logprobs(x, tokens, top, workspace=ws[:ws.numel() - 16])
    with pytest.raises(api.QoqError):
        api.token_logprobs(x, tokens, 33)
    with pytest.raises(ValueError):
        api.token_logprobs(x, tokens[:2].contiguous())
    with pytest.raises(ValueError):
        api.token_logprobs(x.t(), tokens)


# ------------------------------------------------------------------------------------------------------------------
# Together
# ------------------------------------------------------------------------------------------------------------------
def test_a_decode_step_of_many_requests():
    """Two layers' worth of a step, as a server runs them: adapters on the fused QKV projection, append, attention over a shared prefix, adapters on the
    output projection, the last projection's log probabilities; eager and as one graph, replayed as the sequences grow."""
    B, H, Hkv, hidden, V, rank, adapters, prefix = 12, 8, 2, 512, 1024, 16, 5, 192
    N = (H + 2 * Hkv) * D
    s = _Batch([(0, 10, prefix)], [prefix + 3 + i for i in range(10)] + [20, 64], Hkv, 131, width=6)
    weights = [api.pack_weights(wl.make_weights(n, k, seed, DEV)) for n, k, seed in ((N, hidden, 1), (hidden, H * D, 2), (V, hidden, 3))]
    la = [(_half(41, adapters, rank, hidden, scale=0.05), _half(42, adapters, N, rank, scale=0.1)), (_half(43, adapters, rank, H * D, scale=0.05), _half(44, adapters, hidden, rank, scale=0.1))]
    scales = torch.tensor([0.5, 1.0, 2.0, 1.5, 0.25], device=DEV)
    row = _ints([b % 6 for b in range(B)])
    angles = api.rope_angles(s.width * PAGE, device=DEV)
    cu, group_cu, pl = _ints(list(range(B + 1))), _ints(s.cu), _ints(s.prefix)
    # every sequence writes its next token into a page of its own: the tables get them now
    pool = torch.cat((s.pool, torch.zeros(B * 2 * Hkv * 8704, dtype=torch.uint8, device=DEV)))
    table = s.table.clone()
    for b in range(B):
        n = -(-s.lens[b] // PAGE)
        table[b, n:n + 2] = _ints([s.pages + 2 * b, s.pages + 2 * b + 1])[:s.width - n]
    lens = _ints(s.lens)
    starts, tokens = lens.clone(), _ints([3 * b for b in range(B)])
    behind = max(api.lora_workspace_bytes(B, N, hidden, rank, adapters), api.lora_workspace_bytes(B, hidden, H * D, rank, adapters),
                 api.token_logprobs_workspace_bytes(B, V, 5), api.kv4_shared_attention_workspace_bytes(B, H, Hkv, s.width, 1))
    ws = api.new_workspace(max(api.gemm_workspace_bytes(B, N, hidden), api.gemm_workspace_bytes(B, hidden, H * D), api.gemm_workspace_bytes(B, V, hidden),
                               api.GEMM_COUNTER_BYTES + behind), DEV)
    scratch = ws[api.GEMM_COUNTER_BYTES:]                                   # one workspace for all: behind the counters for the calls that have none
    x = wl.make_activations(B, hidden, 7, DEV)
    plan = api.lora_plan(row, adapters)

    def step():
        api.lora_plan(row, adapters, out=plan)
        starts.copy_(lens)
        lens.add_(1)
        qkv = api.w4a8_linear(x, weights[0], N, workspace=ws)[0]
        api.lora_add(qkv, x, *la[0], plan, scales=scales, out=qkv, workspace=scratch)
        heads = qkv.view(B, H + 2 * Hkv, D)
        q, _ = api.qk_rope_kv4_append(heads[:, :H], heads[:, H:H + Hkv], heads[:, H + Hkv:], pool, table, cu, starts, angles)
        att = api.kv4_shared_attention_decode(q, pool, table, lens, group_cu, pl, Hkv, workspace=scratch)
        out = api.w4a8_linear(att.view(B, H * D), weights[1], hidden, workspace=ws)[0]
        api.lora_add(out, att.view(B, H * D), *la[1], plan, scales=scales, out=out, workspace=scratch)
        logits = api.w4a8_linear(out, weights[2], V, workspace=ws)[0]
        return (q, att, out, logits, *api.token_logprobs(logits, tokens, 5, workspace=scratch))

    first = [t.clone() for t in step()]
    q, att, out, logits = first[:4]
    _check_logprobs(first[4:], logits, tokens.tolist(), 5)
    base = api.w4a8_linear(att.view(B, H * D), weights[1], hidden)[0]
    _check_lora(out, base, att.view(B, H * D), *la[1], row.tolist(), scales)
    # the prefix is of whole pages, which every member's table names: each sequence by itself reads the same tokens, and both results are within
    # 2^-11 of themselves and 2^-10 of the values' average of the exact one
    alone = api.kv4_paged_attention_decode(q, pool, table, lens, Hkv)
    rows = [int(n) for n in lens.tolist()]
    _, v = api.kv4_paged_gather(pool, table, _ints(np.concatenate(([0], np.cumsum(rows))).tolist()), None, sum(rows), Hkv)
    most = float(v.float().abs().max())
    assert (alone.float() - att.float()).abs().max() <= 2 * (2.0 ** -11 + 2.0 ** -10) * most
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    lens.copy_(_ints(s.lens))
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        kept = step()
    for _ in range(3):
        lens.copy_(_ints(s.lens))
        graph.replay()
        torch.cuda.synchronize()
        assert all(_same(a, b) for a, b in zip(kept, first))
    graph.replay()                                                          # a step further on: another token in every sequence
    torch.cuda.synchronize()
    assert not _same(kept[1], first[1]) and torch.isfinite(kept[1].float()).all()

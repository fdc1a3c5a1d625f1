"""Refusals of the paged calls, on the CPU: nothing here reaches a device."""
import ctypes
import math
import os
import random

import pytest
import torch

from paper_2405_04532_amd import api


@pytest.fixture(scope="module")
def L():
    return api.lib()


@pytest.fixture(scope="module")
def p():
    buf = (ctypes.c_uint8 * 64)()
    test = (ctypes.addressof(buf) + 15) & ~15
    _keep.append(buf)
    return test


_keep = []
OK, NULL, SHAPE, ALIGN, WORKSPACE, ARCH = 0, 1, 2, 3, 5, 6


def _append(L, p, **over):
    a = dict(q=p, qs=512, k=p, ks=256, v=p, vs=256, gq=None, gk=None, eps=1e-6, angles=p, rows=8, rot=128, inter=0, cu=p, starts=p, M=4, B=1,
             H=4, Hkv=2, D=128, pool=p, pages=2, table=p, width=1, qo=p, qos=512, ko=None, kos=0)
    a.update(over)
    return L.qoq_qk_rope_kv4_append(*a.values(), None)


@pytest.mark.parametrize("over,want", [
    (dict(D=64), SHAPE), (dict(rot=8), SHAPE), (dict(rot=144), SHAPE), (dict(rot=-16), SHAPE), (dict(rows=0), SHAPE), (dict(rows=1 << 31), SHAPE),
    (dict(eps=-1.0), SHAPE), (dict(eps=float("nan")), SHAPE), (dict(eps=float("inf")), SHAPE), (dict(qs=504), SHAPE), (dict(qs=516), SHAPE), (dict(ks=248), SHAPE), (dict(vs=128), SHAPE),
    (dict(ks=1 << 23), SHAPE), (dict(pages=0), SHAPE), (dict(pages=1 << 31), SHAPE), (dict(width=0), SHAPE), (dict(width=(1 << 18) + 1), SHAPE),
    (dict(M=-1), SHAPE), (dict(M=(1 << 24) + 1), SHAPE), (dict(B=-1), SHAPE), (dict(B=(1 << 20) + 1), SHAPE), (dict(H=0), SHAPE), (dict(Hkv=0), SHAPE), (dict(Hkv=1025), SHAPE),
    (dict(qos=0), SHAPE), (dict(ko="p", kos=128), SHAPE),
    (dict(M=0, q=None, k=None, v=None, qo=None), OK), (dict(B=0, k=None), OK),
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(cu=None), NULL), (dict(pool=None), NULL), (dict(table=None), NULL), (dict(qo=None), NULL),
    (dict(q=None), NULL), (dict(angles=None), NULL),
    (dict(q="p8"), ALIGN), (dict(k="p8"), ALIGN), (dict(v="p8"), ALIGN), (dict(gq="p8"), ALIGN), (dict(gk="p2"), ALIGN), (dict(angles="p4"), ALIGN),
    (dict(pool="p8"), ALIGN), (dict(qo="p8"), ALIGN), (dict(ko="p8", kos=256), ALIGN), (dict(cu="p2"), ALIGN), (dict(starts="p2"), ALIGN), (dict(table="p2"), ALIGN)])
def test_append_refusals(L, p, over, want):
    put = {"p": p, "p2": p + 2, "p4": p + 4, "p8": p + 8}
    assert _append(L, p, **{k: put.get(v, v) if isinstance(v, str) else v for k, v in over.items()}) == want


def _decode(L, p, **over):
    a = dict(q=p, qs=512, pool=p, pages=2, table=p, width=64, lens=p, B=1, H=4, Hkv=2, D=128, window=0, sinks=0, out=p, ws=None, nbytes=0)
    a.update(over)
    return L.qoq_kv4_paged_attention_decode(*a.values(), None)


@pytest.mark.parametrize("over,want", [
    (dict(D=96), SHAPE), (dict(H=3), SHAPE), (dict(H=34), SHAPE), (dict(H=0), SHAPE), (dict(qs=500), SHAPE), (dict(window=-1), SHAPE), (dict(sinks=-1), SHAPE), (dict(pages=0), SHAPE),
    (dict(width=0), SHAPE), (dict(B=-1), SHAPE), (dict(B=0, q=None), OK), (dict(q=None), NULL), (dict(pool=None), NULL), (dict(table=None), NULL),
    (dict(lens=None), NULL), (dict(out=None), NULL), (dict(q="p8"), ALIGN), (dict(out="p8"), ALIGN), (dict(pool="p8"), ALIGN), (dict(ws="p8"), ALIGN),
    (dict(lens="p2"), ALIGN), (dict(table="p2"), ALIGN), (dict(ws="p", nbytes=1024), WORKSPACE)])
def test_decode_refusals(L, p, over, want):
    put = {"p": p, "p2": p + 2, "p8": p + 8}
    assert _decode(L, p, **{k: put.get(v, v) if isinstance(v, str) else v for k, v in over.items()}) == want


def test_gather_refusals(L, p):
    g = L.qoq_kv4_paged_gather
    assert g(p, 2, p, 1, p, p, 4, 1, 2, 64, p, p, None) == SHAPE
    assert g(p, 0, p, 1, p, p, 4, 1, 2, 128, p, p, None) == SHAPE
    assert g(p, 2, p, 1, p, p, -4, 1, 2, 128, p, p, None) == SHAPE
    assert g(None, 2, None, 1, None, None, 0, 1, 2, 128, None, None, None) == OK
    for hole in range(5):
        a = [p, p, p, p, p]
        a[hole] = None
        assert g(a[0], 2, a[1], 1, a[2], None, 4, 1, 2, 128, a[3], a[4], None) == NULL
    assert g(p, 2, p, 1, p + 2, p, 4, 1, 2, 128, p, p, None) == ALIGN and g(p, 2, p, 1, p, p, 4, 1, 2, 128, p, p + 8, None) == ALIGN
    assert g(p, 2, p, 1, p, p + 2, 4, 1, 2, 128, p, p, None) == ALIGN


def _prefill(L, p, **over):
    a = dict(q=p, qs=512, k=p, ks=256, v=p, vs=256, cu_q=p, cu_k=p, M=4, Mk=8, B=1, H=4, Hkv=2, D=128, window=0, sinks=0, out=p, ws=None, nbytes=0)
    a.update(over)
    return L.qoq_attention_prefill(*a.values(), None)


@pytest.mark.parametrize("over,want", [
    (dict(D=64), SHAPE), (dict(H=5), SHAPE), (dict(H=130), SHAPE), (dict(Hkv=0), SHAPE), (dict(qs=256), SHAPE), (dict(ks=8), SHAPE), (dict(vs=260), SHAPE), (dict(window=-2), SHAPE),
    (dict(sinks=-2), SHAPE), (dict(M=-1), SHAPE), (dict(Mk=-1), SHAPE), (dict(Mk=(1 << 24) + 1), SHAPE), (dict(M=0, q=None), OK), (dict(B=0, q=None), OK),
    (dict(q=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL), (dict(cu_q=None), NULL), (dict(cu_k=None), NULL), (dict(out=None), NULL),
    (dict(q="p8"), ALIGN), (dict(k="p8"), ALIGN), (dict(v="p8"), ALIGN), (dict(out="p8"), ALIGN), (dict(ws="p8"), ALIGN), (dict(cu_q="p2"), ALIGN), (dict(cu_k="p2"), ALIGN)])
def test_prefill_refusals(L, p, over, want):
    put = {"p2": p + 2, "p8": p + 8}
    assert _prefill(L, p, **{k: put.get(v, v) if isinstance(v, str) else v for k, v in over.items()}) == want


def test_sizes(L):
    assert api.kv4_pool_bytes(3, 8) == 3 * 8 * 8704 and api.kv4_pool_bytes(0, 8) == 0 and api.kv4_pool_bytes(3, 8, 64) == 0
    with pytest.raises(api.QoqError):
        api.kv4_new_pool(0, 8, "cpu")
    # one sequence of few heads is shared by workgroups, a full batch is not; what a window leaves decides, not the table
    assert api.kv4_paged_attention_workspace_bytes(1, 32, 8, 128) > api.GEMM_COUNTER_BYTES
    assert api.kv4_paged_attention_workspace_bytes(128, 32, 8, 128) == 0 and api.kv4_paged_attention_workspace_bytes(1, 32, 8, 1) == 0
    assert api.kv4_paged_attention_workspace_bytes(1, 32, 8, 1024, window=64) == 0
    assert api.kv4_paged_attention_workspace_bytes(1, 34, 2, 128) == 0 and api.kv4_paged_attention_workspace_bytes(0, 32, 8, 128) == 0
    for width in (1, 2, 17, 500, 1 << 18):
        assert api.kv4_paged_attention_workspace_bytes(2, 8, 4, width) % 16 == 0


def test_angles():
    t = api.rope_angles(70, rot=64, theta=500000.0)
    assert t.shape == (70, 64) and t.dtype == torch.float32 and bool((t[0, :32] == 1).all()) and bool((t[0, 32:] == 0).all())
    i, pos = torch.arange(32, dtype=torch.float64), 69
    want = pos * 500000.0 ** (-2 * i / 64)
    assert bool(((t[pos, :32] - want.cos()).abs() <= 2 ** -24).all()) and bool(((t[pos, 32:] - want.sin()).abs() <= 2 ** -24).all())


def test_one_workspace_serves_every_shape(L):
    """The bytes of a call are not monotone in its sizes (a larger batch may need none), but bounded: for any shape by what the header and the
    binding state, and there are shapes that need just that."""
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "qoq_w4a8.h")).read()
    most = {"decode": 0, "prompt": 0}
    rng = random.Random(1)
    log = lambda hi: int(2 ** rng.uniform(0, math.log2(hi + 1)))           # noqa: E731
    for _ in range(20000):
        Hkv, window, sinks = log(1024), rng.choice((0, log(1 << 20))), log(100)
        most["decode"] = max(most["decode"], api.kv4_paged_attention_workspace_bytes(log(1 << 20), Hkv * rng.randint(1, 16), Hkv, log(1 << 18), window, sinks))
        most["prompt"] = max(most["prompt"], api.attention_prefill_workspace_bytes(log(1 << 24), log(1 << 24), log(2000), Hkv * rng.randint(1, 64), Hkv, window, sinks))
    full = {"decode": api.kv4_paged_attention_workspace_bytes(128, 32, 2, 1 << 18),
            "prompt": api.attention_prefill_workspace_bytes(12, 14000000, 4, 784, 16, 30000, 1)}
    assert full == {"decode": 4587520, "prompt": api.ATTENTION_WORKSPACE_MAX}
    assert all(most[x] <= full[x] and str(full[x]) in text for x in full)
    # a batch that needs none, and one of its parts that does
    assert api.kv4_paged_attention_workspace_bytes(128, 32, 8, 128) == 0 < api.kv4_paged_attention_workspace_bytes(16, 32, 8, 128)

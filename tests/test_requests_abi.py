"""Refusals of the calls of a decode step of many requests, on the CPU (nothing here reaches a device), and pins of their oracle."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import requests
from paper_2405_04532_amd import api

OK, NULL, SHAPE, ALIGN, WORKSPACE, ARCH = 0, 1, 2, 3, 5, 6
_keep = []


@pytest.fixture(scope="module")
def L():
    return api.lib()


@pytest.fixture(scope="module")
def p():
    buf = (ctypes.c_uint8 * 64)()
    _keep.append(buf)
    return (ctypes.addressof(buf) + 15) & ~15


def _args(defaults, over, p):
    put = {"p": p, "p1": p + 1, "p2": p + 2, "p4": p + 4, "p8": p + 8}
    a = dict(defaults)
    assert set(over) <= set(a)
    a.update({k: put.get(v, v) if isinstance(v, str) else v for k, v in over.items()})
    return a.values()


def _status(call, want):
    if want == ARCH and torch.cuda.is_available():      # nothing is wrong with these but the device, which is none here
        pytest.skip("host pointers: without a device only")
    return call()


@pytest.mark.parametrize("over,want", [
    (dict(D=64), SHAPE), (dict(H=3), SHAPE), (dict(H=34), SHAPE), (dict(H=0), SHAPE), (dict(qs=500), SHAPE), (dict(qs=516), SHAPE), (dict(pages=0), SHAPE),
    (dict(width=0), SHAPE), (dict(B=-1), SHAPE), (dict(groups=-1), SHAPE), (dict(groups=(1 << 20) + 1), SHAPE), (dict(B=0, q=None), OK),
    (dict(q=None), NULL), (dict(pool=None), NULL), (dict(table=None), NULL), (dict(lens=None), NULL), (dict(out=None), NULL), (dict(cu=None), NULL),
    (dict(prefix=None), NULL), (dict(q="p8"), ALIGN), (dict(pool="p8"), ALIGN), (dict(out="p8"), ALIGN), (dict(ws="p8"), ALIGN), (dict(table="p2"), ALIGN),
    (dict(lens="p2"), ALIGN), (dict(cu="p2"), ALIGN), (dict(prefix="p1"), ALIGN), (dict(ws=None), WORKSPACE), (dict(nbytes=1000), WORKSPACE),
    (dict(), ARCH), (dict(cu=None, prefix=None, groups=0), ARCH)])
def test_shared_refusals(L, p, over, want):
    d = dict(q=p, qs=512, pool=p, pages=2, table=p, width=64, lens=p, cu=p, prefix=p, groups=1, B=1, H=4, Hkv=2, D=128, out=p, ws=p, nbytes=1 << 30)
    assert _status(lambda: L.qoq_kv4_shared_attention_decode(*_args(d, over, p), None), want) == want


def test_shared_workspace_bytes():
    size = api.kv4_shared_attention_workspace_bytes
    assert size(0, 4, 2, 8, 1) == 0 and size(4, 5, 2, 8, 1) == 0 and size(4, 34, 2, 8, 1) == 0 and size(4, 4, 2, 8, -1) == 0
    for B, H, Hkv, width, groups in ((1, 4, 4, 1, 0), (64, 32, 8, 80, 1), (500, 64, 8, 300, 7), (3, 16, 1, 4000, 3)):
        n = size(B, H, Hkv, width, groups)
        assert n >= B * H * 132 * 4 and n % 16 == 0
        assert size(B, H, Hkv, width, groups + 1) > 0


@pytest.mark.parametrize("B,H,Hkv,width", [(1, 4, 4, 1), (3, 32, 8, 100), (40, 16, 1, 3000), (5, 64, 8, 300)])
def test_shared_workspace_of_more_groups_than_sequences(B, H, Hkv, width):
    """No more than B groups hold a sequence, so none beyond them takes workgroups, or their parts."""
    assert len({api.kv4_shared_attention_workspace_bytes(B, H, Hkv, width, groups) for groups in (B, B + 1, 20 * B, 1 << 20)}) == 1


@pytest.mark.parametrize("over,want", [
    (dict(M=-1), SHAPE), (dict(M=(1 << 20) + 1), SHAPE), (dict(adapters=0), SHAPE), (dict(adapters=4097), SHAPE), (dict(plan=None), NULL), (dict(rows=None), NULL),
    (dict(rows=None, M=0), ARCH), (dict(plan="p8"), ALIGN), (dict(rows="p2"), ALIGN), (dict(nbytes=64), WORKSPACE), (dict(), ARCH)])
def test_plan_refusals(L, p, over, want):
    d = dict(rows=p, M=4, adapters=3, plan=p, nbytes=1 << 20)
    assert _status(lambda: L.qoq_lora_plan(*_args(d, over, p), None), want) == want


@pytest.mark.parametrize("over,want", [
    (dict(M=-1), SHAPE), (dict(N=0), SHAPE), (dict(N=12), SHAPE), (dict(K=0), SHAPE), (dict(K=20), SHAPE), (dict(rank=0), SHAPE), (dict(rank=12), SHAPE),
    (dict(rank=520), SHAPE), (dict(adapters=0), SHAPE), (dict(adapters=4097), SHAPE), (dict(bs=32), SHAPE), (dict(bs=68), SHAPE), (dict(xs=8), SHAPE), (dict(os=0), SHAPE),
    (dict(os=1 << 25), SHAPE), (dict(out="p", base="p", os=72), SHAPE), (dict(N=(1 << 22) + 8, bs=1 << 23, os=1 << 23), SHAPE),
    (dict(M=0, base=None, x=None, plan=None), OK),
    (dict(base=None), NULL), (dict(x=None), NULL), (dict(a=None), NULL), (dict(b=None), NULL), (dict(plan=None), NULL), (dict(out=None), NULL),
    (dict(base="p8"), ALIGN), (dict(x="p8"), ALIGN), (dict(a="p8"), ALIGN), (dict(b="p8"), ALIGN), (dict(out="p8"), ALIGN), (dict(plan="p8"), ALIGN), (dict(ws="p8"), ALIGN),
    (dict(scales="p2"), ALIGN), (dict(pbytes=64), WORKSPACE), (dict(ws=None), WORKSPACE), (dict(nbytes=64), WORKSPACE), (dict(), ARCH), (dict(scales="p"), ARCH)])
def test_lora_refusals(L, p, over, want):
    d = dict(base=p, bs=64, x=p, xs=16, a=p, b=p, scales=None, plan=p, pbytes=1 << 20, M=4, N=64, K=16, rank=8, adapters=3, out=p, os=64, ws=p, nbytes=1 << 24)
    assert _status(lambda: L.qoq_lora_add(*_args(d, over, p), None), want) == want


def test_lora_bytes(L):
    assert L.qoq_lora_plan_bytes(-1, 4) == 0 and L.qoq_lora_plan_bytes(4, 0) == 0 and L.qoq_lora_plan_bytes(0, 4) > 0
    assert api.lora_workspace_bytes(0, 64, 16, 8, 3) >= 0 and api.lora_workspace_bytes(4, 64, 20, 8, 3) == 0 and api.lora_workspace_bytes(4, 64, 16, 8, 3) >= 4 * 8 * 4


@pytest.mark.parametrize("over,want", [
    (dict(dtype=2), SHAPE), (dict(V=0), SHAPE), (dict(V=(1 << 24) + 1, stride=1 << 25), SHAPE), (dict(M=-1), SHAPE), (dict(stride=99), SHAPE), (dict(top=-1), SHAPE),
    (dict(top=33), SHAPE), (dict(V=4, top=5), SHAPE), (dict(M=0, x=None), OK),
    (dict(x=None), NULL), (dict(tokens=None), NULL), (dict(ids=None), NULL), (dict(tops=None), NULL),
    (dict(x="p1"), ALIGN), (dict(dtype=1, x="p2"), ALIGN), (dict(ws="p8"), ALIGN), (dict(tokens="p2"), ALIGN), (dict(lp="p2"), ALIGN), (dict(rank="p1"), ALIGN),
    (dict(ent="p2"), ALIGN), (dict(ids="p2"), ALIGN), (dict(tops="p1"), ALIGN), (dict(V=100000, stride=100000, ws="p", nbytes=100), WORKSPACE),
    (dict(), ARCH), (dict(x="p2"), ARCH), (dict(tokens=None, lp=None, rank=None), ARCH), (dict(top=0, ids=None, tops=None, ent=None), ARCH)])
def test_logprobs_refusals(L, p, over, want):
    d = dict(x=p, dtype=0, stride=100, tokens=p, M=3, V=100, top=5, lp=p, rank=p, ent=p, ids=p, tops=p, ws=None, nbytes=0)
    assert _status(lambda: L.qoq_token_logprobs(*_args(d, over, p), None), want) == want


def test_logprobs_workspace_bytes():
    assert api.token_logprobs_workspace_bytes(0, 32000, 5) == 0
    assert api.token_logprobs_workspace_bytes(100000, 32000, 5) == 0                     # a workgroup to a row
    assert api.token_logprobs_workspace_bytes(1, 100, 5) == 0
    assert api.token_logprobs_workspace_bytes(1, 32000, 5) >= 2 * (16 + 5 * 8)
    assert api.token_logprobs_workspace_bytes(1, 32000, 33) == 0                         # refused by the call


def test_the_binding_refuses_tensors_of_the_cpu():
    x = torch.zeros((2, 64), dtype=torch.float16)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError):
        api.token_logprobs(x, i)
    with pytest.raises(TypeError):
        api.lora_plan(i, 3)
    with pytest.raises(TypeError):
        api.lora_add(x, x, x, x, i)
    with pytest.raises(TypeError):
        api.kv4_shared_attention_decode(x.view(1, 1, 128), i, i, i, i, i, 1)


# ------------------------------------------------------------------------------------------------------------------
# Pins of the oracle
# ------------------------------------------------------------------------------------------------------------------
def test_oracle_logprobs_by_hand():
    lp, rank, ent, ids, tops, _ = requests.logprobs(np.log([4.0, 1.0, 2.0, 1.0]), 3, 4)
    assert np.isclose(lp, np.log(0.125)) and rank == 4 and list(ids) == [0, 2, 1, 3]
    assert np.isclose(ent, 0.5 * np.log(2) + 0.25 * np.log(4) + 0.25 * np.log(8)) and np.allclose(np.exp(tops), [0.5, 0.25, 0.125, 0.125])
    lp, rank, ent, ids, tops, _ = requests.logprobs([-np.inf, 0.0, -np.inf], 2, 3)
    assert lp == -np.inf and rank == 3 and ent == 0.0 and list(ids) == [1, 0, 2] and tops[0] == 0.0
    for bad in ([np.nan, 1.0], [np.inf, 0.0], [-np.inf, -np.inf]):
        lp, rank, ent, ids, tops, _ = requests.logprobs(bad, 0, 1)
        assert np.isnan(lp) and rank == 0 and np.isnan(ent) and ids[0] == -1 and np.isnan(tops[0])


def test_oracle_lora_by_hand():
    base, x = np.ones((3, 2)), np.array([[1.0, 2.0], [3.0, 4.0], [5.0, 6.0]])
    a, b = np.array([[[1.0, 0.0]], [[0.0, 1.0]]]), np.array([[[1.0], [2.0]], [[3.0], [4.0]]])
    out, off = requests.lora(base, x, a, b, [1, -1, 0], [0.5, 2.0])
    assert np.array_equal(out, [[1 + 2 * 2 * 3, 1 + 2 * 2 * 4], [1, 1], [1 + 0.5 * 5, 1 + 0.5 * 5 * 2]]) and (off < 1e-4).all()


def test_oracle_shared_attention_is_attention_of_the_concatenation():
    g = np.random.default_rng(1)
    k, v, q = g.normal(size=(2, 9, 1, 4)), g.normal(size=(2, 9, 1, 4)), g.normal(size=(2, 2, 4))
    got = requests.shared_attention(q, lambda b, t: (k[b, t], v[b, t]), [9, 7], [0, 2], [5])
    for b, L in enumerate((9, 7)):
        kk, vv = np.concatenate((k[0, :5], k[b, 5:L])), np.concatenate((v[0, :5], v[b, 5:L]))
        s = np.einsum("td,hd->ht", kk[:, 0], q[b]) / 2.0
        w = np.exp(s) / np.exp(s).sum(1, keepdims=True)
        assert np.allclose(got[b][0], w @ vv[:, 0])

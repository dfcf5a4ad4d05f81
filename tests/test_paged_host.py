"""CPU-side checks of the paged KV4 calls and the adapters: sizes, refusals before any launch, the block layout of the tests."""
import ctypes
import os

import numpy as np
import pytest
import torch

import paged_ref as ref
import paper_2606_02823_b200 as qift
from paper_2606_02823_b200 import binding


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2606_02823_b200 import build
        build.build()
    return qift.lib()


def test_every_nibble_of_a_block_has_one_owner():
    places = np.concatenate([(ref.KB * 2 + ref.KSH // 4).ravel(), (ref.VB * 2 + ref.VSH // 4).ravel()])
    assert np.array_equal(np.sort(places), np.arange(2 * 4096))
    owned = np.concatenate([ref.token_bytes(t) for t in range(ref.TOKENS)])
    assert all(ref.token_bytes(t).size == 138 for t in range(ref.TOKENS)) and np.array_equal(np.sort(owned), np.arange(ref.BLOCK))


def test_sizes(L):
    assert qift.qift_kv4_page_bytes(64, 8) == 8 * 64 * 138
    assert qift.qift_kv4_page_bytes(32, 1) == ref.BLOCK
    for page, H, D in ((48, 8, 128), (16, 8, 128), (0, 8, 128), (2048, 8, 128), (64, 0, 128), (64, 8, 64)):
        assert qift.qift_kv4_page_bytes(page, H, D) == 0
    assert qift.qift_kv4_paged_attention_workspace_bytes(0, 1, 8, 8) == 0
    assert qift.qift_kv4_paged_attention_workspace_bytes(4, 1, 9, 8) == 0
    assert qift.qift_kv4_paged_attention_workspace_bytes(4, 1, 32, 8) > 0
    assert qift.qift_lora_workspace_bytes(0, 16, 64) == 0 and qift.qift_lora_workspace_bytes(5, 16, 64) > 0


P, ODD, NULL = 4096, 4100, None      # addresses that are never dereferenced: the calls fail validation first


def write(L, K=P, V=P, dt=0, ks=1024, vs=1024, total=4, H=8, D=128, kh=0, vh=0, clip=0.95, rs=P, first=P, R=2, table=P, mp=3, pool=P, np_=5, page=64):
    return L.qift_kv4_paged_write(K, V, dt, ks, vs, total, H, D, kh, vh, clip, rs, first, R, table, mp, pool, np_, page, None)


def read(L, K=P, V=P, dt=0, ks=1024, vs=1024, total=4, H=8, D=128, kh=0, vh=0, rs=P, first=P, R=2, table=P, mp=3, pool=P, np_=5, page=64):
    return L.qift_kv4_paged_read(K, V, dt, ks, vs, total, H, D, kh, vh, rs, first, R, table, mp, pool, np_, page, None)


def keep(L, keep=P, kept=P, total=4, H=8, D=128, rs=P, first=P, R=2, table=P, mp=3, pool=P, np_=5, page=64):
    return L.qift_kv4_paged_keep(keep, kept, total, H, D, rs, first, R, table, mp, pool, np_, page, None)


def attend(L, q=P, dt=0, qs=4096, total=4, Hq=32, H=8, D=128, qh=0, scale=0.0, mask=P, words=2, rs=P, first=P, R=2, table=P, mp=3, pool=P, np_=5,
           page=64, out=P, ws=P, wsb=1 << 40):
    return L.qift_kv4_paged_attention(q, dt, qs, total, Hq, H, D, qh, scale, mask, words, rs, first, R, table, mp, pool, np_, page, out, ws, wsb, None)


def lora(L, x=P, dt=0, A=P, B=P, sc=P, n=3, rank=16, M=4, N=64, K=64, rs=P, ad=P, R=2, y=P, out=P, ws=P, wsb=1 << 40):
    return L.qift_lora_linear(x, dt, A, B, sc, n, rank, M, N, K, rs, ad, R, y, out, ws, wsb, None)


BAD_ARG, BAD_SHAPE, BAD_ALIGN = qift.ERR_INVALID_ARG, qift.ERR_UNSUPPORTED_SHAPE, qift.ERR_ALIGNMENT


@pytest.mark.parametrize("call", [write, read, keep, attend])
@pytest.mark.parametrize("bad,status", [
    (dict(rs=NULL), BAD_ARG), (dict(first=NULL), BAD_ARG), (dict(table=NULL), BAD_ARG), (dict(pool=NULL), BAD_ARG), (dict(total=0), BAD_ARG),
    (dict(H=0), BAD_ARG), (dict(R=0), BAD_ARG), (dict(mp=0), BAD_ARG), (dict(np_=-1), BAD_ARG), (dict(D=64), BAD_SHAPE), (dict(page=48), BAD_SHAPE),
    (dict(page=2048), BAD_SHAPE), (dict(pool=ODD), BAD_ALIGN), (dict(rs=4098), BAD_ALIGN), (dict(first=4097), BAD_ALIGN), (dict(table=4098), BAD_ALIGN)])
def test_paged_calls_refuse(L, call, bad, status):
    assert call(L, **bad) == status


@pytest.mark.parametrize("call,bad,status", [
    (write, dict(K=NULL), BAD_ARG), (write, dict(V=NULL), BAD_ARG), (write, dict(dt=2), BAD_ARG), (write, dict(clip=0.0), BAD_ARG),
    (write, dict(clip=float("nan")), BAD_ARG), (write, dict(kh=96), BAD_SHAPE), (write, dict(vh=256), BAD_SHAPE), (write, dict(kh=-2), BAD_SHAPE),
    (write, dict(ks=1020), BAD_SHAPE), (write, dict(vs=1026), BAD_SHAPE), (write, dict(dt=1, ks=1028), BAD_SHAPE), (write, dict(K=ODD), BAD_ALIGN),
    (read, dict(K=NULL, V=NULL), BAD_ARG), (read, dict(dt=7), BAD_ARG), (read, dict(kh=3), BAD_SHAPE), (read, dict(vs=512), BAD_SHAPE),
    (read, dict(V=ODD), BAD_ALIGN),
    (keep, dict(keep=NULL), BAD_ARG), (keep, dict(kept=NULL), BAD_ARG), (keep, dict(keep=4098), BAD_ALIGN),
    (attend, dict(q=NULL), BAD_ARG), (attend, dict(out=NULL), BAD_ARG), (attend, dict(dt=3), BAD_ARG), (attend, dict(Hq=0), BAD_ARG),
    (attend, dict(words=0), BAD_ARG), (attend, dict(words=33), BAD_ARG), (attend, dict(scale=-1.0), BAD_ARG),
    (attend, dict(scale=float("nan")), BAD_ARG), (attend, dict(scale=float("inf")), BAD_ARG), (attend, dict(Hq=12, qs=4096), BAD_SHAPE),
    (attend, dict(Hq=520, qs=1 << 20), BAD_SHAPE), (attend, dict(qh=48), BAD_SHAPE), (attend, dict(qs=4000), BAD_SHAPE),
    (attend, dict(q=ODD), BAD_ALIGN), (attend, dict(mask=4098), BAD_ALIGN), (attend, dict(ws=ODD), BAD_ALIGN),
    (attend, dict(ws=NULL), qift.ERR_WORKSPACE), (attend, dict(wsb=8), qift.ERR_WORKSPACE),
    (lora, dict(x=NULL), BAD_ARG), (lora, dict(A=NULL), BAD_ARG), (lora, dict(B=NULL), BAD_ARG), (lora, dict(sc=NULL), BAD_ARG),
    (lora, dict(rs=NULL), BAD_ARG), (lora, dict(ad=NULL), BAD_ARG), (lora, dict(out=NULL), BAD_ARG), (lora, dict(n=0), BAD_ARG),
    (lora, dict(rank=0), BAD_ARG), (lora, dict(M=0), BAD_ARG), (lora, dict(N=-8), BAD_ARG), (lora, dict(K=0), BAD_ARG), (lora, dict(R=0), BAD_ARG),
    (lora, dict(dt=2), BAD_ARG), (lora, dict(rank=12), BAD_SHAPE), (lora, dict(rank=136), BAD_SHAPE), (lora, dict(K=60), BAD_SHAPE),
    (lora, dict(N=60), BAD_SHAPE), (lora, dict(x=ODD), BAD_ALIGN), (lora, dict(y=ODD), BAD_ALIGN), (lora, dict(rs=4098), BAD_ALIGN),
    (lora, dict(ws=NULL), qift.ERR_WORKSPACE), (lora, dict(wsb=15), qift.ERR_WORKSPACE)])
def test_calls_refuse(L, call, bad, status):
    assert call(L, **bad) == status


def test_binding_checks_its_tensors():
    with pytest.raises(AssertionError):
        qift.Kv4Pages(torch.zeros((2, 8, 8832), dtype=torch.uint8), torch.zeros((1, 2), dtype=torch.int32), 64)   # not on a GPU

"""CPU-side checks of the page-table calls, the norms and rotation, and the gated calls: what they refuse before any launch."""
import ctypes
import os

import pytest

import paper_2606_02823_b200 as qift
from paper_2606_02823_b200 import binding


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2606_02823_b200 import build
        build.build()
    return qift.lib()


P, ODD, NULL = 4096, 4098, None      # addresses that are never dereferenced: the calls fail validation first
ARG, SHAPE, ALIGN, SPACE = qift.ERR_INVALID_ARG, qift.ERR_UNSUPPORTED_SHAPE, qift.ERR_ALIGNMENT, qift.ERR_WORKSPACE


def begin(L, rows=P, first=P, R=2, table=P, most=3, pages=5, page=64, free=P, count=P, mask=P, words=2, total=4, start=P, position=P, slot=P, lost=P):
    return L.qift_kv4_pages_begin(rows, first, R, table, most, pages, page, free, count, mask, words, total, start, position, slot, lost, None)


def end(L, length=P, shared=P, R=2, table=P, most=3, pages=5, page=64, free=P, count=P):
    return L.qift_kv4_pages_end(length, shared, R, table, most, pages, page, free, count, None)


def rope(L, q=P, k=P, dt=0, qs=4096, ks=1024, total=4, Hq=32, H=8, D=128, wq=P, wk=P, eps=1e-6, inv=P, rot=128, pairs=0, pos=P, qo=P, ko=P, qos=4096, kos=1024):
    return L.qift_qk_norm_rope(q, k, dt, qs, ks, total, Hq, H, D, wq, wk, eps, inv, rot, pairs, pos, qo, ko, qos, kos, None)


def outputs(N=64, N2=64, packed=P, s_n=P, acc=None):
    return (binding.LinearOutput * 2)(binding.LinearOutput(packed, s_n, None, acc, N, 0), binding.LinearOutput(packed, s_n, None, acc, N2, 0))


def linear(L, q=P, s=P, M=4, K=256, levels=0, act=0, H=P, dt=0, buf=P, buf_bytes=1 << 40, ready=0, ahead=None, pair=None, **kw):
    pair = pair or outputs(**kw)
    return L.qift_gated_linear(q, s, M, K, levels, ctypes.addressof(pair), act, H, dt, buf, buf_bytes, ready, ahead, None)


def forward(L, x=P, xdt=0, M=4, K=256, had=256, clip=0.9, levels=0, act=0, H=P, dt=0, ws=P, wsb=1 << 40, buf=P, buf_bytes=1 << 40, pair=None, **kw):
    pair = pair or outputs(**kw)
    return L.qift_gated_forward(x, xdt, M, K, had, clip, levels, ctypes.addressof(pair), act, H, dt, ws, wsb, buf, buf_bytes, 0, None, None)


@pytest.mark.parametrize("bad, status", [(dict(rows=NULL), ARG), (dict(first=NULL), ARG), (dict(table=NULL), ARG), (dict(free=NULL), ARG), (dict(count=NULL), ARG),
                                        (dict(start=NULL), ARG), (dict(position=NULL), ARG), (dict(lost=NULL), ARG), (dict(R=0), ARG), (dict(most=0), ARG),
                                        (dict(pages=0), ARG), (dict(total=0), ARG), (dict(total=-1), ARG), (dict(page=48), SHAPE), (dict(page=0), SHAPE),
                                        (dict(page=2048), SHAPE), (dict(words=0), SHAPE), (dict(words=33), SHAPE), (dict(R=1 << 16, most=1 << 15), SHAPE),
                                        (dict(rows=ODD), ALIGN), (dict(first=ODD), ALIGN), (dict(table=ODD), ALIGN), (dict(free=ODD), ALIGN), (dict(count=ODD), ALIGN),
                                        (dict(mask=ODD), ALIGN), (dict(start=ODD), ALIGN), (dict(position=ODD), ALIGN), (dict(slot=4100), ALIGN), (dict(lost=ODD), ALIGN)])
def test_begin_refuses(L, bad, status):
    assert begin(L, **bad) == status


@pytest.mark.parametrize("bad, status", [(dict(length=NULL), ARG), (dict(table=NULL), ARG), (dict(free=NULL), ARG), (dict(count=NULL), ARG), (dict(R=0), ARG),
                                        (dict(most=-1), ARG), (dict(pages=0), ARG), (dict(page=33), SHAPE), (dict(R=1 << 16, most=1 << 15), SHAPE),
                                        (dict(length=ODD), ALIGN), (dict(shared=ODD), ALIGN), (dict(table=ODD), ALIGN), (dict(free=ODD), ALIGN), (dict(count=ODD), ALIGN)])
def test_end_refuses(L, bad, status):
    assert end(L, **bad) == status


@pytest.mark.parametrize("bad, status", [(dict(q=NULL), ARG), (dict(k=NULL), ARG), (dict(qo=NULL), ARG), (dict(ko=NULL), ARG), (dict(inv=NULL), ARG), (dict(pos=NULL), ARG),
                                        (dict(total=0), ARG), (dict(Hq=0), ARG), (dict(H=0), ARG), (dict(D=0), ARG), (dict(rot=0), ARG), (dict(dt=2), ARG),
                                        (dict(eps=0.0), ARG), (dict(eps=-1.0), ARG), (dict(eps=float("nan")), ARG), (dict(eps=float("inf")), ARG), (dict(pairs=2), ARG),
                                        (dict(D=120), SHAPE), (dict(D=528), SHAPE), (dict(rot=144), SHAPE), (dict(rot=24), SHAPE), (dict(Hq=65535, H=1), SHAPE),
                                        (dict(qs=4095), SHAPE), (dict(qs=4098), SHAPE), (dict(ks=1020), SHAPE), (dict(qos=4092), SHAPE), (dict(kos=1026), SHAPE),
                                        (dict(dt=1, qs=4100), SHAPE), (dict(q=ODD), ALIGN), (dict(k=4104), ALIGN), (dict(wq=4104), ALIGN), (dict(wk=ODD), ALIGN),
                                        (dict(qo=ODD), ALIGN), (dict(ko=ODD), ALIGN), (dict(inv=ODD), ALIGN), (dict(pos=ODD), ALIGN)])
def test_rope_refuses(L, bad, status):
    assert rope(L, **bad) == status


@pytest.mark.parametrize("bad, status", [(dict(q=NULL), ARG), (dict(s=NULL), ARG), (dict(H=NULL), ARG), (dict(M=0), ARG), (dict(K=0), ARG), (dict(levels=5), ARG),
                                        (dict(act=2), ARG), (dict(act=-1), ARG), (dict(dt=2), ARG), (dict(N=0), ARG), (dict(N2=65), ARG), (dict(packed=NULL), ARG),
                                        (dict(s_n=NULL), ARG), (dict(K=24), SHAPE), (dict(K=48, levels=qift.INT3), SHAPE), (dict(K=12, levels=qift.INT4), SHAPE),
                                        (dict(q=ODD), ALIGN), (dict(s=ODD), ALIGN), (dict(H=ODD), ALIGN), (dict(packed=4104), ALIGN), (dict(s_n=ODD), ALIGN),
                                        (dict(acc=ODD), ALIGN), (dict(M=5000, buf=NULL), SPACE), (dict(M=5000, buf_bytes=2 * 64 * 256 - 1), SPACE),
                                        (dict(M=5000, buf=4224), ALIGN)])
def test_gated_linear_refuses(L, bad, status):
    assert linear(L, **bad) == status


@pytest.mark.parametrize("bad, status", [(dict(x=NULL), ARG), (dict(xdt=2), ARG), (dict(clip=0.0), ARG), (dict(clip=1.5), ARG), (dict(act=9), ARG), (dict(had=512), SHAPE),
                                        (dict(had=3), SHAPE), (dict(x=ODD), ALIGN), (dict(ws=NULL), SPACE), (dict(wsb=2047), SPACE), (dict(ws=4224), ALIGN),
                                        (dict(M=5000, buf=NULL), SPACE)])
def test_gated_forward_refuses(L, bad, status):
    assert forward(L, **bad) == status


def test_sizes(L):
    assert L.qift_gated_forward_scratch_bytes(4, 256) == 2048 and L.qift_gated_forward_scratch_bytes(0, 256) == 0
    assert 129 <= qift.qift_gated_levels_min_rows() <= 4096
    ahead = binding.DecodeAhead(ctypes.addressof(outputs()), 2, 256, 0, 0, None, 0, None)
    assert linear(L, ahead=ctypes.addressof(ahead)) == ARG


def test_more_requests_than_their_numbers_have_room_for(L):
    assert begin(L, R=(1 << 30) + 1, most=1) == SHAPE and end(L, R=(1 << 30) + 1, most=1) == SHAPE


@pytest.mark.parametrize("bad, status", [(dict(buf=NULL), SPACE), (dict(buf_bytes=2 * 64 * 256 - 1), SPACE), (dict(buf=4224), ALIGN)])
def test_levels_that_are_there_have_to_be_given(L, bad, status):
    assert linear(L, M=1000, ready=1, **bad) == status

"""What the self-test of the gated kernels' waits refuses before any launch (CPU)."""
import ctypes

import pytest

import paper_2606_02823_b200 as qift
from test_step_host import ALIGN, ARG, NULL, ODD, P, SHAPE, SPACE, L, outputs  # noqa: F401  (L: the fixture)


def probe(L, kernel=1, warp=4, waits=0, limit=1000, q=P, s=P, M=4, K=256, H=P, pair=None, **kw):
    pair = pair or outputs(**kw)
    return L.qift_selftest_gated_wait(kernel, warp, waits, limit, q, s, M, K, ctypes.addressof(pair), H, None)


@pytest.mark.parametrize("bad, status", [(dict(q=NULL), ARG), (dict(s=NULL), ARG), (dict(H=NULL), ARG), (dict(kernel=2), ARG), (dict(kernel=-1), ARG), (dict(warp=-1), ARG),
                                        (dict(warp=20), ARG), (dict(kernel=0, warp=16), ARG), (dict(waits=-1), ARG), (dict(limit=0), ARG),
                                        (dict(limit=1_000_001), ARG), (dict(M=0), ARG), (dict(N2=65), ARG), (dict(K=24), SHAPE), (dict(K=1 << 21), SHAPE),
                                        (dict(kernel=0, M=9), SHAPE), (dict(kernel=0, K=1 << 20), SHAPE), (dict(M=5000), SPACE), (dict(q=ODD), ALIGN),
                                        (dict(s=ODD), ALIGN), (dict(H=ODD), ALIGN), (dict(packed=4104), ALIGN)])
def test_refused(L, bad, status):  # noqa: F811
    assert probe(L, **bad) == status


def pairs(L, limit=1000, q=P, s=P, M=500, K=256, H=P, buf=P, bufb=1 << 40, pair=None, **kw):  # noqa: F811
    pair = pair or outputs(**kw)
    return L.qift_selftest_gated_pairs_wait(limit, q, s, M, K, ctypes.addressof(pair), H, buf, bufb, None)


@pytest.mark.parametrize("bad, status", [(dict(q=NULL), ARG), (dict(s=NULL), ARG), (dict(H=NULL), ARG), (dict(limit=0), ARG), (dict(limit=1_000_001), ARG), (dict(N2=65), ARG),
                                        (dict(M=448), SHAPE), (dict(K=24), SHAPE), (dict(buf=NULL), SPACE), (dict(bufb=2 * 64 * 256 - 1), SPACE),
                                        (dict(buf=4224), ALIGN), (dict(q=ODD), ALIGN), (dict(s=ODD), ALIGN), (dict(H=ODD), ALIGN)])
def test_pairs_refused(L, bad, status):  # noqa: F811
    assert pairs(L, **bad) == status

"""Gated kernels in which a wait runs out: what they store is right, the rest stays as it was, the host learns of it, and the next call is an ordinary one."""
import time

import pytest
import torch

import paper_2606_02823_b200 as qift
from gated_ref import Case

pytestmark = pytest.mark.gpu
OLD = 12345.5
FEW, TC = 0, 1
_made = {}


def made(M, N, K):
    """The case of a size, and its result by an ordinary call."""
    if (M, N, K) not in _made:
        c = Case(M + N, M, N, K, "mnz")
        _made[M, N, K] = c, qift.qift_gated_linear(c.q, c.s, *c.weights, c.lv)
    return _made[M, N, K]


def probe(kernel, warp, waits, M, N, K):
    """-> which results were stored, [M, N]; all of them are right.  The status and the time, too."""
    c, want = made(M, N, K)
    assert qift.qift_device_status() == (qift.OK, 0)
    out = torch.full((M, N), OLD, device="cuda")
    t0 = time.perf_counter()
    qift.qift_selftest_gated_wait(kernel, warp, waits, 1000, c.q, c.s, *c.weights, out)
    rc, detail = qift.qift_device_status()
    assert time.perf_counter() - t0 < 1.0, "waits of 1 ms"
    stored = out != OLD
    assert torch.equal(out[stored], want[stored])
    assert rc == qift.OK or (rc == qift.ERR_TIMEOUT and detail & 0xff in ({81} if kernel == FEW else set(range(82, 90)))), (rc, hex(detail))
    assert (rc == qift.OK) == bool(stored.all())
    assert qift.qift_device_status() == (qift.OK, 0)
    return stored


def ordinary(M, N, K):
    c, want = made(M, N, K)
    assert torch.equal(qift.qift_gated_linear(c.q, c.s, *c.weights, c.lv), want)
    c.check(want)


@pytest.mark.parametrize("warp", [0, 1, 2, 4, 9, 14, 19])
@pytest.mark.parametrize("waits", [0, 1, 2, 3, 5])
def test_nothing_of_an_item_without_its_operands(warp, waits):
    """Two to three items for every CTA, of more steps than there are stages: the one warp has not done its share of the first item, so nobody has sums."""
    size = 200, 19200, 1536
    stored = probe(TC, warp, waits, *size)
    assert not stored.any()
    ordinary(*size)


def test_a_warp_that_never_waits():
    size = 200, 19200, 1536
    assert probe(TC, 3, 0, *size).all()
    assert probe(TC, 9, 1 << 20, *size).all()


@pytest.mark.parametrize("K", [256, 1024, 2048])
@pytest.mark.parametrize("warp, waits", [(0, 0), (1, 0), (1, 1), (2, 0), (4, 0), (4, 1), (9, 0), (17, 0), (19, 1)])
def test_calls_that_fit_the_stages(warp, waits, K):
    """All copies of a CTA are asked for at once, so the warp that asks for them has no wait that could run out: they arrive before the CTA ends all
    the same, and calls right behind it have their shared memory to themselves."""
    size = 48, 1300, K
    c, want = made(*size)
    if K == 256 and warp in (17, 19):
        K = 512                                                      # (a single step leaves warps of the odd ones without waits)
        c, want = made(48, 1300, K)
    outs = [torch.full((48, 1300), OLD, device="cuda") for _ in range(4)]
    for out in outs[:2]:
        qift.qift_selftest_gated_wait(TC, warp, waits, 1000, c.q, c.s, *c.weights, out)
        qift.qift_gated_linear(c.q, c.s, *c.weights, c.lv, out=outs[2])
    rc, detail = qift.qift_device_status()
    assert rc == qift.ERR_TIMEOUT and 82 <= (detail & 0xff) <= 89, (rc, hex(detail))
    assert (outs[0] == OLD).all() and (outs[1] == OLD).all() and torch.equal(outs[2], want)
    ordinary(48, 1300, K)


@pytest.mark.parametrize("warp, waits", [(1, 13), (2, 26), (4, 8), (9, 12), (17, 12), (0, 11)])
def test_later_items(warp, waits):
    """The warp stops in a later item of its CTA: those before are there, and right."""
    size = 200, 19200, 1536
    stored = probe(TC, warp, waits, *size)
    items = 300
    whole = [bool(stored[r0:min(r0 + 112, 200), n0:n0 + 128].all()) for n0 in range(0, 19200, 128) for r0 in (0, 112)]
    some = [bool(stored[r0:min(r0 + 112, 200), n0:n0 + 128].any()) for n0 in range(0, 19200, 128) for r0 in (0, 112)]
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert len(whole) == items and whole == some and all(whole[:sms]) and not all(whole)
    ordinary(*size)


@pytest.mark.parametrize("warp", [0, 1, 6, 15])
@pytest.mark.parametrize("waits", [0, 1, 3, 1 << 20])
def test_few_rows(warp, waits):
    """Two or three tiles for every pair of warps, two waits each: the tiles whose sums one of the pair has not finished stay as they were."""
    M, N, K = 5, 38400, 1536
    stored = probe(FEW, warp, waits, M, N, K).view(M, N // 16, 16).any(2).any(0).cpu()
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    tiles = torch.arange(N // 16)
    mine = tiles[(tiles // sms) % 8 == warp // 2]
    done = mine // (8 * sms) < waits // 2
    assert not stored[mine[~done]].any()                             # (of other pairs' tiles those before they learned of it)
    assert waits < 1 << 20 or stored.all()
    ordinary(M, N, K)


@pytest.mark.parametrize("limit", [1, 3, 20, 1_000_000])
@pytest.mark.parametrize("M, N, K", [(450, 264, 512), (600, 9000, 4096), (2100, 3000, 1040)])
def test_pairs_of_ctas(M, N, K, limit):
    """Products on decoded levels whose waits are shorter than a copy, or than a call: what is stored is right, and calls right behind it are ordinary ones."""
    c, _ = made(M, N, K)
    buf = torch.zeros(qift.qift_levels_bytes(K, c.weights), dtype=torch.uint8, device="cuda")
    qift.qift_gated_linear(c.q[:1].clone(), c.s[:1].clone(), *c.weights, c.lv, ahead=(c.weights, K, c.lv, buf))
    want = qift.qift_gated_linear(c.q, c.s, *c.weights, c.lv, levels_buf=buf, levels_ready=True)
    c.check(want)
    out, behind = (torch.full((M, N), OLD, device="cuda") for _ in range(2))
    for _ in range(2):
        qift.qift_selftest_gated_pairs_wait(limit, c.q, c.s, *c.weights, buf, out)
        qift.qift_gated_linear(c.q, c.s, *c.weights, c.lv, levels_buf=buf, levels_ready=True, out=behind)
    rc, detail = qift.qift_device_status()
    stored = out != OLD
    assert torch.equal(out[stored], want[stored]) and torch.equal(behind, want)
    assert rc == qift.OK and stored.all() or rc == qift.ERR_TIMEOUT and limit < 1_000_000 and 30 <= (detail & 0xff) <= 35, (rc, hex(detail))
    assert qift.qift_device_status() == (qift.OK, 0)

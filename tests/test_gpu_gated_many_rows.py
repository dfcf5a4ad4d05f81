"""The gated calls on decoded levels, from as many rows on as they decode the codes for: from X, captured, with gates of any size; and, on every route,
weights that change between calls and calls on two streams at once."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_02823_b200 as qift
from gated_ref import Case

pytestmark = pytest.mark.gpu
ACTS = [qift.ACT_SILU, qift.ACT_GELU_TANH]


def many(more=0):
    return qift.qift_gated_levels_min_rows() + more


def run(c, act=qift.ACT_SILU, **kw):
    return qift.qift_gated_linear(c.q, c.s, *c.weights, c.lv, activation=act, **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("levels, N, K, had", [("mnz", 130, 1024, 1024), ("int4", 264, 1040, 16), ("int3", 97, 544, 32), ("pot", 200, 512, 256)])
def test_from_activations(levels, N, K, had, dtype):
    M = many(N % 7)
    c = Case(K, M, N, K, levels)
    x = torch.from_numpy(np.random.default_rng(N).standard_normal((M, K)).astype(np.float32)).cuda().to(dtype)
    q, s = oracle.quantize_act(x.float().cpu().numpy(), had, 0.9)
    c.q, c.s = torch.from_numpy(q).cuda(), torch.from_numpy(s).cuda()
    h, *accs = qift.qift_gated_forward(x, had, *c.weights, c.lv, 0.9, want_acc=True)
    c.check(h, accs)
    scratch = torch.empty(qift.lib().qift_gated_forward_scratch_bytes(M, K), dtype=torch.uint8, device="cuda")
    buf = torch.empty(qift.qift_levels_bytes(K, c.weights), dtype=torch.uint8, device="cuda")
    for _ in range(2):                                               # the second time the levels are there
        b = qift.qift_gated_forward(x, had, *c.weights, c.lv, 0.9, out_dtype=torch.bfloat16, scratch=scratch, levels_buf=buf, levels_ready=bool(_))
        assert torch.equal(b, h.to(torch.bfloat16))


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("N", [400, 393])
def test_large_and_small_gates(N, act):
    c = Case(3, many(), N, 512, "int4", extreme=True)
    c.s[0], c.s[-1] = 40.0, 0.0
    h = run(c, act)
    assert torch.isfinite(h).all()
    c.check(h, act=act)
    assert (h[-1] == 0).all()


@pytest.mark.parametrize("levels", ["mnz", "int3"])
@pytest.mark.parametrize("rows", [1, 12, 50, 400, "many"])
def test_captured_with_other_weights(rows, levels):
    """A graph decodes anew: activations and packed weights change between replays, and what the buffer of levels held is gone."""
    M = many(5) if rows == "many" else rows
    c, d = (Case(s, M, 500, 1024, levels) for s in (4, 5))
    out = torch.zeros((M, 500), device="cuda")
    buf = torch.empty(qift.qift_levels_bytes(1024, c.weights), dtype=torch.uint8, device="cuda")
    run(c, out=out, levels_buf=buf)
    c.check(out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(c, out=out, levels_buf=buf)
    for i in range(2):
        c.q.copy_(d.q)
        (c.weights[i][0]).copy_(d.weights[i][0]), (c.weights[i][1]).copy_(d.weights[i][1])
        c.values[i] = d.values[i]
        out.zero_(), buf.fill_(0x55)
        graph.replay()
        c.check(out)
    assert qift.qift_device_status() == (qift.OK, 0)


@pytest.mark.parametrize("rows", [1, 12, 50, 400, "many"])
def test_weights_written_right_before(rows):
    """Packed weights that a copy, or the packing call, has written just before, in stream order."""
    M = many() if rows == "many" else rows
    cases = [Case(s, M, 4800, 1024, "mnz") for s in (1, 2)]
    wants = [run(c) for c in cases]
    for c, w in zip(cases, wants):
        c.check(w)
    place = [(torch.zeros_like(p), torch.zeros_like(s)) for p, s in cases[0].weights]
    x = torch.randn((M, 1024), device="cuda")
    got = []
    for i in range(8):
        c = cases[i % 2]
        for (p, s), (p0, s0) in zip(place, c.weights):
            p.copy_(p0), s.copy_(s0)
        if i % 4 > 1:
            qift.qift_quantize_act(x, 1024)                          # a launch between that lets the next begin early
        got.append(qift.qift_gated_linear(c.q, c.s, *place, c.lv))
    assert all(torch.equal(g, wants[i % 2]) for i, g in enumerate(got))
    W = [torch.randn((4800, 1024), device="cuda", generator=torch.Generator("cuda").manual_seed(i)) for i in range(2)]
    c = cases[0]
    plain = [qift.qift_pack_weights(w, qift.MNZ, qift.SCALE_ABSMAX) for w in W]
    torch.cuda.synchronize()
    want = qift.qift_gated_linear(c.q, c.s, *plain, c.lv)
    fresh = [(torch.zeros_like(p), torch.zeros_like(s)) for p, s in plain]
    torch.cuda.synchronize()
    for w, (p, s) in zip(W, fresh):
        qift.qift_pack_weights(w, qift.MNZ, qift.SCALE_ABSMAX, s_n=s, packed=p)
    assert torch.equal(qift.qift_gated_linear(c.q, c.s, *fresh, c.lv), want)


@pytest.mark.parametrize("rows", [(1, 50), (12, 400), (50, "many"), ("many", "many")])
def test_two_streams_at_once(rows):
    """Two graphs, each of several calls, replayed side by side: they share no memory of the library's."""
    cases, outs, graphs, wants = [], [], [], []
    for i, M in enumerate(rows):
        c = Case(20 + i, many(i) if M == "many" else M, 2000 + 8 * i, 1024, ("mnz", "int4")[i])
        wants.append(run(c))
        c.check(wants[-1])
        out = [torch.zeros_like(wants[-1]) for _ in range(6)]
        buf = torch.empty(qift.qift_levels_bytes(1024, c.weights), dtype=torch.uint8, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for o in out:
                run(c, out=o, levels_buf=buf)
        cases.append((c, buf)), outs.append(out), graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in rows]
    for _ in range(5):
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
        for s, g, o in zip(streams, graphs, outs):
            with torch.cuda.stream(s):
                for t in o:
                    t.zero_()
                g.replay()
        for s in streams:
            torch.cuda.current_stream().wait_stream(s)
        assert all(torch.equal(t, w) for o, w in zip(outs, wants) for t in o)
    assert qift.qift_device_status() == (qift.OK, 0)

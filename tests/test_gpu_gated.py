"""The gated half of a feed-forward block: exact sums, h against 64 bits, on every route."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_02823_b200 as qift
from gated_ref import LEVELS, Case, check

pytestmark = pytest.mark.gpu
ACTS = [qift.ACT_SILU, qift.ACT_GELU_TANH]


def run(c, act=qift.ACT_SILU, dtype=torch.float32, **kw):
    return qift.qift_gated_linear(c.q, c.s, *c.weights, c.lv, activation=act, out_dtype=dtype, **kw)


@pytest.mark.parametrize("levels", list(LEVELS))
@pytest.mark.parametrize("M, N, K", [
    (1, 1, 32), (1, 300, 1024), (1, 2400, 4096), (2, 17, 256), (3, 100, 288), (5, 16, 4096), (7, 1000, 2048), (8, 333, 544), (9, 48, 1024),
    (13, 130, 4128), (16, 260, 4096), (16, 100, 14336), (17, 100, 256), (20, 129, 1056), (31, 300, 1024), (33, 257, 2080), (48, 500, 512), (64, 128, 4096),
    (65, 31, 1024), (100, 390, 256), (128, 256, 2048), (129, 200, 256), (200, 131, 1056), (300, 700, 1024), (513, 300, 512), (1025, 515, 256)])
def test_sizes(M, N, K, levels):
    c = Case(M * 7 + N, M, N, K, levels)
    act = ACTS[(M + N) % 2]
    sums = c.sums()
    h, *accs = run(c, act, want_acc=True)
    c.check(h, accs, act, sums)
    b = run(c, act, torch.bfloat16)
    assert torch.equal(b, h.to(torch.bfloat16))                      # the same fp32 value, rounded once


@pytest.mark.parametrize("levels, K", [("mnz", 16), ("mnz", 48), ("pot", 1040), ("sym", 272), ("int4", 8), ("int4", 24), ("int4", 136), ("int4", 4104), ("int3", 96)])
@pytest.mark.parametrize("M", [1, 6, 16, 40, 140])
def test_odd_depths(M, K, levels):
    c = Case(K + M, M, 37, K, levels)
    h, *accs = run(c, want_acc=True)
    c.check(h, accs)


@pytest.mark.parametrize("M", [1, 30, 150])
@pytest.mark.parametrize("act", ACTS)
def test_large_and_small_gates(M, act):
    """Gates beyond +-100: exp(-z) passes the fp32 range, the activation goes to g and to 0."""
    c = Case(3, M, 400, 512, "int4", extreme=True)
    c.s[0] = 40.0
    c.s[-1] = 0.0
    h = run(c, act)
    assert torch.isfinite(h).all()
    c.check(h, act=act)
    assert (h[-1] == 0).all()


def test_same_rows_same_bits_on_every_route():
    """A row's results do not depend on how many others there are."""
    c = Case(5, 700, 333, 512, "mnz")
    whole = run(c)
    for M in (1, 2, 9, 20, 60, 128, 200):
        part = qift.qift_gated_linear(c.q[:M].contiguous(), c.s[:M].contiguous(), *c.weights, c.lv)
        assert torch.equal(part, whole[:M]), M


@pytest.mark.parametrize("M", [1, 4, 40, 200])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_forward_from_activations(M, dtype):
    c = Case(11, M, 130, 1024, "mnz")
    x = torch.from_numpy(np.random.default_rng(M).standard_normal((M, 1024)).astype(np.float32)).cuda().to(dtype)
    q, s = oracle.quantize_act(x.float().cpu().numpy(), 1024, 0.9)
    c.q, c.s = torch.from_numpy(q).cuda(), torch.from_numpy(s).cuda()
    h, *accs = qift.qift_gated_forward(x, 1024, *c.weights, c.lv, 0.9, want_acc=True)
    c.check(h, accs)
    scratch = torch.empty(qift.lib().qift_gated_forward_scratch_bytes(M, 1024), dtype=torch.uint8, device="cuda")
    assert torch.equal(h, qift.qift_gated_forward(x, 1024, *c.weights, c.lv, 0.9, scratch=scratch))


def test_extremes_of_the_codes():
    """Largest sums: every code and activation at the end of its range."""
    for levels, lv in LEVELS.items():
        K, N, M = 16384, 33, 3
        top = int(np.argmax(np.abs(oracle.level_table(lv))))
        packed = torch.from_numpy(oracle.pack(np.full((N, K), top, np.uint8), lv).view(np.int32).ravel()).cuda()
        s_n, s_a = torch.full((N,), 1e-5, device="cuda"), torch.ones(M, device="cuda")
        q = torch.full((M, K), -8, dtype=torch.int8, device="cuda")
        q[1] = 7
        h, a, b = qift.qift_gated_linear(q, s_a, (packed, s_n), (packed, s_n), lv, want_acc=True)
        v = int(oracle.level_table(lv)[top])
        assert (a[0] == -8 * v * K).all() and (a[1] == 7 * v * K).all() and torch.equal(a, b), levels
        check(h, [a, b], s_a, [s_n, s_n], qift.ACT_SILU)


def test_levels_decoded_ahead():
    """The call in a chain: another call decodes its codes, and it decodes another's."""
    M = max(300, qift.qift_gated_levels_min_rows())
    c, d = Case(1, M, 200, 512, "mnz"), Case(2, M, 96, 256, "int3")
    buf = torch.zeros(qift.qift_levels_bytes(512, c.weights), dtype=torch.uint8, device="cuda")
    other = torch.zeros(qift.qift_levels_bytes(256, d.weights), dtype=torch.uint8, device="cuda")
    x = torch.from_numpy(np.random.default_rng(1).standard_normal((M, 512)).astype(np.float32)).cuda()
    qift.qift_forward_multi(x, 512, c.weights, c.lv, ahead=(c.weights, 512, c.lv, buf))
    h = run(c, levels_buf=buf, levels_ready=True, ahead=(d.weights, 256, d.lv, other))
    c.check(h)
    e = run(d, levels_buf=other, levels_ready=True)
    d.check(e)
    small = Case(3, 5, 200, 512, "mnz")                              # few rows decode for later calls all the same
    buf.zero_()
    run(small, ahead=(c.weights, 512, c.lv, buf))
    assert torch.equal(run(c, levels_buf=buf, levels_ready=True), h)


@pytest.mark.parametrize("M", [1, 12, 50, 400])
def test_captured_on_another_stream(M):
    c = Case(4, M, 500, 1024, "mnz")
    out = torch.zeros((M, 500), device="cuda")
    buf = torch.empty(qift.qift_levels_bytes(1024, c.weights), dtype=torch.uint8, device="cuda")
    run(c, out=out, levels_buf=buf)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(c, out=out, levels_buf=buf)
    for seed in range(2):
        c.q.copy_(torch.from_numpy(np.random.default_rng(seed).integers(-8, 8, (M, 1024)).astype(np.int8)))
        out.zero_()
        graph.replay()
        c.check(out)
    rc, detail = qift.qift_device_status()
    assert rc == qift.OK, (rc, detail)


def test_weights_of_another_size_are_refused():
    c = Case(1, 3, 40, 512, "mnz")
    (pg, sg), up = c.weights
    with pytest.raises(AssertionError, match="another size"):
        qift.qift_gated_linear(c.q, c.s, (pg[:-8], sg), up, c.lv)
    with pytest.raises(AssertionError, match="another size"):
        qift.qift_gated_linear(torch.zeros((3, 1024), dtype=torch.int8, device="cuda"), c.s, *c.weights, c.lv)
    with pytest.raises(qift.QiftError):
        qift.qift_gated_linear(c.q, c.s, (pg, sg), (up[0], up[1][:32]), c.lv)


@pytest.mark.parametrize("levels, M, N, K", [
    ("mnz", 5, 40, 28672), ("mnz", 16, 40, 28672), ("int3", 16, 130, 16384), ("int4", 12, 40, 20008), ("int4", 7, 33, 16384), ("pot", 1, 20, 225280),
    ("sym", 1, 20, 231424), ("mnz", 2, 300, 240000), ("int4", 1, 9, 240008), ("int4", 3, 20, 1 << 21)])
def test_long_rows(levels, M, N, K):
    """Few rows whose activations, beside the rings of codes, pass what shared memory holds."""
    c = Case(M + K, M, N, K, levels)
    h, *accs = run(c, want_acc=True)
    c.check(h, accs)
    assert qift.qift_device_status()[0] == qift.OK


def test_longest_sums():
    """Every operand at the end of its range over 2^21 codes: beyond 32 bits once the factors of the tensor cores' operands are on."""
    for K in ((1 << 21) - 16, 1 << 21):
        table = oracle.level_table(qift.INT4)
        low = int(np.min(table))
        packed = torch.from_numpy(oracle.pack(np.full((2, K), int(np.argmin(table)), np.uint8), qift.INT4).view(np.int32).ravel()).cuda()
        s_n, s_a = torch.full((2,), 1e-9, device="cuda"), torch.ones(20, device="cuda")
        q = torch.full((20, K), -8, dtype=torch.int8, device="cuda")
        h, a, b = qift.qift_gated_linear(q, s_a, (packed, s_n), (packed, s_n), qift.INT4, want_acc=True)
        assert (a == -8 * low * K).all() and torch.equal(a, b)
        check(h, [a, b], s_a, [s_n, s_n], qift.ACT_SILU)


@pytest.mark.parametrize("levels", list(LEVELS))
@pytest.mark.parametrize("M, N, K", [(450, 150, 512), (512, 257, 256), (700, 96, 1056), (1025, 264, 288), (1300, 131, 544)])
def test_decoded_by_an_earlier_call(M, N, K, levels):
    """Levels that are there, from the fewest rows on that use them: the same bits as from the codes."""
    c = Case(M + N, M, N, K, levels)
    buf = torch.zeros(qift.qift_levels_bytes(K, c.weights), dtype=torch.uint8, device="cuda")
    few = qift.qift_gated_linear(c.q[:40].contiguous(), c.s[:40].contiguous(), *c.weights, c.lv, ahead=(c.weights, K, c.lv, buf))
    h, *accs = run(c, levels_buf=buf, levels_ready=True, want_acc=True)
    c.check(h, accs)
    assert torch.equal(h, run(c)) and torch.equal(h[:40], few)
    assert torch.equal(run(c, dtype=torch.bfloat16, levels_buf=buf, levels_ready=True), h.to(torch.bfloat16))


@pytest.mark.parametrize("N", [120, 131])
def test_many_rows_same_bits(N):
    """Rows of a call that decodes the codes first against calls of fewer rows."""
    c = Case(N, qift.qift_gated_levels_min_rows() + 70, N, 512, "sym")
    whole = run(c, qift.ACT_GELU_TANH)
    c.check(whole, act=qift.ACT_GELU_TANH)
    for M in (1, 30, 300, 600):
        part = qift.qift_gated_linear(c.q[-M:].clone(), c.s[-M:].clone(), *c.weights, c.lv, activation=qift.ACT_GELU_TANH)
        assert torch.equal(part, whole[-M:]), M


@pytest.mark.parametrize("M, N", [(64, 33_600_016), (1100, 1_960_008)])
def test_more_results_than_32_bits_count(M, N):
    """Row by row the same as calls of one row."""
    K = 32
    assert M * N > 1 << 31
    g = torch.Generator("cuda").manual_seed(N)
    weights = [(torch.randint(-2 ** 31, 2 ** 31 - 1, ((N + 15) // 16 * 256,), dtype=torch.int32, device="cuda", generator=g),
                torch.rand(N, device="cuda", generator=g)) for _ in range(2)]
    q = torch.randint(-8, 8, (M, K), dtype=torch.int8, device="cuda", generator=g)
    s = torch.rand(M, device="cuda", generator=g)
    whole = qift.qift_gated_linear(q, s, *weights, qift.MNZ, out_dtype=torch.bfloat16)
    for m in (0, M // 2, M - 1):
        assert torch.equal(whole[m], qift.qift_gated_linear(q[m:m + 1].clone(), s[m:m + 1].clone(), *weights, qift.MNZ, out_dtype=torch.bfloat16)[0]), m


@pytest.mark.parametrize("levels", list(LEVELS))
@pytest.mark.parametrize("M, K", [(9, 512), (16, 1040), (13, 264)])
def test_some_rows_of_many_channels(M, K, levels):
    """More tiles of channels than a few for every SM."""
    K = K if levels == "int4" else K // 32 * 32
    c = Case(M + K, M, 9600, K, levels)
    h, *accs = run(c, qift.ACT_GELU_TANH, want_acc=True)
    c.check(h, accs, act=qift.ACT_GELU_TANH)

"""A decoder layer of a batch of requests, from page tables to the feed-forward block, as its calls follow one another in a step: on the
values of the calls before, against 64 bits stage by stage, over several steps and captured into a graph."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_02823_b200 as qift
from gated_ref import check as check_gated
from tables_ref import Tables

pytestmark = pytest.mark.gpu
D, Hq, H, E, F = 128, 8, 2, 1024, 1472        # head size, query and KV heads, width of the model and of the block between
P, R, MOST, PAGES, TOTAL = 32, 3, 6, 14, 24   # page size, requests, pages of a request, pages of the pool, rows of a step


def ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


class Layer:
    def __init__(self, seed, dtype):
        r = np.random.default_rng(seed)
        self.dtype = dtype
        W = {}
        for name, (n, k) in dict(qkv=((Hq + 2 * H) * D, E), o=(E, Hq * D), gate=(F, E), up=(F, E), down=(E, F)).items():
            W[name] = qift.qift_pack_weights(torch.from_numpy((r.standard_normal((n, k)) * 0.05).astype(np.float32)).cuda(), qift.MNZ, qift.SCALE_MSE)
        self.W = W
        self.wq, self.wk = (torch.from_numpy((1 + 0.2 * r.standard_normal(D)).astype(np.float32)).cuda().to(dtype) for _ in range(2))
        self.inv = torch.tensor([10000.0 ** (-i / 64) for i in range(64)], dtype=torch.float32, device="cuda")
        self.pages = qift.Kv4Pages.empty(PAGES, H, P, torch.full((R, MOST), -1, dtype=torch.int32, device="cuda"))
        self.free = qift.Kv4FreePages.all_of(PAGES)
        self.plan = qift.Kv4Rows.empty(R, TOTAL)

    def step(self, x, rows, first, length):
        """Every tensor of the step by name."""
        W, s = self.W, {}
        qift.qift_kv4_pages_begin(self.pages, self.free, rows, first, TOTAL, out=self.plan)
        s["qkv"] = qift.qift_forward(x, 1024, *W["qkv"], qift.MNZ, out_dtype=self.dtype).view(TOTAL, Hq + 2 * H, D)
        s["q"], s["k"] = (torch.zeros((TOTAL, n, D), dtype=self.dtype, device="cuda") for n in (Hq, H))
        qift.qift_qk_norm_rope(s["qkv"][:, :Hq], s["qkv"][:, Hq:Hq + H], self.plan.position, self.inv, self.wq, self.wk, q_out=s["q"], k_out=s["k"])
        qift.qift_kv4_paged_write(s["k"], s["qkv"][:, Hq + H:], self.pages, self.plan.row_start, first, k_had_block=D)
        s["attended"] = torch.zeros((TOTAL, Hq, D), dtype=self.dtype, device="cuda")
        qift.qift_kv4_paged_attention(s["q"], self.pages, self.plan.row_start, first, q_had_block=D, out=s["attended"])
        s["o"] = qift.qift_forward(s["attended"].view(TOTAL, Hq * D), 1024, *W["o"], qift.MNZ, out_dtype=self.dtype)
        s["h"], s["acc_g"], s["acc_u"] = qift.qift_gated_forward(s["o"], 1024, W["gate"], W["up"], qift.MNZ, out_dtype=self.dtype, want_acc=True)
        s["y"] = qift.qift_forward(s["h"], 64, *W["down"], qift.MNZ, out_dtype=self.dtype)
        qift.qift_kv4_pages_end(self.pages, self.free, length)
        return s


def steps():
    """Rows, cached tokens before, tokens that stay: prompts, single tokens, a draft of which part stays, one request ends and another begins."""
    yield [9, 0, 14], [0, 0, 0], [9, 0, 14]
    yield [1, 20, 1], [9, 0, 14], [10, 20, 15]
    yield [5, 3, 4], [10, 20, 15], [12, 21, 0]
    yield [1, 1, 22], [12, 21, 0], [13, 22, 22]


def check_step(L, s, plain, rows, first):
    start, position, slot, lost = plain.begin(rows, first, TOTAL)
    assert lost == 0
    for got, want in ((L.plan.row_start, start), (L.plan.position, position), (L.plan.slot, slot)):
        assert np.array_equal(got.cpu().numpy(), want)
    live = position >= 0
    bf16 = L.dtype == torch.bfloat16
    # keys and queries of the rows, from the projection as it is
    x = s["qkv"].double().cpu().numpy()[live]
    angle = position[live][:, None].astype(np.float64) * L.inv.double().cpu().numpy()
    c, si = np.cos(angle)[:, None], np.sin(angle)[:, None]
    for got, a, b, w in ((s["q"], 0, Hq, L.wq), (s["k"], Hq, Hq + H, L.wk)):
        y = x[:, a:b] / np.sqrt((x[:, a:b] ** 2).mean(-1, keepdims=True) + float(np.float32(1e-6))) * w.double().cpu().numpy()
        want = np.concatenate([y[..., :64] * c - y[..., 64:] * si, y[..., 64:] * c + y[..., :64] * si], -1)
        pair = np.tile(np.abs(y[..., :64]) + np.abs(y[..., 64:]), 2)
        got = got.double().cpu().numpy()
        # 30 roundings to fp32 of a pair (as the kernel's own test counts them), and one to the rows' type
        assert (np.abs(got[live] - want) <= pair * 30 * 2.0 ** -24 + (np.abs(want) * 2.0 ** -8 if bf16 else 0) * 1.01).all()
        assert (got[~live] == 0).all()
    # h from the accumulators, and those from the quantized activation
    q, sa = oracle.quantize_act(s["o"].float().cpu().numpy(), 1024, 0.9)
    sums = [torch.from_numpy(oracle.int_matmul(oracle.unpack(L.W[n][0].cpu().numpy().view(np.uint32), F, E, qift.MNZ), qift.MNZ, q).astype(np.int32)).cuda() for n in ("gate", "up")]
    assert torch.equal(s["acc_g"], sums[0]) and torch.equal(s["acc_u"], sums[1])
    check_gated(s["h"], sums, torch.from_numpy(sa).cuda(), [L.W["gate"][1], L.W["up"][1]], qift.ACT_SILU)
    # the cache holds the rows' keys, exactly as the oracle quantizes them, at the slots that were handed out
    keys = s["k"].float().cpu().numpy()[live]
    codes, sc, z = oracle.kv4_quantize(keys.reshape(-1, D), D, 0.95)
    held = (sc[:, None] * (codes.astype(np.float32) - z[:, None])).reshape(-1, H, D)
    got = qift.qift_kv4_paged_read(L.pages, ints(start), ints(first), TOTAL)[0].cpu().numpy()[live]
    assert np.array_equal(got, held)
    assert torch.isfinite(s["y"]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_steps_of_a_layer(dtype):
    L = Layer(1, dtype)
    plain = Tables(np.full((R, MOST), -1), np.arange(PAGES - 1, -1, -1), PAGES, P, PAGES)
    r = np.random.default_rng(2)
    for rows, first, length in steps():
        x = torch.from_numpy(r.standard_normal((TOTAL, E)).astype(np.float32)).cuda().to(dtype)
        # the read in the check wants the pages of this step: they go back in a call of their own
        s = L.step(x, ints(rows), ints(first), ints([a + b for a, b in zip(rows, first)]))
        check_step(L, s, plain, rows, first)
        qift.qift_kv4_pages_end(L.pages, L.free, ints(length))
        plain.end([a + b for a, b in zip(rows, first)])
        plain.end(length)
        assert np.array_equal(L.pages.page_table.cpu().numpy(), plain.table) and int(L.free.count) == plain.count


def test_a_captured_step_goes_on_by_itself():
    """The same steps as one graph that is replayed with other lengths give the same bits."""
    eager, graphed = Layer(3, torch.bfloat16), Layer(3, torch.bfloat16)
    x, rows, first, length = torch.zeros((TOTAL, E), dtype=torch.bfloat16, device="cuda"), ints([0] * R), ints([0] * R), ints([0] * R)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graphed.step(x, rows, first, length)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = graphed.step(x, rows, first, length)
    r = np.random.default_rng(4)
    for n, f, k in steps():
        x.copy_(torch.from_numpy(r.standard_normal((TOTAL, E)).astype(np.float32)))
        rows.copy_(ints(n)), first.copy_(ints(f)), length.copy_(ints(k))
        want = eager.step(x, rows, first, length)
        graph.replay()
        for name in want:
            assert torch.equal(out[name], want[name]), name
        assert torch.equal(eager.pages.page_table, graphed.pages.page_table) and torch.equal(eager.free.pages[:int(eager.free.count)], graphed.free.pages[:int(eager.free.count)])
    rc, detail = qift.qift_device_status()
    assert rc == qift.OK, (rc, detail)

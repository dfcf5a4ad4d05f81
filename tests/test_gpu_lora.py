"""Adapters of many requests beside a shared projection, against 64 bits."""
import numpy as np
import pytest
import torch

import synth
import paper_2606_02823_b200 as qift

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def ints(v):
    return torch.tensor(list(v), dtype=torch.int32, device="cuda")


def normal(seed, shape, dtype, scale=1.0):
    return torch.from_numpy((synth.normal(seed, 3, shape) * scale).astype(np.float32)).cuda().to(dtype)


class Case:
    def __init__(self, seed, rows, ids, n, rank, K, N, dtype, pad_rows=0):
        self.dtype, self.ids, self.rank = DTYPES[dtype], ids, rank
        self.cut = np.concatenate([[0], np.cumsum(rows)])
        M = int(self.cut[-1]) + pad_rows
        self.x, self.y = normal(seed, (M, K), self.dtype), normal(seed + 1, (M, N), self.dtype)
        self.A, self.B = normal(seed + 2, (n, rank, K), torch.bfloat16, K ** -0.5), normal(seed + 3, (n, N, rank), torch.bfloat16, rank ** -0.5)
        self.scaling = normal(seed + 4, (n,), torch.float32).abs() + 0.5
        self.rs, self.adapter = ints(self.cut.tolist()), ints(ids)

    def call(self, **kw):
        kw.setdefault("y", self.y)
        return qift.qift_lora_linear(self.x, self.A, self.B, self.scaling, self.rs, self.adapter, **kw)

    def check(self, got, y=True):
        """Bounds, worst case: A x is an fp32 sum of K products of x held to 2^-17 at least (bf16 exactly), then held to 2^-17 again
        for the second product of rank terms; sums of n terms in fp32 are off by n 2^-24 of the sum of magnitudes."""
        K, M = self.x.shape[1], int(self.cut[-1])
        x, A, B, s = self.x.double(), self.A.double(), self.B.double(), self.scaling.double()
        want = self.y.double().clone() if y else torch.zeros_like(self.y.double())
        bound = torch.zeros_like(want)
        for i, a in enumerate(self.ids):
            at = slice(int(self.cut[i]), int(self.cut[i + 1]))
            if 0 <= a < A.shape[0]:
                want[at] += s[a] * (x[at] @ A[a].T) @ B[a].T
                size = s[a] * (x[at].abs() @ A[a].abs().T) @ B[a].abs().T
                bound[at] = size * (2 * 2.0 ** -17 + (K + self.rank + 8) * 2.0 ** -24) + 2.0 ** -23 * (want[at].abs() + self.y[at].double().abs())
        bound += (2.0 ** -8 if self.dtype == torch.bfloat16 else 2.0 ** -23) * want.abs()
        err = (got.double() - want).abs()[:M]
        assert (err <= bound[:M] + 1e-30).all(), ((err / (bound[:M] + 1e-30)).max().item(), err.max().item())


SHAPES = [([1], [0], 1, 8, 64, 64), ([1] * 5, [2, 0, 2, 1, 0], 3, 16, 256, 136), ([3, 0, 17, 1], [1, 0, 0, 1], 2, 24, 1000, 72),
          ([40, 70], [0, 1], 2, 64, 512, 520), ([130, 5], [1, 0], 2, 128, 264, 1032), ([200], [0], 1, 40, 4096, 1024), ([33] * 6, [0, 1, 2, 3, 4, 0], 5, 16, 768, 264)]


@pytest.mark.parametrize("rows,ids,n,rank,K,N", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_against_64_bits(rows, ids, n, rank, K, N, dtype):
    c = Case(400, rows, ids, n, rank, K, N, dtype)
    c.check(c.call())
    c.check(c.call(y=None), y=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [[2, 3, 1], [50, 21, 40]])
def test_rows_without_adapter_rows_of_nobody_and_in_place(dtype, rows):
    c = Case(410, rows, [1, -1, 7], 2, 16, 512, 264, dtype, pad_rows=2)                # 7: no such adapter
    c.x[-2:] = float("nan")
    out = torch.full_like(c.y, 9.0)
    got = c.call(out=out)
    c.check(got)
    assert torch.equal(got[rows[0]:-2], c.y[rows[0]:-2]) and (got[-2:] == 9).all()
    inplace = c.y.clone()
    c.call(y=inplace, out=inplace)
    assert torch.equal(inplace[:-2], got[:-2]) and torch.equal(inplace[-2:], c.y[-2:])
    zero = c.call(y=None, out=torch.full_like(c.y, 9.0))
    assert not zero[rows[0]:-2].any()


def test_beside_the_quantized_projection():
    """The shared W2A4 product and the adapters of its requests, as a server adds them."""
    M, K, N = 24, 1024, 512
    W = normal(420, (N, K), torch.float32, 0.02)
    packed, s_n = qift.qift_pack_weights(W, qift.MNZ, qift.SCALE_ABSMAX)
    c = Case(421, [1] * M, [i % 4 - 1 for i in range(M)], 3, 16, K, N, "bf16")
    q_a, s_a = qift.qift_quantize_act(c.x, 1024, 0.9)
    c.y = qift.qift_w2a4_linear(packed, s_n, qift.MNZ, q_a, s_a, out_dtype=torch.bfloat16)
    c.y = c.y[0] if isinstance(c.y, tuple) else c.y
    c.check(c.call())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_calls_share_a_workspace(dtype):
    cases = [Case(430, [1] * 20, [i % 3 for i in range(20)], 3, 16, 512, 264, dtype), Case(440, [60, 1, 90], [1, 0, 1], 2, 32, 512, 264, dtype)]
    ws = torch.full((max(qift.qift_lora_workspace_bytes(c.x.shape[0], c.rank, 512) for c in cases),), 0xFF, dtype=torch.uint8, device="cuda")
    graphs = []
    for c in cases:
        want = c.call()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = c.call(workspace=ws)
        graphs.append((g, want, got))
    for _ in range(3):
        for g, _, _ in graphs:
            g.replay()
        for _, want, got in graphs:
            assert torch.equal(want, got)
    cases[0].adapter.copy_(ints([(i + 1) % 3 for i in range(20)]))
    want = cases[0].call()
    graphs[0][0].replay()
    assert torch.equal(want, graphs[0][2])


def test_two_streams_at_once():
    cases = [Case(450, [1] * 40, [i % 5 for i in range(40)], 5, 16, 2048, 1024, "bf16"), Case(460, [300], [0], 1, 64, 2048, 1024, "bf16")]
    wants = [c.call() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(5):
        gots = []
        for s, c in zip(streams, cases):
            with torch.cuda.stream(s):
                gots.append(c.call())
        torch.cuda.synchronize()
        assert all(torch.equal(w, g) for w, g in zip(wants, gots))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rank,rows", [(8, [300, 259, 257]), (16, [129, 0, 400]), (24, [90, 170]), (32, [65, 128, 1, 127]), (72, [33, 63, 31])])
def test_long_requests_of_every_rank(rank, rows, dtype):
    """Items of 128 rows: ends inside a warp's 16 rows, requests without rows, K and N that end inside a step."""
    c = Case(440, rows, [i % 2 for i in range(len(rows))], 2, rank, 328, 200, dtype)
    c.check(c.call())
    c.check(c.call(y=None), y=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_requests_without_adapter_rows_of_nobody_and_in_place(dtype):
    rows = [150, 121, 140]
    c = Case(450, rows, [1, -1, 7], 2, 64, 512, 264, dtype, pad_rows=40)
    c.x[-40:] = float("nan")
    c.x[3] = float("inf")                                                             # spoils its own row alone
    got = c.call(out=torch.full_like(c.y, 9.0))
    c.x[3], got[3] = 0.0, c.y[3]
    c.check(got)
    assert torch.equal(got[rows[0]:-40], c.y[rows[0]:-40]) and (got[-40:] == 9).all()
    inplace = c.y.clone()
    c.call(y=inplace, out=inplace)
    assert torch.equal(inplace[:-40], got[:-40]) and torch.equal(inplace[-40:], c.y[-40:])

"""Norms of queries and keys and their rotation by position, against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2606_02823_b200 as qift

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def normal(seed, shape, dtype=torch.float32):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape).astype(np.float32)).cuda().to(dtype)


def frequencies(rot, base=10000.0):
    return torch.tensor([base ** (-i / (rot // 2)) for i in range(rot // 2)], dtype=torch.float32, device="cuda")


def wanted(x, position, inv_freq, weight, eps, near):
    """-> (64-bit result, its bound in fp32).  The sum of D <= 512 squares runs over 16 of a thread and five exchanges: 22 roundings at
    most, halved by the root, and seven more to y: 18 U.  Sine and cosine: the angle less its whole turns, at most pi, is rounded
    to fp32 (pi U) after three roundings in fp64 (of the angle A: 3 A 2^-53), and the functions are within 2 ulp: 6 U.  Three roundings of
    the products and their sum.  All of that of |a| + |b|: 30 U covers it."""
    D, pairs = x.shape[-1], inv_freq.numel()
    y = x.double()
    if weight is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + float(np.float32(eps))) * weight.double()
    angle = position.double()[:, None] * inv_freq.double()
    c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    out, bound = y.clone(), y.abs() * 30 * U
    ia, ib = (torch.arange(0, 2 * pairs, 2), torch.arange(1, 2 * pairs, 2)) if near else (torch.arange(pairs), torch.arange(pairs, 2 * pairs))
    a, b = y[..., ia], y[..., ib]
    out[..., ia], out[..., ib] = a * c - b * s, b * c + a * s
    off = (a.abs() + b.abs()) * (30 * U + 3 * 2.0 ** -53 * angle.abs()[:, None])
    bound[..., ia], bound[..., ib] = off, off
    return out, bound


def check(got, x, position, inv_freq, weight, eps, near, old=None):
    want, bound = wanted(x, position, inv_freq, weight, eps, near)
    if got.dtype == torch.bfloat16:
        bound = bound + (want.abs() + bound) * 2.0 ** -8
    off = (got.double() - want).abs()
    rows = position >= 0
    assert (off[rows] <= bound[rows] + 1e-37).all(), (off[rows] / (bound[rows] + 1e-37)).max()
    if old is not None:
        assert torch.equal(got[~rows], old[~rows])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("near", [False, True])
@pytest.mark.parametrize("total, Hq, H, D, rot, norm", [
    (1, 32, 8, 128, 128, True), (1, 1, 1, 128, 128, False), (48, 32, 8, 128, 128, False), (333, 32, 32, 128, 96, True),
    (17, 7, 1, 64, 32, True), (5, 3, 2, 16, 16, True), (29, 5, 5, 32, 16, False), (9, 12, 3, 96, 96, True), (301, 2, 2, 256, 224, True),
    (7, 3, 1, 512, 512, True), (11, 2, 1, 400, 64, True), (5000, 4, 1, 128, 128, True)])
def test_sizes(total, Hq, H, D, rot, norm, near, dtype):
    t = DTYPES[dtype]
    row = normal(total, (total, Hq + 2 * H, D), t)                    # one projection's rows
    q, k = row[:, :Hq], row[:, Hq:Hq + H]
    position = torch.from_numpy(np.random.default_rng(D).integers(-2, 40000, total).astype(np.int32)).cuda()
    position[0] = 39999
    wq, wk = (1 + 0.3 * normal(7, (2, D))).to(t) if norm else (None, None)
    inv = frequencies(rot)
    oq, ok = normal(1, q.shape, t), normal(2, k.shape, t)
    gq, gk = qift.qift_qk_norm_rope(q, k, position, inv, wq, wk, 1e-5, near, q_out=oq.clone(), k_out=ok.clone())
    check(gq, q, position, inv, wq, 1e-5, near, oq)
    check(gk, k, position, inv, wk, 1e-5, near, ok)
    # in place in the projection's rows: the same values, and what lies beside them is not touched
    place = row.clone()
    qift.qift_qk_norm_rope(place[:, :Hq], place[:, Hq:Hq + H], position, inv, wq, wk, 1e-5, near, q_out=place[:, :Hq], k_out=place[:, Hq:Hq + H])
    live = position >= 0
    assert torch.equal(place[live][:, :Hq], gq[live]) and torch.equal(place[live][:, Hq:Hq + H], gk[live])
    assert torch.equal(place[:, Hq + H:], row[:, Hq + H:]) and torch.equal(place[~live], row[~live])


@pytest.mark.parametrize("which", ["q", "k"])
def test_one_norm_alone(which):
    q, k, position, inv = normal(1, (9, 8, 128)), normal(2, (9, 2, 128)), torch.arange(9, dtype=torch.int32, device="cuda"), frequencies(128)
    w = 1 + 0.3 * normal(3, (128,))
    wq, wk = (w, None) if which == "q" else (None, w)
    gq, gk = qift.qift_qk_norm_rope(q, k, position, inv, wq, wk)
    check(gq, q, position, inv, wq, 1e-6, False)
    check(gk, k, position, inv, wk, 1e-6, False)


def test_far_positions():
    """Up to 2^31 - 1 turns are counted in fp64."""
    position = torch.tensor([2 ** 31 - 1, 2 ** 30 + 7, 10 ** 8, 1_000_003, 65537, 1, 0], dtype=torch.int32, device="cuda")
    q, k, inv = normal(1, (7, 2, 128)), normal(2, (7, 1, 128)), frequencies(128, 500000.0)
    gq, gk = qift.qift_qk_norm_rope(q, k, position, inv)
    check(gq, q, position, inv, None, 1e-6, False)
    check(gk, k, position, inv, None, 1e-6, False)
    assert torch.equal(gq[6], q[6])                                   # position 0 turns nothing


def test_zeros_and_what_is_no_number():
    q, k = normal(1, (6, 2, 128)), normal(2, (6, 1, 128))
    q[0], q[1, 0, 5], q[2, 1, 100], q[3, 0, :] = 0.0, float("inf"), float("nan"), 1e-30
    q[5, 0, 127] = float("inf")
    position = torch.arange(6, dtype=torch.int32, device="cuda")
    w, inv = 1 + 0.1 * normal(3, (128,)), frequencies(64)
    gq, _ = qift.qift_qk_norm_rope(q, k, position, inv, w, w)
    assert (gq[0] == 0).all() and torch.isnan(gq[1, 0]).any() and torch.isnan(gq[2, 1]).all()
    assert torch.isfinite(gq[1, 1]).all() and torch.isfinite(gq[2, 0]).all() and torch.isfinite(gq[3]).all() and torch.isfinite(gq[4]).all()
    plain, _ = qift.qift_qk_norm_rope(q, k, position, inv)            # without a norm a value stays with its pair
    assert torch.equal(plain[..., 64:].nan_to_num(7.0), q[..., 64:].nan_to_num(7.0))
    bad = ~torch.isfinite(plain[1, 0])
    assert set(bad.nonzero().flatten().tolist()) <= {5, 37}
    assert bad.any() and torch.isfinite(plain[5, 0, :127]).all()


def test_captured_on_another_stream():
    q, k, position, inv = normal(1, (40, 8, 128), torch.bfloat16), normal(2, (40, 2, 128), torch.bfloat16), torch.arange(40, dtype=torch.int32, device="cuda"), frequencies(128)
    oq, ok = torch.zeros_like(q), torch.zeros_like(k)
    qift.qift_qk_norm_rope(q, k, position, inv)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qift.qift_qk_norm_rope(q, k, position, inv, q_out=oq, k_out=ok)
    for shift in (0, 1000):
        position.add_(shift), q.mul_(1.5)
        graph.replay()
        check(oq, q, position, inv, None, 1e-6, False)
        check(ok, k, position, inv, None, 1e-6, False)


def test_rows_far_apart():
    """Strides whose multiples pass 2^31 elements, in and out."""
    step, position, inv = 2 ** 30 + 8, torch.tensor([5, -1, 70], dtype=torch.int32, device="cuda"), frequencies(64)
    q, k, w = normal(1, (3, 2, 64), torch.bfloat16), normal(2, (3, 1, 64), torch.bfloat16), normal(3, (64,), torch.bfloat16)
    space = torch.empty(2 * step + 4096, dtype=torch.bfloat16, device="cuda")
    fq, fk = space.as_strided((3, 2, 64), (step, 64, 1)), space.as_strided((3, 1, 64), (step, 64, 1), 1024)
    fq.copy_(q), fk.copy_(k)
    qift.qift_qk_norm_rope(fq, fk, position, inv, w, w, q_out=fq, k_out=fk)
    check(fq, q, position, inv, w, 1e-6, False, q)
    check(fk, k, position, inv, w, 1e-6, False, k)

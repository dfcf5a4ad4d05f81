"""fp32 adapters: the sums over K and over the rank lose nothing by the way, however long they are and however K is split."""
import numpy as np
import pytest
import torch

import synth
import paper_2606_02823_b200 as qift

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(list(v), dtype=torch.int32, device="cuda")


def normal(seed, shape):
    return torch.from_numpy(synth.normal(seed, 3, shape).astype(np.float32)).cuda()


def compare(x, A, B, rows, limit):
    """One adapter for every request; error against 64 bits: along the result (errors of one direction) and as a whole."""
    R = len(rows)
    cut = np.concatenate([[0], np.cumsum(rows)])
    one = torch.ones(1, device="cuda")
    got = qift.qift_lora_linear(x, A[None].contiguous(), B[None].contiguous(), one, ints(cut.tolist()), ints([0] * R)).double()
    want = x.double() @ A.double().T @ B.double().T
    err, size = got - want, (want * want).sum()
    bias, whole = ((err * want).sum() / size).item(), ((err * err).sum() / size).sqrt().item()
    assert abs(bias) <= limit and whole <= limit, (bias, whole, limit)


# A matrix instruction cuts up to 2^-23 off the sum that it adds to.  A step of 32 k is six of them on a sum of its own, which then joins the
# others by a rounded addition; those, about K / 32 of them in a row, are off by 2^-24 / sqrt(3) each, without a common direction:
# sqrt(K / 32 / 3) 2^-24 of the largest sum.  16 ranks are three on one sum that runs through all of them: it grows evenly, to 9/16 of the
# result on average, and half of 2^-23 of it is cut off on average.  Rows of positive numbers have all their sums grow.
def bound(K, rank):
    return 6 * 2.0 ** -23 + 2.0 ** -24 * (np.sqrt(K / 96) + 2) + 3 * (rank / 16) * 2.0 ** -24 * 9 / 16


# 16-row items with K split and unsplit, 128-row items with K split and unsplit
@pytest.mark.parametrize("rows,rank", [([1] * 8, 16), ([1] * 320, 16), ([3] * 310, 64), ([200], 64), ([40] * 300, 64), ([33] * 300, 128)])
@pytest.mark.parametrize("positive", [True, False])
def test_long_sums_over_k(rows, rank, positive):
    K = 11008
    x, A = normal(700, (sum(rows), K)), normal(701, (rank, K)).bfloat16()
    if positive:
        x, A = x.abs(), A.abs()
    compare(x, A, torch.eye(rank, device="cuda").bfloat16(), rows, bound(K, 0))


@pytest.mark.parametrize("rows", [[1] * 20, [7] * 30, [200], [130, 90]])
@pytest.mark.parametrize("rank", [24, 128])
@pytest.mark.parametrize("positive", [True, False])
def test_sums_over_the_rank(rows, rank, positive):
    x, A, B = normal(710, (sum(rows), 32)), normal(711, (rank, 32)).bfloat16(), normal(712, (512, rank)).bfloat16()
    if positive:
        x, A, B = x.abs(), A.abs(), B.abs()
    compare(x, A, B, rows, bound(32, rank))


@pytest.mark.parametrize("rows", [[1] * 20, [200]])
def test_the_sum_over_ranks_alone(rows):
    """A x is exact here (one bf16 value of x a row): two bf16 parts, the third is zero, so 16 instructions cut off the sum over 128 ranks."""
    rank, M = 128, sum(rows)
    x = torch.zeros((M, 16), device="cuda")
    x[torch.arange(M), torch.arange(M) % 16] = normal(720, (M,)).bfloat16().float().abs()
    A, B = normal(721, (rank, 16)).bfloat16().abs(), normal(722, (512, rank)).bfloat16().abs()
    compare(x, A, B, rows, 16 * 2.0 ** -24 * 9 / 16 + 2.0 ** -24)

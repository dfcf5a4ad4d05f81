"""Adapters of batches that mix one long request with many short ones: either kernel variant, K beyond 4096."""
import pytest

from test_gpu_lora import Case

import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,rank,K,N", [([300] + [1] * 60, 16, 512, 264), ([1] * 20 + [1500] + [1] * 9, 64, 512, 264), ([2, 700, 0, 1], 128, 328, 72),
                                           ([257] + [1] * 300, 16, 6000, 128), ([40] * 7 + [1], 24, 11008, 64)])
def test_one_long_request_among_short_ones(rows, rank, K, N, dtype):
    ids = [(i * 7 + 2) % 5 - 1 for i in range(len(rows))]                             # some without an adapter
    c = Case(800, rows, ids, 4, rank, K, N, dtype, pad_rows=3)
    out = torch.full_like(c.y, 9.0)
    got = c.call(out=out)
    c.check(got)
    assert (got[-3:] == 9).all()
    one = Case(800, rows, ids, 4, rank, K, N, dtype, pad_rows=3).call()               # again: the same bits
    assert torch.equal(one[:-3], got[:-3])

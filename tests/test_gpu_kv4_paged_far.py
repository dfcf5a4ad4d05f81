"""Positions next to 2^31 in a cache of which two pages exist: written, read, kept and seen like any others."""
import numpy as np
import pytest
import torch

import paged_limits as limits
import paper_2606_02823_b200 as qift
from test_gpu_kv4_paged import D, ints, ok, values

pytestmark = pytest.mark.gpu
PAGE = 1024


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,end", [(1, 2 ** 31 - 32), (40, 2 ** 31 - 32), (40, 2 ** 31 - 100), (40, 2 ** 31 - 10)])
def test_the_last_positions(n, end, dtype):
    table = torch.full((1, 2 ** 31 // PAGE), -1, dtype=torch.int32, device="cuda")
    table[0, 0], table[0, -1] = 1, 0
    pages = qift.Kv4Pages.empty(2, 1, PAGE, table)
    last = 2 ** 31 - PAGE
    k, v = values(700, (2 * PAGE, 1, D), "f32", 0.1)[0], values(701, (2 * PAGE, 1, D), "f32")[0]
    for at, first in ((0, 0), (PAGE, last)):
        qift.qift_kv4_paged_write(k[at:at + PAGE], v[at:at + PAGE], pages, ints([0, PAGE]), ints([first]))
    # the same in a cache of two pages in a row, whose last 32 positions (from 2^31 - 32 on) have no place
    near = qift.Kv4Pages.empty(2, 1, PAGE, ints([[1, 0]]))
    qift.qift_kv4_paged_write(k[:2 * PAGE - 32], v[:2 * PAGE - 32], near, ints([0, 2 * PAGE - 32]), ints([0]))
    assert torch.equal(pages.pool, near.pool)
    K, V = (torch.full((PAGE, 1, D), 7.0, device="cuda") for _ in range(2))
    qift.qift_kv4_paged_read(pages, ints([0, PAGE]), ints([last]), PAGE, K=K, V=V)
    assert (K[-32:] == 7).all() and torch.equal(K[:-32], qift.qift_kv4_paged_read(near, ints([0, PAGE - 32]), ints([PAGE]), PAGE - 32)[0])
    q, qn = values(702, (n, 4, D), dtype)
    got = qift.qift_kv4_paged_attention(q, pages, ints([0, n]), ints([end - n])).float().cpu().numpy()
    here = end - n - last + PAGE                                                       # the same place in the near cache
    rows = min(n, 2 * PAGE - 32 - here)                                                # drafted tokens that have a position
    pool = near.pool.cpu().numpy()
    want, limit = limits.attention(qn[:rows], pool, np.array([[1, 0]]), PAGE, [0, rows], [here], None, 0, None, dtype == "f32")
    assert (np.linalg.norm(got[:rows] - want, axis=-1) <= limit).all()
    keep = torch.zeros(n, dtype=torch.int32, device="cuda")
    if n > 4:
        keep[:2] = ints([1, 3])
        for p, f in ((pages, end - n), (near, here)):
            qift.qift_kv4_paged_keep(p, ints([0, n]), ints([f]), keep, ints([0, 2]))
        assert torch.equal(pages.pool, near.pool)
    ok()

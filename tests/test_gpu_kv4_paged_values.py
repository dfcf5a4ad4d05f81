"""Paged KV4 attention and cache: values that are no numbers, scales that differ by many orders, extreme clipping ratios, and the error of
each row as a whole against 64 bits."""
import numpy as np
import pytest
import torch

import paged_limits as limits
import paper_2606_02823_b200 as qift
from test_gpu_kv4_paged import D, DTYPES, Batch, dev, filled, ints, ok, trees, values

pytestmark = pytest.mark.gpu
# rows of a request: with four query heads a KV head they make tiles of 8, 16 and 128 rows (bf16; fp32 always 8)
WIDTHS = [1, 6, 60]


def within(got, want, limit, rows=slice(None), heads=slice(None)):
    err = np.linalg.norm(got.float().cpu().numpy().astype(np.float64) - want, axis=-1)[rows, heads]
    assert (err <= limit[rows, heads]).all(), (err / limit[rows, heads]).max()


def check(b, q, qn, dtype, mask=None, **kw):
    got = qift.qift_kv4_paged_attention(q, b.pages, b.rs, b.f, mask=None if mask is None else dev(mask), **kw)
    want, limit = limits.attention(qn, b.pool(), b.table, b.page, b.row_start, b.first, mask, kw.get("q_had_block", 0), kw.get("scale"), dtype == "f32")
    n = int(b.row_start[-1])
    within(got[:n], want[:n], limit[:n])
    ok()
    return got


# ------------------------------------------------------------------------------------------------------- no numbers
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", WIDTHS)
@pytest.mark.parametrize("first", [[2000, 40], [3, 0]])
def test_a_query_row_that_is_no_number_gives_no_number(first, n, dtype):
    """By the definition every score of such a row is NaN, and so is the row, however its tokens are dealt to the GPU."""
    b = filled(500, [n, n], first, 2, 32)
    q, qn = values(510, (2 * n, 8, D), dtype)
    bad = np.zeros((2 * n, 8), bool)
    q[0, 1], q[n, 3], q[2 * n - 1, 6, 9], q[n - 1, 7, 5] = float("nan"), float("inf"), float("nan"), float("-inf")
    bad[0, 1] = bad[n, 3] = bad[2 * n - 1, 6] = bad[n - 1, 7] = True
    for had in (0, 128):
        b2 = filled(500, [n, n], first, 2, 32, had=had)
        got = qift.qift_kv4_paged_attention(q, b2.pages, b2.rs, b2.f, q_had_block=had)
        isnan = torch.isnan(got).cpu().numpy()
        assert isnan[bad].all() and not isnan[~bad].any()
        want, limit = limits.attention(qn, b2.pool(), b2.table, 32, b2.row_start, b2.first, None, had, None, dtype == "f32")
        err = np.linalg.norm(got.float().cpu().numpy() - want, axis=-1)
        assert (err <= limit)[~bad].all()
    ok()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", WIDTHS)
@pytest.mark.parametrize("where", ["key", "value"])
def test_a_cached_token_that_is_no_number_reaches_the_rows_that_see_it(where, n, dtype):
    """Also where it is the only token of its block that a row sees (a piece of its own)."""
    rows, first = [n, n], [1984, 64]                                                  # the drafted tokens begin a block
    b = filled(520, rows, first, 2, 32)
    K, V = qift.qift_kv4_paged_read(b.pages, b.rs, b.f, 2 * n)
    x = torch.zeros((2 * n, 2, D), device="cuda")
    x[0, 0], x[n, 1] = float("nan"), float("inf")     # the quantizer holds the NaN as zeros, the infinities with a scale of infinity
    qift.qift_kv4_paged_write(*((K + x, V) if where == "key" else (K, V + x)), b.pages, b.rs, b.f)
    mask = np.tile(trees(9, [n], 2), (2, 1))                                          # everyone descends from drafted token 0
    q, qn = values(530, (2 * n, 8, D), dtype)
    got = qift.qift_kv4_paged_attention(q, b.pages, b.rs, b.f, mask=dev(mask))
    want = limits.attention(np.zeros_like(qn), b.pool(), b.table, 32, b.row_start, b.first, mask)[0]
    bad = np.isnan(want).all(axis=-1)
    assert bad[n:, 4:].all() and not bad[n:, :4].any() and not bad[:n, 4:].any()
    isnan = torch.isnan(got).cpu().numpy()
    assert isnan[bad].all() and not isnan[~bad].any()
    ok()

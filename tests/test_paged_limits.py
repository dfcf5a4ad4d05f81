"""The limits of the paged attention's tests see what they are there to see (CPU): one block of 32 tokens left out of a row."""
import numpy as np
import pytest

import paged_limits as limits
import paged_ref as ref

D = 128


@pytest.mark.parametrize("fp32", [True, False])
@pytest.mark.parametrize("tokens", [100, 1000, 9000, 40000])
def test_a_block_left_out_exceeds_the_limit(fp32, tokens):
    rng = np.random.default_rng(tokens)
    k, v, q = rng.standard_normal((tokens, D)), rng.standard_normal((tokens, D)), rng.standard_normal((1, D)) * 1.2
    seen = np.ones((1, tokens), bool)
    scales = (v.max(1) - v.min(1)) / 15
    want, limit = limits.one_head(q, k, v, seen, D ** -0.5, fp32, scales)
    for b in range(0, tokens - 31, max(32, tokens // 1600 * 32)):
        without = seen.copy()
        without[:, b:b + 32] = False
        got = limits.one_head(q, k, v, without, D ** -0.5, fp32)[0]
        assert np.linalg.norm(got - want) > 1.5 * limit[0]
    assert limit[0] < 0.02 * np.linalg.norm(want)


def test_the_two_plain_forms_agree():
    rng = np.random.default_rng(3)
    pool = rng.integers(0, 256, (5, 2, 2 * ref.BLOCK), dtype=np.uint8)
    blocks = pool.reshape(5, 2, 2, ref.BLOCK)
    blocks[..., 4096:4352] = np.ascontiguousarray(rng.random((5, 2, 2, 64)).astype(np.float32)).view(np.uint8)
    blocks[..., 4352:] &= 15
    table, rs, first = np.array([[3, 0, -1], [2, 9, 4]]), [0, 9, 40], [70, 95]
    q = rng.standard_normal((42, 4, D)) * 0.1
    mask = np.concatenate([ref.tree_mask([-1] + [i // 2 for i in range(8)], 1), ref.tree_mask([-1] + [i // 3 for i in range(30)], 1), np.zeros((2, 1), np.int32)])
    for m in (None, mask):
        a = ref.attention(q, pool, table, 64, rs, first, m, 16, 0.2)[0]
        b = limits.attention(q, pool, table, 64, rs, first, m, 16, 0.2)[0]
        assert np.allclose(a, b, rtol=1e-11, atol=1e-12)

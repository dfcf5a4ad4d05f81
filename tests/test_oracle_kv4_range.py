"""The oracle's KV4 quantizer at clipping ratios so small that quotients pass 32-bit integers: end codes."""
import numpy as np
import pytest

import oracle


@pytest.mark.parametrize("clip", [1e-6, 1e-9, 1e-12, 1e-20])
def test_quotients_of_any_size_give_the_end_codes(clip):
    x = np.random.default_rng(1).standard_normal((16, 64)).astype(np.float32)
    x[:4], x[4:8] = np.abs(x[:4]), -np.abs(x[4:8])
    x[:, ::5] = 0.0
    codes, s, z = oracle.kv4_quantize(x, 0, clip)
    want = np.where(x > 0, 15, np.where(x < 0, 0, z[:, None])).astype(np.uint8)
    assert np.array_equal(codes, want)

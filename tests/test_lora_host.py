"""CPU-side checks of the adapters: sizes whose index arithmetic would pass 32 bits are refused before any launch."""
import os

import pytest

import paper_2606_02823_b200 as qift
from paper_2606_02823_b200 import binding

P = 4096      # an address that is never dereferenced


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2606_02823_b200 import build
        build.build()
    return qift.lib()


def lora(L, M=4, N=64, K=64, rank=16, wsb=0):
    return L.qift_lora_linear(P, 0, P, P, P, 3, rank, M, N, K, P, P, 2, P, P, P, wsb, None)


def test_sizes_next_to_32_bits(L):
    top, edge = 2 ** 31 - 8, 2 ** 31 - 2 ** 20
    for bad in (dict(N=top), dict(K=top), dict(N=edge + 8), dict(K=edge + 8), dict(M=2 ** 31 - 255), dict(M=2 ** 31 - 1)):
        assert lora(L, **bad) == qift.ERR_UNSUPPORTED_SHAPE
    for good in (dict(N=edge), dict(K=edge), dict(M=2 ** 31 - 256)):
        assert lora(L, **good) == qift.ERR_WORKSPACE                                  # past the shapes, to the workspace of 0 bytes
    assert qift.qift_lora_workspace_bytes(4, 16, top) == 0 and qift.qift_lora_workspace_bytes(2 ** 31 - 1, 16, 64) == 0
    assert qift.qift_lora_workspace_bytes(4, 136, 64) == 0
    assert qift.qift_lora_workspace_bytes(4, 16, edge) == 16 * 4 * 16 * 4 and qift.qift_lora_workspace_bytes(2 ** 31 - 256, 128, 64) == (2 ** 31 - 256) * 512


def slices(N, K, items, sms=148):
    """Columns of a CTA of the second kernel and k of one of the first, as the launch sizes them; every sum on the way is 32-bit there."""
    n = min(-(-4 * sms // items), fits(N + 255) // 256)
    width = (N + n - 1) // n + 255 >> 8 << 8
    splits = max(1, min(16, fits(K + 511) // 512, -(-2 * sms // items)))
    depth = fits(fits(K + splits - 1) // splits + 63) & ~63
    return fits(width), fits(depth)


def fits(x):
    assert 0 <= x < 2 ** 31
    return x


@pytest.mark.parametrize("items", [1, 2, 3, 7, 100, 591, 592, 10000])
def test_the_last_indexes_fit(items):
    edge = 2 ** 31 - 2 ** 20
    for size in (edge, edge - 8, edge - 1000):
        width, depth = slices(size, size, items)
        fits(((size - 1) // width + 1) * width + 4096)                                 # an end, and a few steps beyond it
        fits(((size - 1) // depth + 1) * depth + 4096)

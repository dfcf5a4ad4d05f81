"""Gates far below zero: h fades out with exp(z), it does not stop at 2^-126."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_02823_b200 as qift

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
K = 64


def one_code(value):
    """64 channels whose codes all stand for `value`."""
    table = list(oracle.level_table(qift.SYM))
    return torch.from_numpy(oracle.pack(np.full((64, K), table.index(value), np.uint8), qift.SYM).view(np.int32).ravel()).cuda()


@pytest.mark.parametrize("M", [1, 7, 12, 40, 200, "levels"])
@pytest.mark.parametrize("act, gates", [(qift.ACT_SILU, np.linspace(-102.0, -80.0, 64)), (qift.ACT_GELU_TANH, np.linspace(-10.6, -9.4, 64))])
def test_far_negative_gates(M, act, gates):
    """Gates of these values beside 2^60: the sums are -64 and 64, scales the rest, so g and u are the scales to a rounding each.
    exp within 2 ulp (4 U) and its argument's roundings (GELU: six, 6 |z| U), the two sums and products around the quotient, at most three (3 U),
    the quotient within 2 ulp (4 U); e below 2^-126 is a multiple of 2^-149, off by 2 of them at most, times |g u|."""
    rows = qift.qift_gated_levels_min_rows() if M == "levels" else M
    q = torch.ones((rows, K), dtype=torch.int8, device="cuda")
    s_a = torch.ones(rows, device="cuda")
    s_g, s_u = torch.from_numpy((gates / -64).astype(np.float32)).cuda(), torch.full((64,), 2.0 ** 54, device="cuda")
    h = qift.qift_gated_linear(q, s_a, (one_code(-1), s_g), (one_code(1), s_u), qift.SYM, activation=act).double()
    g = (-64.0 * s_g.double()).float().double()
    z = g if act == qift.ACT_SILU else 2 * np.sqrt(2 / np.pi) * (g + 0.044715 * g ** 3)
    want = g * torch.sigmoid(z) * 2.0 ** 60
    bound = want.abs() * (11 * U + (0 if act == qift.ACT_SILU else 6 * U * z.abs())) + g.abs() * 2.0 ** 60 * 2.0 ** -148
    assert (want.abs() > 2.0 ** -100).any() and torch.equal(h, h[:1].expand_as(h))
    assert ((h[0] - want).abs() <= bound).all(), ((h[0] - want).abs() / bound).max()

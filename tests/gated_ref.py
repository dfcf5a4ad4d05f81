"""The gated half of a feed-forward block in 64 bits, and how far fp32 may be from it."""
import numpy as np
import torch

import oracle
import paper_2606_02823_b200 as qift

LEVELS = {"mnz": qift.MNZ, "pot": qift.POT, "sym": qift.SYM, "int4": qift.INT4, "int3": qift.INT3}
U = 2.0 ** -24


class Case:
    """Random codes, activations and scales of a call; everything of one seed."""

    def __init__(self, seed, M, N, K, levels, extreme=False):
        r = np.random.default_rng(seed)
        self.M, self.N, self.K, self.lv = M, N, K, LEVELS[levels]
        table = np.array(oracle.level_table(self.lv), np.int64)
        self.weights, self.values = [], []
        for _ in range(2):
            codes = r.integers(0, oracle.num_codes(self.lv), (N, K), dtype=np.uint8)
            packed = torch.from_numpy(oracle.pack(codes, self.lv).view(np.int32).ravel()).cuda()
            top = 30.0 if extreme else 1.0
            s_n = torch.from_numpy(((r.random(N) + 0.5) * top / (4.6 * np.sqrt(K) * np.sqrt((table ** 2).mean()))).astype(np.float32)).cuda()
            self.weights.append((packed, s_n))
            self.values.append(torch.from_numpy(table[codes].astype(np.float32)).cuda())
        self.q = torch.from_numpy(r.integers(-8, 8, (M, K)).astype(np.int8)).cuda()
        self.s = torch.from_numpy((r.random(M) + 0.5).astype(np.float32)).cuda()

    def sums(self):
        """The integer products, exactly."""
        return [torch.matmul(self.q.double(), v.double().T).to(torch.int32) for v in self.values]

    def check(self, h, accs=None, act=qift.ACT_SILU, sums=None, s=None):
        want = sums if sums is not None else self.sums()
        if accs is not None:
            for a, b in zip(accs, want):
                assert torch.equal(a, b)
        check(h, want, self.s if s is None else s, [w[1] for w in self.weights], act)


def check(h, sums, s_a, s_n, act):
    """g and u are two rounded multiplies of the exact sums.  From there on, a unit in the last place being 2 U: exp within 2 ulp, of which the
    quotient passes on at most all (4 U), the sum one rounding (U), the quotient, by way of a reciprocal, within 2 ulp (4 U), the last product one
    rounding (U): 10 U of h.  The GELU's argument z takes six roundings, 6 |z| U of exp(-z), of which the quotient passes on sigmoid(-z).
    Where exp(-z) passes the range, or the quotient is denormal, 2^-126 of the rest."""
    g, u = (a.float() * s_a[:, None] * s for a, s in zip(sums, s_n))
    g, u = g.double(), u.double()
    z = g if act == qift.ACT_SILU else 2 * np.sqrt(2 / np.pi) * (g + 0.044715 * g ** 3)
    want = g * torch.sigmoid(z) * u
    off = 10 * U + (6 * U * z.abs() * torch.sigmoid(-z) if act != qift.ACT_SILU else 0)
    bound = want.abs() * off + (g * u).abs() * 2.0 ** -126 + (1 + u.abs()) * 2.0 ** -148
    if h.dtype == torch.bfloat16:
        bound = bound + (want.abs() + bound) * 2.0 ** -8
    d = (h.double() - want).abs()
    assert (d <= bound).all(), float((d / bound).max())

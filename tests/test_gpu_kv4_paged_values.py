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


# -------------------------------------------------------------------------------------- scales that differ by many orders
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [4, 12, 60])
@pytest.mark.parametrize("factor", [1e6, 1e10, 1e20, 1e30])
def test_large_values_leave_the_rows_that_do_not_see_them(factor, n, dtype):
    rows, first = [n, n], [75, 300]
    b = filled(540, rows, first, 2, 32)
    mask = trees(9, rows, 2)
    K, V = qift.qift_kv4_paged_read(b.pages, b.rs, b.f, 2 * n)
    V[1] *= factor                                                                    # drafted token 1 of request 0, 2 of request 1
    V[n + 2] *= -factor
    qift.qift_kv4_paged_write(K, V, b.pages, b.rs, b.f)
    q, qn = values(550, (2 * n, 8, D), dtype)
    sees = np.array([(mask[i, 0] >> (1 if i < n else 2)) & 1 for i in range(2 * n)], bool)
    assert sees.any() and not sees.all()
    check(b, q, qn, dtype, mask)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", WIDTHS)
@pytest.mark.parametrize("strength,factor", [(2.0, 1e6), (4.0, 1e10), (16.0, 1e30)])
def test_large_values_of_tokens_that_hardly_count(strength, factor, n, dtype):
    """Tokens that every row sees, with values so large and weights so small that their product is nothing, or of the others' size."""
    rows, first = [n, n], [400, 1000]
    b = filled(560, rows, first, 2, 32, had=0)
    w = torch.ones(D, device="cuda")
    w[::2] = -1.0
    at = [[33, 200], [0, 999]]
    for r, where in enumerate(at):
        for pos in where:                                                             # one token of request r
            K = (-strength * w).expand(1, 2, D).contiguous()
            V = values(570 + pos, (1, 2, D), "f32", scale=factor)[0]
            qift.qift_kv4_paged_write(K, V, b.pages, ints([0, 1, 1] if r == 0 else [0, 0, 1]), ints([pos, pos]))
    q, _ = values(580, (2 * n, 8, D), "f32", scale=0.5)
    q = (q + strength * w / 2).to(DTYPES[dtype])
    check(b, q, q.float().cpu().numpy(), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", WIDTHS)
@pytest.mark.parametrize("size", [1e-6, 1e-9, 1e-20])
def test_zero_vectors_among_small_values(size, n, dtype):
    """A vector of zeros is held with scale 1, whatever the others' scales are."""
    rows, first = [n, n], [200, 130]
    b = Batch(590, rows, first, 2, 64)
    cut = np.concatenate([[0], np.cumsum([f + n for f in first])])
    k = values(591, (int(cut[-1]), 2, D), "f32", 0.1)[0]
    v = values(592, (int(cut[-1]), 2, D), "f32", -0.1)[0] * size
    v[3::7] = 0.0
    v[int(cut[1]) - 1, 1] = 0.0
    qift.qift_kv4_paged_write(k, v, b.pages, ints(cut), ints([0, 0]))
    q, qn = values(593, (2 * n, 8, D), dtype)
    check(b, q, qn, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", WIDTHS)
@pytest.mark.parametrize("size", [1e24, 1e-24, 1e32, 3e-25])
def test_values_of_any_size(size, n, dtype):
    rows, first = [n, n], [200, 1300]
    b = Batch(600, rows, first, 2, 64)
    cut = np.concatenate([[0], np.cumsum([f + n for f in first])])
    k = values(601, (int(cut[-1]), 2, D), "f32", 0.1)[0]
    v = values(602, (int(cut[-1]), 2, D), "f32", -0.1)[0] * size
    qift.qift_kv4_paged_write(k, v, b.pages, ints(cut), ints([0, 0]))
    q, qn = values(603, (2 * n, 8, D), dtype)
    check(b, q, qn, dtype)


# ------------------------------------------------------------------------------------------------- every block counts
@pytest.mark.parametrize("rows,first", [([1], [1000]), ([64, 20], [700, 31]), ([1], [40000]), ([64, 40, 7], [5000, 64, 9000]), ([13, 0, 4, 7], [95, 20, 0, 257]),
                                        ([1] * 20 + [64], list(range(900, 920)) + [2000])])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_error_of_each_row(rows, first, dtype):
    """The last batch holds a wide tree beside single tokens."""
    b = filled(610, rows, first, 2, 64)
    q, qn = values(620, (b.total, 8, D), dtype, scale=1.2)
    check(b, q, qn, dtype, trees(11, rows, 2), q_had_block=128)


@pytest.mark.parametrize("Hq,H", [(64, 1), (66, 2), (5, 1)])
@pytest.mark.parametrize("rows,first", [([1], [300]), ([1, 1, 3], [0, 2000, 65])])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_query_heads_and_odd_numbers_of_them(rows, first, Hq, H, dtype):
    """Also single tokens reach the widest tiles: 64 query heads a KV head."""
    b = filled(625, rows, first, H, 32, pad_rows=1)
    q, qn = values(626, (b.total, Hq, D), dtype, scale=1.2)
    check(b, q, qn, dtype, q_had_block=128)


@pytest.mark.parametrize("rows,first", [([700], [0]), ([300, 1, 1, 90], [0, 500, 31, 1000])])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_causal_runs(rows, first, dtype):
    """Prompts over the paged cache, alone and beside single tokens."""
    b = filled(630, rows, first, 2, 64)
    q, qn = values(640, (b.total, 8, D), dtype, scale=1.2)
    check(b, q, qn, dtype, q_had_block=128)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", WIDTHS)
@pytest.mark.parametrize("tokens", [2048, 2100])
def test_rows_that_look_at_one_token_find_it(tokens, n, dtype):
    """Each row's query points at one token, block after block: whatever run, stage or piece a block falls into, it is there."""
    blocks = -(-tokens // 32)
    R = -(-blocks // n)
    b = filled(650, [n], [tokens], 2, 64, had=0)
    b.table = np.repeat(b.table, R, 0)                                                # the same pages for every request
    pages = qift.Kv4Pages(b.pages.pool, ints(b.table), 64)
    K, V = qift.qift_kv4_paged_read(b.pages, ints([0, tokens]), ints([0]), tokens)
    at = np.array([min(tokens - 1, 32 * (i % blocks) + 7 * i % 32) for i in range(R * n)])
    q = (K[torch.from_numpy(at).cuda()].repeat_interleave(4, 1) * 3.0).to(DTYPES[dtype])
    row_start, first = np.arange(R + 1) * n, [tokens] * R
    got = qift.qift_kv4_paged_attention(q, pages, ints(row_start), ints(first))
    want, limit = limits.attention(q.float().cpu().numpy(), b.pool(), b.table, 64, row_start, first, None, 0, None, dtype == "f32")
    within(got, want, limit)
    token = V[torch.from_numpy(at).cuda()].repeat_interleave(4, 1).cpu().numpy()
    assert (np.linalg.norm(want - token, axis=-1) < 0.1 * np.linalg.norm(token, axis=-1)).mean() > 0.9       # the reference's own rows
    ok()


# ------------------------------------------------------------------------------------------------- clipping ratios
def quantized(x, clip):
    """The definition, each step rounded to fp32 once; codes are clamped, however large the quotient."""
    f = np.float32
    lo, hi = (np.minimum(x.min(-1), f(0)) * f(clip)).astype(f), (np.maximum(x.max(-1), f(0)) * f(clip)).astype(f)
    s = ((hi - lo).astype(f) / f(15)).astype(f)
    z = np.rint((-lo / s).astype(f))
    return np.clip(np.rint((x / s[..., None]).astype(f)).astype(np.float64) + z[..., None], 0, 15).astype(np.uint8), s, z


def clip_rows():
    x = values(660, (64, 1, D), "f32")[1].copy()
    x[:8] = np.abs(x[:8])                                                             # one-sided ranges
    x[8:16] = -np.abs(x[8:16])
    x[16, 0, :2], x[17, 0, :2] = (-1.0, -0.9), (1.0, 0.9)
    return x


@pytest.mark.parametrize("clip", [1e-3, 1e-5, 3e-6, 1.2e-6, 1e-6, 8e-7, 6e-7, 5e-7, 3e-7, 1e-7])
def test_write_with_small_clipping_ratios(clip):
    x = clip_rows()
    b = Batch(670, [64], [0], 1, 64)
    qift.qift_kv4_paged_write(torch.from_numpy(x).cuda(), torch.from_numpy(x).cuda(), b.pages, b.rs, b.f, clip_ratio=clip)
    held = limits.ref.cached(b.pool(), b.table, 64, 0, 64)
    code, s, z = quantized(x, clip)
    for got in (held[:3], held[3:]):
        assert np.array_equal(got[1], s) and np.array_equal(got[2], z.astype(np.uint8)) and np.array_equal(got[0], code)
    ok()


# --------------------------------------------------------------------------------- quotients beyond 32-bit integers
@pytest.mark.parametrize("clip", [1e-9, 2e-10, 1e-12, 1e-20])
def test_quotients_beyond_32_bit_integers(clip):
    """All of a vector but its zeros is far outside the range: end codes, in the paged cache and in the contiguous one."""
    x = clip_rows()
    x[20:30, 0, ::3] = 0.0
    X = torch.from_numpy(x).cuda()
    code, s, z = quantized(x, clip)
    assert set(np.unique(code)) > {0, 15}
    b = Batch(680, [64], [0], 1, 64)
    qift.qift_kv4_paged_write(X, X, b.pages, b.rs, b.f, clip_ratio=clip)
    held = limits.ref.cached(b.pool(), b.table, 64, 0, 64)
    for got in (held[:3], held[3:]):
        assert np.array_equal(got[1], s) and np.array_equal(got[2], z.astype(np.uint8)) and np.array_equal(got[0], code)
    one = qift.Kv4Cache(1, 64)
    qift.qift_kv4_quantize(X, one, clip_ratio=clip)
    packed = code[:, 0, 0::2] | code[:, 0, 1::2] << 4
    assert np.array_equal(one.codes.cpu().numpy()[0], packed) and np.array_equal(one.scale.cpu().numpy()[0], s[:, 0])
    ok()


# ------------------------------------------------------------------------------------------------- scales all over
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", WIDTHS)
@pytest.mark.parametrize("orders", [3, 6, 12, 40])
def test_scales_that_differ_from_token_to_token(orders, n, dtype):
    """Values of 2^-orders to 2^orders side by side, vectors of zeros among them."""
    rows, first = [n, n], [700, 1300]
    b = Batch(720, rows, first, 2, 64)
    cut = np.concatenate([[0], np.cumsum([f + n for f in first])])
    k = values(721, (int(cut[-1]), 2, D), "f32", 0.1)[0]
    v = values(722, (int(cut[-1]), 2, D), "f32")[0]
    u = torch.from_numpy(np.random.default_rng(5).random((int(cut[-1]), 2, 1)).astype(np.float32)).cuda()
    v *= torch.exp2((2 * u - 1) * orders) * (u > 0.1)
    qift.qift_kv4_paged_write(k, v, b.pages, ints(cut), ints([0, 0]))
    q, qn = values(723, (2 * n, 8, D), dtype)
    check(b, q, qn, dtype, trees(13, rows, 2))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", WIDTHS)
@pytest.mark.parametrize("strength", [1.0, 2.0, 3.0])
def test_zero_vectors_that_take_the_weight(strength, n, dtype):
    """A row looks at tokens whose values are zeros; its result is what little the others have left (about e^-11, -23, -34 of them)."""
    rows, first = [n, n], [200, 1300]
    b = Batch(730, rows, first, 2, 64)
    cut = np.concatenate([[0], np.cumsum([f + n for f in first])])
    k = values(731, (int(cut[-1]), 2, D), "f32", scale=0.3)[0]
    v = values(732, (int(cut[-1]), 2, D), "f32")[0]
    w = torch.ones(D, device="cuda")
    w[::2] = -1.0
    for at in (0, 70, int(cut[1]), int(cut[1]) + 640, int(cut[1]) + 1299):
        k[at], v[at] = w, 0.0
    qift.qift_kv4_paged_write(k, v, b.pages, ints(cut), ints([0, 0]))
    q = (values(733, (2 * n, 8, D), "f32", scale=0.3)[0] + strength * w).to(DTYPES[dtype])
    check(b, q, q.float().cpu().numpy(), dtype)

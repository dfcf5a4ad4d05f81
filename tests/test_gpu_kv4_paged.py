"""Paged KV4 cache on the GPU: the write bit-exactly against the oracle's quantizer, the read, the moves of accepted tokens, and
the attention of drafted trees against 64 bits."""
import numpy as np
import pytest
import torch

import oracle
import paged_ref as ref
import synth
import paper_2606_02823_b200 as qift

pytestmark = pytest.mark.gpu
D = 128
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def ints(v):
    return torch.tensor(np.asarray(v).tolist(), dtype=torch.int32, device="cuda")


def values(seed, shape, dtype, shift=0.0, scale=1.0):
    x = torch.from_numpy((synth.normal(seed, 3, shape) * scale + shift).astype(np.float32)).cuda().to(DTYPES[dtype])
    return x, x.float().cpu().numpy()


class Batch:
    """A pool filled with the byte 0xA5, shuffled pages, ragged requests."""

    def __init__(self, seed, rows, first, H, page, pad_rows=0, spare_pages=2):
        self.rows, self.first, self.H, self.page = rows, first, H, page
        need = [-(-max(0, n + f) // page) for n, f in zip(rows, first)]
        order = np.random.default_rng(seed).permutation(sum(need) + spare_pages)
        self.table = np.full((len(rows), max(need + [1]) + 1), -1, np.int64)
        at = 0
        for r, n in enumerate(need):
            self.table[r, :n] = order[at:at + n]
            at += n
        self.row_start = np.concatenate([[0], np.cumsum(rows)])
        self.total = int(self.row_start[-1]) + pad_rows
        self.pages = qift.Kv4Pages.empty(sum(need) + spare_pages, H, page, ints(self.table))
        self.pages.pool.fill_(0xA5)
        self.rs, self.f = ints(self.row_start), ints(first)

    def pool(self):
        return self.pages.pool.cpu().numpy()

    def places(self):
        """(row, request, position) of every row."""
        return [(int(self.row_start[r]) + i, r, f + i) for r, (n, f) in enumerate(zip(self.rows, self.first)) for i in range(n)]


def ok():
    rc, detail = qift.qift_device_status()
    assert rc == qift.OK, (rc, detail)


BATCHES = [([1], [0]), ([5, 0, 1, 37], [0, 9, 31, 30]), ([64, 33, 32], [32, 64, 5]), ([100], [63]), ([1] * 9, list(range(60, 69)))]


@pytest.mark.parametrize("rows,first", BATCHES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("had", [(128, 0), (0, 16)])
def test_write_is_bit_exact_and_touches_nothing_else(rows, first, dtype, had):
    H, page = 3, 64
    b = Batch(1, rows, first, H, page, pad_rows=2)
    before = b.pool()
    K, kn = values(100, (b.total, H, D), dtype, 0.2)
    V, vn = values(101, (b.total, H, D), dtype, -0.3)
    K[b.total - 2:], V[b.total - 2:] = float("nan"), float("inf")                  # rows of nobody
    qift.qift_kv4_paged_write(K, V, b.pages, b.rs, b.f, k_had_block=had[0], v_had_block=had[1])
    after = b.pool()
    want = before.copy()
    n = int(b.row_start[-1])
    kc, ks, kz = oracle.kv4_quantize(kn[:n].reshape(n * H, D), had[0], 0.95)
    vc, vs, vz = oracle.kv4_quantize(vn[:n].reshape(n * H, D), had[1], 0.95)
    for row, r, pos in b.places():
        for h in range(H):
            blk = want[b.table[r, pos // page], h].reshape(-1, ref.BLOCK)[pos % page // 32]
            t, i = pos % 32, row * H + h
            for bytes_, shifts, codes in ((ref.KB, ref.KSH, kc), (ref.VB, ref.VSH, vc)):
                blk[bytes_[t]] = 0
                np.bitwise_or.at(blk, bytes_[t], codes[i].astype(np.uint8) << shifts[t].astype(np.uint8))
            blk[4096 + 4 * t:4100 + 4 * t] = ks[i:i + 1].view(np.uint8)
            blk[4224 + 4 * t:4228 + 4 * t] = vs[i:i + 1].view(np.uint8)
            blk[4352 + t], blk[4384 + t] = int(kz[i]), int(vz[i])
    assert np.array_equal(after, want)
    ok()


def test_write_codes_next_to_a_border_and_odd_rows():
    """Rows where x / s falls on halves (equal ends of the range put z on one), constant rows, zeros, tiny and huge values."""
    x = np.zeros((64, 1, D), np.float32)
    grid = np.arange(D) / 127.0
    for i in range(24):
        x[i, 0] = (grid * 2 - 1) * (i + 1) / 8.0                                    # symmetric: -lo / s = 7.5
    for i in range(24, 40):
        x[i, 0] = ((np.arange(D) % 31) - 15) * 0.5 * (1.0 + i / 64.0)               # multiples of half a step
    x[40], x[41, 0, 7], x[42, 0, :3] = 3.0, 1e-30, (-2e30, 1e30, 5.0)
    x[43, 0, 0], x[44, 0, :2] = 1e-44, (3e38, -3e38)
    x[45:] = synth.normal(5, 3, (19, 1, D)) * 1e-3
    for dtype in ("f32", "bf16"):
        for clip in (0.95, 1.0, 0.03):
            b = Batch(2, [64], [0], 1, 64)
            X = torch.from_numpy(x).cuda().to(DTYPES[dtype])
            qift.qift_kv4_paged_write(X, X, b.pages, b.rs, b.f, clip_ratio=clip)
            code, s, z = oracle.kv4_quantize(X.float().cpu().numpy().reshape(64, D), 0, clip)
            kc, ks, kz, vc, vs, vz = ref.cached(b.pool(), b.table, 64, 0, 64)
            # row 43's range, 1e-44, is below 15 * 2^-149 = 2.1e-44: its scale rounds to 0 and the oracle's zero-point is 0 / 0; the
            # cache holds such a row as zeros with scale 1
            if s[43] == 0.0:
                code[43], s[43], z[43] = 0, 1.0, 0.0
            for c_, s_, z_ in ((kc, ks, kz), (vc, vs, vz)):
                assert np.array_equal(c_[:, 0], code) and np.array_equal(s_[:, 0].view(np.uint32), s.view(np.uint32))
                assert np.array_equal(z_[:, 0], z.astype(np.uint8))


def test_rows_may_be_slices_of_a_fused_projection():
    Hq, H = 6, 2
    b = Batch(3, [7, 40], [3, 0], H, 32)
    wide = values(110, (b.total, (Hq + 2 * H) * D), "bf16")[0]
    q, k, v = (t.view(b.total, -1, D) for t in (wide[:, :Hq * D], wide[:, Hq * D:(Hq + H) * D], wide[:, (Hq + H) * D:]))
    assert not k.is_contiguous()
    qift.qift_kv4_paged_write(k, v, b.pages, b.rs, b.f, k_had_block=128)
    pool = b.pages.pool.clone()
    b.pages.pool.fill_(0xA5)
    qift.qift_kv4_paged_write(k.contiguous(), v.contiguous(), b.pages, b.rs, b.f, k_had_block=128)
    assert torch.equal(pool, b.pages.pool)
    a = qift.qift_kv4_paged_attention(q, b.pages, b.rs, b.f, q_had_block=128)
    assert torch.equal(a, qift.qift_kv4_paged_attention(q.contiguous(), b.pages, b.rs, b.f, q_had_block=128))
    out = torch.zeros((b.total, 3 * H, D), device="cuda")                             # read back into slices
    qift.qift_kv4_paged_read(b.pages, b.rs, b.f, b.total, K=out[:, :H], V=out[:, 2 * H:], k_had_block=128)
    K, V = qift.qift_kv4_paged_read(b.pages, b.rs, b.f, b.total, k_had_block=128)
    assert torch.equal(out[:, :H], K) and torch.equal(out[:, 2 * H:], V) and not out[:, H:2 * H].any()


@pytest.mark.parametrize("rows,first", BATCHES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_read_returns_what_the_cache_holds(rows, first, dtype):
    H, page = 3, 32
    b = Batch(4, rows, first, H, page, pad_rows=1)
    X = values(120, (b.total, H, D), "f32", 0.1)[0]
    Y = values(121, (b.total, H, D), "f32", -0.1)[0]
    qift.qift_kv4_paged_write(X, Y, b.pages, b.rs, b.f)
    K = torch.full((b.total, H, D), 77.0, dtype=DTYPES[dtype], device="cuda")
    V = K.clone()
    qift.qift_kv4_paged_read(b.pages, b.rs, b.f, b.total, K=K, V=V)
    pool = b.pool()
    Kn, Vn = K.float().cpu().numpy(), V.float().cpu().numpy()
    Kr = qift.qift_kv4_paged_read(b.pages, b.rs, b.f, b.total, K=K.clone(), V=V.clone(), k_had_block=128)[0].float().cpu().numpy()
    for r in range(len(rows)):
        parts = ref.cached(pool, b.table, page, r, first[r] + rows[r])
        at = slice(int(b.row_start[r]), int(b.row_start[r + 1]))
        k32, v32 = ((p[1][..., None] * (p[0].astype(np.float32) - p[2].astype(np.float32)[..., None]))[first[r]:] for p in (parts[:3], parts[3:]))
        for got, want in ((Kn[at], k32), (Vn[at], v32)):                              # one product in fp32, then one rounding
            assert np.array_equal(got, torch.from_numpy(want).to(DTYPES[dtype]).float().numpy())
        # rotated back: seven additions and a product, each half a step off at most, on sums that |k| bounds by sqrt(128) max|k|
        want = ref.rotate(k32, 128)
        bound = 9 * 2.0 ** -24 * np.abs(k32).sum(-1, keepdims=True) / np.sqrt(D) * 2 + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0)
        assert (np.abs(Kr[at] - want) <= bound + 1e-30).all()
    assert (Kn[int(b.row_start[-1]):] == 77).all() and (Vn[int(b.row_start[-1]):] == 77).all()
    ok()


def test_pages_that_are_none():
    """Table entries outside the pool, positions before 0 and past the table: nothing is written, read or seen there."""
    H, page = 2, 32
    b = Batch(5, [70, 6], [10, 0], H, page)
    b.table[0, 1] = b.pages.num_pages                                                 # positions 32 .. 63 of request 0
    b.first = [10, -3]
    b.pages.page_table, b.f = ints(b.table), ints(b.first)
    before = b.pool()
    X = values(130, (b.total, H, D), "f32")[0]
    qift.qift_kv4_paged_write(X, X, b.pages, b.rs, b.f)
    pool = b.pool()
    pages_written = {int(b.table[0, 0]), int(b.table[0, 2]), int(b.table[1, 0])}
    for i in range(b.pages.num_pages):
        assert (i in pages_written) == bool((pool[i] != before[i]).any())
    K = torch.full((b.total, H, D), 77.0, device="cuda")
    qift.qift_kv4_paged_read(b.pages, b.rs, b.f, b.total, K=K, V=K.clone())
    left = (K == 77).all(dim=2).all(dim=1).cpu().numpy()
    assert left[22:54].all() and not left[:22].any() and not left[54:70].any()        # rows 22 .. 53 <-> positions 32 .. 63
    assert left[70:73].all() and not left[73:].any()                                  # rows at positions -3 .. -1
    q, qn = values(131, (b.total, H, D), "f32")
    out = qift.qift_kv4_paged_attention(q, b.pages, b.rs, b.f).cpu().numpy()
    want, size, top = ref.attention(qn, pool, b.table, page, b.row_start, b.first)
    assert (np.abs(out - want) <= tolerance("f32", want, size, top, 128)).all()
    ok()


def test_kept_tokens_move_to_the_front():
    H, page = 3, 32
    rows, first = [40, 1, 12, 8, 0, 20], [25, 31, 0, 63, 4, 5]
    b = Batch(6, rows, first, H, page)
    keep = [[0, 3, 4, 9, 17, 18, 30, 31, 33, 39], [0], [], list(range(8)), [], [2, 5, 99, 19]]
    flat = np.zeros(b.total, np.int64)
    for r, k in enumerate(keep):
        flat[b.row_start[r]:b.row_start[r] + len(k)] = k
    kept_start = np.concatenate([[0], np.cumsum([len(k) for k in keep])])
    X = values(140, (b.total, H, D), "f32")[0]
    qift.qift_kv4_paged_write(X, -X, b.pages, b.rs, b.f, k_had_block=128)
    before = b.pool()
    qift.qift_kv4_paged_keep(b.pages, b.rs, b.f, ints(flat), ints(kept_start))
    want = before.copy()
    for r, k in enumerate(keep):
        for i, src in enumerate(k):
            if src >= rows[r]:
                continue                                                              # no such drafted token: nothing moves
            s, d = first[r] + src, first[r] + i
            sb = before[b.table[r, s // page]].reshape(H, -1, ref.BLOCK)[:, s % page // 32]
            db = want[b.table[r, d // page]].reshape(H, -1, ref.BLOCK)[:, d % page // 32]
            db[:, ref.token_bytes(d % 32)] = sb[:, ref.token_bytes(s % 32)]
    assert np.array_equal(b.pool(), want)
    ok()


# ------------------------------------------------------------------------------------------------------- attention
def tolerance(dtype, want, size, top, length):
    """Bounds, worst case.  fp32: a score is a 128-term fp32 dot product of a query held to 2^-22 (two fp16 parts) with exact codes,
    times two fp32 factors and the logarithm's base: off by at most (128 + 16) 2^-24 sum|q k|; exp and the sums of `length` positive
    weights add (length + 32) 2^-24 relative.  Each is a relative error of every weight, at most doubled by the normalisation.
    bf16: the rotated query and the weights are rounded to fp16 (2^-11 each), the result to bf16 (2^-8)."""
    score = (144 * 2.0 ** -24 + (2.0 ** -11 if dtype == "bf16" else 0)) * size
    weight = (length + 32) * 2.0 ** -24 + (2.0 ** -11 if dtype == "bf16" else 0)
    return (2.0 * (np.expm1(score) + weight) * top)[..., None] + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0)


def filled(seed, rows, first, H, page, had=128, pad_rows=0):
    """A batch whose cache holds all positions up to first + rows; slots behind them hold NaN scales and 0xFF codes."""
    b = Batch(seed, rows, first, H, page, pad_rows=pad_rows)
    b.pages.pool.fill_(0xFF)
    lengths = [n + f for n, f in zip(rows, first)]
    cut = np.concatenate([[0], np.cumsum(lengths)])
    k = values(seed + 1, (max(1, int(cut[-1])), H, D), "f32", 0.1)[0]
    v = values(seed + 2, (max(1, int(cut[-1])), H, D), "f32", -0.1)[0]
    k[..., 5] *= 6.0
    qift.qift_kv4_paged_write(k, v, b.pages, ints(cut), ints([0] * len(rows)), k_had_block=had)
    return b


def trees(seed, rows, words):
    rng = np.random.default_rng(seed)
    return np.concatenate([np.zeros((0, words), np.int32)] + [
        ref.tree_mask([-1] + [int(rng.integers(max(0, i - 6), i)) for i in range(1, n)], words) for n in rows if n])


def check(b, q, qn, dtype, mask=None, out=None, **kw):
    m = None if mask is None else dev(mask)
    got = qift.qift_kv4_paged_attention(q, b.pages, b.rs, b.f, mask=m, out=out, **kw)
    want, size, top = ref.attention(qn, b.pool(), b.table, b.page, b.row_start, b.first, mask, kw.get("q_had_block", 0), kw.get("scale"))
    n = int(b.row_start[-1])
    g = got.float().cpu().numpy()
    assert np.isfinite(g[:n]).all()
    length = max(f + r for r, f in zip(b.rows, b.first))
    err, bound = np.abs(g[:n] - want[:n]), tolerance(dtype, want, size, top, length)[:n]
    assert (err <= bound).all(), (err.max(), (err / np.maximum(bound, 1e-30)).max())
    ok()
    return got


# rows and cached tokens before them: one token over nothing, single tokens, small trees, ragged, an empty request, wide trees
SHAPES = [([1], [0]), ([1], [31]), ([1], [1000]), ([1, 1, 1], [0, 64, 333]), ([5], [0]), ([13, 0, 4, 7], [95, 20, 0, 257]), ([3] * 5, [1, 2, 31, 32, 33]),
          ([33], [100]), ([64, 20], [700, 31]), ([130], [65])]


@pytest.mark.parametrize("rows,first", SHAPES)
@pytest.mark.parametrize("Hq,H", [(8, 2), (3, 3), (7, 1)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_of_trees(rows, first, Hq, H, dtype):
    b = filled(200, rows, first, H, 64)
    q, qn = values(210, (b.total, Hq, D), dtype, scale=1.2)
    check(b, q, qn, dtype, trees(7, rows, -(-max(rows) // 32)), q_had_block=128)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("page", [32, 96, 1024])
def test_attention_without_a_mask_other_pages_scale_and_rotation(dtype, page):
    rows, first = [17, 1, 70], [140, 999, 0]
    b = filled(220, rows, first, 2, page, had=16)
    q, qn = values(230, (b.total, 4, D), dtype)
    check(b, q, qn, dtype, None, q_had_block=16, scale=0.125)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [4, 40])
def test_rows_that_see_nothing_and_rows_of_nobody(dtype, n):
    """An empty mask over an empty context gives zeros; drafted tokens beyond the mask's bits are not seen; rows behind the last
    request keep what `out` held."""
    rows, first = [n, n, 2], [0, 50, 0]
    b = filled(240, rows, first, 2, 32, pad_rows=3)
    mask = trees(8, rows, -(-n // 32))
    mask[0] = 0
    mask[n - 1] = 0
    mask[2 * n:] = 0
    mask = np.concatenate([mask, np.full((3, mask.shape[1]), -1, np.int32)])
    q, qn = values(250, (b.total, 8, D), dtype)
    q[-3:] = float("nan")
    out = torch.full((b.total, 8, D), 5.0, dtype=DTYPES[dtype], device="cuda")
    got = check(b, q, qn, dtype, mask, out=out).float().cpu().numpy()
    assert not got[0].any() and not got[n - 1].any() and not got[2 * n:2 * n + 2].any() and got[n].any()
    assert (got[-3:] == 5).all()
    if n == 40:
        check(b, q, qn, dtype, mask[:, :1], out=out)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [[1, 1], [24, 9]])
def test_attention_with_large_and_tiny_values(dtype, rows):
    """Scores dominated by one token, uniform scores, value scales from 1e-20 to 1e6 in one cache."""
    first = [300, 77]
    b = Batch(260, rows, first, 2, 64)
    lengths = [n + f for n, f in zip(rows, first)]
    cut = np.concatenate([[0], np.cumsum(lengths)])
    k = values(261, (int(cut[-1]), 2, D), "f32", 0.1)[0]
    v = values(262, (int(cut[-1]), 2, D), "f32", -0.1)[0]
    big = torch.ones((int(cut[-1]), 1, 1), device="cuda")
    for at, factor in ((5, 1e6), (40, 1e-20), (150, 1e-4), (301, 3e4), (310, 1e5)):
        big[at] = factor
    qift.qift_kv4_paged_write(k, v * big, b.pages, ints(cut), ints([0, 0]))
    q, qn = values(263, (b.total, 4, D), dtype)
    check(b, q, qn, dtype)
    check(b, torch.zeros_like(q), np.zeros_like(qn), dtype)
    peaked = (k[123 % lengths[0]].repeat_interleave(2, 0)[None] * 4.0).expand(b.total, 4, D).contiguous().to(q.dtype)
    check(b, peaked, peaked.float().cpu().numpy(), dtype)
    qift.qift_kv4_paged_write(k, v * 1e-6, b.pages, ints(cut), ints([0, 0]))
    check(b, q, qn, dtype)
    tiny = (q.float() * 1e-12).to(q.dtype)
    check(b, tiny, tiny.float().cpu().numpy(), dtype)


def test_requests_share_pages_and_pages_beyond_four_gigabytes():
    H, page = 8, 1024
    num_pages = (5 << 30) // qift.qift_kv4_page_bytes(page, H)
    table = np.array([[num_pages - 1, num_pages - 2, -1], [num_pages - 1, 3, -1]])     # a common first page
    pool = torch.empty((num_pages, H, page // 32 * ref.BLOCK), dtype=torch.uint8, device="cuda")
    pages = qift.Kv4Pages(pool, ints(table), page)
    k = values(270, (2100, H, D), "bf16", 0.1)[0]
    qift.qift_kv4_paged_write(k[:1100], -k[:1100], pages, ints([0, 1100, 1100]), ints([0, 0]))
    qift.qift_kv4_paged_write(k[1100:], -k[1100:], pages, ints([0, 0, 1000]), ints([0, 1024]))
    K, V = qift.qift_kv4_paged_read(pages, ints([0, 1100, 2100]), ints([0, 1024]), 2100)
    assert (K - k.float()).abs().max() < 0.5 and (V + k.float()).abs().max() < 0.5
    q, qn = values(271, (4, 16, D), "bf16")
    got = qift.qift_kv4_paged_attention(q, pages, ints([0, 2, 4]), ints([1098, 2022])).float().cpu().numpy()
    small = np.stack([pool[int(p)].cpu().numpy() for p in (num_pages - 1, num_pages - 2, 3)])
    want, size, top = ref.attention(qn, small, np.array([[0, 1, -1], [0, 2, -1]]), page, [0, 2, 4], [1098, 2022])
    assert (np.abs(got - want) <= tolerance("bf16", want, size, top, 2024)).all()
    ok()


def test_long_context_and_many_requests():
    rows, first = [2], [40000]
    b = filled(280, rows, first, 1, 128)
    for dtype in ("f32", "bf16"):
        q, qn = values(281, (2, 4, D), dtype)
        check(b, q, qn, dtype, q_had_block=128)
    rng = np.random.default_rng(3)
    rows, first = rng.integers(0, 3, 600).tolist(), rng.integers(0, 70, 600).tolist()
    b = filled(290, rows, first, 1, 32)
    for dtype in ("f32", "bf16"):
        q, qn = values(291, (b.total, 2, D), dtype)
        check(b, q, qn, dtype, q_had_block=128)


# ------------------------------------------------------------------------------------------------- used together
def step(b, k, v, q, mask, keep, kept_start, kept, workspace=None):
    qift.qift_kv4_paged_write(k, v, b.pages, b.rs, b.f, k_had_block=128)
    out = qift.qift_kv4_paged_attention(q, b.pages, b.rs, b.f, mask=mask, q_had_block=128, workspace=workspace)
    qift.qift_kv4_paged_keep(b.pages, b.rs, b.f, keep, kept_start)
    K, V = qift.qift_kv4_paged_read(b.pages, kept_start, b.f, kept, q.dtype, k_had_block=128)
    return out, K, V


def make_step(seed, dtype="bf16"):
    rows, first = [12, 5, 30], [40, 0, 333]
    b = filled(seed, rows, first, 2, 64)
    k = values(seed + 5, (b.total, 2, D), dtype)[0]
    v = values(seed + 6, (b.total, 2, D), dtype)[0]
    q, qn = values(seed + 7, (b.total, 8, D), dtype)
    mask = trees(seed, rows, 1)
    keep = np.zeros(b.total, np.int64)
    keep[:3], keep[12:13], keep[17:21] = [0, 2, 11], [0], [0, 1, 5, 29]
    return b, (k, v, q, dev(mask), ints(keep), ints([0, 3, 4, 8]), 8), qn, mask


def test_a_serving_step_and_the_next_one():
    """Drafts are written, checked and kept; a following token sees exactly the kept ones."""
    b, args, qn, mask = make_step(300)
    k, v = args[0], args[1]
    out, K, V = step(b, *args)
    rows_kept = [0, 2, 11, 12, 17, 18, 22, 46]
    assert (K.float() - k[rows_kept].float()).abs().max() < 0.6 and (V.float() - v[rows_kept].float()).abs().max() < 0.6
    # the attention saw the tree before anything moved: the same from a cache that was only written
    b2, args2, _, _ = make_step(300)
    qift.qift_kv4_paged_write(k, v, b2.pages, b2.rs, b2.f, k_had_block=128)
    check(b2, args2[2], qn, "bf16", mask, q_had_block=128)
    assert torch.equal(out, qift.qift_kv4_paged_attention(args2[2], b2.pages, b2.rs, b2.f, mask=args2[3], q_had_block=128))
    b.rows, b.first = [1, 1, 1], [43, 1, 337]
    b.row_start = np.arange(4)
    b.rs, b.f, b.total = ints(b.row_start), ints(b.first), 3
    nk = values(310, (3, 2, D), "bf16")[0]
    qift.qift_kv4_paged_write(nk, nk, b.pages, b.rs, b.f, k_had_block=128)
    q, qn = values(311, (3, 8, D), "bf16")
    check(b, q, qn, "bf16", q_had_block=128)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_steps_share_a_workspace_and_follow_new_lengths(dtype):
    steps = [make_step(320, dtype), make_step(330, dtype)]
    need = qift.qift_kv4_paged_attention_workspace_bytes(47, 3, 8, 2)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    graphs, outs = [], []
    for b, args, _, _ in steps:
        pool = b.pages.pool.clone()
        want = step(b, *args)                                                         # eager, and a warm-up
        b.pages.pool.copy_(pool)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = step(b, *args, workspace=ws)
        graphs.append(g), outs.append((pool, want, got))
    for _ in range(2):
        for (b, _, _, _), (pool, _, _) in zip(steps, outs):
            b.pages.pool.copy_(pool)
        for g in graphs:
            g.replay()
        for _, want, got in outs:
            assert all(torch.equal(x, y) for x, y in zip(want, got))
    # other contents of the same arrays: shorter contexts, an empty request
    b, args, _, _ = steps[0]
    b.f.copy_(ints([3, 0, 100]))
    b.rs.copy_(ints([0, 12, 12, 47]))
    b.pages.pool.copy_(outs[0][0])
    want = step(b, *args)
    b.pages.pool.copy_(outs[0][0])
    graphs[0].replay()
    assert torch.equal(want[0], outs[0][2][0])


def test_calls_on_two_streams_at_once_do_not_disturb_each_other():
    steps = [make_step(340), make_step(350)]
    pools = [b.pages.pool.clone() for b, _, _, _ in steps]
    wants = []
    for b, args, _, _ in steps:
        wants.append(step(b, *args))
    streams = [torch.cuda.Stream() for _ in steps]
    for _ in range(5):
        for (b, _, _, _), pool in zip(steps, pools):
            b.pages.pool.copy_(pool)
        torch.cuda.synchronize()
        gots = []
        for s, (b, args, _, _) in zip(streams, steps):
            with torch.cuda.stream(s):
                gots.append(step(b, *args))
        torch.cuda.synchronize()
        for want, got in zip(wants, gots):
            assert all(torch.equal(x, y) for x, y in zip(want, got))


def test_run_twice_is_the_same():
    b = filled(360, [30, 1, 64], [2000, 5000, 100], 2, 64)
    for dtype in ("f32", "bf16"):
        q = values(361, (b.total, 8, D), dtype)[0]
        a = qift.qift_kv4_paged_attention(q, b.pages, b.rs, b.f, q_had_block=128)
        for _ in range(3):
            assert torch.equal(a, qift.qift_kv4_paged_attention(q, b.pages, b.rs, b.f, q_had_block=128))


def test_many_replays_of_wide_trees_stay_in_step():
    """Wide trees over contexts of many blocks, many times in a row: every pass gives the same bits and no wait runs out."""
    b = filled(370, [64, 64, 40, 7], [5000, 1300, 64, 9000], 4, 64)
    q = values(371, (b.total, 16, D), "bf16")[0]
    want = qift.qift_kv4_paged_attention(q, b.pages, b.rs, b.f, q_had_block=128)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        gots = [qift.qift_kv4_paged_attention(q, b.pages, b.rs, b.f, q_had_block=128) for _ in range(8)]
    for _ in range(25):
        g.replay()
        assert all(torch.equal(want, got) for got in gots)
    ok()


@pytest.mark.parametrize("had", [(2, 64), (8, 32), (4, 128), (1, 0)])
@pytest.mark.parametrize("clip", [1.0, 0.5])
def test_write_with_other_rotations_and_clips(had, clip):
    H, page = 9, 32                                                                   # more heads than one CTA takes
    b = Batch(380, [40, 3, 90], [20, 31, 5], H, page)
    want = b.pool()
    K, kn = values(381, (b.total, H, D), "bf16", 0.2)
    V, vn = values(382, (b.total, H, D), "bf16", -0.3)
    qift.qift_kv4_paged_write(K, V, b.pages, b.rs, b.f, k_had_block=had[0], v_had_block=had[1], clip_ratio=clip)
    kq = oracle.kv4_quantize(kn.reshape(-1, D), had[0], clip)
    vq = oracle.kv4_quantize(vn.reshape(-1, D), had[1], clip)
    for row, r, pos in b.places():
        for h in range(H):
            blk = want[b.table[r, pos // page], h].reshape(-1, ref.BLOCK)[pos % page // 32]
            t, i = pos % 32, row * H + h
            for bytes_, shifts, codes in ((ref.KB, ref.KSH, kq[0]), (ref.VB, ref.VSH, vq[0])):
                blk[bytes_[t]] = 0
                np.bitwise_or.at(blk, bytes_[t], codes[i].astype(np.uint8) << shifts[t].astype(np.uint8))
            blk[4096 + 4 * t:4100 + 4 * t] = kq[1][i:i + 1].view(np.uint8)
            blk[4224 + 4 * t:4228 + 4 * t] = vq[1][i:i + 1].view(np.uint8)
            blk[4352 + t], blk[4384 + t] = int(kq[2][i]), int(vq[2][i])
    assert np.array_equal(b.pool(), want)
    ok()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [4, 12, 60])
def test_what_is_no_number_stays_with_the_rows_that_see_it(dtype, n):
    """Cached NaN and infinities behind a mask, and query rows of NaN and infinities, leave the other rows as they are."""
    rows, first = [n, n], [75, 300]
    b = filled(390, rows, first, 2, 32)
    mask = trees(9, rows, 2)
    bad = [1, n + 2]                                                                  # drafted token 1 of request 0, 2 of request 1
    x = torch.zeros((2 * n, 2, D), device="cuda")
    K, V = qift.qift_kv4_paged_read(b.pages, b.rs, b.f, 2 * n)
    x[1], x[n + 2, :, ::2] = float("nan"), float("inf")
    qift.qift_kv4_paged_write(K + x, V - x, b.pages, b.rs, b.f)
    q, qn = values(391, (2 * n, 8, D), dtype)
    q[n + 3], q[0, 5] = float("nan"), float("inf")
    got = qift.qift_kv4_paged_attention(q, b.pages, b.rs, b.f, mask=dev(mask)).float().cpu().numpy()
    sees = np.array([(mask[i, 0] >> (1 if i < n else 2)) & 1 for i in range(2 * n)], bool)
    sees[n + 3] = True
    want, size, top = ref.attention(qn, b.pool(), b.table, 32, b.row_start, b.first, mask)
    bound = tolerance(dtype, want, size, top, 300 + n)
    fine = np.repeat(~sees[:, None], 8, 1)
    fine[0, 5] = False
    assert 2 <= fine.sum() // 8 and (np.abs(got - want)[fine] <= bound[fine]).all()
    ok()


def test_wide_trees_with_large_and_tiny_values():
    test_attention_with_large_and_tiny_values("bf16", [64, 40])


def test_wide_trees_over_pages_that_are_none():
    """Pages outside the pool inside and at the end of a context, positions before 0 and past the table."""
    H, page = 2, 32
    b = filled(400, [40, 64, 64], [1000, 95, 30], H, page)
    b.table[0, [0, 3, 4, 5, 20, 32]] = -1
    b.table[1, 1:] = b.pages.num_pages                                                # one page is all there is
    b.table[2] = -7
    b.pages.page_table = ints(b.table)
    q, qn = values(401, (b.total, 8, D), "bf16")
    pool = b.pool()
    for first in ([1000, 95, 30], [1100, -20, 0]):
        got = qift.qift_kv4_paged_attention(q, b.pages, b.rs, ints(first)).float().cpu().numpy()
        want, size, top = ref.attention(qn, pool, b.table, page, b.row_start, first)
        err, bound = np.abs(got - want), tolerance("bf16", want, size, top, 1200)
        seen = np.isfinite(want)                                                      # slots that were never written hold NaN
        assert (err[seen] <= bound[seen]).all() and not got[104:].any()
    ok()


def test_long_runs_in_fp32_lose_nothing_by_the_way():
    """A tile over 32000 tokens, values about -1: sums that are cut off instead of rounded would all be cut the same way.
    A block's sums, six products in a row, lose at most 6 x 2^-23 of themselves; the sums of the codes less 8 and of the zero-points
    less 8 that the result is the difference of are together at most four times the result here; rounded additions and the weights' own
    errors have no common direction."""
    R, n, tokens = 37, 8, 32000                                                       # 37 x 64 tiles: one for each warp of the grid
    k = values(410, (tokens, 1, D), "f32", 0.1)[0]
    v = values(411, (tokens, 1, D), "f32", -1.0)[0]
    table = np.arange(tokens // 128)[None]
    b = qift.Kv4Pages.empty(tokens // 128, 1, 128, ints(table))
    qift.qift_kv4_paged_write(k, v, b, ints([0, tokens]), ints([0]))
    b = qift.Kv4Pages(b.pool, ints(np.repeat(table, R, 0)), 128)
    q, qn = values(412, (R * n, 64, D), "f32", scale=0.3)
    got = qift.qift_kv4_paged_attention(q, b, ints(np.arange(R + 1) * n), ints([tokens - n] * R))
    want = ref.attention(qn[:n], b.pool.cpu().numpy(), table, 128, [0, n], [tokens - n])[0]
    err = got[:n].cpu().numpy() - want
    assert abs((err * want).sum() / (want * want).sum()) <= 4 * 6 * 2.0 ** -23
    ok()

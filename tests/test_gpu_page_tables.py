"""Page tables, positions and slots made on the device, against a plain walk over requests and entries."""
import numpy as np
import pytest
import torch

import paper_2606_02823_b200 as qift
from tables_ref import Tables

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


class Both:
    """The device's tables and the plain ones, kept in step."""

    def __init__(self, table, free, count, page, pages):
        self.plain = Tables(table, free, count, page, pages)
        pool = torch.empty((pages, 1, page // 32 * 4416), dtype=torch.uint8, device="cuda")
        self.pages, self.free = qift.Kv4Pages(pool, ints(table), page), qift.Kv4FreePages(ints(free), ints([count]))

    def same(self):
        assert np.array_equal(self.pages.page_table.cpu().numpy(), self.plain.table)
        assert int(self.free.count) == self.plain.count
        assert np.array_equal(self.free.pages.cpu().numpy(), self.plain.free)

    def begin(self, rows, first, total, mask=None):
        got = qift.qift_kv4_pages_begin(self.pages, self.free, ints(rows), ints(first), total, mask=None if mask is None else ints(mask))
        want = self.plain.begin(rows, first, total, mask)
        for x, y in zip((got.row_start, got.position, got.slot), want):
            assert np.array_equal(x.cpu().numpy(), y)
        assert int(got.lost) == want[3]
        self.same()
        return got

    def end(self, length, shared=None):
        qift.qift_kv4_pages_end(self.pages, self.free, ints(length), None if shared is None else ints(shared))
        self.plain.end(length, shared)
        self.same()


def fresh(r, R, most, page, pages):
    return Both(np.full((R, most), -1), r.permutation(pages), pages, page, pages)


@pytest.mark.parametrize("R, page, rows, total_more", [(1, 32, 1, 0), (1, 64, 5000, 3), (3, 96, 40, 0), (33, 32, 200, 11), (700, 64, 3, 1), (600, 32, 2000, 5),
                                                      (2500, 32, 90, 0), (5, 1024, 3000, 0)])
def test_steps(R, page, rows, total_more):
    """Several steps: rows come, some stay, some requests end; pools that are large enough and that are not."""
    r = np.random.default_rng(R)
    most = -(-4 * rows // page) + 2
    for pages in (R * most, max(1, R * most // 5)):
        b = fresh(r, R, most, page, pages)
        first = np.zeros(R, np.int64)
        for step in range(4):
            n = r.integers(0, rows + 1, R)
            b.begin(n, first, max(1, int(n.sum()) + total_more))
            first = first + r.integers(0, n + 1)
            first[r.random(R) < 0.2] = 0
            b.end(first)


def test_trees_get_their_depths():
    r = np.random.default_rng(1)
    rows, first, words = [7, 0, 64, 1], [5, 9, 1000, 0], 2
    masks = []
    for n in rows:
        bits = []
        for k in range(n):
            bits.append((bits[r.integers(max(0, k - 5), k)] if k else 0) | 1 << k)
        masks += [[b & 0xFFFFFFFF, b >> 32] for b in bits]
    mask = np.array(masks + [[0, 0]] * 3, np.uint32).view(np.int32)
    b = fresh(r, 4, 40, 32, 200)
    b.begin(rows, first, len(masks) + 3, mask)
    mask[2] = 0                                                      # a row that sees nothing
    b.begin(rows, first, len(masks) + 3, mask)
    wide = np.full((len(masks), 32), -1, np.int32)                   # all 1024 bits
    b.begin(rows, first, len(masks), wide)


def test_rows_that_do_not_fit_are_cut():
    b = fresh(np.random.default_rng(2), 4, 5, 32, 100)
    got = b.begin([10, 20, 30, 40], [0, 0, 40, 0], 35)
    assert got.row_start.tolist() == [0, 10, 30, 35, 35] and int(got.lost) == 65
    b.begin([10, 20, 30, 40], [0, 0, 40, 0], 1)


def test_odd_positions():
    """Rows before 0, across the table's end and far behind it, and near 2^31."""
    b = fresh(np.random.default_rng(3), 6, 3, 32, 50)
    b.begin([40, 70, 5, 3, -7, 9], [-20, 60, 5000, 2 ** 31 - 2, 0, -2 ** 31], 140)
    b.end([-5, 2 ** 31 - 1, 0, 97, 33, 96])


def test_what_the_stack_holds_is_checked():
    b = Both(np.full((2, 4), -1), [3, -1, 50, 7, 2 ** 30, 0, 1, 2], 6, 32, 8)     # entries that are no pages are no pages
    b.begin([128, 40], [0, 0], 168)
    b.begin([128, 40], [0, 0], 168)
    for count in (-3, 100):                                                       # counts outside the stack
        b = Both(np.full((2, 4), -1), np.arange(8), count, 32, 8)
        b.begin([40, 40], [0, 0], 80)
        b.end([0, 0])


def test_second_call_fills_in_what_was_missing():
    b = fresh(np.random.default_rng(4), 3, 6, 32, 7)
    rows, first = [100, 100, 60], [30, 0, 0]
    got = b.begin(rows, first, 260)
    assert int(got.lost) > 0
    b.end([0, 100, 60])                                                           # the first request gives way
    got = b.begin([0, 100, 60], [0, 0, 0], 260)
    assert int(got.lost) == 0 and (got.slot[:160] >= 0).all()


def test_a_begin_taken_back_restores_the_stack():
    b = fresh(np.random.default_rng(5), 40, 9, 64, 360)
    first = np.random.default_rng(6).integers(0, 200, 40)
    b.begin(first, np.zeros(40), int(first.sum()))
    before = b.free.pages.clone(), b.free.count.clone(), b.pages.page_table.clone()
    b.begin(np.full(40, 300), first, 12000)
    b.end(first)
    assert torch.equal(before[1], b.free.count) and torch.equal(before[0], b.free.pages) and torch.equal(before[2], b.pages.page_table)


def test_shared_pages_stay_out_of_the_stack_and_doubles_are_dropped():
    table = np.full((3, 4), -1)
    table[0], table[1, :2], table[2, :3] = [0, 1, 2, 3], [0, 1], [0, 1, 4]
    free = np.array([5, 6, 7, 0, 0, 0, 0, 0])
    b = Both(table, free, 3, 32, 8)
    b.end([0, 0, 33], [0, 2, 2])
    table[1] = [9, -5, 3, 3]                                                      # a page twice, and what are no pages
    b = Both(table, free, 6, 32, 8)
    b.end([0, 0, 0])


def test_no_slots_and_given_outputs():
    b = fresh(np.random.default_rng(7), 2, 3, 32, 6)
    out = qift.Kv4Rows.empty(2, 9)
    out.slot = None
    got = qift.qift_kv4_pages_begin(b.pages, b.free, ints([4, 4]), ints([30, 0]), 9, out=out)
    assert got is out and got.position.tolist() == [30, 31, 32, 33, 0, 1, 2, 3, -1]


@pytest.mark.parametrize("total", [300, 6000])
def test_captured_and_replayed_on_another_stream(total):
    """A graph of begin and end follows new lengths; a second one shares nothing with it."""
    r = np.random.default_rng(8)
    b = fresh(r, 20, 30, 32, 700)
    rows, first, length = ints(np.zeros(20)), ints(np.zeros(20)), ints(np.zeros(20))
    out = qift.Kv4Rows.empty(20, total)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            qift.qift_kv4_pages_begin(b.pages, b.free, rows, first, total, out=out)
            qift.qift_kv4_pages_end(b.pages, b.free, length)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qift.qift_kv4_pages_begin(b.pages, b.free, rows, first, total, out=out)
        qift.qift_kv4_pages_end(b.pages, b.free, length)
    f = np.zeros(20, np.int64)
    for step in range(3):
        n = r.integers(0, total // 20, 20)
        keep = f + r.integers(0, n + 1)
        rows.copy_(ints(n)), first.copy_(ints(f)), length.copy_(ints(keep))
        graph.replay()
        want = b.plain.begin(n, f, total)
        b.plain.end(keep)
        for x, y in zip((out.row_start, out.position, out.slot), want):
            assert np.array_equal(x.cpu().numpy(), y)
        b.same()
        f = keep


def test_places_beyond_32_bits():
    """Requests that end at 2^31 - 1 tokens, in a pool of 2^32 (whose memory the calls do not touch)."""
    page, most, pages = 1024, 2 ** 21, 2 ** 22
    plain = Tables(np.full((2, most), -1), np.arange(pages), pages, page, pages)
    table, free, count = ints(plain.table), ints(plain.free), ints([pages])
    rows, first, total = ints([3000, 2]), ints([2 ** 31 - 2500, 2 ** 31 - 2]), 3010
    start, position, lost = ints(np.zeros(3)), ints(np.zeros(total)), ints([0])
    slot = torch.zeros(total, dtype=torch.int64, device="cuda")
    at = [t.data_ptr() for t in (rows, first, table, free, count, start, position, slot, lost)]
    stream = torch.cuda.current_stream().cuda_stream
    assert qift.lib().qift_kv4_pages_begin(at[0], at[1], 2, at[2], most, pages, page, at[3], at[4], None, 0, total, at[5], at[6], at[7], at[8], stream) == qift.OK
    want = plain.begin([3000, 2], [2 ** 31 - 2500, 2 ** 31 - 2], total)
    for x, y in zip((start, position, slot), want):
        assert np.array_equal(x.cpu().numpy(), y)
    assert int(lost) == want[3] == 500 and int(slot.max()) > 2 ** 31
    assert np.array_equal(table.cpu().numpy(), plain.table) and int(count) == plain.count
    length = ints([2 ** 31 - 2000, 0])
    assert qift.lib().qift_kv4_pages_end(length.data_ptr(), None, 2, at[2], most, pages, page, at[3], at[4], stream) == qift.OK
    plain.end([2 ** 31 - 2000, 0], None)
    assert np.array_equal(table.cpu().numpy(), plain.table) and int(count) == plain.count and np.array_equal(free.cpu().numpy(), plain.free)

"""Page tables of two pools at once: graphs of begin and end on two streams, eager calls beside them, each against its own plain walk."""
import numpy as np
import pytest
import torch

import paper_2606_02823_b200 as qift
from test_gpu_page_tables import fresh, ints

pytestmark = pytest.mark.gpu


class Graphed:
    """A pool whose steps are one graph: begin, what begin made of the table, end."""

    def __init__(self, seed, R, total, most, pages):
        self.r, self.R, self.total = np.random.default_rng(seed), R, total
        self.b = fresh(self.r, R, most, 32, pages)
        self.rows, self.first, self.length = (ints(np.zeros(R)) for _ in range(3))
        self.out, self.held = qift.Kv4Rows.empty(R, total), torch.zeros_like(self.b.pages.page_table)
        self.stream, self.f = torch.cuda.Stream(), np.zeros(R, np.int64)
        self.step()
        torch.cuda.synchronize()
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.step()

    def step(self):
        qift.qift_kv4_pages_begin(self.b.pages, self.b.free, self.rows, self.first, self.total, out=self.out)
        self.held.copy_(self.b.pages.page_table)
        qift.qift_kv4_pages_end(self.b.pages, self.b.free, self.length)

    def lengths(self):
        self.n = self.r.integers(0, 2 * self.total // self.R, self.R)     # (some steps ask for more rows than there is room for)
        self.keep = np.where(self.r.random(self.R) < 0.2, 0, self.f + self.r.integers(0, self.n + 1))
        self.rows.copy_(ints(self.n)), self.first.copy_(ints(self.f)), self.length.copy_(ints(self.keep))

    def launch(self, eager):
        self.stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(self.stream):
            self.step() if eager else self.graph.replay()

    def check(self):
        start, position, slot, lost = self.b.plain.begin(self.n, self.f, self.total)
        assert np.array_equal(self.held.cpu().numpy(), self.b.plain.table)
        self.b.plain.end(self.keep)
        for x, y in ((self.out.row_start, start), (self.out.position, position), (self.out.slot, slot)):
            assert np.array_equal(x.cpu().numpy(), y)
        assert int(self.out.lost) == lost
        self.b.same()
        self.f = self.keep
        return lost


@pytest.mark.parametrize("sizes", [((20, 300, 30, 700), (20, 6000, 90, 300)), ((700, 5000, 20, 6000), (300, 40000, 60, 9000)), ((3, 9, 40, 40), (2500, 3000, 8, 9000))])
def test_two_pools_on_two_streams(sizes):
    """One CTA each, one CTA beside a cluster, two clusters: neither takes the other's pages, sums or places."""
    pools = [Graphed(i, *s) for i, s in enumerate(sizes)]
    lost = [0, 0]
    for step in range(8):
        for p in pools:
            p.lengths()
        for i, p in enumerate(pools):
            p.launch(eager=(step + i) % 4 == 3)
        torch.cuda.synchronize()
        for i, p in enumerate(pools):
            lost[i] += p.check()
    assert any(lost)                                                      # places ran out somewhere, and their count was right, too

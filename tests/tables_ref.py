"""Page tables of a batch of requests, entry by entry in Python."""
import numpy as np


class Tables:
    def __init__(self, table, free, count, page, pages):
        self.table, self.free, self.page, self.pages = np.array(table, np.int64), np.array(free, np.int64), page, pages
        self.count = min(max(int(count), 0), pages)

    def is_page(self, v):
        return 0 <= v < self.pages

    def begin(self, rows, first, total, mask=None):
        """-> row_start, position, slot, lost"""
        P, most = self.page, self.table.shape[1]
        start, position, slot, at = [0], np.full(total, -1, np.int64), np.full(total, -1, np.int64), 0
        for r, (n, f) in enumerate(zip(rows, first)):
            n = min(max(int(n), 0), total - at)
            f = int(f)
            if n:
                for i in range(max(f, 0) // P, min(-(-(f + n) // P), most)):
                    if not self.is_page(self.table[r, i]):
                        page = -1
                        if self.count:
                            self.count -= 1
                            page = self.free[self.count]
                        self.table[r, i] = page if self.is_page(page) else -1
            for i in range(n):
                p = f + i
                if 0 <= p < most * P and self.is_page(self.table[r, p // P]):
                    slot[at + i] = self.table[r, p // P] * P + p % P
                if mask is not None:
                    p = f + max(sum(bin(int(w) & 0xFFFFFFFF).count("1") for w in mask[at + i]) - 1, 0)
                position[at + i] = min(max(p, -1), 2 ** 31 - 1)
            at += n
            start.append(at)
        lost = sum(max(int(n), 0) for n in rows) - int((slot >= 0).sum())
        return np.array(start), position, slot, min(lost, 2 ** 31 - 1)

    def end(self, length, shared=None):
        back = []
        for r, n in enumerate(length):
            for i in range(-(-max(int(n), 0) // self.page), self.table.shape[1]):
                if self.is_page(self.table[r, i]) and not (shared is not None and i < shared[r]):
                    back.append(self.table[r, i])
                self.table[r, i] = -1
        for k, page in enumerate(back):
            to = self.count + len(back) - 1 - k
            if to < self.pages:
                self.free[to] = page
        self.count = min(self.count + len(back), self.pages)

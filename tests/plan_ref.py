"""Plans of the paged cache, one page at a time."""


class Plan:
    """State as lists; step() returns (cu_rows, row_pos, slot), or None where it
    cannot be met (the state then stays as it was)."""

    def __init__(self, n_pages, batch, max_pages, page):
        self.n_pages, self.max_pages, self.page = n_pages, max_pages, page
        self.len = [0] * batch
        self.table = [[-1] * max_pages for _ in range(batch)]
        self.free = list(range(n_pages))

    def _pages(self, n):
        return -(-n // self.page)

    def step(self, add, rows=None):
        """rows: room for new rows, or None where positions are not asked for."""
        new = [max(0, n + a) for n, a in zip(self.len, add)]
        most = min(self.max_pages * self.page, 2 ** 31 - 1)
        if any(n > most for n in new) or (rows is not None and sum(max(a, 0) for a in add) > rows):
            return None
        moves = [self._pages(n) - self._pages(o) for n, o in zip(new, self.len)]
        if sum(m for m in moves if m > 0) > len(self.free) - sum(m for m in moves if m < 0):
            return None
        for b in reversed(range(len(add))):
            for i in range(self._pages(self.len[b]) - 1, self._pages(new[b]) - 1, -1):
                self.free.append(self.table[b][i])
                self.table[b][i] = -1
        cu, pos, slot = [0], [], []
        for b, a in enumerate(add):
            for i in range(self._pages(self.len[b]), self._pages(new[b])):
                self.table[b][i] = self.free.pop()
            for p in range(self.len[b], self.len[b] + max(a, 0)):
                pos.append(p)
                slot.append(self.table[b][p // self.page] * self.page + p % self.page)
            cu.append(len(pos))
        self.len = new
        return cu, pos, slot

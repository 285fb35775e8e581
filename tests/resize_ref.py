"""The resize of a paged cache on host lists, sequence by sequence from its definition."""


class State:
    def __init__(self, pages, length, columns, free, page):
        self.pages = [list(r) for r in pages]
        self.length, self.columns, self.free, self.page = list(length), list(columns), list(free), page

    def resize(self, want, held):
        """start, (slot, position) of each row, granted. Pages given back are free afterwards."""
        per = len(self.pages[0]) if self.pages else 0
        start, rows, granted, back, asked, had = [0], [], [], [], 0, len(self.free)
        taken = list(self.free)
        for s in range(len(self.pages)):
            w = min(max(want[s], 0), per * self.page)
            need = max(-(-w // self.page), min(max(held[s], 0), per))
            asks = max(0, need - self.columns[s])
            asked += asks
            ok = asks == 0 or asked <= had
            granted.append(int(ok))
            if ok:
                for c in range(self.columns[s], need):
                    self.pages[s][c] = taken.pop()
                for c in range(need, self.columns[s]):
                    back.append(self.pages[s][c])
                    self.pages[s][c] = -1
                self.columns[s] = need
                for pos in range(self.length[s], w):
                    rows.append((self.pages[s][pos // self.page] * self.page + pos % self.page, pos))
                self.length[s] = w
            start.append(len(rows))
        self.free = taken + back[::-1]
        return start, rows, granted

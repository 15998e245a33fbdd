"""Plain model of a pool of pages for the tests: lists, one entry after the other, as the definitions in include/floe.h read."""


class Pool:
    def __init__(self, n_pages, block, refs=None):
        self.n, self.block = n_pages, block
        self.refs = [0] * n_pages if refs is None else list(refs)

    def is_page(self, e):
        return 0 <= e < self.n

    def count(self, *tables):
        self.refs = [0] * self.n
        for t in tables:
            for row in t:
                for e in row:
                    if self.is_page(e):
                        self.refs[e] += 1
        return self

    def reorder(self, table, length, parent):
        width = len(table[0]) if table else 0
        out, out_len = [], []
        for p in parent:
            there = 0 <= p < len(table)
            out.append(list(table[p]) if there else [-1] * width)
            out_len.append(length[p] if there else 0)
        for rows, by in ((table, -1), (out, 1)):
            for row in rows:
                for e in row:
                    if self.is_page(e):
                        self.refs[e] += by
        return out, out_len

    def blocks(self, length, rows, s, width):
        """The blocks that rows behind length[s] tokens touch, and how many of them lie behind the table."""
        L, n = min(max(length[s], 0), 1 << 30), max(rows[s], 0)
        b = list(range(L // self.block, (L + n - 1) // self.block + 1)) if n else []
        return [x for x in b if x < width], len([x for x in b if x >= width])

    def reserve(self, table, length, rows):
        width = len(table[0]) if table else 0
        pairs, missing = [[-1, -1] for _ in table], 0
        writers = {}
        for s in range(len(table)):
            for b in self.blocks(length, rows, s, width)[0]:
                if self.is_page(table[s][b]):
                    writers.setdefault(table[s][b], []).append(s)
        before = list(self.refs)
        free = [p for p in range(self.n) if self.refs[p] <= 0]
        for s in range(len(table)):
            inside, outside = self.blocks(length, rows, s, width)
            missing += outside
            for b in inside:
                e = table[s][b]
                if self.is_page(e) and (before[e] <= 1 or (writers[e][0] == s and len(writers[e]) >= before[e])):
                    continue
                if not free:
                    missing += 1
                    continue
                new = free.pop(0)
                if self.is_page(e):
                    self.refs[e] -= 1
                    if b == length[s] // self.block and length[s] % self.block:
                        pairs[s] = [e, new]
                table[s][b] = new
                self.refs[new] = 1
        return pairs, missing

    def trim(self, table, length, window, sinks):
        for s, row in enumerate(table):
            for b, e in enumerate(row):
                tokens = range(b * self.block, min((b + 1) * self.block, max(length[s], 0)))
                if any(window == 0 or t > length[s] - window or t < sinks for t in tokens):
                    continue
                if self.is_page(e):
                    self.refs[e] -= 1
                row[b] = -1

    def compact(self, table, moves):
        pairs, where = [], list(range(self.n))
        while len(pairs) < moves:
            used = [p for p in range(self.n) if self.refs[p] > 0]
            free = [p for p in range(self.n) if self.refs[p] <= 0]
            if not used or not free or used[-1] < free[0]:
                break
            pairs.append([used[-1], free[0]])
            where[used[-1]] = free[0]
            self.refs[free[0]], self.refs[used[-1]] = self.refs[used[-1]], 0
        for row in table:
            row[:] = [where[e] if self.is_page(e) else e for e in row]
        return pairs + [[-1, -1]] * (moves - len(pairs)), where

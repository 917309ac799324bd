"""A cache in pages in plain Python: the books as include/fw.h defines them, and every cell's rows as lists of numbers
(a row's identity), shared by the tests of the pages."""
OK, INVALID, WORKSPACE = 0, 1, 5


class Model:
    def __init__(self, cells, N, P, width):
        self.cells, self.N, self.P, self.width = cells, N, P, width
        self.table = [[0] * width for _ in range(cells)]
        self.held, self.counts = [0] * cells, [0] * cells
        self.refs, self.free, self.next = [0] * N, [True] * N, 0
        self.mem = [[None] * P for _ in range(N)]  # row identities in the pool

    # ---- reading
    def rows(self, h):
        return [self.mem[self.table[h][r // self.P]][r % self.P] for r in range(self.counts[h])]

    def bits(self):
        out = []
        for w in range((self.N + 31) // 32):
            x = sum(1 << b for b in range(32) if w * 32 + b < self.N and self.free[w * 32 + b])
            out.append(x - (1 << 32) if x >= 1 << 31 else x)
        return out

    def sound(self, h):
        return 0 <= self.held[h] <= self.width and 0 <= self.counts[h] <= self.held[h] * self.P

    # ---- pages
    def _hand_out(self, needs):
        """Pages for the cells' needs in order (None for a cell that gets none)."""
        free = [(self.next + i) % self.N for i in range(self.N) if self.free[(self.next + i) % self.N]]
        at, got, last, over = 0, [], None, False
        for n in needs:
            over = over or (n > 0 and at + n > len(free))
            if n > 0 and over:
                got.append(None)
                continue
            got.append(free[at:at + n])
            if n:
                last = free[at + n - 1]
            at += n
        for pages in got:
            for p in pages or []:
                self.refs[p], self.free[p] = 1, False
        if last is not None:
            self.next = (last + 1) % self.N
        return got

    def _release(self, pages):
        for p in pages:
            if 0 <= p < self.N:
                self.refs[p] -= 1
                if self.refs[p] == 0:
                    self.free[p] = True

    # ---- calls
    def append(self, m, ident):
        """ident(h, i): what new row i of cell h is."""
        P, st, needs, plans = self.P, [OK] * self.cells, [], []
        for h in range(self.cells):
            n, want = self.counts[h], []
            if not self.sound(h):
                st[h] = INVALID
            elif (n + m - 1) // P >= self.width:
                st[h] = WORKSPACE
            else:
                for i in range(n // P, (n + m - 1) // P + 1):
                    if i < self.held[h] and not 0 <= self.table[h][i] < self.N:
                        st[h] = INVALID
                    elif i >= self.held[h] or self.refs[self.table[h][i]] > 1:
                        want.append(i)
            if st[h] != OK:
                want = []
            plans.append(want)
            needs.append(len(want))
        gone = []
        for h, got in enumerate(self._hand_out(needs)):
            if got is None:
                st[h] = WORKSPACE
            if st[h] != OK:
                continue
            n = self.counts[h]
            for i, p in zip(plans[h], got):
                if i < self.held[h]:
                    was = self.table[h][i]
                    gone.append(was)
                    for r in range(P):
                        if i * P + r < n:
                            self.mem[p][r] = self.mem[was][r]
                self.table[h][i] = p
            self.held[h] = max(self.held[h], (n + m - 1) // P + 1)
            for j in range(m):
                self.mem[self.table[h][(n + j) // P]][(n + j) % P] = ident(h, j)
            self.counts[h] = n + m
        self._release(gone)
        return st

    def compact(self, offsets, kept_pos, source=None, T=None):
        """source(h, t): what row t of cell h of the outer cache is; None: the cells' own rows."""
        P, st, needs = self.P, [OK] * self.cells, []
        for h in range(self.cells):
            o0, o1 = offsets[h], offsets[h + 1]
            if not self.sound(h) or o0 < 0 or o1 < o0 or o1 > len(kept_pos):
                st[h] = INVALID
            elif -(-(o1 - o0) // P) > self.width:
                st[h] = WORKSPACE
            needs.append(0 if st[h] else -(-(o1 - o0) // P))
        gone = []
        for h, got in enumerate(self._hand_out(needs)):
            if got is None:
                st[h] = WORKSPACE
            if st[h] != OK:
                continue
            for j, pos in enumerate(kept_pos[offsets[h]:offsets[h + 1]]):
                if source is None:
                    page = self.table[h][pos // P] if 0 <= pos < self.counts[h] else -1
                    row = self.mem[page][pos % P] if 0 <= page < self.N else 0
                    bad = not 0 <= page < self.N
                else:
                    bad = not 0 <= pos < T
                    row = 0 if bad else source(h, pos)
                if bad:
                    st[h] = INVALID
                self.mem[got[j // P]][j % P] = row
            gone += self.table[h][:self.held[h]]
            self.table[h][:len(got)] = got
            self.held[h], self.counts[h] = len(got), offsets[h + 1] - offsets[h]
        self._release(gone)
        return st

    def fork(self, src):
        P, st, new, gone = self.P, [OK] * self.cells, {}, []
        for h, f in enumerate(src):
            if not self.sound(h) or f >= self.cells or (f >= 0 and not self.sound(f)):
                st[h] = INVALID
                continue
            if f == h:
                continue
            n = self.counts[f] if f >= 0 else 0
            pages = self.table[f][:-(-n // P)] if f >= 0 else []
            if any(not 0 <= p < self.N for p in pages):
                st[h] = INVALID
                continue
            new[h] = (pages, n)
        for pages, _ in new.values():
            for p in pages:
                self.refs[p] += 1
        for h, (pages, n) in new.items():
            gone += self.table[h][:self.held[h]]
        self._release(gone)
        for h, (pages, n) in new.items():
            self.table[h][:len(pages)] = pages
            self.held[h], self.counts[h] = len(pages), n
        return st

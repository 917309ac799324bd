"""The cache in pages: appends, compaction and forks against a model of the books in plain Python (every table entry, every
count and bit, every row)."""
import random

import pytest

from tests.pages_model import Model

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def fw():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2608_25230_gb300 import fw as _fw

    return _fw


def row_of(ident, d):
    """The row that a number stands for: its bits over the columns, as bf16 bit patterns of their own (keys; values differ)."""
    i = torch.as_tensor(ident, dtype=torch.int64, device="cuda")
    c = torch.arange(d, device="cuda")
    return ((i[..., None] * 40503 + c * 977) % 32500).to(torch.int16)


def as_rows(ident, d):
    k = row_of(ident, d)
    return k.view(torch.bfloat16), (k ^ 257).view(torch.bfloat16)


class Both:
    """A cache on the GPU and its model, stepped together."""

    def __init__(self, fw, cells, N, P, width, d):
        self.fw, self.d = fw, d
        self.m = Model(cells, N, P, width)
        self.p = fw.pages_empty(cells, N, d, max_pages=width, page_rows=P)
        self.p.k.view(torch.int16).fill_(-1)
        self.p.v.view(torch.int16).fill_(-1)
        self.status = torch.full((cells,), -1, dtype=torch.int32, device="cuda")
        self.fresh = 1

    def idents(self, cells, n):
        a = self.fresh
        self.fresh += cells * n
        return torch.arange(a, self.fresh).view(cells, n)

    def append(self, m, heads=None, **kw):
        cells = self.m.cells
        heads = heads or cells
        ids = self.idents(cells, m)
        x = ids.view(-1, heads, m).transpose(1, 2)  # [sequences][m][heads]
        k, v = as_rows(x, self.d)
        self.status.fill_(-1)
        self.fw.pages_append(self.p, k, v, status=self.status, **kw)
        self.check(self.m.append(m, lambda h, j: int(ids[h, j])))

    def compact(self, T, offsets, pos, **kw):
        ids = self.idents(self.m.cells, T)
        k, v = as_rows(ids, self.d)
        o, q = torch.tensor(offsets, device="cuda"), torch.tensor(pos, dtype=torch.int32, device="cuda")
        self.status.fill_(-1)
        self.fw.pages_compact(self.p, k, v, o, q, status=self.status, **kw)
        self.check(self.m.compact(offsets, pos, lambda h, t: int(ids[h, t]), T))

    def keep(self, offsets, pos, **kw):
        o, q = torch.tensor(offsets, device="cuda"), torch.tensor(pos, dtype=torch.int32, device="cuda")
        self.status.fill_(-1)
        self.fw.pages_keep(self.p, o, q, status=self.status, **kw)
        self.check(self.m.compact(offsets, pos))

    def fork(self, src, **kw):
        self.status.fill_(-1)
        self.fw.pages_fork(self.p, torch.tensor(src, dtype=torch.int32, device="cuda"), status=self.status, **kw)
        self.check(self.m.fork(src))

    def set_counts(self, counts):
        self.m.counts = list(counts)
        self.p.counts.copy_(torch.tensor(counts, dtype=torch.int32))

    def check(self, status):
        m, p = self.m, self.p
        torch.cuda.synchronize()
        assert self.status.tolist() == status
        assert p.counts.tolist() == m.counts and p.held.tolist() == m.held
        assert p.next.tolist() == [m.next]
        assert p.refs.tolist() == m.refs
        assert p.free.tolist()[:-1] == m.bits()[:-1]
        last = (1 << (m.N - 1) % 32 + 1) - 1
        assert int(p.free[-1]) & last == m.bits()[-1] & last
        table = p.table.tolist()
        assert all(table[h][:m.held[h]] == m.table[h][:m.held[h]] for h in range(m.cells) if 0 <= m.held[h] <= m.width)
        # the pool: what was never written is as it was, rows of a failed position are zeros
        want = torch.tensor([[-1 if x is None else x for x in page] for page in m.mem], device="cuda")
        k, v = as_rows(want, self.d)
        gone, zero = (want == -1)[..., None], (want == 0)[..., None]
        k = torch.where(gone, torch.full_like(k.view(torch.int16), -1), torch.where(zero, 0, k.view(torch.int16)))
        v = torch.where(gone, torch.full_like(k, -1), torch.where(zero, 0, v.view(torch.int16)))
        assert torch.equal(p.k.view(torch.int16), k) and torch.equal(p.v.view(torch.int16), v)


def picks(r, counts):
    """Ascending positions of every cell below its count, some cells all or none of them."""
    off, pos = [0], []
    for n in counts:
        share = r.choice([0, 0.1, 0.5, 0.9, 1])
        mine = [t for t in range(n) if r.random() < share]
        pos += mine
        off.append(len(pos))
    return off, pos


@pytest.mark.parametrize("P,d", [(16, 64), (16, 128), (32, 64), (64, 128), (128, 64)])
@pytest.mark.parametrize("seed", [0, 1])
def test_sequences_of_calls(fw, P, d, seed):
    r = random.Random(f"{P} {d} {seed}")
    cells = r.choice([1, 6, 12])
    b = Both(fw, cells, r.choice([97, 160, 333]), P, 12, d)
    for _ in range(14):
        what = r.choice(["append", "append", "append", "fork", "keep", "compact", "back"])
        if what == "append":
            b.append(r.choice([1, 1, 2, 5, P - 1, P, P + 1, 3 * P + 7]), heads=r.choice([x for x in (1, 2, 3, 6) if cells % x == 0]))
        elif what == "fork":
            b.fork([r.choice([h, h, r.randrange(cells), r.randrange(cells), -1]) for h in range(cells)])
        elif what == "keep":
            b.keep(*picks(r, b.m.counts))
        elif what == "compact":
            T = r.choice([1, 33, 200])
            b.compact(T, *picks(r, [T] * cells))
        else:
            b.set_counts([max(0, n - r.choice([0, 1, 3, P, n])) for n in b.m.counts])


def test_twins_append_beside_each_other(fw):
    """Cells that share an incomplete page and all append: each gets its own, and the shared one is free when the last has left."""
    b = Both(fw, 4, 40, 32, 6, 64)
    b.append(45)
    b.fork([0, 0, 0, 3])
    b.append(1)
    b.fork([0, 0, 2, -1])
    b.append(30, heads=2)
    b.set_counts([64, 40, 33, 5])  # back over a page's border
    b.fork([0, 0, 0, 0])
    b.append(3)
    b.fork([-1] * 4)
    assert all(b.m.free)


def test_beams_change_places(fw):
    b = Both(fw, 6, 64, 16, 8, 128)
    for m in (17, 16, 1):
        b.append(m, heads=2)
        b.fork([2, 3, 0, 1, 0, 1])
    b.fork([1, 2, 3, 4, 5, 0])


@pytest.mark.parametrize("N", [1, 31, 32, 33, 64, 130])
def test_pool_runs_out(fw, N):
    """What is left goes to the first cells; the first that it does not hold and those behind it get none."""
    b = Both(fw, 5, N, 16, 40, 64)
    for m in (20, 1, 150, 16, 5, 333, 1):
        b.append(m)
    b.fork([-1, 1, 0, 3, 4])
    b.append(40)
    b.keep([0] * 6, [])
    b.append(16 * max(1, N // 5))


def test_tables_end(fw):
    b = Both(fw, 3, 50, 16, 4, 64)
    b.append(60)
    b.append(5)      # beyond four pages
    b.append(4)
    b.append(1)
    b.compact(90, [0, 65, 129, 129], list(range(65)) + list(range(64)))  # 5 pages, 4, none
    b.compact(90, [0, 64, 64, 90], list(range(90)))


@pytest.mark.parametrize("own", [False, True])
def test_bad_positions_and_offsets(fw, own):
    b = Both(fw, 6, 80, 16, 8, 64)
    b.append(40)
    pos = [0, 39, 5, -1, 40, 1 << 30, -(1 << 31), 7, 7, 3] + list(range(30))
    for off in ([0, 3, 7, 10, 10, 40, 40], [0, 3, 2, 10, 41, 40, 40], [-1, 3, 3, 3, 20, 20, 1 << 40], [40, 40, 0, 40, 0, 40, 0]):
        if own:
            b.keep(off, pos)
        else:
            b.compact(40, off, pos)


def test_bad_books(fw):
    """Cells whose counts, held entries or pages are out of range are left as they were, and all others served."""
    b = Both(fw, 8, 90, 16, 6, 64)
    b.append(40)

    def spoil(h, **kw):
        for name, x in kw.items():
            if name == "page":
                i, x = x
                b.m.table[h][i] = x
                b.p.table[h, i] = x
            else:
                getattr(b.m, name)[h] = x
                getattr(b.p, name)[h] = x

    spoil(1, counts=-1)
    spoil(2, counts=49)
    spoil(3, held=-2)
    spoil(4, held=7)
    spoil(5, page=(2, 90))
    spoil(6, page=(2, -1))
    spoil(7, page=(0, 1 << 30))
    b.append(1)
    b.append(20)
    b.fork([0, 1, 0, 3, 4, 0, 5, 7])
    b.keep([0, 3, 3, 6, 6, 9, 12, 15, 16], [0, 1, 2] * 5 + [0])
    b.compact(20, [0, 3, 3, 6, 6, 9, 12, 15, 15], list(range(3)) * 5)
    b.fork([8, 1 << 30, -(1 << 31), 0, 0, 0, 6, 0])
    b.p.next.fill_(-5)  # (a place to search from that is none: the first page)
    b.m.next = 0
    b.append(17)

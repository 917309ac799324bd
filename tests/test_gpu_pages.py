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


def test_kept_rows_on_an_entry_that_is_no_page(fw):
    """They become zeros, with a status; the cell's other rows are kept, its good pages are given back, other cells are served."""
    P, d, n = 16, 64, 40
    p = fw.pages_empty(3, 20, d, max_pages=4, page_rows=P)
    ids = torch.arange(1, 3 * n + 1, device="cuda").view(1, 3, n).transpose(1, 2)
    fw.pages_append(p, *as_rows(ids, d))
    k, v = (x[0].transpose(0, 1) for x in as_rows(ids, d))  # [cells][rows][d]
    gone = int(p.table[1, 1])
    p.table[1, 1] = 20
    status = torch.full((3,), -1, dtype=torch.int32, device="cuda")
    pos = [0, 39, 3, 15, 16, 31, 32, 5]
    off = torch.tensor([0, 2, 6, 8], device="cuda")
    fw.pages_keep(p, off, torch.tensor(pos, dtype=torch.int32, device="cuda"), status=status)
    torch.cuda.synchronize()
    assert status.tolist() == [fw.FW_OK, fw.FW_ERR_INVALID_ARG, fw.FW_OK]
    assert p.counts.tolist() == [2, 4, 2] and p.held.tolist() == [1, 1, 1]
    for h in range(3):
        for j, t in enumerate(pos[int(off[h]):int(off[h + 1])]):
            page = int(p.table[h, 0])
            for pool, want in ((p.k, k), (p.v, v)):
                row = torch.zeros_like(want[h, t]) if h == 1 and t // P == 1 else want[h, t]
                assert torch.equal(pool[page, j].view(torch.int16), row.view(torch.int16))
    # all that the books named but the three new pages is free again; the page that an entry named no more is nobody's
    assert [i for i, x in enumerate(p.refs.tolist()) if x] == sorted([gone] + p.table[:, 0].tolist())


@pytest.mark.parametrize("cells,width,N,P,d", [(40, 12, 700, 16, 64), (7, 300, 1700, 16, 64), (33, 600, 3000, 16, 128)])
def test_forks_of_many_cells_and_long_tables(fw, cells, width, N, P, d):
    """More cells than one CTA takes, tables longer than what is asked for early."""
    r = random.Random(f"{cells} {width}")
    b = Both(fw, cells, N, P, width, d)
    b.append(min(P * (width - 1), P * N // cells // 2))
    b.set_counts([r.randint(0, n) for n in b.m.counts])
    b.append(1)
    for _ in range(4):
        b.fork([r.choice([h, r.randrange(cells), r.randrange(cells), -1, cells + 3]) for h in range(cells)])
        b.append(r.choice([1, P + 1]))
    b.fork([-1] * cells)
    assert all(b.m.free)


def test_many_cells_in_a_large_pool(fw):
    """More cells than the plan's CTA has threads, more words of free bits than it asks for at a time, a search round the
    end."""
    r = random.Random(3)
    cells, N, P, width = 2500, 140000, 16, 70
    b = Both(fw, cells, N, P, width, 64)
    b.p.next.fill_(N - 1000)
    b.m.next = N - 1000
    b.append(3)
    b.append(200)  # (13 pages more a cell)
    b.fork([r.choice([h, h, r.randrange(cells), -1]) for h in range(cells)])
    b.append(1)
    b.append(700)  # (32,000 pages are in use, these do not all fit)
    b.set_counts([n // 2 for n in b.m.counts])
    b.keep(*picks(r, b.m.counts))
    b.compact(40, *picks(r, [40] * cells))
    b.append(60)


def test_pool_nearly_full(fw):
    """Free pages far from where the search begins, a few among many words of none."""
    b = Both(fw, 3, 300000, 16, 100000, 64)
    b.append(16 * 99990)
    b.fork([0, 1, 2])
    b.set_counts([16 * 99990 - 5, 7, 16 * 500])
    b.append(40)
    b.fork([0, -1, 2])
    b.append(16 * 70000)
    b.append(16 * 30000)


def test_calls_in_a_graph(fw):
    """A captured step (append, fork, keep), replayed: it goes by the books as they are then."""
    cells, P, d = 6, 16, 64
    b = Both(fw, cells, 200, P, 12, d)
    b.append(21)
    ids = b.idents(cells, 1)
    k, v = as_rows(ids.view(1, cells, 1).transpose(1, 2), d)
    src = torch.tensor([0, 0, 2, 3, 2, -1], dtype=torch.int32, device="cuda")
    off, pos = [0, 3, 5, 5, 9, 9, 9], [0, 2, 20, 1, 19, 0, 1, 2, 3]
    o, q = torch.tensor(off, device="cuda"), torch.tensor(pos, dtype=torch.int32, device="cuda")
    st = [torch.empty(cells, dtype=torch.int32, device="cuda") for _ in range(3)]
    ws = [fw.pages_append_workspace(b.p, 1), fw.pages_fork_workspace(b.p), fw.pages_compact_workspace(b.p, 9)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fw.pages_append(b.p, k, v, status=st[0], workspace=ws[0])
        fw.pages_fork(b.p, src, status=st[1], workspace=ws[1])
        fw.pages_append(b.p, k, v, status=st[2], workspace=ws[0])
    one = torch.cuda.CUDAGraph()
    with torch.cuda.graph(one):
        fw.pages_keep(b.p, o, q, status=b.status, workspace=ws[2])
    for _ in range(3):
        for w in ws:
            w.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        assert st[0].tolist() == b.m.append(1, lambda h, j: int(ids[h, 0]))
        assert st[1].tolist() == b.m.fork(src.tolist())
        b.status.copy_(st[2])
        b.check(b.m.append(1, lambda h, j: int(ids[h, 0])))
    one.replay()
    b.check(b.m.compact(off, pos))


def test_a_book_put_back_undoes_a_step(fw):
    b = Both(fw, 4, 60, 32, 5, 128)
    b.append(40)
    b.fork([0, 0, 2, 3])
    before, k, v = b.p.book.clone(), b.p.k.clone(), b.p.v.clone()
    rows = [[(b.p.table[h, r // 32].item(), r % 32) for r in range(40)] for h in range(4)]
    new = torch.ones(1, 5, 4, 128, dtype=torch.bfloat16, device="cuda")
    fw.pages_append(b.p, new, new)
    b.p.book.copy_(before)
    torch.cuda.synchronize()
    for h in range(4):
        for page, r in rows[h]:
            assert torch.equal(b.p.k[page, r].view(torch.int16), k[page, r].view(torch.int16))
            assert torch.equal(b.p.v[page, r].view(torch.int16), v[page, r].view(torch.int16))


def test_strides_streams_and_broadcast_rows(fw):
    """New rows out of wider projections, one row for all, on another stream; a cache of one cell."""
    gen = torch.Generator("cuda").manual_seed(1)
    p = fw.pages_empty(6, 40, 64, max_pages=4, page_rows=16)
    x = torch.randn(3, 7, 10, 64, generator=gen, device="cuda").to(torch.bfloat16)  # [sequences][tokens][heads]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    fw.pages_append(p, x[:, :, 3:5], x[:, :, 5:7], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    fw.pages_append(p, x[:, 2:3, 8:10].expand(3, 13, 2, 64), x[0, 0, 0].expand(3, 13, 2, 64))
    torch.cuda.synchronize()
    assert p.counts.tolist() == [20] * 6
    for c in range(6):
        s, h = divmod(c, 2)
        t = torch.arange(20, device="cuda")
        k, v = (y[p.table[c].long()[t // 16], t % 16] for y in (p.k, p.v))
        assert torch.equal(k[:7], x[s, :, 3 + h]) and torch.equal(v[:7], x[s, :, 5 + h])
        assert torch.equal(k[7:], x[s, 2, 8 + h].expand(13, 64)) and torch.equal(v[7:], x[0, 0, 0].expand(13, 64))
    one = fw.pages_empty(1, 3, 128, max_pages=3, page_rows=128)
    y = torch.randn(1, 300, 1, 128, generator=gen, device="cuda").to(torch.bfloat16)
    fw.pages_append(one, y, y)
    # a token-major cache's kept rows
    z = torch.randn(90, 6, 64, generator=gen, device="cuda").to(torch.bfloat16)
    o = torch.arange(7, device="cuda") * 10
    pos = torch.arange(60, dtype=torch.int32, device="cuda")
    fw.pages_compact(p, z.transpose(0, 1), z.transpose(0, 1), o, pos)
    torch.cuda.synchronize()
    assert torch.equal(one.k.view(-1, 128)[:300], y[0, :, 0]) and one.counts.tolist() == [300]
    for c in range(6):
        assert torch.equal(p.k[p.table[c, 0].long(), :10], z[10 * c:10 * c + 10, c])

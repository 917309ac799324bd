"""Calls that change the books of a cache in pages right behind one another, with nothing between them: forks of more than 32 cells or of
tables beyond 256 entries (whose second kernel reads tables before the first has ended), appends of several pages a cell, compaction
from a contiguous cache and of the cells' own rows."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def fw():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2608_25230_gb300 import fw as _fw

    return _fw


class Loop:
    """Calls whose every input is ready before the first of them, on one cache."""

    def __init__(self, fw, cells, width, rows, m, d, P=16, steps=4):
        self.fw, self.cells, self.steps = fw, cells, steps
        gen = torch.Generator("cuda").manual_seed(cells + width + m + d)
        self.p = p = fw.pages_empty(cells, 3 * cells * width, d, max_pages=width, page_rows=P)
        p.k.zero_(), p.v.zero_()

        def rand(*shape):
            return torch.randn(*shape, generator=gen, device="cuda").to(torch.bfloat16)

        def positions(T, n):
            keep = torch.argsort(torch.rand(cells, T, generator=gen, device="cuda"), 1)[:, :n].sort(1)[0]
            return torch.arange(cells + 1, device="cuda") * n, keep.to(torch.int32).flatten().contiguous()

        first = rand(1, rows, cells, d)
        fw.pages_append(p, first, first * 0.5)
        self.new = [[rand(1, x, cells, d) for x in (m, 1, 3 * P + 5)] for _ in range(steps)]
        # forks into neighbours' places, beams that change places, sequences that end, cells that stay
        src = [torch.randint(0, cells, (cells,), generator=gen, device="cuda") for _ in range(2 * steps)]
        for i, s in enumerate(src):
            s[i % 3::5] = torch.arange(i % 3, cells, 5, device="cuda")
            s[i % 7::11] = -1
        self.src = [s.to(torch.int32) for s in src]
        # (what a cell has not as many rows for is a row of zeros)
        self.own = [positions(rows, rows - 40 - i) for i in range(steps)]
        self.outer = rand(cells, rows + 9, d)
        self.kept = [positions(rows + 9, rows - 7 * i) for i in range(steps)]
        self.q = rand(cells, 1, 4, d)
        self.outs = [fw.pages_attend(p, self.q, kv_heads=1) for _ in range(3 * steps)]
        self.status = [torch.full((cells,), -1, dtype=torch.int32, device="cuda") for _ in range(9 * steps)]
        self.ws = [fw.pages_append_workspace(p, max(m, 3 * P + 5)), fw.pages_fork_workspace(p),
                   fw.pages_compact_workspace(p, cells * (rows + 9)), fw.pages_attend_workspace(p, self.q, kv_heads=1)]

    def run(self, wait):
        fw, p = self.fw, self.p
        status, outs = iter(self.status), iter(self.outs)

        def attend():
            fw.pages_attend(p, self.q, kv_heads=1, out=next(outs), workspace=self.ws[3])
            wait()

        def append(x):
            fw.pages_append(p, x, x, status=next(status), workspace=self.ws[0])
            wait()

        def fork(i):
            fw.pages_fork(p, self.src[i], status=next(status), workspace=self.ws[1])
            wait()

        for i in range(self.steps):
            one, two, three = self.new[i]
            append(one)
            fork(2 * i)
            append(two)
            attend()
            fw.pages_keep(p, *self.own[i], status=next(status), workspace=self.ws[2])
            wait()
            fork(2 * i + 1)
            fork(2 * i)
            append(three)
            attend()
            fw.pages_compact(p, self.outer, self.outer, *self.kept[i], status=next(status), workspace=self.ws[2])
            wait()
            fork(2 * i + 1)
            attend()

    def rows(self):
        """All cells' rows, zeros behind them."""
        p = self.p
        there = torch.arange(p.max_pages, device="cuda") < p.held[:, None]
        page = torch.where(there, p.table, 0).long()
        r = torch.arange(p.max_pages * p.page_rows, device="cuda") < p.counts[:, None]
        return [torch.where(r[..., None], x[page].flatten(1, 2), 0) for x in (p.k, p.v)]


# cells, table entries, rows at first: more cells than one CTA's, tables beyond 256 entries that are held, and both
@pytest.mark.parametrize("cells,width,rows,m,d", [(40, 40, 300, 1, 64), (70, 48, 500, 2, 128), (6, 330, 4400, 1, 64), (40, 300, 4300, 7, 64)])
@pytest.mark.parametrize("how", ["stream", "graph"])
def test_calls_without_a_wait_are_calls_with_one(fw, cells, width, rows, m, d, how):
    one, other = Loop(fw, cells, width, rows, m, d), Loop(fw, cells, width, rows, m, d)
    torch.cuda.synchronize()
    one.run(torch.cuda.synchronize)
    if how == "stream":
        other.run(lambda: None)
    else:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            other.run(lambda: None)
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(one.p.book, other.p.book)
    for a, b in zip(one.status, other.status):
        assert torch.equal(a, b)
    for a, b in zip(one.outs, other.outs):
        assert torch.equal(a["o"], b["o"]) and torch.equal(a["lse"], b["lse"]) and torch.equal(a["status"], b["status"])
    for a, b in zip(one.rows(), other.rows()):
        assert torch.equal(a, b)
    refs, free = one.p.refs, one.p.free
    there = torch.arange(width, device="cuda") < one.p.held[:, None]
    named = torch.bincount(one.p.table[there].long(), minlength=refs.numel())
    assert torch.equal(named.to(torch.int32), refs)
    bits = (free[:, None] >> torch.arange(32, dtype=torch.int32, device="cuda") & 1).flatten()[:refs.numel()]
    assert torch.equal(bits == 1, refs == 0)

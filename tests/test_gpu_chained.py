"""Calls on pages right behind one another and behind other kernels: they start before the one in front has ended, and must not
be seen to."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def fw():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2608_25230_gb300 import fw as _fw

    return _fw


class Decode:
    """A decode loop whose every call reads what the one before wrote, with buffers that are used again at once."""

    def __init__(self, fw, d, m, seqs=6, heads=2, group=4, far=300):
        self.fw, self.d, self.m, self.seqs, self.heads = fw, d, m, seqs, heads
        gen = torch.Generator("cuda").manual_seed(d + m)
        cells = seqs * heads
        self.p = fw.pages_empty(cells, 40 * cells, d, max_pages=40, page_rows=16)
        k = torch.randn(seqs, far, heads, d, generator=gen, device="cuda").to(torch.bfloat16)
        fw.pages_append(self.p, k, k * 0.5)
        rows = seqs * m
        self.x = torch.randn(rows, (group + 2) * heads, d, generator=gen, device="cuda").to(torch.bfloat16)
        self.mix = torch.randn(2048, 2048, generator=gen, device="cuda")
        self.q = torch.empty(rows, group * heads, d, dtype=torch.bfloat16, device="cuda")
        self.k = torch.empty(rows, heads, d, dtype=torch.bfloat16, device="cuda")
        self.pos = torch.arange(rows, dtype=torch.int32, device="cuda")
        self.freq = 1.0 / 1e4 ** (torch.arange(0, d, 2, device="cuda") / d)
        self.ws = [fw.pages_append_workspace(self.p, m), fw.pages_fork_workspace(self.p),
                   fw.pages_attend_workspace(self.p, self.q.view(seqs, m, -1, d), kv_heads=heads, longest=400)]
        self.out = dict(o=torch.empty(seqs, m, group * heads, d, dtype=torch.bfloat16, device="cuda"))
        self.src = torch.arange(cells, dtype=torch.int32, device="cuda")
        self.saved = []

    def step(self, i, wait, stream=None):
        fw, x, hq = self.fw, self.x, self.q.shape[1]
        # a long kernel in front, whose result the queries take
        y = self.mix @ self.mix
        x[:, 0] += y[0, :self.d].to(torch.bfloat16) * 1e-3
        wait()
        fw.qk_rotate(x[:, :hq], x[:, hq:hq + self.heads], self.pos, self.freq, eps=1e-5, out=(self.q, self.k), stream=stream)
        wait()
        view = (self.seqs, self.m, -1, self.d)
        fw.pages_append(self.p, self.k.view(view), x[:, hq + self.heads:].view(view), workspace=self.ws[0], stream=stream)
        wait()
        for longest in (400, 0):
            fw.pages_attend(self.p, self.q.view(view), kv_heads=self.heads, longest=longest, out=self.out, stream=stream,
                            workspace=self.ws[2] if longest else None)
            wait()
            x[:, :hq] += self.out["o"].reshape(x[:, :hq].shape)  # the next step's input
            self.saved.append(self.out["o"].clone())
            wait()
        self.src.copy_(torch.roll(self.src, self.heads))
        fw.pages_fork(self.p, self.src, workspace=self.ws[1], stream=stream)
        wait()
        if i % 3 == 2:
            n = self.p.counts.long()
            off = torch.cat([n.new_zeros(1), (n * 0 + 290).cumsum(0)])
            pos = torch.arange(290, dtype=torch.int32, device="cuda").repeat(self.p.cells)
            fw.pages_keep(self.p, off, pos, stream=stream)
            wait()


@pytest.mark.parametrize("d,m", [(64, 1), (128, 1), (128, 3), (64, 5)])
@pytest.mark.parametrize("how", ["stream", "side", "graph"])
def test_steps_without_a_wait_are_steps_with_one(fw, d, m, how):
    one, other = Decode(fw, d, m), Decode(fw, d, m)
    torch.cuda.synchronize()
    for i in range(7):
        one.step(i, torch.cuda.synchronize)
    torch.cuda.synchronize()
    if how == "stream":
        for i in range(7):
            other.step(i, lambda: None)
    elif how == "side":
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for i in range(7):
                other.step(i, lambda: None)
        torch.cuda.current_stream().wait_stream(side)
    else:
        g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(g):
            for i in range(7):
                if i % 2:  # (a step on a branch of the graph)
                    side.wait_stream(torch.cuda.current_stream())
                    with torch.cuda.stream(side):
                        other.step(i, lambda: None)
                    torch.cuda.current_stream().wait_stream(side)
                else:
                    other.step(i, lambda: None)
        g.replay()
    torch.cuda.synchronize()
    assert len(one.saved) == len(other.saved) == 14
    for a, b in zip(one.saved, other.saved):
        assert bool(torch.isfinite(a.float()).all()) and torch.equal(a, b)
    assert torch.equal(one.p.book, other.p.book)

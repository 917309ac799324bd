"""Attention over a cache in pages against plain attention in 64 bits."""
import math
import random

import pytest

from tests.attention64 import attend64, check_rows

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# weights enter the second product as the sum of two bf16 numbers: half a step of the second, 2^-8 of what the first
# leaves, itself at most 2^-8 of the weight
U_P = 2.0 ** -16


@pytest.fixture(scope="module")
def fw():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2608_25230_gb300 import fw as _fw

    return _fw


def rand(gen, *shape, amp=1.0):
    x = amp * torch.randn(*shape, generator=gen, device="cuda")
    return (x * torch.exp2(torch.randint(-3, 4, shape[:-1] + (1,), generator=gen, device="cuda"))).to(torch.bfloat16)


def cache_of(fw, gen, counts, P, d, *, width=None, spare=5, fill=float("nan")):
    """Pages scattered over a pool; rows behind the counts and pages of nobody hold `fill`."""
    need = [-(-n // P) for n in counts]
    N = sum(need) + spare
    p = fw.pages_empty(len(counts), N, d, max_pages=width or max(need + [1]) + 1, page_rows=P)
    order = torch.randperm(N, generator=gen, device="cuda").to(torch.int32)
    p.table.fill_(-7)
    at = 0
    for h, e in enumerate(need):
        p.table[h, :e] = order[at:at + e]
        at += e
    p.held.copy_(torch.tensor(need, dtype=torch.int32))
    p.counts.copy_(torch.tensor(counts, dtype=torch.int32))
    p.k.copy_(rand(gen, N, P, d))
    p.v.copy_(rand(gen, N, P, d))
    used = torch.zeros(N, P, dtype=torch.bool, device="cuda")
    for h, n in enumerate(counts):
        r = torch.arange(n, device="cuda")
        used[p.table[h].long()[r // P], r % P] = True
    p.k[~used], p.v[~used] = fill, fill
    return p


def rows_of(p, h, n):
    r = torch.arange(n, device="cuda")
    page = p.table[h].long()[r // p.page_rows]
    return p.k[page, r % p.page_rows].double(), p.v[page, r % p.page_rows].double()


def check_cell(p, h, n, q, out, kv_heads, scale, skip=()):
    b, hk = divmod(h, kv_heads)
    m, g = q.shape[1], q.shape[2] // kv_heads
    k, v = rows_of(p, h, n)
    seen = (torch.arange(m, device="cuda") + n - m + 1).clamp(min=0).repeat_interleave(g)
    mine = slice(hk * g, (hk + 1) * g)
    want = attend64(q[b, :, mine].reshape(m * g, -1).double(), k, v, seen, scale)
    check_rows(out["o"][b, :, mine].reshape(m * g, -1), out["lse"][b, :, mine].reshape(-1), want, U_P)


def check_all(fw, p, counts, q, kv_heads, scale=None, **kw):
    out = fw.pages_attend(p, q, kv_heads=kv_heads, scale=scale, **kw)
    torch.cuda.synchronize()
    assert not bool(out["status"].any())
    for h, n in enumerate(counts):
        check_cell(p, h, n, q, out, kv_heads, 1.0 / math.sqrt(q.shape[-1]) if scale is None else scale)
    again = fw.pages_attend(p, q, kv_heads=kv_heads, scale=scale, **kw)
    assert torch.equal(out["o"].view(torch.int16), again["o"].view(torch.int16)) and torch.equal(out["lse"], again["lse"])
    return out


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("group,m", [(1, 1), (4, 1), (7, 1), (8, 2), (3, 7), (16, 5), (128, 1), (1, 40)])
def test_lengths(fw, d, P, group, m):
    gen = torch.Generator("cuda").manual_seed(d + P + group)
    counts = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 333, 7, 1000, 40]
    p = cache_of(fw, gen, counts, P, d)
    q = rand(gen, 5, m, 4 * group, d)
    check_all(fw, p, counts, q, 4)
    check_all(fw, p, counts, q, 4, longest=1000)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cells,mean", [(1, 5), (1, 20000), (2, 700), (7, 3000), (8, 4097), (20, 1100), (40, 900), (100, 300),
                                        (700, 50), (1300, 1), (3000, 20)])
def test_splits(fw, d, cells, mean):
    """Few long cells, many short ones: every way in which the rows are divided."""
    r = random.Random(f"{d} {cells} {mean}")
    gen = torch.Generator("cuda").manual_seed(cells + mean)
    counts = [r.choice([0, mean, r.randint(0, 2 * mean), r.randint(0, 2 * mean)]) if cells > 1 else mean for _ in range(cells)]
    p = cache_of(fw, gen, counts, r.choice([16, 32, 64]), d)
    for group, m in ((4, 1), (5, 2), (9, 3)):
        q = rand(gen, cells, m, group, d)
        for longest in (0, max(counts)):
            out = fw.pages_attend(p, q, kv_heads=1, longest=longest)
            torch.cuda.synchronize()
            assert not bool(out["status"].any())
            for h in sorted(set(range(cells) if cells <= 40 else r.sample(range(cells), 40))):
                check_cell(p, h, counts[h], q, out, 1, 1.0 / math.sqrt(d))


def test_one_cell_holds_most_rows(fw):
    gen = torch.Generator("cuda").manual_seed(2)
    counts = [3] * 5 + [30000] + [0] * 60 + [17] * 62
    p = cache_of(fw, gen, counts, 32, 128)
    for longest in (0, 10, 30000):  # (a bound that is wrong leaves nothing out)
        check_all(fw, p, counts, rand(gen, 128, 1, 4, 128), 1, longest=longest)


@pytest.mark.parametrize("d", [64, 128])
def test_strides_parts_and_scales(fw, d):
    gen = torch.Generator("cuda").manual_seed(d)
    counts = [50, 0, 131, 77, 16, 900, 33, 64]
    p = cache_of(fw, gen, counts, 16, d)
    # the queries out of a wider projection
    x = rand(gen, 4, 3, 14, d + 16)
    q = x[:, :, 2:12, 8:8 + d]
    for scale in (None, 1.0, 3.0, 1e-3):
        check_all(fw, p, counts, q, 2, scale=scale)
    part = p.part(2, 4)
    check_all(fw, part, counts[2:6], q[1:3], 2)
    # one row of queries for all heads and tokens
    check_all(fw, p, counts, rand(gen, 4, 1, 1, d).expand(4, 3, 10, d), 2)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_a_token_does_not_see_has_no_part(fw, d, bad):
    """Values and keys of a draft's later rows that are not finite: rows that do not see them stay clean, those that
    do are not finite."""
    gen = torch.Generator("cuda").manual_seed(d)
    m, g, counts = 6, 3, [5, 18, 40, 300, 6, 70]
    p = cache_of(fw, gen, counts, 16, d, fill=bad)
    q = rand(gen, 6, m, g, d)
    clean = fw.pages_attend(p, q, kv_heads=1)
    torch.cuda.synchronize()
    for where in ("k", "v"):
        for back in (1, 3, 5):  # that row from the end: tokens from m - back on see it
            x = p.v if where == "v" else p.k
            kept = x.clone()
            for h, n in enumerate(counts):
                r = n - back
                if r >= 0:
                    row = x[int(p.table[h, r // 16]), r % 16]
                    row[5 if where == "v" else 0] = bad
            out = fw.pages_attend(p, q, kv_heads=1)
            torch.cuda.synchronize()
            for h, n in enumerate(counts):
                if n - back < 0:
                    continue
                for t in range(m):
                    if n - m + 1 + t <= n - back:
                        assert torch.equal(out["o"][h, t], clean["o"][h, t]) and torch.equal(out["lse"][h, t], clean["lse"][h, t])
                    elif where == "v":
                        rest = [c for c in range(d) if c != 5]
                        assert not bool(torch.isfinite(out["o"][h, t, :, 5]).any())
                        assert bool(torch.isfinite(out["o"][h, t][:, rest]).all())
                        # the other columns are what they were (their sums may be taken in another order)
                        k, v = rows_of(p, h, n)
                        v[:, 5] = 0.0
                        if not math.isnan(bad):
                            # a weight below 2^-149 of the largest is 0 in 32 bits, and 0 times infinity is NaN: the sign
                            # is certain where the weight is above 2^-100 of the sum
                            logits = (q[h, t].double() @ k[:n - m + 1 + t].T) / math.sqrt(d)
                            sure = torch.softmax(logits, 1)[:, n - back] > 2.0 ** -100
                            assert bool((out["o"][h, t, sure, 5] == bad).all())
                        seen = torch.full((g,), n - m + 1 + t, device="cuda")
                        want = attend64(q[h, t].double(), k, v, seen, 1.0 / math.sqrt(d))
                        got = out["o"][h, t].clone()
                        got[:, 5] = 0.0
                        check_rows(got, out["lse"][h, t], want, U_P)
                    elif math.isnan(bad):
                        assert bool(torch.isnan(out["o"][h, t]).all())
            x.copy_(kept)


def test_pages_and_books_out_of_range(fw):
    """A page that is none has no part, a count or an entry out of range leaves the cell empty; the status says so, and
    other cells are served."""
    gen = torch.Generator("cuda").manual_seed(8)
    d, P, counts = 128, 16, [100, 200, 300, 40, 500, 64, 48]
    p = cache_of(fw, gen, counts, P, d)
    q = rand(gen, 7, 2, 4, d)
    p.table[1, 3], p.table[2, 0], p.table[4, 31] = p.num_pages, -1, 1 << 30
    p.counts[3] = p.held[3] * P + 1
    p.held[5] = p.max_pages + 1
    p.counts[6] = -3
    for longest in (0, 500):
        out = fw.pages_attend(p, q, kv_heads=1, longest=longest)
        torch.cuda.synchronize()
        assert out["status"].tolist() == [0] + [fw.FW_ERR_INVALID_ARG] * 6
        check_cell(p, 0, 100, q, out, 1, 1.0 / math.sqrt(d))
        for h in (3, 5, 6):
            assert not bool(out["o"][h].any()) and bool(torch.isneginf(out["lse"][h]).all())
        for h, page in ((1, 3), (2, 0), (4, 31)):
            n = counts[h]
            r = torch.arange(n, device="cuda")
            ok = r // P != page
            pg = p.table[h].long()[r // P].clamp(0, p.num_pages - 1)
            k, v = p.k[pg, r % P].double()[ok], p.v[pg, r % P].double()[ok]
            for t in range(2):
                seen = ((r < n - 1 + t) & ok).sum().expand(4)
                want = attend64(q[h, t].double(), k, v, seen, 1.0 / math.sqrt(d))
                check_rows(out["o"][h, t], out["lse"][h, t], want, U_P)


def test_rows_beyond_two_to_the_31_elements(fw):
    """A pool whose offsets pass 32 bits: pages at its end."""
    gen = torch.Generator("cuda").manual_seed(3)
    d, P, counts = 128, 128, [700, 129, 1]
    N = (1 << 31) // (P * d) + 300  # 4.9 GB of keys
    p = fw.pages_empty(3, N, d, max_pages=8, page_rows=P)
    need = [-(-n // P) for n in counts]
    order = list(range(N - sum(need), N))
    for h, e in enumerate(need):
        p.table[h, :e] = torch.tensor(order[:e], dtype=torch.int32)
        del order[:e]
    p.k[-20:], p.v[-20:] = rand(gen, 20, P, d), rand(gen, 20, P, d)
    p.held.copy_(torch.tensor(need, dtype=torch.int32))
    p.counts.copy_(torch.tensor(counts, dtype=torch.int32))
    q = rand(gen, 3, 1, 8, d)
    check_all(fw, p, counts, q, 1)
    # and appends there
    p.refs[p.table[0, :6].long()] = 1
    p.refs[p.table[1, :2].long()] = 1
    p.refs[p.table[2, :1].long()] = 1
    p.next.fill_(N - 30)
    new = rand(gen, 3, 1, 1, d)
    fw.pages_append(p, new, new)
    torch.cuda.synchronize()
    for h, n in enumerate(counts):
        assert torch.equal(rows_of(p, h, n + 1)[0][-1], new[h, 0, 0].double())
    check_all(fw, p, [n + 1 for n in counts], q, 1)


def test_side_streams_and_graphs(fw):
    """Two captured calls that share a workspace, replayed one after another with other counts."""
    gen = torch.Generator("cuda").manual_seed(6)
    counts = [200, 3, 0, 77, 500, 64, 1, 31]
    p = cache_of(fw, gen, counts, 16, 64)
    q = [rand(gen, 4, 1, 8, 64) for _ in "ab"]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = fw.pages_attend(p, q[0], kv_heads=2, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for h, n in enumerate(counts):
        check_cell(p, h, n, q[0], out, 2, 0.125)
    ws = fw.pages_attend_workspace(p, q[0], kv_heads=2)
    outs, graphs = [], []
    for x in q:
        o = dict(o=torch.empty_like(x), lse=torch.empty(x.shape[:-1], device="cuda"),
                 status=torch.empty(8, dtype=torch.int32, device="cuda"))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            fw.pages_attend(p, x, kv_heads=2, out=o, workspace=ws)
        outs.append(o)
        graphs.append(g)
    counts = [n // 2 for n in counts]
    p.counts.copy_(torch.tensor(counts, dtype=torch.int32))
    ws.fill_(255)
    for g in graphs:
        g.replay()
    torch.cuda.synchronize()
    for x, o in zip(q, outs):
        for h, n in enumerate(counts):
            check_cell(p, h, n, x, o, 2, 0.125)


def test_a_kept_workspace_and_a_bound_that_grows(fw):
    """A workspace made at the first step, whose bound asks for clusters, serves the steps whose bound asks for ranges."""
    gen = torch.Generator("cuda").manual_seed(9)
    counts = [300] * 64
    p = cache_of(fw, gen, counts, 16, 128, width=2000)
    q = rand(gen, 64, 1, 4, 128)
    ws = fw.pages_attend_workspace(p, q, kv_heads=1, longest=300)
    for longest in (300, 600, 3000, 32000, 0):
        check_all(fw, p, counts, q, 1, longest=longest, workspace=ws)


def test_without_lse_and_status(fw):
    gen = torch.Generator("cuda").manual_seed(7)
    p = cache_of(fw, gen, [90, 0, 3], 32, 64)
    q = rand(gen, 3, 1, 4, 64)
    want = fw.pages_attend(p, q, kv_heads=1)
    o = torch.empty_like(q)
    fw.pages_attend(p, q, kv_heads=1, out=dict(o=o))
    torch.cuda.synchronize()
    assert torch.equal(o, want["o"])


@pytest.mark.parametrize("group,m", [(100, 40), (7, 33), (5, 17), (60, 1)])
def test_many_query_rows(fw, group, m):
    """Tiles of rows beyond one team's, the last of them nearly empty."""
    gen = torch.Generator("cuda").manual_seed(group)
    counts = [33, 400, 5]
    p = cache_of(fw, gen, counts, 32, 128)
    q = rand(gen, 3, m, group, 128)
    for longest in (0, 400):
        check_all(fw, p, counts, q, 1, longest=longest)


def test_rows_that_see_nothing_beside_rows_that_do(fw):
    """Drafts longer than their cells' rows."""
    gen = torch.Generator("cuda").manual_seed(4)
    counts = [1, 3, 0, 16, 17, 30]
    p = cache_of(fw, gen, counts, 16, 64, fill=float("inf"))
    for longest in (0, 30):
        out = check_all(fw, p, counts, rand(gen, 6, 20, 3, 64), 1, longest=longest)
        assert bool(torch.isneginf(out["lse"][2]).all()) and not bool(out["o"][0, :19].any())


@pytest.mark.parametrize("d", [64, 128])
def test_logits_that_grow_and_are_far_apart(fw, d):
    """Maxima that move in every block, by little and by much, up and down; rows of equal logits."""
    gen = torch.Generator("cuda").manual_seed(d)
    n = 700
    p = cache_of(fw, gen, [n] * 5, 16, d)
    q = torch.zeros(5, 1, 2, d, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 8.0
    t = torch.arange(n, device="cuda").float()
    for h, f in enumerate((0.1 * t, -0.1 * t, 40 * torch.sin(t), 0 * t, torch.where(t % 97 == 0, 90.0, -3e38 / 8))):
        page = p.table[h].long()[torch.arange(n, device="cuda") // 16]
        p.k[page, torch.arange(n, device="cuda") % 16, 0] = f.to(torch.bfloat16)
        p.k[page, torch.arange(n, device="cuda") % 16, 1:] = 0
    for longest in (0, n):
        check_all(fw, p, [n] * 5, q, 1, scale=1.0, longest=longest)


def test_as_many_blocks_as_are_numbered(fw):
    """Tables that name few pages over and over: all cells' blocks of 16 rows together are 2^31 - 128, so that a share of them
    rounded up passes 2^31.  Every weight is 1 and every value 0 or 1, so all sums of a team (14 million rows) are whole
    numbers below 2^24, exact in 32 bits.  About 2,432 of these in 16 cells are joined by 153 sums each, 2^-24 off relative, so
    o, whose values 2^-6 apart are bf16 numbers, is exact, and lse off by 2^-24 * 153, a step of the logarithm to base 2 of
    about 31 (2^-19) and two roundings at 21.5: below 2^-15."""
    cells, P, d, width, N = 16, 128, 64, (1 << 24) - 1, 64
    table = (torch.arange(width, device="cuda", dtype=torch.int32) % N).expand(cells, width).contiguous()
    r, c = torch.arange(P, device="cuda")[:, None], torch.arange(d, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    p = fw.Pages(k=rand(torch.Generator("cuda").manual_seed(1), N, P, d), v=(r % 64 <= c).to(torch.bfloat16).expand(N, P, d).contiguous(),
                 table=table, held=torch.full((cells,), width, **i32), counts=torch.full((cells,), width * P, **i32),
                 refs=torch.ones(N, **i32), free=torch.zeros(2, **i32), next=torch.zeros(1, **i32))
    out = fw.pages_attend(p, torch.zeros(cells, 1, 1, d, dtype=torch.bfloat16, device="cuda"), kv_heads=1)
    torch.cuda.synchronize()
    assert not bool(out["status"].any())
    assert torch.equal(out["o"].double(), ((c + 1) / 64).double().expand_as(out["o"]))
    assert bool(((out["lse"].double() - math.log(width * P)).abs() < 2.0 ** -15).all())


@pytest.mark.parametrize("d,group,m,tile,warp,rows", [
    (128, 4, 1, 0, 0, range(0, 4)), (64, 5, 2, 0, 0, range(0, 8)), (64, 5, 2, 0, 1, range(8, 10)), (128, 4, 5, 0, 2, range(16, 20)),
    (64, 20, 1, 0, 1, range(8, 16)), (64, 30, 1, 0, 3, range(24, 30)), (128, 12, 5, 0, 3, range(24, 32)),
    (128, 12, 5, 1, 0, range(32, 40)), (128, 12, 5, 1, 3, range(56, 60)), (64, 45, 2, 1, 5, range(88, 90))])
def test_a_wait_that_gives_up_shows(fw, d, group, m, tile, warp, rows):
    """Whichever warp of whichever tile gives up: its rows are NaN, its cells' statuses say so, and all else is as it was.  (As if a
    wait had given up: no wait runs out.  Cells are so short that no other warp waits for what this one would have asked for.)"""
    gen = torch.Generator("cuda").manual_seed(group)
    counts = [40, 0, 16, 17, 70, 48, 33, 1, 90, 0, 64, 5]
    p = cache_of(fw, gen, counts, 16, d)
    q = rand(gen, 12, m, group, d)
    p.table[4, 1] = -1  # (a page that is none beside it)
    mine = torch.tensor([r in rows for r in range(m * group)], device="cuda").view(m, group)
    for longest in (0, 90):
        want = fw.pages_attend(p, q, kv_heads=1, longest=longest)
        fw.raw().fw_pages_attend_give_up(tile, warp)
        try:
            out = fw.pages_attend(p, q, kv_heads=1, longest=longest)
        finally:
            fw.raw().fw_pages_attend_give_up(-1, -1)
        again = fw.pages_attend(p, q, kv_heads=1, longest=longest)
        torch.cuda.synchronize()
        assert want["status"].tolist() == [fw.FW_ERR_INVALID_ARG if h == 4 else 0 for h in range(12)]
        assert out["status"].tolist() == [fw.FW_ERR_TIMEOUT if n else 0 for n in counts]
        hit = mine & (torch.tensor(counts, device="cuda")[:, None, None] > 0)
        assert bool(torch.isnan(out["o"][hit]).all()) and bool(torch.isnan(out["lse"][hit]).all())
        assert torch.equal(out["o"][~hit].view(torch.int16), want["o"][~hit].view(torch.int16))
        assert torch.equal(out["lse"][~hit], want["lse"][~hit])
        for x in ("o", "lse", "status"):
            assert torch.equal(again[x], want[x])


@pytest.mark.parametrize("d,beams", [(64, 4), (128, 8)])
def test_cells_that_share_pages(fw, d, beams):
    """Beams of two prompts that fork, decode on and fork again: every cell's attention is that over its own rows, and bit for bit
    that over copies of them in pages of its own."""
    gen = torch.Generator("cuda").manual_seed(d)
    heads, P = 2, 16
    cells = 2 * beams * heads
    p = fw.pages_empty(cells, 40 * cells, d, max_pages=40, page_rows=P)
    first = rand(gen, 2 * beams, 333, heads, d)
    fw.pages_append(p, first, rand(gen, 2 * beams, 333, heads, d))
    for i in range(3):
        lead = [s // beams * beams + (s * (i + 1) + i) % beams // 2 for s in range(2 * beams)]  # (half of the beams go on, twice each)
        fw.pages_fork(p, torch.tensor([s * heads + h for s in lead for h in range(heads)], dtype=torch.int32, device="cuda"))
        fw.pages_append(p, rand(gen, 2 * beams, 5, heads, d), rand(gen, 2 * beams, 5, heads, d))
    torch.cuda.synchronize()
    counts = p.counts.tolist()
    assert counts == [348] * cells and int((p.refs > 1).sum()) > 20 * heads
    q = rand(gen, 2 * beams, 3, 4 * heads, d)
    own = cache_of(fw, gen, counts, P, d)
    r = torch.arange(348, device="cuda")
    for h in range(cells):
        to, at = own.table[h].long()[r // P], p.table[h].long()[r // P]
        own.k[to, r % P], own.v[to, r % P] = p.k[at, r % P], p.v[at, r % P]
    for longest in (0, 348):
        out = check_all(fw, p, counts, q, heads, longest=longest)
        other = fw.pages_attend(own, q, kv_heads=heads, longest=longest)
        assert torch.equal(out["o"].view(torch.int16), other["o"].view(torch.int16)) and torch.equal(out["lse"], other["lse"])

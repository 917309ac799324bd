"""The 8-bit ragged store: compaction into it and appends to it against a plain quantisation in
64 bits (every bit), and the attention over it against plain attention in 64 bits."""
import math

import pytest

from tests.attention64 import attend64, check_rows

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TOP = {"e4m3": 448.0, "int8": 127.0}
U_P = 2.0 ** -11  # weights are rounded to fp16 for the second product


@pytest.fixture(scope="module")
def fw():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2608_25230_gb300 import fw as _fw

    return _fw


def quantise64(rows, fmt):
    """(values of the codes, scale) of one block's rows, from the definition."""
    x = rows.double()
    finite = torch.isfinite(x)
    top = float(torch.where(finite, x.abs(), torch.zeros_like(x)).max())
    e = -120
    while top > TOP[fmt] * 2.0 ** e:
        e += 1
    y = torch.nan_to_num(x, nan=0.0, posinf=TOP[fmt] * 2.0 ** e, neginf=-TOP[fmt] * 2.0 ** e) / 2.0 ** e
    if fmt == "int8":
        return torch.round(y), 2.0 ** e
    table = torch.tensor([(m / 8 * 2.0 ** -6 if x == 0 else (1 + m / 8) * 2.0 ** (x - 7)) for x in range(16)
                          for m in range(8)][:127], dtype=torch.float64, device=x.device)
    mid = (table[1:] + table[:-1]) / 2
    a = y.abs()
    up = torch.searchsorted(mid, a, right=True)   # a tie goes up ...
    down = torch.searchsorted(mid, a, right=False)
    i = torch.where(up != down, torch.where(up % 2 == 0, up, down), up)  # ... or to the even code
    return torch.sign(y) * table[i], 2.0 ** e


def check_cell(cache, h, kv, rows, first=0):
    """The cell's blocks from row `first` on hold exactly the quantised rows."""
    base, n = int(cache.base[h]), rows.shape[0]
    codes, scales, tail = ((cache.k, cache.k_scale, cache.k_tail), (cache.v, cache.v_scale, cache.v_tail))[kv]
    assert int(cache.counts[h]) == n
    for b in range(first // 32 * 32, n, 32):
        val, sc = quantise64(rows[b:b + 32], cache.fmt)
        assert float(scales[(base + b) // 32]) == sc
        assert torch.equal(codes[base + b:base + min(b + 32, n)].double(), val)
    for r in range(max(first, n // 32 * 32), n):
        assert torch.equal(tail[h, r % 64].view(torch.int16), rows[r].view(torch.int16))


def rand(gen, *shape, amp=1.0):
    x = amp * torch.randn(*shape, generator=gen, device="cuda")
    return (x * torch.exp2(torch.randint(-3, 4, shape[:-1] + (1,), generator=gen, device="cuda"))).to(torch.bfloat16)


def off(counts):
    return torch.tensor([sum(counts[:i]) for i in range(len(counts) + 1)], dtype=torch.int64, device="cuda")


def picks(gen, counts, T):
    return torch.cat([torch.randperm(T, generator=gen, device="cuda")[:c].sort().values for c in counts] or
                     [torch.zeros(0, device="cuda")]).to(torch.int32)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("room", [0, 40])
def test_compact(fw, fmt, d, room):
    gen = torch.Generator("cuda").manual_seed(d + room)
    counts, T = [0, 1, 31, 32, 33, 64, 100, 257, 7, 500], 500
    K, V = rand(gen, len(counts), T, d), rand(gen, len(counts), T, d)
    pos, o = picks(gen, counts, T), off(counts)
    cache = fw.cache8_empty(o, pos.numel() + 77, d, fmt=fmt, room=room)
    assert bool((cache.capacity >= torch.tensor(counts, device="cuda") + room).all())
    cache.k.view(torch.int8).fill_(85)
    st = torch.full((len(counts),), -1, dtype=torch.int32, device="cuda")
    fw.cache8_compact(cache, K, V, o, torch.cat([pos, pos.new_full((77,), -5)]), status=st)
    torch.cuda.synchronize()
    assert not bool(st.any())
    used = torch.zeros(cache.k.shape[0], dtype=torch.bool, device="cuda")
    for h, c in enumerate(counts):
        p = pos[int(o[h]):int(o[h + 1])].long()
        check_cell(cache, h, 0, K[h, p])
        check_cell(cache, h, 1, V[h, p])
        used[int(cache.base[h]):int(cache.base[h]) + c] = True
    assert bool((cache.k.view(torch.int8)[~used] == 85).all())  # other rows keep what they held


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_compact_token_major_cache(fw, fmt):
    gen = torch.Generator("cuda").manual_seed(3)
    T, H, d = 300, 4, 64
    K, V = rand(gen, T, H, d), rand(gen, T, H, d)
    counts = [40, 300, 0, 129]
    pos, o = picks(gen, counts, T), off(counts)
    cache = fw.cache8_empty(o, pos.numel(), d, fmt=fmt)
    fw.cache8_compact(cache, K.transpose(0, 1), V.transpose(0, 1), o, pos)
    torch.cuda.synchronize()
    for h in range(H):
        p = pos[int(o[h]):int(o[h + 1])].long()
        check_cell(cache, h, 0, K[p, h])
        check_cell(cache, h, 1, V[p, h])


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_scales_at_their_edges(fw, fmt):
    """Blocks whose largest value lies at, just below and just above a scale's limit; blocks of zeros, of
    subnormals, of the type's extremes; ties; infinities and NaN."""
    d, tops = 64, []
    for m in range(128):
        tops += [(1 + m / 128) * 2.0 ** x for x in (0, 7, -9, 100, -120, 127)]
    tops += [0.0, 2.0 ** -133, 3 * 2.0 ** -133, 2.0 ** -126, 3.3895313892515355e38]
    n = len(tops)
    gen = torch.Generator("cuda").manual_seed(1)
    t = torch.tensor(tops, dtype=torch.float64, device="cuda")
    x = (torch.rand(n, 32, d, generator=gen, device="cuda", dtype=torch.float64) * 2 - 1) * t[:, None, None] * 0.99
    # multiples of an eighth of the top's last code: ties in plenty
    x[:, 1] = torch.randint(-8, 9, (n, d), generator=gen, device="cuda") / 16 * t[:, None]
    x[:, 0, 0] = -t
    K = x.to(torch.bfloat16)
    o, pos = off([32] * n), torch.arange(32, dtype=torch.int32, device="cuda").repeat(n)
    cache = fw.cache8_empty(o, 32 * n, d, fmt=fmt)
    st = torch.empty(n, dtype=torch.int32, device="cuda")
    fw.cache8_compact(cache, K, K, o, pos, status=st)
    torch.cuda.synchronize()
    assert not bool(st.any())
    for h in range(n):
        check_cell(cache, h, 0, K[h])
    K = K[:3].clone()
    K[0, 5, 7], K[1, 31, 63], K[2, 0, 0], K[2, 1, 1] = float("nan"), float("inf"), float("-inf"), float("nan")
    cache = fw.cache8_empty(off([32] * 3), 96, d, fmt=fmt)
    fw.cache8_compact(cache, K, K, off([32] * 3), pos[:96], status=st[:3])
    torch.cuda.synchronize()
    assert st[:3].tolist() == [fw.FW_ERR_NONFINITE] * 3
    for h in range(3):
        check_cell(cache, h, 1, K[h])


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("steps", [[1] * 70, [33, 1, 30, 2, 64, 7], [100, 200], [5, 31, 31, 1, 1, 32]])
def test_appends_equal_the_rows_quantised_at_once(fw, fmt, d, steps):
    gen = torch.Generator("cuda").manual_seed(sum(steps))
    start = [0, 1, 31, 32, 63, 90]
    T, cells = 90, len(start)
    K, V = rand(gen, cells, T, d), rand(gen, cells, T, d)
    o = off(start)
    pos = torch.cat([torch.arange(c, device="cuda") for c in start]).to(torch.int32)
    cache = fw.cache8_empty(o, pos.numel(), d, fmt=fmt, room=sum(steps))
    fw.cache8_compact(cache, K, V, o, pos)
    rows = [[K[h, :start[h]] for h in range(cells)], [V[h, :start[h]] for h in range(cells)]]
    st = torch.empty(cells, dtype=torch.int32, device="cuda")
    for m in steps:
        new = [rand(gen, cells, m, d), rand(gen, cells, m, d)]
        fw.cache8_append(cache, new[0], new[1], status=st)
        for kv in range(2):
            rows[kv] = [torch.cat([rows[kv][h], new[kv][h]]) for h in range(cells)]
        assert not bool(st.any())
    torch.cuda.synchronize()
    for h in range(cells):
        for kv in range(2):
            check_cell(cache, h, kv, rows[kv][h])


def test_append_after_counts_are_set_back(fw):
    """A draft of up to 32 rows is taken back, also across a block's end, and other rows follow."""
    gen = torch.Generator("cuda").manual_seed(4)
    d, start = 64, [0, 20, 31, 32, 50]
    cells = len(start)
    K = rand(gen, cells, 64, d)
    o, pos = off(start), torch.cat([torch.arange(c, device="cuda") for c in start]).to(torch.int32)
    cache = fw.cache8_empty(o, pos.numel(), d, room=80)
    fw.cache8_compact(cache, K, K, o, pos)
    have = [K[h, :start[h]] for h in range(cells)]
    for draft, kept in [(32, 0), (7, 3), (32, 1), (5, 5), (13, 0), (1, 1)]:
        new = rand(gen, cells, draft, d, amp=100.0 if kept == 0 else 1.0)
        fw.cache8_append(cache, new, new)
        cache.counts.sub_(draft - kept)
        have = [torch.cat([have[h], new[h, :kept]]) for h in range(cells)]
    new = rand(gen, cells, 2, d)
    before = [x.shape[0] for x in have]
    fw.cache8_append(cache, new, new)
    torch.cuda.synchronize()
    for h in range(cells):  # (the block that the last append touches is the quantised rows')
        check_cell(cache, h, 0, torch.cat([have[h], new[h]]), first=before[h])


def test_store_refusals_per_cell(fw):
    d, cells = 64, 5
    K = torch.ones(cells, 100, d, dtype=torch.bfloat16, device="cuda")
    o, pos = off([40] * cells), torch.arange(40, dtype=torch.int32, device="cuda").repeat(cells)
    cache = fw.cache8_empty(o, 200, d)
    cache.k.view(torch.int8).fill_(17)
    cache.capacity[0], cache.capacity[1] = 64, 39
    cache.base[2] += 1
    cache.capacity[3] = cache.k.shape[0]
    pos[4 * 40 + 3] = 100
    st = torch.empty(cells, dtype=torch.int32, device="cuda")
    fw.cache8_compact(cache, K, K, o, pos, status=st)
    torch.cuda.synchronize()
    I, W = fw.FW_ERR_INVALID_ARG, fw.FW_ERR_WORKSPACE
    assert st.tolist() == [0, W, I, I, I] and cache.counts.tolist() == [40, 0, 0, 0, 40]
    assert bool((cache.k.view(torch.int8)[64:192] == 17).all())
    new = torch.ones(cells, 25, d, dtype=torch.bfloat16, device="cuda")
    cache.counts.copy_(torch.tensor([40, 20, 0, 0, -1], dtype=torch.int32))
    fw.cache8_append(cache, new, new, status=st)
    torch.cuda.synchronize()
    assert st.tolist() == [W, W, I, I, I] and cache.counts.tolist() == [40, 20, 0, 0, -1]
    q = torch.ones(1, 1, cells, d, dtype=torch.bfloat16, device="cuda")
    out = fw.cache8_attend(cache, q, kv_heads=cells)
    torch.cuda.synchronize()
    assert out["status"].tolist() == [0, 0, I, I, I]
    assert not bool(out["o"][0, 0, 2:].any()) and bool(torch.isneginf(out["lse"][0, 0, 2:]).all())


# ------------------------------------------------------------------ attention
def filled(fw, gen, counts, d, fmt, room=0):
    o = off(counts)
    cache = fw.cache8_empty(o, sum(counts), d, fmt=fmt, room=room)
    for x in (cache.k, cache.v):
        if fmt == "e4m3":
            x.copy_((80 * torch.randn(x.shape, generator=gen, device="cuda")).clamp_(-448, 448).to(x.dtype))
        else:
            x.copy_((30 * torch.randn(x.shape, generator=gen, device="cuda")).round_().clamp_(-127, 127).to(x.dtype))
    for x in (cache.k_scale, cache.v_scale):
        x.copy_(torch.exp2(torch.randint(-8, -4, x.shape, generator=gen, device="cuda").float()))
    cache.counts.copy_(torch.tensor(counts, dtype=torch.int32))
    return cache


def values(cache, h):
    b, n = int(cache.base[h]), int(cache.counts[h])
    blk = (torch.arange(n, device="cuda") + b) // 32
    return [(x[b:b + n].double() * s[blk].double()[:, None]) for x, s in
            ((cache.k, cache.k_scale), (cache.v, cache.v_scale))]


def check_attend(cache, q, out, kv_heads, scale):
    seqs, m, hq, d = q.shape
    g = hq // kv_heads
    for h in range(cache.cells):
        b, hk = divmod(h, kv_heads)
        k, v = values(cache, h)
        Q = q[b, :, hk * g:(hk + 1) * g].reshape(-1, d).double()
        n = k.shape[0]
        seen = (n - m + 1 + torch.arange(m, device="cuda")).clamp(min=0).repeat_interleave(g)
        want = attend64(Q, k, v, seen, scale)
        kmax = float(k.abs().sum(1).max()) if n else 0.0
        # (queries keep 2^-24 of a row's largest)
        extra = 2.0 ** -24 * scale * kmax * Q.abs().amax(1)
        check_rows(out["o"][b, :, hk * g:(hk + 1) * g].reshape(-1, d), out["lse"][b, :, hk * g:(hk + 1) * g].reshape(-1),
                   want, U_P, extra)
    assert not bool(out["status"].any())


COUNTS = {"short": [0, 1, 2, 31, 32, 33], "odd": [300, 5, 1025, 0, 64, 777], "long": [9001, 31, 2000, 20000, 12000, 1]}


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("counts", list(COUNTS))
@pytest.mark.parametrize("kv_heads,g,m", [(1, 1, 1), (2, 4, 1), (3, 8, 1), (2, 4, 3), (6, 7, 5), (1, 16, 2), (1, 40, 3)])
def test_attend(fw, fmt, d, counts, kv_heads, g, m):
    gen = torch.Generator("cuda").manual_seed(g * m + d)
    cache = filled(fw, gen, COUNTS[counts], d, fmt)
    q = (1.5 * torch.randn(6 // kv_heads, m, kv_heads * g, d, generator=gen, device="cuda")).to(torch.bfloat16)
    scale = 1 / math.sqrt(d)
    out = fw.cache8_attend(cache, q, kv_heads=kv_heads, scale=scale)
    torch.cuda.synchronize()
    check_attend(cache, q, out, kv_heads, float(torch.tensor(scale, dtype=torch.float32)))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_attend_many_cells(fw, fmt):
    gen = torch.Generator("cuda").manual_seed(8)
    counts = [int(x) for x in torch.randint(0, 900, (600,), generator=torch.Generator().manual_seed(8))]
    cache = filled(fw, gen, counts, 64, fmt)
    q = torch.randn(75, 1, 32, 64, generator=gen, device="cuda").to(torch.bfloat16)
    out = fw.cache8_attend(cache, q, kv_heads=8)
    torch.cuda.synchronize()
    check_attend(cache, q, out, 8, 0.125)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("d", [64, 128])
def test_attend_rows_past_the_count_have_no_part(fw, fmt, d):
    """Rows behind a cell's count hold anything, e4m3's NaN among it, and so do scales of blocks behind it."""
    gen = torch.Generator("cuda").manual_seed(6)
    cache = filled(fw, gen, [70, 0, 33, 500], d, fmt, room=100)
    q = torch.randn(2, 2, 8, d, generator=gen, device="cuda").to(torch.bfloat16)
    used = torch.zeros(cache.k.shape[0], dtype=torch.bool, device="cuda")
    for h in range(4):
        b = int(cache.base[h])
        used[b:b + int(cache.counts[h])] = True
    free = ~used.view(-1, 32).any(1)
    for x in (cache.k, cache.v):
        x.view(torch.int8)[~used] = 0x7f
    for x in (cache.k_scale, cache.v_scale):
        x[free] = float("nan")
    out = fw.cache8_attend(cache, q, kv_heads=2)
    torch.cuda.synchronize()
    check_attend(cache, q, out, 2, float(torch.tensor(1 / math.sqrt(d), dtype=torch.float32)))


@pytest.mark.parametrize("d", [64, 128])
def test_attend_ranges(fw, d):
    """Queries of any size (rows of zeros, of 1e-30 and 1e30 among ordinary ones), value scales far apart, logits
    whose maximum moves by hundreds both ways."""
    gen = torch.Generator("cuda").manual_seed(7)
    cache = filled(fw, gen, [600, 600], d, "e4m3")
    q = torch.randn(2, 1, 8, d, generator=gen, device="cuda")
    q[0, 0, 0] = 0
    q[0, 0, 1] *= 1e-30
    q[0, 0, 2] *= 100.0
    q[1, 0, 3, 1:] *= 1e-6
    q = q.to(torch.bfloat16)
    cache.v_scale.copy_(torch.exp2(torch.randint(-60, 60, cache.v_scale.shape, generator=gen, device="cuda").float()))
    cache.k_scale.copy_(torch.exp2(torch.randint(-12, -1, cache.k_scale.shape, generator=gen, device="cuda").float()))
    out = fw.cache8_attend(cache, q, kv_heads=1, scale=0.25)
    torch.cuda.synchronize()
    check_attend(cache, q, out, 1, 0.25)
    big = q.clone()
    big[0, 0, 0] = 1e30
    cache.k_scale.fill_(2.0 ** -110)
    out = fw.cache8_attend(cache, big, kv_heads=1, scale=0.25)
    torch.cuda.synchronize()
    check_attend(cache, big, out, 1, 0.25)


@pytest.mark.parametrize("m", [1, 3])
def test_attend_strides_streams_and_repeats(fw, m):
    gen = torch.Generator("cuda").manual_seed(11)
    cache = filled(fw, gen, [400, 3, 77, 2500, 129, 1000], 128, "int8")
    fused = torch.randn(3, m, 24, 128, generator=gen, device="cuda").to(torch.bfloat16)
    q = fused[:, :, 4:12]
    a = fw.cache8_attend(cache, q, kv_heads=2)
    b = fw.cache8_attend(cache, q.contiguous(), kv_heads=2, workspace=fw.cache8_attend_workspace(cache, q, kv_heads=2))
    t = q.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c = fw.cache8_attend(cache, t, kv_heads=2, stream=side)
    only = fw.cache8_attend(cache, q, kv_heads=2, out=dict(o=torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")))
    torch.cuda.synchronize()
    check_attend(cache, q, a, 2, float(torch.tensor(1 / math.sqrt(128), dtype=torch.float32)))
    for x in (b, c, only):
        assert torch.equal(a["o"], x["o"])
    assert torch.equal(a["lse"], b["lse"]) and torch.equal(a["lse"], c["lse"])


def test_attend_offsets_past_32_bits(fw):
    """A store of more than 2^31 codes, its cells at both ends."""
    gen = torch.Generator("cuda").manual_seed(12)
    rows, d = 18 << 20, 128
    z = dict(device="cuda")
    store = dict(k=torch.zeros(rows, d, dtype=torch.int8, **z), v=torch.zeros(rows, d, dtype=torch.int8, **z),
                 k_scale=torch.ones(rows // 32, **z), v_scale=torch.ones(rows // 32, **z),
                 k_tail=torch.zeros(2, 64, d, dtype=torch.bfloat16, **z), v_tail=torch.zeros(2, 64, d, dtype=torch.bfloat16, **z),
                 base=torch.tensor([32, rows - 2080], **z), capacity=torch.tensor([64, 2080], dtype=torch.int32, **z),
                 counts=torch.zeros(2, dtype=torch.int32, **z))
    cache = fw.Cache8(fmt="int8", **store)
    K, V = rand(gen, 2, 2000, d), rand(gen, 2, 2000, d)
    pos = torch.cat([torch.arange(40, **z), torch.arange(2000, **z)]).to(torch.int32)
    fw.cache8_compact(cache, K, V, off([40, 2000]), pos)
    new = rand(gen, 2, 9, d)
    fw.cache8_append(cache, new, new)
    q = torch.randn(1, 1, 8, d, generator=gen, device="cuda").to(torch.bfloat16)
    out = fw.cache8_attend(cache, q, kv_heads=2)
    torch.cuda.synchronize()
    check_cell(cache, 1, 0, torch.cat([K[1], new[1]]))
    check_cell(cache, 0, 1, torch.cat([V[0, :40], new[0]]))
    check_attend(cache, q, out, 2, float(torch.tensor(1 / math.sqrt(d), dtype=torch.float32)))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_compact_many_cells_of_unlike_counts(fw, fmt):
    """Thousands of cells, most with fewer rows than a block, some empty; without a status too."""
    cells, T, d = 3001, 70, 64
    gen = torch.Generator("cuda").manual_seed(21)
    counts = torch.randint(0, 71, (cells,), generator=torch.Generator().manual_seed(21)) * (torch.arange(cells) % 3 != 1)
    counts[1500:1700] = 0
    counts = counts.tolist()
    K, V = rand(gen, cells, T, d), rand(gen, cells, T, d)
    pos, o = picks(gen, counts, T), off(counts)
    caches = [fw.cache8_empty(o, pos.numel(), d, fmt=fmt) for _ in range(2)]
    st = torch.empty(cells, dtype=torch.int32, device="cuda")
    fw.cache8_compact(caches[0], K, V, o, pos, status=st)
    fw.cache8_compact(caches[1], K, V, o, pos)
    torch.cuda.synchronize()
    assert not bool(st.any()) and caches[1].counts.tolist() == counts
    for h in list(range(0, cells, 97)) + [1499, 1500, 1699, 1700, cells - 1]:
        for c in caches:
            p = pos[int(o[h]):int(o[h + 1])].long()
            check_cell(c, h, 0, K[h, p])
            check_cell(c, h, 1, V[h, p])


def test_long_appends_report_and_refuse(fw):
    """Appends of several blocks: non-finite rows and full cells, cell by cell."""
    gen = torch.Generator("cuda").manual_seed(22)
    d, start, m = 128, [5, 40, 32], 150
    K = rand(gen, 3, 64, d)
    o, pos = off(start), torch.cat([torch.arange(c, device="cuda") for c in start]).to(torch.int32)
    cache = fw.cache8_empty(o, pos.numel(), d, room=m)
    fw.cache8_compact(cache, K, K, o, pos)
    cache.capacity[1] = 40 + m - 1
    new = rand(gen, 3, m, d)
    new[2, 77, 5] = float("inf")
    st = torch.empty(3, dtype=torch.int32, device="cuda")
    fw.cache8_append(cache, new, new, status=st)
    torch.cuda.synchronize()
    assert st.tolist() == [0, fw.FW_ERR_WORKSPACE, fw.FW_ERR_NONFINITE]
    for h in (0, 2):
        check_cell(cache, h, 1, torch.cat([K[h, :start[h]], new[h]]))
    check_cell(cache, 1, 0, K[1, :40])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kv_heads,g,m,counts", [(1, 4, 1, [40000]), (2, 8, 3, [70000, 20]), (8, 4, 5, [1] * 40 + [30000] + [3] * 39)])
def test_attend_one_long_cell(fw, d, kv_heads, g, m, counts):
    """One cell with nearly all rows, shared by most of the GPU's warps."""
    gen = torch.Generator("cuda").manual_seed(d + g)
    cache = filled(fw, gen, counts, d, "int8")
    q = (1.5 * torch.randn(len(counts) // kv_heads, m, kv_heads * g, d, generator=gen, device="cuda")).to(torch.bfloat16)
    out = fw.cache8_attend(cache, q, kv_heads=kv_heads)
    again = fw.cache8_attend(cache, q, kv_heads=kv_heads)
    torch.cuda.synchronize()
    check_attend(cache, q, out, kv_heads, float(torch.tensor(1 / math.sqrt(d), dtype=torch.float32)))
    assert torch.equal(out["o"], again["o"]) and torch.equal(out["lse"], again["lse"])


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("seqs,kv_heads,g,m", [(3, 8, 4, 1), (7, 4, 8, 2), (20, 3, 7, 1), (9, 8, 16, 1), (1, 14, 4, 9)])
def test_attend_cells_between_few_and_many(fw, fmt, d, seqs, kv_heads, g, m):
    """Short cells in clusters of every size, among them empty ones, and the calls around where the rule changes."""
    gen = torch.Generator("cuda").manual_seed(seqs)
    cells = seqs * kv_heads
    for top in (40, 1500, 6000):
        counts = [int(x) for x in torch.randint(0, top, (cells,), generator=torch.Generator().manual_seed(cells + top))]
        counts[1] = 0
        cache = filled(fw, gen, counts, d, fmt)
        q = (1.5 * torch.randn(seqs, m, kv_heads * g, d, generator=gen, device="cuda")).to(torch.bfloat16)
        out = fw.cache8_attend(cache, q, kv_heads=kv_heads)
        torch.cuda.synchronize()
        check_attend(cache, q, out, kv_heads, float(torch.tensor(1 / math.sqrt(d), dtype=torch.float32)))


@pytest.mark.parametrize("d,fmt", [(64, "int8"), (128, "e4m3")])
@pytest.mark.parametrize("offsets,total", [
    ([0, 100, 50, 150], 150), ([0, 500, 100, 600], 600), ([0, 40, 400, 80, 120], 400), ([0, 150, 0, 150, 0, 150], 150),
    ([0, 40, 80, 120, 160], 60), ([-5, 40, 80], 80), ([0, 40, -2 ** 62, 80, 2 ** 62, 80], 80), ([70, 33, 33, 0], 70)])
def test_compact_offsets_out_of_order_concern_their_cells_only(fw, offsets, total, d, fmt):
    """Cells whose offsets descend or leave the positions are refused, with a count of 0; all others get their rows, in a
    store that held others before."""
    gen = torch.Generator("cuda").manual_seed(total)
    cells, T = len(offsets) - 1, 600
    K, V = rand(gen, cells, T, d), rand(gen, cells, T, d)
    pos = torch.randint(0, T, (total,), generator=gen, device="cuda", dtype=torch.int32)
    o = torch.tensor(offsets, dtype=torch.int64, device="cuda")
    ok = [0 <= a <= b <= total for a, b in zip(offsets, offsets[1:])]
    for status in (torch.full((cells,), -1, dtype=torch.int32, device="cuda"), None):
        cache = fw.cache8_empty(off([600] * cells), 600 * cells, d, fmt=fmt)
        cache.counts.fill_(77)
        cache.k.view(torch.int8).fill_(17)
        fw.cache8_compact(cache, K, V, o, pos, status=status)
        torch.cuda.synchronize()
        if status is not None:
            assert status.tolist() == [0 if x else fw.FW_ERR_INVALID_ARG for x in ok]
        for h in range(cells):
            if ok[h]:
                p = pos[offsets[h]:offsets[h + 1]].long()
                check_cell(cache, h, 0, K[h, p])
                check_cell(cache, h, 1, V[h, p])
            else:
                assert int(cache.counts[h]) == 0
            b, n = int(cache.base[h]), int(cache.counts[h])
            assert bool((cache.k.view(torch.int8)[b + n:b + 600] == 17).all())


@pytest.mark.parametrize("bad", [[3], [1400], [5, 700, 1999], [511, 512, 1024]])
def test_compact_offsets_out_of_order_among_many_cells(fw, bad):
    cells, T, d = 2000, 70, 64
    gen = torch.Generator("cuda").manual_seed(bad[0])
    counts = torch.randint(0, 71, (cells,), generator=torch.Generator().manual_seed(bad[0])).tolist()
    K = rand(gen, cells, T, d)
    pos, o = picks(gen, counts, T), off(counts)
    cache = fw.cache8_empty(off([T] * cells), T * cells, d)
    cache.counts.fill_(9)
    for b in bad:  # (an offset that both of its cells cannot take)
        o[b] = pos.numel() + 1 + b
    st = torch.empty(cells, dtype=torch.int32, device="cuda")
    fw.cache8_compact(cache, K, K, o, pos, status=st)
    torch.cuda.synchronize()
    refused = sorted({c for b in bad for c in (b - 1, b)})
    assert torch.nonzero(st).flatten().tolist() == refused
    want = [0 if h in refused else c for h, c in enumerate(counts)]
    assert cache.counts.tolist() == want
    for h in [h for h in range(0, cells, 61) if want[h]] + [h for b in bad for h in (b - 3, b - 2, b + 1, b + 2) if h < cells and want[h]]:
        check_cell(cache, h, 0, K[h, pos[int(o[h]):int(o[h + 1])].long()])


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("top", [1.0, 2.0 ** 100, 2.9e38, 3.0e38, 3.3895313892515355e38])
def test_infinities_beside_the_largest_values(fw, fmt, top):
    """Infinities become the largest code of their sign and NaN 0 whatever the block's scale is, in the compaction and in an
    append."""
    gen = torch.Generator("cuda").manual_seed(17)
    d, n = 64, 40
    K = ((torch.rand(1, n, d, generator=gen, device="cuda") * 2 - 1) * top).to(torch.bfloat16)
    K[0, 0, 0] = K[0, 35, 1] = top
    K[0, 3, 5], K[0, 31, 63], K[0, 7, 7], K[0, 36, 8], K[0, 39, 9] = (float(x) for x in ("inf", "-inf", "nan", "-inf", "nan"))
    caches = [fw.cache8_empty(off([n]), n, d, fmt=fmt) for _ in range(2)]
    st = torch.empty(2, dtype=torch.int32, device="cuda")
    fw.cache8_compact(caches[0], K, K, off([n]), torch.arange(n, dtype=torch.int32, device="cuda"), status=st[:1])
    fw.cache8_append(caches[1], K[:, :32].contiguous(), K[:, :32].contiguous())
    fw.cache8_append(caches[1], K[:, 32:].contiguous(), K[:, 32:].contiguous(), status=st[1:])
    torch.cuda.synchronize()
    assert st.tolist() == [fw.FW_ERR_NONFINITE] * 2
    for b in (0, 32):
        val, sc = quantise64(K[0, b:b + 32], fmt)
        for c in caches:
            at = int(c.base[0]) + b
            for codes, scales in ((c.k, c.k_scale), (c.v, c.v_scale)):
                assert float(scales[at // 32]) == sc and torch.equal(codes[at:at + val.shape[0]].double(), val)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("m", [1, 3])
def test_attend_on_a_part_of_a_large_store(fw, d, m):
    """A layer's cells within a store whose other cells hold most of the rows, and the same cells in a store of their own."""
    gen = torch.Generator("cuda").manual_seed(d + m)
    counts = [3000, 17, 0, 2900, 3100, 64, 1, 2048]
    whole = filled(fw, gen, [70000] + counts + [40000], d, "e4m3")
    part = whole.part(1, 8)
    lo, hi = int(whole.base[1]), int(whole.base[9])
    own = fw.Cache8(fmt="e4m3", k=whole.k[lo:hi].clone(), v=whole.v[lo:hi].clone(), k_scale=whole.k_scale[lo // 32:hi // 32].clone(),
                    v_scale=whole.v_scale[lo // 32:hi // 32].clone(), k_tail=part.k_tail.clone(), v_tail=part.v_tail.clone(),
                    base=part.base - lo, capacity=part.capacity.clone(), counts=part.counts.clone())
    q = (1.5 * torch.randn(1, m, 32, d, generator=gen, device="cuda")).to(torch.bfloat16)
    for cache in (part, own):
        out = fw.cache8_attend(cache, q, kv_heads=8)
        torch.cuda.synchronize()
        check_attend(cache, q, out, 8, float(torch.tensor(1 / math.sqrt(d), dtype=torch.float32)))

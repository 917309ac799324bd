"""Norms and rotation of queries and keys against the formula in 64 bits."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def fw():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2608_25230_gb300 import fw as _fw

    return _fw


def rotate64(x, w, eps, pos, inv_freq, interleaved):
    """(y, |y_a| + |y_b| of each column's pair) in 64 bits."""
    y = x.double()
    if eps is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps)
        if w is not None:
            y = y * w.double()
    half = inv_freq.numel()
    out, mag = y.clone(), y.abs()
    t = (pos.double()[:, None] * inv_freq.double())[:, None]
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    u, v = y[..., a], y[..., b]
    out[..., a], out[..., b] = u * torch.cos(t) - v * torch.sin(t), v * torch.cos(t) + u * torch.sin(t)
    mag[..., a] = mag[..., b] = u.abs() + v.abs()
    return out, mag


def check(got, want):
    """One rounding to bf16 (2^-8 of the value), before it fp32: the mean of at most 256 squares is summed in 16 steps
    a lane and 4 over lanes (2^-19 relative with the root and three products), cosine and sine are off by at most
    2 pi 2^-26 + 2^-24 for the angle and 2^-22 themselves, one product and one sum: 2^-18 of the pair's magnitude."""
    y, mag = want
    tol = 2.0 ** -8 * y.abs() + 2.0 ** -18 * mag * (1 + 2.0 ** -8) + 2.0 ** -133
    err = (got.double() - y).abs()
    assert bool((err <= tol).all()), f"off by {float((err / tol).max())} of the bound"


def freqs(rot, base=5e5):
    return (base ** (-2 * torch.arange(rot // 2, device="cuda", dtype=torch.float64) / max(rot, 1))).float()


def packed(gen, rows, hq, hk, d):
    """A projection's queries, keys and values side by side."""
    x = torch.randn(rows, hq + 2 * hk, d, generator=gen, device="cuda")
    x *= torch.exp2(torch.randint(-6, 7, (rows, hq + 2 * hk, 1), generator=gen, device="cuda"))
    x = x.to(torch.bfloat16)
    return x[:, :hq], x[:, hq:hq + hk]


@pytest.mark.parametrize("d,rot", [(16, 16), (48, 16), (64, 64), (64, 32), (64, 0), (80, 48), (96, 96), (128, 128), (128, 96),
                                   (128, 32), (192, 64), (256, 256), (240, 240)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,hq,hk", [(1, 1, 1), (3, 7, 3), (67, 32, 8), (300, 5, 1)])
def test_against_64_bits(fw, d, rot, interleaved, rows, hq, hk):
    gen = torch.Generator("cuda").manual_seed(d + rot + rows)
    q, k = packed(gen, rows, hq, hk, d)
    pos = torch.randint(-5000, 1 << 20, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    f = freqs(rot)
    for eps, dtype in ((1e-6, torch.bfloat16), (0.0, torch.float32), (1e-2, None), (None, None)):
        w = [None, None] if dtype is None else [torch.randn(d, generator=gen, device="cuda").to(dtype) for _ in "qk"]
        a, b = fw.qk_rotate(q, k, pos, f, q_weight=w[0], k_weight=w[1], eps=eps, interleaved=interleaved)
        torch.cuda.synchronize()
        check(a, rotate64(q, w[0], eps, pos, f, interleaved))
        check(b, rotate64(k, w[1], eps, pos, f, interleaved))


def test_far_positions_and_odd_frequencies(fw):
    """Angles of the farthest positions, of frequencies above one and below zero, of zero and of subnormals."""
    gen = torch.Generator("cuda").manual_seed(9)
    d, rows = 64, 200
    q, k = packed(gen, rows, 2, 1, d)
    pos = torch.randint(-(1 << 31), (1 << 31) - 1, (rows,), generator=gen, device="cuda").to(torch.int32)
    pos[:4] = torch.tensor([(1 << 31) - 1, -(1 << 31), 0, -1], dtype=torch.int32)
    f = torch.rand(32, generator=gen, device="cuda") * 2
    f[:12] = torch.tensor([1.0, -1.0, math.pi, -2.5e-9, 0.0, -0.0, 1e-40, 1e-30, 6.2831855, 100.0, -127.5, 1e-12])
    for inter in (False, True):
        a, b = fw.qk_rotate(q, k, pos, f, interleaved=inter)
        torch.cuda.synchronize()
        check(a, rotate64(q, None, None, pos, f, inter))
        check(b, rotate64(k, None, None, pos, f, inter))


def test_in_place_head_major_and_broadcast(fw):
    gen = torch.Generator("cuda").manual_seed(4)
    rows, hq, hk, d = 33, 6, 2, 128
    q, k = packed(gen, rows, hq, hk, d)
    pos, f = torch.arange(rows, dtype=torch.int32, device="cuda") + 100000, freqs(d)
    want = [rotate64(x, None, 1e-5, pos, f, False) for x in (q, k)]
    # keys straight into a cache [heads][tokens][d], queries in tokens' order
    cache = torch.zeros(hk, rows + 7, d, dtype=torch.bfloat16, device="cuda")
    out = (torch.empty(rows, hq, d, dtype=torch.bfloat16, device="cuda"), cache[:, 3:3 + rows].transpose(0, 1))
    fw.qk_rotate(q, k, pos, f, eps=1e-5, out=out)
    torch.cuda.synchronize()
    check(out[0], want[0])
    check(out[1], want[1])
    assert not bool(cache[:, :3].any()) and not bool(cache[:, 3 + rows:].any())
    # one row for all positions
    one = q[:1].expand(rows, hq, d)
    a, none = fw.qk_rotate(one, None, pos, f, eps=1e-5)
    torch.cuda.synchronize()
    assert none is None
    check(a, rotate64(one, None, 1e-5, pos, f, False))
    # in place, values behind the keys untouched
    base = q._base if q._base is not None else q
    values = base[:, hq + hk:].clone()
    a, b = fw.qk_rotate(q, k, pos, f, eps=1e-5, out=(q, k))
    torch.cuda.synchronize()
    assert a is q and b is k
    check(q, want[0])
    check(k, want[1])
    assert torch.equal(base[:, hq + hk:], values)
    a, b = fw.qk_rotate(q[:0], k[:0], pos[:0], f)
    assert a.shape == (0, hq, d) and b.shape == (0, hk, d)


def test_values_that_are_not_finite_stay_in_their_heads(fw):
    gen = torch.Generator("cuda").manual_seed(5)
    rows, hq, hk, d = 9, 4, 4, 64
    q, k = packed(gen, rows, hq, hk, d)
    pos, f = torch.arange(rows, dtype=torch.int32, device="cuda"), freqs(d)
    want = [rotate64(x, None, 1e-6, pos, f, False) for x in (q, k)]
    q[2, 1, 5], q[3, 0, 0], k[4, 3, 63] = float("nan"), float("inf"), float("-inf")
    a, b = fw.qk_rotate(q, k, pos, f, eps=1e-6)
    torch.cuda.synchronize()
    for got, w, heads in ((a, want[0], [(2, 1), (3, 0)]), (b, want[1], [(4, 3)])):
        keep = torch.ones(got.shape[:2], dtype=torch.bool, device="cuda")
        for r, h in heads:
            keep[r, h] = False
        assert bool(torch.isnan(got[~keep]).any(-1).all())
        check(got[keep], (w[0][keep], w[1][keep]))
    # a frequency that is none: its pair of columns alone
    f2 = f.clone()
    f2[3] = float("inf")
    q, k = packed(gen, rows, hq, hk, d)
    a, _ = fw.qk_rotate(q, k, pos, f2)
    torch.cuda.synchronize()
    cols = torch.zeros(d, dtype=torch.bool, device="cuda")
    cols[3] = cols[35] = True
    assert bool(torch.isnan(a[..., cols]).all())
    w = rotate64(q, None, None, pos, f, False)
    check(a[..., ~cols], (w[0][..., ~cols], w[1][..., ~cols]))


def test_on_a_side_stream_and_in_a_graph(fw):
    gen = torch.Generator("cuda").manual_seed(6)
    rows, hq, hk, d = 40, 8, 2, 64
    q, k = packed(gen, rows, hq, hk, d)
    pos, f = torch.arange(rows, dtype=torch.int32, device="cuda"), freqs(d)
    a, b = fw.qk_rotate(q, k, pos, f, eps=1e-6)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c, e = fw.qk_rotate(q, k, pos, f, eps=1e-6, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a, c) and torch.equal(b, e)
    out = (torch.empty_like(a), torch.empty_like(b))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fw.qk_rotate(q, k, pos, f, eps=1e-6, out=out)
    pos += 77
    g.replay()
    torch.cuda.synchronize()
    check(out[0], rotate64(q, None, 1e-6, pos, f, False))
    check(out[1], rotate64(k, None, 1e-6, pos, f, False))


@pytest.mark.parametrize("rows,hq,hk,d,rot", [(5003, 32, 8, 128, 128), (5003, 7, 3, 256, 96), (5000, 3, 50, 48, 48), (1500, 40, 9, 64, 64),
                                              (1500, 41, 7, 208, 208), (700, 64, 9, 128, 32), (6001, 29, 0, 128, 0),
                                              (2501, 33, 15, 80, 16)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_warps_that_take_many_heads(fw, rows, hq, hk, d, rot, interleaved):
    """So many tokens that a warp takes several chunks of a token's heads, all or every 2nd to 7th of up to 25: the heads that it asks
    for ahead come round in their places, and it goes over from queries to keys, with full and ragged chunks, not in place and in
    place."""
    gen = torch.Generator("cuda").manual_seed(rows + d)
    q, k = packed(gen, rows, hq, hk, d)
    base = q._base
    pos = torch.randint(-5000, 1 << 20, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    f = freqs(rot)
    w = [torch.randn(d, generator=gen, device="cuda") for _ in "qk"]
    for eps, (wq, wk) in ((1e-6, w), (None, (None, None))):
        want = [rotate64(x, y, eps, pos, f, interleaved) for x, y in ((q, wq), (k, wk))]
        args = dict(q_weight=wq, k_weight=wk if hk else None, eps=eps, interleaved=interleaved)
        a, b = fw.qk_rotate(q, k if hk else None, pos, f, **args)
        torch.cuda.synchronize()
        check(a, want[0])
        if hk:
            check(b, want[1])
    values = base[:, hq + hk:].clone()
    fw.qk_rotate(q, k if hk else None, pos, f, out=(q, k if hk else None), **args)
    torch.cuda.synchronize()
    assert torch.equal(q, a) and (not hk or torch.equal(k, b)) and torch.equal(base[:, hq + hk:], values)

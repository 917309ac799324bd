"""Attention over packed prompts (fw_prompt_attention) against plain attention in 64 bits."""
import math

import pytest

from tests.attention64 import attend64, check_rows

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U_P = 2.0 ** -8  # weights are rounded to bf16 for the second product


@pytest.fixture(scope="module")
def fw():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2608_25230_gb300 import fw as _fw

    return _fw


def cu(lens, first=0):
    t = [first]
    for n in lens:
        t.append(t[-1] + n)
    return torch.tensor(t, dtype=torch.int32, device="cuda")


def rand(gen, *shape, amp=1.0):
    return (amp * torch.randn(*shape, generator=gen, device="cuda")).to(torch.bfloat16)


def check(out, q, k, v, lens, scale, first=(0, 0), rows=None):
    """Every row (or, of long sequences, the last `rows`, the first and some between) of every head."""
    g = q.shape[1] // k.shape[1]
    aq, ak = first
    for lq, lk in lens:
        pos = torch.arange(lq, device="cuda")
        if rows is not None and lq > 3 * rows:
            pos = torch.cat([pos[:rows], pos[lq // 2:lq // 2 + rows], pos[-rows:]])
        seen = (lk - lq + 1 + pos).clamp(max=lk)
        for h in range(q.shape[1]):
            K, V = k[ak:ak + lk, h // g].double(), v[ak:ak + lk, h // g].double()
            want = attend64(q[aq + pos, h].double(), K, V, seen, scale)
            check_rows(out["o"][aq + pos, h], out["lse"][aq + pos, h], want, U_P)
        aq, ak = aq + lq, ak + lk
    assert bool((out["status"] == 0).all())


LENS = {
    "one": [(1, 1)], "short": [(17, 17)], "tile": [(128, 128)], "ragged": [(129, 129), (1, 1), (0, 0), (255, 255), (64, 64)],
    "behind": [(5, 300), (64, 1064), (1, 777), (130, 131)], "empty_rows": [(10, 4), (3, 0), (300, 150), (7, 7)],
    "long": [(2049, 2049), (513, 3000)],
}


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", list(LENS))
@pytest.mark.parametrize("hk,g", [(1, 1), (2, 4), (2, 3), (1, 8)])
def test_prompt_lengths(fw, lens, hk, g, d):
    gen = torch.Generator("cuda").manual_seed(hk * 100 + g + d)
    lens = LENS[lens]
    lq, lk = [a for a, _ in lens], [b for _, b in lens]
    q, k, v = (rand(gen, sum(lq), hk * g, d, amp=1.5), rand(gen, sum(lk), hk, d), rand(gen, sum(lk), hk, d))
    out = fw.prompt_attention(q, k, v, cu(lq), cu(lk))
    torch.cuda.synchronize()
    check(out, q, k, v, lens, 1 / math.sqrt(d))


@pytest.mark.parametrize("hk,g,d", [(1, 5, 64), (3, 7, 128), (1, 16, 128), (2, 33, 64), (1, 100, 64), (1, 128, 128), (8, 2, 64)])
def test_prompt_groups(fw, hk, g, d):
    gen = torch.Generator("cuda").manual_seed(g)
    lens = [(37, 37), (66, 200), (2, 1)]
    q, k, v = (rand(gen, 105, hk * g, d, amp=1.5), rand(gen, 238, hk, d), rand(gen, 238, hk, d))
    out = fw.prompt_attention(q, k, v, cu([37, 66, 2]), cu([37, 200, 1]), scale=0.2)
    torch.cuda.synchronize()
    check(out, q, k, v, lens, float(torch.tensor(0.2, dtype=torch.float32)))


@pytest.mark.parametrize("d", [64, 128])
def test_prompt_strides(fw, d):
    """Slices of one fused projection, and the head-major layout of the framework's caches."""
    gen = torch.Generator("cuda").manual_seed(d)
    lens, hk, g = [(150, 150), (33, 33)], 2, 4
    qkv = rand(gen, 183, hk * (g + 2), d)
    q, k, v = qkv[:, :hk * g], qkv[:, hk * g:hk * (g + 1)], qkv[:, hk * (g + 1):]
    out = fw.prompt_attention(q, k, v, cu([150, 33]))
    torch.cuda.synchronize()
    check(out, q, k, v, lens, 1 / math.sqrt(d))
    K, V, Q = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (k, v, q))
    again = fw.prompt_attention(Q, K, V, cu([150, 33]))
    torch.cuda.synchronize()
    assert torch.equal(out["o"], again["o"]) and torch.equal(out["lse"], again["lse"])


@pytest.mark.parametrize("d,T", [(128, 9001), (64, 12345)])
def test_prompt_one_long_sequence(fw, d, T):
    gen = torch.Generator("cuda").manual_seed(T)
    q, k, v = rand(gen, T, 4, d, amp=2.0), rand(gen, T, 1, d), rand(gen, T, 1, d)
    out = fw.prompt_attention(q, k, v, cu([T]))
    torch.cuda.synchronize()
    check(out, q, k, v, [(T, T)], 1 / math.sqrt(d), rows=150)


@pytest.mark.parametrize("d", [64, 128])
def test_prompt_large_logits_rising_and_falling(fw, d):
    """Logits whose running maximum moves by hundreds from tile to tile, both ways."""
    gen = torch.Generator("cuda").manual_seed(5)
    T = 1000
    q, k, v = rand(gen, T, 2, d), rand(gen, T, 1, d), rand(gen, T, 1, d)
    ramp = torch.linspace(-30, 30, T, device="cuda")[:, None, None].to(torch.bfloat16)
    q[..., 0] = 8
    for sgn in (1, -1):
        kk = k.clone()
        kk[..., :1] = sgn * ramp
        out = fw.prompt_attention(q, kk, v, cu([T]), scale=1.0)
        torch.cuda.synchronize()
        check(out, q, kk, v, [(T, T)], 1.0)


@pytest.mark.parametrize("d", [64, 128])
def test_prompt_unseen_keys_have_no_part(fw, d):
    """NaN and infinities around a sequence's rows, and at keys that earlier rows do not see."""
    gen = torch.Generator("cuda").manual_seed(9)
    nan, inf = float("nan"), float("inf")
    lens = [(100, 100), (70, 90), (200, 200)]
    q, k, v = rand(gen, 380, 8, d), rand(gen, 420, 2, d), rand(gen, 420, 2, d)
    clean = fw.prompt_attention(q, k, v, cu([100, 70, 200], 5), cu([100, 90, 200], 10))
    for x in (k, v):
        x[:10], x[400:] = nan, inf
    q[:5], q[375:] = nan, nan
    dirty = fw.prompt_attention(q, k, v, cu([100, 70, 200], 5), cu([100, 90, 200], 10))
    torch.cuda.synchronize()
    check(dirty, q, k, v, lens, 1 / math.sqrt(d), first=(5, 10))
    assert torch.equal(clean["o"][5:375], dirty["o"][5:375])
    # the key at position 60 of the first sequence and at 150 of the last, in the values only, then in the keys
    for a, (bad, at) in enumerate([(nan, 10 + 60), (inf, 10 + 190 + 150), (-inf, 10 + 190 + 150)]):
        for x in (v, k):
            y = x.clone()
            y[at, 1, 3 + a] = bad
            out = fw.prompt_attention(q, y if x is k else k, y if x is v else v, cu([100, 70, 200], 5),
                                      cu([100, 90, 200], 10))
            torch.cuda.synchronize()
            lo, hi = (5, 105) if at < 110 else (175, 375)  # rows of the sequence
            first = lo + at - (10 if at < 110 else 200)    # the first row that sees the key
            o, co = out["o"], clean["o"]
            assert torch.equal(o[lo:first], co[lo:first]) and torch.equal(o[hi:375], co[hi:375])
            assert torch.equal(o[5:lo], co[5:lo]) and torch.equal(o[first:hi, :4], co[first:hi, :4])
            hit = o[first:hi, 4:]
            if x is v:
                assert not bool(torch.isfinite(hit[..., 3 + a]).any())
                rest = [c for c in range(d) if c != 3 + a]
                assert torch.equal(hit[..., rest], co[first:hi, 4:][..., rest])
                if bad == bad:
                    assert bool((hit[..., 3 + a] == bad).all())
            elif bad != bad:
                assert bool(torch.isnan(hit).all())


def test_prompt_no_keys_and_no_rows(fw):
    q = torch.ones(6, 4, 64, dtype=torch.bfloat16, device="cuda")
    kv = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    out = fw.prompt_attention(q, kv, kv, cu([6]), cu([0]))
    torch.cuda.synchronize()
    assert not bool(out["o"].any()) and bool(torch.isneginf(out["lse"]).all()) and out["status"].tolist() == [0]
    none = fw.prompt_attention(q[:0], kv, kv, cu([0, 0]), cu([0, 0]))
    torch.cuda.synchronize()
    assert none["o"].numel() == 0 and none["status"].tolist() == [0, 0]


def test_prompt_repeats_streams_and_optional_outputs(fw):
    gen = torch.Generator("cuda").manual_seed(2)
    lens = [700, 1, 300, 45]
    q, k, v = rand(gen, 1046, 8, 128), rand(gen, 1046, 2, 128), rand(gen, 1046, 2, 128)
    a = fw.prompt_attention(q, k, v, cu(lens))
    side = torch.cuda.Stream()
    bounds = cu(lens)
    side.wait_stream(torch.cuda.current_stream())
    b = fw.prompt_attention(q, k, v, bounds, stream=side)
    only = dict(o=torch.empty_like(q))
    fw.prompt_attention(q, k, v, cu(lens), out=only)
    torch.cuda.synchronize()
    assert torch.equal(a["o"], b["o"]) and torch.equal(a["lse"], b["lse"]) and torch.equal(a["o"], only["o"])


def test_prompt_bad_bounds_are_reported(fw):
    q = torch.ones(40, 2, 64, dtype=torch.bfloat16, device="cuda")
    for bounds in ([0, 20, 10, 40], [0, 20, 41], [-1, 20, 40]):
        t = torch.tensor(bounds, dtype=torch.int32, device="cuda")
        out = fw.prompt_attention(q, q[:, :1], q[:, :1], t)
        torch.cuda.synchronize()
        bad = [b < a or a < 0 or b > 40 for a, b in zip(bounds, bounds[1:])]
        got = out["status"].tolist()
        assert [s == fw.FW_ERR_INVALID_ARG for s in got] == bad


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[(1, 20000)], [(17, 4097)], [(3, 9000), (130, 7000)], [(300, 2100), (1, 4000), (0, 9000)],
                                  [(64, 1024)], [(40, 20), (5, 9000)]])
@pytest.mark.parametrize("hk,g", [(1, 1), (2, 4), (1, 12)])
def test_prompt_few_rows_against_long_keys(fw, hk, g, d, lens):
    """Slots so few that their keys are split over several CTAs and joined."""
    gen = torch.Generator("cuda").manual_seed(hk + g + d)
    lq, lk = [a for a, _ in lens], [b for _, b in lens]
    q, k, v = rand(gen, sum(lq), hk * g, d, amp=1.5), rand(gen, sum(lk), hk, d), rand(gen, sum(lk), hk, d)
    out = fw.prompt_attention(q, k, v, cu(lq), cu(lk))
    torch.cuda.synchronize()
    check(out, q, k, v, lens, 1 / math.sqrt(d))
    again = fw.prompt_attention(q, k, v, cu(lq), cu(lk))
    torch.cuda.synchronize()
    assert torch.equal(out["o"], again["o"]) and torch.equal(out["lse"], again["lse"])


@pytest.mark.parametrize("d", [64, 128])
def test_prompt_unseen_values_with_keys_split(fw, d):
    gen = torch.Generator("cuda").manual_seed(31)
    T, lq = 6000, 90
    q, k, v = rand(gen, lq, 4, d), rand(gen, T, 2, d), rand(gen, T, 2, d)
    clean = fw.prompt_attention(q, k, v, cu([lq]), cu([T]))
    for at, bad in ((T - 50, float("nan")), (T - lq, float("inf")), (T - 1, float("-inf")), (700, float("inf"))):
        y = v.clone()
        y[at, 0, 5] = bad
        out = fw.prompt_attention(q, k, y, cu([lq]), cu([T]))
        torch.cuda.synchronize()
        first = max(0, at - (T - lq))
        o, co = out["o"], clean["o"]
        assert torch.equal(o[:first], co[:first]) and torch.equal(o[:, 2:], co[:, 2:])
        assert not bool(torch.isfinite(o[first:, :2, 5]).any())
        rest = [c for c in range(d) if c != 5]
        assert torch.equal(o[first:, :2][..., rest], co[first:, :2][..., rest])


@pytest.mark.parametrize("cu_q,cu_k", [([0, 0, 0], [0, 5, 9]), ([0, 1, 0], [0, 5, 9]), ([0, 0, 0], [0, 9, 5]), ([0, 0, 0], [0, 5, 10]),
                                       ([-1, 0, 0], [0, 5, 9]), ([0, 0, 0], [-2, 5, 9])])
def test_prompt_bounds_are_reported_without_any_rows_too(fw, cu_q, cu_k):
    """No query rows at all: the sequences' bounds are looked at all the same."""
    q = torch.ones(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    kv = torch.ones(9, 2, 64, dtype=torch.bfloat16, device="cuda")
    a, b = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (cu_q, cu_k))
    out = fw.prompt_attention(q, kv, kv, a, b)
    torch.cuda.synchronize()
    bad = [not (0 <= a0 <= a1 <= 0 and 0 <= b0 <= b1 <= 9) for a0, a1, b0, b1 in zip(cu_q, cu_q[1:], cu_k, cu_k[1:])]
    assert out["status"].tolist() == [fw.FW_ERR_INVALID_ARG if x else 0 for x in bad]


def fills_two_tiles(hk, g, lq):
    """Whether the CTAs of two tiles fill more than half of the SMs (with d = 128 they are taken then)."""
    return (sum(lq) // (2 * (128 // g)) + len(lq)) * hk * 2 > torch.cuda.get_device_properties(0).multi_processor_count


@pytest.mark.parametrize("hk,g", [(8, 1), (8, 3), (4, 7)])
def test_prompt_two_tiles_a_cta_rows_and_groups(fw, hk, g):
    """Rows that see nothing in the first tile of a CTA, in both and in part of one, sequences without keys, groups that do not
    divide a tile."""
    lens = [(300, 120), (900, 400), (513, 0), (1200, 1200), (40, 39), (0, 7), (257, 258), (700, 900)]
    lq, lk = [a for a, _ in lens], [b for _, b in lens]
    assert fills_two_tiles(hk, g, lq)
    gen = torch.Generator("cuda").manual_seed(10 * hk + g)
    q, k, v = rand(gen, sum(lq), hk * g, 128, amp=1.5), rand(gen, sum(lk), hk, 128), rand(gen, sum(lk), hk, 128)
    out = fw.prompt_attention(q, k, v, cu(lq), cu(lk))
    torch.cuda.synchronize()
    check(out, q, k, v, lens, 1 / math.sqrt(128))


@pytest.mark.parametrize("hk,g", [(8, 1), (8, 3)])
def test_prompt_two_tiles_a_cta_large_logits(fw, hk, g):
    """The running maximum moves by hundreds from block to block, both ways."""
    gen = torch.Generator("cuda").manual_seed(15)
    T = 2700
    assert fills_two_tiles(hk, g, [T])
    q, k, v = rand(gen, T, hk * g, 128), rand(gen, T, hk, 128), rand(gen, T, hk, 128)
    ramp = torch.linspace(-60, 60, T, device="cuda")[:, None, None].to(torch.bfloat16)
    q[..., 0] = 8
    for sgn in (1, -1):
        kk = k.clone()
        kk[..., :1] = sgn * ramp
        out = fw.prompt_attention(q, kk, v, cu([T]), scale=1.0)
        torch.cuda.synchronize()
        check(out, q, kk, v, [(T, T)], 1.0, rows=300)


@pytest.mark.parametrize("hk,g", [(8, 1), (8, 3)])
def test_prompt_two_tiles_a_cta_unseen_values(fw, hk, g):
    """Values that are not finite, at keys that some rows of a CTA do not see: up to three blocks of them with one head a
    key head, whose CTAs hold 256 tokens."""
    gen = torch.Generator("cuda").manual_seed(19)
    lens = [(1300, 1300), (700, 900), (1000, 1000)]
    lq, lk = [a for a, _ in lens], [b for _, b in lens]
    assert fills_two_tiles(hk, g, lq)
    q, k, v = rand(gen, sum(lq), hk * g, 128), rand(gen, sum(lk), hk, 128), rand(gen, sum(lk), hk, 128)
    clean = fw.prompt_attention(q, k, v, cu(lq), cu(lk))
    torch.cuda.synchronize()
    check(clean, q, k, v, lens, 1 / math.sqrt(128), rows=100)
    nan, inf = float("nan"), float("inf")
    for seq, at, bad in ((0, 130, nan), (0, 255, inf), (0, 256, -inf), (1, 201, nan), (1, 330, inf), (1, 455, nan), (1, 456, -inf),
                         (2, 511, nan), (2, 999, inf), (2, 0, nan)):
        y = v.clone()
        y[sum(lk[:seq]) + at, 1, 77] = bad
        out = fw.prompt_attention(q, k, y, cu(lq), cu(lk))
        torch.cuda.synchronize()
        first = sum(lq[:seq]) + max(0, at - (lk[seq] - lq[seq]))  # rows that see it: first .. end of the sequence's
        end = sum(lq[:seq + 1])
        o, co = out["o"], clean["o"]
        assert torch.equal(o[:first], co[:first]) and torch.equal(o[end:], co[end:])
        hit, was = o[first:end], co[first:end]
        heads = torch.arange(hk * g, device="cuda") // g == 1
        assert torch.equal(hit[:, ~heads], was[:, ~heads])
        cols = torch.arange(128, device="cuda") != 77
        assert torch.equal(hit[:, heads][..., cols], was[:, heads][..., cols])
        assert not bool(torch.isfinite(hit[:, heads][..., 77]).any())
        assert torch.equal(out["lse"], clean["lse"])

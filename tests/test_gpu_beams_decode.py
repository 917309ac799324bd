"""Rotation, pages and their attention as a decoding program uses them together: the example's run against the same steps
on plain rows in 64 bits."""
import pytest

from tests.attention64 import attend64, check_rows

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("kw", [dict(tokens=500, layers=2, beams=3, kv_heads=2, group=3, d=64, steps=9, page_rows=16),
                                dict(tokens=1111, layers=1, beams=4, kv_heads=4, group=4, d=128, steps=12, page_rows=32),
                                dict(tokens=70, layers=3, beams=1, kv_heads=1, group=8, d=128, steps=6, page_rows=128)])
def test_beams_against_plain_rows(kw):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from examples import beams_decode

    r = beams_decode.run(**kw)
    torch.cuda.synchronize()
    assert not any(bool(s.any()) for s in r["statuses"])
    layers, beams, hk, g, d = r["shape"]
    # every cell's rows, as the steps say
    off, pos = r["kept"]["offsets"].tolist(), r["kept"]["kept_pos"].long()
    rows = [None] * (layers * beams * hk)
    for c in range(layers * hk):
        p = pos[off[c]:off[c + 1]]
        rows[c // hk * beams * hk + c % hk] = (r["K"][c, p], r["V"][c, p])
    outs = iter(r["decoded"])
    for what, *x in r["record"]:
        if what == "fork":
            rows = [rows[s] for s in x[0].tolist()]
        elif what == "keep":
            rows = [(k[torch.tensor(t, device="cuda")], v[torch.tensor(t, device="cuda")]) for (k, v), t in zip(rows, x[0])]
        else:
            layer, new_k, new_v, q = x
            out = next(outs)
            for b in range(beams):
                for h in range(hk):
                    c = (layer * beams + b) * hk + h
                    k, v = rows[c] = tuple(torch.cat([old, new[b, :, h]]) for old, new in zip(rows[c], (new_k, new_v)))
                    mine = slice(h * g, (h + 1) * g)
                    seen = torch.full((g,), k.shape[0], device="cuda")
                    want = attend64(q[b, mine].double(), k.double(), v.double(), seen, r["scale"])
                    check_rows(out[b, mine], None, want, 2.0 ** -16)
    # and what the pages hold in the end
    p = r["pages"]
    P = p.page_rows
    for c, (k, v) in enumerate(rows):
        assert int(p.counts[c]) == k.shape[0]
        t = torch.arange(k.shape[0], device="cuda")
        page = p.table[c].long()[t // P]
        assert torch.equal(p.k[page, t % P], k) and torch.equal(p.v[page, t % P], v)
    refs = torch.zeros_like(p.refs)
    for c, n in enumerate(p.held.tolist()):
        refs.index_add_(0, p.table[c, :n].long(), torch.ones(n, dtype=torch.int32, device="cuda"))
    assert torch.equal(refs, p.refs)
    free = (p.free[:, None] >> torch.arange(32, device="cuda", dtype=torch.int32) & 1).flatten()[:p.num_pages]
    assert torch.equal(free == 1, p.refs == 0)

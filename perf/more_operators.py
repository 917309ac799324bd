"""The operators around a cache held in pages, with their plain forms and the calls
they are measured on: norms and rotation of queries and keys, appends to the pages,
compaction into and inside them, forks, and the attention of new tokens over them.

Where `own` is false, run() computes them from elementary torch operations in 32 bits
(the rotation's angles in 64); where it is true, it makes the library's calls.  Both
write the same tensors.

The pages: pools k, v [pages][rows of a page][d], and int32 books: per cell (a KV head
of a sequence) a table of pages, how many of its entries are held and how many rows are
filled; per page how many entries name it; a bit per page that none does; and the page
at which the search for free ones begins.  Free pages are handed out in ascending
order from there, round the end, to cells in order: which page goes where does not
depend on what computes it.  All books lie in one tensor, so that a program takes a step
back by one copy of it; that is how every pass here begins.
"""
import math
import random

import torch

own = False


# ------------------------------------------------------------------------ cases
def listed():
    return [
        # a draft of 5 tokens of 8 sequences at far positions, half of each head's 64 columns rotated in neighbouring
        # pairs: one small launch
        dict(name="rotate_draft", op="rotate", rows=40, kv_heads=2, group=7, d=64, rot=32, pairs="next", norm=True, far=1 << 20),
        # a prompt chunk of an odd number of tokens, 32 query and 8 KV heads out of one projection
        dict(name="rotate_prompt", op="rotate", rows=16381, kv_heads=8, group=4, d=128, rot=128, pairs="half", norm=True,
             far=1 << 17),
        # one decoded token of 32 sequences, every fourth of which was just forked from its neighbour
        dict(name="append_token", op="append", seqs=32, kv_heads=8, m=1, length=700, page=32, d=128, twins=4),
        # a prompt chunk of 509 tokens of 4 sequences, small pages
        dict(name="append_chunk", op="append", seqs=4, kv_heads=8, m=509, length=1200, page=16, d=64, twins=0),
        # a whole cache (32 layers x 8 heads) of a prompt into pages, an eighth of its tokens kept
        dict(name="compact_prompt", op="compact", cells=256, T=32768, keep=0.125, page=32, d=128),
        # eight sequences evicted again while they decode: half of the rows of each head's pages kept
        dict(name="keep_decoding", op="keep", cells=64, T=7001, keep=0.5, page=64, d=128),
        # beams of 3 prompts change places, 4 each
        dict(name="fork_beams", op="fork", seqs=12, kv_heads=2, length=300, page=16, d=64, family=4),
        # 256 sequences that share long prefixes, 8 heads each: some end, others fork into their place
        dict(name="fork_batch", op="fork", seqs=256, kv_heads=8, length=8192, page=32, d=64, family=8),
        # one layer of one sequence: a latency-bound decode step
        dict(name="attend_layer", op="attend", seqs=1, kv_heads=8, group=4, m=1, length=4096, page=16, d=128),
        # a draft of 5 tokens verified for 8 sequences of odd lengths
        dict(name="attend_draft", op="attend", seqs=8, kv_heads=8, group=4, m=5, length=1537, page=32, d=64),
        # a batch of 24 sequences after eviction, groups of 7 heads
        dict(name="attend_batch", op="attend", seqs=24, kv_heads=4, group=7, m=1, length=5000, page=128, d=128),
        # a batch of 64 long caches
        dict(name="attend_large", op="attend", seqs=64, kv_heads=8, group=4, m=1, length=16384, page=64, d=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotate", "rotate", "append", "append", "compact", "keep", "fork", "attend", "attend", "attend"])
    d, page = rng.choice([64, 128]), rng.choice([16, 32, 64, 128])
    kv_heads, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 7, 8, 16])
    if op == "rotate":
        rot = rng.choice([d, d, d // 2, 3 * d // 4, 0])
        while True:
            rows = _log(rng, 1, 65536)
            if rows * kv_heads * (group + 1) * d <= 16381 * 40 * 128:
                return dict(op=op, rows=rows, kv_heads=kv_heads, group=group, d=d, rot=rot, pairs=rng.choice(["half", "next"]),
                            norm=rng.random() < 0.8 or rot == 0, far=rng.choice([1 << 12, 1 << 17, 1 << 24]))
    if op == "append":
        while True:
            seqs, m, length = _log(rng, 1, 256), rng.choice([1, 1, rng.randint(2, 8), _log(rng, 9, 2048)]), _log(rng, 1, 8192)
            if seqs * kv_heads * (m + length) * d <= 64 * 8192 * 128:
                return dict(op=op, seqs=seqs, kv_heads=kv_heads, m=m, length=length, page=page, d=d, twins=rng.choice([0, 2, 4]))
    if op in ("compact", "keep"):
        while True:
            cells, T = _log(rng, 1, 512), _log(rng, 33, 32768)
            if cells * T * d <= 96 * 32768 * 128:
                return dict(op=op, cells=cells, T=T, keep=rng.choice([0.06, 0.125, 0.25, 0.5, 0.8]), page=page, d=d)
    if op == "fork":
        while True:
            seqs, length = _log(rng, 1, 256), _log(rng, 1, 16384)
            family = rng.choice([1, 2, 4, 8])
            if seqs * kv_heads * length <= 2048 * 8192 and seqs * kv_heads * length * d / family <= 512 * 8192 * 64:
                return dict(op=op, seqs=seqs, kv_heads=kv_heads, length=length, page=page, d=d, family=family)
    while True:
        seqs, length = _log(rng, 1, 128), _log(rng, 1, 32768)
        m = rng.choice([1, 1, 1, rng.randint(2, 8)])
        # (no more work than the large batch, and the plain form's scores within reason)
        if seqs * kv_heads * length * d * max(1.0, group * m / 8) <= 64 * 8 * 16384 * 128 / 2:
            return dict(op=op, seqs=seqs, kv_heads=kv_heads, group=group, m=m, length=length, page=page, d=d)


def _rng(case, *keys):
    return random.Random(" ".join(str(case[k]) for k in keys))


def _spread(r, cells, mean, top):
    """Rows of every cell as a global threshold leaves them: unlike from head to head, every 29th cell with a few."""
    n = []
    for c in range(cells):
        x = mean * math.exp(r.gauss(-0.18, 0.6)) if cells > 1 else mean
        n.append(min(top, r.randint(0, 31) if c % 29 == 28 else int(x)))
    return n


def _append_counts(case):
    """Rows of every cell before the append; a twin (the second of every `twins` sequences) has its neighbour's."""
    n = _spread(_rng(case, "seqs", "kv_heads", "m", "length"), case["seqs"] * case["kv_heads"], case["length"], 3 * case["length"])
    hk, tw = case["kv_heads"], case["twins"]
    for s in range(case["seqs"]):
        if tw and s % tw == 1:
            n[s * hk:(s + 1) * hk] = n[(s - 1) * hk:s * hk]
    return n


def _kept_counts(case):
    r = _rng(case, "cells", "T", "keep")
    w = [math.exp(r.gauss(0, 0.6)) for _ in range(case["cells"])]
    k = case["T"] * case["keep"] * case["cells"] / sum(w)
    return [min(case["T"], max(min(32, case["T"]), int(x * k))) for x in w]


def _fork_counts(case):
    """Rows of every sequence's heads; a family shares the pages of its first seven eighths."""
    n = _spread(_rng(case, "seqs", "kv_heads", "length"), case["seqs"] * case["kv_heads"], case["length"], 2 * case["length"])
    hk, f = case["kv_heads"], case["family"]
    for s in range(case["seqs"]):
        if s % f:  # (a sequence of a family has decoded a little further than the one before)
            for h in range(hk):
                n[s * hk + h] = n[(s - 1) * hk + h] + s % 3
    return n


def _fork_sources(case):
    """Where every cell comes from: of each family's sequences one ends for good (-1), one forks into the place of another,
    two change places, the others stay."""
    r, hk, f, S = _rng(case, "seqs", "kv_heads", "family"), case["kv_heads"], case["family"], case["seqs"]
    src = list(range(S))
    for a in range(0, S, f):
        b = min(S, a + f)
        p = list(range(a, b))
        r.shuffle(p)
        if len(p) >= 2:
            src[p[0]] = p[1]  # forks
        if len(p) >= 4:
            src[p[2]], src[p[3]] = p[3], p[2]  # change places
        if len(p) >= 6 or len(p) == 1 and a % 3 == 0:
            src[p[-1]] = -1
    return [s * hk + h if s >= 0 else -1 for s in src for h in range(hk)]


def _cell_counts(case):
    m = case["m"]
    r = _rng(case, "seqs", "kv_heads", "length", "m")
    return [m + x for x in _spread(r, case["seqs"] * case["kv_heads"], case["length"], 3 * case["length"])]


def work(case):
    op, d = case["op"], case["d"]
    if op == "rotate":
        x = case["rows"] * case["kv_heads"] * (case["group"] + 1) * d
        return {"bytes": 4 * x + 4 * case["rows"], "flops": x * ((4 if case["norm"] else 0) + 3 * case["rot"] / d)}
    if op == "append":
        P, tw, hk = case["page"], case["twins"], case["kv_heads"]
        n = _append_counts(case)
        # the rows of pages that twins share are copied, for both of them
        copied = sum(x % P for c, x in enumerate(n) if tw and (c // hk) % tw < 2 and (c // hk) // tw * tw + 1 < case["seqs"])
        return {"bytes": 8 * d * (len(n) * case["m"] + copied) + 24 * len(n), "flops": 0}
    if op in ("compact", "keep"):
        return {"bytes": sum(_kept_counts(case)) * (8 * d + 4), "flops": 0}
    if op == "fork":
        P, n, src = case["page"], _fork_counts(case), _fork_sources(case)
        # per entry that comes or goes: itself, and how many name its page (read and written)
        came = sum(-(-n[s] // P) for c, s in enumerate(src) if s >= 0 and s != c)
        went = sum(-(-n[c] // P) for c, s in enumerate(src) if s != c)
        return {"bytes": 16 * came + 12 * went + 20 * len(n), "flops": 0}
    n = _cell_counts(case)
    rows = len(n) * case["group"] * case["m"]
    return {"bytes": sum(n) * 4 * d + rows * (4 * d + 4), "flops": 4 * d * sum(n) * case["group"] * case["m"]}


# ----------------------------------------------------------------------- inputs
def _keys(shape, gen):
    """Keys or values as a cache has them: channels of unlike size."""
    x = torch.randn(shape, device="cuda", generator=gen, dtype=torch.bfloat16)
    x *= torch.exp(0.5 * torch.randn(shape[-1], device="cuda", generator=gen)).to(torch.bfloat16)
    return x


def _pages(case, counts, shared, gen, *, need, spare_rows):
    """Pages as a running server has them: every cell's scattered over the pool.  `shared`: (leader, entries) per cell, the
    entries that it has in common with an earlier cell's first ones.  `need`: pages that must be free."""
    P, d, cells = case["page"], case["d"], len(counts)
    held = [-(-n // P) for n in counts]
    width = max(held) + -(-spare_rows // P) + 1
    fresh = [e - min(s[1], e) for e, s in zip(held, shared)]
    N = sum(fresh) + need + need // 8 + 37
    order = torch.randperm(N, device="cuda", generator=gen).to(torch.int32)
    # entries of a cell's own: a run of the shuffled pages, behind those that it shares
    start = torch.tensor([0] + fresh[:-1], device="cuda").cumsum(0)
    i = torch.arange(width, device="cuda")
    common = torch.tensor([min(s[1], e) for e, s in zip(held, shared)], device="cuda")
    held_t = torch.tensor(held, device="cuda")
    mine = (i >= common[:, None]) & (i < held_t[:, None])
    at = (start[:, None] + i - common[:, None]).clamp(0, N - 1)
    sizes = [("next", 4), ("counts", cells), ("held", cells), ("table", cells * width), ("refs", N), ("free", -(-N // 32))]
    book = torch.zeros(sum(-(-z // 4) * 4 for _, z in sizes), dtype=torch.int32, device="cuda")
    st, a = {}, 0
    for name, z in sizes:
        st[name] = book[a:a + (1 if name == "next" else z)]
        a += -(-z // 4) * 4
    st["table"] = table = st["table"].view(cells, width)
    table.copy_(torch.where(mine, order[at], torch.full_like(order[at], -1)))
    leader = torch.tensor([s[0] for s in shared], device="cuda")
    table.copy_(torch.where(i < common[:, None], table[leader], table))
    st["held"].copy_(held_t)
    st["counts"].copy_(torch.tensor(counts, device="cuda"))
    used = table[(i < held_t[:, None])].long()
    st["refs"].index_add_(0, used, torch.ones(used.numel(), dtype=torch.int32, device="cuda"))
    st["free"].copy_(_free_bits(st["refs"]))
    st["next"].fill_(N // 3)
    st["k"], st["v"] = _keys((N, P, d), gen), _keys((N, P, d), gen)
    return st, book


def _free_bits(refs):
    N = refs.numel()
    f = torch.zeros(-(-N // 32) * 32, dtype=torch.int64, device=refs.device)
    f[:N] = (refs == 0).long()
    bits = (f.view(-1, 32) << torch.arange(32, device=refs.device)).sum(1)
    return torch.where(bits >= 1 << 31, bits - (1 << 32), bits).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    op, d = case["op"], case["d"]
    st = dict(op=op, d=d)
    if op == "rotate":
        rows, hk, hq = case["rows"], case["kv_heads"], case["kv_heads"] * case["group"]
        # the projection of a token holds its queries, keys and values side by side
        x = torch.randn(rows, hq + 2 * hk, d, device="cuda", generator=gen, dtype=torch.bfloat16)
        x *= torch.exp(0.4 * torch.randn(rows, 1, 1, device="cuda", generator=gen)).to(torch.bfloat16)
        rot = case["rot"]
        pos = torch.randint(0, case["far"], (rows,), device="cuda", generator=gen, dtype=torch.int32)
        if rows >= 64:  # a prompt's positions follow one another
            pos = torch.arange(rows, device="cuda", dtype=torch.int32) + (pos[0] % max(1, case["far"] - rows)).int()
        w = [(1 + 0.2 * torch.randn(d, device="cuda", generator=gen)).to(torch.bfloat16) if case["norm"] else None for _ in "qk"]
        st.update(q=x[:, :hq], k=x[:, hq:hq + hk], pos=pos, q_weight=w[0], k_weight=w[1], eps=1e-6 if case["norm"] else None,
                  inv_freq=torch.exp(torch.arange(rot // 2, device="cuda", dtype=torch.float64) * (-2 * math.log(5e5) /
                                     max(rot, 1))).float(), next=case["pairs"] == "next",
                  out=(torch.empty(rows, hq, d, device="cuda", dtype=torch.bfloat16),
                       torch.empty(rows, hk, d, device="cuda", dtype=torch.bfloat16)))
        return st
    P = case["page"]
    st["P"] = P
    if op == "append":
        hk, m, tw = case["kv_heads"], case["m"], case["twins"]
        n = _append_counts(case)
        shared = [(c - hk, 1 << 30) if tw and (c // hk) % tw == 1 else (c, 0) for c in range(len(n))]
        need = len(n) * (-(-m // P) + 1)
        st["store"], book = _pages(case, n, shared, gen, need=need, spare_rows=m)
        st.update(new_k=_keys((case["seqs"], m, hk, d), gen), new_v=_keys((case["seqs"], m, hk, d), gen))
    elif op in ("compact", "keep"):
        cells, T = case["cells"], case["T"]
        n = _kept_counts(case)
        nt = torch.tensor(n, device="cuda")
        # kept positions as an allocation gives them: ascending, the recent ones and those of largest score
        score = torch.rand(cells, T, device="cuda", generator=gen)
        score[:, -32:] += 1.0
        keep = torch.zeros(cells, T, dtype=torch.bool, device="cuda")
        keep.scatter_(1, torch.argsort(score, 1, descending=True), torch.arange(T, device="cuda") < nt[:, None])
        del score
        st["offsets"] = torch.cat([nt.new_zeros(1), torch.cumsum(nt, 0)])
        st["kept_pos"] = keep.nonzero()[:, 1].to(torch.int32).contiguous()
        need = sum(-(-x // P) for x in n)
        # (into pages: cells that are empty; inside pages: whole caches)
        st["store"], book = _pages(case, [T if op == "keep" else 0] * cells, [(c, 0) for c in range(cells)], gen, need=need,
                                   spare_rows=max(n) if op == "compact" else 0)
        if op == "compact":
            st.update(K=_keys((cells, T, d), gen), V=_keys((cells, T, d), gen))
    elif op == "fork":
        hk, f = case["kv_heads"], case["family"]
        n = _fork_counts(case)
        shared = []
        for c in range(len(n)):
            lead = (c // hk) // f * f * hk + c % hk
            shared.append((lead, n[lead] // P * 7 // 8) if lead != c else (c, 0))
        st["store"], book = _pages(case, n, shared, gen, need=0, spare_rows=2 * P)
        st["src"] = torch.tensor(_fork_sources(case), dtype=torch.int32, device="cuda")
    else:
        n, hk = _cell_counts(case), case["kv_heads"]
        st["store"], book = _pages(case, n, [(c, 0) for c in range(len(n))], gen, need=0, spare_rows=0)
        st.update(q=1.5 * torch.randn(case["seqs"], case["m"], hk * case["group"], d, device="cuda", generator=gen,
                                      dtype=torch.bfloat16), kv_heads=hk, longest=max(n), scale=1.0 / math.sqrt(d))
    if op != "attend":
        st.update(book=book, before=book.clone())
    if own:  # the handle over the pages that a program keeps, and its buffers for a step
        from paper_2608_25230_gb300 import fw

        st["pages"] = pages = fw.Pages(**st["store"])
        if op == "append":
            st["workspace"] = fw.pages_append_workspace(pages, case["m"])
        elif op in ("compact", "keep"):
            st["workspace"] = fw.pages_compact_workspace(pages, st["kept_pos"].numel())
        elif op == "fork":
            st["workspace"] = fw.pages_fork_workspace(pages)
        else:
            q = st["q"]
            st["out"] = dict(o=torch.empty_like(q), lse=torch.empty(q.shape[:-1], device="cuda"),
                             status=torch.empty(len(n), dtype=torch.int32, device="cuda"))
            st["workspace"] = fw.pages_attend_workspace(pages, q, kv_heads=st["kv_heads"], longest=st["longest"])
    return st


# ------------------------------------------------------------------ plain forms
def _rotate_plain(st):
    half = st["inv_freq"].numel()
    angle = st["pos"].double()[:, None] * st["inv_freq"].double()
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    for x, w, y in ((st["q"], st["q_weight"], st["out"][0]), (st["k"], st["k_weight"], st["out"][1])):
        f = x.float()
        if st["eps"] is not None:
            f = f * torch.rsqrt((f * f).mean(-1, keepdim=True) + st["eps"]) * w.float()
        if half:
            a, b = (f[..., 0:2 * half:2], f[..., 1:2 * half:2]) if st["next"] else (f[..., :half], f[..., half:2 * half])
            r = (a * cos - b * sin, b * cos + a * sin)
            r = torch.stack(r, -1).flatten(-2) if st["next"] else torch.cat(r, -1)
            f = torch.cat([r, f[..., 2 * half:]], -1)
        y.copy_(f)
    return st["out"]


def _hand_out(s):
    """The free pages in the order in which they are handed out (behind them N's of no meaning)."""
    N = s["refs"].numel()
    at = (s["next"].long() + torch.arange(N, device="cuda")) % N
    free = (s["refs"] == 0)[at]
    place = torch.where(free, torch.cumsum(free, 0) - 1, torch.full_like(at, N))
    return torch.zeros(N + 1, dtype=torch.int64, device="cuda").scatter_(0, place, at)


def _take(s, pages, wanted):
    """Pages for the entries of the mask `wanted`, in its order; the search goes on behind the last one."""
    flat = wanted.flatten()
    rank = torch.cumsum(flat, 0)
    got = pages[(rank - 1).clamp(min=0)].view(wanted.shape)
    s["next"].copy_(torch.where(rank[-1:] > 0, (pages[(rank[-1:] - 1).clamp(min=0)] + 1) % s["refs"].numel(), s["next"].long()))
    return got


def _count(s, table, live, sign):
    """The entries of `table` that are `live` come (+1) or go (-1)."""
    s["refs"].index_add_(0, table.clamp(min=0).long().flatten(), (live.int() * sign).flatten())


def _books(s, names):
    s["free"].copy_(_free_bits(s["refs"]))
    return {x: s[x] for x in names + ("table", "held", "counts", "refs", "free", "next")}


def _append_plain(st):
    s, P, d = st["store"], st["P"], st["d"]
    S, m, hk = st["new_k"].shape[:3]
    n, held = s["counts"].long(), s["held"].long()
    cells, width = s["table"].shape
    span = (m + P - 2) // P + 1
    i = (n // P)[:, None] + torch.arange(span, device="cuda")            # the entries that the rows touch
    touched = i <= (n + m - 1)[:, None] // P
    ic = i.clamp(max=width - 1)
    old = torch.gather(s["table"].long(), 1, ic)
    have = touched & (i < held[:, None])
    shared = have & (s["refs"][old.clamp(min=0)] > 1)
    wanted = touched & (~have | shared)
    got = _take(s, _hand_out(s), wanted)
    page = torch.where(wanted, got, old)
    # the rows that a shared page holds already (where there are none, the first new row's place stands for them)
    j = torch.arange(P, device="cuda")
    moved = shared[:, 0, None] & (j < (n % P)[:, None])
    first = (page[:, 0] * P + n % P)[:, None]
    for x, new in (("k", st["new_k"]), ("v", st["new_v"])):
        rows = s[x].view(-1, d)
        to = torch.where(moved, page[:, 0, None] * P + j, first)
        rows[to.flatten()] = rows[torch.where(moved, old[:, 0, None] * P + j, first).flatten()]
        r = n[:, None] + torch.arange(m, device="cuda")
        to = torch.gather(page, 1, r // P - (n // P)[:, None]) * P + r % P
        rows[to.flatten()] = new.permute(0, 2, 1, 3).reshape(-1, d)
    _count(s, page, wanted, 1)
    _count(s, old, shared, -1)
    c = torch.arange(cells, device="cuda")[:, None].expand_as(i)
    s["table"].view(-1).scatter_(0, (c * width + ic).flatten(), torch.where(touched, page, old).to(torch.int32).flatten())
    s["held"].copy_(torch.maximum(held, (n + m + P - 1) // P))
    s["counts"].copy_(n + m)
    return _books(s, ("k", "v"))


def _compact_plain(st):
    s, P, d, off, pos = st["store"], st["P"], st["d"], st["offsets"], st["kept_pos"].long()
    n = off[1:] - off[:-1]
    cells, width = s["table"].shape
    i = torch.arange(width, device="cuda")
    wanted = i < ((n + P - 1) // P)[:, None]
    got = _take(s, _hand_out(s), wanted)
    r = torch.arange(pos.numel(), device="cuda")
    cell = torch.searchsorted(off[1:].contiguous(), r, right=True)
    j = r - off[cell]
    to = got[cell, j // P] * P + j % P
    for x, src in (("k", "K"), ("v", "V")):
        rows = s[x].view(-1, d)
        rows[to] = st[src][cell, pos] if st["op"] == "compact" else rows[s["table"][cell, pos // P].long() * P + pos % P]
    _count(s, got, wanted, 1)
    _count(s, s["table"], i < s["held"][:, None], -1)
    s["table"].copy_(torch.where(wanted, got, s["table"].long()))
    s["held"].copy_((n + P - 1) // P)
    s["counts"].copy_(n)
    return _books(s, ("k", "v"))


def _fork_plain(st):
    s, P = st["store"], st["P"]
    src = st["src"].long()
    cells, width = s["table"].shape
    h, i = torch.arange(cells, device="cuda"), torch.arange(width, device="cuda")
    from_ = src.clamp(min=0)
    stays = src == h
    n = torch.where(src < 0, torch.zeros_like(src), s["counts"].long()[from_])
    held = torch.where(stays, s["held"].long(), (n + P - 1) // P)
    came = (i < held[:, None]) & ~stays[:, None]
    table = torch.where(came, s["table"][from_], s["table"])
    _count(s, table, came, 1)
    _count(s, s["table"], (i < s["held"][:, None]) & ~stays[:, None], -1)
    s["table"].copy_(table)
    s["held"].copy_(held)
    s["counts"].copy_(n)
    return _books(s, ())


def _attend_plain(st):
    s, q, P = st["store"], st["q"], st["P"]
    S, m, hq, d = q.shape
    hk, L = st["kv_heads"], st["longest"]
    n = s["counts"].long()
    cells, j = n.numel(), torch.arange(L, device="cuda")
    there = j < n[:, None]
    row = s["table"].long()[:, j // P].clamp_(min=0) * P + j % P
    row = torch.where(there, row, row[:, :1])              # (rows that are not there: any)
    k, v = (s[x].view(-1, d)[row].float() for x in "kv")
    v.masked_fill_(~there[..., None], 0.0)
    qc = q.view(S, m, hk, hq // hk, d).permute(0, 2, 1, 3, 4).reshape(cells, -1, d).float()
    x = torch.matmul(qc, k.transpose(1, 2)).mul_(st["scale"]).view(cells, m, hq // hk, L)
    seen = n[:, None] - m + 1 + torch.arange(m, device="cuda")
    x.masked_fill_((j >= seen[..., None])[:, :, None], float("-inf"))
    mx = x.amax(-1, keepdim=True)
    mx = torch.where(mx == float("-inf"), torch.zeros_like(mx), mx)
    x.sub_(mx).exp_()
    l = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(cells, -1, L), v).view(cells, m, hq // hk, d) / torch.where(l > 0, l, torch.ones_like(l))
    o = o.view(S, hk, m, -1, d).permute(0, 2, 1, 3, 4).reshape(S, m, hq, d).to(torch.bfloat16)
    lse = (mx + torch.log(l))[..., 0].view(S, hk, m, -1).permute(0, 2, 1, 3).reshape(S, m, hq)
    return {"o": o, "lse": lse}


def run(st):
    op = st["op"]
    if "book" in st:
        st["book"].copy_(st["before"])  # the step is taken back
    if not own:
        return {"rotate": _rotate_plain, "append": _append_plain, "compact": _compact_plain, "keep": _compact_plain,
                "fork": _fork_plain, "attend": _attend_plain}[op](st)
    from paper_2608_25230_gb300 import fw

    if op == "rotate":
        return fw.qk_rotate(st["q"], st["k"], st["pos"], st["inv_freq"], q_weight=st["q_weight"], k_weight=st["k_weight"],
                            eps=st["eps"], interleaved=st["next"], out=st["out"])
    pages, ws = st["pages"], st["workspace"]
    if op == "attend":
        r = fw.pages_attend(pages, st["q"], kv_heads=st["kv_heads"], scale=st["scale"], longest=st["longest"], out=st["out"],
                            workspace=ws)
        return {"o": r["o"], "lse": r["lse"]}
    if op == "append":
        fw.pages_append(pages, st["new_k"], st["new_v"], workspace=ws)
    elif op == "compact":
        fw.pages_compact(pages, st["K"], st["V"], st["offsets"], st["kept_pos"], workspace=ws)
    elif op == "keep":
        fw.pages_keep(pages, st["offsets"], st["kept_pos"], workspace=ws)
    else:
        fw.pages_fork(pages, st["src"], workspace=ws)
    s = st["store"]
    return {x: s[x] for x in (() if op == "fork" else ("k", "v")) + ("table", "held", "counts", "refs", "free", "next")}


# ---------------------------------------------------------------- in 64 bits
def _rotate64(st, x, w):
    y = x.double()
    if st["eps"] is not None:
        y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / y.shape[-1] + st["eps"]) * w.double()
    for p in range(st["inv_freq"].numel()):
        a, b = (2 * p, 2 * p + 1) if st["next"] else (p, p + st["inv_freq"].numel())
        t = (st["pos"].double() * st["inv_freq"][p].double())[:, None]
        u, z = y[..., a].clone(), y[..., b].clone()
        y[..., a], y[..., b] = u * torch.cos(t) - z * torch.sin(t), u * torch.sin(t) + z * torch.cos(t)
    return y


class _Hand:
    """Free pages one after another, on the host."""

    def __init__(self, s):
        self.refs, self.at = s["refs"].tolist(), int(s["next"])

    def page(self):
        N = len(self.refs)
        for z in range(N):
            p = (self.at + z) % N
            if self.refs[p] == 0:
                self.refs[p], self.at = 1, (p + 1) % N
                return p
        raise ValueError("no page is free")


def exact(case, seed):
    op, d = case["op"], case["d"]
    st = prepare(case, seed)
    if op == "rotate":
        return (_rotate64(st, st["q"], st["q_weight"]), _rotate64(st, st["k"], st["k_weight"]))
    if op == "fork":
        return None  # (books alone: whole numbers)
    s, P = st["store"], case["page"]
    table, counts, held = s["table"].tolist(), s["counts"].tolist(), s["held"].tolist()
    pool = {x: s[x].double().view(-1, d) for x in "kv"}
    if op == "attend":
        q, hk, g, m = st["q"].double(), case["kv_heads"], case["group"], case["m"]
        o, lse = torch.zeros_like(q), torch.full(q.shape[:3], float("-inf"), dtype=torch.float64, device="cuda")
        for c, n in enumerate(counts):
            b, h = divmod(c, hk)
            pages = s["table"][c, :held[c]].long()
            k, v = (pool[x].view(-1, P, d)[pages].reshape(-1, d)[:n] for x in "kv")
            for t in range(m):
                e = n - m + 1 + t
                if e < 1:
                    continue
                x = st["scale"] * (q[b, t, h * g:(h + 1) * g] @ k[:e].T)
                z = torch.logsumexp(x, 1)
                lse[b, t, h * g:(h + 1) * g] = z
                o[b, t, h * g:(h + 1) * g] = torch.exp(x - z[:, None]) @ v[:e]
        return {"o": o, "lse": lse}
    hand = _Hand(s)
    if op == "append":
        hk, m = case["kv_heads"], case["m"]
        refs = s["refs"].tolist()
        for c, n in enumerate(counts):
            mine = table[c][:held[c]]
            for i in range(n // P, (n + m - 1) // P + 1):
                if i >= len(mine):
                    mine.append(hand.page())
                elif refs[mine[i]] > 1:
                    fresh, was = hand.page(), mine[i]
                    keep = max(0, min(P, n - i * P))
                    for x in "kv":
                        pool[x][fresh * P:fresh * P + keep] = s[x].view(-1, d)[was * P:was * P + keep].double()
                    mine[i] = fresh
            r = torch.arange(n, n + m, device="cuda")
            to = torch.tensor(mine, device="cuda")[r // P] * P + r % P
            pool["k"][to], pool["v"][to] = st["new_k"][c // hk, :, c % hk].double(), st["new_v"][c // hk, :, c % hk].double()
    else:
        off = st["offsets"].tolist()
        for c in range(case["cells"]):
            pos = st["kept_pos"][off[c]:off[c + 1]].long()
            fresh = torch.tensor([hand.page() for _ in range(-(-pos.numel() // P))], device="cuda")
            r = torch.arange(pos.numel(), device="cuda")
            to = fresh[r // P] * P + r % P
            for x in "kv":
                src = st[x.upper()][c, pos] if op == "compact" else s[x].view(-1, d)[s["table"][c].long()[pos // P] * P + pos % P]
                pool[x][to] = src.double()
    return dict({x: pool[x].view(s[x].shape) for x in "kv"}, **dict.fromkeys(("table", "held", "counts", "refs", "free", "next")))

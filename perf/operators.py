"""The serving operators around the evicted cache, with their plain forms and the
calls they are measured on: attention over packed prompts, the ragged store held in
8 bits (compaction into it, appends to it) and the attention that reads it.

Where `own` is false, run() computes them from elementary torch operations in 32
bits; where it is true, it makes the library's calls.  Both write the same tensors.

The store holds a code per value and a power-of-two scale per block of 32 tokens and
head, so a code is the exact rounding of value / scale whatever computes it.  run()
returns the codes as they are held (float8 values, or whole numbers for int8) beside
their scales: the value a code stands for is their product, exactly.
"""
import math
import random

import torch

own = False

BLOCK = 32  # tokens per scale
RING = 64   # bf16 rows kept per cell, by row index modulo RING
TOP = {"e4m3": 448.0, "int8": 127.0}
# the largest code as mantissa in [1/2, 1) and exponent
TOP_MANT = {"e4m3": 0.875, "int8": 0.9921875}
TOP_EXP = {"e4m3": 9, "int8": 7}


# ------------------------------------------------------------------------ cases
def listed():
    return [
        # a short question: one small launch, latency only
        dict(name="prompt_short", op="prompt", seqs=1, q_len=17, context=0, ragged=False, kv_heads=8, group=4, d=128),
        # a prefill batch of prompts of unlike lengths, one of a single token
        dict(name="prompt_packed", op="prompt", seqs=12, q_len=2048, context=0, ragged=True, kv_heads=8, group=4, d=64),
        # a chunk of 512 tokens per sequence behind contexts already in the cache
        dict(name="prompt_chunk", op="prompt", seqs=4, q_len=512, context=7680, ragged=True, kv_heads=8, group=4, d=128),
        # one long prompt
        dict(name="prompt_long", op="prompt", seqs=1, q_len=16384, context=0, ragged=False, kv_heads=8, group=4, d=128),
        # one layer of one short sequence compacted
        dict(name="compact_layer", op="compact", cells=8, T=4097, share=8, d=64, fmt="int8"),
        # a whole cache (32 layers x 8 heads) compacted to an eighth of its tokens
        dict(name="compact_cache", op="compact", cells=256, T=32768, share=8, d=128, fmt="e4m3"),
        # one decoded token for every head of a 32-layer cache
        dict(name="append_token", op="append", cells=256, m=1, d=128, fmt="e4m3"),
        # a draft of 7 tokens for a batch of 64 sequences of one layer, heads of 64
        dict(name="append_draft", op="append", cells=512, m=7, d=64, fmt="int8"),
        # one layer, one sequence, one token: a latency-bound decode step
        dict(name="attend_layer", op="attend", seqs=1, kv_heads=8, group=4, m=1, length=4096, d=128, fmt="e4m3"),
        # a draft of 5 tokens verified for 8 sequences of odd lengths
        dict(name="attend_draft", op="attend", seqs=8, kv_heads=8, group=4, m=5, length=1537, d=64, fmt="e4m3"),
        # a batch of 32 sequences after eviction, a token each
        dict(name="attend_batch", op="attend", seqs=32, kv_heads=8, group=4, m=1, length=4096, d=128, fmt="e4m3"),
        # a batch of 64 long caches
        dict(name="attend_large", op="attend", seqs=64, kv_heads=8, group=4, m=1, length=16384, d=128, fmt="int8"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["prompt", "prompt", "compact", "append", "attend", "attend"])
    d = rng.choice([64, 128])
    fmt = rng.choice(["e4m3", "int8"])
    if op == "prompt":
        kv_heads, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 8])
        while True:
            seqs, q_len = _log(rng, 1, 24), _log(rng, 1, 16384)
            context = rng.choice([0, 0, _log(rng, 1, 16384)])
            # (the plain form's padded scores, and no more work than the longest prompt)
            if seqs * kv_heads * group * q_len * (q_len + context) <= 16384 * 16384 * 16 and context + q_len <= 16384:
                break
        return dict(op=op, seqs=seqs, q_len=q_len, context=context, ragged=rng.random() < 0.7, kv_heads=kv_heads,
                    group=group, d=d)
    if op == "compact":
        while True:
            cells, T = _log(rng, 1, 512), _log(rng, 33, 32768)
            if cells * T <= 256 * 32768:
                # (no more rows kept than the whole cache's eighth)
                return dict(op=op, cells=cells, T=T, share=rng.choice([2, 4, 8, 16]) if cells * T <= 64 * 32768
                            else rng.choice([8, 16]), d=d, fmt=fmt)
    if op == "append":
        return dict(op=op, cells=_log(rng, 1, 2048), m=rng.choice([1, 1, 1, rng.randint(2, 32)]), d=d, fmt=fmt)
    while True:
        seqs, length = _log(rng, 1, 128), _log(rng, 1, 32768)
        kv_heads, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 7, 8, 16])
        m = rng.choice([1, 1, rng.randint(2, 8)])
        if seqs * kv_heads * length * max(1.0, group * m / 8) <= 64 * 8 * 16384:
            return dict(op=op, seqs=seqs, kv_heads=kv_heads, group=group, m=m, length=length, d=d, fmt=fmt)


def _prompt_lengths(case):
    """(query tokens, keys) of every sequence: ragged ones spread from 1 to q_len."""
    r = random.Random("%d %d %d" % (case["seqs"], case["q_len"], case["context"]))
    lq, lk = [], []
    for s in range(case["seqs"]):
        q, c = case["q_len"], case["context"]
        if case["ragged"] and s > 0:
            if c:  # a chunk: the contexts differ
                c = r.randint(0, c)
            else:
                q = 1 if s == 1 else r.randint(1, q)
        lq.append(q)
        lk.append(q + c)
    return lq, lk


def _cell_counts(case):
    """Rows of every cell: what a global threshold leaves is unlike from head to head;
    an average of about `length`, every 29th cell with fewer rows than a block."""
    cells = case["seqs"] * case["kv_heads"]
    r = random.Random("%d %d %d" % (cells, case["length"], case["m"]))
    n = []
    for c in range(cells):
        x = case["length"] * math.exp(r.gauss(-0.18, 0.6)) if cells > 1 else case["length"]
        if c % 29 == 28:
            x = r.randint(0, BLOCK - 1)
        n.append(case["m"] + min(int(x), 3 * case["length"]))
    return n


def _append_counts(case):
    r = random.Random("%d %d" % (case["cells"], case["m"]))
    return [r.randint(0, 160) for _ in range(case["cells"])]


def _kept_counts(case):
    """Kept rows of every cell: the recent block always, shares unlike from cell to cell."""
    r = random.Random("%d %d %d" % (case["cells"], case["T"], case["share"]))
    w = [math.exp(r.gauss(0, 0.6)) for _ in range(case["cells"])]
    k = case["T"] / case["share"] * case["cells"] / sum(w)
    return [min(case["T"], max(min(BLOCK, case["T"]), int(x * k))) for x in w]


def work(case):
    d, op = case["d"], case["op"]
    if op == "prompt":
        lq, lk = _prompt_lengths(case)
        hq, hk = case["kv_heads"] * case["group"], case["kv_heads"]
        seen = sum(q * (k - q) + q * (q + 1) // 2 for q, k in zip(lq, lk))
        return {"bytes": 2 * d * (2 * hq * sum(lq) + 2 * hk * sum(lk)) + 4 * hq * sum(lq), "flops": 4 * d * hq * seen}
    if op == "compact":
        kept = sum(_kept_counts(case))
        return {"bytes": kept * (3 * 2 * d + 4 + 8 / BLOCK), "flops": kept * 2 * d * 3}
    if op == "append":
        opened = sum(c % BLOCK for c in _append_counts(case))
        new = case["cells"] * case["m"]
        return {"bytes": 2 * d * (2 * (new + opened) + 2 * new + (new + opened)) + 16 * case["cells"],
                "flops": (new + opened) * 2 * d * 3}
    n = sum(_cell_counts(case))
    rows = case["seqs"] * case["kv_heads"] * case["group"] * case["m"]
    return {"bytes": n * (2 * d + 8 / BLOCK) + rows * (4 * d + 4), "flops": 4 * d * n * case["group"] * case["m"]}


# ----------------------------------------------------------------------- inputs
def _code_dtype(fmt):
    return torch.float8_e4m3fn if fmt == "e4m3" else torch.int8


def _keys(shape, gen, *, spread):
    """Keys or values as a cache has them: channels of unlike size, tokens too."""
    x = torch.randn(shape, device="cuda", generator=gen, dtype=torch.bfloat16)
    ch = torch.exp(0.5 * torch.randn(shape[-1], device="cuda", generator=gen)).to(torch.bfloat16)
    x *= ch
    if spread:
        x *= torch.exp(0.3 * torch.randn(shape[:-1] + (1,), device="cuda", generator=gen)).to(torch.bfloat16)
    return x


def _store(base, capacity, d, fmt):
    rows = int((base[-1] + capacity[-1]).item())
    cells = base.numel()
    z = dict(device="cuda")
    return dict(k=torch.zeros(rows, d, dtype=torch.int8, **z).view(_code_dtype(fmt)),
                v=torch.zeros(rows, d, dtype=torch.int8, **z).view(_code_dtype(fmt)),
                k_scale=torch.ones(rows // BLOCK, **z), v_scale=torch.ones(rows // BLOCK, **z),
                k_tail=torch.zeros(cells, RING, d, dtype=torch.bfloat16, **z),
                v_tail=torch.zeros(cells, RING, d, dtype=torch.bfloat16, **z),
                base=base, capacity=capacity, counts=torch.zeros(cells, dtype=torch.int32, **z))


def _layout(counts, room):
    """Rows of every cell in a store: its count and `room` more, in whole blocks."""
    capacity = (counts.to(torch.int64) + room + BLOCK - 1) // BLOCK * BLOCK
    base = torch.cumsum(capacity, 0) - capacity
    return base.contiguous(), capacity.to(torch.int32).contiguous()


def _outputs(q, items):
    """Buffers for the outputs: `items` sequences or cells have a status each."""
    return dict(o=torch.empty_like(q), lse=torch.empty(q.shape[:-1], device="cuda"),
                status=torch.empty(items, dtype=torch.int32, device="cuda"))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    st = dict(op=case["op"], d=case["d"])
    d, op = case["d"], case["op"]
    if op == "prompt":
        lq, lk = _prompt_lengths(case)
        hk, g = case["kv_heads"], case["group"]
        cu = [torch.tensor([sum(x[:i]) for i in range(len(x) + 1)], dtype=torch.int32, device="cuda") for x in (lq, lk)]
        q = torch.randn(sum(lq), hk * g, d, device="cuda", generator=gen, dtype=torch.bfloat16)
        st.update(q=q * 1.5, k=_keys((sum(lk), hk, d), gen, spread=False), v=_keys((sum(lk), hk, d), gen, spread=True),
                  cu_q=cu[0], cu_k=cu[1], max_q=max(lq), max_k=max(lk), scale=1.0 / math.sqrt(d))
        if own:
            st["out"] = _outputs(st["q"], len(lq))
        return st
    st["fmt"] = fmt = case["fmt"]
    if op == "compact":
        cells, T = case["cells"], case["T"]
        st.update(K=_keys((cells, T, d), gen, spread=True), V=_keys((cells, T, d), gen, spread=True))
        # kept positions as an allocation gives them: ascending, the recent ones and those of largest score
        n = torch.tensor(_kept_counts(case), device="cuda")
        score = torch.rand(cells, T, device="cuda", generator=gen)
        score[:, -BLOCK:] += 1.0
        order = torch.argsort(score, 1, descending=True)
        keep = torch.zeros(cells, T, dtype=torch.bool, device="cuda")
        keep.scatter_(1, order, torch.arange(T, device="cuda") < n[:, None])
        st["offsets"] = torch.cat([n.new_zeros(1), torch.cumsum(n, 0)])
        st["kept_pos"] = keep.nonzero()[:, 1].to(torch.int32).contiguous()
        base, capacity = _layout(n, 0)
        st["store"] = _store(base, capacity, d, fmt)
    elif op == "append":
        cells, m = case["cells"], case["m"]
        st["counts0"] = torch.tensor(_append_counts(case), dtype=torch.int32, device="cuda")
        base, capacity = _layout(torch.full((cells,), 160, device="cuda"), m + BLOCK)
        st["store"] = s = _store(base, capacity, d, fmt)
        # the cells' rows so far arrived by appends
        for old in range(0, 160, BLOCK):
            rows = torch.clamp(st["counts0"] - old, 0, BLOCK)
            x = [_keys((cells, BLOCK, d), gen, spread=True) for _ in "kv"]
            _append_plain(s, x[0], x[1], d, fmt, rows)
        st.update(new_k=_keys((cells, m, d), gen, spread=True), new_v=_keys((cells, m, d), gen, spread=True))
    else:
        n = torch.tensor(_cell_counts(case), dtype=torch.int32, device="cuda")
        base, capacity = _layout(n, 0)
        st["store"] = s = _store(base, capacity, d, fmt)
        s["counts"].copy_(n)
        # codes of blocks whose largest value sits in the top octave of the code's range
        for x in "kv":
            if fmt == "e4m3":
                c = torch.randn(s[x].shape, device="cuda", generator=gen, dtype=torch.bfloat16)
                s[x].copy_((c * 80).clamp_(-448, 448).to(torch.float8_e4m3fn))
            else:
                c = torch.randn(s[x].shape, device="cuda", generator=gen, dtype=torch.bfloat16)
                s[x].copy_((c * 30).round_().clamp_(-127, 127).to(torch.int8))
            e = torch.randint(0, 3, s[x + "_scale"].shape, device="cuda", generator=gen)
            s[x + "_scale"].copy_(torch.exp2((e - (7 if fmt == "e4m3" else 6)).float()))
        st.update(q=torch.randn(case["seqs"], case["m"], case["kv_heads"] * case["group"], d, device="cuda",
                                generator=gen, dtype=torch.bfloat16) * 1.5,
                  kv_heads=case["kv_heads"], max_n=int(n.max().item()), scale=1.0 / math.sqrt(d))
    if own:  # the handle over the store's tensors that a program keeps, and its buffers for a step
        from paper_2608_25230_gb300 import fw

        st["cache"] = fw.Cache8(fmt=fmt, **st["store"])
        if op == "attend":
            st["out"] = _outputs(st["q"], s["base"].numel())
            st["workspace"] = fw.cache8_attend_workspace(st["cache"], st["q"], kv_heads=st["kv_heads"])
    return st


# ------------------------------------------------------------------ plain forms
def _prompt_plain(st):
    q, k, v, cu_q, cu_k = st["q"], st["k"], st["v"], st["cu_q"], st["cu_k"]
    total, hq, d = q.shape
    hk, S, MQ, MK = k.shape[1], cu_q.numel() - 1, st["max_q"], st["max_k"]
    lq, lk = (cu_q[1:] - cu_q[:-1]).long(), (cu_k[1:] - cu_k[:-1]).long()
    iq, ik = torch.arange(MQ, device=q.device), torch.arange(MK, device=q.device)
    qp = q[(cu_q[:-1, None] + iq).clamp_(max=total - 1).long()].float()       # [S, MQ, hq, d]
    kp = k[(cu_k[:-1, None] + ik).clamp_(max=k.shape[0] - 1).long()].float()  # [S, MK, hk, d]
    vp = v[(cu_k[:-1, None] + ik).clamp_(max=k.shape[0] - 1).long()].float()
    qp = qp.view(S, MQ, hk, hq // hk, d).permute(0, 2, 3, 1, 4).reshape(S, hk, -1, d)
    s = torch.matmul(qp, kp.permute(0, 2, 3, 1)).mul_(st["scale"]).view(S, hk, hq // hk, MQ, MK)
    last = (lk - lq)[:, None] + iq                                            # the last key a row sees
    unseen = ik > torch.minimum(last, lk[:, None] - 1)[:, :, None]            # [S, MQ, MK]
    s.masked_fill_(unseen[:, None, None], float("-inf"))
    mx = s.amax(-1, keepdim=True)
    mx = torch.where(mx == float("-inf"), torch.zeros_like(mx), mx)
    s.sub_(mx).exp_()
    l = s.sum(-1, keepdim=True)
    o = torch.matmul(s.view(S, hk, -1, MK), vp.permute(0, 2, 1, 3)).view(S, hk, hq // hk, MQ, d)
    o = o / torch.where(l > 0, l, torch.ones_like(l))
    lse = (mx + torch.log(l))[..., 0]
    row = torch.arange(total, device=q.device)
    sq = torch.searchsorted(cu_q[1:].long(), row, right=True)
    at = row - cu_q.long()[sq]
    o = o.permute(0, 3, 1, 2, 4)[sq, at].reshape(total, hq, d).to(torch.bfloat16)
    return {"o": o, "lse": lse.permute(0, 3, 1, 2)[sq, at].reshape(total, hq)}


def _scale_exponent(amax, fmt):
    """The least e >= -120 with amax <= TOP 2^e (0 in a block of zeros: -120)."""
    mant, ex = torch.frexp(amax)
    e = ex - TOP_EXP[fmt] + (mant > TOP_MANT[fmt]).to(ex.dtype)
    return torch.where(amax > 0, e.clamp(min=-120), torch.full_like(e, -120))


def _codes(x, e, fmt):
    y = torch.ldexp(x, -e)
    return y.to(torch.float8_e4m3fn).view(torch.int8) if fmt == "e4m3" else torch.round(y).to(torch.int8)


def _bytes(t):
    return t.view(torch.int8)


def _state(s):
    return {x: s[x] for x in ("k", "v", "k_scale", "v_scale", "k_tail", "v_tail", "counts")}


def _compact_plain(st):
    s, off, pos, fmt = st["store"], st["offsets"], st["kept_pos"].long(), st["fmt"]
    p = torch.arange(pos.numel(), device=pos.device)
    cell = torch.searchsorted(off[1:], p, right=True)
    row = p - off[cell]
    dest = s["base"][cell] + row
    n = (off[1:] - off[:-1])
    opened = row >= n[cell] // BLOCK * BLOCK
    # rows of complete blocks leave the ring as it is: they are sent to a spare slot behind it
    slot = torch.where(opened, cell * RING + row % RING, torch.full_like(row, s["k_tail"].shape[0] * RING))
    for x, src in (("k", st["K"]), ("v", st["V"])):
        r = src[cell, pos]
        f = r.float()
        amax = torch.zeros_like(s[x + "_scale"]).scatter_reduce_(0, dest // BLOCK, f.abs().amax(1), "amax")
        e = _scale_exponent(amax, fmt)
        used = torch.zeros_like(amax, dtype=torch.bool).index_fill_(0, dest // BLOCK, True)
        s[x + "_scale"].copy_(torch.where(used, torch.ldexp(torch.ones_like(amax), e), s[x + "_scale"]))
        _bytes(s[x]).index_copy_(0, dest, _codes(f, e[dest // BLOCK][:, None], fmt))
        ring = torch.cat([s[x + "_tail"].view(-1, st["d"]), r.new_zeros(1, st["d"])])
        ring.index_copy_(0, slot, r)
        s[x + "_tail"].copy_(ring[:-1].view_as(s[x + "_tail"]))
    s["counts"].copy_(n)
    return _state(s)


def _append_plain(s, new_k, new_v, d, fmt, take=None):
    """`take`: rows of each cell's m that are appended (all, where it is None)."""
    cells, m = new_k.shape[:2]
    n = s["counts"].long()
    t = torch.full_like(n, m) if take is None else take.long()
    i = torch.arange((m + 2 * BLOCK - 2) // BLOCK * BLOCK, device=n.device)   # rows of the blocks that m rows can touch
    row = (n // BLOCK * BLOCK)[:, None] + i                                   # [cells, rows]
    live = row < (n + t)[:, None]
    fresh = live & (row >= n[:, None])
    dest = (s["base"][:, None] + row)
    c = torch.arange(cells, device=n.device)[:, None].expand_as(row)
    for x, new in (("k", new_k), ("v", new_v)):
        old = s[x + "_tail"][c, row % RING]
        r = torch.where(fresh[..., None], new[c, (row - n[:, None]).clamp(0, m - 1)], old)
        f = torch.where(live[..., None], r, torch.zeros_like(r)).float().view(cells, -1, BLOCK, d)
        e = _scale_exponent(f.abs().amax((2, 3)), fmt)
        block = dest.view(cells, -1, BLOCK)[:, :, 0] // BLOCK
        any_live = live.view(cells, -1, BLOCK)[:, :, 0] & (t > 0)[:, None]
        s[x + "_scale"][block] = torch.where(any_live, torch.ldexp(torch.ones_like(f[:, :, 0, 0]), e),
                                             s[x + "_scale"][block])
        code = _codes(f, e[:, :, None, None], fmt).view(cells, -1, d)
        flat = dest.reshape(-1)
        _bytes(s[x])[flat] = torch.where(live[..., None], code, _bytes(s[x])[dest]).view(-1, d)
        # ring slots of rows that are not new get what they hold (slots repeat only beyond RING rows)
        slots = row[:, :RING] % RING
        s[x + "_tail"][c[:, :RING], slots] = torch.where(fresh[:, :RING, None], r[:, :RING], old[:, :RING])
    s["counts"].copy_(n + t)
    return _state(s)


def _attend_plain(st):
    s, q, fmt = st["store"], st["q"], st["fmt"]
    seqs, m, hq, d = q.shape
    hk = st["kv_heads"]
    n = s["counts"].long()
    cells = n.numel()
    j = torch.arange(st["max_n"], device=q.device)
    row = (s["base"][:, None] + j).clamp_(max=s["k"].shape[0] - 1)
    kv = [(_bytes(s[x])[row].view(_code_dtype(fmt)).float().mul_(s[x + "_scale"][row // BLOCK][..., None])) for x in "kv"]
    qc = q.view(seqs, m, hk, hq // hk, d).permute(0, 2, 1, 3, 4).reshape(cells, -1, d).float()  # rows (token, head)
    x = torch.matmul(qc, kv[0].transpose(1, 2)).mul_(st["scale"]).view(cells, m, hq // hk, -1)
    seen = n[:, None] - m + 1 + torch.arange(m, device=q.device)                                # keys a token sees
    x.masked_fill_((j >= seen[..., None])[:, :, None], float("-inf"))
    mx = x.amax(-1, keepdim=True)
    mx = torch.where(mx == float("-inf"), torch.zeros_like(mx), mx)
    x.sub_(mx).exp_()
    l = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(cells, -1, j.numel()), kv[1]).view(cells, m, hq // hk, d)
    o = o / torch.where(l > 0, l, torch.ones_like(l))
    lse = (mx + torch.log(l))[..., 0]
    o = o.view(seqs, hk, m, -1, d).permute(0, 2, 1, 3, 4).reshape(seqs, m, hq, d).to(torch.bfloat16)
    return {"o": o, "lse": lse.view(seqs, hk, m, -1).permute(0, 2, 1, 3).reshape(seqs, m, hq)}


def run(st):
    op = st["op"]
    if own:
        from paper_2608_25230_gb300 import fw

        if op == "prompt":
            r = fw.prompt_attention(st["q"], st["k"], st["v"], st["cu_q"], st["cu_k"], scale=st["scale"], out=st["out"])
            return {"o": r["o"], "lse": r["lse"]}
        if op == "compact":
            fw.cache8_compact(st["cache"], st["K"], st["V"], st["offsets"], st["kept_pos"])
            return _state(st["store"])
        if op == "append":  # (the counts of a draft that was not accepted are set back like this)
            st["store"]["counts"].copy_(st["counts0"])
            fw.cache8_append(st["cache"], st["new_k"], st["new_v"])
            return _state(st["store"])
        r = fw.cache8_attend(st["cache"], st["q"], kv_heads=st["kv_heads"], scale=st["scale"], out=st["out"],
                             workspace=st["workspace"])
        return {"o": r["o"], "lse": r["lse"]}
    if op == "prompt":
        return _prompt_plain(st)
    if op == "compact":
        return _compact_plain(st)
    if op == "append":
        st["store"]["counts"].copy_(st["counts0"])
        return _append_plain(st["store"], st["new_k"], st["new_v"], st["d"], st["fmt"])
    return _attend_plain(st)


# ---------------------------------------------------------------- in 64 bits
def _softmax64(q, k, v, seen, scale):
    """One head: q [rows, d], k, v [keys, d] in 64 bits, row r sees keys below seen[r]."""
    o = torch.zeros(q.shape[0], v.shape[1], dtype=torch.float64, device=q.device)
    lse = torch.full((q.shape[0],), float("-inf"), dtype=torch.float64, device=q.device)
    for a in range(0, q.shape[0], 4096):
        lo = seen[a:a + 4096]
        n = max(0, int(lo.max().item()))
        if n == 0:
            continue
        x = scale * (q[a:a + 4096] @ k[:n].T)
        x[torch.arange(n, device=q.device)[None] >= lo[:, None]] = float("-inf")
        z = torch.logsumexp(x, 1)
        lse[a:a + 4096] = z
        p = torch.exp(x - torch.where(torch.isinf(z), torch.zeros_like(z), z)[:, None])
        o[a:a + 4096] = p @ v[:n]
    return o, lse


def _quantise64(rows, fmt):
    """Codes' values of rows [n, d] in 64 bits and the scale of each of their blocks, from the
    definition: the least power of two (from 2^-120 on) that holds the block, then the nearest
    code, to even on ties."""
    n, d = rows.shape
    x = torch.cat([rows, rows.new_zeros(-n % BLOCK, d)]).view(-1, BLOCK * d)
    top = x.abs().max(1, keepdim=True).values
    scale = torch.full_like(top, 2.0 ** -120)
    for e in range(-119, 121):
        scale = torch.where(top > TOP[fmt] * scale, 2.0 * scale, scale)
    y = x / scale
    if fmt == "int8":
        y = torch.round(y)
    else:
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)  # spacing of the codes there
        y = torch.round(y / step) * step
    return y.view(-1, d)[:n], scale[:, 0]


def exact(case, seed):
    d, op = case["d"], case["op"]
    if op == "prompt":
        st = prepare(case, seed)
        lq, lk = _prompt_lengths(case)
        q, k, v = (st[x].double() for x in "qkv")
        g = case["group"]
        o, lse = torch.empty(q.shape, dtype=torch.float64, device=q.device), q.new_empty(q.shape[:2])
        aq = ak = 0
        for nq, nk in zip(lq, lk):
            seen = (torch.arange(nq, device=q.device) + nk - nq + 1).clamp(max=nk)
            for h in range(q.shape[1]):
                o[aq:aq + nq, h], lse[aq:aq + nq, h] = _softmax64(q[aq:aq + nq, h], k[ak:ak + nk, h // g], v[ak:ak + nk, h // g],
                                                                 seen, st["scale"])
            aq, ak = aq + nq, ak + nk
        return {"o": o, "lse": lse}
    st = prepare(case, seed)
    s, fmt = st["store"], case["fmt"]
    if op == "attend":
        n, m, g = _cell_counts(case), case["m"], case["group"]
        q = st["q"].double()
        o, lse = torch.empty(q.shape, dtype=torch.float64, device=q.device), q.new_empty(q.shape[:3])
        base = s["base"].tolist()
        for c, cnt in enumerate(n):
            b, h = divmod(c, case["kv_heads"])
            rows = slice(base[c], base[c] + cnt)
            blocks = (torch.arange(cnt, device=q.device) + base[c]) // BLOCK
            k, v = (s[x][rows].double() * s[x + "_scale"][blocks].double()[:, None] for x in "kv")
            seen = (torch.arange(m, device=q.device) + cnt - m + 1).clamp(min=0).repeat_interleave(g)
            oc, lc = _softmax64(q[b, :, h * g:(h + 1) * g].reshape(-1, d), k, v, seen, st["scale"])
            o[b, :, h * g:(h + 1) * g], lse[b, :, h * g:(h + 1) * g] = oc.view(m, g, d), lc.view(m, g)
        return {"o": o, "lse": lse}
    # the store after the call: the codes of every touched block from its rows
    cells = s["base"].numel()
    out = {x: None for x in ("k", "v", "k_scale", "v_scale", "k_tail", "v_tail", "counts")}
    base = s["base"].tolist()
    off = st["offsets"].tolist() if op == "compact" else None
    n0 = [0] * cells if op == "compact" else _append_counts(case)
    for x in "kv":
        vals, sc, ring = s[x].double(), s[x + "_scale"].double(), s[x + "_tail"].double()
        for c in range(cells):
            first = n0[c] // BLOCK * BLOCK
            if op == "compact":
                rows = st["KV"["kv".index(x)]][c, st["kept_pos"][off[c]:off[c + 1]].long()].double()
            else:
                held = s[x + "_tail"][c, torch.arange(first, n0[c]) % RING].double()
                rows = torch.cat([held, st["new_" + x][c].double()])
            end = first + rows.shape[0]
            y, scale = _quantise64(rows, fmt)
            vals[base[c] + first:base[c] + end] = y
            sc[(base[c] + first) // BLOCK:(base[c] + first) // BLOCK + scale.numel()] = scale
            a = end // BLOCK * BLOCK if op == "compact" else n0[c]
            ring[c, torch.arange(a, end) % RING] = rows[a - first:]
        out.update({x: vals if fmt == "e4m3" else None, x + "_scale": sc, x + "_tail": ring})
    return out

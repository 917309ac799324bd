"""A prompt, its cache evicted into pages, and beams decoded after it that share what they have in common.

One sequence through the attention of a stack of layers with random projections: queries and keys normed and rotated, the
prompt's attention, the observation window's score of its keys, ContourKV's budgets, the kept rows compacted into pages.
The beams fork from it and decode: per token and layer rotation, append and attention over the pages; every few tokens
the beams change places, and half way the heads are evicted again inside their pages.  Prints how many pages the beams hold
together and what they would hold apart.

    python examples/beams_decode.py [--tokens 2048] [--layers 2] [--beams 4] [--steps 16] [--keep 0.25]
"""
import argparse
import math
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2608_25230_gb300 import fw  # noqa: E402


def run(*, tokens=2048, layers=2, beams=4, kv_heads=8, group=4, d=128, steps=16, keep=0.25, window=32, page_rows=32, seed=0):
    """Returns a dict: the pages, the decoded outputs and a record of what came in, step by step."""
    gen = torch.Generator("cuda").manual_seed(seed)
    heads, cells, scale = kv_heads * group, layers * kv_heads, 1.0 / math.sqrt(d)
    inv_freq = (1e4 ** (-torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d)).float()
    weights = [(1 + 0.1 * torch.randn(d, generator=gen, device="cuda")).to(torch.bfloat16) for _ in "qk"]

    def project(rows):
        """A projection's queries, keys and values, side by side as a model has them."""
        x = torch.randn(rows, heads + 2 * kv_heads, d, generator=gen, device="cuda", dtype=torch.bfloat16)
        return x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:]

    def rotate(q, k, positions, out=None):
        return fw.qk_rotate(q, k, positions, inv_freq, q_weight=weights[0], k_weight=weights[1], eps=1e-6, out=out)

    # the prompt: rotated keys go straight into the caches of heads that the score and the compaction read
    K = torch.empty(cells, tokens, d, dtype=torch.bfloat16, device="cuda")
    V = torch.empty_like(K)
    pos = torch.arange(tokens, dtype=torch.int32, device="cuda")
    bounds = torch.tensor([0, tokens], dtype=torch.int32, device="cuda")
    w, prompt, Qw = min(window, tokens), [], []
    for layer in range(layers):
        cut = slice(layer * kv_heads, (layer + 1) * kv_heads)
        q, k, v = project(tokens)
        V[cut].copy_(v.transpose(0, 1))
        qr, kr = rotate(q, k, pos, out=(torch.empty(tokens, heads, d, dtype=torch.bfloat16, device="cuda"), K[cut].transpose(0, 1)))
        prompt.append(fw.prompt_attention(qr, kr, v, bounds, scale=scale)["o"])
        Qw.append(qr[-w:].view(w, kv_heads, group, d).float().mean(2).to(torch.bfloat16).transpose(0, 1))
    scores, _ = fw.window_score(torch.cat(Qw).contiguous(), K, scale=scale)
    budget = max(cells * w, int(cells * tokens * keep))
    kept = fw.contour_alloc(scores, floor=w, total_budget=budget, uniform_s=budget // cells)

    # pages for all layers' cells [layer][beam][head]; the kept rows become the first beam's
    entries = -(-(tokens + steps) // page_rows) + 1
    # (room for what the beams share, and for what each keeps for itself when it is evicted again)
    pages = fw.pages_empty(layers * beams * kv_heads, (1 + beams) * (budget // page_rows + 4 * cells), d, max_pages=entries,
                           page_rows=page_rows)
    status = torch.empty(pages.cells, dtype=torch.int32, device="cuda")
    per = beams * kv_heads
    parts = [pages.part(layer * per, per) for layer in range(layers)]
    statuses = []

    def check(part):
        statuses.append(status[:part.cells].clone())

    for layer in range(layers):
        cut = slice(layer * kv_heads, (layer + 1) * kv_heads)
        first = pages.part(layer * per, kv_heads)
        fw.pages_compact(first, K[cut], V[cut], kept["offsets"][cut.start:cut.stop + 1].contiguous(), kept["kept_pos"],
                         status=status)
        check(first)
    places = torch.arange(pages.cells, dtype=torch.int32, device="cuda") // per * per
    places += torch.arange(kv_heads, dtype=torch.int32, device="cuda").repeat(layers * beams)
    fw.pages_fork(pages, places, status=status)  # every beam begins as the first
    check(pages)
    record = [("fork", places.clone())]

    workspace = fw.pages_append_workspace(parts[0], 1)
    decoded = []
    for step in range(steps):
        at = torch.full((beams,), tokens + step, dtype=torch.int32, device="cuda")
        for layer, part in enumerate(parts):
            q, k, v = project(beams)
            qr, kr = rotate(q, k, at)
            kr, v = kr.unsqueeze(1), v.unsqueeze(1)  # [beams][one token][heads][d]
            fw.pages_append(part, kr, v, status=status, workspace=workspace)
            check(part)
            out = fw.pages_attend(part, qr.unsqueeze(1), kv_heads=kv_heads, scale=scale, longest=tokens + steps)
            statuses.append(out["status"])
            decoded.append(out["o"][:, 0])
            record.append(("append", layer, kr, v, qr))
        if step % 4 == 3:  # the beams that go on: some twice, others no more
            best = torch.randint(0, beams, (beams,), generator=gen, device="cuda")
            places = (torch.arange(layers, device="cuda")[:, None, None] * per + best[None, :, None] * kv_heads +
                      torch.arange(kv_heads, device="cuda")).flatten().to(torch.int32)
            fw.pages_fork(pages, places, status=status)
            check(pages)
            record.append(("fork", places))
        if step == steps // 2:  # the heads evicted again: every second row and the last `window`
            rows = [[r for r in range(n) if r % 2 == 0 or r >= n - w] for n in pages.counts.tolist()]
            offsets = torch.tensor([0] + [len(r) for r in rows], device="cuda").cumsum(0)
            positions = torch.tensor([r for x in rows for r in x], dtype=torch.int32, device="cuda")
            fw.pages_keep(pages, offsets, positions, status=status)
            check(pages)
            record.append(("keep", rows))
    return dict(pages=pages, prompt=prompt, kept=kept, K=K, V=V, decoded=decoded, record=record, statuses=statuses,
                shape=(layers, beams, kv_heads, group, d), scale=scale)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--beams", type=int, default=4)
    ap.add_argument("--steps", type=int, default=16)
    ap.add_argument("--keep", type=float, default=0.25)
    a = ap.parse_args()
    r = run(tokens=a.tokens, layers=a.layers, beams=a.beams, steps=a.steps, keep=a.keep)
    torch.cuda.synchronize()
    p = r["pages"]
    bad = sum(int(s.count_nonzero()) for s in r["statuses"])
    print(f"{a.beams} beams, {int(p.counts.sum())} rows in {int((p.refs > 0).sum())} pages ({int(p.held.sum())} apart), "
          f"{bad} cells with a status")


if __name__ == "__main__":
    main()

"""A prompt, its cache evicted and held in 8 bits, and the tokens decoded after it.

One sequence through the attention of a stack of layers with random weights' worth of queries, keys and values:
the prompt's attention, the observation window's score of its keys, ContourKV's budgets, the kept rows compacted into the
8-bit store, then per token and layer an append and the attention over the store.  Prints what the eviction and the 8 bits
cost against attention over the whole cache.

    python examples/evicted_decode.py [--tokens 4096] [--layers 4] [--steps 16] [--keep 0.25] [--fmt e4m3]
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


def run(*, tokens=4096, layers=4, kv_heads=8, group=4, d=128, steps=16, keep=0.25, window=32, fmt="e4m3", seed=0):
    """Returns a dict: the inputs, the prompt's outputs, the store, the decoded outputs and what the whole cache gives."""
    gen = torch.Generator("cuda").manual_seed(seed)
    heads, cells, scale = kv_heads * group, layers * kv_heads, 1.0 / math.sqrt(d)

    def rand(*shape):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.bfloat16)

    # the caches of all layers, a head's rows together: [layers x heads][tokens][d]
    # (a head's queries look along one direction, and a few of its keys lie along it, more of them in some heads)
    K, V, u = rand(cells, tokens, d), rand(cells, tokens, d), rand(cells, 1, d)
    share = torch.rand(cells, 1, 1, generator=gen, device="cuda") * 2 * keep
    K += 0.6 * u * (torch.rand(cells, tokens, 1, generator=gen, device="cuda") < 0.5 * share)
    look = u.view(layers, 1, kv_heads, 1, d).expand(layers, 1, kv_heads, group, d).reshape(layers, 1, heads, d)
    q = rand(layers, tokens, heads, d) * 0.5 + look
    bounds = torch.tensor([0, tokens], dtype=torch.int32, device="cuda")
    prompt = []
    for layer in range(layers):  # (the prompt call reads [tokens][heads][d] through strides)
        k, v = (x[layer * kv_heads:(layer + 1) * kv_heads].transpose(0, 1) for x in (K, V))
        prompt.append(fw.prompt_attention(q[layer], k, v, bounds, scale=scale))

    # the last queries of each KV head's group judge the keys; budgets over all layers and heads at once
    w = min(window, tokens)
    Qw = q[:, -w:].view(layers, w, kv_heads, group, d).float().mean(3).to(torch.bfloat16)
    Qw = Qw.permute(0, 2, 1, 3).reshape(cells, w, d).contiguous()
    scores, _ = fw.window_score(Qw, K, scale=scale)
    budget = max(cells * min(w, tokens), int(cells * tokens * keep))
    kept = fw.contour_alloc(scores, floor=w, total_budget=budget, uniform_s=budget // cells)

    cache = fw.cache8_empty(kept["offsets"], budget, d, fmt=fmt, room=steps)
    status = torch.empty(cells, dtype=torch.int32, device="cuda")
    fw.cache8_compact(cache, K, V, kept["offsets"], kept["kept_pos"], status=status)

    # decoding: each layer appends its heads' new rows and attends over what it kept
    parts = [cache.part(layer * kv_heads, kv_heads) for layer in range(layers)]
    workspace = fw.cache8_attend_workspace(parts[0], rand(1, 1, heads, d), kv_heads=kv_heads)
    decoded, whole, drawn = [], [], []
    for _ in range(steps):
        for layer, part in enumerate(parts):
            new_k, new_v = rand(kv_heads, 1, d), rand(kv_heads, 1, d)
            new_q = rand(1, 1, heads, d) * 0.5 + look[layer]
            drawn.append((new_k, new_v, new_q))
            fw.cache8_append(part, new_k, new_v)
            out = fw.cache8_attend(part, new_q, kv_heads=kv_heads, scale=scale, workspace=workspace)
            decoded.append(out["o"][0, 0])
            # what the whole cache in 16 bits gives, by the prompt call of one token
            cut = slice(layer * kv_heads, (layer + 1) * kv_heads)
            k, v = (torch.cat([x[cut], y], 1).transpose(0, 1) for x, y in ((K, new_k), (V, new_v)))
            one = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
            ref = fw.prompt_attention(new_q[0], k, v, one, torch.tensor([0, tokens + 1], dtype=torch.int32, device="cuda"),
                                      scale=scale)
            whole.append(ref["o"][0])
    return dict(prompt=prompt, kept=kept, cache=cache, status=status, K=K, V=V, drawn=drawn,
                decoded=torch.stack(decoded), whole=torch.stack(whole))


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--steps", type=int, default=16)
    ap.add_argument("--keep", type=float, default=0.25)
    ap.add_argument("--fmt", choices=("e4m3", "int8"), default="e4m3")
    a = ap.parse_args()
    r = run(tokens=a.tokens, layers=a.layers, steps=a.steps, keep=a.keep, fmt=a.fmt)
    torch.cuda.synchronize()
    counts = r["cache"].counts.float()
    err = (r["decoded"].float() - r["whole"].float()).norm() / r["whole"].float().norm()
    print(f"kept {int(r['kept']['offsets'][-1])} of {r['cache'].cells * a.tokens} rows in 8 bits "
          f"({counts.min():.0f} to {counts.max():.0f} a head); decoded outputs {float(err):.3f} from the whole cache's")


if __name__ == "__main__":
    main()

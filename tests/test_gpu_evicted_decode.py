"""The serving calls together, as examples/evicted_decode.py runs them."""
import importlib.util
import math
import os

import pytest

from tests.attention64 import attend64, check_rows
from tests.test_gpu_cache8 import quantise64

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("evicted_decode", os.path.join(ROOT, "examples", "evicted_decode.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("tokens,d", [(333, 64), (700, 128)])
def test_example_path(example, fmt, tokens, d):
    steps, layers = 40, 2
    r = example.run(tokens=tokens, layers=layers, kv_heads=2, group=4, d=d, steps=steps, keep=0.3, fmt=fmt)
    torch.cuda.synchronize()
    kept, cache = r["kept"], r["cache"]
    assert not bool(r["status"].any())
    assert torch.equal(cache.counts, (kept["offsets"][1:] - kept["offsets"][:-1]).to(torch.int32) + steps)
    for p in r["prompt"]:
        assert bool(torch.isfinite(p["o"].float()).all()) and p["status"].tolist() == [0]
    assert bool(torch.isfinite(r["decoded"].float()).all())


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_nothing_evicted_is_the_whole_cache_in_8_bits(example, fmt):
    """With every row kept, the decoded outputs are attention over the quantised rows of the whole cache."""
    tokens, d, steps, layers = 300, 64, 3, 2
    r = example.run(tokens=tokens, layers=layers, kv_heads=2, group=2, d=d, steps=steps, keep=1.0, fmt=fmt, seed=5)
    torch.cuda.synchronize()
    rows = [[r["K"][c], r["V"][c]] for c in range(4)]
    scale, i = float(torch.tensor(1.0 / math.sqrt(d), dtype=torch.float32)), 0
    for _ in range(steps):
        for layer in range(layers):
            nk, nv, nq = r["drawn"][i]
            for h in range(2):
                c = layer * 2 + h
                rows[c] = [torch.cat([rows[c][0], nk[h]]), torch.cat([rows[c][1], nv[h]])]
                q64 = [torch.cat([v * s for v, s in (quantise64(x[b:b + 32], fmt) for b in range(0, x.shape[0], 32))])
                       for x in rows[c]]
                q = nq[0, 0, 2 * h:2 * h + 2].double()
                want = attend64(q, q64[0], q64[1], torch.full((2,), rows[c][0].shape[0], device="cuda"), scale)
                extra = 2.0 ** -24 * scale * float(q64[0].abs().sum(1).max()) * q.abs().amax(1)
                check_rows(r["decoded"][i][2 * h:2 * h + 2], None, want, 2.0 ** -11, extra)
            i += 1


def test_buffers_of_a_call_on_another_stream():
    """The outputs and the workspace that a call makes come from the memory of the stream that it runs on."""
    from paper_2608_25230_gb300 import fw

    def stream_of(ptr):
        for seg in torch.cuda.memory_snapshot():
            if seg["address"] <= ptr < seg["address"] + seg["total_size"]:
                return seg["stream"]

    side = torch.cuda.Stream()
    q = torch.randn(40, 4, 64, device="cuda").to(torch.bfloat16)
    bounds = torch.tensor([0, 40], dtype=torch.int32, device="cuda")
    want = fw.prompt_attention(q, q[:, :2], q[:, :2], bounds)
    cache = fw.cache8_empty(torch.arange(121, device="cuda") * 20, 2400, 64)
    qd = torch.randn(60, 1, 2, 64, device="cuda").to(torch.bfloat16)
    torch.cuda.synchronize()
    side.wait_stream(torch.cuda.current_stream())
    outs = [fw.prompt_attention(q, q[:, :2], q[:, :2], bounds, stream=side), fw.cache8_attend(cache, qd, kv_heads=2, stream=side)]
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(outs[0]["o"], want["o"]) and torch.equal(outs[0]["lse"], want["lse"])
    for out in outs:
        for x in out.values():
            assert stream_of(x.data_ptr()) == side.cuda_stream
    torch.cuda.synchronize()

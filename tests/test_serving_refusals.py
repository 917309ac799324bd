"""What the binding of the serving calls refuses before it calls the library (no GPU needed: nothing gets that far)."""
import pytest
import torch


@pytest.fixture(scope="module")
def fw():
    from paper_2608_25230_gb300 import _build

    _build.build()
    from paper_2608_25230_gb300 import fw as _fw

    return _fw


def bf(*shape):
    return torch.zeros(*shape, dtype=torch.bfloat16)


def store(**kw):
    a = dict(fmt="e4m3", k=torch.zeros(64, 64, dtype=torch.int8).view(torch.float8_e4m3fn),
             v=torch.zeros(64, 64, dtype=torch.int8).view(torch.float8_e4m3fn), k_scale=torch.ones(2), v_scale=torch.ones(2),
             k_tail=bf(2, 64, 64), v_tail=bf(2, 64, 64), base=torch.tensor([0, 32]),
             capacity=torch.tensor([32, 32], dtype=torch.int32), counts=torch.zeros(2, dtype=torch.int32))
    a.update(kw)
    return a


def test_prompt_refusals(fw):
    q, kv, cu = bf(5, 8, 64), bf(5, 2, 64), torch.tensor([0, 5], dtype=torch.int32)
    before = fw.launch_count()
    for args in [(q.float(), kv, kv, cu), (q, kv.half(), kv, cu), (q, kv, bf(4, 2, 64), cu), (q, bf(5, 2, 32), bf(5, 2, 32), cu),
                 (q, kv, kv, cu.long()), (q, kv, kv, cu, torch.tensor([0, 1, 5], dtype=torch.int32)),
                 (bf(5, 64, 8).transpose(1, 2), kv, kv, cu), (q, kv, kv, cu)]:  # (the last: not on a GPU)
        with pytest.raises(ValueError):
            fw.prompt_attention(*args)
    assert fw.launch_count() == before


def test_store_refusals(fw):
    bad = [dict(fmt="e5m2"), dict(fmt="int8"), dict(k_scale=torch.ones(3)), dict(k=torch.zeros(65, 64, dtype=torch.float8_e4m3fn)),
           dict(k_tail=bf(2, 32, 64)), dict(base=torch.tensor([0, 32], dtype=torch.int32)),
           dict(counts=torch.zeros(3, dtype=torch.int32)), dict(v_scale=torch.ones(4)[::2]), dict()]  # (the last: not on a GPU)
    for kw in bad:
        with pytest.raises(ValueError):
            fw.Cache8(**store(**kw))
    with pytest.raises(ValueError):
        fw.cache8_empty(torch.tensor([0, 3]), 3, 64, fmt="fp8")


def test_calls_on_a_store_refuse(fw):
    """A stand-in with the fields the checks read, so that no GPU is needed."""
    class Stand:
        cells, d, device, index = 2, 64, torch.device("cuda", 0), 0

    c, off, pos = Stand(), torch.tensor([0, 1, 2]), torch.zeros(2, dtype=torch.int32)
    K = bf(2, 9, 64)
    for args in [(K.float(), K, off, pos), (K, bf(2, 8, 64), off, pos), (bf(3, 9, 64), bf(3, 9, 64), off, pos),
                 (K, bf(9, 2, 64).transpose(0, 1), off, pos), (K, K, off.int(), pos), (K, K, off[:2], pos),
                 (K, K, off, pos.long()), (K, K, off, pos)]:
        with pytest.raises(ValueError):
            fw.cache8_compact(c, *args)
    for args in [(K.float(), K), (K, bf(2, 8, 64)), (bf(2, 18, 64)[:, ::2], bf(2, 18, 64)[:, ::2]), (bf(1, 9, 64), bf(1, 9, 64)),
                 (K, K)]:
        with pytest.raises(ValueError):
            fw.cache8_append(c, *args)
    for q, h in [(torch.zeros(1, 1, 4, 64), 2), (bf(1, 1, 4, 128), 2), (bf(1, 1, 5, 64), 2), (bf(2, 1, 4, 64), 2),
                 (bf(1, 1, 4, 64), 0), (bf(1, 1, 64, 4).transpose(2, 3), 2), (bf(1, 1, 4, 64), 2)]:
        with pytest.raises(ValueError):
            fw.cache8_attend(c, q, kv_heads=h)

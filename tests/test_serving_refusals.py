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


class On(torch.Tensor):
    """A tensor that says it is on the GPU of its `index`."""
    index = 0

    def get_device(self):
        return type(self).index


class OnSecond(On):
    index = 1


class StandInLibrary:
    """Takes the calls that the binding lets through."""
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 0
        return call


class StandInStream:
    def __init__(self, index, handle):
        self.device, self.cuda_stream = torch.device("cuda", index), handle


def serving_calls(fw, kind, stream=None):
    """The four calls and the workspace's on tensors of `kind`, ready to be made."""
    def t(*shape, dtype=torch.bfloat16):
        return torch.zeros(*shape, dtype=dtype).as_subclass(kind)

    class Stand:
        cells, d, device, index, _ref = 2, 64, torch.device("cpu"), kind.index, None

    i32, K, q = torch.int32, t(2, 9, 64), t(1, 1, 4, 64)
    outs = dict(o=t(1, 1, 4, 64), lse=t(1, 1, 4, dtype=torch.float32), status=t(2, dtype=i32))
    return {
        "fw_prompt_attention": lambda: fw.prompt_attention(t(5, 8, 64), t(5, 2, 64), t(5, 2, 64), t(2, dtype=i32), stream=stream,
                                                           out=dict(o=t(5, 8, 64))),
        "fw_cache8_compact": lambda: fw.cache8_compact(Stand(), K, K, t(3, dtype=torch.int64), t(2, dtype=i32), stream=stream),
        "fw_cache8_append": lambda: fw.cache8_append(Stand(), K, K, stream=stream),
        "fw_cache8_attend": lambda: fw.cache8_attend(Stand(), q, kv_heads=2, out=outs, workspace=t(256, dtype=torch.uint8),
                                                     stream=stream),
        "fw_cache8_attend_workspace": lambda: fw.cache8_attend_workspace(Stand(), q, kv_heads=2),
    }


def test_calls_off_the_current_gpu_are_refused(fw, monkeypatch):
    """The library launches on the current GPU: tensors or a stream of another one do not get that far."""
    lib = StandInLibrary()
    monkeypatch.setattr(fw, "_lib", lib)
    monkeypatch.setattr(fw, "_current_raw", lambda index: 70 + index)
    monkeypatch.setattr(fw, "_current_device", lambda: 0, raising=False)
    for name, call in serving_calls(fw, OnSecond).items():
        with pytest.raises(ValueError, match="current"):
            call()
    for name, call in serving_calls(fw, On, StandInStream(1, 5)).items():
        if name != "fw_cache8_attend_workspace":
            with pytest.raises(ValueError, match="stream"):
                call()
    assert not lib.calls
    # on the current GPU, with its current stream or one that is given
    for kind, index in ((On, 0), (OnSecond, 1)):
        monkeypatch.setattr(fw, "_current_device", lambda: index)
        for stream, handle in ((None, 70 + index), (StandInStream(index, 5), 5)):
            for name, call in serving_calls(fw, kind, stream).items():
                lib.calls.clear()
                call()
                assert [c[0] for c in lib.calls] == [name]
                if name != "fw_cache8_attend_workspace":
                    assert lib.calls[0][1][-1] == handle


def test_status_and_workspace_elsewhere_are_refused(fw, monkeypatch):
    """A status or a workspace that the GPU of the store does not hold, or not in one piece, does not reach the library."""
    lib = StandInLibrary()
    monkeypatch.setattr(fw, "_lib", lib)
    monkeypatch.setattr(fw, "_current_raw", lambda index: 0)
    monkeypatch.setattr(fw, "_current_device", lambda: 0)

    class Stand:
        cells, d, device, index, _ref = 2, 64, torch.device("cpu"), 0, None

    def t(*shape, dtype=torch.bfloat16, kind=On):
        return torch.zeros(*shape, dtype=dtype).as_subclass(kind)

    i32, u8, K, q = torch.int32, torch.uint8, t(2, 9, 64), t(1, 1, 4, 64)
    off, pos = t(3, dtype=torch.int64), t(2, dtype=i32)
    outs = dict(o=t(1, 1, 4, 64))
    for kind in (OnSecond, torch.Tensor):
        st, ws = t(2, dtype=i32, kind=kind), t(256, dtype=u8, kind=kind)
        with pytest.raises(ValueError):
            fw.cache8_compact(Stand(), K, K, off, pos, status=st)
        with pytest.raises(ValueError):
            fw.cache8_append(Stand(), K, K, status=st)
        with pytest.raises(ValueError):
            fw.cache8_attend(Stand(), q, kv_heads=2, out=outs, workspace=ws)
    with pytest.raises(ValueError):
        fw.cache8_attend(Stand(), q, kv_heads=2, out=outs, workspace=t(1, dtype=u8).expand(256))
    assert not lib.calls
    fw.cache8_append(Stand(), K, K, status=t(2, dtype=i32))
    fw.cache8_attend(Stand(), q, kv_heads=2, out=outs, workspace=t(256, dtype=u8))
    assert [c[0] for c in lib.calls] == ["fw_cache8_append", "fw_cache8_attend"]


def test_buffers_made_for_another_stream_come_from_its_memory(fw, monkeypatch):
    """What a call with stream= makes for itself is allocated on that stream: a block that the current stream has freed may
    still be in use there.  Outputs, which the caller reads, are recorded on the current stream."""
    import contextlib

    lib, side, made, recorded, inside = StandInLibrary(), StandInStream(0, 5), [], [], []

    @contextlib.contextmanager
    def on(stream):
        inside.append(stream)
        yield
        inside.pop()

    empty = torch.empty

    def noted(*args, **kw):
        made.append(inside[-1] if inside else None)
        return empty(*args, **kw)

    monkeypatch.setattr(fw, "_lib", lib)
    monkeypatch.setattr(fw, "_current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: "current")
    monkeypatch.setattr(torch, "empty", noted)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, s: recorded.append(s))

    class Stand:
        cells, d, device, index, _ref = 2, 64, torch.device("cpu"), 0, None

    def t(*shape, dtype=torch.bfloat16):
        return torch.zeros(*shape, dtype=dtype).as_subclass(On)

    fw.prompt_attention(t(5, 8, 64), t(5, 2, 64), t(5, 2, 64), t(2, dtype=torch.int32), stream=side)
    assert made == [side] * 3 and recorded == ["current"] * 3
    made.clear(), recorded.clear()
    fw.cache8_attend(Stand(), t(1, 1, 4, 64), kv_heads=2, stream=side)
    assert made == [side] * 4 and recorded == ["current"] * 3  # (the workspace is used on that stream only)
    made.clear(), recorded.clear()
    monkeypatch.setattr(fw, "_current_raw", lambda index: 0)
    fw.cache8_attend(Stand(), t(1, 1, 4, 64), kv_heads=2)
    assert made == [None] * 4 and not recorded and not inside

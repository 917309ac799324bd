"""What the calls on a cache in pages and the rotation refuse, in the library and in its binding (no GPU needed: nothing gets
that far)."""
import ctypes as C

import pytest
import torch

from tests.test_serving_refusals import On, OnSecond, StandInLibrary, StandInStream


@pytest.fixture(scope="module")
def fw():
    from paper_2608_25230_gb300 import _build

    _build.build()
    from paper_2608_25230_gb300 import fw as _fw

    return _fw


P = 256  # an address that is never read


def cache(fw, **kw):
    a = dict(cells=4, d=64, page_rows=16, num_pages=40, max_pages=9, k=P, v=P, table=P, held=P, counts=P, refs=P, free_bits=P,
             next=P)
    a.update(kw)
    return C.byref(fw.FwPages(**a))


def test_the_library_refuses_on_the_host(fw):
    I, U, W, lib = fw.FW_ERR_INVALID_ARG, fw.FW_ERR_UNSUPPORTED, fw.FW_ERR_WORKSPACE, fw._lib
    before = fw.launch_count()

    def rows(**kw):
        a = dict(kv_heads=2, m=3, k=P, v=P, k_seq=384, k_tok=128, k_head=64, v_seq=384, v_tok=128, v_head=64)
        a.update(kw)
        return C.byref(fw.FwPagesNew(**a))

    def query(**kw):
        a = dict(kv_heads=2, group=4, m=1, longest=0, q=P, q_seq=512, q_tok=512, q_head=64, scale=0.125)
        a.update(kw)
        return C.byref(fw.FwPagesQuery(**a))

    big = 1 << 40
    for want, kw in [(I, dict(cells=0)), (U, dict(d=96)), (U, dict(page_rows=8)), (U, dict(page_rows=48)), (I, dict(num_pages=0)),
                     (I, dict(max_pages=0)), (I, dict(k=None)), (I, dict(v=P + 8)), (I, dict(table=None)), (I, dict(held=None)),
                     (I, dict(counts=None)), (I, dict(refs=None)), (I, dict(free_bits=None)), (I, dict(next=None)),
                     (U, dict(num_pages=1 << 27)), (U, dict(cells=1 << 20, max_pages=1 << 11)), (U, dict(cells=(1 << 24) + 1)),
                     (U, dict(max_pages=1 << 27, cells=1))]:
        c = cache(fw, **kw)
        assert lib.fw_pages_append(c, rows(), P, P, big, None) == want, kw
        assert lib.fw_pages_compact(c, P, P, 9, 576, 64, P, P, 4, P, P, big, None) == want, kw
        assert lib.fw_pages_fork(c, P, P, P, big, None) == want, kw
        assert lib.fw_pages_attend(c, query(), P, P, P, P, big, None) == want, kw
        assert lib.fw_pages_append_workspace(c, 1) == lib.fw_pages_compact_workspace(c, 4) == lib.fw_pages_fork_workspace(c) == 0
        assert lib.fw_pages_attend_workspace(c, query()) == 0
    c = cache(fw)
    for want, kw in [(I, dict(kv_heads=3)), (I, dict(kv_heads=0)), (I, dict(m=0)), (I, dict(m=-1)), (I, dict(k=None)),
                     (I, dict(v=P + 2)), (I, dict(k_tok=4)), (I, dict(v_seq=1 << 40)), (U, dict(m=(1 << 29)))]:
        assert lib.fw_pages_append(c, rows(**kw), P, P, big, None) == want, kw
    assert lib.fw_pages_append(c, None, P, P, big, None) == I
    for args in [(None, P, 9, 576, 64, P, P, 4), (P, P + 2, 9, 576, 64, P, P, 4), (P, P, 0, 576, 64, P, P, 4),
                 (P, P, 9, 576, 63, P, P, 4), (P, P, 9, -8, 64, P, P, 4), (P, P, 9, 576, 64, None, P, 4),
                 (P, P, 9, 576, 64, P, None, 4), (P, P, 9, 576, 64, P, P, -1), (P, None, 9, 576, 64, P, P, 4),
                 (None, None, 0, 0, 0, None, P, 4)]:
        assert lib.fw_pages_compact(c, *args, P, P, big, None) == I, args
    assert lib.fw_pages_fork(c, None, P, P, big, None) == I
    for want, kw in [(I, dict(kv_heads=3)), (I, dict(kv_heads=0)), (I, dict(group=0)), (I, dict(m=0)), (I, dict(q=None)),
                     (I, dict(q=P + 8)), (I, dict(q_tok=4)), (I, dict(scale=-1.0)), (I, dict(scale=float("nan"))),
                     (I, dict(longest=-1)), (U, dict(group=256, m=512))]:
        assert lib.fw_pages_attend(c, query(**kw), P, P, P, P, big, None) == want, kw
    assert lib.fw_pages_attend(c, query(), None, P, P, P, big, None) == I
    # workspaces: missing, too small, misaligned
    for need, call in [(lib.fw_pages_append_workspace(c, 3), lambda w, n: lib.fw_pages_append(c, rows(), P, w, n, None)),
                       (lib.fw_pages_compact_workspace(c, 4),
                        lambda w, n: lib.fw_pages_compact(c, None, None, 0, 0, 0, P, P, 4, P, w, n, None)),
                       (lib.fw_pages_fork_workspace(c), lambda w, n: lib.fw_pages_fork(c, P, P, w, n, None)),
                       (lib.fw_pages_attend_workspace(c, query()), lambda w, n: lib.fw_pages_attend(c, query(), P, P, P, w, n, None))]:
        if need:
            assert call(None, need) == call(P, need - 1) == call(P + 8, need) == W

    def rotation(**kw):
        a = dict(rows=5, q_heads=4, kv_heads=2, d=64, rot=32, interleaved=0, w_dtype=1, eps=1e-6, q=P, k=P, q_out=P, k_out=P,
                 q_weight=P, k_weight=P, pos=P, inv_freq=P, q_row=512, q_head=64, k_row=512, k_head=64, q_out_row=256,
                 q_out_head=64, k_out_row=128, k_out_head=64)
        a.update(kw)
        return lib.fw_qk_rotate(C.byref(fw.FwRotation(**a)), None)

    for want, kw in [(I, dict(rows=-1)), (U, dict(rows=1 << 31)), (I, dict(q_heads=0)), (I, dict(kv_heads=-1)), (U, dict(d=72)),
                     (U, dict(d=272)), (I, dict(d=0, rot=0)), (I, dict(rot=80)), (I, dict(rot=-16)), (U, dict(rot=24)),
                     (I, dict(interleaved=2)), (I, dict(w_dtype=2)), (I, dict(eps=float("nan"))), (I, dict(eps=float("inf"))),
                     (I, dict(eps=-1.0)), (I, dict(q=None)), (I, dict(k=P + 8)), (I, dict(q_out=None)), (I, dict(k_out=P + 2)),
                     (I, dict(q_weight=P + 8)), (I, dict(pos=None)), (I, dict(inv_freq=None)), (I, dict(q_row=4)),
                     (I, dict(k_head=-4)), (I, dict(q_out_row=0)), (I, dict(k_out_head=-64)), (U, dict(q_heads=70000))]:
        assert rotation(**kw) == want, kw
    assert rotation(rows=0, q=None, pos=None) == fw.FW_OK
    assert lib.fw_qk_rotate(None, None) == I
    assert fw.launch_count() == before


def test_a_bound_beyond_the_tables_is_theirs(fw):
    """The way over the cells for a `longest` that no table holds, up to the largest number, is the one for full tables: here ranges,
    which want a workspace (clusters would not)."""
    for d, pages, cells in ((64, 200, 100), (128, 5000, 300)):
        c = cache(fw, d=d, max_pages=pages, cells=cells)
        for longest in (16 * pages, 16 * pages + 1, 1 << 30, (1 << 31) - 16, (1 << 31) - 15, (1 << 31) - 1):
            q = C.byref(fw.FwPagesQuery(kv_heads=2, group=4, m=1, longest=longest, q=P, q_seq=512, q_tok=512, q_head=64, scale=0.125))
            assert fw._lib.fw_pages_attend(c, q, P, P, P, None, 0, None) == fw.FW_ERR_WORKSPACE, longest


def test_an_attention_workspace_serves_every_bound(fw):
    for d, cells, group, m in ((64, 8, 4, 1), (128, 64, 4, 5), (128, 2, 16, 4)):
        c, size = cache(fw, d=d, max_pages=5000, cells=cells), set()
        for longest in (0, 1, 100, 3000, 80000, (1 << 31) - 1):
            q = fw.FwPagesQuery(kv_heads=2, group=group, m=m, longest=longest, q=P, q_seq=512, q_tok=512, q_head=64, scale=0.125)
            size.add(fw._lib.fw_pages_attend_workspace(c, C.byref(q)))
        assert len(size) == 1 and min(size) > 0, size


def bf(*shape, kind=torch.Tensor):
    return torch.zeros(*shape, dtype=torch.bfloat16).as_subclass(kind)


def i32(*shape, kind=torch.Tensor):
    return torch.zeros(*shape, dtype=torch.int32).as_subclass(kind)


def tensors(**kw):
    a = dict(k=bf(5, 16, 64), v=bf(5, 16, 64), table=i32(2, 3), held=i32(2), counts=i32(2), refs=i32(5), free=i32(1), next=i32(1))
    a.update(kw)
    return a


class Stand:
    """The fields of a cache that the checks read, so that no GPU is needed."""
    cells, d, device, index, _ref = 2, 64, torch.device("cpu"), 0, None


def test_cache_refusals(fw):
    for kw in [dict(k=bf(5, 16, 32)), dict(k=bf(5, 8, 64), v=bf(5, 8, 64)), dict(k=bf(80, 64), v=bf(80, 64)),
               dict(v=bf(4, 16, 64)), dict(k=bf(5, 16, 64).float()), dict(table=i32(6)), dict(held=i32(3)), dict(counts=i32(1)),
               dict(refs=i32(6)), dict(free=i32(2)), dict(next=i32(2)), dict(counts=i32(2).long()), dict(table=i32(3, 2).T),
               dict(k=bf(5, 64, 16).transpose(1, 2)), dict()]:  # (the last: not on a GPU)
        with pytest.raises(ValueError):
            fw.Pages(**tensors(**kw))


def test_calls_refuse(fw, monkeypatch):
    lib = StandInLibrary()
    monkeypatch.setattr(fw, "_lib", lib)
    monkeypatch.setattr(fw, "_current_raw", lambda index: 0)
    monkeypatch.setattr(fw, "_current_device", lambda: 0)
    c, on = Stand(), dict(kind=On)
    off, pos, x, ws = torch.zeros(3, dtype=torch.int64).as_subclass(On), i32(4, **on), bf(1, 3, 2, 64, **on), bf(256, **on)
    for k, v in [(x.float(), x), (x, bf(1, 2, 2, 64, **on)), (bf(2, 3, 2, 64, **on), bf(2, 3, 2, 64, **on)),
                 (bf(1, 3, 2, 128, **on), bf(1, 3, 2, 128, **on)), (bf(1, 0, 2, 64, **on), bf(1, 0, 2, 64, **on)),
                 (bf(1, 3, 64, 2, **on).transpose(2, 3), x), (bf(1, 3, 2, 64), x), (x, bf(1, 3, 2, 64, kind=OnSecond))]:
        with pytest.raises(ValueError):
            fw.pages_append(c, k, v, workspace=ws)
    K = bf(2, 9, 64, **on)
    for args in [(K.float(), K, off, pos), (K, bf(2, 8, 64, **on), off, pos), (bf(3, 9, 64, **on), bf(3, 9, 64, **on), off, pos),
                 (K, bf(9, 2, 64, **on).transpose(0, 1), off, pos), (K, K, off.int(), pos), (K, K, off[:2], pos),
                 (K, K, off, pos.long()), (K, K, off, i32(8, **on)[::2]), (bf(2, 9, 64), K, off, pos), (K, K, off, i32(4))]:
        with pytest.raises(ValueError):
            fw.pages_compact(c, *args, workspace=ws)
        if args[0] is K and args[1] is K:
            with pytest.raises(ValueError):
                fw.pages_keep(c, *args[2:], workspace=ws)
    for src in (i32(3, **on), i32(2, **on).long(), i32(4, **on)[::2], i32(2)):
        with pytest.raises(ValueError):
            fw.pages_fork(c, src, workspace=ws)
    q = bf(1, 1, 4, 64, **on)
    for args, h in [(q.float(), 2), (bf(1, 1, 4, 128, **on), 2), (bf(1, 1, 5, 64, **on), 2), (bf(2, 1, 4, 64, **on), 2), (q, 0),
                    (bf(1, 1, 64, 4, **on).transpose(2, 3), 2), (bf(1, 1, 4, 64), 2)]:
        with pytest.raises(ValueError):
            fw.pages_attend(c, args, kv_heads=h, workspace=ws)
    # statuses and workspaces elsewhere, or not in one piece
    for kind in (OnSecond, torch.Tensor):
        st, w = i32(2, kind=kind), bf(256, kind=kind)
        for kw in (dict(status=st, workspace=ws), dict(workspace=w)):
            for call in (lambda: fw.pages_append(c, x, x, **kw), lambda: fw.pages_compact(c, K, K, off, pos, **kw),
                         lambda: fw.pages_keep(c, off, pos, **kw), lambda: fw.pages_fork(c, i32(2, **on), **kw)):
                with pytest.raises(ValueError):
                    call()
        with pytest.raises(ValueError):
            fw.pages_attend(c, q, kv_heads=2, out=dict(o=q), workspace=w)
    f, p = torch.zeros(16).as_subclass(On), i32(5, **on)
    a, b, w = bf(5, 4, 64, **on), bf(5, 2, 64, **on), bf(64, **on)
    for args, kw in [((a.float(), b, p, f), {}), ((a, bf(4, 2, 64, **on), p, f), {}), ((a, bf(5, 2, 32, **on), p, f), {}),
                     ((a, b, p.long(), f), {}), ((a, b, i32(4, **on), f), {}), ((a, b, p, f.double()), {}),
                     ((a, b, p, torch.zeros(4, 4).as_subclass(On)), {}), ((a, b, p, f), dict(q_weight=w)),
                     ((a, b, p, f), dict(q_weight=w, k_weight=w.float(), eps=0.0)), ((a, b, p, f), dict(eps=-1.0)),
                     ((a, b, p, f), dict(q_weight=bf(32, **on), eps=0.0)), ((a, b, p, f), dict(q_weight=w.half(), eps=0.0)),
                     ((bf(5, 64, 4, **on).transpose(1, 2), b, p, f), {}), ((bf(5, 4, 64), b, p, f), {}),
                     ((a, b, i32(5, kind=OnSecond), f), {}), ((a, b, p, f), dict(out=(a, None))),
                     ((a, b, p, f), dict(out=(b, b))), ((a, b, p, f), dict(out=(a.float(), b)))]:
        with pytest.raises(ValueError):
            fw.qk_rotate(*args, **kw)
    assert not lib.calls


def calls(fw, kind, stream=None):
    x, K = bf(1, 3, 2, 64, kind=kind), bf(2, 9, 64, kind=kind)
    off, pos, ws = torch.zeros(3, dtype=torch.int64).as_subclass(kind), i32(4, kind=kind), bf(256, kind=kind)
    q = bf(1, 1, 4, 64, kind=kind)

    class Here(Stand):
        index = kind.index

    kw = dict(workspace=ws, stream=stream)
    c, a, b = Here(), bf(5, 4, 64, kind=kind), bf(5, 2, 64, kind=kind)
    return [("fw_pages_append", lambda: fw.pages_append(c, x, x, **kw)),
            ("fw_pages_compact", lambda: fw.pages_compact(c, K, K, off, pos, **kw)),
            ("fw_pages_compact", lambda: fw.pages_keep(c, off, pos, **kw)),
            ("fw_pages_fork", lambda: fw.pages_fork(c, i32(2, kind=kind), **kw)),
            ("fw_pages_attend", lambda: fw.pages_attend(c, q, kv_heads=2, out=dict(o=q), **kw)),
            ("fw_qk_rotate", lambda: fw.qk_rotate(a, b, i32(5, kind=kind), torch.zeros(16).as_subclass(kind), out=(a, b), stream=stream))]


def test_calls_off_the_current_gpu_are_refused(fw, monkeypatch):
    lib = StandInLibrary()
    monkeypatch.setattr(fw, "_lib", lib)
    monkeypatch.setattr(fw, "_current_raw", lambda index: 70 + index)
    monkeypatch.setattr(fw, "_current_device", lambda: 0)
    for _, call in calls(fw, OnSecond):
        with pytest.raises(ValueError, match="current"):
            call()
    for _, call in calls(fw, On, StandInStream(1, 5)):
        with pytest.raises(ValueError, match="stream"):
            call()
    assert not lib.calls
    for stream, handle in ((None, 70), (StandInStream(0, 5), 5)):
        for name, call in calls(fw, On, stream):
            lib.calls.clear()
            call()
            assert [c[0] for c in lib.calls] == [name] and lib.calls[0][1][-1] == handle


def test_buffers_made_for_another_stream_come_from_its_memory(fw, monkeypatch):
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
    c, x, q = Stand(), bf(1, 3, 2, 64, kind=On), bf(1, 1, 4, 64, kind=On)
    fw.pages_append(c, x, x, stream=side)
    fw.pages_fork(c, i32(2, kind=On), stream=side)
    assert made == [side] * 2 and not recorded
    made.clear()
    fw.pages_attend(c, q, kv_heads=2, stream=side)
    assert made == [side] * 4 and recorded == ["current"] * 3
    made.clear(), recorded.clear()
    fw.qk_rotate(bf(5, 4, 64, kind=On), bf(5, 2, 64, kind=On), i32(5, kind=On), torch.zeros(16).as_subclass(On), stream=side)
    assert made == [side] * 2 and recorded == ["current"] * 2

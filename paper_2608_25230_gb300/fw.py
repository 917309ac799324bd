"""Thin ctypes binding of libfw.so (include/fw.h).

Marshalling only: every step of the computation runs in the library's CUDA
kernels.  torch provides device memory and the current stream; the library
never allocates.  If libfw.so is missing this module raises on import -- there
is no fallback path.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import math
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfw.so")

FW_OK, FW_ERR_INVALID_ARG, FW_ERR_UNSUPPORTED, FW_ERR_CUDA = 0, 1, 2, 3
FW_ERR_TIMEOUT, FW_ERR_WORKSPACE, FW_ERR_NONFINITE = 4, 5, 6
FW_F32, FW_BF16 = 0, 1

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
                      "(nvcc, sm_103a); there is no CPU fallback")
_lib = C.CDLL(LIB_PATH)

vp = C.c_void_p


class FwRows(C.Structure):
    _fields_ = [("num_groups", C.c_int64), ("rows_per_group", C.c_int32), ("d", C.c_int32),
                ("max_n", C.c_int32), ("v_dtype", C.c_int32), ("logits", vp), ("logit_off", vp),
                ("n", vp), ("v", vp), ("v_off", vp)]


class FwGapOut(C.Structure):
    _fields_ = [("o", vp), ("o_kept", vp), ("gap", vp), ("dropped", vp), ("phi", vp), ("row_max", vp),
                ("row_sum", vp), ("thr_key", vp), ("thr_idx", vp), ("kept_bits", vp),
                ("kept_words", C.c_int32), ("row_status", vp)]


class FwBestSubsetStats(C.Structure):
    _fields_ = [("rows_exhaustive", C.c_int64), ("candidates", C.c_int64), ("inner_nodes", C.c_uint64),
                ("inner_leaves", C.c_uint64), ("inner_ops", C.c_uint64), ("skipped", C.c_uint64)]


class FwSwapParams(C.Structure):
    _fields_ = [("E", C.c_int32), ("max_swaps", C.c_int32)]


class FwPrompt(C.Structure):
    _fields_ = [("num_seqs", C.c_int32), ("q_heads", C.c_int32), ("kv_heads", C.c_int32), ("d", C.c_int32),
                ("total_q", C.c_int64), ("total_k", C.c_int64), ("q", vp), ("k", vp), ("v", vp),
                ("q_row", C.c_int64), ("q_head", C.c_int64), ("k_row", C.c_int64), ("k_head", C.c_int64),
                ("v_row", C.c_int64), ("v_head", C.c_int64), ("cu_q", vp), ("cu_k", vp), ("scale", C.c_float)]


class FwCache8(C.Structure):
    _fields_ = [("cells", C.c_int32), ("d", C.c_int32), ("format", C.c_int32), ("rows", C.c_int64), ("k", vp),
                ("v", vp), ("k_scale", vp), ("v_scale", vp), ("k_tail", vp), ("v_tail", vp), ("base", vp),
                ("capacity", vp), ("counts", vp)]


class FwCache8Query(C.Structure):
    _fields_ = [("kv_heads", C.c_int32), ("group", C.c_int32), ("m", C.c_int32), ("q", vp), ("q_seq", C.c_int64),
                ("q_tok", C.c_int64), ("q_head", C.c_int64), ("scale", C.c_float)]


_lib.fw_prompt_attention.argtypes = [C.POINTER(FwPrompt), vp, vp, vp, vp]
_lib.fw_cache8_compact.argtypes = [C.POINTER(FwCache8), vp, vp, C.c_int32, C.c_int64, C.c_int64, vp, vp, C.c_int64, vp,
                                   vp]
_lib.fw_cache8_append.argtypes = [C.POINTER(FwCache8), vp, vp, C.c_int32, vp, vp]
_lib.fw_cache8_attend.argtypes = [C.POINTER(FwCache8), C.POINTER(FwCache8Query), vp, vp, vp, vp, C.c_size_t, vp]
_lib.fw_cache8_attend_workspace.argtypes = [C.POINTER(FwCache8), C.POINTER(FwCache8Query)]
_lib.fw_cache8_attend_workspace.restype = C.c_size_t
_lib.fw_dense_and_topk_gap.argtypes = [C.POINTER(FwRows), vp, C.c_int32, C.POINTER(FwGapOut), vp, C.c_size_t, vp]
_lib.fw_dense_and_topk_gap_workspace.argtypes = [C.POINTER(FwRows), C.c_int32]
_lib.fw_dense_and_topk_gap_workspace.restype = C.c_size_t
_lib.fw_swap_refine.argtypes = [C.POINTER(FwRows), vp, C.c_int32, C.POINTER(FwGapOut), C.POINTER(FwSwapParams),
                                vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
_lib.fw_swap_refine_workspace.argtypes = [C.POINTER(FwRows), C.c_int32, C.POINTER(FwSwapParams)]
_lib.fw_swap_refine_workspace.restype = C.c_size_t
_lib.fw_best_subset.argtypes = [C.POINTER(FwRows), vp, vp, vp, vp, C.c_int32, vp, vp, vp, C.c_size_t, vp]
_lib.fw_best_subset_workspace.argtypes = [C.POINTER(FwRows)]
_lib.fw_best_subset_workspace.restype = C.c_size_t
_lib.fw_fp32_fma_probe.argtypes = [C.c_int32, C.c_int32, vp, vp]
_lib.fw_fp32_fma_probe.restype = C.c_int
_lib.fw_best_subset_read_stats.argtypes = [C.POINTER(FwRows), vp, C.POINTER(FwBestSubsetStats), vp]
_lib.fw_best_subset_read_stats.restype = C.c_int
_lib.fw_contour_alloc.argtypes = [vp, C.c_int32, C.c_int32, C.c_int32, C.c_int64, C.c_int32, vp, vp, vp, vp, vp,
                                  vp, vp, C.c_size_t, vp]
_lib.fw_contour_alloc_workspace.argtypes = [C.c_int32, C.c_int32]
_lib.fw_contour_alloc_workspace.restype = C.c_size_t
_lib.fw_contour_alloc_capped.argtypes = [vp, C.c_int32, C.c_int32, C.c_int32, C.c_int64, C.c_int32, C.c_int32, vp, vp,
                                         vp, vp, vp, vp, vp, C.c_size_t, vp]
_lib.fw_contour_alloc_capped.restype = C.c_int
_lib.fw_contour_alloc_capped_workspace.argtypes = [C.c_int32, C.c_int32]
_lib.fw_contour_alloc_capped_workspace.restype = C.c_size_t
_lib.fw_ragged_compact_to.argtypes = [vp, vp, C.c_int32, C.c_int32, C.c_int32, vp, vp, vp, vp, vp, vp, vp, vp]
_lib.fw_ragged_compact_to.restype = C.c_int
_lib.fw_ragged_append.argtypes = [vp, vp, vp, vp, vp, vp, vp, C.c_int32, C.c_int32, C.c_int32, vp, vp]
_lib.fw_ragged_append.restype = C.c_int
_lib.fw_window_score.argtypes = [vp, vp, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_float, C.c_int32, vp, vp,
                                 vp, C.c_size_t, vp]
_lib.fw_window_score.restype = C.c_int
_lib.fw_window_score_workspace.argtypes = [C.c_int32, C.c_int32]
_lib.fw_window_score_workspace.restype = C.c_size_t
_lib.fw_selector_audit.argtypes = [C.POINTER(FwRows), vp, C.c_int32, C.POINTER(FwGapOut), vp, vp, C.c_int32, vp,
                                   C.c_size_t, vp]
_lib.fw_selector_audit.restype = C.c_int
_lib.fw_selector_audit_workspace.argtypes = [C.POINTER(FwRows), C.c_int32]
_lib.fw_selector_audit_workspace.restype = C.c_size_t
_lib.fw_ragged_compact.argtypes = [vp, vp, C.c_int32, C.c_int32, C.c_int32, vp, vp, C.c_int64, vp, vp, vp]
_lib.fw_group_vote.argtypes = [C.POINTER(FwRows), vp, C.c_int32, C.POINTER(FwGapOut), vp, vp, vp, C.c_int32, vp,
                               vp, C.c_size_t, vp]
_lib.fw_group_vote_workspace.argtypes = [C.POINTER(FwRows), C.c_int32]
_lib.fw_group_vote_workspace.restype = C.c_size_t
_lib.fw_pool_best_subset.argtypes = [C.POINTER(FwRows), vp, C.c_int32, vp, C.POINTER(FwGapOut), vp, vp, C.c_int32,
                                     vp, vp, vp, vp, C.c_size_t, vp]
_lib.fw_pool_best_subset_workspace.argtypes = [C.POINTER(FwRows), C.c_int32]
_lib.fw_pool_best_subset_workspace.restype = C.c_size_t
_lib.fw_sync_status.argtypes = [vp, C.c_int64, C.POINTER(C.c_int64), vp]
_lib.fw_status_string.argtypes = [C.c_int]
_lib.fw_status_string.restype = C.c_char_p
_lib.fw_launch_count.restype = C.c_uint64
for _f in ("fw_dense_and_topk_gap", "fw_swap_refine", "fw_best_subset", "fw_contour_alloc", "fw_ragged_compact",
           "fw_group_vote", "fw_pool_best_subset", "fw_sync_status", "fw_prompt_attention", "fw_cache8_compact",
           "fw_cache8_append", "fw_cache8_attend"):
    getattr(_lib, _f).restype = C.c_int


class FwError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: {_lib.fw_status_string(status).decode()} ({status})")


def _check(st, where):
    if st != FW_OK:
        raise FwError(st, where)


def launch_count() -> int:
    return int(_lib.fw_launch_count())


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream(stream=None):
    s = stream if stream is not None else torch.cuda.current_stream()
    return C.c_void_p(s.cuda_stream)


def _ws(nbytes, device):
    # 256-byte aligned scratch for the library (torch's caching allocator aligns to 512)
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


class Rows:
    """Device-side row batch (fw_rows) built from tensors."""

    def __init__(self, *, rows_per_group, d, n_host, logits, logit_off, n, v, v_off, v_dtype):
        self.rows_per_group = int(rows_per_group)
        self.d = int(d)
        self.n_host = n_host
        self.num_groups = int(len(n_host))
        self.num_rows = self.num_groups * self.rows_per_group
        self.max_n = int(max(n_host)) if self.num_groups else 1
        self.logits, self.logit_off, self.n, self.v, self.v_off = logits, logit_off, n, v, v_off
        self.v_dtype = FW_BF16 if v_dtype == "bf16" else FW_F32
        self.device = logits.device
        self.c = FwRows(self.num_groups, self.rows_per_group, self.d, self.max_n, self.v_dtype,
                        _ptr(logits), _ptr(logit_off), _ptr(n), _ptr(v), _ptr(v_off))


def _to_dev(a, dtype, device):
    if isinstance(a, torch.Tensor):
        return a.to(device=device, dtype=dtype).contiguous()
    import numpy as np

    return torch.from_numpy(np.ascontiguousarray(a)).to(device=device, dtype=dtype).contiguous()


def rows_from_batch(batch, device="cuda") -> Rows:
    """Copy a workloads.RowBatch (numpy or torch) to the device."""
    import numpy as np

    if batch.v_dtype == "bf16":
        v = batch.v
        if isinstance(v, torch.Tensor):
            v = v.to(device).contiguous().view(torch.int16)
        else:
            v = torch.from_numpy(np.ascontiguousarray(v).view(np.int16)).to(device)
    else:
        v = _to_dev(batch.v, torch.float32, device)
    return Rows(rows_per_group=batch.rows_per_group, d=batch.d, n_host=np.asarray(batch.n_host),
                logits=_to_dev(batch.logits, torch.float32, device),
                logit_off=_to_dev(batch.logit_off, torch.int64, device),
                n=_to_dev(batch.n, torch.int32, device), v=v,
                v_off=_to_dev(batch.v_off, torch.int64, device), v_dtype=batch.v_dtype)


def dense_and_topk_gap(rows: Rows, k: torch.Tensor, *, o_kept=True, kept_bits=True, phi=True, stream=None):
    """fw_dense_and_topk_gap.  k: int32 [rows][nb] on the device.  Returns a dict
    of device tensors (the fw_gap_out fields)."""
    dev = rows.device
    R, d = rows.num_rows, rows.d
    nb = int(k.shape[1])
    words = (rows.max_n + 31) // 32
    f32 = dict(dtype=torch.float32, device=dev)
    out = dict(o=torch.empty(R, d, **f32), gap=torch.empty(R, nb, **f32), dropped=torch.empty(R, nb, **f32),
               row_max=torch.empty(R, **f32), row_sum=torch.empty(R, **f32),
               thr_key=torch.empty(R, nb, dtype=torch.int32, device=dev),
               thr_idx=torch.empty(R, nb, dtype=torch.int32, device=dev),
               row_status=torch.empty(R, dtype=torch.int32, device=dev))
    if o_kept:
        out["o_kept"] = torch.empty(R, nb, d, **f32)
    if phi:
        out["phi"] = torch.empty(R, nb, **f32)
    if kept_bits:
        out["kept_bits"] = torch.empty(R, nb, words, dtype=torch.int32, device=dev)
    c_out = gap_out_struct(out, words)
    nbytes = _lib.fw_dense_and_topk_gap_workspace(C.byref(rows.c), nb)
    ws = _ws(nbytes, dev)
    st = _lib.fw_dense_and_topk_gap(C.byref(rows.c), _ptr(k), nb, C.byref(c_out), _ptr(ws), ws.numel(),
                                    _stream(stream))
    _check(st, "fw_dense_and_topk_gap")
    out["_ws"] = ws
    out["_c"] = c_out
    return out


def gap_out_struct(out, words):
    return FwGapOut(_ptr(out.get("o")), _ptr(out.get("o_kept")), _ptr(out["gap"]), _ptr(out["dropped"]),
                    _ptr(out.get("phi")), _ptr(out.get("row_max")), _ptr(out.get("row_sum")),
                    _ptr(out.get("thr_key")), _ptr(out.get("thr_idx")), _ptr(out.get("kept_bits")),
                    int(words), _ptr(out.get("row_status")))


def swap_refine(rows: Rows, k: torch.Tensor, topk: dict, *, E: int, max_swaps: int = 64, stream=None):
    dev = rows.device
    R = rows.num_rows
    nb = int(k.shape[1])
    prm = FwSwapParams(int(E), int(max_swaps))
    out = dict(n_swaps=torch.empty(R, nb, dtype=torch.int32, device=dev),
               swap_out=torch.empty(R, nb, max_swaps, dtype=torch.int32, device=dev),
               swap_in=torch.empty(R, nb, max_swaps, dtype=torch.int32, device=dev),
               refined_gap=torch.empty(R, nb, dtype=torch.float32, device=dev),
               topk_gap=torch.empty(R, nb, dtype=torch.float32, device=dev),
               capped=torch.empty(R, nb, dtype=torch.int32, device=dev))
    nbytes = _lib.fw_swap_refine_workspace(C.byref(rows.c), nb, C.byref(prm))
    ws = _ws(nbytes, dev)
    st = _lib.fw_swap_refine(C.byref(rows.c), _ptr(k), nb, C.byref(topk["_c"]), C.byref(prm),
                             _ptr(out["n_swaps"]), _ptr(out["swap_out"]), _ptr(out["swap_in"]),
                             _ptr(out["refined_gap"]), _ptr(out["topk_gap"]), _ptr(out["capped"]), _ptr(ws),
                             ws.numel(), _stream(stream))
    _check(st, "fw_swap_refine")
    out["_ws"] = ws
    return out


def group_vote(rows: Rows, s: torch.Tensor, topk: dict, *, bits=True, stream=None):
    """fw_group_vote.  s: int32 [groups][nb] budgets on the device; topk: the
    dict dense_and_topk_gap returned for the same rows.  Returns gap, dropped,
    row_status ([rows][nb] / [rows]) and bits ([groups][nb][words])."""
    dev = rows.device
    R, nb = rows.num_rows, int(s.shape[1])
    words = (rows.max_n + 31) // 32
    out = dict(gap=torch.empty(R, nb, dtype=torch.float32, device=dev),
               dropped=torch.empty(R, nb, dtype=torch.float32, device=dev),
               row_status=torch.empty(R, dtype=torch.int32, device=dev))
    if bits:
        out["bits"] = torch.empty(rows.num_groups, nb, words, dtype=torch.int32, device=dev)
    nbytes = _lib.fw_group_vote_workspace(C.byref(rows.c), nb)
    ws = _ws(nbytes, dev)
    st = _lib.fw_group_vote(C.byref(rows.c), _ptr(s), nb, C.byref(topk["_c"]), _ptr(out["gap"]),
                            _ptr(out["dropped"]), _ptr(out.get("bits")), words, _ptr(out["row_status"]), _ptr(ws),
                            ws.numel(), _stream(stream))
    _check(st, "fw_group_vote")
    out["_ws"] = ws
    return out


def best_subset(rows: Rows, k: torch.Tensor, *, k_max=None, stream=None, ws=None):
    """fw_best_subset.  k: int32 [rows] (or [rows][1]) on the device."""
    dev = rows.device
    R = rows.num_rows
    k = k.reshape(-1)
    if k_max is None:  # one device read; pass k_max to avoid it
        k_max = int(k.max().item()) if k.numel() else 1
    k_max = int(k_max)
    out = dict(best_rank=torch.empty(R, dtype=torch.int64, device=dev),
               best_gap=torch.empty(R, dtype=torch.float32, device=dev),
               best_idx=torch.empty(R, k_max, dtype=torch.int32, device=dev),
               topk_gap=torch.empty(R, dtype=torch.float32, device=dev),
               row_status=torch.empty(R, dtype=torch.int32, device=dev))
    nbytes = _lib.fw_best_subset_workspace(C.byref(rows.c))
    if ws is None or ws.numel() < nbytes:
        ws = _ws(nbytes, dev)
    st = _lib.fw_best_subset(C.byref(rows.c), _ptr(k), _ptr(out["best_rank"]), _ptr(out["best_gap"]),
                             _ptr(out["best_idx"]), k_max, _ptr(out["topk_gap"]), _ptr(out["row_status"]),
                             _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "fw_best_subset")
    out["_ws"] = ws
    return out


def best_subset_stats(rows: Rows, out: dict, stream=None) -> dict:
    """fw_best_subset_read_stats for the call that returned `out` (waits for
    the stream): rows sent to the exhaustive path, re-scored candidates, and
    the walk's inner enumerations, leaves, fp32 operations and skipped nodes."""
    st = FwBestSubsetStats()
    _check(_lib.fw_best_subset_read_stats(C.byref(rows.c), _ptr(out["_ws"]), C.byref(st), _stream(stream)),
           "fw_best_subset_read_stats")
    return {name: int(getattr(st, name)) for name, _ in FwBestSubsetStats._fields_}


def pool_best_subset(rows: Rows, k: torch.Tensor, topk: dict, *, E, k_max: int = 32, stream=None):
    """fw_pool_best_subset (ES_pool, Definition 2.2).  k: int32 [rows][nb] on
    the device (the budgets of the gap call `topk`); E: extras per budget slot
    (host sequence of nb ints).  Returns best_gap, best_idx, topk_gap, n_cand,
    row_status."""
    dev, R, nb = rows.device, rows.num_rows, int(k.shape[1])
    E = [int(e) for e in E]
    if len(E) != nb:
        raise ValueError("E needs one entry per budget slot")
    Eh = (C.c_int32 * nb)(*E)
    out = dict(best_gap=torch.empty(R, nb, dtype=torch.float32, device=dev),
               best_idx=torch.empty(R, nb, int(k_max), dtype=torch.int32, device=dev),
               topk_gap=torch.empty(R, nb, dtype=torch.float32, device=dev),
               n_cand=torch.empty(R, nb, dtype=torch.int64, device=dev),
               row_status=torch.empty(R, dtype=torch.int32, device=dev))
    ws = _ws(_lib.fw_pool_best_subset_workspace(C.byref(rows.c), nb), dev)
    st = _lib.fw_pool_best_subset(C.byref(rows.c), _ptr(k), nb, Eh, C.byref(topk["_c"]), _ptr(out["best_gap"]),
                                  _ptr(out["best_idx"]), int(k_max), _ptr(out["topk_gap"]), _ptr(out["n_cand"]),
                                  _ptr(out["row_status"]), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "fw_pool_best_subset")
    out["_ws"] = ws
    return out


def sync_status(row_status: torch.Tensor, stream=None):
    """fw_sync_status: wait for the stream, then (status, first bad row) of a
    per-row status array (FW_OK, -1 when every row is fine)."""
    first = C.c_int64(-1)
    st = _lib.fw_sync_status(_ptr(row_status), int(row_status.numel()), C.byref(first), _stream(stream))
    return int(st), int(first.value)


def _contour_outputs(cells, total_budget, dev, out):
    if out is not None:  # caller-owned buffers of the same shapes, reused across calls
        return out
    return dict(counts=torch.empty(cells, dtype=torch.int32, device=dev),
                offsets=torch.empty(cells + 1, dtype=torch.int64, device=dev),
                kept_pos=torch.empty(int(total_budget), dtype=torch.int32, device=dev),
                tau=torch.empty(1, dtype=torch.float32, device=dev),
                dropped_uniform=torch.empty(cells, dtype=torch.float32, device=dev),
                dropped_alloc=torch.empty(cells, dtype=torch.float32, device=dev))


def _contour_ws(nbytes, dev, workspace):
    if workspace is None:
        return _ws(nbytes, dev)
    if workspace.numel() * workspace.element_size() < nbytes:
        raise ValueError(f"workspace holds {workspace.numel() * workspace.element_size()} bytes, {nbytes} needed")
    return workspace


def contour_alloc(scores: torch.Tensor, *, floor: int, total_budget: int, uniform_s: int, stream=None, out=None,
                  workspace=None):
    """fw_contour_alloc.  out (a dict as returned) and workspace (a uint8
    tensor of fw_contour_alloc_workspace bytes) may be passed to reuse
    buffers across calls."""
    dev = scores.device
    cells, T = scores.shape
    out = _contour_outputs(cells, total_budget, dev, out)
    ws = _contour_ws(_lib.fw_contour_alloc_workspace(cells, T), dev, workspace)
    st = _lib.fw_contour_alloc(_ptr(scores), cells, T, int(floor), int(total_budget), int(uniform_s),
                               _ptr(out["counts"]), _ptr(out["offsets"]), _ptr(out["kept_pos"]), _ptr(out["tau"]),
                               _ptr(out["dropped_uniform"]), _ptr(out["dropped_alloc"]), _ptr(ws), ws.numel(),
                               _stream(stream))
    _check(st, "fw_contour_alloc")
    out["_ws"] = ws
    return out


def contour_alloc_capped(scores: torch.Tensor, *, floor: int, total_budget: int, uniform_s: int, cap: int,
                         stream=None, out=None, workspace=None):
    """fw_contour_alloc_capped: the allocation truncated to `cap` entries per
    cell.  kept_pos holds total_budget entries; offsets[-1] of them are valid.
    out and workspace as for contour_alloc (the capped workspace size)."""
    dev = scores.device
    cells, T = scores.shape
    out = _contour_outputs(cells, total_budget, dev, out)
    ws = _contour_ws(_lib.fw_contour_alloc_capped_workspace(cells, T), dev, workspace)
    st = _lib.fw_contour_alloc_capped(_ptr(scores), cells, T, int(floor), int(total_budget), int(uniform_s), int(cap),
                                      _ptr(out["counts"]), _ptr(out["offsets"]), _ptr(out["kept_pos"]),
                                      _ptr(out["tau"]), _ptr(out["dropped_uniform"]), _ptr(out["dropped_alloc"]),
                                      _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "fw_contour_alloc_capped")
    out["_ws"] = ws
    return out


def ragged_compact(K: torch.Tensor, V: torch.Tensor, offsets: torch.Tensor, kept_pos: torch.Tensor, total: int,
                   *, out=None, stream=None):
    cells, T, d = K.shape
    row_bytes = d * K.element_size()
    if out is None:
        Ko = torch.empty(int(total), d, dtype=K.dtype, device=K.device)
        Vo = torch.empty(int(total), d, dtype=V.dtype, device=V.device)
    else:
        Ko, Vo = out
    st = _lib.fw_ragged_compact(_ptr(K), _ptr(V), cells, T, row_bytes, _ptr(offsets), _ptr(kept_pos), int(total),
                                _ptr(Ko), _ptr(Vo), _stream(stream))
    _check(st, "fw_ragged_compact")
    return Ko, Vo


def ragged_compact_to(K: torch.Tensor, V: torch.Tensor, offsets: torch.Tensor, kept_pos: torch.Tensor,
                      base: torch.Tensor, capacity: torch.Tensor, K_store: torch.Tensor, V_store: torch.Tensor,
                      status: torch.Tensor = None, stream=None):
    """fw_ragged_compact_to: kept rows into a store with room per cell."""
    cells, T, d = K.shape
    st = _lib.fw_ragged_compact_to(_ptr(K), _ptr(V), cells, T, d * K.element_size(), _ptr(offsets), _ptr(kept_pos),
                                   _ptr(base), _ptr(capacity), _ptr(K_store), _ptr(V_store), _ptr(status),
                                   _stream(stream))
    _check(st, "fw_ragged_compact_to")


def ragged_append(K_store: torch.Tensor, V_store: torch.Tensor, base: torch.Tensor, capacity: torch.Tensor,
                  counts: torch.Tensor, new_K: torch.Tensor, new_V: torch.Tensor, status: torch.Tensor = None,
                  stream=None):
    """fw_ragged_append: new_K / new_V [cells][m][d] behind each cell's rows."""
    cells, m, d = new_K.shape
    st = _lib.fw_ragged_append(_ptr(K_store), _ptr(V_store), _ptr(base), _ptr(capacity), _ptr(counts), _ptr(new_K),
                               _ptr(new_V), cells, m, d * new_K.element_size(), _ptr(status), _stream(stream))
    _check(st, "fw_ragged_append")


def window_score(Qw: torch.Tensor, K: torch.Tensor, *, scale: float = None, pool: int = 7, out=None, stream=None):
    """fw_window_score.  Qw: bf16 (or int16 bits) [cells][w][d]; K: [cells][T][d].
    Returns (scores [cells][T] fp32, status [cells])."""
    cells, w, d = Qw.shape
    T = K.shape[1]
    scale = 1.0 / math.sqrt(d) if scale is None else float(scale)
    scores = out if out is not None else torch.empty(cells, T, dtype=torch.float32, device=K.device)
    status = torch.empty(cells, dtype=torch.int32, device=K.device)
    ws = _ws(_lib.fw_window_score_workspace(cells, T), K.device)
    st = _lib.fw_window_score(_ptr(Qw), _ptr(K), cells, T, d, w, C.c_float(scale), int(pool), _ptr(scores),
                              _ptr(status), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "fw_window_score")
    return scores, status


SELECTORS = ("streamingllm", "h2o", "snapkv", "quest", "quest16")


def selector_audit(rows: Rows, s, topk: dict, *, bits=False, stream=None):
    """fw_selector_audit: es of every deployed rule's kept set ([rows][5][nb],
    rules in SELECTORS order) at the host budgets s; optionally the sets."""
    dev, R = rows.device, rows.num_rows
    s = [int(x) for x in s]
    nb = len(s)
    words = (rows.max_n + 31) // 32
    out = dict(es=torch.empty(R, len(SELECTORS), nb, dtype=torch.float32, device=dev))
    if bits:
        out["bits"] = torch.empty(R, len(SELECTORS), nb, words, dtype=torch.int32, device=dev)
    sh = (C.c_int32 * nb)(*s)
    ws = _ws(_lib.fw_selector_audit_workspace(C.byref(rows.c), nb), dev)
    st = _lib.fw_selector_audit(C.byref(rows.c), sh, nb, C.byref(topk["_c"]), _ptr(out["es"]), _ptr(out.get("bits")),
                                words, _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "fw_selector_audit")
    out["_ws"] = ws
    return out


def _need(ok, what):
    if not ok:
        raise ValueError(what)


# the raw handle of a device's current stream, without the Stream object that torch.cuda.current_stream makes (2 us)
_current_raw = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _on_current(dev):
    # the library launches on the current GPU, and a default stream's handle is 0 on every GPU
    if dev != _current_device():
        raise ValueError(f"the tensors are on GPU {dev}, which is not the current one")


def _raw_stream(stream, dev):
    """The handle of the stream that a call on GPU `dev` runs on."""
    if stream is None and dev == _current_device():
        return _current_raw(dev)
    _on_current(dev)
    if stream.device.index != dev:
        raise ValueError("the stream is one of the tensors' GPU")
    return stream.cuda_stream


def _one_device(*tensors):
    dev = tensors[0].get_device()
    for t in tensors:
        if t.get_device() != dev or dev < 0:
            raise ValueError("the tensors of a call are on one GPU")


def _made_on(stream):
    # buffers for a call on another stream come from that stream's memory: what the current stream has
    # freed, work still under way there may be using
    return torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext()


def _attention_out(out, q, items, stream):
    """(o, lse, status, the dict) of a call's outputs: those of `out`, checked, or new ones."""
    if out is None:
        with _made_on(stream):
            out = dict(o=torch.empty(q.shape, dtype=torch.bfloat16, device=q.device),
                       lse=torch.empty(q.shape[:-1], dtype=torch.float32, device=q.device),
                       status=torch.empty(items, dtype=torch.int32, device=q.device))
        if stream is not None:  # the caller reads them on the current one
            for t in out.values():
                t.record_stream(torch.cuda.current_stream(q.device))
        return out["o"].data_ptr(), out["lse"].data_ptr(), out["status"].data_ptr(), out
    o, lse, status = out["o"], out.get("lse"), out.get("status")
    if o.shape != q.shape or o.dtype is not torch.bfloat16 or not o.is_contiguous():
        raise ValueError("out['o'] is contiguous bfloat16 of q's shape")
    if lse is not None and (lse.shape != q.shape[:-1] or lse.dtype is not torch.float32 or not lse.is_contiguous()):
        raise ValueError("out['lse'] is contiguous float32 of q's shape without its last axis")
    if status is not None and (status.numel() < items or status.dtype is not torch.int32 or not status.is_contiguous()):
        raise ValueError(f"out['status'] is contiguous int32, {items} entries")
    dev = q.get_device()
    if o.get_device() != dev or (lse is not None and lse.get_device() != dev) or (
            status is not None and status.get_device() != dev):
        raise ValueError("out's tensors are on q's GPU")
    return o.data_ptr(), lse.data_ptr() if lse is not None else None, status.data_ptr() if status is not None else None, out


def prompt_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_q: torch.Tensor, cu_k: torch.Tensor = None, *,
                     scale: float = None, out=None, stream=None):
    """fw_prompt_attention.  q: bf16 [rows][q_heads][d], k and v: bf16 [rows][kv_heads][d], any strides that are
    multiples of 8 with d contiguous; cu_q, cu_k: int32 [sequences + 1] row bounds (cu_k = cu_q if not given).
    Returns a dict of o (bf16, as q), lse (fp32 [rows][q_heads]) and status [sequences]; such a dict passed as out
    is written instead."""
    if cu_k is None:
        cu_k = cu_q
    rows, hq, d = q.shape
    keys, hk, dk = k.shape
    bf16, i32 = torch.bfloat16, torch.int32
    if q.dtype is not bf16 or k.dtype is not bf16 or v.dtype is not bf16:
        raise ValueError("q, k and v are bfloat16")
    if v.shape != k.shape or dk != d:
        raise ValueError("k and v are [rows][kv_heads][d], d as in q")
    (qr, qh, q1), (kr, kh, k1), (vr, vh, v1) = q.stride(), k.stride(), v.stride()
    if not q1 == k1 == v1 == 1:
        raise ValueError("d is the contiguous axis of q, k and v")
    if cu_q.dtype is not i32 or cu_k.dtype is not i32 or cu_q.dim() != 1 or cu_q.shape != cu_k.shape or not (
            cu_q.is_contiguous() and cu_k.is_contiguous()):
        raise ValueError("cu_q and cu_k are contiguous int32 [sequences + 1]")
    dev = q.get_device()
    if dev < 0 or k.get_device() != dev or v.get_device() != dev or cu_q.get_device() != dev or cu_k.get_device() != dev:
        raise ValueError("the tensors of a call are on one GPU")
    handle = _raw_stream(stream, dev)
    # (strides of axes of one entry, which torch leaves open)
    if hq == 1:
        qh = d
    if hk == 1:
        kh = vh = d
    if rows <= 1:
        qr = hq * qh
    if keys <= 1:
        kr, vr = hk * kh, hk * vh
    seqs = cu_q.shape[0] - 1
    o, lse, status, out = _attention_out(out, q, seqs, stream)
    p = FwPrompt(seqs, hq, hk, d, rows, keys, q.data_ptr(), k.data_ptr(), v.data_ptr(), qr, qh, kr, kh, vr, vh,
                 cu_q.data_ptr(), cu_k.data_ptr(), 1.0 / math.sqrt(d) if scale is None else scale)
    st = _lib.fw_prompt_attention(C.byref(p), o, lse, status, handle)
    if st != FW_OK:
        raise FwError(st, "fw_prompt_attention")
    return out


CACHE8_BLOCK, CACHE8_TAIL = 32, 64
_CACHE8_FORMATS = {"e4m3": (0, torch.float8_e4m3fn), "int8": (1, torch.int8)}


class Cache8:
    """A ragged per-head store in 8 bits (fw_cache8) over the caller's tensors: codes k, v [rows][d] (float8_e4m3fn
    for fmt "e4m3", int8 for "int8"), their scales fp32 [rows / 32], the open blocks' bf16 rows k_tail, v_tail
    [cells][64][d], and base (int64), capacity and counts (int32), [cells] each."""

    def __init__(self, *, fmt, k, v, k_scale, v_scale, k_tail, v_tail, base, capacity, counts):
        _need(fmt in _CACHE8_FORMATS, f"fmt is one of {sorted(_CACHE8_FORMATS)}")
        code, dtype = _CACHE8_FORMATS[fmt]
        rows, d = k.shape
        cells = base.numel()
        _need(k.dtype == v.dtype == dtype and k.shape == v.shape, f"k and v are {dtype} [rows][d]")
        _need(rows % CACHE8_BLOCK == 0 and k_scale.numel() == v_scale.numel() == rows // CACHE8_BLOCK and
              k_scale.dtype == v_scale.dtype == torch.float32, "k_scale and v_scale are float32 [rows / 32]")
        _need(k_tail.dtype == v_tail.dtype == torch.bfloat16 and
              tuple(k_tail.shape) == tuple(v_tail.shape) == (cells, CACHE8_TAIL, d), "tails are bfloat16 [cells][64][d]")
        _need(base.dtype == torch.int64 and capacity.dtype == counts.dtype == torch.int32 and
              capacity.numel() == counts.numel() == cells, "base is int64, capacity and counts are int32, [cells] each")
        _need(d in (64, 128) and cells >= 1, "d is 64 or 128, and there is a cell")
        self.tensors = (k, v, k_scale, v_scale, k_tail, v_tail, base, capacity, counts)
        _need(all(t.is_contiguous() for t in self.tensors), "the store's tensors are contiguous")
        _one_device(*self.tensors)
        self.k, self.v, self.k_scale, self.v_scale, self.k_tail, self.v_tail, self.base, self.capacity, self.counts = \
            self.tensors
        self.fmt, self.d, self.cells, self.device, self.index = fmt, d, cells, k.device, k.get_device()
        self.c = FwCache8(cells, d, code, rows, *(t.data_ptr() for t in self.tensors))
        self._ref = C.byref(self.c)

    def part(self, first: int, cells: int) -> "Cache8":
        """The cells first .. first + cells (a layer's, say) as a store of their own over the same memory."""
        _need(0 <= first and cells >= 1 and first + cells <= self.cells, "cells within the store's")
        cut = slice(first, first + cells)
        return Cache8(fmt=self.fmt, k=self.k, v=self.v, k_scale=self.k_scale, v_scale=self.v_scale,
                      k_tail=self.k_tail[cut], v_tail=self.v_tail[cut], base=self.base[cut],
                      capacity=self.capacity[cut], counts=self.counts[cut])


def cache8_empty(offsets: torch.Tensor, total: int, d: int, *, fmt: str = "e4m3", room: int = 0) -> Cache8:
    """A store for cells of offsets[h + 1] - offsets[h] rows (offsets int64 [cells + 1] on the device, at most `total`
    rows in all) and `room` more each.  Sized on the host from total alone: cell h starts at the multiple of 32 at or
    behind offsets[h] + h (room + 31), which leaves it its rows without a prefix sum or a synchronisation."""
    _need(fmt in _CACHE8_FORMATS, f"fmt is one of {sorted(_CACHE8_FORMATS)}")
    cells, dev = offsets.numel() - 1, offsets.device
    rows = (int(total) + cells * (room + 31) + 31) // 32 * 32
    h = torch.arange(cells + 1, device=dev)
    edge = (offsets + h * (room + 31) + 31) // 32 * 32
    f = dict(dtype=_CACHE8_FORMATS[fmt][1], device=dev)
    tail = dict(dtype=torch.bfloat16, device=dev)
    return Cache8(fmt=fmt, k=torch.empty(rows, d, **f), v=torch.empty(rows, d, **f),
                  k_scale=torch.empty(rows // 32, dtype=torch.float32, device=dev),
                  v_scale=torch.empty(rows // 32, dtype=torch.float32, device=dev),
                  k_tail=torch.empty(cells, CACHE8_TAIL, d, **tail), v_tail=torch.empty(cells, CACHE8_TAIL, d, **tail),
                  base=edge[:-1].contiguous(), capacity=(edge[1:] - edge[:-1]).to(torch.int32),
                  counts=torch.zeros(cells, dtype=torch.int32, device=dev))


def _status_ptr(status, cache):
    if status is None:
        return None
    if status.dtype is not torch.int32 or status.numel() < cache.cells or not status.is_contiguous() or (
            status.get_device() != cache.index):
        raise ValueError("status is contiguous int32 [cells] on the store's GPU")
    return status.data_ptr()


def cache8_compact(cache: Cache8, K: torch.Tensor, V: torch.Tensor, offsets: torch.Tensor, kept_pos: torch.Tensor, *,
                   status: torch.Tensor = None, stream=None):
    """fw_cache8_compact: the kept rows of K, V (bf16 [cells][T][d], equal strides that are multiples of 8, d
    contiguous) quantised into the store, whose counts are set."""
    cells, T, d = K.shape
    if K.dtype is not torch.bfloat16 or V.dtype is not torch.bfloat16 or V.shape != K.shape or cells != cache.cells or \
            d != cache.d:
        raise ValueError("K and V are bfloat16 [cells][T][d], as the store's")
    (cs, rs, one), (vcs, vrs, vone) = K.stride(), V.stride()
    if cells == 1:
        cs = vcs = T * d
    if T == 1:
        rs = vrs = d
    if one != 1 or vone != 1 or cs != vcs or rs != vrs:
        raise ValueError("K and V have equal strides and d contiguous")
    if offsets.dtype is not torch.int64 or offsets.numel() != cells + 1 or kept_pos.dtype is not torch.int32 or not (
            offsets.is_contiguous() and kept_pos.is_contiguous()):
        raise ValueError("offsets is contiguous int64 [cells + 1], kept_pos contiguous int32")
    if not K.get_device() == V.get_device() == offsets.get_device() == kept_pos.get_device() == cache.index:
        raise ValueError("the tensors of a call are on the store's GPU")
    st = _lib.fw_cache8_compact(cache._ref, K.data_ptr(), V.data_ptr(), T, cs, rs, offsets.data_ptr(),
                                kept_pos.data_ptr(), kept_pos.numel(), _status_ptr(status, cache),
                                _raw_stream(stream, cache.index))
    if st != FW_OK:
        raise FwError(st, "fw_cache8_compact")


def cache8_append(cache: Cache8, new_K: torch.Tensor, new_V: torch.Tensor, *, status: torch.Tensor = None, stream=None):
    """fw_cache8_append: new_K, new_V (bf16 [cells][m][d], contiguous) behind each cell's rows."""
    cells, m, d = new_K.shape
    if new_K.dtype is not torch.bfloat16 or new_V.dtype is not torch.bfloat16 or new_V.shape != new_K.shape or not (
            new_K.is_contiguous() and new_V.is_contiguous()) or cells != cache.cells or d != cache.d:
        raise ValueError("new_K and new_V are contiguous bfloat16 [cells][m][d], as the store's")
    if not new_K.get_device() == new_V.get_device() == cache.index:
        raise ValueError("the tensors of a call are on the store's GPU")
    st = _lib.fw_cache8_append(cache._ref, new_K.data_ptr(), new_V.data_ptr(), m, _status_ptr(status, cache),
                               _raw_stream(stream, cache.index))
    if st != FW_OK:
        raise FwError(st, "fw_cache8_append")


def _cache8_query(cache, q, kv_heads, scale):
    seqs, m, hq, d = q.shape
    s0, s1, s2, one = q.stride()
    if q.dtype is not torch.bfloat16 or one != 1 or d != cache.d:
        raise ValueError("q is bfloat16 [sequences][m][heads][d], d contiguous and the store's")
    if kv_heads < 1 or hq % kv_heads or seqs * kv_heads != cache.cells:
        raise ValueError("sequences x kv_heads is the store's cells, heads a multiple of kv_heads")
    # (strides of axes of one entry, which torch leaves open)
    return FwCache8Query(kv_heads, hq // kv_heads, m, q.data_ptr(), s0 if seqs > 1 else d, s1 if m > 1 else d,
                         s2 if hq > 1 else d, 1.0 / math.sqrt(d) if scale is None else scale)


def cache8_attend_workspace(cache: Cache8, q: torch.Tensor, *, kv_heads: int) -> torch.Tensor:
    """A workspace for cache8_attend calls with queries of q's shape (fw_cache8_attend_workspace)."""
    c_q = _cache8_query(cache, q, kv_heads, None)
    _on_current(cache.index)
    return _ws(_lib.fw_cache8_attend_workspace(cache._ref, C.byref(c_q)), cache.device)


def cache8_attend(cache: Cache8, q: torch.Tensor, *, kv_heads: int, scale: float = None, out=None, workspace=None,
                  stream=None):
    """fw_cache8_attend.  q: bf16 [sequences][m][q_heads][d] (strides multiples of 8, d contiguous), the queries of
    each sequence's last m tokens; the store's cells are [sequences][kv_heads].  Returns a dict of o (bf16, as q), lse
    (fp32 [sequences][m][q_heads]) and status [cells]; such a dict passed as out is written instead.  A workspace
    (cache8_attend_workspace) serves one call at a time."""
    c_q = _cache8_query(cache, q, kv_heads, scale)
    if q.get_device() != cache.index:
        raise ValueError("q is on the store's GPU")
    handle = _raw_stream(stream, cache.index)
    o, lse, status, out = _attention_out(out, q, cache.cells, stream)
    if workspace is None:
        with _made_on(stream):
            workspace = _ws(_lib.fw_cache8_attend_workspace(cache._ref, C.byref(c_q)), cache.device)
    elif workspace.get_device() != cache.index or not workspace.is_contiguous():
        raise ValueError("workspace is contiguous on the store's GPU")
    st = _lib.fw_cache8_attend(cache._ref, C.byref(c_q), o, lse, status, workspace.data_ptr(), workspace.numel(), handle)
    if st != FW_OK:
        raise FwError(st, "fw_cache8_attend")
    return out


def raw():
    """The loaded ctypes library (for callers that marshal their own arguments)."""
    return _lib


def fp32_fma_probe(blocks: int, iters: int, out: torch.Tensor, stream=None):
    """fw_fp32_fma_probe (a measurement aid): blocks x 256 threads x 16 chains x
    iters fp32 FMAs; out: float32 [blocks * 256] on the device."""
    _check(_lib.fw_fp32_fma_probe(int(blocks), int(iters), _ptr(out), _stream(stream)), "fw_fp32_fma_probe")

"""Thin ctypes binding of libsparsebal (include/sparsebal.h): argument marshalling only.

Every step of the hot path runs inside the library's HIP kernels; torch is used here for device
memory and the current stream.  There is no CPU fallback: if the shared library is missing the
import of `lib()` raises.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libsparsebal.so")

SB_OK = 0
SB_BF16, SB_F32 = 0, 1
SB_SELECT_PER_QHEAD, SB_SELECT_PER_KVGROUP = 0, 1
SB_CU_SLOTS = 512

EXPORTS = ["sb_get_layout", "sb_keep_ratio_to_topk", "sb_sel_rowptr_host", "sb_block_scores", "sb_select_topk", "sb_select_topk_static", "sb_score_select",
           "sb_plan_worklist", "sb_plan_sections", "sb_sparse_attn_fwd", "sb_sparse_attn_bwd", "sb_score_coverage", "sb_perf_predict", "sb_perf_align", "sb_dst_tune",
           "sb_rope_init", "sb_rope_apply", "sb_window_ws_bytes", "sb_window_attn_fwd", "sb_window_attn_bwd", "sb_cache_append",
           "sb_cache_attn_ws_bytes", "sb_cache_attn", "sb_spar_update", "sb_spar_predict", "sb_balanced_partition", "sb_sab_batches",
           "sb_set_instrumentation", "sb_read_cu_busy", "sb_read_kernel_times",
           "sb_last_error", "sb_version"]


class sb_problem(C.Structure):
    _fields_ = [("total_tokens", C.c_int32), ("num_seqs", C.c_int32), ("num_q_heads", C.c_int32),
                ("num_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("block_size", C.c_int32), ("dtype", C.c_int32),
                ("select_mode", C.c_int32), ("softmax_scale", C.c_float), ("score_scale", C.c_float),
                ("cu_seqlens_host", C.c_void_p), ("cu_seqlens_dev", C.c_void_p), ("topk_host", C.c_void_p),
                ("topk_dev", C.c_void_p)]


class sb_layout(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("num_qblocks", "sel_heads", "scores_elems", "pooled_elems", "sel_rows", "sel_nnz",
                                         "plan_bytes", "scores_ws_bytes", "select_ws_bytes", "fwd_ws_bytes", "bwd_ws_bytes",
                                         "attended_pairs_per_head_sum", "coverage_ws_bytes")]


class sb_perf_table(C.Structure):
    _fields_ = [("num_lengths", C.c_int32), ("num_budgets", C.c_int32), ("lengths", C.c_void_p), ("budgets", C.c_void_p),
                ("latency", C.c_void_p)]


SB_ROPE_MAX_PAIRS = 64


class sb_rope(C.Structure):
    _fields_ = [("rot_dim", C.c_int32), ("layout", C.c_int32), ("amplitude", C.c_float), ("reserved", C.c_int32),
                ("turns", C.c_double * SB_ROPE_MAX_PAIRS)]


class sb_cache(C.Structure):
    _fields_ = [("num_pages", C.c_int32), ("page_size", C.c_int32), ("num_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32),
                ("max_pages", C.c_int32), ("k", C.c_void_p), ("v", C.c_void_p), ("page_table", C.c_void_p)]


class sb_chunk(C.Structure):
    _fields_ = [("num_seqs", C.c_int32), ("num_q_heads", C.c_int32), ("total_new", C.c_int32), ("max_new", C.c_int32), ("max_length", C.c_int32),
                ("softmax_scale", C.c_float), ("cu_new", C.c_void_p), ("cached", C.c_void_p)]


_lib = None


class SparseBalError(RuntimeError):
    pass


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise SparseBalError(f"{LIB_PATH} is not built; run `python -c 'import __graft_entry__ as g; g.build()'`")
        loaded = C.CDLL(LIB_PATH)
        loaded.sb_last_error.restype = C.c_char_p
        loaded.sb_version.restype = C.c_char_p
        _lib = loaded  # (complete: another thread may be here too)
    return _lib


def _check(rc):
    if rc != SB_OK:
        raise SparseBalError(f"libsparsebal error {rc}: {lib().sb_last_error().decode()}")


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, torch.Tensor):
        assert t.is_contiguous()
        return C.c_void_p(t.data_ptr())
    return t.ctypes.data_as(C.c_void_p)


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


class Problem:
    """Holds sb_problem plus the host/device arrays it points to."""

    def __init__(self, cu_seqlens, topk, Hq, Hkv, D, B=64, dtype=SB_BF16, select_mode=SB_SELECT_PER_QHEAD,
                 softmax_scale=0.0, score_scale=0.0, device=None):
        self.cu_host = np.ascontiguousarray(cu_seqlens, dtype=np.int32)
        self.topk_host = np.ascontiguousarray(topk, dtype=np.int32)
        self.S, self.T = len(self.cu_host) - 1, int(self.cu_host[-1]) if len(self.cu_host) else 0
        self.device = device
        if device is not None:
            self.cu_dev = torch.from_numpy(self.cu_host).to(device)
            self.topk_dev = torch.from_numpy(self.topk_host).to(device) if self.S else torch.zeros(1, dtype=torch.int32, device=device)
        else:
            self.cu_dev = self.topk_dev = None
        self.c = sb_problem(self.T, self.S, Hq, Hkv, D, B, dtype, select_mode, softmax_scale, score_scale,
                            self.cu_host.ctypes.data, self.cu_dev.data_ptr() if device is not None else None,
                            self.topk_host.ctypes.data if self.S else None,
                            self.topk_dev.data_ptr() if device is not None else None)
        self.Hq, self.Hkv, self.D, self.B, self.dtype, self.select_mode = Hq, Hkv, D, B, dtype, select_mode
        self.layout = sb_get_layout(self)

    def ref(self):
        return C.byref(self.c)


def sb_get_layout(pb: Problem) -> sb_layout:
    out = sb_layout()
    _check(lib().sb_get_layout(pb.ref(), C.byref(out)))
    return out


def sb_keep_ratio_to_topk(cu_seqlens, block_size, keep_ratio) -> np.ndarray:
    cu = np.ascontiguousarray(cu_seqlens, dtype=np.int32)
    rho = np.ascontiguousarray(keep_ratio, dtype=np.float32)
    out = np.zeros(len(rho), dtype=np.int32)
    _check(lib().sb_keep_ratio_to_topk(_ptr(cu), len(rho), block_size, _ptr(rho), _ptr(out)))
    return out


def sb_sel_rowptr_host(pb: Problem) -> np.ndarray:
    out = np.zeros(pb.layout.sel_rows + 1, dtype=np.int32)
    _check(lib().sb_sel_rowptr_host(pb.ref(), _ptr(out)))
    return out


def _bytes(n, device):
    return torch.empty(max(int(n), 256), dtype=torch.uint8, device=device)


def sb_block_scores(pb: Problem, q, k, want_kbar=False, ws=None):
    lay = pb.layout
    scores = torch.empty(max(lay.scores_elems, 1), dtype=torch.float32, device=q.device)
    kbar = torch.empty(max(lay.pooled_elems, 1), dtype=torch.float32, device=q.device) if want_kbar else None
    ws = ws if ws is not None else _bytes(lay.scores_ws_bytes, q.device)
    _check(lib().sb_block_scores(pb.ref(), _ptr(q), _ptr(k), _ptr(kbar), _ptr(scores), _ptr(ws), _stream()))
    return (scores, kbar) if want_kbar else scores


def sb_select_topk(pb: Problem, scores, ws=None):
    lay = pb.layout
    rowptr = torch.empty(lay.sel_rows + 1, dtype=torch.int32, device=scores.device)
    idx = torch.empty(max(lay.sel_nnz, 1), dtype=torch.int32, device=scores.device)
    ws = ws if ws is not None else _bytes(lay.select_ws_bytes, scores.device)
    _check(lib().sb_select_topk(pb.ref(), _ptr(scores), _ptr(rowptr), _ptr(idx), _ptr(ws), _stream()))
    return rowptr, idx


def sb_select_topk_static(pb: Problem, scores, rowptr=None, idx=None):
    """sb_select_topk without a workspace argument (the library's built-in scratch); outputs may be passed in."""
    lay = pb.layout
    rowptr = rowptr if rowptr is not None else torch.empty(lay.sel_rows + 1, dtype=torch.int32, device=scores.device)
    idx = idx if idx is not None else torch.empty(max(lay.sel_nnz, 1), dtype=torch.int32, device=scores.device)
    _check(lib().sb_select_topk_static(pb.ref(), _ptr(scores), _ptr(rowptr), _ptr(idx), _stream()))
    return rowptr, idx


def sb_score_select(pb: Problem, q, k, ws=None, want_scores=True):
    """Scores and selection in one call; returns (scores, sel_rowptr, sel_idx); scores is None with want_scores=False
    (the single-kernel form that keeps the scores on chip)."""
    lay = pb.layout
    scores = torch.empty(max(lay.scores_elems, 1), dtype=torch.float32, device=q.device) if want_scores else None
    rowptr = torch.empty(lay.sel_rows + 1, dtype=torch.int32, device=q.device)
    idx = torch.empty(max(lay.sel_nnz, 1), dtype=torch.int32, device=q.device)
    ws = ws if ws is not None else _bytes(lay.scores_ws_bytes, q.device)
    _check(lib().sb_score_select(pb.ref(), _ptr(q), _ptr(k), None, _ptr(scores), _ptr(rowptr), _ptr(idx), _ptr(ws), _stream()))
    return scores, rowptr, idx


def sb_plan_worklist(pb: Problem, sel_rowptr, sel_idx, plan=None):
    plan = plan if plan is not None else _bytes(pb.layout.plan_bytes, sel_rowptr.device)
    _check(lib().sb_plan_worklist(pb.ref(), _ptr(sel_rowptr), _ptr(sel_idx), _ptr(plan), _stream()))
    return plan


def sb_sparse_attn_fwd(pb: Problem, q, k, v, sel_rowptr, sel_idx, plan, o=None, lse=None, ws=None):
    o = o if o is not None else torch.empty_like(q)
    lse = lse if lse is not None else torch.empty((pb.Hq, pb.T), dtype=torch.float32, device=q.device)
    ws = ws if ws is not None else _bytes(pb.layout.fwd_ws_bytes, q.device)
    _check(lib().sb_sparse_attn_fwd(pb.ref(), _ptr(q), _ptr(k), _ptr(v), _ptr(sel_rowptr), _ptr(sel_idx), _ptr(plan),
                                    _ptr(o), _ptr(lse), _ptr(ws), _stream()))
    return o, lse


def sb_sparse_attn_bwd(pb: Problem, q, k, v, o, lse, d_o, sel_rowptr, sel_idx, plan, dq=None, dk=None, dv=None, ws=None):
    dq = dq if dq is not None else torch.empty_like(q)
    dk = dk if dk is not None else torch.empty_like(k)
    dv = dv if dv is not None else torch.empty_like(v)
    ws = ws if ws is not None else _bytes(pb.layout.bwd_ws_bytes, q.device)
    _check(lib().sb_sparse_attn_bwd(pb.ref(), _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(d_o), _ptr(sel_rowptr),
                                    _ptr(sel_idx), _ptr(plan), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(ws), _stream()))
    return dq, dk, dv


SB_ANCHOR_MIN, SB_ANCHOR_MEAN, SB_ANCHOR_MAX = 0, 1, 2


def sb_score_coverage(pb: Problem, scores, ws=None):
    """Coverage curves C_s(k) of the routing scores: NQB floats on the device."""
    cov = torch.empty(max(pb.layout.num_qblocks, 1), dtype=torch.float32, device=scores.device)
    ws = ws if ws is not None else _bytes(pb.layout.coverage_ws_bytes, scores.device)
    _check(lib().sb_score_coverage(pb.ref(), _ptr(scores), _ptr(cov), _ptr(ws), _stream()))
    return cov


class PerfTable:
    """Holds sb_perf_table plus the host arrays it points to."""

    def __init__(self, lengths, budgets, latency):
        self.lengths = np.ascontiguousarray(lengths, dtype=np.float32)
        self.budgets = np.ascontiguousarray(budgets, dtype=np.float32)
        self.latency = np.ascontiguousarray(latency, dtype=np.float32).reshape(len(self.lengths), len(self.budgets))
        self.c = sb_perf_table(len(self.lengths), len(self.budgets), self.lengths.ctypes.data, self.budgets.ctypes.data,
                               self.latency.ctypes.data)

    def ref(self):
        return C.byref(self.c)

    @classmethod
    def from_json(cls, path):
        """A table written by paper_2604_13847_amd/profile_latency.py."""
        import json
        with open(path) as f:
            j = json.load(f)
        return cls(j["lengths"], j["budgets"], j["latency_ms"])


def sb_perf_predict(tab: PerfTable, length, budget) -> float:
    out = C.c_double()
    _check(lib().sb_perf_predict(tab.ref(), C.c_double(length), C.c_double(budget), C.byref(out)))
    return out.value


def sb_perf_align(tab: PerfTable, length, target, max_budget) -> int:
    out = C.c_int32()
    _check(lib().sb_perf_align(tab.ref(), C.c_double(length), C.c_double(target), int(max_budget), C.byref(out)))
    return out.value


def sb_dst_tune(pb: Problem, coverage_host, tab: PerfTable, anchor, threshold_p):
    """Algorithm 1 for every sequence; pb's topk are the base budgets.  Returns (k_final, k_anchor, T_anchor)."""
    cov = np.ascontiguousarray(coverage_host, dtype=np.float32)
    kf, ka = np.zeros(max(pb.S, 1), dtype=np.int32), np.zeros(max(pb.S, 1), dtype=np.int32)
    ta = C.c_double()
    _check(lib().sb_dst_tune(pb.ref(), _ptr(cov), tab.ref(), int(anchor), C.c_double(threshold_p), _ptr(kf), _ptr(ka), C.byref(ta)))
    return kf[: pb.S], ka[: pb.S], ta.value


class SparsityPredictor:
    """Spar of Algorithm 2: per length bin, a moving average of the budgets the tuning step produced."""

    def __init__(self, bin_edges, decay=0.9):
        self.edges = np.ascontiguousarray(bin_edges, dtype=np.float32)
        self.nb = len(self.edges) - 1
        self.ema = np.zeros(self.nb, dtype=np.float32)
        self.seen = np.zeros(self.nb, dtype=np.uint8)
        self.decay = float(decay)

    def update(self, lengths, k_final):
        L, k = np.ascontiguousarray(lengths, dtype=np.int32), np.ascontiguousarray(k_final, dtype=np.int32)
        _check(lib().sb_spar_update(_ptr(self.ema), _ptr(self.seen), _ptr(self.edges), self.nb, C.c_double(self.decay), _ptr(L), _ptr(k), len(L)))

    def predict(self, length, k_base) -> float:
        out = C.c_double()
        _check(lib().sb_spar_predict(_ptr(self.ema), _ptr(self.seen), _ptr(self.edges), self.nb, int(length), C.c_double(k_base), C.byref(out)))
        return out.value


def sb_balanced_partition(weights, num_bins) -> np.ndarray:
    w = np.ascontiguousarray(weights, dtype=np.float64)
    out = np.zeros(max(len(w), 1), dtype=np.int32)
    _check(lib().sb_balanced_partition(_ptr(w), len(w), int(num_bins), _ptr(out)))
    return out[: len(w)]


def sb_sab_batches(tab: PerfTable, lengths, k_pred, dp_size, dp_rank, num_microbatches):
    """Algorithm 2.  Returns (weights, dp_bin_of, mb_bin_of)."""
    L, k = np.ascontiguousarray(lengths, dtype=np.int32), np.ascontiguousarray(k_pred, dtype=np.float64)
    n = len(L)
    w, dp, mb = np.zeros(max(n, 1)), np.zeros(max(n, 1), dtype=np.int32), np.zeros(max(n, 1), dtype=np.int32)
    _check(lib().sb_sab_batches(tab.ref(), _ptr(L), _ptr(k), n, int(dp_size), int(dp_rank), int(num_microbatches), _ptr(w), _ptr(dp), _ptr(mb)))
    return w[:n], dp[:n], mb[:n]


# ------------------------------------------------------------------ rotary positions, window attention, paged cache
# A call of a serving step takes the GPU a few microseconds, so what the binding takes counts: a tensor is checked by one expression (and looked at again for the message
# if that fails), addresses go to the library as plain integers, and device and stream are asked for once a call.
SB_ROPE_HALF, SB_ROPE_INTERLEAVED = 0, 1
SB_ROPE_PLAIN, SB_ROPE_LINEAR, SB_ROPE_NTK, SB_ROPE_YARN, SB_ROPE_BANDS = range(5)
_TORCH_DTYPE = {SB_BF16: torch.bfloat16, SB_F32: torch.float32}


def _call(name, *args):
    """One of the calls below, by a function object whose argument types are set."""
    global _calls
    if _calls is None:
        P, I, L = C.c_void_p, C.c_int32, C.c_int64
        types = {"sb_rope_apply": [P, P, P, P, L, P, L, P, P, I, P], "sb_window_attn_fwd": [P, I, I] + [P] * 7, "sb_window_attn_bwd": [P, I, I] + [P] * 11,
                 "sb_cache_append": [P, P, P, P, L, P, L, P, L, P, P], "sb_cache_attn": [P, P, I, I] + [P] * 5}
        # (function objects of their own: those of `lib()` keep taking what ctypes makes of their arguments.  All at once: another thread may be here too)
        _calls = {n: C.CFUNCTYPE(C.c_int, *t)((n, lib())) for n, t in types.items()}
    rc = _calls[name](*args)
    if rc != SB_OK:
        _check(rc)


_calls = None


def _here():
    """(current device, its current stream)"""
    try:
        device = torch._C._cuda_getDevice()
        return device, torch._C._cuda_getCurrentRawStream(device)
    except RuntimeError:
        return -2, 0  # no GPU: no tensor lies on the device, and each is refused


def _tensor(name, t, shape, dtype, device, pitch=False):
    """Refuses a tensor that the library could not use as it lies in memory.  pitch: tokens [T][H][D] may be further apart than their elements."""
    if isinstance(t, torch.Tensor) and t.get_device() == device and t.dtype is dtype and t.shape == shape:
        if t.is_contiguous():
            return
        if pitch:
            token, head, element = t.stride()
            if element == 1 and (head == shape[2] or shape[1] == 1) and (shape[0] == 1 or token >= shape[1] * shape[2]):
                return
    def need(ok, what):
        if not ok:
            raise SparseBalError(f"{name}: {what}")
    need(isinstance(t, torch.Tensor) and t.is_cuda, "a GPU tensor is needed")
    need(t.get_device() == device, f"lies on {t.device}, the current device is cuda:{device}")
    need(t.dtype is dtype, f"{t.dtype} given, {dtype} needed")
    need(t.shape == shape, f"shape {tuple(t.shape)} given, {tuple(shape)} needed")
    need(False, "a token's heads must be contiguous, and tokens in order" if pitch else "must be contiguous")


def _elsewhere(name, there, device):
    raise SparseBalError(f"{name}: lies on {'cuda:' + str(there) if there >= 0 else 'the CPU'}, the current device is cuda:{device}")


def _batch(pb, device):
    """Refuses a batch whose lengths the kernels would have to read on another device.  (Without any on a device the library refuses it.)"""
    if pb.cu_dev is not None and pb.cu_dev.get_device() != device:
        _elsewhere("cu_seqlens", pb.cu_dev.get_device(), device)


def _pitch(t):
    return 0 if t is None or t.shape[0] < 2 else t.stride(0)


def _address(t):
    return None if t is None else t.data_ptr()


def _workspace(ws, need, device):
    if ws is None:
        return _bytes(need, torch.device("cuda", device)) if need else None
    if ws.get_device() != device or not ws.is_contiguous() or ws.numel() * ws.element_size() < need:
        raise SparseBalError(f"ws: {need} contiguous bytes on cuda:{device} are needed")
    return ws


class Rope:
    """Holds sb_rope: how many revolutions a token each pair of elements turns.  `low`, `high`: 0 for the scaling's own values."""

    def __init__(self, rot_dim, layout=SB_ROPE_HALF, base=10000.0, scaling=SB_ROPE_PLAIN, factor=1.0, original_length=0.0, low=0.0, high=0.0):
        self.c = sb_rope()
        _check(lib().sb_rope_init(C.byref(self.c), int(rot_dim), int(layout), C.c_double(base), int(scaling), C.c_double(factor),
                                  C.c_double(original_length), C.c_double(low), C.c_double(high)))

    def ref(self):
        return C.byref(self.c)


def sb_rope_apply(pb: Problem, rope: Rope, q, k, positions=None, backward=False, q_out=None, k_out=None):
    """(q, k) turned by their positions (the tokens' indices in their sequences, or `positions`), or gradients turned back.  q and k may
    be slices of a fused projection; either may be None.  q_out, k_out may be q and k where these are contiguous."""
    dt, (device, stream) = _TORCH_DTYPE[pb.dtype], _here()
    if positions is None:
        _batch(pb, device)
    if q is not None:
        shape = (pb.T, pb.Hq, pb.D)
        _tensor("q", q, shape, dt, device, pitch=True)
        if q_out is None:
            q_out = torch.empty(shape, dtype=dt, device=q.device)
        else:
            _tensor("q_out", q_out, shape, dt, device)
    if k is not None:
        shape = (pb.T, pb.Hkv, pb.D)
        _tensor("k", k, shape, dt, device, pitch=True)
        if k_out is None:
            k_out = torch.empty(shape, dtype=dt, device=k.device)
        else:
            _tensor("k_out", k_out, shape, dt, device)
    if positions is not None:
        _tensor("positions", positions, (pb.T,), torch.int32, device)
    _call("sb_rope_apply", C.addressof(pb.c), C.addressof(rope.c), _address(positions), _address(q), _pitch(q), _address(k), _pitch(k), _address(q_out),
          _address(k_out), 1 if backward else 0, stream)
    return q_out, k_out


def _window(window, sinks):
    """Both as the library's 32-bit numbers; a larger one would lose its upper bits on the way."""
    if window > 2 ** 31 - 1 or sinks > 2 ** 31 - 1 or window < 1 or sinks < 0:
        raise SparseBalError(f"window ({window}) must be 1 .. 2^31 - 1 and sinks ({sinks}) 0 .. 2^31 - 1")
    return int(window), int(sinks)


def sb_window_ws_bytes(pb: Problem, window, sinks):
    """(forward, backward) bytes of the workspaces of sb_window_attn_fwd and sb_window_attn_bwd."""
    window, sinks = _window(window, sinks)
    f, b = C.c_int64(), C.c_int64()
    _check(lib().sb_window_ws_bytes(pb.ref(), int(window), int(sinks), C.byref(f), C.byref(b)))
    return f.value, b.value


def sb_window_attn_fwd(pb: Problem, window, sinks, q, k, v, o=None, lse=None, ws=None):
    """Attention with a sliding window and sinks; pb's budgets and blocks are not read.  Returns (o, lse).  (ws: the forward needs none.)"""
    dt, (device, stream) = _TORCH_DTYPE[pb.dtype], _here()
    _batch(pb, device)
    queries, keys, rows = (pb.T, pb.Hq, pb.D), (pb.T, pb.Hkv, pb.D), (pb.Hq, pb.T)
    _tensor("q", q, queries, dt, device)
    _tensor("k", k, keys, dt, device)
    _tensor("v", v, keys, dt, device)
    if o is None:
        o = torch.empty_like(q)
    else:
        _tensor("o", o, queries, dt, device)
    if lse is None:
        lse = torch.empty(rows, dtype=torch.float32, device=q.device)
    else:
        _tensor("lse", lse, rows, torch.float32, device)
    window, sinks = _window(window, sinks)
    ws = _workspace(ws, 0, device)
    _call("sb_window_attn_fwd", C.addressof(pb.c), window, sinks, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), _address(ws),
          stream)
    return o, lse


def sb_window_attn_bwd(pb: Problem, window, sinks, q, k, v, o, lse, d_o, dq=None, dk=None, dv=None, ws=None):
    dt, (device, stream) = _TORCH_DTYPE[pb.dtype], _here()
    _batch(pb, device)
    queries, keys = (pb.T, pb.Hq, pb.D), (pb.T, pb.Hkv, pb.D)
    for name, x, shape in (("q", q, queries), ("k", k, keys), ("v", v, keys), ("o", o, queries), ("d_o", d_o, queries)):
        _tensor(name, x, shape, dt, device)
    _tensor("lse", lse, (pb.Hq, pb.T), torch.float32, device)
    dq = dq if dq is not None else torch.empty_like(q)
    dk = dk if dk is not None else torch.empty_like(k)
    dv = dv if dv is not None else torch.empty_like(v)
    for name, x, shape in (("dq", dq, queries), ("dk", dk, keys), ("dv", dv, keys)):
        _tensor(name, x, shape, dt, device)
    window, sinks = _window(window, sinks)
    ws = _workspace(ws, sb_window_ws_bytes(pb, window, sinks)[1], device)
    _call("sb_window_attn_bwd", C.addressof(pb.c), window, sinks, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(),
          d_o.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), _address(ws), stream)
    return dq, dk, dv


class Cache:
    """Holds sb_cache plus the tensors it points to: k, v [pages][KV heads][tokens of a page][head_dim], page_table [sequences][most pages of one] int32."""

    def __init__(self, k, v, page_table):
        if k.dim() != 4 or k.dtype not in _TORCH_DTYPE.values():
            raise SparseBalError("k: [pages][KV heads][tokens of a page][head_dim] in bfloat16 or float32 is needed")
        if page_table.dim() != 2:
            raise SparseBalError("page_table: [sequences][pages] is needed")
        self.device = device = _here()[0]
        _tensor("k", k, k.shape, k.dtype, device)
        _tensor("v", v, k.shape, k.dtype, device)
        _tensor("page_table", page_table, page_table.shape, torch.int32, device)
        self.k, self.v, self.page_table = k, v, page_table
        self.c = sb_cache(k.shape[0], k.shape[2], k.shape[1], k.shape[3], SB_F32 if k.dtype == torch.float32 else SB_BF16, page_table.shape[1],
                          k.data_ptr(), v.data_ptr(), page_table.data_ptr())

    def ref(self):
        return C.byref(self.c)


class Chunk:
    """Holds sb_chunk plus the tensors it points to: the new tokens of every sequence.  Sizes on the host are bounds (see sb_chunk); the tensors may change between calls."""

    def __init__(self, cu_new, cached, Hq, total_new, max_new, max_length, softmax_scale=0.0):
        S, device = cached.shape[0], _here()[0]
        self.device = device
        _tensor("cu_new", cu_new, (S + 1,), torch.int32, device)
        _tensor("cached", cached, (S,), torch.int32, device)
        for name, x in (("Hq", Hq), ("total_new", total_new), ("max_new", max_new), ("max_length", max_length)):
            if not -2 ** 31 <= x < 2 ** 31:
                raise SparseBalError(f"{name}: {x} does not fit 32 bits")
        self.cu_new, self.cached, self.Hq, self.total_new = cu_new, cached, int(Hq), int(total_new)
        self.c = sb_chunk(S, int(Hq), int(total_new), int(max_new), int(max_length), float(softmax_scale), cu_new.data_ptr(), cached.data_ptr())

    def ref(self):
        return C.byref(self.c)


def _same_sequences(cache, chunk, device):
    if cache.device != device:
        _elsewhere("cache", cache.device, device)
    if chunk.device != device:
        _elsewhere("chunk", chunk.device, device)
    if cache.page_table.shape[0] != chunk.c.num_seqs:
        raise SparseBalError(f"page_table: {cache.page_table.shape[0]} rows for {chunk.c.num_seqs} sequences")


def sb_cache_append(cache: Cache, chunk: Chunk, k, v, rope: Rope = None, q=None, q_out=None):
    """New tokens' k (turned) and v into their pages; returns q turned likewise (None without q)."""
    n, D, dt, (device, stream) = chunk.total_new, cache.c.head_dim, cache.k.dtype, _here()
    _same_sequences(cache, chunk, device)
    keys, queries = (n, cache.c.num_kv_heads, D), (n, chunk.Hq, D)
    _tensor("k", k, keys, dt, device, pitch=True)
    _tensor("v", v, keys, dt, device, pitch=True)
    if q is not None:
        _tensor("q", q, queries, dt, device, pitch=True)
        if q_out is None:
            q_out = torch.empty(queries, dtype=dt, device=q.device)
        else:
            _tensor("q_out", q_out, queries, dt, device)
    elif q_out is not None:
        raise SparseBalError("q_out without q")
    _call("sb_cache_append", C.addressof(cache.c), C.addressof(chunk.c), C.addressof(rope.c) if rope is not None else None, _address(q), _pitch(q),
          k.data_ptr(), _pitch(k), v.data_ptr(), _pitch(v), _address(q_out), stream)
    return q_out


def sb_cache_attn_ws_bytes(cache: Cache, chunk: Chunk, window, sinks) -> int:
    out, (window, sinks) = C.c_int64(), _window(window, sinks)
    _check(lib().sb_cache_attn_ws_bytes(cache.ref(), chunk.ref(), int(window), int(sinks), C.byref(out)))
    return out.value


def sb_cache_attn(cache: Cache, chunk: Chunk, q, window=2 ** 31 - 1, sinks=0, o=None, lse=None, ws=None):
    """Attention of the new tokens over the cache, which holds them already.  Returns (o, lse)."""
    dt, (device, stream) = cache.k.dtype, _here()
    _same_sequences(cache, chunk, device)
    queries, rows = (chunk.total_new, chunk.Hq, cache.c.head_dim), (chunk.Hq, chunk.total_new)
    _tensor("q", q, queries, dt, device)
    if o is None:
        o = torch.empty_like(q)
    else:
        _tensor("o", o, queries, dt, device)
    if lse is None:
        lse = torch.empty(rows, dtype=torch.float32, device=q.device)
    else:
        _tensor("lse", lse, rows, torch.float32, device)
    window, sinks = _window(window, sinks)
    ws = _workspace(ws, sb_cache_attn_ws_bytes(cache, chunk, window, sinks), device)
    _call("sb_cache_attn", C.addressof(cache.c), C.addressof(chunk.c), window, sinks, q.data_ptr(), o.data_ptr(), lse.data_ptr(), _address(ws), stream)
    return o, lse


SB_INSTR_CU_BUSY, SB_INSTR_KERNEL_EVENTS = 1, 2
KERNEL_NAMES = ["pool", "score", "topk", "plan", "fwd", "bwd_prep", "bwd_dq", "bwd_dkv", "coverage", "score_select", "rope", "window_fwd", "window_dq", "window_dkv",
                "cache_attn"]


def sb_set_instrumentation(flag: int):
    _check(lib().sb_set_instrumentation(int(flag)))


def sb_read_kernel_times():
    """{kernel: (total_ms, launches)} since the last call."""
    ms = np.zeros(len(KERNEL_NAMES), dtype=np.float64)
    cnt = np.zeros(len(KERNEL_NAMES), dtype=np.int64)
    _check(lib().sb_read_kernel_times(_ptr(ms), _ptr(cnt)))
    return {n: (float(ms[i]), int(cnt[i])) for i, n in enumerate(KERNEL_NAMES)}


def sb_read_cu_busy(ws) -> np.ndarray:
    out = np.zeros(SB_CU_SLOTS, dtype=np.uint64)
    _check(lib().sb_read_cu_busy(_ptr(ws), _ptr(out), _stream()))
    return out


def sb_version() -> str:
    return lib().sb_version().decode()


# ------------------------------------------------------------------ plan inspection (tests only)
_PLAN_KEYS = ["qb_off", "bm_off", "qb_seq", "work_fwd", "colcost", "bitmap", "bwd_items", "counters", "split_cols",
              "bwd_items_count", "split_weight", "split_max"]


def plan_views(pb: Problem, plan: torch.Tensor):
    """Decode the opaque plan for property tests, from the section offsets the library reports.  Everything is at the
    granularity of 64-token tiles (NT of them), whatever the selection block size."""
    sec = np.zeros(len(_PLAN_KEYS), dtype=np.int64)
    _check(lib().sb_plan_sections(pb.ref(), _ptr(sec)))
    o = dict(zip(_PLAN_KEYS, (int(x) for x in sec)))
    S, Hkv = pb.S, pb.Hkv
    raw = plan.cpu().numpy()

    def view(start, count, dt):
        return raw[start:start + count * np.dtype(dt).itemsize].view(dt)

    qb_off = view(o["qb_off"], S + 1, np.int32)
    NT = int(qb_off[-1])
    Hs = pb.layout.sel_heads
    counters = view(o["counters"], 3, np.int32)
    return {
        "qb_off": qb_off, "bm_off": view(o["bm_off"], S + 1, np.int64), "qb_seq": view(o["qb_seq"], NT, np.int32),
        "work_fwd": view(o["work_fwd"], Hs * NT, np.int32), "colcost": view(o["colcost"], Hkv * NT, np.int32),
        "bitmap": raw[o["bitmap"]:o["bwd_items"]].view(np.uint32),
        "bwd_items": view(o["bwd_items"], 4 * o["bwd_items_count"], np.int32).reshape(-1, 4),
        "slots_used": int(counters[0]), "sub_slots_used": int(counters[2]), "split_cols": view(o["split_cols"], 3 * int(counters[1]), np.int32).reshape(-1, 3),
        "split_weight": o["split_weight"], "split_max": o["split_max"],
    }

"""ctypes binding of include/tokenselect.h: argument marshalling only.

Every function takes torch tensors that already live on the GPU (PyTorch is used for device memory
and streams, nothing else) and forwards their data pointers; all arithmetic runs in the HIP kernels
of libtokenselect.so.  There is no CPU fallback: if the library is missing, load() raises.
"""
from __future__ import annotations

import ctypes
import os
import re
from typing import Optional

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libtokenselect.so")
_HEADER = os.path.join(os.path.dirname(_HERE), "include", "tokenselect.h")

TS_F32, TS_BF16 = 0, 1
TS_TOPK_FLAT_VOTES = 1
TS_TOPK_VOTE_HIST = 2


class TokenSelectError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s failed: %s (%d)" % (where, ts_strerror(status), status))


class _CProblem(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("chunk", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
        ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32),
        ("max_seq_len", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("k_pool", ctypes.c_void_p), ("v_pool", ctypes.c_void_p), ("page_indptr", ctypes.c_void_p),
        ("page_indices", ctypes.c_void_p), ("seq_lens", ctypes.c_void_p),
        ("num_initial", ctypes.c_int32), ("num_local", ctypes.c_int32),
    ]


class _CSelcache(ctypes.Structure):
    _fields_ = [("cached_q", ctypes.c_void_p), ("cached_q_next", ctypes.c_void_p), ("first", ctypes.c_void_p),
                ("first_next", ctypes.c_void_p), ("reuse", ctypes.c_void_p), ("theta", ctypes.c_float)]


class _CRope(ctypes.Structure):
    _fields_ = [("inv_freq", ctypes.c_void_p), ("rotary_dim", ctypes.c_int32), ("num_axes", ctypes.c_int32),
                ("adjacent", ctypes.c_int32), ("scale", ctypes.c_float), ("pair_axis", ctypes.c_uint8 * 64)]


_lib = None


def lib_path() -> str:
    return _LIB_PATH


def declared_symbols():
    """Names of the functions include/tokenselect.h declares."""
    text = open(_HEADER).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(ts_[a-z_]+)\s*\(", text)))


def load():
    """Loads libtokenselect.so (built by paper_2411_02886_amd.build).  Raises if it is not there."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise FileNotFoundError("%s is missing: run `python -m paper_2411_02886_amd.build` (no CPU fallback exists)"
                                    % _LIB_PATH)
        L = ctypes.CDLL(_LIB_PATH)
        vp, i32, i64, f32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
        pp = ctypes.POINTER(_CProblem)
        L.ts_version.restype = i32
        L.ts_strerror.restype = ctypes.c_char_p
        L.ts_strerror.argtypes = [i32]
        L.ts_workspace_bytes.argtypes = [pp, i32, ctypes.POINTER(sz)]
        L.ts_workspace_init.argtypes = [vp, sz, vp]
        L.ts_paged_qk_scores.argtypes = [pp, vp, vp, f32, vp, vp, sz, vp]
        L.ts_soft_vote.argtypes = [pp, vp, f32, vp, vp, vp, vp, sz, vp]
        L.ts_soft_vote_ranked.argtypes = [pp, vp, f32, vp, vp, vp, vp, sz, vp]
        L.ts_topk.argtypes = [pp, vp, i32, vp, vp, vp, i32, vp, sz, vp]
        L.ts_topk_noalloc.argtypes = [pp, vp, i32, vp, vp, vp, i32, vp]
        L.ts_paged_qk_codes.argtypes = [pp, vp, vp, f32, vp, vp, sz, vp]
        L.ts_soft_vote_bounds.argtypes = [pp, vp, f32, vp, vp, vp, vp, vp, sz, vp]
        L.ts_topk_exact.argtypes = [pp, vp, vp, vp, f32, i32, vp, vp, vp, vp, vp, sz, vp]
        L.ts_selcache_check.argtypes = [pp, vp, vp, vp, f32, vp, vp]
        L.ts_paged_qk_scores_checked.argtypes = [pp, vp, ctypes.POINTER(_CSelcache), vp, f32, vp, sz, vp]
        L.ts_paged_qk_codes_checked.argtypes = [pp, vp, ctypes.POINTER(_CSelcache), vp, f32, vp, sz, vp]
        L.ts_sparse_paged_attn.argtypes = [pp, vp, vp, i32, vp, f32, vp, vp, vp, sz, vp]
        L.ts_chunk_row_stats.argtypes = [pp, vp, f32, vp, vp, sz, vp]
        L.ts_chunk_soft_vote.argtypes = [pp, vp, vp, f32, vp, vp, sz, vp]
        L.ts_chunk_mean_query.argtypes = [pp, vp, vp, vp]
        L.ts_sum_vote.argtypes = [pp, vp, vp, vp, vp]
        L.ts_head_vote_scratch_bytes.argtypes = [pp, ctypes.POINTER(sz)]
        L.ts_head_vote.argtypes = [pp, vp, i32, vp, vp, vp, sz, vp]
        L.ts_paged_attn_workspace_bytes.argtypes = [pp, i32, ctypes.POINTER(sz)]
        L.ts_paged_attn.argtypes = [pp, vp, vp, i32, i32, f32, vp, vp, vp, sz, vp]
        L.ts_paged_attn_rounded.argtypes = L.ts_paged_attn.argtypes
        L.ts_rope_append.argtypes = [pp, ctypes.POINTER(_CRope), vp, i64, vp, i64, vp, i64, vp, i32, vp, vp, vp]
        L.ts_pages_copy.argtypes = [pp, vp, vp, i32, i32, vp]
        L.ts_cache_compact.argtypes = [pp, vp, i32, vp, vp, vp, vp, vp, vp]
        L.ts_debug_set_score_variant.argtypes = [i32, i32, i32]
        L.ts_debug_set_topk_path.argtypes = [i32]
        L.ts_debug_set_codes_path.argtypes = [i32, i32]
        L.ts_debug_event_create.argtypes = [ctypes.POINTER(vp)]
        L.ts_debug_event_destroy.argtypes = [vp]
        L.ts_debug_event_elapsed_ms.argtypes = [vp, vp, ctypes.POINTER(f32)]
        L.ts_debug_set_score_timing_events.argtypes = [vp, vp]
        for name in ("ts_workspace_bytes", "ts_workspace_init", "ts_paged_qk_scores", "ts_soft_vote", "ts_topk",
                     "ts_selcache_check", "ts_sparse_paged_attn", "ts_debug_set_score_variant", "ts_chunk_row_stats",
                     "ts_chunk_soft_vote", "ts_chunk_mean_query", "ts_sum_vote", "ts_head_vote_scratch_bytes",
                     "ts_head_vote", "ts_debug_set_topk_path", "ts_debug_event_create", "ts_debug_event_destroy",
                     "ts_debug_event_elapsed_ms", "ts_debug_set_score_timing_events", "ts_paged_qk_codes",
                     "ts_soft_vote_bounds", "ts_topk_exact", "ts_debug_set_codes_path", "ts_topk_noalloc",
                     "ts_paged_qk_scores_checked", "ts_paged_qk_codes_checked", "ts_soft_vote_ranked",
                     "ts_paged_attn_workspace_bytes", "ts_paged_attn", "ts_paged_attn_rounded", "ts_rope_append", "ts_pages_copy", "ts_cache_compact"):
            getattr(L, name).restype = i32
        _lib = L
    return _lib


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


_raw_stream = _device = None


def _current_stream() -> int:
    """Handle of the current stream of the current device.  Four of these are in every decode step, so the Stream object
    that torch.cuda.current_stream() builds (about 2 us) is left out."""
    if _raw_stream is None:
        _find_raw_stream()
    return _raw_stream(_device())


def _find_raw_stream() -> None:
    global _raw_stream, _device
    import torch
    torch.cuda.init()
    _raw_stream, _device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
    if _raw_stream is None or _device is None:
        _raw_stream, _device = (lambda i: torch.cuda.current_stream(i).cuda_stream), torch.cuda.current_device


def _stream(stream) -> Optional[int]:
    if stream is None:
        return _current_stream() or None
    return getattr(stream, "cuda_stream", stream) or None


def _ok(status: int, where: str) -> None:
    if status != 0:
        raise TokenSelectError(status, where)


class Problem:
    """ts_problem plus references that keep the tensors it points at alive."""

    def __init__(self, *, batch, chunk=1, num_q_heads, num_kv_heads, head_dim, page_size, max_seq_len, dtype,
                 k_pool, v_pool, page_indptr, page_indices, seq_lens, num_initial=0, num_local=0):
        self._keep = (k_pool, v_pool, page_indptr, page_indices, seq_lens)
        self.c = _CProblem(batch, chunk, num_q_heads, num_kv_heads, head_dim, page_size, max_seq_len, dtype,
                           _ptr(k_pool), _ptr(v_pool), _ptr(page_indptr), _ptr(page_indices), _ptr(seq_lens),
                           int(num_initial), int(num_local))
        self.q_row, self.kv_row = num_q_heads * head_dim, num_kv_heads * head_dim      # elements of a token's q, and of its k or v
        self._ref = ctypes.byref(self.c)
        self.batch, self.heads, self.dtype = batch, num_q_heads, dtype
        self.device = -1 if k_pool is None else k_pool.get_device()                    # -1: not on a GPU

    def ref(self):
        return self._ref

    def with_chunk(self, chunk: int):
        """The same problem with another number of new tokens per sequence."""
        c = self.c
        k_pool, v_pool, page_indptr, page_indices, seq_lens = self._keep
        return Problem(batch=c.batch, chunk=chunk, num_q_heads=c.num_q_heads, num_kv_heads=c.num_kv_heads, head_dim=c.head_dim, page_size=c.page_size,
                       max_seq_len=c.max_seq_len, dtype=c.dtype, k_pool=k_pool, v_pool=v_pool, page_indptr=page_indptr, page_indices=page_indices,
                       seq_lens=seq_lens, num_initial=c.num_initial, num_local=c.num_local)


class Rope:
    """ts_rope plus a reference that keeps the frequencies alive.  pair_axis: the position axis of each pair (rotary_dim / 2
    numbers), or None: every pair turns with the first axis.  inv_freq: float tensor on the GPU, one per pair."""

    def __init__(self, *, inv_freq, pair_axis=None, num_axes=1, adjacent=False, scale=1.0):
        n = int(inv_freq.numel())
        axes = [0] * n if pair_axis is None else [int(i) for i in pair_axis]
        if len(axes) != n or n > 64 or any(not 0 <= i < 256 for i in axes):
            raise ValueError("pair_axis: one axis for each of the %d pairs (at most 64)" % n)
        if str(inv_freq.dtype) != "torch.float32" or not inv_freq.is_contiguous():
            raise ValueError("inv_freq: a contiguous float32 tensor")
        self._keep = inv_freq
        self.num_axes, self.device = int(num_axes), inv_freq.get_device()
        self.c = _CRope(_ptr(inv_freq), 2 * n, int(num_axes), int(bool(adjacent)), float(scale), (ctypes.c_uint8 * 64)(*axes))
        self._ref = ctypes.byref(self.c)

    def ref(self):
        return self._ref


def rope_axes(sections, dealt=False):
    """Axis of each pair for position axes that get sections[a] pairs each: the first axis' pairs, then the next one's; dealt:
    in turn, axis after axis, as long as an axis has pairs left."""
    sections = [int(n) for n in sections]
    if not dealt:
        return [a for a, n in enumerate(sections) for _ in range(n)]
    left, axes = list(sections), []
    while any(left):
        for a in range(len(left)):
            if left[a]:
                left[a] -= 1
                axes.append(a)
    return axes


def ts_version() -> int:
    return int(load().ts_version())


def ts_strerror(status: int) -> str:
    return load().ts_strerror(int(status)).decode()


def ts_workspace_bytes(p: Problem, k: int) -> int:
    out = ctypes.c_size_t(0)
    _ok(load().ts_workspace_bytes(p.ref(), int(k), ctypes.byref(out)), "ts_workspace_bytes")
    return int(out.value)


def ts_workspace_init(ws, stream=None) -> None:
    _ok(load().ts_workspace_init(_ptr(ws), ws.numel() * ws.element_size(), _stream(stream)), "ts_workspace_init")


def ts_debug_set_score_variant(variant: int, wg: int = 0, run_tiles: int = 0) -> None:
    _ok(load().ts_debug_set_score_variant(int(variant), int(wg), int(run_tiles)), "ts_debug_set_score_variant")


def ts_debug_set_codes_path(mfma: int, run_tiles: int = 0) -> None:
    _ok(load().ts_debug_set_codes_path(int(mfma), int(run_tiles)), "ts_debug_set_codes_path")


def ts_debug_set_topk_path(five_pass: int) -> None:
    _ok(load().ts_debug_set_topk_path(int(five_pass)), "ts_debug_set_topk_path")


def ts_debug_event_create() -> int:
    ev = ctypes.c_void_p(0)
    _ok(load().ts_debug_event_create(ctypes.byref(ev)), "ts_debug_event_create")
    return int(ev.value)


def ts_debug_event_destroy(ev: int) -> None:
    _ok(load().ts_debug_event_destroy(ctypes.c_void_p(ev)), "ts_debug_event_destroy")


def ts_debug_event_elapsed_ms(start: int, stop: int) -> float:
    ms = ctypes.c_float(0.0)
    _ok(load().ts_debug_event_elapsed_ms(ctypes.c_void_p(start), ctypes.c_void_p(stop), ctypes.byref(ms)),
        "ts_debug_event_elapsed_ms")
    return float(ms.value)


def ts_debug_set_score_timing_events(start, stop) -> None:
    _ok(load().ts_debug_set_score_timing_events(ctypes.c_void_p(start) if start else None,
                                                ctypes.c_void_p(stop) if stop else None),
        "ts_debug_set_score_timing_events")


def _nbytes(ws) -> int:
    return ws.numel() * ws.element_size() if ws is not None else 0


def ts_paged_qk_scores(p: Problem, q, scores, score_scale: float, skip, ws, stream=None) -> None:
    _ok(load().ts_paged_qk_scores(p.ref(), _ptr(q), _ptr(scores), float(score_scale), _ptr(skip), _ptr(ws), _nbytes(ws),
                                  _stream(stream)), "ts_paged_qk_scores")


def ts_soft_vote(p: Problem, scores, score_scale: float, row_stats, votes, skip, ws, stream=None) -> None:
    _ok(load().ts_soft_vote(p.ref(), _ptr(scores), float(score_scale), _ptr(row_stats), _ptr(votes), _ptr(skip),
                            _ptr(ws), _nbytes(ws), _stream(stream)), "ts_soft_vote")


def _selcache(cached_q, cached_q_next, first, first_next, reuse, theta) -> _CSelcache:
    return _CSelcache(_ptr(cached_q), _ptr(cached_q_next), _ptr(first), _ptr(first_next), _ptr(reuse), float(theta))


def ts_paged_qk_scores_checked(p: Problem, q, cached_q, cached_q_next, first, first_next, reuse, theta: float, scores,
                               score_scale: float, ws, stream=None) -> None:
    sc = _selcache(cached_q, cached_q_next, first, first_next, reuse, theta)
    _ok(load().ts_paged_qk_scores_checked(p.ref(), _ptr(q), ctypes.byref(sc), _ptr(scores), float(score_scale), _ptr(ws),
                                          _nbytes(ws), _stream(stream)), "ts_paged_qk_scores_checked")


def ts_paged_qk_codes_checked(p: Problem, q, cached_q, cached_q_next, first, first_next, reuse, theta: float, codes,
                              score_scale: float, ws, stream=None) -> None:
    sc = _selcache(cached_q, cached_q_next, first, first_next, reuse, theta)
    _ok(load().ts_paged_qk_codes_checked(p.ref(), _ptr(q), ctypes.byref(sc), _ptr(codes), float(score_scale), _ptr(ws),
                                         _nbytes(ws), _stream(stream)), "ts_paged_qk_codes_checked")


def ts_soft_vote_ranked(p: Problem, scores, score_scale: float, row_stats, votes, skip, ws, stream=None) -> None:
    _ok(load().ts_soft_vote_ranked(p.ref(), _ptr(scores), float(score_scale), _ptr(row_stats), _ptr(votes), _ptr(skip),
                                   _ptr(ws), _nbytes(ws), _stream(stream)), "ts_soft_vote_ranked")


def ts_paged_qk_codes(p: Problem, q, codes, score_scale: float, skip, ws, stream=None) -> None:
    _ok(load().ts_paged_qk_codes(p.ref(), _ptr(q), _ptr(codes), float(score_scale), _ptr(skip), _ptr(ws), _nbytes(ws),
                                 _stream(stream)), "ts_paged_qk_codes")


def ts_soft_vote_bounds(p: Problem, codes, score_scale: float, row_stats, vote_hi, vote_lo, skip, ws, stream=None) -> None:
    _ok(load().ts_soft_vote_bounds(p.ref(), _ptr(codes), float(score_scale), _ptr(row_stats), _ptr(vote_hi),
                                   _ptr(vote_lo), _ptr(skip), _ptr(ws), _nbytes(ws), _stream(stream)),
        "ts_soft_vote_bounds")


def ts_topk_exact(p: Problem, q, vote_hi, row_stats, score_scale: float, k: int, idx, count, skip, ws, stream=None,
                  sel_votes=None) -> None:
    _ok(load().ts_topk_exact(p.ref(), _ptr(q), _ptr(vote_hi), _ptr(row_stats), float(score_scale), int(k), _ptr(idx),
                             _ptr(count), _ptr(sel_votes), _ptr(skip), _ptr(ws), _nbytes(ws), _stream(stream)), "ts_topk_exact")


def ts_chunk_row_stats(p: Problem, q, score_scale: float, row_stats, ws, stream=None) -> None:
    _ok(load().ts_chunk_row_stats(p.ref(), _ptr(q), float(score_scale), _ptr(row_stats), _ptr(ws), _nbytes(ws),
                                  _stream(stream)), "ts_chunk_row_stats")


def ts_chunk_soft_vote(p: Problem, q, row_stats, score_scale: float, votes, ws, stream=None) -> None:
    _ok(load().ts_chunk_soft_vote(p.ref(), _ptr(q), _ptr(row_stats), float(score_scale), _ptr(votes), _ptr(ws),
                                  _nbytes(ws), _stream(stream)), "ts_chunk_soft_vote")


def ts_sum_vote(p: Problem, scores, votes, skip, stream=None) -> None:
    _ok(load().ts_sum_vote(p.ref(), _ptr(scores), _ptr(votes), _ptr(skip), _stream(stream)), "ts_sum_vote")


def ts_head_vote_scratch_bytes(p: Problem) -> int:
    out = ctypes.c_size_t(0)
    _ok(load().ts_head_vote_scratch_bytes(p.ref(), ctypes.byref(out)), "ts_head_vote_scratch_bytes")
    return int(out.value)


def ts_head_vote(p: Problem, scores, k_head: int, votes, skip, scratch, stream=None) -> None:
    _ok(load().ts_head_vote(p.ref(), _ptr(scores), int(k_head), _ptr(votes), _ptr(skip), _ptr(scratch), _nbytes(scratch),
                            _stream(stream)), "ts_head_vote")


def ts_chunk_mean_query(p: Problem, q, q_mean, stream=None) -> None:
    _ok(load().ts_chunk_mean_query(p.ref(), _ptr(q), _ptr(q_mean), _stream(stream)), "ts_chunk_mean_query")


def ts_topk(p: Problem, votes, k: int, idx, count, skip, ws, stream=None, flags: int = 0) -> None:
    _ok(load().ts_topk(p.ref(), _ptr(votes), int(k), _ptr(idx), _ptr(count), _ptr(skip), int(flags), _ptr(ws), _nbytes(ws),
                       _stream(stream)), "ts_topk")


def ts_topk_noalloc(p: Problem, votes, k: int, idx, count, skip, stream=None, flags: int = 0) -> None:
    _ok(load().ts_topk_noalloc(p.ref(), _ptr(votes), int(k), _ptr(idx), _ptr(count), _ptr(skip), int(flags),
                               _stream(stream)), "ts_topk_noalloc")


def ts_selcache_check(p: Problem, q, cached_q, first, theta: float, reuse, stream=None) -> None:
    _ok(load().ts_selcache_check(p.ref(), _ptr(q), _ptr(cached_q), _ptr(first), float(theta), _ptr(reuse),
                                 _stream(stream)), "ts_selcache_check")


def ts_sparse_paged_attn(p: Problem, q, idx, idx_stride: int, count, sm_scale: float, out, lse, ws,
                         stream=None) -> None:
    _ok(load().ts_sparse_paged_attn(p.ref(), _ptr(q), _ptr(idx), int(idx_stride), _ptr(count), float(sm_scale),
                                    _ptr(out), _ptr(lse), _ptr(ws),
                                    ws.numel() * ws.element_size() if ws is not None else 0, _stream(stream)),
        "ts_sparse_paged_attn")


_INT = _FLOAT = _MASK = _STORED = None      # element types: of index arrays, of lse, of skip masks, of q, k, v and results by the problem's


def _load_types():
    global _INT, _FLOAT, _MASK, _STORED
    import torch
    bits = [getattr(torch, name) for name in ("bfloat16", "int16", "uint16") if hasattr(torch, name)]      # bf16 may travel as raw bits
    _FLOAT, _MASK, _INT = (torch.float32,), (torch.uint8, torch.bool), (torch.int32,)
    _STORED = {TS_F32: _FLOAT, TS_BF16: tuple(bits)}


def _refuse(p: Problem, t, name: str, types, need: str):
    if t.dtype not in types:
        raise ValueError("%s: a tensor of %s" % (name, " or ".join(str(x) for x in types)))
    if t.get_device() != p.device:
        raise ValueError("%s: on the device of the pools" % name)
    raise ValueError("%s: %s" % (name, need))


def _at(p: Problem, t, name: str, types, count: int):
    """Address of a tensor that the library takes as an array of `count` elements, or an error where it would read something else."""
    if t is None:
        return None
    if t.dtype in types and t.get_device() == p.device and t.numel() >= count and t.is_contiguous():
        return t.data_ptr()
    _refuse(p, t, name, types, "%d elements one after the other" % count)


def _stream_of(p: Problem, stream):
    """The stream that a call on the problem's pools goes to; without one the current device has to be theirs."""
    if p.device < 0 and p.c.k_pool is not None:
        raise ValueError("the pools are not on a GPU")
    if stream is not None or p.device < 0:
        return _stream(stream)
    if _raw_stream is None:
        _find_raw_stream()
    device = _device()
    if device != p.device:
        raise ValueError("the pools are on device %d, the current one is %d" % (p.device, device))
    return _raw_stream(device) or None


def ts_paged_attn_workspace_bytes(p: Problem, num_rows: int) -> int:
    out = ctypes.c_size_t(0)
    _ok(load().ts_paged_attn_workspace_bytes(p.ref(), int(num_rows), ctypes.byref(out)), "ts_paged_attn_workspace_bytes")
    return int(out.value)


def _attend(call, where, p: Problem, q, q_indptr, num_rows, window, sm_scale, out, lse, ws, stream):
    n = int(num_rows)
    if _STORED is None:
        _load_types()
    stored = _STORED.get(p.dtype, ())
    if ws is not None and ws.get_device() != p.device:
        raise ValueError("ws: on the device of the pools")
    _ok(call(p.ref(), _at(p, q, "q", stored, n * p.q_row), _at(p, q_indptr, "q_indptr", _INT, p.batch + 1), n, int(window), float(sm_scale),
             _at(p, out, "out", stored, n * p.q_row), _at(p, lse, "lse", _FLOAT, n * p.heads), _ptr(ws), _nbytes(ws), _stream_of(p, stream)), where)


def ts_paged_attn(p: Problem, q, q_indptr, num_rows: int, window: int, sm_scale: float, out, lse, ws, stream=None) -> None:
    _attend(load().ts_paged_attn, "ts_paged_attn", p, q, q_indptr, num_rows, window, sm_scale, out, lse, ws, stream)


def ts_paged_attn_rounded(p: Problem, q, q_indptr, num_rows: int, window: int, sm_scale: float, out, lse, ws, stream=None) -> None:
    _attend(load().ts_paged_attn_rounded, "ts_paged_attn_rounded", p, q, q_indptr, num_rows, window, sm_scale, out, lse, ws, stream)


def _row_stride(t, row: int, name: str) -> int:
    """Elements between the rows of a [rows][...] tensor whose rows are packed; row: elements of one."""
    if t is None:
        return 0
    shape = t.shape
    if len(shape) > 1 and t.is_contiguous() and t.numel() == shape[0] * row:      # the usual case, and the quickest answer
        return 0
    strides, want = t.stride(), 1
    if len(shape) > 1 and shape[0] > 1 and strides[0] < row:                      # (0 would mean packed)
        raise ValueError("%s: rows that overlap, such as one that is expanded" % name)
    if len(shape) == 2 and shape[1] == row and strides[1] == 1:
        return strides[0] if shape[0] > 1 else 0
    for i in range(len(shape) - 1, 0, -1):
        if strides[i] != want and shape[i] > 1:
            raise ValueError("%s: the elements of a row must follow each other" % name)
        want *= shape[i]
    if want != row:
        raise ValueError("%s: rows of %d elements, the problem's have %d" % (name, want, row))
    return strides[0] if shape[0] > 1 else 0


def _rows_at(p: Problem, t, row: int, name: str, types, num_rows: int):
    """(address, elements between the rows or 0 for packed) of a [rows][...] tensor; row: elements of one."""
    if t is None:
        return None, 0
    shape = t.shape
    if t.dtype in types and t.get_device() == p.device and shape[0] >= num_rows:
        if len(shape) == 2 and shape[1] == row and shape[0] > 1:                  # parts of a projection, the quickest answer
            strides = t.stride()
            if strides[1] == 1 and strides[0] >= row:
                return t.data_ptr(), strides[0]
        return t.data_ptr(), _row_stride(t, row, name)
    _refuse(p, t, name, types, "%d rows" % num_rows)


def ts_rope_append(p: Problem, rope, q, k, v, q_indptr, num_rows: int, positions, q_out, stream=None) -> None:
    """q, k, v: [rows][heads][D] or [rows][heads * D], rows any multiple of 16 bytes apart; q and q_out, or k and v, may be None."""
    n = int(num_rows)
    if _STORED is None:
        _load_types()
    stored, axes = _STORED.get(p.dtype, ()), 0
    q_at, q_stride = _rows_at(p, q, p.q_row, "q", stored, n)
    k_at, k_stride = _rows_at(p, k, p.kv_row, "k", stored, n)
    v_at, v_stride = _rows_at(p, v, p.kv_row, "v", stored, n)
    if rope is not None:
        axes = rope.num_axes
        if rope.device != p.device and rope.c.rotary_dim:
            raise ValueError("inv_freq: on the device of the pools")
    _ok(load().ts_rope_append(p.ref(), None if rope is None else rope.ref(), q_at, q_stride, k_at, k_stride, v_at, v_stride,
                              _at(p, q_indptr, "q_indptr", _INT, p.batch + 1), n, _at(p, positions, "positions", _INT, axes * n),
                              _at(p, q_out, "q_out", stored, n * p.q_row), _stream_of(p, stream)), "ts_rope_append")


def ts_pages_copy(p: Problem, src, dst, n: int, num_pages: int, stream=None) -> None:
    if _STORED is None:
        _load_types()
    n, elements = int(n), int(num_pages) * p.c.page_size * p.kv_row
    for pool in p._keep[:2]:
        if pool is not None and pool.numel() < elements:
            raise ValueError("num_pages: %d, the pools hold fewer" % num_pages)
    _ok(load().ts_pages_copy(p.ref(), _at(p, src, "src", _INT, n), _at(p, dst, "dst", _INT, n), n, int(num_pages), _stream_of(p, stream)),
        "ts_pages_copy")


def ts_cache_compact(p: Problem, idx, idx_stride: int, count, skip, to_indptr, to_indices, to_lens, stream=None) -> None:
    if _STORED is None:
        _load_types()
    B = p.batch
    _ok(load().ts_cache_compact(p.ref(), _at(p, idx, "idx", _INT, B * int(idx_stride)), int(idx_stride), _at(p, count, "count", _INT, B),
                                _at(p, skip, "skip", _MASK, B), _at(p, to_indptr, "to_indptr", _INT, B + 1),
                                _at(p, to_indices, "to_indices", _INT, 1), _at(p, to_lens, "to_lens", _INT, B), _stream_of(p, stream)),
        "ts_cache_compact")

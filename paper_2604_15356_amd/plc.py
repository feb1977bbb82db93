"""Thin ctypes binding over libplc.so: argument marshalling only.

Every function takes torch tensors that already live on the GPU, passes their
device pointers and the current HIP stream to the C entry point of the same
name (see include/plc.h), and returns.  No step of the coding path runs in
Python or in torch; torch only owns the memory and the stream.  If the library
has not been built, loading fails with an error -- there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libplc.so")

PLC_OK, PLC_ERR_INVALID, PLC_ERR_CAPACITY, PLC_ERR_CORRUPT, PLC_ERR_HIP, PLC_ERR_SCRATCH = 0, 1, 2, 3, 4, 5
STATIC_SCRATCH_BYTES = 48 << 20
PLC_ESCAPE = 255

EXPORTS = ("plc_version", "plc_strerror", "plc_workspace_bytes", "plc_units_per_stream",
           "plc_predict_residual", "plc_predict_residual_hist", "plc_predict_residual_noalloc", "plc_histogram", "plc_build_freq", "plc_rans_encode",
           "plc_rans_decode", "plc_reconstruct", "plc_rans_decode_reconstruct", "plc_rans_decode_reconstruct_cond",
           "plc_rans_decode_reconstruct_adapt",
           "plc_trace_kernel_events", "plc_trace_kernel_name",
           "plc_predict_residual_cond", "plc_reconstruct_cond", "plc_select_candidate",
           "plc_index_encode", "plc_index_decode",
           "plc_surprisal_thresholds", "plc_surprisal_bits", "plc_predict_residual_adapt", "plc_reconstruct_adapt",
           "plc_histogram_bucketed", "plc_build_freq_bucketed", "plc_rans_encode_bucketed",
           "plc_rans_decode_bucketed",
           "plc_restart_points", "plc_decode_one_kernel", "plc_rans_encode_restart", "plc_rans_decode_restart",
           "plc_rans_encode_bucketed_restart", "plc_rans_decode_bucketed_restart",
           "plc_rans_decode_reconstruct_restart", "plc_rans_decode_reconstruct_cond_restart",
           "plc_rans_decode_reconstruct_adapt_restart",
           "plc_expected_embedding", "plc_predict_residual_linear", "plc_reconstruct_linear",
           "plc_pages_workspace_bytes", "plc_pages_fork", "plc_pages_extend", "plc_pages_trim", "plc_pages_accept",
           "plc_pages_compact", "plc_pages_store", "plc_pages_load", "plc_attend_workspace_bytes", "plc_attend",
           "plc_rotary_frequencies", "plc_rotary_turns", "plc_rotate", "plc_rotate_store", "plc_attend_weights", "plc_pages_evict",
           "plc_score_workspace_bytes", "plc_score_tokens",
           "plc_trie_create", "plc_trie_destroy", "plc_trie_size", "plc_trie_nodes", "plc_trie_insert",
           "plc_trie_best_match", "plc_trie_evict")

MAX_BITS = 4
PLC_FP16, PLC_BF16, PLC_FP32 = 0, 1, 2
ROTARY_SCALINGS = ("none", "linear", "stretched", "parts", "ramp")  # PLC_ROTARY_*
MOST_ALTERNATIVES = 32
TREE_NODES = 256
RESTART_WORDS = 34

(TRACE_PREDICT, TRACE_RECONSTRUCT, TRACE_HISTOGRAM, TRACE_RANS_ENCODE, TRACE_RANS_DECODE,
 TRACE_PREDICT_COND, TRACE_RECONSTRUCT_COND, TRACE_EXPECTED_EMBEDDING, TRACE_PREDICT_LINEAR,
 TRACE_RECONSTRUCT_LINEAR) = range(10)


class PlcError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {strerror(code)} (code {code})")


class plc_dims(C.Structure):
    _fields_ = [("S", C.c_int32), ("L", C.c_int32), ("H", C.c_int32), ("n", C.c_int32),
                ("k", C.c_int32), ("d", C.c_int32),
                ("cand_stride", C.c_int64 * 5), ("act_stride", C.c_int64 * 4),
                ("delta", C.c_float), ("qmax", C.c_int32)]


class plc_restart(C.Structure):
    _fields_ = [("points", C.c_void_p), ("scratch", C.c_void_p), ("per_stream", C.c_int32)]


class plc_pages(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("stride", C.c_int64 * 4),
                ("P", C.c_int32), ("L", C.c_int32), ("H", C.c_int32), ("B", C.c_int32), ("d", C.c_int32),
                ("S", C.c_int32), ("M", C.c_int32),
                ("table", C.c_void_p), ("lens", C.c_void_p), ("refs", C.c_void_p)]


class plc_rows(C.Structure):
    _fields_ = [("layer", C.c_int32), ("layers", C.c_int32), ("packed", C.c_int32), ("rows", C.c_int64),
                ("stride", C.c_int64 * 4)]


class plc_rotary_spec(C.Structure):
    _fields_ = [("r", C.c_int32), ("scaling", C.c_int32), ("base", C.c_double), ("factor", C.c_double),
                ("low", C.c_double), ("high", C.c_double), ("trained", C.c_int64)]


class plc_rotary(C.Structure):
    _fields_ = [("turns", C.c_void_p), ("r", C.c_int32), ("interleaved", C.c_int32), ("magnitude", C.c_float)]


class plc_weights(C.Structure):
    _fields_ = [("w", C.c_void_p), ("stride", C.c_int64 * 3), ("width", C.c_int64)]


_lib = None


def lib() -> C.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it first "
                               "(python -m paper_2604_15356_amd.build); there is no fallback path")
        L = C.CDLL(LIB_PATH)
        p, u64, i64, i32, sz = C.c_void_p, C.c_uint64, C.c_int64, C.c_int32, C.c_size_t
        dp = C.POINTER(plc_dims)
        L.plc_version.restype = C.c_int
        L.plc_strerror.restype = C.c_char_p
        L.plc_strerror.argtypes = [C.c_int]
        L.plc_workspace_bytes.restype = sz
        L.plc_workspace_bytes.argtypes = [dp]
        L.plc_units_per_stream.restype = i64
        L.plc_units_per_stream.argtypes = [i64, i32]
        L.plc_predict_residual.argtypes = [dp, p, p, p, p, p, p, p, u64, p, p, p, p, sz, p, p]
        L.plc_predict_residual_hist.argtypes = [dp, p, p, p, p, p, p, p, u64, p, p, p, p, p, sz, p, p]
        L.plc_predict_residual_noalloc.argtypes = [dp, p, p, p, p, p, p, p, u64, p, p, p, p, p]
        L.plc_histogram.argtypes = [p, i64, i64, p, p]
        L.plc_build_freq.argtypes = [p, i64, p, p, p, p]
        L.plc_rans_encode.argtypes = [p, i64, i64, i32, p, p, p, p, u64, p, p, p]
        L.plc_rans_decode.argtypes = [p, p, p, u64, p, p, i64, i64, i32, p, p, p]
        L.plc_reconstruct.argtypes = [dp, p, p, p, p, p, u64, p, p, p, p, sz, p, p]
        L.plc_rans_decode_reconstruct.argtypes = [dp, p, p, p, u64, p, p, i32, p, p, p, p, u64, p, p, p, p, p, sz,
                                                  p, p]
        L.plc_rans_decode_reconstruct_cond.argtypes = [dp, p, p, p, u64, p, p, i32, p, p, p, p, p, u64, p, p, p, p, p,
                                                       sz, p, p]
        L.plc_rans_decode_reconstruct_adapt.argtypes = [dp, p, p, p, u64, p, p, i32, i32, p, p, p, p, p, C.c_float, p,
                                                        u64, p, p, p, p, p, sz, p, p]
        L.plc_trace_kernel_events.argtypes = [C.c_int, p, p]
        L.plc_trace_kernel_name.restype = C.c_char_p
        L.plc_trace_kernel_name.argtypes = [C.c_int]
        L.plc_predict_residual_cond.argtypes = [dp, p, p, p, p, p, p, p, p, u64, p, p, p, p, sz, p, p]
        L.plc_reconstruct_cond.argtypes = [dp, p, p, p, p, p, p, u64, p, p, p, p, sz, p, p]
        L.plc_select_candidate.argtypes = [dp, p, p, C.c_float, p, p]
        L.plc_index_encode.argtypes = [p, p, i32, i32, i32, p, p, p, u64, p, p, p]
        L.plc_index_decode.argtypes = [p, p, p, u64, p, p, i32, i32, i32, p, p, p]
        L.plc_surprisal_thresholds.argtypes = [C.c_double, C.c_double, i32, C.POINTER(C.c_uint16)]
        L.plc_surprisal_bits.argtypes = [p, p, i32, i32, i32, C.POINTER(C.c_uint16), i32, p, p, p]
        L.plc_predict_residual_adapt.argtypes = [dp, p, p, p, p, p, C.c_float, p, p, p, p, u64, p, p, p, p, sz, p, p]
        L.plc_reconstruct_adapt.argtypes = [dp, p, p, p, p, p, C.c_float, p, p, u64, p, p, p, p, sz, p, p]
        L.plc_histogram_bucketed.argtypes = [p, i64, i64, i32, i32, p, i32, p, p, p]
        L.plc_build_freq_bucketed.argtypes = [p, i64, i32, p, p, p]
        L.plc_rans_encode_bucketed.argtypes = [p, i64, i64, i32, i32, i32, p, i32, p, p, p, p, u64, p, p, p]
        L.plc_rans_decode_bucketed.argtypes = [p, p, p, u64, p, p, i64, i64, i32, i32, i32, p, i32, p, p, p]
        rp = C.POINTER(plc_restart)
        L.plc_restart_points.restype = i32
        L.plc_restart_points.argtypes = [i64, i64, i32]
        L.plc_decode_one_kernel.restype = i32
        L.plc_decode_one_kernel.argtypes = [i64, i64, i32, i32, i32, i32, i32]
        L.plc_rans_encode_restart.argtypes = [p, i64, i64, i32, p, p, p, p, u64, p, rp, p, p]
        L.plc_rans_decode_restart.argtypes = [p, p, p, u64, p, p, i64, i64, i32, rp, p, p, p]
        L.plc_rans_encode_bucketed_restart.argtypes = [p, i64, i64, i32, i32, i32, p, i32, p, p, p, p, u64, p, rp, p,
                                                       p]
        L.plc_rans_decode_bucketed_restart.argtypes = [p, p, p, u64, p, p, i64, i64, i32, i32, i32, p, i32, rp, p, p,
                                                       p]
        L.plc_rans_decode_reconstruct_restart.argtypes = [dp, p, p, p, u64, p, p, i32, p, p, p, p, u64, p, p, p, p, p,
                                                          sz, rp, p, p]
        L.plc_rans_decode_reconstruct_cond_restart.argtypes = [dp, p, p, p, u64, p, p, i32, p, p, p, p, p, u64, p, p,
                                                               p, p, p, sz, rp, p, p]
        L.plc_rans_decode_reconstruct_adapt_restart.argtypes = [dp, p, p, p, u64, p, p, i32, i32, p, p, p, p, p,
                                                                C.c_float, p, u64, p, p, p, p, p, sz, rp, p, p]
        gp, kp, i64s = C.POINTER(plc_pages), C.POINTER(plc_rows), C.POINTER(i64)
        L.plc_pages_workspace_bytes.restype = sz
        L.plc_pages_workspace_bytes.argtypes = [gp]
        L.plc_pages_fork.argtypes = [gp, p, p, p]
        L.plc_pages_extend.argtypes = [gp, p, p, sz, p, p]
        L.plc_pages_trim.argtypes = [gp, p, p, p]
        L.plc_pages_accept.argtypes = [gp, p, p, i64, p, p, p]
        L.plc_pages_compact.argtypes = [gp, p, p, sz, p, p]
        L.plc_pages_store.argtypes = [gp, kp, p, p, p, p, p]
        L.plc_pages_load.argtypes = [gp, kp, p, p, p, p, p]
        L.plc_attend_workspace_bytes.restype = sz
        L.plc_attend_workspace_bytes.argtypes = [gp, i32, i64, i32, i32]
        L.plc_attend.argtypes = [gp, i32, i32, p, i64s, i32, i64, p, p, i32, i32, C.c_float, p, i64s, p, p, sz, p, p]
        yp, wp, f32 = C.POINTER(plc_rotary), C.POINTER(plc_weights), C.c_float
        L.plc_rotary_frequencies.argtypes = [C.POINTER(plc_rotary_spec), p]
        L.plc_rotary_turns.argtypes = [p, i32, p]
        L.plc_rotate.argtypes = [yp, i32, p, i64s, i64, i32, i32, p, i32, p, i64s, p]
        L.plc_rotate_store.argtypes = [gp, kp, yp, i32, p, p, p, p, p, p, i64s, i32, p, i64s, p, p]
        L.plc_attend_weights.argtypes = [gp, i32, i32, p, i64s, i32, i64, p, i32, i32, f32, p, f32, wp, p, p]
        L.plc_pages_evict.argtypes = [gp, p, i32, i32, wp, p, i32, i32, p, sz, p, p]
        L.plc_score_workspace_bytes.restype = sz
        L.plc_score_workspace_bytes.argtypes = [i32, i32]
        L.plc_score_tokens.argtypes = [i32, p, i64, i64, i32, f32, p, i32, p, p, p, p, p, p, p, p, sz, p, p]
        L.plc_trie_create.restype = p
        L.plc_trie_create.argtypes = [C.c_double]
        L.plc_trie_destroy.restype = None
        L.plc_trie_destroy.argtypes = [p]
        L.plc_trie_size.restype = i64
        L.plc_trie_size.argtypes = [p]
        L.plc_trie_nodes.restype = i64
        L.plc_trie_nodes.argtypes = [p]
        L.plc_trie_insert.argtypes = [p, p, p, i64, i64, C.POINTER(i64)]
        L.plc_trie_best_match.argtypes = [p, p, i64, C.POINTER(i64), C.POINTER(i64), C.POINTER(C.c_double)]
        L.plc_trie_evict.argtypes = [p, i64]
        L.plc_expected_embedding.argtypes = [p, p, i64, i32, i32, p, p]
        L.plc_predict_residual_linear.argtypes = [dp, p, i32, p, p, p, p, p, p, p, u64, p, p, p, sz, p, p]
        L.plc_reconstruct_linear.argtypes = [dp, p, i32, p, p, p, p, p, u64, p, p, p, p, sz, p, p]
        _lib = L
    return _lib


def strerror(code: int) -> str:
    return lib().plc_strerror(int(code)).decode()


def plc_version() -> int:
    return int(lib().plc_version())


def make_dims(S, L, H, n, k, d, delta, qmax=127, cand_stride=None, act_stride=None) -> plc_dims:
    if cand_stride is None:
        cand_stride = (L * H * n * k * d, H * n * k * d, n * k * d, k * d, d)
    if act_stride is None:
        act_stride = (L * H * n * d, H * n * d, n * d, d)
    dm = plc_dims()
    dm.S, dm.L, dm.H, dm.n, dm.k, dm.d = S, L, H, n, k, d
    dm.cand_stride = (C.c_int64 * 5)(*[int(x) for x in cand_stride])
    dm.act_stride = (C.c_int64 * 4)(*[int(x) for x in act_stride])
    dm.delta = float(delta)
    dm.qmax = int(qmax)
    return dm


def plc_workspace_bytes(dims: plc_dims) -> int:
    return int(lib().plc_workspace_bytes(C.byref(dims)))


def plc_units_per_stream(syms_per_stream: int, chunk_syms: int) -> int:
    return int(lib().plc_units_per_stream(int(syms_per_stream), int(chunk_syms)))


def plc_restart_points(n_streams: int, syms_per_stream: int, chunk_syms: int) -> int:
    return int(lib().plc_restart_points(int(n_streams), int(syms_per_stream), int(chunk_syms)))


def plc_decode_one_kernel(n_streams, syms_per_stream, chunk_syms, k, cond=False, per_depth=False, per_stream=0) -> bool:
    return bool(lib().plc_decode_one_kernel(int(n_streams), int(syms_per_stream), int(chunk_syms), int(k), int(cond),
                                            int(per_depth), int(per_stream)))


def _ptr(t, dtype=None):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("plc takes device tensors")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"expected {dtype}, got {t.dtype}")
    return C.c_void_p(t.data_ptr())


def _contig(t, dtype):
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return _ptr(t, dtype)


def _restart(points_and_scratch):
    """(points int32 [streams, per_stream, RESTART_WORDS], scratch int32 [streams, per_stream, 2] or None) as a
    plc_restart, or None."""
    if points_and_scratch is None:
        return None
    points, scratch = points_and_scratch
    r = plc_restart()
    r.points, r.scratch = _contig(points, torch.int32), _contig(scratch, torch.int32)
    r.per_stream = points.shape[1]
    return C.byref(r)


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _check(rc, where):
    if rc != PLC_OK:
        raise PlcError(rc, where)


def plc_predict_residual(dims, cand_k, cand_v, probs, act_k, act_v, symbols, esc_vals, esc_cnt,
                         esc_off, ws, status, pred_out=None):
    """cand_*/act_* fp16 (strides in dims); probs fp32 [S,n,k]; symbols u8 out; esc_vals int16/uint16
    out (its numel is the capacity); esc_cnt int32 out; esc_off int64 out; ws uint8; status int32[1]."""
    rc = lib().plc_predict_residual(
        C.byref(dims), _ptr(cand_k, torch.float16), _ptr(cand_v, torch.float16),
        _contig(probs, torch.float32), _ptr(act_k, torch.float16), _ptr(act_v, torch.float16),
        _contig(symbols, torch.uint8), _contig(esc_vals, None), esc_vals.numel(),
        _contig(esc_cnt, torch.int32), _contig(esc_off, torch.int64), _contig(pred_out, torch.float32),
        _contig(ws, torch.uint8), ws.numel(), _contig(status, torch.int32), _stream())
    _check(rc, "plc_predict_residual")


def plc_predict_residual_hist(dims, cand_k, cand_v, probs, act_k, act_v, symbols, esc_vals, esc_cnt,
                              esc_off, counts, ws, status, pred_out=None):
    """plc_predict_residual that also leaves the symbols' per-stream counts (int32 [streams, 256]) in `counts`."""
    rc = lib().plc_predict_residual_hist(
        C.byref(dims), _ptr(cand_k, torch.float16), _ptr(cand_v, torch.float16),
        _contig(probs, torch.float32), _ptr(act_k, torch.float16), _ptr(act_v, torch.float16),
        _contig(symbols, torch.uint8), _contig(esc_vals, None), esc_vals.numel(),
        _contig(esc_cnt, torch.int32), _contig(esc_off, torch.int64), _contig(pred_out, torch.float32),
        _contig(counts, torch.int32), _contig(ws, torch.uint8), ws.numel(), _contig(status, torch.int32), _stream())
    _check(rc, "plc_predict_residual_hist")


def plc_predict_residual_noalloc(dims, cand_k, cand_v, probs, act_k, act_v, symbols, esc_vals, esc_cnt,
                                 esc_off, status, pred_out=None):
    """plc_predict_residual with the library's own static workspace (no ws argument)."""
    rc = lib().plc_predict_residual_noalloc(
        C.byref(dims), _ptr(cand_k, torch.float16), _ptr(cand_v, torch.float16),
        _contig(probs, torch.float32), _ptr(act_k, torch.float16), _ptr(act_v, torch.float16),
        _contig(symbols, torch.uint8), _contig(esc_vals, None), esc_vals.numel(),
        _contig(esc_cnt, torch.int32), _contig(esc_off, torch.int64), _contig(pred_out, torch.float32),
        _contig(status, torch.int32), _stream())
    _check(rc, "plc_predict_residual_noalloc")


def plc_histogram(symbols, n_streams, syms_per_stream, counts):
    rc = lib().plc_histogram(_contig(symbols, torch.uint8), n_streams, syms_per_stream,
                             _contig(counts, torch.int32), _stream())
    _check(rc, "plc_histogram")


def plc_build_freq(counts, n_streams, freq, cum, status):
    rc = lib().plc_build_freq(_contig(counts, torch.int32), n_streams, _contig(freq, torch.int16),
                              _contig(cum, torch.int16), _contig(status, torch.int32), _stream())
    _check(rc, "plc_build_freq")


def plc_rans_encode(symbols, n_streams, syms_per_stream, chunk_syms, freq, states, words, word_off,
                    word_cap_per_unit, n_words, status, restart=None):
    rc = lib().plc_rans_encode_restart(_contig(symbols, torch.uint8), n_streams, syms_per_stream, chunk_syms,
                               _contig(freq, torch.int16), _contig(states, torch.int32),
                               _contig(words, torch.int16), _contig(word_off, torch.int64),
                               int(word_cap_per_unit), _contig(n_words, torch.int32),
                               _restart(restart), _contig(status, torch.int32), _stream())
    _check(rc, "plc_rans_encode")


def plc_rans_decode(freq, states, words, word_off, n_words, n_streams, syms_per_stream, chunk_syms,
                    symbols, status, restart=None):
    rc = lib().plc_rans_decode_restart(_contig(freq, torch.int16), _contig(states, torch.int32),
                               _contig(words, torch.int16), words.numel(),
                               _contig(word_off, torch.int64), _contig(n_words, torch.int32),
                               n_streams, syms_per_stream, chunk_syms, _restart(restart),
                               _contig(symbols, torch.uint8),
                               _contig(status, torch.int32), _stream())
    _check(rc, "plc_rans_decode")


def plc_reconstruct(dims, cand_k, cand_v, probs, symbols, esc_vals, esc_off, out_k, out_v, ws, status):
    rc = lib().plc_reconstruct(
        C.byref(dims), _ptr(cand_k, torch.float16), _ptr(cand_v, torch.float16),
        _contig(probs, torch.float32), _contig(symbols, torch.uint8), _contig(esc_vals, None),
        esc_vals.numel(), _contig(esc_off, torch.int64), _ptr(out_k, torch.float16),
        _ptr(out_v, torch.float16), _contig(ws, torch.uint8), ws.numel(),
        _contig(status, torch.int32), _stream())
    _check(rc, "plc_reconstruct")


def plc_rans_decode_reconstruct(dims, freq, states, words, word_off, n_words, chunk_syms, cand_k, cand_v, probs,
                                esc_vals, esc_off, symbols, out_k, out_v, ws, status, restart=None):
    rc = lib().plc_rans_decode_reconstruct_restart(
        C.byref(dims), _contig(freq, torch.int16), _contig(states, torch.int32), _contig(words, torch.int16),
        words.numel(), _contig(word_off, torch.int64), _contig(n_words, torch.int32), chunk_syms,
        _ptr(cand_k, torch.float16), _ptr(cand_v, torch.float16), _contig(probs, torch.float32),
        _contig(esc_vals, None), esc_vals.numel(), _contig(esc_off, torch.int64), _contig(symbols, torch.uint8),
        _ptr(out_k, torch.float16), _ptr(out_v, torch.float16), _contig(ws, torch.uint8), ws.numel(),
        _restart(restart), _contig(status, torch.int32), _stream())
    _check(rc, "plc_rans_decode_reconstruct")


def plc_rans_decode_reconstruct_cond(dims, freq, states, words, word_off, n_words, chunk_syms, cand_k, cand_v,
                                     probs, chosen, esc_vals, esc_off, symbols, out_k, out_v, ws, status, restart=None):
    rc = lib().plc_rans_decode_reconstruct_cond_restart(
        C.byref(dims), _contig(freq, torch.int16), _contig(states, torch.int32), _contig(words, torch.int16),
        words.numel(), _contig(word_off, torch.int64), _contig(n_words, torch.int32), chunk_syms,
        _ptr(cand_k, torch.float16), _ptr(cand_v, torch.float16), _contig(probs, torch.float32),
        _contig(chosen, torch.int32), _contig(esc_vals, None), esc_vals.numel(), _contig(esc_off, torch.int64),
        _contig(symbols, torch.uint8), _ptr(out_k, torch.float16), _ptr(out_v, torch.float16),
        _contig(ws, torch.uint8), ws.numel(), _restart(restart), _contig(status, torch.int32), _stream())
    _check(rc, "plc_rans_decode_reconstruct_cond")


def plc_predict_residual_cond(dims, cand_k, cand_v, probs, chosen, act_k, act_v, symbols, esc_vals,
                              esc_cnt, esc_off, ws, status, pred_out=None):
    """As plc_predict_residual, with chosen int32 [S,n] (candidate index of the true token, -1 = none)."""
    rc = lib().plc_predict_residual_cond(
        C.byref(dims), _ptr(cand_k, torch.float16), _ptr(cand_v, torch.float16),
        _contig(probs, torch.float32), _contig(chosen, torch.int32), _ptr(act_k, torch.float16),
        _ptr(act_v, torch.float16), _contig(symbols, torch.uint8), _contig(esc_vals, None),
        esc_vals.numel(), _contig(esc_cnt, torch.int32), _contig(esc_off, torch.int64),
        _contig(pred_out, torch.float32), _contig(ws, torch.uint8), ws.numel(),
        _contig(status, torch.int32), _stream())
    _check(rc, "plc_predict_residual_cond")


def plc_reconstruct_cond(dims, cand_k, cand_v, probs, chosen, symbols, esc_vals, esc_off, out_k, out_v,
                         ws, status):
    rc = lib().plc_reconstruct_cond(
        C.byref(dims), _ptr(cand_k, torch.float16), _ptr(cand_v, torch.float16),
        _contig(probs, torch.float32), _contig(chosen, torch.int32), _contig(symbols, torch.uint8),
        _contig(esc_vals, None), esc_vals.numel(), _contig(esc_off, torch.int64),
        _ptr(out_k, torch.float16), _ptr(out_v, torch.float16), _contig(ws, torch.uint8), ws.numel(),
        _contig(status, torch.int32), _stream())
    _check(rc, "plc_reconstruct_cond")


def plc_select_candidate(dims, cand_k, act_k, max_mean_sq, chosen):
    rc = lib().plc_select_candidate(C.byref(dims), _ptr(cand_k, torch.float16), _ptr(act_k, torch.float16),
                                    float(max_mean_sq), _contig(chosen, torch.int32), _stream())
    _check(rc, "plc_select_candidate")


def plc_index_encode(probs, chosen, S, n, k, states, words, word_off, word_cap, n_words, status):
    rc = lib().plc_index_encode(_contig(probs, torch.float32), _contig(chosen, torch.int32), S, n, k,
                                _contig(states, torch.int32), _contig(words, torch.int16),
                                _contig(word_off, torch.int64), int(word_cap),
                                _contig(n_words, torch.int32), _contig(status, torch.int32), _stream())
    _check(rc, "plc_index_encode")


def plc_index_decode(probs, states, words, word_off, n_words, S, n, k, chosen, status):
    rc = lib().plc_index_decode(_contig(probs, torch.float32), _contig(states, torch.int32),
                                _contig(words, torch.int16), words.numel(),
                                _contig(word_off, torch.int64), _contig(n_words, torch.int32), S, n, k,
                                _contig(chosen, torch.int32), _contig(status, torch.int32), _stream())
    _check(rc, "plc_index_decode")


def plc_surprisal_thresholds(b0, hbar, bmax=MAX_BITS):
    """Host call: the bmax + 1 thresholds (entries 0, 1 unused) that plc_surprisal_bits compares with."""
    arr = (C.c_uint16 * (int(bmax) + 1))()
    _check(lib().plc_surprisal_thresholds(float(b0), float(hbar), int(bmax), arr), "plc_surprisal_thresholds")
    return list(arr)


surprisal_thresholds = plc_surprisal_thresholds


def plc_surprisal_bits(probs, chosen, S, n, k, thr, bits, status):
    """thr: host sequence of bmax + 1 integers (see surprisal_thresholds); bits: uint8 [S,n] out."""
    arr = (C.c_uint16 * len(thr))(*[int(t) for t in thr])
    rc = lib().plc_surprisal_bits(_contig(probs, torch.float32), _contig(chosen, torch.int32), S, n, k, arr,
                                  len(thr) - 1, _contig(bits, torch.uint8), _contig(status, torch.int32), _stream())
    _check(rc, "plc_surprisal_bits")


def plc_predict_residual_adapt(dims, cand_k, cand_v, probs, chosen, bits, step_range, act_k, act_v, symbols,
                               esc_vals, esc_cnt, esc_off, ws, status, pred_out=None):
    rc = lib().plc_predict_residual_adapt(
        C.byref(dims), _ptr(cand_k, torch.float16), _ptr(cand_v, torch.float16),
        _contig(probs, torch.float32), _contig(chosen, torch.int32), _contig(bits, torch.uint8),
        float(step_range), _ptr(act_k, torch.float16), _ptr(act_v, torch.float16),
        _contig(symbols, torch.uint8), _contig(esc_vals, None), esc_vals.numel(),
        _contig(esc_cnt, torch.int32), _contig(esc_off, torch.int64), _contig(pred_out, torch.float32),
        _contig(ws, torch.uint8), ws.numel(), _contig(status, torch.int32), _stream())
    _check(rc, "plc_predict_residual_adapt")


def plc_reconstruct_adapt(dims, cand_k, cand_v, probs, chosen, bits, step_range, symbols, esc_vals, esc_off,
                          out_k, out_v, ws, status):
    rc = lib().plc_reconstruct_adapt(
        C.byref(dims), _ptr(cand_k, torch.float16), _ptr(cand_v, torch.float16),
        _contig(probs, torch.float32), _contig(chosen, torch.int32), _contig(bits, torch.uint8),
        float(step_range), _contig(symbols, torch.uint8), _contig(esc_vals, None), esc_vals.numel(),
        _contig(esc_off, torch.int64), _ptr(out_k, torch.float16), _ptr(out_v, torch.float16),
        _contig(ws, torch.uint8), ws.numel(), _contig(status, torch.int32), _stream())
    _check(rc, "plc_reconstruct_adapt")


def plc_histogram_bucketed(symbols, n_streams, syms_per_stream, syms_per_pos, streams_per_session, bits,
                           n_tables, counts, status):
    rc = lib().plc_histogram_bucketed(_contig(symbols, torch.uint8), n_streams, syms_per_stream, syms_per_pos,
                                      streams_per_session, _contig(bits, torch.uint8), n_tables,
                                      _contig(counts, torch.int32), _contig(status, torch.int32), _stream())
    _check(rc, "plc_histogram_bucketed")


def plc_build_freq_bucketed(counts, n_streams, n_tables, freq, status):
    rc = lib().plc_build_freq_bucketed(_contig(counts, torch.int32), n_streams, n_tables,
                                       _contig(freq, torch.int16), _contig(status, torch.int32), _stream())
    _check(rc, "plc_build_freq_bucketed")


def plc_rans_encode_bucketed(symbols, n_streams, syms_per_stream, chunk_syms, syms_per_pos,
                             streams_per_session, bits, n_tables, freq, states, words, word_off,
                             word_cap_per_unit, n_words, status, restart=None):
    rc = lib().plc_rans_encode_bucketed_restart(_contig(symbols, torch.uint8), n_streams, syms_per_stream, chunk_syms,
                                        syms_per_pos, streams_per_session, _contig(bits, torch.uint8), n_tables,
                                        _contig(freq, torch.int16), _contig(states, torch.int32),
                                        _contig(words, torch.int16), _contig(word_off, torch.int64),
                                        int(word_cap_per_unit), _contig(n_words, torch.int32),
                                        _restart(restart), _contig(status, torch.int32), _stream())
    _check(rc, "plc_rans_encode_bucketed")


def plc_rans_decode_bucketed(freq, states, words, word_off, n_words, n_streams, syms_per_stream, chunk_syms,
                             syms_per_pos, streams_per_session, bits, n_tables, symbols, status, restart=None):
    rc = lib().plc_rans_decode_bucketed_restart(_contig(freq, torch.int16), _contig(states, torch.int32),
                                        _contig(words, torch.int16), words.numel(),
                                        _contig(word_off, torch.int64), _contig(n_words, torch.int32),
                                        n_streams, syms_per_stream, chunk_syms, syms_per_pos,
                                        streams_per_session, _contig(bits, torch.uint8), n_tables,
                                        _restart(restart), _contig(symbols, torch.uint8), _contig(status, torch.int32), _stream())
    _check(rc, "plc_rans_decode_bucketed")


def plc_rans_decode_reconstruct_adapt(dims, freq, states, words, word_off, n_words, chunk_syms, n_tables, cand_k,
                                      cand_v, probs, chosen, bits, step_range, esc_vals, esc_off, symbols, out_k,
                                      out_v, ws, status, restart=None):
    rc = lib().plc_rans_decode_reconstruct_adapt_restart(
        C.byref(dims), _contig(freq, torch.int16), _contig(states, torch.int32), _contig(words, torch.int16),
        words.numel(), _contig(word_off, torch.int64), _contig(n_words, torch.int32), chunk_syms, n_tables,
        _ptr(cand_k, torch.float16), _ptr(cand_v, torch.float16), _contig(probs, torch.float32),
        _contig(chosen, torch.int32), _contig(bits, torch.uint8), float(step_range), _contig(esc_vals, None),
        esc_vals.numel(), _contig(esc_off, torch.int64), _contig(symbols, torch.uint8),
        _ptr(out_k, torch.float16), _ptr(out_v, torch.float16), _contig(ws, torch.uint8), ws.numel(),
        _restart(restart), _contig(status, torch.int32), _stream())
    _check(rc, "plc_rans_decode_reconstruct_adapt")


def plc_expected_embedding(probs_full, embed_t, ebar):
    """probs_full fp16 [rows, V], embed_t fp16 [m, V] -> ebar fp16 [rows, m]."""
    rows, V = probs_full.shape
    m = embed_t.shape[0]
    rc = lib().plc_expected_embedding(_contig(probs_full, torch.float16), _contig(embed_t, torch.float16), rows, V,
                                      m, _contig(ebar, torch.float16), _stream())
    _check(rc, "plc_expected_embedding")


def plc_predict_residual_linear(dims, ebar, A, bias_k, bias_v, act_k, act_v, symbols, esc_vals, esc_cnt, esc_off,
                                ws, status):
    m = A.shape[-1]
    rc = lib().plc_predict_residual_linear(
        C.byref(dims), _contig(ebar, torch.float16), m, _contig(A, torch.float16), _ptr(bias_k, torch.float16),
        _ptr(bias_v, torch.float16), _ptr(act_k, torch.float16), _ptr(act_v, torch.float16),
        _contig(symbols, torch.uint8), _contig(esc_vals, None), esc_vals.numel(), _contig(esc_cnt, torch.int32),
        _contig(esc_off, torch.int64), _contig(ws, torch.uint8), ws.numel(), _contig(status, torch.int32), _stream())
    _check(rc, "plc_predict_residual_linear")


def plc_reconstruct_linear(dims, ebar, A, bias_k, bias_v, symbols, esc_vals, esc_off, out_k, out_v, ws, status):
    m = A.shape[-1]
    rc = lib().plc_reconstruct_linear(
        C.byref(dims), _contig(ebar, torch.float16), m, _contig(A, torch.float16), _ptr(bias_k, torch.float16),
        _ptr(bias_v, torch.float16), _contig(symbols, torch.uint8), _contig(esc_vals, None), esc_vals.numel(),
        _contig(esc_off, torch.int64), _ptr(out_k, torch.float16), _ptr(out_v, torch.float16),
        _contig(ws, torch.uint8), ws.numel(), _contig(status, torch.int32), _stream())
    _check(rc, "plc_reconstruct_linear")


def make_pages(k, v, table, lens, refs) -> plc_pages:
    """k, v [P, L, H, B, d] of 16-bit elements (same strides, components contiguous); table int32 [S, M]; lens int32 [S];
    refs int32 [P].  The tensors have to outlive what is made here."""
    if k.dim() != 5 or k.shape != v.shape or k.dtype != v.dtype or k.stride() != v.stride() or k.stride(4) != 1:
        raise ValueError("k and v are [pages, layers, heads, rows, components] of one shape, type and layout")
    if k.dtype not in (torch.float16, torch.bfloat16):
        raise TypeError(f"expected float16 or bfloat16, got {k.dtype}")
    if table.dim() != 2 or lens.shape != table.shape[:1] or refs.shape != k.shape[:1]:
        raise ValueError("table [sessions, entries], lens [sessions], refs [pages]")
    if len({t.device for t in (k, v, table, lens, refs)}) != 1:
        raise ValueError("k, v, table, lens and refs are on one device")
    pages = plc_pages()
    pages.k, pages.v = _ptr(k), _ptr(v)
    pages.stride = (C.c_int64 * 4)(*k.stride()[:4])
    pages.P, pages.L, pages.H, pages.B, pages.d = k.shape
    pages.S, pages.M = table.shape
    pages.table, pages.lens, pages.refs = (_contig(t, torch.int32) for t in (table, lens, refs))
    return pages


def plc_pages_workspace_bytes(pages) -> int:
    return int(lib().plc_pages_workspace_bytes(pages))


# The calls of the paged cache come once or more a token, and last as long as a launch or two: their arguments go over as
# plain addresses, and the stream is asked for directly.
_I64x2 = C.c_int64 * 2
_raw_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
_int32 = torch.int32


def _stream_of(t):
    """The current stream, of the device that launches go to: tensors of another are not for it."""
    device = t.get_device()
    if device != _current_device():
        raise ValueError(f"plc works on the current device, {_current_device()}; the tensors are on {device}")
    return _raw_stream(device)


def _ints(t):
    if t.dtype is _int32 and t.is_cuda and t.is_contiguous():
        return t.data_ptr()
    if t.dtype is not _int32:
        raise TypeError(f"expected {torch.int32}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError("plc takes device tensors")
    raise ValueError("tensor must be contiguous")


def _on_device(t):
    if not t.is_cuda:
        raise ValueError("plc takes device tensors")
    return t.data_ptr()


def plc_pages_fork(pages, src, status):
    """src int32 [S]: what each session becomes; -1: empty."""
    _check(lib().plc_pages_fork(pages, _ints(src), _ints(status), _stream_of(src)), "plc_pages_fork")


def plc_pages_extend(pages, grow, ws, status):
    _check(lib().plc_pages_extend(pages, _ints(grow), _on_device(ws), ws.numel(), _ints(status),
                                  _stream_of(grow)), "plc_pages_extend")


def plc_pages_trim(pages, new_lens, status):
    _check(lib().plc_pages_trim(pages, _ints(new_lens), _ints(status), _stream_of(new_lens)), "plc_pages_trim")


def plc_pages_accept(pages, off, path, path_off, status):
    """off, path_off int32 [S+1]; path int32: numbers of the nodes to keep, ascending in each session."""
    _check(lib().plc_pages_accept(pages, _ints(off), _ints(path), path.numel(), _ints(path_off), _ints(status),
                                  _stream_of(off)), "plc_pages_accept")


def plc_pages_compact(pages, used, ws, status):
    """used int32 [1] out, or None: pages in use."""
    _check(lib().plc_pages_compact(pages, None if used is None else _ints(used), _on_device(ws), ws.numel(), _ints(status),
                                   _stream_of(ws)), "plc_pages_compact")


_rows_known = {}  # descriptions of rows by their layout


def _rows_of(pages, k, v, layer):
    """Rows in a buffer: packed [rows, layers, heads, d], or [S, layers, heads, rows, d], of any strides but the last."""
    st, shape = k.stride(), k.shape
    if shape != v.shape or k.dtype is not v.dtype or st != v.stride():
        raise ValueError("k and v are [rows, layers, heads, d] or [sessions, layers, heads, rows, d] of one layout")
    rows = _rows_known.get((shape, st, layer, k.dtype))
    if rows is None:
        if len(shape) not in (4, 5) or st[-1] != 1:
            raise ValueError("k and v are [rows, layers, heads, d] or [sessions, layers, heads, rows, d] of one layout")
        if k.dtype is not torch.float16 and k.dtype is not torch.bfloat16:
            raise TypeError(f"expected float16 or bfloat16, got {k.dtype}")
        if len(_rows_known) >= 1024:
            _rows_known.clear()
        rows = plc_rows(layer, shape[1], 1, shape[0], (0, st[1], st[2], st[0])) if len(shape) == 4 else \
            plc_rows(layer, shape[1], 0, shape[3], st[:4])
        _rows_known[shape, st, layer, k.dtype] = rows
    if shape[2] != pages.H or shape[-1] != pages.d or (len(shape) == 5 and shape[0] != pages.S):
        raise ValueError("rows have the pool's heads and components, and a part for each of its sessions")
    return rows


def plc_pages_store(pages, off, k, v, layer, status):
    """k, v [rows, layers, H, d] packed, or [S, layers, H, rows, d]; off int32 [S+1]; layer: the first of the pool's."""
    _check(lib().plc_pages_store(pages, _rows_of(pages, k, v, layer), _ints(off), _on_device(k), _on_device(v), _ints(status),
                                 _stream_of(off)), "plc_pages_store")


def plc_pages_load(pages, off, k, v, layer, status):
    """plc_pages_store the other way round."""
    _check(lib().plc_pages_load(pages, _rows_of(pages, k, v, layer), _ints(off), _on_device(k), _on_device(v), _ints(status),
                                _stream_of(off)), "plc_pages_load")


def plc_attend_workspace_bytes(pages, G, N, max_nodes, max_len) -> int:
    return int(lib().plc_attend_workspace_bytes(pages, G, N, max_nodes, max_len))


def plc_attend(pages, layer, q, off, parents, max_nodes, max_len, scale, out, lse, ws, status):
    """q, out [N, H*G, d], components contiguous; parents int32 [N] or None (a chain); lse float32 [N, H*G] or None."""
    shape, qs, os_ = q.shape, q.stride(), out.stride()
    if shape != out.shape or q.dtype is not out.dtype or len(shape) != 3 or qs[2] != 1 or os_[2] != 1:
        raise ValueError("q and out are [nodes, heads, d] of one type, with contiguous components")
    if q.dtype is not torch.float16 and q.dtype is not torch.bfloat16:
        raise TypeError(f"expected float16 or bfloat16, got {q.dtype}")
    if shape[1] % pages.H or shape[2] != pages.d:
        raise ValueError("query heads are a multiple of the cache's, with as many components")
    if lse is not None and (lse.dtype is not torch.float32 or not lse.is_contiguous()):
        raise TypeError("lse is contiguous float32")
    if not (q.is_cuda and out.is_cuda and ws.is_cuda and (lse is None or lse.is_cuda)):
        raise ValueError("plc takes device tensors")
    q_stride = _I64x2(qs[0], qs[1])
    _check(lib().plc_attend(pages, layer, PLC_FP16 if q.dtype is torch.float16 else PLC_BF16, q.data_ptr(), q_stride,
                            shape[1] // pages.H, shape[0], _ints(off), None if parents is None else _ints(parents), max_nodes,
                            max_len, scale, out.data_ptr(), q_stride if os_ == qs else _I64x2(os_[0], os_[1]),
                            None if lse is None else lse.data_ptr(), ws.data_ptr(), ws.numel(), _ints(status),
                            _stream_of(q)), "plc_attend")


# ---- rotary positions, weights of positions, scores of tokens ------------------------------------------------------------

def plc_rotary_frequencies(r, scaling="none", base=10000.0, factor=1.0, low=1.0, high=2.0, trained=1):
    """Radians a position of each of r / 2 pairs: a list.  Host call."""
    if scaling not in ROTARY_SCALINGS:
        raise ValueError(f"scaling is one of {', '.join(ROTARY_SCALINGS)}")
    theta = (C.c_double * max(int(r) // 2, 1))()
    spec = plc_rotary_spec(r, ROTARY_SCALINGS.index(scaling), base, factor, low, high, trained)
    _check(lib().plc_rotary_frequencies(spec, theta), "plc_rotary_frequencies")
    return list(theta)


def plc_rotary_turns(theta):
    """theta: radians a position, any numbers.  Their turns, in 2^-64: a list of whole numbers.  Host call."""
    theta = (C.c_double * len(theta))(*theta)
    turns = (C.c_uint64 * len(theta))()
    _check(lib().plc_rotary_turns(theta, len(theta), turns), "plc_rotary_turns")
    return list(turns)


def make_rotary(turns, interleaved, magnitude) -> plc_rotary:
    """turns: int64 [r / 2], the bits of plc_rotary_turns; it has to outlive what is made here."""
    return plc_rotary(_contig(turns, torch.int64), 2 * turns.numel(), 1 if interleaved else 0, magnitude)


def _on(device, *tensors):
    """All of them (None aside) on the device that launches go to."""
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError(f"plc works on the current device, {device}; a tensor is on {t.device}")


def _floats(t):
    if t is None:
        return None
    if t.dtype is not torch.float32 or not t.is_contiguous():
        raise TypeError("expected contiguous float32")
    return t.data_ptr()


def _ints_or_none(t):
    return None if t is None else _ints(t)


def _type16(t):
    if t.dtype is torch.float16:
        return PLC_FP16
    if t.dtype is torch.bfloat16:
        return PLC_BF16
    raise TypeError(f"expected float16 or bfloat16, got {t.dtype}")


def _rows_in_and_out(x, out):
    """[rows, heads, d] twice, of one type and shape: the strides of row and head of each."""
    shape, xs, os_ = x.shape, x.stride(), out.stride()
    if len(shape) != 3 or shape != out.shape or x.dtype is not out.dtype or xs[2] != 1 or os_[2] != 1:
        raise ValueError("rows in and out are [rows, heads, d] of one type, with contiguous components")
    return _I64x2(xs[0], xs[1]), _I64x2(os_[0], os_[1])


def plc_rotate(rotary, x, positions, inverse, out):
    """x, out [rows, heads, d], components contiguous; positions int32 [rows].  out may be x."""
    stream = _stream_of(x)
    _on(x.get_device(), positions, out)
    x_stride, out_stride = _rows_in_and_out(x, out)
    if positions.dim() != 1 or positions.shape[0] != x.shape[0]:
        raise ValueError("positions are int32 [rows]")
    _check(lib().plc_rotate(rotary, _type16(x), x.data_ptr(), x_stride, x.shape[0], x.shape[1], x.shape[2], _ints(positions),
                            1 if inverse else 0, out.data_ptr(), out_stride, stream), "plc_rotate")


def plc_rotate_store(pages, rotary, off, base, rel, k, v, layer, q, q_out, status):
    """k, v as for plc_pages_store; base int32 [S] or None; rel int32, one for each row of k (packed [rows], else [S, rows]), or
    None; q, q_out [rows, H*G, d] or None (packed rows only)."""
    stream = _stream_of(off)
    _on(off.get_device(), base, rel, k, v, q, q_out, status)
    rows = _rows_of(pages, k, v, layer)
    if base is not None and (base.dim() != 1 or base.shape[0] != pages.S):
        raise ValueError("base is int32 [sessions]")
    if rel is not None and tuple(rel.shape) != ((k.shape[0],) if rows.packed else (k.shape[0], k.shape[3])):
        raise ValueError("rel has a number for each row")
    q_stride = out_stride = None
    G = 1
    if q is not None:
        q_stride, out_stride = _rows_in_and_out(q, q_out)
        if q.dtype is not k.dtype or q.shape[0] != k.shape[0] or q.shape[1] % pages.H or q.shape[2] != pages.d or not rows.packed:
            raise ValueError("q is [rows, heads, d], packed like k and of its type, its heads a multiple of the cache's")
        G = q.shape[1] // pages.H
    _check(lib().plc_rotate_store(pages, rows, rotary, _type16(k), _ints(off), _ints_or_none(base), _ints_or_none(rel), k.data_ptr(),
                                  v.data_ptr(), None if q is None else q.data_ptr(), q_stride, G,
                                  None if q is None else q_out.data_ptr(), out_stride, _ints(status), stream), "plc_rotate_store")


def make_weights(pages, w) -> plc_weights:
    """w float32 [S, L, H, width]; it has to outlive what is made here."""
    if w.dim() != 4 or w.dtype is not torch.float32 or tuple(w.shape[:3]) != (pages.S, pages.L, pages.H) or w.stride(3) != 1:
        raise ValueError("weights are float32 [sessions, layers, heads, positions] of the cache, positions contiguous")
    return plc_weights(_ptr(w, torch.float32), w.stride()[:3], w.shape[3])


def plc_attend_weights(pages, layer, q, off, max_nodes, max_len, scale, lse, decay, weights, status):
    """q [N, H*G, d], components contiguous; lse float32 [N, H*G]; weights: make_weights."""
    stream = _stream_of(q)
    _on(q.get_device(), off, lse, status)
    shape, qs = q.shape, q.stride()
    if len(shape) != 3 or qs[2] != 1 or shape[1] % pages.H or shape[2] != pages.d:
        raise ValueError("q is [nodes, heads, d], its heads a multiple of the cache's, with contiguous components")
    if lse.shape != shape[:2]:
        raise ValueError("lse is [nodes, heads]")
    _check(lib().plc_attend_weights(pages, layer, _type16(q), q.data_ptr(), _I64x2(qs[0], qs[1]), shape[1] // pages.H, shape[0],
                                    _ints(off), max_nodes, max_len, scale, _floats(lse), decay, weights, _ints(status), stream),
           "plc_attend_weights")


def plc_pages_evict(pages, keep, first, last, weights, kept, max_len, ws, status):
    """keep int32 [S]; weights: make_weights; kept int32 [S, L, H, W] out."""
    stream = _stream_of(keep)
    _on(keep.get_device(), kept, ws, status)
    if kept.dim() != 4 or tuple(kept.shape[:3]) != (pages.S, pages.L, pages.H):
        raise ValueError("kept is int32 [sessions, layers, heads, numbers]")
    _check(lib().plc_pages_evict(pages, _ints(keep), first, last, weights, _ints(kept), kept.shape[3], max_len, _on_device(ws),
                                 ws.numel(), _ints(status), stream), "plc_pages_evict")


def plc_score_workspace_bytes(V, k) -> int:
    return int(lib().plc_score_workspace_bytes(V, k))


_LOGIT_TYPES = {torch.float16: PLC_FP16, torch.bfloat16: PLC_BF16, torch.float32: PLC_FP32}


def plc_score_tokens(logits, scale, tokens, k, logprob, entropy, lse, ids, top_logprobs, probs, chosen, ws, status):
    """logits [N, V], the tokens contiguous; tokens int32 [N] or None; out, or None: logprob, entropy, lse float32 [N], ids int32 and
    top_logprobs, probs float32 [N, k], chosen int32 [N]."""
    _on(_current_device(), logits, tokens, logprob, entropy, lse, ids, top_logprobs, probs, chosen, ws, status)
    N = logits.shape[0]
    for t, n in ((logprob, N), (entropy, N), (lse, N), (chosen, N), (ids, N * k), (top_logprobs, N * k), (probs, N * k)):
        if t is not None and t.numel() != n:
            raise ValueError("a result does not have a place for each row (and alternative)")
    _score_tokens(logits, scale, tokens, k, *(_floats(t) for t in (logprob, entropy, lse)), _ints_or_none(ids), _floats(top_logprobs),
                  _floats(probs), _ints_or_none(chosen), _on_device(ws), ws.numel(), _ints(status))


def _score_tokens(logits, scale, tokens, k, *results):
    """The same with the results' addresses, the workspace's, its size and the status'."""
    stream = _stream_of(logits)
    if logits.dim() != 2 or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError("logits are [rows, tokens], the tokens contiguous")
    kind = _LOGIT_TYPES.get(logits.dtype)
    if kind is None:
        raise TypeError(f"expected float16, bfloat16 or float32, got {logits.dtype}")
    N, V = logits.shape
    if tokens is not None:
        _on(logits.get_device(), tokens)
        if tokens.numel() != N:
            raise ValueError("tokens has a number for each row")
        tokens = _ints(tokens)
    _check(lib().plc_score_tokens(kind, logits.data_ptr(), logits.stride(0), N, V, scale, tokens, k, *results, stream), "plc_score_tokens")


class PrefixTrie:
    """Host-side prefix index (plc_trie_*): insert / best_match / evict over token sequences (numpy int32
    arrays; `bits` = per-token surprisal, float32, optional)."""

    def __init__(self, max_bits=float("inf")):
        import numpy as np
        self._np = np
        self._t = lib().plc_trie_create(float(min(max_bits, 1e300)))
        if not self._t:
            raise PlcError(PLC_ERR_INVALID, "plc_trie_create")

    def close(self):
        if getattr(self, "_t", None):
            lib().plc_trie_destroy(self._t)
            self._t = None

    def __del__(self):
        try:
            self.close()
        except Exception:           # interpreter shutdown: the module globals may be gone already
            pass

    def __len__(self):
        return int(lib().plc_trie_size(self._t))

    @property
    def nodes(self):
        return int(lib().plc_trie_nodes(self._t))

    def _arr(self, a, dtype):
        a = self._np.ascontiguousarray(a, dtype=dtype)
        return a, a.ctypes.data_as(C.c_void_p)

    def insert(self, tokens, ident, bits=None):
        """Returns the number of tokens kept (the path is cut where its surprisal sum would exceed max_bits)."""
        tok, tp = self._arr(tokens, self._np.int32)
        bp = None
        if bits is not None:
            b, bp = self._arr(bits, self._np.float32)
            assert b.size == tok.size
        kept = C.c_int64(0)
        _check(lib().plc_trie_insert(self._t, tp, bp, tok.size, int(ident), C.byref(kept)), "plc_trie_insert")
        return int(kept.value)

    def best_match(self, tokens):
        """(id, lcp, dist): a stored prefix with the longest common prefix with the query (-1 if empty)."""
        tok, tp = self._arr(tokens, self._np.int32)
        ident, lcp, dist = C.c_int64(0), C.c_int64(0), C.c_double(0.0)
        _check(lib().plc_trie_best_match(self._t, tp, tok.size, C.byref(ident), C.byref(lcp), C.byref(dist)),
               "plc_trie_best_match")
        return int(ident.value), int(lcp.value), float(dist.value)

    def evict(self, ident):
        _check(lib().plc_trie_evict(self._t, int(ident)), "plc_trie_evict")


def plc_trace_kernel_events(kernel_id, start=None, stop=None):
    """start/stop: raw hipEvent_t handles (ints) or None to clear."""
    rc = lib().plc_trace_kernel_events(int(kernel_id), C.c_void_p(start) if start else None,
                                       C.c_void_p(stop) if stop else None)
    _check(rc, "plc_trace_kernel_events")


def plc_trace_kernel_name(kernel_id) -> str:
    """Kernel that the last call under trace events launched between them (the entropy coder's two)."""
    return lib().plc_trace_kernel_name(int(kernel_id)).decode()

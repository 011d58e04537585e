"""ctypes binding of libw2v.so: one Python function per C entry point, same names,
argument marshalling only.  Torch provides device memory and streams; every step of
the method runs in the library's kernels.  There is no fallback: if the library is
missing or cannot be built, loading raises.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np
import torch

from . import build as _build

W2V_OK = 0
W2V_ERR_ARG, W2V_ERR_STATE, W2V_ERR_NOMEM, W2V_ERR_CUDA = -1, -2, -3, -4
W2V_ERR_TOKEN_RANGE, W2V_ERR_CAPACITY = -5, -6
MODE_SNAPSHOT, MODE_HOGWILD = 0, 1
TABLE_U, TABLE_V = 0, 1
MAX_SHARDS = 16                  # most column shards (and epoch words per barrier array)

EXPORTS = (
    "w2v_create", "w2v_create_strided", "w2v_create_shard", "w2v_shard_dots", "w2v_shard_adjust",
    "w2v_get_row_stride", "w2v_set_interleave", "w2v_cbow_step", "w2v_cbow_step_host", "w2v_sample_cbow",
    "w2v_topk_cosine", "w2v_set_retrieval_kernel", "w2v_destroy", "w2v_build_alias", "w2v_get_tables", "w2v_sgns_step",
    "w2v_sgns_step_host", "w2v_sample_pairs", "w2v_partial_dots", "w2v_read_rows", "w2v_write_rows",
    "w2v_set_step", "w2v_get_step", "w2v_get_table_ptrs", "w2v_sync", "w2v_profile_enable",
    "w2v_profile_read", "w2v_get_launch_count", "w2v_set_tuning", "w2v_last_error",
    "w2v_sample_pairs_noalloc", "w2v_peer_barrier", "w2v_probe_rows",
    "w2v_selftest_bounded_wait", "w2v_probe_bulk_ring", "w2v_probe_mma_ring",
    "w2v_layer_norm", "w2v_layer_norm_backward", "w2v_sentence_spans", "w2v_bucket_starts", "w2v_attend",
    "w2v_attend_backward", "w2v_attend_token", "w2v_fourbit_pack", "w2v_fourbit_scores",
)


class StepStats(C.Structure):
    _fields_ = [("tokens", C.c_uint64), ("kept", C.c_uint64), ("centres", C.c_uint64),
                ("pairs", C.c_uint64), ("neg_draws", C.c_uint64), ("neg_redraws", C.c_uint64),
                ("oov", C.c_uint64), ("status", C.c_uint32), ("reserved", C.c_uint32)]

    def as_dict(self):
        return {k: int(getattr(self, k)) for k, _ in self._fields_ if k != "reserved"}


class Window(C.Structure):
    """w2v_window: what an attention call sees and how it is laid out."""
    _fields_ = [("type", C.c_uint32), ("heads", C.c_uint32), ("kv_heads", C.c_uint32), ("head_dim", C.c_uint32),
                ("left", C.c_uint32), ("right", C.c_uint32), ("sinks", C.c_uint32), ("buckets", C.c_uint32),
                ("reach", C.c_uint32), ("two_sided", C.c_uint32), ("scale", C.c_float)]


class W2VError(RuntimeError):
    def __init__(self, code, text):
        super().__init__(f"libw2v error {code}: {text}")
        self.code = code


_lib = None


def library_path() -> str:
    return _build.LIB


def load():
    """Load libw2v.so (building it first if the sources are newer and nvcc is here)."""
    global _lib
    if _lib is not None:
        return _lib
    try:
        _build.build()
    except Exception as exc:                     # no nvcc on this machine: use the shipped binary
        if not os.path.exists(_build.LIB):
            raise RuntimeError(f"libw2v.so is missing and could not be built: {exc}") from exc
    L = C.CDLL(_build.LIB)
    vp, u32, u64, i32 = C.c_void_p, C.c_uint32, C.c_uint64, C.c_int32
    sig = {
        "w2v_create": [u64, u32, u64, vp, vp, vp, C.POINTER(vp)],
        "w2v_create_strided": [u64, u32, u32, u64, vp, vp, vp, C.POINTER(vp)],
        "w2v_get_row_stride": [vp, C.POINTER(u32)],
        "w2v_create_shard": [u64, u32, u32, u32, u32, u64, vp, vp, vp, C.POINTER(vp)],
        "w2v_shard_dots": [vp, vp, u64, u32, u32, C.POINTER(vp), u32, u64, C.POINTER(StepStats)],
        "w2v_shard_adjust": [vp, vp, C.c_float],
        "w2v_peer_barrier": [vp, C.POINTER(vp), u32, u32, u32, u32],
        "w2v_probe_rows": [vp, u32, u64, u64, C.POINTER(C.c_double), C.POINTER(u64)],
        "w2v_selftest_bounded_wait": [vp, u32],
        "w2v_probe_bulk_ring": [vp, u32, u32, u32, u64, C.POINTER(C.c_double), C.POINTER(u64)],
        "w2v_probe_mma_ring": [vp, u32, u32, u32, u32, C.POINTER(C.c_double), C.POINTER(C.c_double)],
        "w2v_destroy": [vp],
        "w2v_build_alias": [vp, vp, C.c_double],
        "w2v_get_tables": [vp, vp, vp, vp],
        "w2v_sgns_step": [vp, vp, u64, u32, u32, C.c_float, u32, C.POINTER(StepStats)],
        "w2v_sgns_step_host": [vp, vp, u64, u32, u32, C.c_float, u32, C.POINTER(StepStats)],
        "w2v_cbow_step": [vp, vp, u64, u32, u32, C.c_float, u32, C.POINTER(StepStats)],
        "w2v_cbow_step_host": [vp, vp, u64, u32, u32, C.c_float, u32, C.POINTER(StepStats)],
        "w2v_sample_cbow": [vp, vp, u64, u32, u32, vp, vp, u64, C.POINTER(u64), C.POINTER(StepStats)],
        "w2v_sample_pairs": [vp, vp, u64, u32, u32, vp, vp, vp, u64, C.POINTER(u64), C.POINTER(StepStats)],
        "w2v_sample_pairs_noalloc": [vp, vp, u64, u32, u32, vp, vp, vp, u64, C.POINTER(u64), C.POINTER(StepStats)],
        "w2v_partial_dots": [vp, vp, u64, u32, u32, vp],
        "w2v_read_rows": [vp, u32, vp, u64, vp],
        "w2v_write_rows": [vp, u32, vp, u64, vp],
        "w2v_topk_cosine": [vp, u32, vp, u64, u64, u64, u32, C.c_float, vp, vp],
        "w2v_set_retrieval_kernel": [vp, u32],
        "w2v_layer_norm": [vp, u64, u32, vp, u64, u32, vp, vp, C.c_float, vp, u64, u32, vp, vp],
        "w2v_layer_norm_backward": [vp, u64, u32, vp, u64, u32, vp, u64, u32, vp, vp, vp, vp, u64, vp, vp],
        "w2v_sentence_spans": [vp, vp, u64, vp],
        "w2v_bucket_starts": [u32, u32, u32, vp],
        "w2v_attend": [vp, C.POINTER(Window), u64, vp, vp, u64, vp, u64, vp, u64, vp, vp, u64, vp],
        "w2v_attend_backward": [vp, C.POINTER(Window), u64, vp, vp, u64, vp, u64, vp, u64, vp, vp, u64, vp,
                                vp, u64, vp, u64, vp, u64, vp, u64, vp],
        "w2v_attend_token": [vp, C.POINTER(Window), u32, vp, vp, vp, vp, vp, vp, u64, vp, vp],
        "w2v_fourbit_pack": [vp, vp, u64, u32, u64, u32, vp, vp],
        "w2v_fourbit_scores": [vp, vp, u32, u64, vp, vp, u64, u32, u32, vp, u64],
        "w2v_set_step": [vp, u64],
        "w2v_set_interleave": [vp, u32, u32],
        "w2v_get_step": [vp, C.POINTER(u64)],
        "w2v_get_table_ptrs": [vp, C.POINTER(vp), C.POINTER(vp)],
        "w2v_sync": [vp],
        "w2v_profile_enable": [vp, i32],
        "w2v_profile_read": [vp, C.POINTER(C.c_double), C.POINTER(u64)],
        "w2v_get_launch_count": [vp, C.POINTER(u64)],
        "w2v_set_tuning": [vp, u32, u32],
        "w2v_last_error": [vp],
    }
    for name, argtypes in sig.items():
        fn = getattr(L, name)
        fn.argtypes = argtypes
        fn.restype = C.c_char_p if name == "w2v_last_error" else i32
    _lib = L
    return L


def _check(h, rc, allow=()):
    if rc != W2V_OK and rc not in allow:
        text = load().w2v_last_error(h)
        raise W2VError(rc, text.decode() if text else "?")
    return rc


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, torch.Tensor):
        assert t.is_contiguous()
        return t.data_ptr()
    if isinstance(t, np.ndarray):
        assert t.flags["C_CONTIGUOUS"]
        return t.ctypes.data
    return int(t)


# ---- one function per C entry point ---------------------------------------------------
def w2v_create(vocab, d, seed, U, V, stream):
    h = C.c_void_p()
    rc = load().w2v_create(int(vocab), int(d), int(seed), _ptr(U), _ptr(V), stream, C.byref(h))
    if rc != W2V_OK:
        raise W2VError(rc, "w2v_create rejected its arguments or could not allocate")
    return h


def w2v_create_strided(vocab, d, row_stride, seed, U, V, stream):
    h = C.c_void_p()
    rc = load().w2v_create_strided(int(vocab), int(d), int(row_stride), int(seed), _ptr(U), _ptr(V), stream,
                                   C.byref(h))
    if rc != W2V_OK:
        raise W2VError(rc, "w2v_create_strided rejected its arguments or could not allocate")
    return h


def w2v_create_shard(vocab, d_full, col_lo, col_hi, row_stride, seed, U, V, stream):
    h = C.c_void_p()
    rc = load().w2v_create_shard(int(vocab), int(d_full), int(col_lo), int(col_hi), int(row_stride), int(seed),
                                 _ptr(U), _ptr(V), stream, C.byref(h))
    if rc != W2V_OK:
        raise W2VError(rc, "w2v_create_shard rejected its arguments or could not allocate")
    return h


def w2v_shard_dots(h, tokens, n, window, negatives, F_peers, cap, stats=None, allow=()):
    """F_peers: device pointers (ints or tensors), one array of `cap` floats per shard."""
    ptrs = (C.c_void_p * len(F_peers))(*[_ptr(f) for f in F_peers])
    ref = C.byref(stats) if stats is not None else None
    return _check(h, load().w2v_shard_dots(h, _ptr(tokens), int(n), window, negatives, ptrs, len(F_peers),
                                           int(cap), ref), allow)


def w2v_shard_adjust(h, F, lr):
    return _check(h, load().w2v_shard_adjust(h, _ptr(F), float(lr)))


def w2v_peer_barrier(h, flags_peers, rank, epoch, timeout_ms):
    """flags_peers: device pointers (ints or tensors), one array of len(flags_peers) uint32 per shard."""
    ptrs = (C.c_void_p * len(flags_peers))(*[_ptr(f) for f in flags_peers])
    return _check(h, load().w2v_peer_barrier(h, ptrs, len(flags_peers), int(rank), int(epoch), int(timeout_ms)))


PROBE_GATHER, PROBE_GATHER_RED, PROBE_GATHER_ALIAS, PROBE_GATHER_RED_ALIAS, PROBE_TOUCH_RED = range(5)


def w2v_probe_rows(h, access, span_rows, rows):
    """(milliseconds, rows touched) of one probe launch."""
    ms, done = C.c_double(0.0), C.c_uint64(0)
    _check(h, load().w2v_probe_rows(h, int(access), int(span_rows), int(rows), C.byref(ms), C.byref(done)))
    return ms.value, int(done.value)


def w2v_probe_bulk_ring(h, stage_bytes, stages, producers, bytes_per_sm):
    """(milliseconds, bytes copied per SM) of one launch of the bulk-copy ring probe."""
    ms, done = C.c_double(0.0), C.c_uint64(0)
    _check(h, load().w2v_probe_bulk_ring(h, int(stage_bytes), int(stages), int(producers), int(bytes_per_sm),
                                         C.byref(ms), C.byref(done)))
    return ms.value, int(done.value)


def w2v_probe_mma_ring(h, kblocks_per_stage, stages, tiles, span_tiles):
    """(SM cycles per tile, cycles of them spent waiting for data) of the producer / ring / MMA probe."""
    cyc, waited = C.c_double(0.0), C.c_double(0.0)
    _check(h, load().w2v_probe_mma_ring(h, int(kblocks_per_stage), int(stages), int(tiles), int(bool(span_tiles)),
                                        C.byref(cyc), C.byref(waited)))
    return cyc.value, waited.value


def w2v_selftest_bounded_wait(h, timeout_ms):
    return _check(h, load().w2v_selftest_bounded_wait(h, int(timeout_ms)))


def w2v_get_row_stride(h):
    s = C.c_uint32(0)
    _check(h, load().w2v_get_row_stride(h, C.byref(s)))
    return int(s.value)


def w2v_destroy(h):
    return load().w2v_destroy(h)


def w2v_build_alias(h, counts, subsample_t):
    counts = np.ascontiguousarray(counts, dtype=np.uint64)
    return _check(h, load().w2v_build_alias(h, counts.ctypes.data, float(subsample_t)))


def w2v_get_tables(h, vocab):
    thr = np.empty(vocab, dtype=np.uint32)
    alias = np.empty(vocab, dtype=np.uint32)
    keep = np.empty(vocab, dtype=np.uint32)
    _check(h, load().w2v_get_tables(h, thr.ctypes.data, alias.ctypes.data, keep.ctypes.data))
    return thr, alias, keep


def w2v_sgns_step(h, tokens, n, window, negatives, lr, mode, stats=None, allow=()):
    ref = C.byref(stats) if stats is not None else None
    return _check(h, load().w2v_sgns_step(h, _ptr(tokens), int(n), window, negatives, float(lr), mode, ref), allow)


def w2v_sgns_step_host(h, tokens_host, n, window, negatives, lr, mode, stats=None, allow=()):
    ref = C.byref(stats) if stats is not None else None
    return _check(h, load().w2v_sgns_step_host(h, _ptr(tokens_host), int(n), window, negatives, float(lr), mode, ref), allow)


def w2v_cbow_step(h, tokens, n, window, negatives, lr, mode, stats=None, allow=()):
    ref = C.byref(stats) if stats is not None else None
    return _check(h, load().w2v_cbow_step(h, _ptr(tokens), int(n), window, negatives, float(lr), mode, ref), allow)


def w2v_cbow_step_host(h, tokens_host, n, window, negatives, lr, mode, stats=None, allow=()):
    ref = C.byref(stats) if stats is not None else None
    return _check(h, load().w2v_cbow_step_host(h, _ptr(tokens_host), int(n), window, negatives, float(lr), mode, ref), allow)


def w2v_sample_cbow(h, tokens, n, window, negatives, centre, negs, cap, stats=None, allow=()):
    nex = C.c_uint64(0)
    ref = C.byref(stats) if stats is not None else None
    rc = _check(h, load().w2v_sample_cbow(h, _ptr(tokens), int(n), window, negatives, _ptr(centre), _ptr(negs),
                                          int(cap), C.byref(nex), ref), allow)
    return rc, int(nex.value)


def w2v_sample_pairs(h, tokens, n, window, negatives, centre, context, negs, cap, stats=None, allow=()):
    npairs = C.c_uint64(0)
    ref = C.byref(stats) if stats is not None else None
    rc = _check(h, load().w2v_sample_pairs(h, _ptr(tokens), int(n), window, negatives, _ptr(centre), _ptr(context),
                                           _ptr(negs), int(cap), C.byref(npairs), ref), allow)
    return rc, int(npairs.value)


def w2v_sample_pairs_noalloc(h, tokens, n, window, negatives, centre, context, negs, cap, stats=None, allow=()):
    """w2v_sample_pairs on the library's fixed scratch: no device allocation, at most 65536 tokens."""
    npairs = C.c_uint64(0)
    ref = C.byref(stats) if stats is not None else None
    rc = _check(h, load().w2v_sample_pairs_noalloc(h, _ptr(tokens), int(n), window, negatives, _ptr(centre),
                                                   _ptr(context), _ptr(negs), int(cap), C.byref(npairs), ref), allow)
    return rc, int(npairs.value)


def w2v_partial_dots(h, pairs, m, col_lo, col_hi, out):
    return _check(h, load().w2v_partial_dots(h, _ptr(pairs), int(m), col_lo, col_hi, _ptr(out)))


def w2v_read_rows(h, which, ids, m, out):
    return _check(h, load().w2v_read_rows(h, which, _ptr(ids), int(m), _ptr(out)))


def w2v_write_rows(h, which, ids, m, rows):
    return _check(h, load().w2v_write_rows(h, which, _ptr(ids), int(m), _ptr(rows)))


def w2v_topk_cosine(h, which, queries, m, cand_lo, cand_hi, K, tau, out_ids, out_cos):
    return _check(h, load().w2v_topk_cosine(h, int(which), _ptr(queries), int(m), int(cand_lo), int(cand_hi), int(K),
                                            float(tau), _ptr(out_ids), _ptr(out_cos)))


def w2v_set_retrieval_kernel(h, kind):
    return _check(h, load().w2v_set_retrieval_kernel(h, int(kind)))


# The reader operators take device addresses (`data_ptr()`), since rows may be strided views.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)           # the current stream of a device, without an object for it
TYPE_F32, TYPE_BF16, TYPE_F16 = 0, 1, 2
_TYPES = {torch.float32: TYPE_F32, torch.bfloat16: TYPE_BF16, torch.float16: TYPE_F16}


def w2v_layer_norm(h, rows, d, x, x_stride, x_type, gamma, beta, eps, y, y_stride, y_type, mean, rstd):
    return _check(h, (_lib or load()).w2v_layer_norm(h, rows, d, x, x_stride, x_type, gamma, beta, eps, y, y_stride, y_type, mean, rstd))


def w2v_layer_norm_backward(h, rows, d, dy, dy_stride, y_type, x, x_stride, x_type, gamma, mean, rstd, dx, dx_stride,
                            dgamma, dbeta):
    return _check(h, (_lib or load()).w2v_layer_norm_backward(h, rows, d, dy, dy_stride, y_type, x, x_stride, x_type, gamma, mean, rstd,
                                                    dx, dx_stride, dgamma, dbeta))


def w2v_sentence_spans(h, tokens, n, spans):
    return _check(h, (_lib or load()).w2v_sentence_spans(h, tokens, n, spans))


def w2v_bucket_starts(buckets, reach, two_sided):
    """First distance of each bucket of one side (int32 numpy array)."""
    starts = np.empty(max(1, buckets // 2 if two_sided else buckets), dtype=np.int32)
    rc = load().w2v_bucket_starts(buckets, reach, int(two_sided), starts.ctypes.data)
    if rc != W2V_OK:
        raise W2VError(rc, "buckets must be in 2..64 (two-sided: even, at least 4), reach above half of a side's and at most 1024")
    return starts


def w2v_attend(h, window, n, spans, q, q_stride, k, k_stride, v, v_stride, bias, o, o_stride, lse):
    return _check(h, (_lib or load()).w2v_attend(h, window, n, spans, q, q_stride, k, k_stride, v, v_stride, bias, o, o_stride, lse))


def w2v_attend_backward(h, window, n, spans, q, q_stride, k, k_stride, v, v_stride, bias, o, o_stride, lse,
                        d_o, do_stride, dq, dq_stride, dk, dk_stride, dv, dv_stride, dbias):
    return _check(h, (_lib or load()).w2v_attend_backward(h, window, n, spans, q, q_stride, k, k_stride, v, v_stride, bias, o, o_stride,
                                                lse, d_o, do_stride, dq, dq_stride, dk, dk_stride, dv, dv_stride, dbias))


def w2v_attend_token(h, window, batch, pos, q, k, v, cache_k, cache_v, places, bias, o):
    return _check(h, (_lib or load()).w2v_attend_token(h, window, batch, pos, q, k, v, cache_k, cache_v, places, bias, o))


def w2v_fourbit_pack(h, rows, n, d, row_stride, group, packed, scales):
    return _check(h, (_lib or load()).w2v_fourbit_pack(h, rows, n, d, row_stride, group, packed, scales))


def w2v_fourbit_scores(h, x, m, x_stride, packed, scales, rows, d, group, out, out_stride):
    return _check(h, (_lib or load()).w2v_fourbit_scores(h, x, m, x_stride, packed, scales, rows, d, group, out, out_stride))


def w2v_set_step(h, step_id):
    return _check(h, load().w2v_set_step(h, int(step_id)))


def w2v_set_interleave(h, phase, stride):
    return _check(h, load().w2v_set_interleave(h, int(phase), int(stride)))


def w2v_get_step(h):
    s = C.c_uint64(0)
    _check(h, load().w2v_get_step(h, C.byref(s)))
    return int(s.value)


def w2v_sync(h):
    return _check(h, load().w2v_sync(h))


def w2v_profile_enable(h, on):
    return _check(h, load().w2v_profile_enable(h, 1 if on else 0))


def w2v_profile_read(h):
    ms, k = C.c_double(0.0), C.c_uint64(0)
    _check(h, load().w2v_profile_read(h, C.byref(ms), C.byref(k)))
    return ms.value, int(k.value)


def w2v_get_launch_count(h):
    k = C.c_uint64(0)
    _check(h, load().w2v_get_launch_count(h, C.byref(k)))
    return int(k.value)


def w2v_set_tuning(h, rows_in_flight, blocks_per_sm):
    return _check(h, load().w2v_set_tuning(h, int(rows_in_flight), int(blocks_per_sm)))


def aligned_row_stride(d):
    """Smallest row stride (in floats) >= d that puts every row on a 128-byte boundary, the
    granularity at which the GPU's L2 cache fetches and writes back: a gathered row then moves
    no bytes of its neighbours."""
    return (int(d) + 31) // 32 * 32


# ---- convenience wrapper: owns the torch tensors the handle points at ----------------------
class W2V:
    """Tables U and V as torch tensors on one GPU plus the library handle."""

    def __init__(self, vocab, d, seed, device="cuda:0", row_stride=None, columns=None):
        """columns=(col_lo, col_hi) makes this model one column shard of vectors with d columns;
        its own d is then the slice width."""
        load()
        if not torch.cuda.is_available():
            raise RuntimeError("libw2v needs a CUDA device; there is no CPU path")
        self.device = torch.device(device)
        self.vocab, self.seed = int(vocab), int(seed)
        self.d_full = int(d)
        self.col_lo, self.col_hi = (0, self.d_full) if columns is None else (int(columns[0]), int(columns[1]))
        self.d = self.col_hi - self.col_lo
        self.row_stride = self.d if row_stride is None else int(row_stride)
        with torch.cuda.device(self.device):
            self.U = torch.empty(self.vocab * self.row_stride, dtype=torch.float32, device=self.device)
            self.V = torch.empty(self.vocab * self.row_stride, dtype=torch.float32, device=self.device)
            self._index = self.U.get_device()
            self._windows = {}
            self.stream = torch.cuda.current_stream(self.device)
            self.h = w2v_create_shard(self.vocab, self.d_full, self.col_lo, self.col_hi, self.row_stride,
                                      self.seed, self.U, self.V, self.stream.cuda_stream)
            self._raw = self.stream.cuda_stream

    def close(self):
        if getattr(self, "h", None):
            w2v_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def build_alias(self, counts, subsample_t):
        assert len(counts) == self.vocab
        w2v_build_alias(self.h, counts, subsample_t)

    def tables(self):
        return w2v_get_tables(self.h, self.vocab)

    def _dev_tokens(self, tokens):
        if isinstance(tokens, torch.Tensor):
            return tokens.to(device=self.device, dtype=torch.int32).contiguous()
        return torch.from_numpy(np.ascontiguousarray(tokens, dtype=np.int32)).to(self.device)

    def sgns_step(self, tokens, window, negatives, lr, mode, want_stats=True, allow=()):
        t = self._dev_tokens(tokens)
        st = StepStats() if want_stats else None
        w2v_sgns_step(self.h, t, t.numel(), window, negatives, lr, mode, st, allow)
        return st.as_dict() if want_stats else None

    def sgns_step_host(self, tokens_host, window, negatives, lr, mode, want_stats=True, allow=()):
        n = tokens_host.numel() if isinstance(tokens_host, torch.Tensor) else len(tokens_host)
        st = StepStats() if want_stats else None
        w2v_sgns_step_host(self.h, tokens_host, n, window, negatives, lr, mode, st, allow)
        return st.as_dict() if want_stats else None

    def cbow_step(self, tokens, window, negatives, lr, mode, want_stats=True, allow=()):
        t = self._dev_tokens(tokens)
        st = StepStats() if want_stats else None
        w2v_cbow_step(self.h, t, t.numel(), window, negatives, lr, mode, st, allow)
        return st.as_dict() if want_stats else None

    def sample_cbow(self, tokens, window, negatives, cap=None, allow=()):
        """(centre[E], negs[E, N], counters) of the examples the next cbow_step would use."""
        t = self._dev_tokens(tokens)
        n = t.numel()
        if cap is None:
            cap = max(1, n)
        centre = torch.empty(cap, dtype=torch.int32, device=self.device)
        negs = torch.empty(cap * negatives, dtype=torch.int32, device=self.device)
        st = StepStats()
        rc, E = w2v_sample_cbow(self.h, t, n, window, negatives, centre, negs, cap, st, allow)
        m = min(E, cap)
        return centre[:m].cpu().numpy(), negs[: m * negatives].view(m, negatives).cpu().numpy(), st.as_dict()

    def sample_pairs(self, tokens, window, negatives, cap=None, allow=()):
        t = self._dev_tokens(tokens)
        n = t.numel()
        if cap is None:
            cap = max(1, n * 2 * window)
        centre = torch.empty(cap, dtype=torch.int32, device=self.device)
        context = torch.empty(cap, dtype=torch.int32, device=self.device)
        negs = torch.empty(cap * negatives, dtype=torch.int32, device=self.device)
        st = StepStats()
        rc, P = w2v_sample_pairs(self.h, t, n, window, negatives, centre, context, negs, cap, st, allow)
        m = min(P, cap)
        return (centre[:m].cpu().numpy(), context[:m].cpu().numpy(),
                negs[: m * negatives].view(m, negatives).cpu().numpy(), st.as_dict(), rc, P)

    def partial_dots(self, pairs, col_lo, col_hi):
        p = torch.as_tensor(np.ascontiguousarray(pairs, dtype=np.int32)).reshape(-1, 2).to(self.device)
        out = torch.empty(p.shape[0], dtype=torch.float32, device=self.device)
        w2v_partial_dots(self.h, p, p.shape[0], col_lo, col_hi, out)
        return out.cpu().numpy()

    def read_rows(self, which, ids):
        i = torch.as_tensor(np.ascontiguousarray(ids, dtype=np.int64)).to(self.device)
        out = torch.zeros(i.numel() * self.d, dtype=torch.float32, device=self.device)
        w2v_read_rows(self.h, which, i, i.numel(), out)
        return out.view(i.numel(), self.d).cpu().numpy()

    def write_rows(self, which, ids, rows):
        i = torch.as_tensor(np.ascontiguousarray(ids, dtype=np.int64)).to(self.device)
        r = torch.as_tensor(np.ascontiguousarray(rows, dtype=np.float32)).reshape(-1).to(self.device)
        assert r.numel() == i.numel() * self.d
        w2v_write_rows(self.h, which, i, i.numel(), r)
        w2v_sync(self.h)

    def topk_cosine(self, which, queries, cand_lo, cand_hi, K, tau):
        """(ids[m, K] padded with -1, cosines[m, K]) of the K nearest candidate rows above tau."""
        q = torch.as_tensor(np.ascontiguousarray(queries, dtype=np.int64)).to(self.device)
        ids = torch.empty(q.numel() * K, dtype=torch.int64, device=self.device)
        cs = torch.empty(q.numel() * K, dtype=torch.float32, device=self.device)
        w2v_topk_cosine(self.h, which, q, q.numel(), cand_lo, cand_hi, K, tau, ids, cs)
        w2v_sync(self.h)
        return ids.view(-1, K).cpu().numpy(), cs.view(-1, K).cpu().numpy()

    # ---- reader operators: tensors on this model's device ----
    # They run on this model's stream, in the order of the caller's current stream: after what that was given before, and
    # before what it is given next, also for memory: copies made within a call and its results belong to the current stream.
    # (Written for short calls: a small operator's time is what happens here.)
    def join_streams(self):
        """What this model's stream and the caller's current stream are given from here on waits for all that both have
        been given; False if they are the same.  For programs that read or write U and V by other means than this class."""
        if _raw_stream(self._index) != self._raw:
            here = torch.cuda.current_stream(self._index)
            self.stream.wait_stream(here)
            here.wait_stream(self.stream)
            return True
        return False

    def _on(self, *tensors):
        for t in tensors:
            if t is not None and t.get_device() != self._index:
                raise ValueError(f"tensor on {t.device}, this model is on {self.U.device}")

    @staticmethod
    def _type(t):
        code = _TYPES.get(t.dtype)
        if code is None:
            raise TypeError(f"{t.dtype} is not one of float32, bfloat16, float16")
        return code

    @staticmethod
    def _weights(d, *tensors):
        for t in tensors:
            if t.dtype is not torch.float32 or t.dim() != 1 or t.numel() != d or not t.is_contiguous():
                raise ValueError(f"weights must be contiguous float32 of shape ({d},)")

    @staticmethod
    def _rows(t):
        """A tensor whose last dimension is dense, as (rows, d, stride between rows, tensor)."""
        if t.dim() == 2:
            rows, d = t.shape
            ld, one = t.stride()
            if (one == 1 or d == 1) and (ld >= d or rows <= 1) and d < 1 << 32:
                return rows, d, ld if ld >= d else d, t
        d = t.shape[-1]
        if d >= 1 << 32:
            raise ValueError("rows must be shorter than 2^32")
        t = t.contiguous()
        return t.numel() // max(d, 1), d, d, t

    def layer_norm(self, x, gamma, beta, eps=1e-5, out_dtype=None):
        """(y, what layer_norm_backward needs).  x: [..., d], rows of a padded table included."""
        self._on(x, gamma, beta)
        rows, d, ld, xv = self._rows(x)
        self._weights(d, gamma, beta)
        y = x.new_empty(x.shape, dtype=out_dtype or x.dtype)
        stats = gamma.new_empty((2, rows))
        at = stats.data_ptr()
        apart = self.join_streams()
        w2v_layer_norm(self.h, rows, d, xv.data_ptr(), ld, self._type(x), gamma.data_ptr(), beta.data_ptr(), eps, y.data_ptr(), d,
                       self._type(y), at, at + 4 * rows)
        if apart:
            self.join_streams()
        return y, (xv, gamma, stats, y.dtype, x.shape)

    def layer_norm_backward(self, dy, saved):
        """(dx, dgamma, dbeta) from dy and what layer_norm returned."""
        x, gamma, stats, y_dtype, shape = saved
        self._on(dy)
        if dy.dtype is not y_dtype or dy.shape != shape:
            raise ValueError(f"dy must be {y_dtype} of shape {tuple(shape)}")
        rows, d, ld, dy = self._rows(dy)
        _, _, ldx, _ = self._rows(x)
        dx = x.new_empty(shape)
        dw = gamma.new_empty((2, d))
        at, to = stats.data_ptr(), dw.data_ptr()
        apart = self.join_streams()
        w2v_layer_norm_backward(self.h, rows, d, dy.data_ptr(), ld, _TYPES[y_dtype], x.data_ptr(), ldx, self._type(x),
                                gamma.data_ptr(), at, at + 4 * rows, dx.data_ptr(), d, to, to + 4 * d)
        if apart:
            self.join_streams()
        return dx, dw[0], dw[1]

    def sentence_spans(self, tokens):
        """[n, 2] int32: sentence bounds of every position of a token stream (-1 ends a sentence)."""
        self._on(tokens)
        if tokens.dtype is torch.int32:
            t = tokens.contiguous()
        elif tokens.dtype.is_floating_point or tokens.dtype.is_complex:
            raise TypeError(f"tokens must be whole numbers, not {tokens.dtype}")
        else:                                                        # an id beyond 32 bits stays one that no vocabulary has
            t = tokens.long().clamp(-2, 2 ** 31 - 1).to(torch.int32).contiguous()
        n = t.numel()
        spans = t.new_empty((n, 2))
        apart = self.join_streams()
        w2v_sentence_spans(self.h, t.data_ptr(), n, spans.data_ptr())
        if apart:
            self.join_streams()
        return spans

    @staticmethod
    def _heads(t, what):
        """[n, heads, dim] with dense heads side by side: (tensor, elements from position to position)."""
        if t.dim() != 3:
            raise ValueError(f"{what} must be [n, heads, head_dim]")
        n, heads, dim = t.shape
        width = heads * dim
        ld, between, one = t.stride()
        if one == 1 and (heads == 1 or between == dim) and t.data_ptr() % 16 == 0:
            if n <= 1:
                return t, width
            if ld >= width and ld % 8 == 0:
                return t, ld
        t = t.contiguous()
        return (t if t.data_ptr() % 16 == 0 else t.clone()), width

    def _window(self, q, k, v, bias, left, right, sinks, reach, two_sided, scale):
        """The w2v_window of a call, made once for a set of values."""
        self._on(q, k, v, bias)
        dtype = q.dtype
        if k.dtype is not dtype or v.dtype is not dtype or dtype not in (torch.bfloat16, torch.float16):
            raise TypeError("q, k and v must all be bfloat16 or all float16")
        qs, ks = q.shape, k.shape
        if len(qs) != 3 or len(ks) != 3 or v.shape != ks or ks[0] != qs[0] or ks[2] != qs[2]:
            raise ValueError("q [n, heads, dim], k and v [n, kv_heads, dim] do not fit together")
        buckets = 0
        if bias is not None:
            if bias.dtype is not torch.float32 or bias.dim() != 2 or bias.shape[1] != qs[1] or not bias.is_contiguous():
                raise ValueError("bias must be contiguous float32 [buckets, heads]")
            buckets = bias.shape[0]
        key = (dtype, qs[1], ks[1], qs[2], left, right, sinks, buckets, reach, two_sided, scale)
        w = self._windows.get(key)
        if w is None:
            for what, x in (("heads", qs[1]), ("kv_heads", ks[1]), ("head_dim", qs[2]), ("left", left), ("right", right), ("sinks", sinks), ("reach", reach)):
                if not 0 <= x < 1 << 32:                             # the struct's fields would take it modulo 2^32
                    raise ValueError(f"{what} = {x} is out of range")
            w = Window(_TYPES[dtype], qs[1], ks[1], qs[2], left, right, sinks, buckets, reach, int(two_sided),
                       qs[2] ** -0.5 if scale is None else scale)
            if len(self._windows) > 256:
                self._windows.clear()
            self._windows[key] = w
        return w

    def attend(self, q, k, v, spans, bias=None, left=0, right=0, sinks=0, reach=128, two_sided=False, scale=None, train=False):
        """o [n, heads, dim] of attention over a window of the sentence (w2v_attend); with train=True
        (o, what attend_backward needs)."""
        w = self._window(q, k, v, bias, left, right, sinks, reach, two_sided, scale)
        n = q.shape[0]
        if spans.dtype is not torch.int32 or spans.shape != (n, 2) or not spans.is_contiguous():
            raise ValueError(f"spans must be the contiguous int32 [{n}, 2] of sentence_spans")
        self._on(spans)
        (q, ldq), (k, ldk), (v, ldv) = self._heads(q, "q"), self._heads(k, "k"), self._heads(v, "v")
        o = q.new_empty(q.shape)
        lse = q.new_empty((w.heads, n), dtype=torch.float32) if train else None
        apart = self.join_streams()
        w2v_attend(self.h, w, n, spans.data_ptr(), q.data_ptr(), ldq, k.data_ptr(), ldk, v.data_ptr(), ldv,
                   None if bias is None else bias.data_ptr(), o.data_ptr(), w.heads * w.head_dim, None if lse is None else lse.data_ptr())
        if apart:
            self.join_streams()
        return (o, (w, spans, q, k, v, bias, o, lse)) if train else o

    def attend_backward(self, d_o, saved):
        """(dq, dk, dv, dbias) from d_o and what attend(train=True) returned; dbias is None without a bias."""
        w, spans, q, k, v, bias, o, lse = saved
        self._on(d_o)
        if d_o.dtype is not q.dtype or d_o.shape != q.shape:
            raise ValueError(f"d_o must be {q.dtype} of shape {tuple(q.shape)}")
        d_o, ld_do = self._heads(d_o, "d_o")
        (q, ldq), (k, ldk), (v, ldv) = self._heads(q, "q"), self._heads(k, "k"), self._heads(v, "v")
        dq, dk, dv = q.new_empty(q.shape), k.new_empty(k.shape), v.new_empty(v.shape)
        dbias = None if bias is None else torch.empty_like(bias)
        wq, wk = w.heads * w.head_dim, w.kv_heads * w.head_dim
        apart = self.join_streams()
        w2v_attend_backward(self.h, w, q.shape[0], spans.data_ptr(), q.data_ptr(), ldq, k.data_ptr(), ldk, v.data_ptr(), ldv,
                            None if bias is None else bias.data_ptr(), o.data_ptr(), wq, lse.data_ptr(), d_o.data_ptr(), ld_do,
                            dq.data_ptr(), wq, dk.data_ptr(), wk, dv.data_ptr(), wk, None if dbias is None else dbias.data_ptr())
        if apart:
            self.join_streams()
        return dq, dk, dv, dbias

    def attend_token(self, q, k, v, cache_k, cache_v, pos, bias=None, left=0, right=0, sinks=0, reach=128, two_sided=False, scale=None):
        """o [batch, heads, dim] of one new token per sequence at positions `pos`; writes k and v into the
        caches [batch, places, kv_heads, dim] (w2v_attend_token)."""
        w = self._window(q, k, v, bias, left, right, sinks, reach, two_sided, scale)
        batch = q.shape[0]
        if pos.dtype is not torch.int32 or pos.shape != (batch,) or not pos.is_contiguous():
            raise ValueError(f"pos must be contiguous int32 of shape ({batch},)")
        shape = cache_k.shape
        if cache_v.shape != shape:
            raise ValueError("cache_k and cache_v must have the same shape")
        if len(shape) != 4 or shape[0] != batch or shape[2:] != k.shape[1:] or cache_k.dtype is not q.dtype or cache_v.dtype is not q.dtype or \
                not cache_k.is_contiguous() or not cache_v.is_contiguous():
            raise ValueError("caches must be contiguous [batch, places, kv_heads, dim] of the type of q")
        self._on(pos, cache_k, cache_v)
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        o = q.new_empty(q.shape)
        apart = self.join_streams()
        w2v_attend_token(self.h, w, batch, pos.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), cache_k.data_ptr(),
                         cache_v.data_ptr(), shape[1], None if bias is None else bias.data_ptr(), o.data_ptr())
        if apart:
            self.join_streams()
        return o

    def fourbit_pack(self, rows, group=32):
        """(packed [n, 16 ceil(d/32)] uint8, scales [n, ceil(d/group)] bfloat16) of fp32 rows [n, d]."""
        self._on(rows)
        if rows.dtype is not torch.float32 or rows.dim() != 2:
            raise ValueError("rows must be float32 [n, d]")
        n, d, ld, rows = self._rows(rows)
        if d < 1 or group not in (32, 64, 128):
            raise ValueError("d must be positive and group 32, 64 or 128")
        packed = rows.new_empty((n, 16 * ((d + 31) // 32)), dtype=torch.uint8)
        scales = rows.new_empty((n, (d + group - 1) // group), dtype=torch.bfloat16)
        apart = self.join_streams()
        w2v_fourbit_pack(self.h, rows.data_ptr(), n, d, ld, group, packed.data_ptr(), scales.data_ptr())
        if apart:
            self.join_streams()
        return packed, scales

    def fourbit_scores(self, x, packed, scales, group=32):
        """[m, rows] fp32: products of m <= 8 fp32 vectors with every row of a table of fourbit_pack."""
        self._on(x, packed, scales)
        if x.dtype is not torch.float32 or x.dim() != 2:
            raise ValueError("x must be float32 [m, d]")
        m, d, ld, x = self._rows(x)
        if m > 8:
            raise ValueError("m must be at most 8")
        if d < 1 or group not in (32, 64, 128):
            raise ValueError("d must be positive and group 32, 64 or 128")
        n = packed.shape[0]
        if packed.dtype is not torch.uint8 or packed.shape != (n, 16 * ((d + 31) // 32)) or not packed.is_contiguous():
            raise ValueError(f"packed must be contiguous uint8 [rows, {16 * ((d + 31) // 32)}] for d = {d}")
        if scales.dtype is not torch.bfloat16 or scales.shape != (n, (d + group - 1) // group) or not scales.is_contiguous():
            raise ValueError("scales must be contiguous bfloat16 [rows, ceil(d / group)]")
        out = x.new_empty((m, n))
        apart = self.join_streams()
        w2v_fourbit_scores(self.h, x.data_ptr(), m, ld, packed.data_ptr(), scales.data_ptr(), n, d, group, out.data_ptr(), max(n, 1))
        if apart:
            self.join_streams()
        return out

    def set_step(self, s):
        w2v_set_step(self.h, s)

    def get_step(self):
        return w2v_get_step(self.h)

    def set_interleave(self, phase, stride):
        w2v_set_interleave(self.h, phase, stride)

    def sync(self):
        w2v_sync(self.h)

    def set_tuning(self, rows_in_flight=0, blocks_per_sm=0):
        w2v_set_tuning(self.h, rows_in_flight, blocks_per_sm)

    def launch_count(self):
        return w2v_get_launch_count(self.h)

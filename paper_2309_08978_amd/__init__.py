"""Python binding of libnnjit (include/nnjit.h): argument marshalling only.

Every ``nnjit_*`` function here has the name and argument order of the C
entry point it calls and returns its integer code unchanged; pointer
arguments accept a ``torch.Tensor`` (its ``data_ptr()``), an int or None, and
``stream`` accepts a ``torch.cuda.Stream``, an int handle or None (the default
stream, as NULL in C).  All the work runs in the HIP library; if
``libnnjit.so`` is missing the binding raises instead of falling back to
anything else.

``matmul`` / ``batched_matmul`` are conveniences that take tensors, derive
(M, N, K), leading dimensions and batch strides from them, call the entry
point and raise ``NnjitError`` on a negative code.  ``rotary`` /
``kv_append`` / ``paged_attention`` do the same for the operators of a served
decoder, with ``RotaryTable``, ``PagedCache`` and ``PagedBatch`` as the
handles that a program keeps, and ``paged_step`` / ``kv_append_slots`` /
``norm_rotary`` / ``norm_rotary_grad`` / ``tree_attention`` / ``kv_move`` /
``adjust_logits`` for a step of drafted tokens, with ``PagePool``, ``PagedStep``,
``HeadNorm`` and ``LogitRules``.  All of these run on the tensors' GPU, on
``stream`` or, without one, on the stream that torch works on there; an output
that they allocate belongs to that stream.  None of them is recorded by autograd, whatever
requires a gradient: gradients are calls of their own (``rotary`` with ``transpose``,
``norm_rotary_grad``), for an autograd function of the program's to make.
"""
from __future__ import annotations

import ctypes
import os
import threading
from typing import Optional

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libnnjit.so")

NNJIT_F32, NNJIT_F16 = 0, 1
NNJIT_KIND_GEMM, NNJIT_KIND_BATCHED, NNJIT_KIND_GEMV, NNJIT_KIND_GEMV_Q4 = 0, 1, 2, 3
NNJIT_ROTARY_HALF, NNJIT_ROTARY_INTERLEAVED = 0, 1
NNJIT_ROTARY_PLAIN, NNJIT_ROTARY_LINEAR, NNJIT_ROTARY_BASE, NNJIT_ROTARY_TURNS, NNJIT_ROTARY_INDEX = 0, 1, 2, 3, 4
NNJIT_OK, NNJIT_EINVAL, NNJIT_EDTYPE, NNJIT_ENOCFG, NNJIT_EHIP, NNJIT_ENOMEM = 0, -1, -2, -3, -4, -5
ERROR_NAMES = {-1: "NNJIT_EINVAL", -2: "NNJIT_EDTYPE", -3: "NNJIT_ENOCFG", -4: "NNJIT_EHIP", -5: "NNJIT_ENOMEM"}

EXPORTED = ["nnjit_matmul", "nnjit_batched_matmul", "nnjit_batched_matmul_noalloc", "nnjit_tune", "nnjit_tune_batched", "nnjit_matmul_config",
            "nnjit_gemv_q4", "nnjit_tune_gemv_q4", "nnjit_gemv_q4_config",
            "nnjit_num_configs", "nnjit_config_info", "nnjit_config_resources", "nnjit_lite_space",
            "nnjit_last_tune_stats", "nnjit_last_tune_stats_ex", "nnjit_last_tune_trace", "nnjit_cached_config", "nnjit_cached_ranked",
            "nnjit_set_online", "nnjit_online_status", "nnjit_cache_clear",
            "nnjit_cache_save", "nnjit_cache_load", "nnjit_stream_read", "nnjit_rotary_fill", "nnjit_rotary",
            "nnjit_kv_append", "nnjit_paged_attention", "nnjit_paged_step", "nnjit_kv_append_slots", "nnjit_norm_rotary",
            "nnjit_norm_rotary_grad", "nnjit_tree_attention", "nnjit_kv_move", "nnjit_adjust_logits", "nnjit_last_error", "nnjit_version"]


class NnjitError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{ERROR_NAMES.get(code, code)}: {msg}")
        self.code = code


class DeviceLimits(ctypes.Structure):
    _fields_ = [("num_cus", ctypes.c_int), ("simds_per_cu", ctypes.c_int), ("vgprs_per_lane", ctypes.c_int),
                ("vgpr_granule", ctypes.c_int), ("max_waves_per_simd", ctypes.c_int), ("wave_size", ctypes.c_int),
                ("lds_per_cu", ctypes.c_int64), ("lds_per_wg", ctypes.c_int64), ("max_threads_per_wg", ctypes.c_int)]


class Resources(ctypes.Structure):
    _fields_ = [("regs_per_lane", ctypes.c_int), ("regs_measured", ctypes.c_int), ("lds_per_wg", ctypes.c_int64),
                ("threads_per_wg", ctypes.c_int), ("waves_per_wg", ctypes.c_int), ("reg_limit", ctypes.c_int),
                ("lds_limit", ctypes.c_int), ("wave_limit", ctypes.c_int), ("wg_per_cu", ctypes.c_int)]


class TuneStats(ctypes.Structure):
    _fields_ = [("wall_ms", ctypes.c_double), ("eval_ms", ctypes.c_double), ("n_enumerated", ctypes.c_int),
                ("n_lite", ctypes.c_int), ("n_timed", ctypes.c_int), ("n_aborted", ctypes.c_int),
                ("n_failed", ctypes.c_int), ("chosen", ctypes.c_int), ("best_us", ctypes.c_double),
                ("default_us", ctypes.c_double), ("cache_hit", ctypes.c_int)]


class PagedKvDesc(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p)] + [
        (n, ctypes.c_int64) for n in ("k_page", "k_token", "k_head", "v_page", "v_token", "v_head", "pages", "page_size",
                                      "kv_heads", "head_dim")] + [("dtype", ctypes.c_int)]


class PagedBatchDesc(ctypes.Structure):
    _fields_ = [("sequences", ctypes.c_int64), ("tokens", ctypes.c_int64), ("q_start", ctypes.c_void_p),
                ("kv_len", ctypes.c_void_p), ("page_table", ctypes.c_void_p)] + [
        (n, ctypes.c_int64) for n in ("ld_table", "table_pages", "max_q", "max_kv")]


class RotaryDesc(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("positions", ctypes.c_int64), ("rotary_dim", ctypes.c_int64),
                ("layout", ctypes.c_int)]


class RotaryScaling(ctypes.Structure):
    """nnjit_rotary_scaling: RotaryScaling(kind, factor, original, fast, slow, magnitude)."""
    _fields_ = [("kind", ctypes.c_int)] + [(n, ctypes.c_double) for n in ("factor", "original", "fast", "slow", "magnitude")]


class PagePoolDesc(ctypes.Structure):
    _fields_ = [("free_pages", ctypes.c_void_p), ("capacity", ctypes.c_int64), ("count", ctypes.c_void_p),
                ("count_out", ctypes.c_void_p)]


class StepDesc(ctypes.Structure):
    _fields_ = [("sequences", ctypes.c_int64), ("tokens", ctypes.c_int64)] + [
        (n, ctypes.c_void_p) for n in ("held", "keep", "added", "parent", "page_table")] + [
        (n, ctypes.c_int64) for n in ("ld_table", "table_pages", "page_size")] + [
        (n, ctypes.c_void_p) for n in ("q_start", "kv_len", "positions", "slots", "mask")] + [
        ("ld_mask", ctypes.c_int64), ("mask_words", ctypes.c_int64), ("status", ctypes.c_void_p)]


class HeadNormDesc(ctypes.Structure):
    _fields_ = [("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("q_head", ctypes.c_int64), ("k_head", ctypes.c_int64),
                ("dtype", ctypes.c_int), ("eps", ctypes.c_float)]


class LogitRulesDesc(ctypes.Structure):
    _fields_ = [("history", ctypes.c_void_p), ("ld_history", ctypes.c_int64), ("history_len", ctypes.c_int64)] + [
        (n, ctypes.c_void_p) for n in ("length", "prompt", "repetition", "presence", "frequency", "bias_token", "bias_value")] + [
        ("ld_bias", ctypes.c_int64), ("bias_len", ctypes.c_int64), ("mask", ctypes.c_void_p), ("ld_mask", ctypes.c_int64),
        ("mask_rows", ctypes.c_int64), ("mask_row", ctypes.c_void_p)]


def mi355x_limits() -> DeviceLimits:
    """MI355X constants for the host-only resource model."""
    return DeviceLimits(256, 4, 512, 8, 8, 64, 163840, 163840, 1024)


_lock = threading.Lock()
_lib = None


def load(build_if_missing: bool = False) -> ctypes.CDLL:
    """Load libnnjit.so (built in-tree by ``paper_2309_08978_amd.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is not None:
            return _lib
        if not os.path.exists(LIB_PATH):
            if not build_if_missing:
                raise RuntimeError(f"{LIB_PATH} is not built; run `python -m paper_2309_08978_amd.build`")
            from . import build as _b
            _b.build()
        lib = ctypes.CDLL(LIB_PATH)
        i64, vp, ci = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int
        sig = {
            "nnjit_matmul": [i64, i64, i64, vp, i64, vp, i64, vp, i64, ci, vp],
            "nnjit_batched_matmul": [i64, i64, i64, i64, vp, i64, i64, vp, i64, i64, vp, i64, i64, ci, vp],
            "nnjit_batched_matmul_noalloc": [i64, i64, i64, i64, vp, i64, i64, vp, i64, i64, vp, i64, i64, ci, vp],
            "nnjit_tune": [i64, i64, i64, ci],
            "nnjit_tune_batched": [i64, i64, i64, i64, ci],
            "nnjit_matmul_config": [ci, i64, i64, i64, i64, vp, i64, i64, vp, i64, i64, vp, i64, i64, ci, vp],
            "nnjit_gemv_q4": [i64, i64, i64, vp, vp, i64, vp, i64, vp, vp],
            "nnjit_tune_gemv_q4": [i64, i64, i64],
            "nnjit_gemv_q4_config": [ci, i64, i64, i64, vp, vp, i64, vp, i64, vp, vp],
            "nnjit_num_configs": [],
            "nnjit_config_info": [ci, ctypes.c_char_p, i64],
            "nnjit_config_resources": [ci, ctypes.POINTER(DeviceLimits), ctypes.POINTER(Resources)],
            "nnjit_lite_space": [ci, ci, i64, i64, i64, i64, ctypes.POINTER(DeviceLimits),
                                 ctypes.POINTER(ci), ci, ctypes.POINTER(ci), ctypes.POINTER(i64)],
            "nnjit_last_tune_stats": [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ci), ctypes.POINTER(ci),
                                      ctypes.POINTER(ci)],
            "nnjit_last_tune_stats_ex": [ctypes.POINTER(TuneStats)],
            "nnjit_last_tune_trace": [ctypes.POINTER(ci), ctypes.POINTER(ctypes.c_double),
                                      ctypes.POINTER(ctypes.c_double), ci],
            "nnjit_cached_config": [ci, ci, i64, i64, i64, i64],
            "nnjit_cached_ranked": [ci, ci, i64, i64, i64, i64, ctypes.POINTER(ci), ctypes.POINTER(ctypes.c_double), ci],
            "nnjit_set_online": [ci],
            "nnjit_online_status": [ci, ci, i64, i64, i64, i64, ctypes.POINTER(ci), ctypes.POINTER(ci),
                                    ctypes.POINTER(ci)],
            "nnjit_cache_clear": [],
            "nnjit_cache_save": [ctypes.c_char_p],
            "nnjit_cache_load": [ctypes.c_char_p],
            "nnjit_stream_read": [vp, i64, vp, ci, vp],
            "nnjit_rotary_fill": [vp, i64, i64, ctypes.c_double, vp, vp],
            "nnjit_rotary": [vp, i64, i64, i64, vp, vp, i64, i64, ci, vp, i64, i64, ci, ci, vp],
            "nnjit_kv_append": [vp, vp, vp, vp, i64, i64, vp, i64, i64, i64, vp, i64, i64, vp, i64, i64, ci, vp],
            "nnjit_paged_attention": [vp, vp, i64, vp, i64, i64, vp, i64, i64, ctypes.c_float, ci, i64, vp],
            "nnjit_paged_step": [vp, vp, vp],
            "nnjit_kv_append_slots": [vp, i64, vp, vp, vp, vp, vp, i64, i64, vp, i64, i64, i64, vp, i64, i64, vp, i64, i64, ci, vp],
            "nnjit_norm_rotary": [vp, i64, i64, i64, vp, vp, i64, ci, ctypes.c_float, vp, i64, i64, ci, vp, i64, i64, ci, vp],
            "nnjit_norm_rotary_grad": [vp, i64, i64, i64, vp, vp, i64, ci, ctypes.c_float, vp, i64, i64, ci, vp, i64, i64, ci,
                                       vp, i64, i64, vp, vp],
            "nnjit_tree_attention": [vp, vp, vp, i64, i64, vp, i64, vp, i64, i64, vp, i64, i64, ctypes.c_float, i64, vp],
            "nnjit_kv_move": [vp, vp, vp, i64, i64, vp, vp],
            "nnjit_adjust_logits": [vp, i64, i64, vp, i64, ci, vp, i64, ci, vp],
            "nnjit_last_error": [],
            "nnjit_version": [],
        }
        for name, args in sig.items():
            f = getattr(lib, name)
            f.argtypes = args
            f.restype = ctypes.c_char_p if name == "nnjit_last_error" else ctypes.c_int
        _lib = lib
        return lib


def _ptr(x) -> Optional[int]:
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return int(x.data_ptr())


def _stream(s) -> Optional[int]:
    if s is None:
        return None
    if isinstance(s, int):
        return s
    return int(s.cuda_stream)


# ------------------------------------------------------ entry points (1:1)

def nnjit_matmul(M, N, K, A, lda, B, ldb, C, ldc, dtype, stream=None) -> int:
    return load().nnjit_matmul(M, N, K, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc, dtype, _stream(stream))


def nnjit_batched_matmul(batch, M, N, K, A, lda, strideA, B, ldb, strideB, C, ldc, strideC, dtype,
                         stream=None) -> int:
    return load().nnjit_batched_matmul(batch, M, N, K, _ptr(A), lda, strideA, _ptr(B), ldb, strideB,
                                       _ptr(C), ldc, strideC, dtype, _stream(stream))


def nnjit_batched_matmul_noalloc(batch, M, N, K, A, lda, strideA, B, ldb, strideB, C, ldc, strideC, dtype,
                                 stream=None) -> int:
    return load().nnjit_batched_matmul_noalloc(batch, M, N, K, _ptr(A), lda, strideA, _ptr(B), ldb, strideB,
                                               _ptr(C), ldc, strideC, dtype, _stream(stream))


def nnjit_tune(M, N, K, dtype) -> int:
    return load().nnjit_tune(M, N, K, dtype)


def nnjit_tune_batched(batch, M, N, K, dtype) -> int:
    return load().nnjit_tune_batched(batch, M, N, K, dtype)


def nnjit_matmul_config(cfg, batch, M, N, K, A, lda, strideA, B, ldb, strideB, C, ldc, strideC, dtype,
                        stream=None) -> int:
    return load().nnjit_matmul_config(cfg, batch, M, N, K, _ptr(A), lda, strideA, _ptr(B), ldb, strideB,
                                      _ptr(C), ldc, strideC, dtype, _stream(stream))


def nnjit_gemv_q4(N, K, group, x, Wq, ldq, scales, lds, y, stream=None) -> int:
    return load().nnjit_gemv_q4(N, K, group, _ptr(x), _ptr(Wq), ldq, _ptr(scales), lds, _ptr(y), _stream(stream))


def nnjit_tune_gemv_q4(N, K, group) -> int:
    return load().nnjit_tune_gemv_q4(N, K, group)


def nnjit_gemv_q4_config(cfg, N, K, group, x, Wq, ldq, scales, lds, y, stream=None) -> int:
    return load().nnjit_gemv_q4_config(cfg, N, K, group, _ptr(x), _ptr(Wq), ldq, _ptr(scales), lds, _ptr(y),
                                       _stream(stream))


def nnjit_num_configs() -> int:
    return load().nnjit_num_configs()


def nnjit_config_info(cfg) -> str:
    buf = ctypes.create_string_buffer(512)
    rc = load().nnjit_config_info(cfg, buf, len(buf))
    if rc < 0:
        raise NnjitError(rc, nnjit_last_error())
    return buf.value.decode()


def nnjit_config_resources(cfg, dev: Optional[DeviceLimits] = None) -> dict:
    out = Resources()
    rc = load().nnjit_config_resources(cfg, ctypes.byref(dev) if dev is not None else None, ctypes.byref(out))
    if rc < 0:
        raise NnjitError(rc, nnjit_last_error())
    return {f: getattr(out, f) for f, _ in Resources._fields_}


def nnjit_lite_space(kind, dtype, batch, M, N, K, dev: Optional[DeviceLimits] = None, cap: int = 4096):
    """-> (ids in evaluation order, n_surviving, n_enumerated, n_naive)."""
    ids = (ctypes.c_int * cap)()
    n_enum = ctypes.c_int(0)
    n_naive = ctypes.c_int64(0)
    rc = load().nnjit_lite_space(kind, dtype, batch, M, N, K, ctypes.byref(dev) if dev is not None else None,
                                 ids, cap, ctypes.byref(n_enum), ctypes.byref(n_naive))
    if rc < 0:
        raise NnjitError(rc, nnjit_last_error())
    return list(ids[:min(rc, cap)]), rc, n_enum.value, n_naive.value


def nnjit_last_tune_stats() -> dict:
    """-> {'wall_ms', 'n_enum', 'n_pruned', 'n_timed'} of the last tune on this thread."""
    w = ctypes.c_double(0.0)
    e, p, t = ctypes.c_int(0), ctypes.c_int(0), ctypes.c_int(0)
    check(load().nnjit_last_tune_stats(ctypes.byref(w), ctypes.byref(e), ctypes.byref(p), ctypes.byref(t)))
    return {"wall_ms": w.value, "n_enum": e.value, "n_pruned": p.value, "n_timed": t.value}


def nnjit_last_tune_stats_ex() -> dict:
    """-> every field of nnjit_tune_stats for the last tune on this thread."""
    st = TuneStats()
    check(load().nnjit_last_tune_stats_ex(ctypes.byref(st)))
    return {f: getattr(st, f) for f, _ in TuneStats._fields_}


def nnjit_last_tune_trace(cap: int = 256):
    ids = (ctypes.c_int * cap)()
    us = (ctypes.c_double * cap)()
    at = (ctypes.c_double * cap)()
    n = load().nnjit_last_tune_trace(ids, us, at, cap)
    return [(ids[i], us[i], at[i]) for i in range(min(n, cap))]


def nnjit_cached_config(kind, dtype, batch, M, N, K) -> int:
    return load().nnjit_cached_config(kind, dtype, batch, M, N, K)


def nnjit_cached_ranked(kind, dtype, batch, M, N, K, cap: int = 5):
    """-> [(config id, us)] ranked candidates of a tuned shape (raises if not tuned)."""
    ids = (ctypes.c_int * cap)()
    us = (ctypes.c_double * cap)()
    rc = load().nnjit_cached_ranked(kind, dtype, batch, M, N, K, ids, us, cap)
    if rc < 0:
        raise NnjitError(rc, nnjit_last_error())
    return [(ids[i], us[i]) for i in range(min(rc, cap))]


def nnjit_set_online(enable: bool) -> int:
    """Switch online just-in-time tuning on or off; returns the previous setting."""
    return load().nnjit_set_online(1 if enable else 0)


def nnjit_online_status(kind, dtype, batch, M, N, K) -> dict:
    """{'state': 'online'|'tuned', 'measured', 'total', 'registered'} (raises if neither)."""
    m, t, r = ctypes.c_int(-1), ctypes.c_int(-1), ctypes.c_int(-1)
    rc = load().nnjit_online_status(kind, dtype, batch, M, N, K, ctypes.byref(m), ctypes.byref(t), ctypes.byref(r))
    if rc < 0:
        raise NnjitError(rc, nnjit_last_error())
    return {"state": "online" if rc == 0 else "tuned", "measured": m.value, "total": t.value,
            "registered": r.value}


def nnjit_cache_clear() -> int:
    return load().nnjit_cache_clear()


def nnjit_cache_save(path) -> int:
    return load().nnjit_cache_save(os.fsencode(path))


def nnjit_cache_load(path) -> int:
    return load().nnjit_cache_load(os.fsencode(path))


def nnjit_stream_read(src, nbytes, sink, workgroups, stream=None) -> int:
    return load().nnjit_stream_read(_ptr(src), nbytes, _ptr(sink), workgroups, _stream(stream))


def _desc(d) -> Optional[int]:
    """Address of a descriptor: a handle, a ctypes structure, an int or None."""
    if d is None or isinstance(d, int):
        return d
    return ctypes.addressof(getattr(d, "desc", d))


def nnjit_rotary_fill(table, positions, rotary_dim, base, scaling=None, stream=None) -> int:
    return load().nnjit_rotary_fill(_ptr(table), positions, rotary_dim, base, _desc(scaling), _stream(stream))


def nnjit_rotary(rotary, tokens, heads, head_dim, positions, x, x_token, x_head, x_dtype, y, y_token, y_head, y_dtype,
                 transpose=0, stream=None) -> int:
    return load().nnjit_rotary(_desc(rotary), tokens, heads, head_dim, _ptr(positions), _ptr(x), x_token, x_head, x_dtype,
                               _ptr(y), y_token, y_head, y_dtype, transpose, _stream(stream))


def nnjit_kv_append(cache, batch, rotary, k, k_token, k_head, v, v_token, v_head, q_heads, q, q_token, q_head, q_out,
                    qo_token, qo_head, src_dtype, stream=None) -> int:
    return load().nnjit_kv_append(_desc(cache), _desc(batch), _desc(rotary), _ptr(k), k_token, k_head, _ptr(v), v_token,
                                  v_head, q_heads, _ptr(q), q_token, q_head, _ptr(q_out), qo_token, qo_head, src_dtype,
                                  _stream(stream))


def nnjit_paged_attention(cache, batch, q_heads, q, q_token, q_head, out, out_token, out_head, scale, causal=1, window=0,
                          stream=None) -> int:
    return load().nnjit_paged_attention(_desc(cache), _desc(batch), q_heads, _ptr(q), q_token, q_head, _ptr(out), out_token,
                                        out_head, scale, causal, window, _stream(stream))


def nnjit_paged_step(pool, step, stream=None) -> int:
    return load().nnjit_paged_step(_desc(pool), _desc(step), _stream(stream))


def nnjit_kv_append_slots(cache, tokens, slots, positions, rotary, norm, k, k_token, k_head, v, v_token, v_head, q_heads, q, q_token,
                          q_head, q_out, qo_token, qo_head, src_dtype, stream=None) -> int:
    return load().nnjit_kv_append_slots(_desc(cache), tokens, _ptr(slots), _ptr(positions), _desc(rotary), _desc(norm), _ptr(k),
                                        k_token, k_head, _ptr(v), v_token, v_head, q_heads, _ptr(q), q_token, q_head, _ptr(q_out),
                                        qo_token, qo_head, src_dtype, _stream(stream))


def nnjit_norm_rotary(rotary, tokens, heads, head_dim, positions, weight, w_head, w_dtype, eps, x, x_token, x_head, x_dtype, y, y_token,
                      y_head, y_dtype, stream=None) -> int:
    return load().nnjit_norm_rotary(_desc(rotary), tokens, heads, head_dim, _ptr(positions), _ptr(weight), w_head, w_dtype, eps, _ptr(x),
                                    x_token, x_head, x_dtype, _ptr(y), y_token, y_head, y_dtype, _stream(stream))


def nnjit_norm_rotary_grad(rotary, tokens, heads, head_dim, positions, weight, w_head, w_dtype, eps, x, x_token, x_head, x_dtype, dy,
                           dy_token, dy_head, dy_dtype, dx, dx_token, dx_head, dw, stream=None) -> int:
    return load().nnjit_norm_rotary_grad(_desc(rotary), tokens, heads, head_dim, _ptr(positions), _ptr(weight), w_head, w_dtype, eps,
                                         _ptr(x), x_token, x_head, x_dtype, _ptr(dy), dy_token, dy_head, dy_dtype, _ptr(dx), dx_token,
                                         dx_head, _ptr(dw), _stream(stream))


def nnjit_tree_attention(cache, batch, mask, ld_mask, mask_words, positions, q_heads, q, q_token, q_head, out, out_token, out_head,
                         scale, window=0, stream=None) -> int:
    return load().nnjit_tree_attention(_desc(cache), _desc(batch), _ptr(mask), ld_mask, mask_words, _ptr(positions), q_heads, _ptr(q),
                                       q_token, q_head, _ptr(out), out_token, out_head, scale, window, _stream(stream))


def nnjit_kv_move(cache, batch, path, ld_path, path_len, accepted, stream=None) -> int:
    return load().nnjit_kv_move(_desc(cache), _desc(batch), _ptr(path), ld_path, path_len, _ptr(accepted), _stream(stream))


def nnjit_adjust_logits(rules, rows, vocab, x, ldx, x_dtype, y, ldy, y_dtype, stream=None) -> int:
    return load().nnjit_adjust_logits(_desc(rules), rows, vocab, _ptr(x), ldx, x_dtype, _ptr(y), ldy, y_dtype, _stream(stream))


def nnjit_last_error() -> str:
    r = load().nnjit_last_error()
    return r.decode() if r else ""


def nnjit_version() -> int:
    return load().nnjit_version()


# ------------------------------------------------------------ conveniences

_NOT_PRODUCTS = ("attention_", "rotary.", "serving")   # csrc/ sources that no product runs


def kernel_digest() -> str:
    """Short digest of the kernel and launch sources of the products (csrc/
    without the serving operators'): counter measurements recorded against
    one digest are stale under another."""
    import hashlib
    h = hashlib.sha256()
    d = os.path.join(HERE, "csrc")
    for name in sorted(os.listdir(d)):
        if name.startswith(_NOT_PRODUCTS):
            continue
        with open(os.path.join(d, name), "rb") as f:
            h.update(name.encode() + b"\0" + f.read())
    return h.hexdigest()[:16]


def dtype_code(t) -> int:
    import torch
    if t.dtype == torch.float32:
        return NNJIT_F32
    if t.dtype == torch.float16:
        return NNJIT_F16
    raise TypeError(f"unsupported dtype {t.dtype}")


def check(rc: int) -> int:
    if rc < 0:
        raise NnjitError(rc, nnjit_last_error())
    return rc


def _ld(t) -> int:
    """Leading dimension of the row-major matrices of t (last two dims):
    unit column stride, and a row stride that separates the rows."""
    rows, cols = int(t.shape[-2]), int(t.shape[-1])
    if t.stride(-1) != 1 and cols > 1:
        raise ValueError("operands must have unit stride along the last dimension")
    if rows > 1 and int(t.stride(-2)) < cols:
        raise ValueError(f"row stride {t.stride(-2)} < {cols} columns: rows overlap (an expanded or "
                         "transposed view); pass a contiguous copy")
    return max(int(t.stride(-2)), cols, 1)


def _check_operands(A, B, C, batched: bool):
    """Reject, before any library call, operands the C entry points would
    read or write out of bounds: mismatched dtypes or shapes, an output that
    is not fp32, overlapping rows or output slices, tensors not on one GPU."""
    import torch
    nd = 3 if batched else 2
    for name, t in (("A", A), ("B", B), ("C", C)):
        if t.dim() != nd:
            raise ValueError(f"{name} must be {nd}-D, got shape {tuple(t.shape)}")
    if A.dtype not in (torch.float32, torch.float16):
        raise TypeError(f"unsupported dtype {A.dtype}")
    if B.dtype != A.dtype:
        raise TypeError(f"A is {A.dtype} but B is {B.dtype}")
    if C.dtype != torch.float32:
        raise TypeError(f"C must be float32, got {C.dtype}")
    M, K = A.shape[-2:]
    K2, N = B.shape[-2:]
    if K2 != K:
        raise ValueError(f"inner dimensions differ: {tuple(A.shape)} . {tuple(B.shape)}")
    want = ((A.shape[0],) if batched else ()) + (M, N)
    if batched and B.shape[0] != A.shape[0]:
        raise ValueError(f"batch sizes differ: {tuple(A.shape)} . {tuple(B.shape)}")
    if tuple(C.shape) != want:
        raise ValueError(f"C has shape {tuple(C.shape)}, expected {want}")
    lds = [_ld(t) for t in (A, B, C)]
    if batched:
        for name, t in (("A", A), ("B", B), ("C", C)):
            if t.stride(0) < 0:
                raise ValueError(f"negative batch stride of {name}")
        span = (M - 1) * lds[2] + N if M > 0 and N > 0 else 0
        if C.shape[0] > 1 and span > 0 and C.stride(0) < span:
            raise ValueError(f"batch stride {C.stride(0)} of C < {span}: output slices overlap")
    devs = {t.device for t in (A, B, C)}
    if len(devs) != 1 or next(iter(devs)).type != "cuda":
        raise ValueError(f"A, B and C must be on one GPU, got {sorted(str(d) for d in devs)}")
    return lds


def _plain_lds(A, B, C, sa, sb, sc):
    """Leading dimensions and batch strides (lda, ldb, ldc, sA, sB, sC) of
    operands that plainly pass every check of _check_operands, read with as few
    tensor attribute accesses as that takes; None for any other operands
    (wrong, or right in an unusual way), which the full checks then settle."""
    ta, tb, tc = A.stride(), B.stride(), C.stride()
    dt = A.dtype
    M, K, N = sa[-2], sa[-1], sb[-1]
    lda, ldb, ldc = ta[-2], tb[-2], tc[-2]
    if not (dt in _CODES and B.dtype is dt and C.dtype is _F32 and sb[-2] == K and sc[-2] == M and sc[-1] == N
            and ta[-1] == 1 and tb[-1] == 1 and tc[-1] == 1
            and lda >= K > 0 and ldb >= N > 0 and ldc >= N and M > 0
            and A.is_cuda and B.is_cuda and C.is_cuda
            and A.get_device() == B.get_device() == C.get_device()):
        return None
    if len(sa) == 2:
        return lda, ldb, ldc, 0, 0, 0
    if not (sa[0] == sb[0] == sc[0] and ta[0] >= 0 and tb[0] >= 0 and tc[0] >= (M - 1) * ldc + N):
        return None
    return lda, ldb, ldc, ta[0], tb[0], tc[0]


_CODES: dict = {}     # torch dtype -> code; filled on first use (torch is imported lazily)
_F32 = _I32 = _I64 = None
_torch_module = None
_torch_stream = _torch_device = None     # handle of torch's current stream on a GPU; the current GPU (0.1 us each)


def _torch():
    global _F32, _I32, _I64, _torch_module, _torch_stream, _torch_device
    if _torch_module is None:
        import torch
        _CODES.update({torch.float32: NNJIT_F32, torch.float16: NNJIT_F16})
        _F32, _I32, _I64 = torch.float32, torch.int32, torch.int64
        _torch_stream, _torch_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
        _torch_module = torch
    return _torch_module


def _launch(entry, device_index: int, stream, *args) -> int:
    """entry(*args, stream), checked, with the operands' GPU current: on
    ``stream`` or, if None, on torch's current one there, so that the call is
    ordered with the other work on its tensors and with the reuse of their
    memory."""
    s = _torch_stream(device_index) if stream is None else _stream(stream)
    if _torch_device() == device_index:
        rc = entry(*args, s)
        return rc if rc >= 0 else check(rc)
    with _torch_module.cuda.device(device_index):
        return check(entry(*args, s))


def _empty(shape, dtype, device, stream):
    """An output from the memory of the stream that will write it: another
    stream's could still be in use there."""
    torch = _torch()
    if stream is None or device.type != "cuda" or _stream(stream) == _torch_stream(
            _torch_device() if device.index is None else device.index):
        return torch.empty(shape, dtype=dtype, device=device)
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=device) if stream else torch.cuda.default_stream(device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def matmul(A, B, C=None, stream=None, cfg: Optional[int] = None):
    """C = A . B for 2-D fp32/fp16 CUDA tensors (C fp32, allocated if None)."""
    torch = _torch()
    sa, sb = A.shape, B.shape
    if len(sa) != 2 or len(sb) != 2:
        raise ValueError(f"matmul takes 2-D operands, got {tuple(sa)} . {tuple(sb)}")
    M, K = sa
    N = sb[1]
    if C is None:
        C = _empty((M, N), torch.float32, A.device, stream)
    sc = C.shape
    p = _plain_lds(A, B, C, sa, sb, sc) if len(sc) == 2 else None
    lda, ldb, ldc = p[:3] if p else _check_operands(A, B, C, batched=False)
    dt = dtype_code(A) if not p else _CODES[A.dtype]
    if cfg is None:
        _launch((_lib or load()).nnjit_matmul, A.get_device(), stream, M, N, K, A.data_ptr(), lda, B.data_ptr(), ldb,
                C.data_ptr(), ldc, dt)
    else:
        _launch(nnjit_matmul_config, A.get_device(), stream, cfg, 1, M, N, K, A, lda, 0, B, ldb, 0, C, ldc, 0, dt)
    return C


def batched_matmul(A, B, C=None, stream=None, cfg: Optional[int] = None):
    """C[b] = A[b] . B[b] for 3-D fp32/fp16 CUDA tensors (C fp32)."""
    torch = _torch()
    sa, sb = A.shape, B.shape
    if len(sa) != 3 or len(sb) != 3:
        raise ValueError(f"batched_matmul takes 3-D operands, got {tuple(sa)} . {tuple(sb)}")
    batch, M, K = sa
    N = sb[2]
    if C is None:
        C = _empty((batch, M, N), torch.float32, A.device, stream)
    sc = C.shape
    p = _plain_lds(A, B, C, sa, sb, sc) if len(sc) == 3 else None
    if p:
        lda, ldb, ldc, sA, sB, sC = p
        dt = _CODES[A.dtype]
    else:
        lda, ldb, ldc = _check_operands(A, B, C, batched=True)
        dt = dtype_code(A)
        sA, sB, sC = (int(t.stride(0)) for t in (A, B, C))
    if cfg is None:
        _launch((_lib or load()).nnjit_batched_matmul, A.get_device(), stream, batch, M, N, K, A.data_ptr(), lda, sA,
                B.data_ptr(), ldb, sB, C.data_ptr(), ldc, sC, dt)
    else:
        _launch(nnjit_matmul_config, A.get_device(), stream, cfg, batch, M, N, K, A, lda, sA, B, ldb, sB, C, ldc, sC, dt)
    return C


def gemv_q4(x, Wq, scales, group: int, N: int, y=None, stream=None, cfg: Optional[int] = None):
    """y = x . W for a 4-bit weight-only W (include/nnjit.h, nnjit_gemv_q4):
    x fp16 [K], Wq int32 [N, ldq] (uint32 code words, reinterpreted), scales
    fp16 [N, lds]; y fp32 [N] (allocated if None)."""
    torch = _torch()
    if y is not None and cfg is None:
        # operands that plainly pass every check below, with few accesses
        sx, sw, ss, tw, ts = x.shape, Wq.shape, scales.shape, Wq.stride(), scales.stride()
        K = sx[0] if len(sx) == 1 else 0
        if (K > 0 and group >= 1 and N > 1 and len(sw) == 2 and len(ss) == 2 and x.stride(0) == 1
                and sw[0] >= N and ss[0] >= N and sw[1] >= -(-K // 8) and ss[1] >= -(-K // group)
                and tw[1] == 1 and ts[1] == 1 and tw[0] >= sw[1] and ts[0] >= ss[1]
                and x.dtype is torch.float16 and scales.dtype is torch.float16 and Wq.element_size() == 4
                and y.dtype is _F32 and y.shape == (N,) and y.stride(0) == 1
                and x.is_cuda and Wq.is_cuda and scales.is_cuda and y.is_cuda
                and x.get_device() == Wq.get_device() == scales.get_device() == y.get_device()):
            _launch((_lib or load()).nnjit_gemv_q4, x.get_device(), stream, N, K, group, x.data_ptr(), Wq.data_ptr(), tw[0],
                    scales.data_ptr(), ts[0], y.data_ptr())
            return y
    if x.dim() != 1 or (x.shape[0] > 1 and x.stride(0) != 1):
        raise ValueError(f"x must be a contiguous vector, got shape {tuple(x.shape)}")
    K = int(x.shape[0])
    if group < 1:
        raise ValueError(f"group must be >= 1, got {group}")
    if Wq.dim() != 2 or scales.dim() != 2 or Wq.shape[0] < N or scales.shape[0] < N:
        raise ValueError(f"shape mismatch x {tuple(x.shape)}, Wq {tuple(Wq.shape)}, scales {tuple(scales.shape)}")
    if Wq.shape[1] < -(-K // 8) or scales.shape[1] < -(-K // group):
        raise ValueError(f"rows too short for K={K}: Wq {tuple(Wq.shape)}, scales {tuple(scales.shape)}")
    if x.dtype != torch.float16 or scales.dtype != torch.float16 or Wq.element_size() != 4:
        raise TypeError("x and scales must be float16, Wq 32-bit words")
    if y is None:
        y = _empty((N,), torch.float32, x.device, stream)
    if y.dtype != torch.float32 or tuple(y.shape) != (N,) or (N > 1 and y.stride(0) != 1):
        raise ValueError(f"y must be a contiguous float32 vector of {N}, got {y.dtype} {tuple(y.shape)}")
    devs = {t.device for t in (x, Wq, scales, y)}
    if len(devs) != 1 or next(iter(devs)).type != "cuda":
        raise ValueError(f"x, Wq, scales and y must be on one GPU, got {sorted(str(d) for d in devs)}")
    ldq, lds = _ld(Wq), _ld(scales)
    if cfg is None:
        _launch(nnjit_gemv_q4, x.get_device(), stream, N, K, group, x, Wq, ldq, scales, lds, y)
    else:
        _launch(nnjit_gemv_q4_config, x.get_device(), stream, cfg, N, K, group, x, Wq, ldq, scales, lds, y)
    return y


def _separate(name: str, t):
    """Reject a tensor that is written to if elements of it share memory."""
    room = 1
    for stride, size in sorted((t.stride(i), t.shape[i]) for i in range(t.dim())):
        if size > 1:
            if stride < room:
                raise ValueError(f"elements of {name} overlap: shape {tuple(t.shape)}, strides {tuple(t.stride())}")
            room = stride * (size - 1) + room
    return t


def _on_one_gpu(**tensors):
    devs = {t.device for t in tensors.values()}
    if len(devs) != 1 or next(iter(devs)).type != "cuda":
        raise ValueError(f"{', '.join(tensors)} must be on one GPU, got {sorted(str(d) for d in devs)}")


def _unit_dims(name: str, t):
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name} must have unit stride along the last dimension")


def _int32(name: str, t, *shape):
    import torch
    if t.dtype != torch.int32 or t.dim() != len(shape) or any(w is not None and n != w for n, w in zip(t.shape, shape)):
        raise ValueError(f"{name} must be int32 of shape {shape}, got {t.dtype} {tuple(t.shape)}")
    if t.dim() == 1 and t.shape[0] > 1 and t.stride(0) != 1:
        raise ValueError(f"{name} must be contiguous")


class RotaryTable:
    """Cos and sin of rotary positions: ``table`` fp32 [positions, rotary_dim]
    (per position the cos of every pair, then their sin), ``layout`` 'half'
    (pairs i, i + rotary_dim / 2) or 'interleaved' (pairs 2 i, 2 i + 1)."""

    def __init__(self, table, layout: str = "half"):
        import torch
        if layout not in ("half", "interleaved"):
            raise ValueError(f"layout must be 'half' or 'interleaved', got {layout!r}")
        if table.dtype != torch.float32 or table.dim() != 2 or table.shape[0] < 1 or table.shape[1] < 2 or table.shape[1] % 2:
            raise ValueError(f"table must be float32 [positions, even rotary_dim], got {table.dtype} {tuple(table.shape)}")
        if not table.is_contiguous():
            raise ValueError("table must be contiguous")
        _on_one_gpu(table=table)
        self.table, self.layout = table, layout
        self.rotary_dim, self.device_index = int(table.shape[1]), table.get_device()
        self.desc = RotaryDesc(table.data_ptr(), table.shape[0], table.shape[1],
                               NNJIT_ROTARY_HALF if layout == "half" else NNJIT_ROTARY_INTERLEAVED)
        self.address = ctypes.addressof(self.desc)


def rotary_table(positions: int, rotary_dim: int, base: float = 10000.0, layout: str = "half",
                 scaling: Optional[RotaryScaling] = None, device="cuda", stream=None) -> RotaryTable:
    """A RotaryTable for positions 0 .. positions - 1 (nnjit_rotary_fill)."""
    torch = _torch()
    table = _empty((positions, rotary_dim), torch.float32, torch.device(device), stream)
    _launch(nnjit_rotary_fill, table.get_device(), stream, table, positions, rotary_dim, base, scaling)
    return RotaryTable(table, layout)


class PagedCache:
    """A pool of pages of keys and values: ``k`` and ``v`` fp32 or fp16
    [pages, page_size, kv_heads, head_dim], any strides with contiguous dims
    (a [pages, kv_heads, page_size, head_dim] pool is passed as its
    ``transpose(1, 2)``)."""

    def __init__(self, k, v):
        _torch()
        for name, t in (("k", k), ("v", v)):
            if t.dim() != 4 or 0 in t.shape:
                raise ValueError(f"{name} must be [pages, page_size, kv_heads, head_dim], got {tuple(t.shape)}")
            if t.dtype not in _CODES:
                raise TypeError(f"unsupported dtype {t.dtype}")
            _unit_dims(name, t)
            _separate(name, t)
        if k.shape != v.shape or k.dtype != v.dtype:
            raise ValueError(f"k is {k.dtype} {tuple(k.shape)} but v is {v.dtype} {tuple(v.shape)}")
        _on_one_gpu(k=k, v=v)
        self.k, self.v, self.dtype, self.device_index = k, v, k.dtype, k.get_device()
        pages, page_size, self.kv_heads, self.head_dim = k.shape
        self.desc = PagedKvDesc(k.data_ptr(), v.data_ptr(), k.stride(0), k.stride(1), k.stride(2), v.stride(0), v.stride(1),
                                v.stride(2), pages, page_size, self.kv_heads, self.head_dim, _CODES[k.dtype])
        self.address = ctypes.addressof(self.desc)


class PagedBatch:
    """The sequences of one step (nnjit_paged_batch): ``q_start`` int32
    [sequences + 1], ``kv_len`` int32 [sequences], ``page_table`` int32
    [sequences, columns], all on the GPU; ``tokens`` rows of q, k, v and out;
    ``max_q`` / ``max_kv`` bound the new tokens and keys of a sequence (default:
    all rows; all that the table's columns hold)."""

    def __init__(self, q_start, kv_len, page_table, tokens: int, max_q: Optional[int] = None, max_kv: Optional[int] = None):
        sequences = int(kv_len.shape[0]) if kv_len.dim() == 1 else -1
        _int32("kv_len", kv_len, max(sequences, 0))
        _int32("q_start", q_start, sequences + 1)
        _int32("page_table", page_table, sequences, None)
        _unit_dims("page_table", page_table)
        if sequences > 1 and page_table.stride(0) < page_table.shape[1]:
            raise ValueError("rows of page_table overlap")
        _on_one_gpu(q_start=q_start, kv_len=kv_len, page_table=page_table)
        self.q_start, self.kv_len, self.page_table = q_start, kv_len, page_table
        self.tokens, self.device_index = int(tokens), q_start.get_device()
        self.desc = PagedBatchDesc(sequences, tokens, q_start.data_ptr(), kv_len.data_ptr(), page_table.data_ptr(),
                                   max(page_table.stride(0), page_table.shape[1]), page_table.shape[1],
                                   tokens if max_q is None else max_q, 1 << 30 if max_kv is None else max_kv)
        self.address = ctypes.addressof(self.desc)


def _head_rows(name: str, t, tokens, heads, dim, dtype, device_index):
    """Strides (token, head) of head rows, checked."""
    st = t.stride()
    if t.shape == (tokens, heads, dim) and t.dtype is dtype and st[2] == 1 and t.get_device() == device_index:
        return st
    if t.dim() != 3 or t.shape[0] != tokens or t.shape[1] != heads or t.shape[2] != dim:
        raise ValueError(f"{name} must be [{tokens}, {heads}, {dim}], got {tuple(t.shape)}")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if st[2] != 1 and dim > 1:
        raise ValueError(f"{name} must have unit stride along the last dimension")
    if not t.is_cuda or t.get_device() != device_index:
        raise ValueError(f"{name} must be on one GPU with the other operands, got {t.device}")
    return st


def _written_rows(name: str, t, tokens, heads, dim, dtype, device_index):
    st = _head_rows(name, t, tokens, heads, dim, dtype, device_index)
    if not (st[1] >= dim and st[0] >= st[1] * heads):     # plain rows need no closer look
        _separate(name, t)
    return st


def _rows_in_and_out(name: str, x, out_name: str, out, shape, dtype, out_dtype, device_index):
    """Strides of head rows x and out of this shape, checked; plain ones by as few tensor accesses as that takes."""
    sx, so = x.stride(), out.stride()
    if not (x.shape == shape and out.shape == shape and x.dtype is dtype and out.dtype is out_dtype and sx[2] == 1 and so[2] == 1
            and so[1] >= shape[2] and so[0] >= so[1] * shape[1] and x.get_device() == device_index and out.get_device() == device_index):
        sx = _head_rows(name, x, *shape, dtype, device_index)
        so = _written_rows(out_name, out, *shape, out_dtype, device_index)
    return sx, so


def rotary(x, positions, table: RotaryTable, out=None, transpose: bool = False, stream=None):
    """x [tokens, heads, head_dim] turned by the angles of positions (int32
    [tokens]); ``transpose``: by the opposite ones (the gradient).  ``out``
    (fp32 or fp16, allocated like x if None) may be x."""
    torch = _torch()
    shape = x.shape
    if len(shape) != 3:
        raise ValueError(f"x must be [tokens, heads, head_dim], got {tuple(shape)}")
    tokens, heads, dim = shape
    if out is None:
        out = _empty((tokens, heads, dim), x.dtype, x.device, stream)
    xd, yd, dev = x.dtype, out.dtype, table.device_index
    if xd not in _CODES or yd not in _CODES:
        raise TypeError(f"unsupported dtype {xd} to {yd}")
    sx = _head_rows("x", x, tokens, heads, dim, xd, dev)
    sy = _written_rows("out", out, tokens, heads, dim, yd, dev)
    if positions.shape != (tokens,) or positions.dtype is not torch.int32 or positions.get_device() != dev:
        raise ValueError(f"positions must be int32 of shape ({tokens},) on x's GPU, got {positions.dtype} {tuple(positions.shape)}")
    if tokens > 1 and positions.stride(0) != 1:
        raise ValueError("positions must be contiguous")
    _launch((_lib or load()).nnjit_rotary, dev, stream, table.address, tokens, heads, dim, positions.data_ptr(), x.data_ptr(),
            sx[0], sx[1], _CODES[xd], out.data_ptr(), sy[0], sy[1], _CODES[yd], 1 if transpose else 0)
    return out


def kv_append(cache: PagedCache, batch: PagedBatch, k, v, rotary: Optional[RotaryTable] = None, q=None, q_out=None,
              stream=None):
    """Writes k (turned) and v [tokens, kv_heads, head_dim], fp32 or fp16, to
    the batch's slots of the cache; turns q [tokens, heads, head_dim] of the
    same type into q_out (of the cache's type, allocated if None), which is
    returned (None without q).  ``rotary`` has to hold every position that the
    sequences reach: later ones are turned by its last angles."""
    _torch()
    n, dim, dev = batch.tokens, cache.head_dim, cache.device_index
    dt = k.dtype
    if dt not in _CODES:
        raise TypeError(f"unsupported dtype {dt}")
    if batch.device_index != dev or (rotary is not None and rotary.device_index != dev):
        raise ValueError("cache, batch and rotary must be on one GPU")
    sk = _head_rows("k", k, n, cache.kv_heads, dim, dt, dev)
    sv = _head_rows("v", v, n, cache.kv_heads, dim, dt, dev)
    heads, sq, so, qp, op = 0, (0, 0), (0, 0), None, None
    if q is not None:
        heads = q.shape[1] if q.dim() == 3 else -1
        sq = _head_rows("q", q, n, heads, dim, dt, dev)
        if q_out is None:
            q_out = _empty((n, heads, dim), cache.dtype, q.device, stream)
        so = _written_rows("q_out", q_out, n, heads, dim, cache.dtype, dev)
        qp, op = q.data_ptr(), q_out.data_ptr()
    elif q_out is not None:
        raise ValueError("q_out without q")
    _launch((_lib or load()).nnjit_kv_append, dev, stream, cache.address, batch.address,
            None if rotary is None else rotary.address, k.data_ptr(), sk[0], sk[1], v.data_ptr(), sv[0], sv[1], heads, qp,
            sq[0], sq[1], op, so[0], so[1], _CODES[dt])
    return q_out


def paged_attention(q, cache: PagedCache, batch: PagedBatch, out=None, scale: Optional[float] = None, causal: bool = True,
                    window: int = 0, stream=None):
    """Attention of q [tokens, heads, head_dim] over the cached keys and values
    of every row's sequence; q and out are of the cache's type.  ``scale``
    defaults to head_dim ** -0.5; ``window`` > 0: the last ``window`` keys only."""
    _torch()
    shape = q.shape
    if len(shape) != 3:
        raise ValueError(f"q must be [tokens, heads, head_dim], got {tuple(shape)}")
    heads, dim, dev = shape[1], cache.head_dim, cache.device_index
    if batch.device_index != dev:
        raise ValueError("cache and batch must be on one GPU")
    sq = _head_rows("q", q, batch.tokens, heads, dim, cache.dtype, dev)
    if out is None:
        out = _empty((batch.tokens, heads, dim), cache.dtype, q.device, stream)
    so = _written_rows("out", out, batch.tokens, heads, dim, cache.dtype, dev)
    _launch((_lib or load()).nnjit_paged_attention, dev, stream, cache.address, batch.address, heads, q.data_ptr(), sq[0],
            sq[1], out.data_ptr(), so[0], so[1], dim ** -0.5 if scale is None else scale, 1 if causal else 0, window)
    return out


class PagePool:
    """The free pages of a cache: ``free_pages`` int32 [capacity], a stack whose
    first ``count`` (int32 [1]) ids are free; a step writes the new count to
    ``count_out`` (default: ``count`` itself)."""

    def __init__(self, free_pages, count, count_out=None):
        _torch()
        count_out = count if count_out is None else count_out
        _int32("free_pages", free_pages, None)
        _int32("count", count, 1)
        _int32("count_out", count_out, 1)
        _on_one_gpu(free_pages=free_pages, count=count, count_out=count_out)
        self.free_pages, self.count, self.count_out, self.device_index = free_pages, count, count_out, count.get_device()
        self.desc = PagePoolDesc(free_pages.data_ptr(), free_pages.shape[0], count.data_ptr(), count_out.data_ptr())
        self.address = ctypes.addressof(self.desc)


class PagedStep:
    """The arrays of a step of up to ``tokens`` new rows, which ``paged_step``
    fills: ``q_start``, ``kv_len``, ``positions``, ``slots``, ``status`` and, with
    ``mask_words`` > 0 (32 drafted tokens of a sequence each, at most 32 words),
    ``mask``.  ``page_table`` int32 [sequences, columns] is the program's; ``kv_len``
    (default: an array of the step's own) may be the tensor that is passed as
    ``held`` or ``keep``."""

    def __init__(self, page_table, page_size: int, tokens: int, mask_words: int = 0, kv_len=None):
        torch = _torch()
        _int32("page_table", page_table, None, None)
        _unit_dims("page_table", page_table)
        sequences, columns = page_table.shape
        if sequences > 1 and page_table.stride(0) < columns:
            raise ValueError("rows of page_table overlap")
        if tokens < 0 or not 0 <= mask_words <= 32:
            raise ValueError(f"tokens must be >= 0 and mask_words 0 .. 32, got {tokens} and {mask_words}")
        if kv_len is not None:
            _int32("kv_len", kv_len, sequences)
            _on_one_gpu(page_table=page_table, kv_len=kv_len)
        else:
            _on_one_gpu(page_table=page_table)
        dev = page_table.device
        self.page_table, self.page_size, self.tokens, self.mask_words = page_table, page_size, tokens, mask_words
        self.sequences, self.device_index = sequences, page_table.get_device()
        self.q_start = torch.zeros(sequences + 1, dtype=torch.int32, device=dev)
        self.kv_len = torch.zeros(sequences, dtype=torch.int32, device=dev) if kv_len is None else kv_len
        self.positions = torch.zeros(tokens, dtype=torch.int32, device=dev)
        self.slots = torch.full((tokens,), -1, dtype=torch.int64, device=dev)
        self.mask = torch.zeros((tokens, mask_words), dtype=torch.int32, device=dev) if mask_words else None
        self.status = torch.zeros(4, dtype=torch.int32, device=dev)
        self.desc = StepDesc(sequences, tokens, None, None, None, None, page_table.data_ptr(), max(page_table.stride(0), columns), columns,
                             page_size, self.q_start.data_ptr(), self.kv_len.data_ptr(), self.positions.data_ptr(),
                             self.slots.data_ptr(), self.mask.data_ptr() if mask_words else None, mask_words, mask_words,
                             self.status.data_ptr())

    def batch(self, max_q: Optional[int] = None, max_kv: Optional[int] = None) -> PagedBatch:
        """The step as a PagedBatch over the same arrays."""
        return PagedBatch(self.q_start, self.kv_len, self.page_table, self.tokens, max_q, max_kv)


def _step_ints(name: str, t, count: int, device_index: int) -> int:
    if t.dtype is _I32 and t.shape == (count,) and t.get_device() == device_index and (count < 2 or t.stride(0) == 1):
        return t.data_ptr()
    _int32(name, t, count)
    raise ValueError(f"{name} must be on one GPU with the step, got {t.device}")


def paged_step(step: PagedStep, pool: PagePool, held, added, keep=None, parent=None, stream=None) -> PagedStep:
    """Fills the step's arrays from lengths on the GPU (nnjit_paged_step):
    sequence b holds the pages of held[b] tokens, of which keep[b] (default: all)
    stay, and gets added[b] new ones (int32 [sequences] each).  ``parent`` int32
    [tokens] makes the new tokens of a sequence a drafted tree; without it a step with masks
    gets those of chains (up to the 32 mask_words new tokens that they hold).  Unless
    ``step.status[0]`` is 0 afterwards nothing was changed and the step is empty."""
    _torch()
    n, dev = step.sequences, step.device_index
    if pool.device_index != dev:
        raise ValueError("pool and step must be on one GPU")
    d = StepDesc.from_buffer_copy(step.desc)           # (a copy: another thread may fill the step's with its own)
    d.held, d.added = _step_ints("held", held, n, dev), _step_ints("added", added, n, dev)
    if keep is not None:
        d.keep = _step_ints("keep", keep, n, dev)
    if parent is not None:
        if not step.mask_words:
            raise ValueError("parent needs a step with mask_words")
        d.parent = _step_ints("parent", parent, step.tokens, dev)
    _launch((_lib or load()).nnjit_paged_step, dev, stream, pool.address, ctypes.addressof(d))
    return step


def _norm_weight(name: str, w, dtype):
    """A norm's weight [dim] or [heads, dim] -> (heads or None, head stride)."""
    if w.dtype not in _CODES or (dtype is not None and w.dtype != dtype):
        raise TypeError(f"{name} must be float32 or float16 (both weights alike), got {w.dtype}")
    if w.dim() not in (1, 2) or w.shape[-1] < 1:
        raise ValueError(f"{name} must be [head_dim] or [heads, head_dim], got {tuple(w.shape)}")
    _unit_dims(name, w)
    if w.dim() == 1:
        return None, 0
    if w.shape[0] > 1 and w.stride(0) < w.shape[1]:
        raise ValueError(f"rows of {name} overlap")
    return int(w.shape[0]), max(int(w.stride(0)), int(w.shape[1]))


class HeadNorm:
    """Norms of query and key heads: ``q_weight`` and ``k_weight`` fp32 or fp16
    [head_dim], or [heads, head_dim] for a weight a head; None: not normed."""

    def __init__(self, q_weight=None, k_weight=None, eps: float = 1e-6):
        _torch()
        given = {n: w for n, w in (("q_weight", q_weight), ("k_weight", k_weight)) if w is not None}
        if not given:
            raise ValueError("q_weight, k_weight or both are needed")
        if not 0.0 <= eps < float("inf"):
            raise ValueError(f"eps must be finite and >= 0, got {eps}")
        dtype = next(iter(given.values())).dtype
        shapes = {n: _norm_weight(n, w, dtype) for n, w in given.items()}
        if len({w.shape[-1] for w in given.values()}) != 1:
            raise ValueError("q_weight and k_weight must be of one head_dim")
        _on_one_gpu(**given)
        one = next(iter(given.values()))
        self.q_weight, self.k_weight, self.eps, self.head_dim, self.device_index = q_weight, k_weight, eps, int(one.shape[-1]), one.get_device()
        self.q_heads, q_head = shapes.get("q_weight", (None, 0))
        self.k_heads, k_head = shapes.get("k_weight", (None, 0))
        self.desc = HeadNormDesc(_ptr(q_weight), _ptr(k_weight), q_head, k_head, _CODES[dtype], eps)
        self.address = ctypes.addressof(self.desc)


def kv_append_slots(cache: PagedCache, slots, k, v, positions=None, rotary: Optional[RotaryTable] = None, q=None, q_out=None,
                    norm: Optional[HeadNorm] = None, stream=None):
    """Writes k (normed, turned) and v [tokens, kv_heads, head_dim], fp32 or
    fp16, to slots int64 [tokens] (page * page_size + slot; negative: the row is left
    alone); norms and turns q [tokens, heads, head_dim] of the same type into
    q_out (of the cache's type, allocated if None), which is returned (None without
    q).  ``rotary`` turns by the angles of ``positions`` int32 [tokens]."""
    _torch()
    dim, dev, dt = cache.head_dim, cache.device_index, k.dtype
    code = _CODES.get(dt)
    if code is None:
        raise TypeError(f"unsupported dtype {dt}")
    if slots.dtype is not _I64 or slots.dim() != 1 or slots.get_device() != dev or (slots.shape[0] > 1 and slots.stride(0) != 1):
        raise ValueError(f"slots must be a contiguous int64 vector on the cache's GPU, got {slots.dtype} {tuple(slots.shape)}")
    n = slots.shape[0]
    pp = None
    if rotary is not None:
        if rotary.device_index != dev:
            raise ValueError("cache and rotary must be on one GPU")
        if positions is None:
            raise ValueError("rotary needs positions")
        pp = _step_ints("positions", positions, n, dev)
    shape = k.shape
    sk, sv = k.stride(), v.stride()
    if not (shape == (n, cache.kv_heads, dim) and shape == v.shape and v.dtype is dt and sk[2] == 1 and sv[2] == 1
            and k.get_device() == dev and v.get_device() == dev):
        sk = _head_rows("k", k, n, cache.kv_heads, dim, dt, dev)
        sv = _head_rows("v", v, n, cache.kv_heads, dim, dt, dev)
    heads, sq, so, qp, op = 0, (0, 0), (0, 0), None, None
    if q is not None:
        shape = q.shape
        if len(shape) != 3:
            raise ValueError(f"q must be [tokens, heads, head_dim], got {tuple(shape)}")
        heads = shape[1]
        if q_out is None:
            q_out = _empty((n, heads, dim), cache.dtype, q.device, stream)
        sq, so = _rows_in_and_out("q", q, "q_out", q_out, (n, heads, dim), dt, cache.dtype, dev)
        qp, op = q.data_ptr(), q_out.data_ptr()
    elif q_out is not None:
        raise ValueError("q_out without q")
    if norm is not None:
        if norm.device_index != dev or norm.head_dim != dim:
            raise ValueError(f"norm weights must be on the cache's GPU and of its head_dim {dim}, got {norm.head_dim}")
        if norm.k_heads not in (None, cache.kv_heads) or (heads and norm.q_heads not in (None, heads)):
            raise ValueError(f"weights of {norm.q_heads} query and {norm.k_heads} key heads for {heads} and {cache.kv_heads}")
    _launch((_lib or load()).nnjit_kv_append_slots, dev, stream, cache.address, n, slots.data_ptr(), pp,
            None if rotary is None else rotary.address, None if norm is None else norm.address, k.data_ptr(), sk[0], sk[1],
            v.data_ptr(), sv[0], sv[1], heads, qp, sq[0], sq[1], op, so[0], so[1], code)
    return q_out


def _norm_operands(x, weight, positions, table):
    """(tokens, heads, dim, device, pointer of positions, table's address, weight's head stride) of norm_rotary and its gradient."""
    shape = x.shape
    if len(shape) != 3:
        raise ValueError(f"x must be [tokens, heads, head_dim], got {tuple(shape)}")
    tokens, heads, dim = shape
    dev = x.get_device()
    if dev < 0 or weight.get_device() != dev or (table is not None and table.device_index != dev):
        raise ValueError("x, weight and table must be on one GPU")
    if x.dtype not in _CODES:
        raise TypeError(f"unsupported dtype {x.dtype}")
    if not (weight.shape == (dim,) and weight.stride(0) == 1 and weight.dtype in _CODES):       # one plain weight needs no closer look
        w_heads, w_head = _norm_weight("weight", weight, None)
        if weight.shape[-1] != dim or w_heads not in (None, heads):
            raise ValueError(f"weight must be [{dim}] or [{heads}, {dim}], got {tuple(weight.shape)}")
    else:
        w_head = 0
    if table is None:
        return tokens, heads, dim, dev, None, None, w_head
    if positions is None:
        raise ValueError("a table needs positions")
    return tokens, heads, dim, dev, _step_ints("positions", positions, tokens, dev), table.address, w_head


def norm_rotary(x, weight, positions=None, table: Optional[RotaryTable] = None, eps: float = 1e-6, out=None, stream=None):
    """x [tokens, heads, head_dim] with every head scaled to a mean square of 1,
    times weight ([head_dim] or [heads, head_dim]), turned by the angles of positions
    (int32 [tokens]; without a table: not turned).  ``out`` (fp32 or fp16,
    allocated like x if None) may be x.  The result carries no graph: its gradients are
    ``norm_rotary_grad``'s."""
    _torch()
    tokens, heads, dim, dev, pp, tp, w_head = _norm_operands(x, weight, positions, table)
    if out is None:
        out = _empty((tokens, heads, dim), x.dtype, x.device, stream)
    xd, yd = x.dtype, out.dtype
    if yd not in _CODES:
        raise TypeError(f"unsupported dtype {yd}")
    sx, sy = _rows_in_and_out("x", x, "out", out, (tokens, heads, dim), xd, yd, dev)
    _launch((_lib or load()).nnjit_norm_rotary, dev, stream, tp, tokens, heads, dim, pp, weight.data_ptr(), w_head, _CODES[weight.dtype],
            eps, x.data_ptr(), sx[0], sx[1], _CODES[xd], out.data_ptr(), sy[0], sy[1], _CODES[yd])
    return out


def norm_rotary_grad(dy, x, weight, positions=None, table: Optional[RotaryTable] = None, eps: float = 1e-6, dx=None, dweight=None,
                     stream=None):
    """(dx, dweight) of norm_rotary from its result's gradient dy: dx of x's type
    (allocated if None; may be dy or x), dweight fp32 of weight's shape."""
    torch = _torch()
    tokens, heads, dim, dev, pp, tp, w_head = _norm_operands(x, weight, positions, table)
    if dx is None:
        dx = _empty((tokens, heads, dim), x.dtype, x.device, stream)
    if dweight is None:
        dweight = _empty(tuple(weight.shape), torch.float32, x.device, stream)
    xd, dd = x.dtype, dy.dtype
    if dd not in _CODES:
        raise TypeError(f"unsupported dtype {dd}")
    sx = x.stride()
    if sx[2] != 1:
        sx = _head_rows("x", x, tokens, heads, dim, xd, dev)
    sd = _head_rows("dy", dy, tokens, heads, dim, dd, dev)
    so = _written_rows("dx", dx, tokens, heads, dim, xd, dev)
    if dweight.shape != weight.shape or dweight.dtype is not _F32 or not dweight.is_contiguous() or dweight.get_device() != dev:
        raise ValueError(f"dweight must be contiguous float32 {tuple(weight.shape)} on x's GPU, got {dweight.dtype} {tuple(dweight.shape)}")
    _launch((_lib or load()).nnjit_norm_rotary_grad, dev, stream, tp, tokens, heads, dim, pp, weight.data_ptr(), w_head,
            _CODES[weight.dtype], eps, x.data_ptr(), sx[0], sx[1], _CODES[xd], dy.data_ptr(), sd[0], sd[1], _CODES[dd],
            dx.data_ptr(), so[0], so[1], dweight.data_ptr())
    return dx, dweight


def tree_attention(q, cache: PagedCache, batch: PagedBatch, mask, out=None, scale: Optional[float] = None, positions=None,
                   window: int = 0, stream=None):
    """Attention of drafted tokens q [tokens, heads, head_dim] over the keys
    before their sequence's new ones and over those new ones that mask (int32
    [tokens, words], bit i % 32 of word i / 32: new token i) names.  ``window`` > 0: of
    the keys before the new ones the last only, those above positions (int32
    [tokens]) - window.  Otherwise as ``paged_attention``."""
    _torch()
    shape = q.shape
    if len(shape) != 3:
        raise ValueError(f"q must be [tokens, heads, head_dim], got {tuple(shape)}")
    heads, dim, dev, n = shape[1], cache.head_dim, cache.device_index, batch.tokens
    if batch.device_index != dev:
        raise ValueError("cache and batch must be on one GPU")
    ms = mask.shape
    if len(ms) != 2 or ms[0] != n or ms[1] < 1 or mask.dtype is not _I32 or mask.get_device() != dev:
        raise ValueError(f"mask must be int32 [{n}, words] on the cache's GPU, got {mask.dtype} {tuple(ms)}")
    words = ms[1]
    ld, step = mask.stride()
    if words > 1 and step != 1:
        raise ValueError("mask must have unit stride along the last dimension")
    pp = None
    if window > 0:
        if positions is None:
            raise ValueError("a window needs positions")
        pp = _step_ints("positions", positions, n, dev)
    if out is None:
        out = _empty((n, heads, dim), cache.dtype, q.device, stream)
    sq, so = _rows_in_and_out("q", q, "out", out, (n, heads, dim), cache.dtype, cache.dtype, dev)
    _launch((_lib or load()).nnjit_tree_attention, dev, stream, cache.address, batch.address, mask.data_ptr(), ld, words, pp, heads,
            q.data_ptr(), sq[0], sq[1], out.data_ptr(), so[0], so[1], dim ** -0.5 if scale is None else scale, window)
    return out


def kv_move(cache: PagedCache, batch: PagedBatch, path, accepted, stream=None) -> None:
    """Keys and values of the accepted nodes of each drafted tree go to the
    places behind the cached ones: new token path[b, i] of sequence b to the place
    of its new token i, i < accepted[b] (path int32 [sequences, nodes], accepted int32
    [sequences]), as if all were read before any is written."""
    _torch()
    dev, sequences = cache.device_index, batch.kv_len.shape[0]
    if batch.device_index != dev:
        raise ValueError("cache and batch must be on one GPU")
    if path.dtype is not _I32 or path.dim() != 2 or path.shape[0] != sequences:
        raise ValueError(f"path must be int32 [{sequences}, nodes], got {path.dtype} {tuple(path.shape)}")
    nodes, ld = path.shape[1], path.stride(0)
    if path.get_device() != dev or (nodes > 1 and path.stride(1) != 1) or (sequences > 1 and ld < nodes):
        raise ValueError(f"path must be rows of their own on the cache's GPU with unit stride along the last dimension, got {path.device} {tuple(path.stride())}")
    _launch((_lib or load()).nnjit_kv_move, dev, stream, cache.address, batch.address, path.data_ptr(), ld if ld > nodes else nodes, nodes,
            _step_ints("accepted", accepted, sequences, dev))


class LogitRules:
    """What adjust_logits applies to ``rows`` rows of logits (nnjit_logit_rules);
    each is optional: ``history`` int32 [rows, columns] with ``length`` and
    ``prompt`` int32 [rows] (its tokens, and how many of them are the prompt's);
    ``repetition``, ``presence``, ``frequency`` fp32 [rows]; ``bias_token`` int32 and
    ``bias_value`` fp32 [rows, entries] (tokens outside the vocabulary, such as -1, are ignored);
    ``mask`` int32 [grammars, words], a bit a token, and ``mask_row`` int32 [rows], the
    grammar of every row, negative: none (without it row r has mask row r)."""

    def __init__(self, history=None, length=None, prompt=None, repetition=None, presence=None, frequency=None, bias_token=None,
                 bias_value=None, mask=None, mask_row=None):
        torch = _torch()
        given = {n: t for n, t in (("history", history), ("length", length), ("prompt", prompt), ("repetition", repetition),
                                   ("presence", presence), ("frequency", frequency), ("bias_token", bias_token),
                                   ("bias_value", bias_value), ("mask", mask), ("mask_row", mask_row)) if t is not None}
        if not given:
            raise ValueError("no rule is given")
        if (bias_token is None) != (bias_value is None):
            raise ValueError("bias_token and bias_value go together")
        if history is None and any(n in given for n in ("length", "prompt", "repetition", "presence", "frequency")):
            raise ValueError("lengths and penalties need a history")
        if mask is None and mask_row is not None:
            raise ValueError("mask_row without mask")
        rows = {n: int(t.shape[0]) for n, t in given.items() if t.dim() and (n != "mask" or mask_row is None)}
        if len(set(rows.values())) != 1:
            raise ValueError(f"the rules are for different numbers of rows: {rows}")
        self.rows = next(iter(rows.values()))
        for n, t in given.items():
            want = torch.float32 if n in ("repetition", "presence", "frequency", "bias_value") else torch.int32
            dims = 2 if n in ("history", "bias_token", "bias_value", "mask") else 1
            if t.dtype != want or t.dim() != dims:
                raise ValueError(f"{n} must be {want} with {dims} dimensions, got {t.dtype} {tuple(t.shape)}")
            if t.shape[-1] > 1 and t.stride(-1) != 1:
                raise ValueError(f"{n} must have unit stride along the last dimension")
        if bias_token is not None and (bias_token.shape != bias_value.shape or (self.rows > 1 and bias_token.stride(0) != bias_value.stride(0))):
            raise ValueError("bias_token and bias_value must have the same shape and strides")
        if mask is not None and mask.shape[0] < 1:
            raise ValueError("mask has no row")
        _on_one_gpu(**given)
        self.given, self.device_index = given, next(iter(given.values())).get_device()
        self.words = None if mask is None else int(mask.shape[1])
        ptr = {n: t.data_ptr() for n, t in given.items()}
        ld = {n: int(t.stride(0)) for n, t in given.items() if t.dim() == 2}
        self.desc = LogitRulesDesc(ptr.get("history"), ld.get("history", 0), 0 if history is None else history.shape[1],
                                   ptr.get("length"), ptr.get("prompt"), ptr.get("repetition"), ptr.get("presence"), ptr.get("frequency"),
                                   ptr.get("bias_token"), ptr.get("bias_value"), ld.get("bias_token", 0),
                                   0 if bias_token is None else bias_token.shape[1], ptr.get("mask"), ld.get("mask", 0),
                                   0 if mask is None else mask.shape[0], ptr.get("mask_row"))
        self.address = ctypes.addressof(self.desc)


def adjust_logits(logits, rules: LogitRules, out=None, stream=None):
    """logits [rows, vocab], fp32 or fp16, under the rules: penalties for tokens
    that are there already, biases, -infinity where a mask has no bit.  ``out`` (fp32 or
    fp16, allocated like logits if None) may be logits."""
    _torch()
    shape = logits.shape
    if len(shape) != 2:
        raise ValueError(f"logits must be [rows, vocab], got {tuple(shape)}")
    rows, vocab = shape
    dev = rules.device_index
    if out is None:
        out = _empty((rows, vocab), logits.dtype, logits.device, stream)
    if rules.rows != rows:
        raise ValueError(f"{rows} rows of logits, rules for {rules.rows}")
    if rules.words is not None and 32 * rules.words < vocab:
        raise ValueError(f"mask rows of {rules.words} words for {vocab} tokens")
    sx, sy, xc, yc = logits.stride(), out.stride(), _CODES.get(logits.dtype), _CODES.get(out.dtype)
    if not (out.shape == shape and sx[1] == 1 and sy[1] == 1 and sy[0] >= vocab and xc is not None and yc is not None
            and logits.get_device() == dev and out.get_device() == dev):       # plain rows need no closer look
        for name, t in (("logits", logits), ("out", out)):
            if t.dtype not in _CODES:
                raise TypeError(f"unsupported dtype {t.dtype}")
            if t.shape != shape or (vocab > 1 and t.stride(1) != 1) or t.get_device() != dev:
                raise ValueError(f"{name} must be [{rows}, {vocab}] with unit stride along the last dimension on the rules' GPU, got {tuple(t.shape)} on {t.device}")
        if rows > 1 and sy[0] < vocab:
            raise ValueError("rows of out overlap")
    _launch((_lib or load()).nnjit_adjust_logits, dev, stream, rules.address, rows, vocab, logits.data_ptr(), sx[0], xc,
            out.data_ptr(), sy[0], yc)
    return out


def configs() -> list:
    """Descriptions of every configuration id."""
    out = []
    for i in range(nnjit_num_configs()):
        d = {}
        for kv in nnjit_config_info(i).split():
            k, v = kv.split("=", 1)
            d[k] = int(v) if v.lstrip("-").isdigit() else v
        out.append(d)
    return out

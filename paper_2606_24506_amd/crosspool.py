"""ctypes binding of libcrosspool.so (include/crosspool.h).

Argument marshalling only: every step of the hot path runs in the library's
HIP kernels. PyTorch is used for device buffers and streams. The functions
keep the C names; ``Pool`` is a small convenience wrapper over them.

Importing this module loads the library and fails loudly if it has not been
built (``python -m paper_2606_24506_amd.build``); there is no fallback.
"""
from __future__ import annotations

import array
import ctypes as C
import os
from typing import Optional, Sequence

import numpy as np

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libcrosspool.so")

CP_OK, CP_EINVAL, CP_ENOMEM, CP_ENOSPC, CP_EHIP, CP_ESTATE = 0, -1, -2, -3, -4, -5
CP_KIND_MLA, CP_KIND_GQA = 0, 1
CP_PATH_AUTO, CP_PATH_VALU, CP_PATH_MFMA = 0, 1, 2
CP_SCHED_BALANCED, CP_SCHED_QUEUE, CP_SCHED_GRID = 0, 1, 2
CP_BACKING_BUFFER, CP_BACKING_VIRTUAL = 0, 1
CP_ROPE_HALF, CP_ROPE_INTERLEAVED = 0, 1
CP_ROPE_PLAIN, CP_ROPE_LINEAR, CP_ROPE_NTK, CP_ROPE_PARTS, CP_ROPE_TABLE = 0, 1, 2, 3, 4
CP_ROPE_BF16, CP_ROPE_F32 = 0, 1
_NAMES = {0: "CP_OK", -1: "CP_EINVAL", -2: "CP_ENOMEM", -3: "CP_ENOSPC", -4: "CP_EHIP", -5: "CP_ESTATE"}


class CrossPoolError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{_NAMES.get(status, status)}: {message}")
        self.status = status
        self.message = message


class cp_pool_desc(C.Structure):
    _fields_ = [
        ("page_tokens", C.c_int32),
        ("device", C.c_int32),
        ("pool_bytes", C.c_uint64),
        ("chunk_bytes", C.c_uint64),
        ("placement_seed", C.c_uint64),
        ("device_mem", C.c_void_p),
        ("max_requests", C.c_int32),
        ("backing", C.c_int32),
        ("max_workspace_bytes", C.c_uint64),
        ("device_pages", C.c_int32),
    ]


class cp_pool_stats_t(C.Structure):
    _fields_ = [
        ("chunks_total", C.c_uint64),
        ("chunks_used", C.c_uint64),
        ("pages_used", C.c_uint64),
        ("pages_reserved", C.c_uint64),
        ("requests_open", C.c_int32),
        ("models", C.c_int32),
        ("span_bytes", C.c_uint64),
        ("backing", C.c_int32),
        ("max_models", C.c_int32),
    ]


class cp_model_desc(C.Structure):
    _fields_ = [
        ("kind", C.c_int32),
        ("n_q_heads", C.c_int32),
        ("n_kv_heads", C.c_int32),
        ("head_dim", C.c_int32),
        ("latent_dim", C.c_int32),
        ("rope_dim", C.c_int32),
        ("softmax_scale", C.c_float),
        ("dtype", C.c_int32),
        ("n_layers", C.c_int32),
    ]


class cp_model_info_t(C.Structure):
    _fields_ = [
        ("d_k", C.c_int32),
        ("d_v", C.c_int32),
        ("kappa", C.c_int32),
        ("page_bytes", C.c_int32),
        ("pages_per_chunk", C.c_int32),
        ("row_elems", C.c_int32),
        ("n_layers", C.c_int32),
    ]


class cp_decode_opts(C.Structure):
    _fields_ = [
        ("num_splits", C.c_int32),
        ("schedule", C.c_int32),
        ("path", C.c_int32),
        ("reserved0", C.c_int32),
        ("ev_begin", C.c_void_p),
        ("ev_end", C.c_void_p),
    ]


class cp_rope_desc(C.Structure):
    _fields_ = [
        ("rot_dim", C.c_int32),
        ("layout", C.c_int32),
        ("scaling", C.c_int32),
        ("reserved0", C.c_int32),
        ("base", C.c_double),
        ("factor", C.c_double),
        ("orig_len", C.c_double),
        ("low_turns", C.c_double),
        ("high_turns", C.c_double),
        ("magnitude", C.c_double),
        ("table", C.POINTER(C.c_double)),
    ]


class cp_rope_tensor(C.Structure):
    _fields_ = [
        ("src", C.c_void_p),
        ("dst", C.c_void_p),
        ("src_token", C.c_int64),
        ("src_head", C.c_int64),
        ("dst_token", C.c_int64),
        ("dst_head", C.c_int64),
        ("heads", C.c_int32),
        ("width", C.c_int32),
        ("offset", C.c_int32),
        ("dtype", C.c_int32),
    ]


class cp_extend_opts(C.Structure):
    _fields_ = [
        ("softcap", C.c_float),
        ("window", C.c_int32),
        ("slopes", C.c_void_p),
        ("prefix", C.c_void_p),
        ("doc_begin", C.c_void_p),
        ("num_splits", C.c_int32),
        ("path", C.c_int32),
        ("rope", C.c_void_p),
    ]


class cp_tree(C.Structure):
    _fields_ = [
        ("mask", C.c_void_p),
        ("words", C.c_int32),
        ("reserved0", C.c_int32),
        ("depth", C.c_void_p),
    ]


class cp_token_rows(C.Structure):
    _fields_ = [
        ("data", C.c_void_p),
        ("len", C.c_int64),
        ("head", C.c_int64),
        ("layer", C.c_int64),
    ]


class cp_evict_opts(C.Structure):
    _fields_ = [
        ("first", C.c_int32),
        ("last", C.c_int32),
        ("new_weights", C.c_void_p),
        ("kept", C.c_void_p),
    ]


class cp_plan_model(C.Structure):
    _fields_ = [("kappa_bytes", C.c_double), ("arrival_rate", C.c_double), ("n_samples", C.c_int64),
                ("prompt_tokens", C.POINTER(C.c_int64)), ("output_tokens", C.POINTER(C.c_int64)),
                ("service_time_s", C.POINTER(C.c_double))]


class cp_plan_opts(C.Structure):
    _fields_ = [("horizon_s", C.c_double), ("n_obs", C.c_int64), ("quantile", C.c_double), ("seed", C.c_uint64),
                ("chunk_bytes", C.c_uint64)]


class cp_plan_result(C.Structure):
    _fields_ = [("quantile_bytes", C.c_double), ("mean_bytes", C.c_double), ("max_bytes", C.c_double),
                ("pool_bytes", C.c_uint64), ("n_arrivals", C.c_int64)]


def _load() -> C.CDLL:
    # PyTorch ships its own HIP runtime (soname libamdhip64.so.7, like the
    # system one). Loading torch first makes the library bind to that same
    # runtime instance, so torch's streams and allocations are valid here.
    try:
        import torch  # noqa: F401
    except ImportError:  # pragma: no cover - plain C users do not need torch
        pass
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is not built; run `python -m paper_2606_24506_amd.build`")
    lib = C.CDLL(_LIB_PATH)
    P, I32, I64, VP = C.c_void_p, C.c_int32, C.c_int64, C.c_void_p
    sig = {
        "cp_last_error": ([], C.c_char_p),
        "cp_version": ([], I32),
        "cp_pool_create": ([C.POINTER(cp_pool_desc), C.POINTER(P)], I32),
        "cp_pool_destroy": ([P], I32),
        "cp_pool_stats": ([P, C.POINTER(cp_pool_stats_t)], I32),
        "cp_model_register": ([P, C.POINTER(cp_model_desc), C.POINTER(I32)], I32),
        "cp_model_info": ([P, I32, C.POINTER(cp_model_info_t)], I32),
        "cp_request_open": ([P, I32, I64, C.POINTER(I32)], I32),
        "cp_request_close": ([P, I32], I32),
        "cp_request_len": ([P, I32, C.POINTER(I64)], I32),
        "cp_request_cursor": ([P, I32, C.POINTER(I32), C.POINTER(I32)], I32),
        "cp_request_pages": ([P, I32, I64, I64, C.POINTER(C.c_uint32)], I32),
        "cp_kv_append": ([P, I32, VP, VP, VP, VP], I32),
        "cp_attn_decode": ([P, I32, VP, VP, VP, VP, VP], I32),
        "cp_attn_decode_ex": ([P, I32, VP, VP, VP, VP, VP, C.POINTER(cp_decode_opts)], I32),
        "cp_attn_decode_noalloc": ([P, I32, VP, VP, VP, VP, VP, C.POINTER(cp_decode_opts)], I32),
        "cp_attn_decode_step": ([P, I32, VP, VP, VP, VP, VP, VP, VP, C.POINTER(cp_decode_opts)],
                                I32),
        "cp_attn_decode_layers": ([P, I32, VP, VP, VP, VP, VP, VP, VP,
                                   C.POINTER(cp_decode_opts)], I32),
        "cp_request_layer_state": ([P, I32, C.POINTER(I32), C.POINTER(I64)], I32),
        "cp_kv_gather": ([P, I32, I64, I64, VP, VP], I32),
        "cp_request_fork": ([P, I32, VP, VP, VP, VP], I32),
        "cp_request_truncate": ([P, I32, VP, VP, VP], I32),
        "cp_rope_create": ([C.POINTER(cp_rope_desc), I32, C.POINTER(P)], I32),
        "cp_rope_destroy": ([P], I32),
        "cp_rope_angles": ([P, C.POINTER(C.c_double)], I32),
        "cp_rope_apply": ([P, I32, VP, I64, VP, I64, I32, VP], I32),
        "cp_kv_append_rope": ([P, I32, VP, VP, VP, P, VP], I32),
        "cp_attn_extend": ([P, I32, VP, VP, VP, VP, VP, VP, C.POINTER(cp_extend_opts)], I32),
        "cp_attn_extend_step": ([P, I32, VP, VP, VP, VP, VP, VP, VP, C.POINTER(cp_extend_opts)], I32),
        "cp_tree_build": ([I32, I32, VP, VP, I32, VP, VP, VP], I32),
        "cp_attn_tree": ([P, I32, VP, VP, VP, VP, VP, C.POINTER(cp_tree), VP, C.POINTER(cp_extend_opts)], I32),
        "cp_attn_tree_step": ([P, I32, VP, VP, VP, VP, VP, VP, C.POINTER(cp_tree), VP, C.POINTER(cp_extend_opts)], I32),
        "cp_attn_weights": ([P, I32, VP, VP, VP, VP, I32, C.c_float, VP, VP, VP, C.POINTER(cp_extend_opts)], I32),
        "cp_request_position": ([P, I32, C.POINTER(I64)], I32),
        "cp_request_keep": ([P, I32, VP, VP, VP, VP, VP], I32),
        "cp_kv_evict": ([P, I32, VP, VP, VP, C.POINTER(cp_evict_opts), VP], I32),
        "cp_plan_pool": ([C.POINTER(cp_plan_model), I32, C.POINTER(cp_plan_opts), C.POINTER(cp_plan_result)], I32),
    }
    for name, (args, res) in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = res
    return lib


LIB = _load()


def _check(rc: int):
    if rc != CP_OK:
        raise CrossPoolError(rc, LIB.cp_last_error().decode(errors="replace"))


def _int_array(kind, code: str, xs):
    """xs as a ctypes array of the kind; one of that kind passes as it is.
    Numbers out of its range are refused (OverflowError)."""
    if isinstance(xs, C.Array) and xs._type_ is kind:
        return xs
    return (kind * len(xs)).from_buffer(array.array(code, [int(x) for x in xs]))


def i32_array(xs: Sequence[int]):
    """A host int32 array argument built once, for callers that repeat a
    call with the same request ids (it is passed as it is)."""
    return _int_array(C.c_int32, "i", list(xs))


def i64_array(xs: Sequence[int]):
    """The same of int64, for lengths."""
    return _int_array(C.c_int64, "q", list(xs))


def _i64_array(xs):
    return None if xs is None else _int_array(C.c_int64, "q", xs)


def _i32_array(xs: Sequence[int]):
    """A host int32 array argument: an array from i32_array passes as it is,
    a contiguous numpy int32 array passes its address (no copy), anything
    else (arrays of other integers too) is copied into a ctypes array."""
    if isinstance(xs, np.ndarray) and xs.dtype == np.int32 and xs.flags.c_contiguous:
        return xs.__array_interface__["data"][0]
    return _int_array(C.c_int32, "i", xs)


def _ptr(t) -> Optional[int]:
    """Device pointer of a tensor (or None / raw int)."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return t.data_ptr()


_OPTS = {}


def _event(e):
    if e is None:
        return None
    return e.cuda_event if hasattr(e, "cuda_event") else int(e)


def _opts(num_splits: int, schedule: int, path: int, ev_begin, ev_end):
    """Pointer to a cp_decode_opts; the event-free ones are built once per
    (num_splits, schedule, path) and reused."""
    if ev_begin is None and ev_end is None:
        key = (num_splits, schedule, path)
        o = _OPTS.get(key)
        if o is None:
            o = _OPTS[key] = C.pointer(cp_decode_opts(num_splits, schedule, path, 0, None, None))
        return o
    return C.pointer(cp_decode_opts(num_splits, schedule, path, 0, _event(ev_begin), _event(ev_end)))


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch

        if not torch.cuda.is_available():
            return None
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


# ------------------------------------------------------------ C names ----

def cp_version() -> int:
    return int(LIB.cp_version())


class _Known:
    """What the checks of tensor arguments need of a pool: its device, and the
    query heads of its models and open requests."""

    def __init__(self, device: int):
        self.device, self.models, self.requests = device, {}, {}
        self.kv, self.shapes = {}, {}  # (layers, KV heads) of models and open requests


_POOLS: dict = {}  # by handle


def cp_pool_create(page_tokens: int = 64, pool_bytes: int = 0, chunk_bytes: int = 0, placement_seed: int = 0,
                   device: int = 0, device_mem=None, max_requests: int = 0, backing: int = 0,
                   max_workspace_bytes: int = 0, device_pages: int = 0) -> int:
    d = cp_pool_desc(page_tokens, device, pool_bytes, chunk_bytes, placement_seed, _ptr(device_mem), max_requests,
                     backing, max_workspace_bytes, device_pages)
    out = C.c_void_p()
    _check(LIB.cp_pool_create(C.byref(d), C.byref(out)))
    _POOLS[out.value] = _Known(device)
    return out.value


def cp_pool_destroy(pool: int) -> None:
    _check(LIB.cp_pool_destroy(pool))
    _POOLS.pop(pool, None)


def cp_pool_stats(pool: int) -> dict:
    s = cp_pool_stats_t()
    _check(LIB.cp_pool_stats(pool, C.byref(s)))
    return {f: getattr(s, f) for f, _ in s._fields_}


def cp_model_register(pool: int, kind: int, n_q_heads: int, n_kv_heads: int, head_dim: int = 0,
                      latent_dim: int = 0, rope_dim: int = 0, softmax_scale: float = 0.0, n_layers: int = 1) -> int:
    m = cp_model_desc(kind, n_q_heads, n_kv_heads, head_dim, latent_dim, rope_dim, softmax_scale, 0, n_layers)
    mid = C.c_int32()
    _check(LIB.cp_model_register(pool, C.byref(m), C.byref(mid)))
    if pool in _POOLS:
        _POOLS[pool].models[mid.value] = n_q_heads
        _POOLS[pool].kv[mid.value] = (max(1, n_layers), n_kv_heads)
    return mid.value


def cp_model_info(pool: int, model_id: int) -> dict:
    s = cp_model_info_t()
    _check(LIB.cp_model_info(pool, model_id, C.byref(s)))
    return {f: getattr(s, f) for f, _ in s._fields_}


def cp_request_open(pool: int, model_id: int, reserve_tokens: int) -> int:
    rid = C.c_int32()
    _check(LIB.cp_request_open(pool, model_id, reserve_tokens, C.byref(rid)))
    if pool in _POOLS:
        _POOLS[pool].requests[rid.value] = _POOLS[pool].models.get(model_id, 0)
        _POOLS[pool].shapes[rid.value] = _POOLS[pool].kv.get(model_id)
    return rid.value


def cp_request_close(pool: int, req_id: int) -> None:
    _check(LIB.cp_request_close(pool, req_id))


def cp_request_len(pool: int, req_id: int) -> int:
    n = C.c_int64()
    _check(LIB.cp_request_len(pool, req_id, C.byref(n)))
    return n.value


def cp_request_cursor(pool: int, req_id: int):
    """(layer, in_flight) of the request's layer cursor."""
    layer, inflight = C.c_int32(), C.c_int32()
    _check(LIB.cp_request_cursor(pool, req_id, C.byref(layer), C.byref(inflight)))
    return layer.value, inflight.value


def cp_request_pages(pool: int, req_id: int, first: int, count: int, layers: int = 1) -> np.ndarray:
    """Page-table entries, [count] for one layer or [layers][count]."""
    out = np.zeros((layers, count), dtype=np.uint32)
    _check(LIB.cp_request_pages(pool, req_id, first, count, out.ctypes.data_as(C.POINTER(C.c_uint32))))
    return out[0] if layers == 1 else out


def cp_kv_append(pool: int, req_ids: Sequence[int], n_new: Sequence[int], rows, stream=None) -> None:
    n = len(req_ids)
    if len(n_new) != n:
        raise ValueError("req_ids and n_new differ in length")
    _check(LIB.cp_kv_append(pool, n, _i32_array(req_ids), _i32_array(n_new), _ptr(rows), _stream(stream)))


def cp_attn_decode(pool: int, req_ids: Sequence[int], q, out, lse, stream=None) -> None:
    _check(LIB.cp_attn_decode(pool, len(req_ids), _i32_array(req_ids), _ptr(q), _ptr(out), _ptr(lse), _stream(stream)))


def cp_attn_decode_ex(pool: int, req_ids: Sequence[int], q, out, lse, stream=None, *, num_splits: int = 0,
                      schedule: int = CP_SCHED_BALANCED, path: int = CP_PATH_AUTO, ev_begin=None,
                      ev_end=None) -> None:
    o = _opts(num_splits, schedule, path, ev_begin, ev_end)
    _check(LIB.cp_attn_decode_ex(pool, len(req_ids), _i32_array(req_ids), _ptr(q), _ptr(out), _ptr(lse),
                                 _stream(stream), o))


def cp_attn_decode_noalloc(pool: int, req_ids: Sequence[int], q, out, lse, stream=None, *, num_splits: int = 0,
                           schedule: int = CP_SCHED_BALANCED, path: int = CP_PATH_AUTO, ev_begin=None,
                           ev_end=None) -> None:
    o = _opts(num_splits, schedule, path, ev_begin, ev_end)
    _check(LIB.cp_attn_decode_noalloc(pool, len(req_ids), _i32_array(req_ids), _ptr(q), _ptr(out), _ptr(lse),
                                      _stream(stream), o))


def cp_attn_decode_step(pool: int, req_ids: Sequence[int], n_new: Sequence[int], rows, q, out, lse, stream=None, *,
                        num_splits: int = 0, schedule: int = CP_SCHED_BALANCED, path: int = CP_PATH_AUTO,
                        ev_begin=None, ev_end=None) -> None:
    n = len(req_ids)
    if len(n_new) != n:
        raise ValueError("req_ids and n_new differ in length")
    o = _opts(num_splits, schedule, path, ev_begin, ev_end)
    _check(LIB.cp_attn_decode_step(pool, n, _i32_array(req_ids), _i32_array(n_new), _ptr(rows), _ptr(q), _ptr(out),
                                   _ptr(lse), _stream(stream), o))


def cp_attn_decode_layers(pool: int, req_ids: Sequence[int], n_new: Sequence[int], rows, q, out, lse, stream=None, *,
                          num_splits: int = 0, schedule: int = CP_SCHED_BALANCED, path: int = CP_PATH_AUTO,
                          ev_begin=None, ev_end=None) -> None:
    o = _opts(num_splits, schedule, path, ev_begin, ev_end)
    n = len(req_ids)
    _check(LIB.cp_attn_decode_layers(pool, n, _i32_array(req_ids), _i32_array(n_new), _ptr(rows), _ptr(q), _ptr(out),
                                     _ptr(lse), _stream(stream), o))


def cp_request_layer_state(pool: int, req_id: int):
    layer, tokens = C.c_int32(), C.c_int64()
    _check(LIB.cp_request_layer_state(pool, req_id, C.byref(layer), C.byref(tokens)))
    return layer.value, tokens.value


def cp_kv_gather(pool: int, req_id: int, start: int, n_tok: int, dst, stream=None) -> None:
    _check(LIB.cp_kv_gather(pool, req_id, start, n_tok, _ptr(dst), _stream(stream)))


def cp_request_fork(pool: int, src_ids: Sequence[int], dst_ids: Sequence[int], n_tok=None, stream=None) -> None:
    n = len(dst_ids)
    if len(src_ids) != n or (n_tok is not None and len(n_tok) != n):
        raise ValueError("src_ids, dst_ids and n_tok differ in length")
    _check(LIB.cp_request_fork(pool, n, _i32_array(src_ids), _i32_array(dst_ids), _i64_array(n_tok), _stream(stream)))


def cp_request_truncate(pool: int, req_ids: Sequence[int], new_len: Sequence[int], stream=None) -> None:
    n = len(req_ids)
    if len(new_len) != n:
        raise ValueError("req_ids and new_len differ in length")
    _check(LIB.cp_request_truncate(pool, n, _i32_array(req_ids), _i64_array(new_len), _stream(stream)))


def cp_rope_create(rot_dim: int, device: int = 0, layout: int = CP_ROPE_HALF, scaling: int = CP_ROPE_PLAIN,
                   base: float = 10000.0, factor: float = 1.0, orig_len: float = 0.0, low_turns: float = 1.0,
                   high_turns: float = 32.0, magnitude: float = 0.0, table=None) -> int:
    tab = None if table is None else (C.c_double * len(table))(*[float(x) for x in table])
    if tab is not None and len(tab) != rot_dim // 2:
        raise ValueError("table holds rot_dim / 2 angles")
    d = cp_rope_desc(rot_dim, layout, scaling, 0, base, factor, orig_len, low_turns, high_turns, magnitude, tab)
    out = C.c_void_p()
    _check(LIB.cp_rope_create(C.byref(d), device, C.byref(out)))
    return out.value


def cp_rope_destroy(rope: int) -> None:
    _check(LIB.cp_rope_destroy(rope))


def cp_rope_angles(rope: int, rot_dim: int) -> np.ndarray:
    out = np.zeros(rot_dim // 2)
    _check(LIB.cp_rope_angles(rope, out.ctypes.data_as(C.POINTER(C.c_double))))
    return out


def rope_parts(pairs, offset: int = 0):
    """The tensor records of cp_rope_apply, built once for callers that repeat
    a call: (src, dst) tensors [tokens][heads][width], bf16 or float32, whose
    last dimension is contiguous; dst may be src. Elements [offset, offset +
    rot_dim) of each head are rotated."""
    import torch

    pairs = list(pairs)
    arr = (cp_rope_tensor * len(pairs))()
    tokens = None
    for i, (s, d) in enumerate(pairs):
        if s.dim() != 3 or s.shape != d.shape or s.dtype != d.dtype:
            raise ValueError("src and dst are [tokens][heads][width] of one dtype")
        if s.dtype not in (torch.bfloat16, torch.float32):
            raise ValueError("rotated tensors are bf16 or float32")
        if any(t.stride(2) != 1 and t.shape[2] > 1 for t in (s, d)):
            raise ValueError("the last dimension must be contiguous")
        if tokens not in (None, s.shape[0]):
            raise ValueError("the tensors differ in tokens")
        if s.device != d.device or s.device.type != "cuda" or s.device != pairs[0][0].device:
            raise ValueError("the tensors are on one GPU")
        tokens = s.shape[0]
        arr[i] = cp_rope_tensor(s.data_ptr(), d.data_ptr(), s.stride(0), s.stride(1), d.stride(0), d.stride(1),
                                s.shape[1], s.shape[2], offset, CP_ROPE_F32 if s.dtype == torch.float32 else CP_ROPE_BF16)
    arr.tokens, arr.keep, arr.device = tokens or 0, pairs, pairs[0][0].device.index if pairs else None
    return arr


def cp_rope_apply(rope: int, parts, positions=None, first: int = 0, inverse: bool = False, stream=None) -> None:
    """parts: from rope_parts. positions: int32 device tensor (or address) with
    one entry per token, or None: first, first + 1, ..."""
    if hasattr(positions, "dtype") and (str(positions.dtype) != "torch.int32" or positions.numel() != parts.tokens or
                                        not positions.is_cuda or
                                        getattr(parts, "device", None) not in (None, positions.device.index)):
        raise ValueError("positions holds one int32 per token, on the GPU of the tensors")
    _check(LIB.cp_rope_apply(rope, len(parts), parts, parts.tokens, _ptr(positions), first, int(inverse),
                             _stream(stream)))


def _rope(rope) -> Optional[int]:
    if isinstance(rope, Rope):
        if not rope.handle:
            raise ValueError("the rotation is destroyed")
        return rope.handle
    return rope


def cp_kv_append_rope(pool: int, req_ids: Sequence[int], n_new: Sequence[int], rows, rope, stream=None) -> None:
    n = len(req_ids)
    if len(n_new) != n:
        raise ValueError("req_ids and n_new differ in length")
    _check(LIB.cp_kv_append_rope(pool, n, _i32_array(req_ids), _i32_array(n_new), _ptr(rows), _rope(rope),
                                 _stream(stream)))


def _extend_opts(pool, req_ids, n_q, tensors, softcap, window, slopes, prefix, doc_begin, num_splits, path, rope):
    n, known = len(req_ids), _POOLS.get(pool)
    for t in (*tensors, slopes, doc_begin):
        if hasattr(t, "is_cuda") and not (t.is_cuda and (known is None or t.device.index == known.device)):
            raise ValueError("tensors of attention are on the GPU of the pool")
    if hasattr(slopes, "dtype"):
        heads = known.requests.get(int(req_ids[0]), 0) if known and n else 0
        if str(slopes.dtype) != "torch.float32" or slopes.numel() < heads:
            raise ValueError("slopes holds one float32 per query head")
    if hasattr(doc_begin, "dtype") and (str(doc_begin.dtype) != "torch.int32" or doc_begin.numel() != sum(n_q)):
        raise ValueError("doc_begin holds one int32 per query token")
    if prefix is not None:
        if len(prefix) != n:
            raise ValueError("prefix and req_ids differ in length")
        prefix = _i32_array(prefix)
    o = cp_extend_opts(softcap, window, _ptr(slopes), None, _ptr(doc_begin), num_splits, path, _rope(rope))
    if prefix is not None:
        o.prefix = prefix if isinstance(prefix, int) else C.addressof(prefix)
        o.keep = prefix
    return o


def cp_attn_extend(pool: int, req_ids: Sequence[int], n_q: Sequence[int], q, out, lse, stream=None, *,
                   softcap: float = 0.0, window: int = 0, slopes=None, prefix=None, doc_begin=None,
                   num_splits: int = 0, path: int = CP_PATH_AUTO) -> None:
    n = len(req_ids)
    if len(n_q) != n:
        raise ValueError("req_ids and n_q differ in length")
    o = _extend_opts(pool, req_ids, n_q, (q, out, lse), softcap, window, slopes, prefix, doc_begin, num_splits, path, None)
    _check(LIB.cp_attn_extend(pool, n, _i32_array(req_ids), _i32_array(n_q), _ptr(q), _ptr(out), _ptr(lse),
                              _stream(stream), C.byref(o)))


def cp_attn_extend_step(pool: int, req_ids: Sequence[int], n_new: Sequence[int], rows, q, out, lse, stream=None, *,
                        rope=None, softcap: float = 0.0, window: int = 0, slopes=None, prefix=None, doc_begin=None,
                        num_splits: int = 0, path: int = CP_PATH_AUTO) -> None:
    n = len(req_ids)
    if len(n_new) != n:
        raise ValueError("req_ids and n_new differ in length")
    o = _extend_opts(pool, req_ids, n_new, (rows, q, out, lse), softcap, window, slopes, prefix, doc_begin, num_splits, path, rope)
    _check(LIB.cp_attn_extend_step(pool, n, _i32_array(req_ids), _i32_array(n_new), _ptr(rows), _ptr(q), _ptr(out),
                                   _ptr(lse), _stream(stream), C.byref(o)))


_DTYPES: dict = {}


def _dtype(t) -> str:
    """The name of a tensor's type (each looked up once: str() takes a microsecond)."""
    name = _DTYPES.get(t.dtype)
    if name is None:
        name = _DTYPES[t.dtype] = str(t.dtype)
    return name


def _tree(known, n_q, mask, depth):
    """The record of a call's trees: mask int32 [tokens][words], depth int32
    [tokens], on the GPU."""
    total = sum(n_q)
    if mask.dim() != 2 or mask.shape[0] != total or depth.numel() != total:
        raise ValueError("mask is [tokens][words] and depth [tokens] of the call's trees")
    for t in (mask, depth):
        if _dtype(t) != "torch.int32" or not t.is_cuda or (known is not None and t.device.index != known.device):
            raise ValueError("mask and depth are int32, on the GPU of the pool")
    return cp_tree(_ptr(mask), mask.shape[1], 0, _ptr(depth))


def cp_tree_build(n_tok: Sequence[int], parents, mask, depth, stream=None) -> None:
    """parents int32 [tokens of every tree]; mask int32 [tokens][words] and depth
    int32 [tokens] are written. All on one GPU."""
    total = sum(n_tok)
    if parents.numel() != total or _dtype(parents) != "torch.int32":
        raise ValueError("parents holds one int32 per token")
    t = _tree(None, n_tok, mask, depth)
    device = mask.device
    if parents.device != device or depth.device != device:
        raise ValueError("the tensors are on one GPU")
    _check(LIB.cp_tree_build(device.index, len(n_tok), _i32_array(n_tok), _ptr(parents), t.words, t.mask, t.depth,
                             _stream(stream)))


def cp_attn_tree(pool: int, req_ids: Sequence[int], n_q: Sequence[int], q, out, lse, mask, depth, stream=None, *,
                 softcap: float = 0.0, window: int = 0, slopes=None, doc_begin=None, num_splits: int = 0,
                 path: int = CP_PATH_AUTO) -> None:
    n = len(req_ids)
    if len(n_q) != n:
        raise ValueError("req_ids and n_q differ in length")
    t = _tree(_POOLS.get(pool), n_q, mask, depth)
    o = _extend_opts(pool, req_ids, n_q, (q, out, lse), softcap, window, slopes, None, doc_begin, num_splits, path, None)
    _check(LIB.cp_attn_tree(pool, n, _i32_array(req_ids), _i32_array(n_q), _ptr(q), _ptr(out), _ptr(lse), C.byref(t),
                            _stream(stream), C.byref(o)))


def cp_attn_tree_step(pool: int, req_ids: Sequence[int], n_new: Sequence[int], rows, q, out, lse, mask, depth,
                      stream=None, *, rope=None, softcap: float = 0.0, window: int = 0, slopes=None, doc_begin=None,
                      num_splits: int = 0, path: int = CP_PATH_AUTO) -> None:
    n = len(req_ids)
    if len(n_new) != n:
        raise ValueError("req_ids and n_new differ in length")
    t = _tree(_POOLS.get(pool), n_new, mask, depth)
    o = _extend_opts(pool, req_ids, n_new, (rows, q, out, lse), softcap, window, slopes, None, doc_begin, num_splits, path, rope)
    _check(LIB.cp_attn_tree_step(pool, n, _i32_array(req_ids), _i32_array(n_new), _ptr(rows), _ptr(q), _ptr(out),
                                 _ptr(lse), C.byref(t), _stream(stream), C.byref(o)))


def token_rows(tensors):
    """The records of what a call's requests keep per token, built once for
    callers that repeat a call: one tensor per request, [KV heads][tokens] or
    [layers][KV heads][tokens], float32 (sums) or int32 (token numbers), the last
    dimension contiguous."""
    tensors = list(tensors)
    arr = (cp_token_rows * len(tensors))()
    for i, t in enumerate(tensors):
        if t.dim() not in (2, 3) or (t.shape[-1] > 1 and t.stride(-1) != 1):
            raise ValueError("rows are [KV heads][tokens] or [layers][KV heads][tokens], tokens contiguous")
        if str(t.dtype) not in ("torch.float32", "torch.int32") or t.dtype != tensors[0].dtype:
            raise ValueError("rows are float32 or int32")
        if not t.is_cuda or t.device != tensors[0].device:
            raise ValueError("rows are on one GPU")
        arr[i] = cp_token_rows(t.data_ptr(), t.shape[-1], t.stride(-2), t.stride(0) if t.dim() == 3 else 0)
    arr.keep = tensors
    arr.shapes = {(t.shape[0] if t.dim() == 3 else 1, t.shape[-2]) for t in tensors}  # (layers, KV heads)
    arr.floats = str(tensors[0].dtype) == "torch.float32" if tensors else None
    arr.device = tensors[0].device.index if tensors else None
    return arr


def _rows_arg(pool, req_ids, rows, floats: bool):
    """Records of token_rows (or tensors), one per request of the call and as many
    rows as its model has KV heads and layers."""
    if rows is None:
        return None
    if not isinstance(rows, C.Array):
        rows = token_rows(rows)
    known = _POOLS.get(pool)
    if len(rows) != len(req_ids):
        raise ValueError("one record of rows per request")
    if rows.floats not in (None, floats):
        raise ValueError("sums are float32, token numbers int32")
    if known is not None:
        if rows.device not in (None, known.device):
            raise ValueError("rows are on the GPU of the pool")
        # (the requests of a call are of one model, or the call is refused)
        shape = known.shapes.get(int(req_ids[0])) if len(req_ids) else None
        if shape is not None and rows.shapes - {shape}:
            raise ValueError("rows for every layer and KV head of the requests' model")
    return rows


def cp_attn_weights(pool: int, req_ids: Sequence[int], n_q: Sequence[int], q, lse, new, stream=None, *, old=None,
                    decay: float = 1.0, layer: int = 0, softcap: float = 0.0, window: int = 0, slopes=None, prefix=None,
                    doc_begin=None, num_splits: int = 0, path: int = CP_PATH_AUTO) -> None:
    """new (written) and old: token_rows of the requests' sums, or their tensors."""
    n = len(req_ids)
    if len(n_q) != n:
        raise ValueError("req_ids and n_q differ in length")
    o = _extend_opts(pool, req_ids, n_q, (q, lse), softcap, window, slopes, prefix, doc_begin, num_splits, path, None)
    new, old = _rows_arg(pool, req_ids, new, True), _rows_arg(pool, req_ids, old, True)
    _check(LIB.cp_attn_weights(pool, n, _i32_array(req_ids), _i32_array(n_q), _ptr(q), _ptr(lse), layer, decay, old, new,
                               _stream(stream), C.byref(o)))


def cp_request_position(pool: int, req_id: int) -> int:
    n = C.c_int64()
    _check(LIB.cp_request_position(pool, req_id, C.byref(n)))
    return n.value


def cp_request_keep(pool: int, req_ids: Sequence[int], first: Sequence[int], n_keep: Sequence[int], keep: Sequence[int],
                    stream=None) -> None:
    """keep: the requests' lists one behind the other, n_keep[i] entries each."""
    n = len(req_ids)
    if len(first) != n or len(n_keep) != n:
        raise ValueError("req_ids, first and n_keep differ in length")
    if len(keep) != sum(n_keep):
        raise ValueError("keep holds n_keep entries of each request")
    _check(LIB.cp_request_keep(pool, n, _i32_array(req_ids), _i64_array(first), _i32_array(n_keep), _i32_array(keep),
                               _stream(stream)))


def cp_kv_evict(pool: int, req_ids: Sequence[int], n_keep: Sequence[int], weights, stream=None, *, new=None, kept=None,
                first: int = 0, last: int = 0) -> None:
    """weights, new (float32) and kept (int32): token_rows, or their tensors."""
    n = len(req_ids)
    if len(n_keep) != n:
        raise ValueError("req_ids and n_keep differ in length")
    weights, new = _rows_arg(pool, req_ids, weights, True), _rows_arg(pool, req_ids, new, True)
    kept = _rows_arg(pool, req_ids, kept, False)
    o = cp_evict_opts(first, last, None if new is None else C.addressof(new), None if kept is None else C.addressof(kept))
    _check(LIB.cp_kv_evict(pool, n, _i32_array(req_ids), _i64_array(n_keep), weights, C.byref(o), _stream(stream)))


def cp_plan_pool(models, horizon_s: float, n_obs: int, quantile: float, seed: int, chunk_bytes: int = 2 << 20) -> dict:
    """models: sequence of dicts with kappa_bytes, arrival_rate and equal-length
    prompt_tokens / output_tokens / service_time_s sequences (trace records)."""
    keep = []
    arr = (cp_plan_model * len(models))()
    for i, m in enumerate(models):
        op = (C.c_int64 * len(m["prompt_tokens"]))(*[int(x) for x in m["prompt_tokens"]])
        od = (C.c_int64 * len(m["output_tokens"]))(*[int(x) for x in m["output_tokens"]])
        tr = (C.c_double * len(m["service_time_s"]))(*[float(x) for x in m["service_time_s"]])
        if not (len(op) == len(od) == len(tr)):
            raise ValueError("trace columns differ in length")
        keep += [op, od, tr]
        arr[i] = cp_plan_model(float(m["kappa_bytes"]), float(m["arrival_rate"]), len(op), op, od, tr)
    o = cp_plan_opts(float(horizon_s), int(n_obs), float(quantile), int(seed) & ((1 << 64) - 1), int(chunk_bytes))
    r = cp_plan_result()
    _check(LIB.cp_plan_pool(arr, len(models), C.byref(o), C.byref(r)))
    return dict(quantile_bytes=r.quantile_bytes, mean_bytes=r.mean_bytes, max_bytes=r.max_bytes,
                pool_bytes=r.pool_bytes, n_arrivals=r.n_arrivals)


# -------------------------------------------------------- convenience ----

class Rope:
    """Owns one cp_rope handle. layout: "half" or "interleaved"; scaling:
    "none", "linear", "ntk", "parts" or "table"."""

    _LAYOUT = {"half": CP_ROPE_HALF, "interleaved": CP_ROPE_INTERLEAVED}
    _SCALING = {"none": CP_ROPE_PLAIN, "linear": CP_ROPE_LINEAR, "ntk": CP_ROPE_NTK, "parts": CP_ROPE_PARTS,
                "table": CP_ROPE_TABLE}

    def __init__(self, rot_dim: int, device: int = 0, layout: str = "half", scaling: str = "none", **desc):
        self.handle = None
        if layout not in self._LAYOUT or scaling not in self._SCALING:
            raise ValueError(f"unknown layout {layout!r} or scaling {scaling!r}")
        self.rot_dim, self.device = rot_dim, device
        self.handle = cp_rope_create(rot_dim, device, self._LAYOUT[layout], self._SCALING[scaling], **desc)

    def angles(self) -> np.ndarray:
        return cp_rope_angles(_rope(self), self.rot_dim)

    def apply(self, parts, positions=None, first: int = 0, inverse: bool = False, stream=None) -> None:
        if parts.device not in (None, self.device):
            raise ValueError(f"the rotation is on device {self.device}, the tensors on {parts.device}")
        cp_rope_apply(_rope(self), parts, positions, first, inverse, stream)

    def destroy(self) -> None:
        if self.handle:
            cp_rope_destroy(self.handle)
            self.handle = None


class Pool:
    """Owns one cp_pool handle; methods forward to the C names above."""

    def __init__(self, **desc):
        self.handle = cp_pool_create(**desc)
        self.device = desc.get("device", 0)
        self.page_tokens = desc.get("page_tokens", 64)

    def register(self, kind: int, n_q_heads: int, n_kv_heads: int, **kw) -> int:
        return cp_model_register(self.handle, kind, n_q_heads, n_kv_heads, **kw)

    def register_spec(self, spec, n_layers: int = 1) -> int:
        """Register a model described by an object with kind / head fields."""
        if spec.kind == "mla":
            return self.register(CP_KIND_MLA, spec.n_q_heads, 1, latent_dim=spec.latent_dim,
                                 rope_dim=spec.rope_dim, softmax_scale=spec.scale, n_layers=n_layers)
        return self.register(CP_KIND_GQA, spec.n_q_heads, spec.n_kv_heads, head_dim=spec.head_dim,
                             softmax_scale=spec.scale, n_layers=n_layers)

    def info(self, model_id: int) -> dict:
        return cp_model_info(self.handle, model_id)

    def open(self, model_id: int, reserve_tokens: int) -> int:
        return cp_request_open(self.handle, model_id, reserve_tokens)

    def close(self, req_id: int) -> None:
        cp_request_close(self.handle, req_id)

    def ctx_len(self, req_id: int) -> int:
        return cp_request_len(self.handle, req_id)

    def cursor(self, req_id: int):
        return cp_request_cursor(self.handle, req_id)

    def pages(self, req_id: int, first: int = 0, count: Optional[int] = None, layers: int = 1) -> np.ndarray:
        if count is None:
            count = -(-self.ctx_len(req_id) // self.page_tokens) - first
        return cp_request_pages(self.handle, req_id, first, count, layers)

    def stats(self) -> dict:
        return cp_pool_stats(self.handle)

    def append(self, req_ids, n_new, rows, stream=None) -> None:
        cp_kv_append(self.handle, req_ids, n_new, rows, stream)

    def decode(self, req_ids, q, out, lse, stream=None, **opts) -> None:
        if opts:
            cp_attn_decode_ex(self.handle, req_ids, q, out, lse, stream, **opts)
        else:
            cp_attn_decode(self.handle, req_ids, q, out, lse, stream)

    def decode_noalloc(self, req_ids, q, out, lse, stream=None, **opts) -> None:
        cp_attn_decode_noalloc(self.handle, req_ids, q, out, lse, stream, **opts)

    def decode_step(self, req_ids, n_new, rows, q, out, lse, stream=None, **opts) -> None:
        cp_attn_decode_step(self.handle, req_ids, n_new, rows, q, out, lse, stream, **opts)

    def decode_layers(self, req_ids, n_new, rows, q, out, lse, stream=None, **opts) -> None:
        cp_attn_decode_layers(self.handle, req_ids, n_new, rows, q, out, lse, stream, **opts)

    def append_rope(self, req_ids, n_new, rows, rope, stream=None) -> None:
        cp_kv_append_rope(self.handle, req_ids, n_new, rows, rope, stream)

    def extend(self, req_ids, n_q, q, out, lse, stream=None, **opts) -> None:
        cp_attn_extend(self.handle, req_ids, n_q, q, out, lse, stream, **opts)

    def extend_step(self, req_ids, n_new, rows, q, out, lse, stream=None, **opts) -> None:
        cp_attn_extend_step(self.handle, req_ids, n_new, rows, q, out, lse, stream, **opts)

    def tree(self, req_ids, n_q, q, out, lse, mask, depth, stream=None, **opts) -> None:
        cp_attn_tree(self.handle, req_ids, n_q, q, out, lse, mask, depth, stream, **opts)

    def tree_step(self, req_ids, n_new, rows, q, out, lse, mask, depth, stream=None, **opts) -> None:
        cp_attn_tree_step(self.handle, req_ids, n_new, rows, q, out, lse, mask, depth, stream, **opts)

    def weights(self, req_ids, n_q, q, lse, new, stream=None, **opts) -> None:
        cp_attn_weights(self.handle, req_ids, n_q, q, lse, new, stream, **opts)

    def keep(self, req_ids, first, n_keep, keep, stream=None) -> None:
        cp_request_keep(self.handle, req_ids, first, n_keep, keep, stream)

    def evict(self, req_ids, n_keep, weights, stream=None, **opts) -> None:
        cp_kv_evict(self.handle, req_ids, n_keep, weights, stream, **opts)

    def position(self, req_id: int) -> int:
        return cp_request_position(self.handle, req_id)

    def fork(self, src_ids, dst_ids, n_tok=None, stream=None) -> None:
        cp_request_fork(self.handle, src_ids, dst_ids, n_tok, stream)

    def truncate(self, req_ids, new_len, stream=None) -> None:
        cp_request_truncate(self.handle, req_ids, new_len, stream)

    def layer_state(self, req_id: int):
        return cp_request_layer_state(self.handle, req_id)

    def gather(self, req_id, start, n_tok, dst, stream=None) -> None:
        cp_kv_gather(self.handle, req_id, start, n_tok, dst, stream)

    def destroy(self) -> None:
        if self.handle:
            cp_pool_destroy(self.handle)
            self.handle = None

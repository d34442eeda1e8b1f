"""ctypes binding of ``include/ead.h``: same names, argument marshalling only.

PyTorch is used by callers for device memory and streams; every step of the
gate path runs inside the CUDA library.  Tensors are passed as raw device
pointers (``tensor.data_ptr()``), bf16 matrices as ``torch.bfloat16``.
"""
from __future__ import annotations

import ctypes as C
import os

_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_DIR, "libead_b200.so")

EAD_OK = 0
EAD_EINVALID_ARG = -1
EAD_EALIGNMENT = -2
EAD_ECUDA = -3
EAD_EUNSUPPORTED_ARCH = -4
EAD_EDEVICE_FAULT = -5
EAD_ESTATE = -6
EAD_ELIMIT = -7
EAD_STATIC_MAX_B = 128
EAD_STATIC_MAX_H = 8192
EAD_STATUS_NONFINITE = 0x1
EAD_STATUS_WAIT_EXPIRED = 0x2
EAD_STATUS_BAD_COUNT = 0x4
EAD_STATUS_SHARD_MISMATCH = 0x8
EAD_SHARD_RECORD_BYTES = 32
EAD_SHARD_MAX = 16
EAD_STATUS_BAD_PAGE = 0x10
EAD_FMT_BF16 = 0
EAD_FMT_E4M3 = 1
EAD_FMT_BLOCK = 32
EAD_KV_WORKSPACE_BYTES = 64 << 20
EAD_NORM_MAX_H = 16384

SYMBOLS = ["ead_create", "ead_step", "ead_run", "ead_run_host", "ead_run_timed", "ead_reset", "ead_status",
           "ead_state_size", "ead_get_state", "ead_set_state", "ead_kernel_launches",
           "ead_launch_info", "ead_destroy", "ead_strerror", "ead_head_entropy_static",
           "ead_plan_split", "ead_plan_units", "ead_usage", "ead_parameter_ratio", "ead_set_done", "ead_get_done",
           "ead_shard_range", "ead_shard_partials", "ead_shard_gate", "ead_shard_connect",
           "ead_shard_exchange_bytes", "ead_kv_write", "ead_kv_read", "ead_kv_attention", "ead_add_rmsnorm",
           "ead_plan_chunk", "ead_kv_wait_limit"]


class EadConfig(C.Structure):
    _fields_ = [("B", C.c_int32), ("V", C.c_int32), ("H_small", C.c_int32), ("H_large", C.c_int32),
                ("w", C.c_int32), ("d_min", C.c_int32), ("tau", C.c_float), ("unit", C.c_int32),
                ("start_model", C.c_int32), ("device", C.c_int32), ("stream", C.c_void_p),
                ("temperature", C.c_float), ("seed", C.c_uint64), ("eos_token", C.c_int32),
                ("V_large", C.c_int32), ("shard_count", C.c_int32), ("vocab_offset_small", C.c_int32),
                ("vocab_offset_large", C.c_int32)]


class EadKvCache(C.Structure):
    """``struct ead_kv_cache``; made by ``ead_kv_cache``."""
    _fields_ = [("format", C.c_int32), ("heads_kv", C.c_int32), ("head_dim", C.c_int32), ("page_size", C.c_int32),
                ("n_pages", C.c_int32), ("reserved", C.c_int32), ("page_stride", C.c_int64),
                ("head_stride", C.c_int64), ("slot_stride", C.c_int64), ("k", C.c_void_p), ("v", C.c_void_p),
                ("k_scale", C.c_void_p), ("v_scale", C.c_void_p)]


class EadKvBatch(C.Structure):
    """``struct ead_kv_batch``; made by ``ead_kv_batch``."""
    _fields_ = [("B", C.c_int32), ("n_tokens", C.c_int32), ("max_new", C.c_int32), ("max_len", C.c_int32),
                ("new_start", C.c_void_p), ("kv_len", C.c_void_p), ("page_table", C.c_void_p),
                ("table_stride", C.c_int32), ("reserved", C.c_int32)]


class EadError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {strerror(code)} ({code})")


_lib = None


def lib() -> C.CDLL:
    """Loads the CUDA library; fails loudly when it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: run `python -m paper_2502_06833_b200.build` "
                              "(there is no fallback path)")
        L = C.CDLL(LIB_PATH)
        vp, i32p, f32p, u8p = C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p
        L.ead_create.restype = C.c_int
        L.ead_create.argtypes = [C.POINTER(EadConfig), vp, vp, C.POINTER(C.c_void_p)]
        L.ead_step.restype = C.c_int
        L.ead_step.argtypes = [vp, vp, vp, i32p, f32p, f32p, u8p, u8p]
        for name in ("ead_run", "ead_run_host"):
            f = getattr(L, name)
            f.restype = C.c_int
            f.argtypes = [vp, C.c_int32, vp, vp, i32p, f32p, f32p, u8p, u8p]
        L.ead_run_timed.restype = C.c_int
        L.ead_run_timed.argtypes = [vp, C.c_int32, vp, vp, i32p, f32p, f32p, u8p, u8p,
                                    C.POINTER(C.c_float)]
        L.ead_reset.restype = C.c_int
        L.ead_reset.argtypes = [vp]
        L.ead_status.restype = C.c_int
        L.ead_status.argtypes = [vp, C.POINTER(C.c_uint32)]
        L.ead_state_size.restype = C.c_size_t
        L.ead_state_size.argtypes = [vp]
        L.ead_get_state.restype = C.c_int
        L.ead_get_state.argtypes = [vp, vp, C.c_size_t]
        L.ead_set_state.restype = C.c_int
        L.ead_set_state.argtypes = [vp, vp, C.c_size_t]
        L.ead_kernel_launches.restype = C.c_int64
        L.ead_kernel_launches.argtypes = [vp]
        L.ead_launch_info.restype = C.c_int
        L.ead_launch_info.argtypes = [vp, C.POINTER(C.c_int32), C.c_int32]
        L.ead_destroy.restype = None
        L.ead_destroy.argtypes = [vp]
        L.ead_head_entropy_static.restype = C.c_int
        L.ead_head_entropy_static.argtypes = [vp, vp, C.c_int32, C.c_int32, C.c_int32, i32p, f32p, vp,
                                              C.c_int32, vp]
        L.ead_set_done.restype = C.c_int
        L.ead_set_done.argtypes = [vp, vp]
        L.ead_get_done.restype = C.c_int
        L.ead_get_done.argtypes = [vp, vp]
        L.ead_usage.restype = C.c_int
        L.ead_usage.argtypes = [vp, C.POINTER(C.c_uint64), vp]
        L.ead_parameter_ratio.restype = C.c_double
        L.ead_parameter_ratio.argtypes = [C.c_uint64, C.c_uint64, C.c_double, C.c_double]
        L.ead_plan_split.restype = C.c_int
        L.ead_plan_split.argtypes = [C.c_int32] * 4 + [C.POINTER(C.c_int32)]
        L.ead_plan_units.restype = C.c_int
        L.ead_plan_units.argtypes = [C.c_int32] * 5 + [C.POINTER(C.c_int32)]
        L.ead_shard_range.restype = C.c_int
        L.ead_shard_range.argtypes = [C.c_int32] * 3 + [C.POINTER(C.c_int32)] * 2
        L.ead_shard_exchange_bytes.restype = C.c_size_t
        L.ead_shard_exchange_bytes.argtypes = [C.c_int32, C.c_int32]
        L.ead_shard_connect.restype = C.c_int
        L.ead_shard_connect.argtypes = [vp, C.c_int32, C.POINTER(C.c_void_p)]
        L.ead_shard_partials.restype = C.c_int
        L.ead_shard_partials.argtypes = [vp, vp, vp, vp]
        L.ead_shard_gate.restype = C.c_int
        L.ead_shard_gate.argtypes = [vp, vp, C.c_int32, i32p, f32p, f32p, u8p, u8p]
        i32, i64 = C.c_int32, C.c_int64
        L.ead_kv_write.restype = C.c_int
        L.ead_kv_write.argtypes = [vp, vp, vp, vp, i64, vp, i32, vp]
        L.ead_kv_read.restype = C.c_int
        L.ead_kv_read.argtypes = [vp, vp, vp, vp, vp, i64, vp, i32, vp]
        L.ead_kv_attention.restype = C.c_int
        L.ead_kv_attention.argtypes = [vp, vp, vp, i64, i32, C.c_float, i32, i32, vp, i64, vp, vp, vp, i32, vp]
        L.ead_kv_wait_limit.restype = C.c_int
        L.ead_kv_wait_limit.argtypes = [i32]
        L.ead_plan_chunk.restype = C.c_int
        L.ead_plan_chunk.argtypes = [i32] * 6 + [C.POINTER(C.c_int64)]
        L.ead_add_rmsnorm.restype = C.c_int
        L.ead_add_rmsnorm.argtypes = [vp, i64, vp, i64, vp, i64, vp, C.c_float, i32, i32, i32, vp, i64, vp, i32, vp]
        L.ead_strerror.restype = C.c_char_p
        L.ead_strerror.argtypes = [C.c_int]
        _lib = L
    return _lib


def strerror(code: int) -> str:
    return lib().ead_strerror(int(code)).decode()


def _check(code: int, where: str) -> None:
    if code != EAD_OK:
        raise EadError(code, where)


def _ptr(t):
    """Device (or host) address of a torch tensor / numpy array / int / None."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if hasattr(t, "data_ptr"):
        return t.data_ptr()
    return t.ctypes.data


def ead_create(*, B, V, H_small, H_large, w, d_min, tau, W_small, W_large, unit=0, start_model=0,
               device=0, stream=0, temperature=0.0, seed=0, eos_token=-1, V_large=0, shard_count=0,
               vocab_offset_small=0, vocab_offset_large=0):
    """Returns an opaque context handle (int).  ``W_*`` are device bf16 ``[V, H]``; they are
    borrowed, keep them alive until ``ead_destroy``."""
    cfg = EadConfig(B, V, H_small, H_large, w, d_min, float(tau), unit, start_model, device,
                    C.c_void_p(int(stream)), float(temperature), int(seed), int(eos_token), int(V_large),
                    int(shard_count), int(vocab_offset_small), int(vocab_offset_large))
    out = C.c_void_p()
    _check(lib().ead_create(C.byref(cfg), _ptr(W_small), _ptr(W_large), C.byref(out)), "ead_create")
    return out.value


def ead_step(ctx, h_small, h_large, tok=None, H=None, Hbar=None, model_used=None, next_model=None):
    _check(lib().ead_step(ctx, _ptr(h_small), _ptr(h_large), _ptr(tok), _ptr(H), _ptr(Hbar),
                          _ptr(model_used), _ptr(next_model)), "ead_step")


def ead_run(ctx, T, h_small_seq, h_large_seq, tok=None, H=None, Hbar=None, model_used=None,
            next_model=None):
    _check(lib().ead_run(ctx, int(T), _ptr(h_small_seq), _ptr(h_large_seq), _ptr(tok), _ptr(H),
                         _ptr(Hbar), _ptr(model_used), _ptr(next_model)), "ead_run")


def ead_run_host(ctx, T, h_small_seq, h_large_seq, tok=None, H=None, Hbar=None, model_used=None,
                 next_model=None):
    """All buffers are HOST memory (numpy arrays or CPU tensors, ideally pinned)."""
    _check(lib().ead_run_host(ctx, int(T), _ptr(h_small_seq), _ptr(h_large_seq), _ptr(tok), _ptr(H),
                              _ptr(Hbar), _ptr(model_used), _ptr(next_model)), "ead_run_host")


def ead_run_timed(ctx, T, h_small_seq, h_large_seq, tok=None, H=None, Hbar=None, model_used=None,
                  next_model=None) -> dict:
    """ead_run with CUDA events around every kernel; returns summed milliseconds per kernel."""
    ms = (C.c_float * 3)()
    _check(lib().ead_run_timed(ctx, int(T), _ptr(h_small_seq), _ptr(h_large_seq), _ptr(tok), _ptr(H),
                               _ptr(Hbar), _ptr(model_used), _ptr(next_model), ms), "ead_run_timed")
    return dict(compact_ms=ms[0], lmhead_ms=ms[1], merge_gate_ms=ms[2])


def ead_reset(ctx):
    _check(lib().ead_reset(ctx), "ead_reset")


def ead_status(ctx, raise_on_fault: bool = True) -> int:
    word = C.c_uint32()
    rc = lib().ead_status(ctx, C.byref(word))
    if rc != EAD_OK and (raise_on_fault or rc != EAD_EDEVICE_FAULT):
        raise EadError(rc, f"ead_status (status word {word.value:#x})")
    return int(word.value)


def ead_state_size(ctx) -> int:
    return int(lib().ead_state_size(ctx))


def ead_get_state(ctx) -> bytes:
    n = ead_state_size(ctx)
    buf = C.create_string_buffer(n)
    _check(lib().ead_get_state(ctx, C.cast(buf, C.c_void_p), n), "ead_get_state")
    return buf.raw


def ead_set_state(ctx, blob: bytes) -> None:
    buf = C.create_string_buffer(bytes(blob), len(blob))
    _check(lib().ead_set_state(ctx, C.cast(buf, C.c_void_p), len(blob)), "ead_set_state")


def ead_kernel_launches(ctx) -> int:
    return int(lib().ead_kernel_launches(ctx))


def ead_launch_info(ctx) -> dict:
    a = (C.c_int32 * 4)()
    _check(lib().ead_launch_info(ctx, a, 4), "ead_launch_info")
    return dict(ctas=a[0], stages=a[1], a_rows=a[2], smem_bytes=a[3])


def ead_head_entropy_static(W, h, B, V, H, tok=None, H_out=None, status=None, device=0, stream=0):
    """Entropy (nats) and greedy token of one LM head for a dense batch, for callers that
    may not allocate device memory: the library uses a scratch array compiled into it
    (B <= EAD_STATIC_MAX_B, H <= EAD_STATIC_MAX_H).  All buffers are device memory owned
    by the caller; asynchronous on ``stream``."""
    _check(lib().ead_head_entropy_static(_ptr(W), _ptr(h), int(B), int(V), int(H), _ptr(tok),
                                         _ptr(H_out), _ptr(status), int(device),
                                         C.c_void_p(int(stream))), "ead_head_entropy_static")


def ead_set_done(ctx, done) -> None:
    """``done``: uint8 numpy array [B] of 0/1 (host memory)."""
    _check(lib().ead_set_done(ctx, _ptr(done)), "ead_set_done")


def ead_get_done(ctx, B: int):
    import numpy as np
    out = np.zeros(B, dtype=np.uint8)
    _check(lib().ead_get_done(ctx, _ptr(out)), "ead_get_done")
    return out


def ead_usage(ctx, per_row=None) -> dict:
    """Tokens produced by each model and switches since the last reset (summed over rows);
    ``per_row`` may be a uint32 numpy array of shape [3, B] to receive the per-row counters."""
    a = (C.c_uint64 * 3)()
    _check(lib().ead_usage(ctx, a, _ptr(per_row)), "ead_usage")
    return dict(tokens_small=int(a[0]), tokens_large=int(a[1]), switches=int(a[2]))


def ead_parameter_ratio(tokens_small, tokens_large, P_small, P_large) -> float:
    return float(lib().ead_parameter_ratio(int(tokens_small), int(tokens_large), float(P_small),
                                           float(P_large)))


def ead_plan_split(cta, G, n_rows, V) -> dict:
    a = (C.c_int32 * 6)()
    _check(lib().ead_plan_split(int(cta), int(G), int(n_rows), int(V), a), "ead_plan_split")
    return dict(active=a[0], row_block=a[1], slot=a[2], col_begin=a[3], col_end=a[4], group=a[5])


def ead_plan_units(cta, G, n_rows, V, two_blocks=True) -> dict:
    a = (C.c_int32 * 13)()
    _check(lib().ead_plan_units(int(cta), int(G), int(n_rows), int(V), int(bool(two_blocks)), a), "ead_plan_units")
    return dict(active=a[0], two_blocks=a[1], row_block=a[2], slot=a[3], group=a[4], rounds=a[5],
                tail_col0=a[6], tail_cols=a[7], thin16=a[8], tile_n=a[9], n_hi=a[10], w_hi=a[11], w_lo=a[12])


def ead_shard_range(V, n_shards, shard) -> tuple:
    """Rows ``[begin, end)`` of a head of V rows held by ``shard`` of ``n_shards``."""
    b, e = C.c_int32(), C.c_int32()
    _check(lib().ead_shard_range(int(V), int(n_shards), int(shard), C.byref(b), C.byref(e)), "ead_shard_range")
    return int(b.value), int(e.value)


def ead_shard_exchange_bytes(B, n_shards) -> int:
    return int(lib().ead_shard_exchange_bytes(int(B), int(n_shards)))


def ead_shard_connect(ctx, shard, exchange) -> None:
    """``exchange``: one device address (or tensor) per shard, as addressable from this GPU."""
    ptrs = (C.c_void_p * len(exchange))(*[_ptr(e) for e in exchange])
    _check(lib().ead_shard_connect(ctx, int(shard), ptrs), "ead_shard_connect")


def ead_shard_partials(ctx, h_small, h_large, records) -> None:
    _check(lib().ead_shard_partials(ctx, _ptr(h_small), _ptr(h_large), _ptr(records)), "ead_shard_partials")


def ead_shard_gate(ctx, all_records, n_shards, tok=None, H=None, Hbar=None, model_used=None,
                   next_model=None) -> None:
    _check(lib().ead_shard_gate(ctx, _ptr(all_records), int(n_shards), _ptr(tok), _ptr(H), _ptr(Hbar),
                                _ptr(model_used), _ptr(next_model)), "ead_shard_gate")


_torch = None


def _t():
    """torch, on first use: the gate step's calls do not need it."""
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


def _rows3(t, shape, what: str) -> int:
    """Checks a bf16 tensor ``[n, heads, dim]`` whose rows are contiguous; elements between rows."""
    if t.dtype is not _t().bfloat16 or t.shape != shape:
        raise ValueError(f"{what}: {t.dtype} {tuple(t.shape)}, want bfloat16 {tuple(shape)}")
    s0, s1, s2 = t.stride()
    if s2 != 1 or (s1 != shape[2] and shape[1] != 1):
        raise ValueError(f"{what}: want rows that are contiguous")
    return s0 if shape[0] > 1 else shape[1] * shape[2]


def _rows2(t, shape, what: str, dtypes) -> int:
    if t.dtype not in dtypes or t.shape != shape:
        raise ValueError(f"{what}: {t.dtype} {tuple(t.shape)}, want {dtypes} {tuple(shape)}")
    s0, s1 = t.stride()
    if s1 != 1 and shape[1] != 1:
        raise ValueError(f"{what}: want rows that are contiguous")
    return s0 if shape[0] > 1 else shape[1]


def _dense(t, shape, dtype, what: str) -> None:
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what}: {t.dtype} {tuple(t.shape)}, want contiguous {dtype} {tuple(shape)}")


def ead_kv_cache(k, v, k_scale=None, v_scale=None) -> EadKvCache:
    """Describes a paged cache held in tensors; they are borrowed (the description keeps them alive).

    ``k``, ``v``: ``[n_pages, heads_kv, page_size, head_dim]``, bf16, or 8-bit (``torch.float8_e4m3fn`` or
    ``torch.uint8``) with ``*_scale`` uint8 ``[n_pages, heads_kv, page_size, head_dim / 32]``.  The last
    dimension is contiguous, the others have any strides (a cache laid out token by token is a
    ``transpose(1, 2)`` of its tensor), the same for both."""
    T = _t()
    e4m3 = k_scale is not None
    strides = lambda t: [s if n > 1 else t.shape[3] for s, n in zip(t.stride()[:3], t.shape)]   # noqa: E731  (of one element: any)
    for t, name in ((k, "k"), (v, "v")):
        if t.dtype not in ((T.float8_e4m3fn, T.uint8) if e4m3 else (T.bfloat16,)):
            raise ValueError(f"{name}: {t.dtype} does not fit a cache {'with' if e4m3 else 'without'} scales")
        if t.dim() != 4 or t.stride(3) != 1 or t.shape != k.shape or strides(t) != strides(k):
            raise ValueError(f"{name}: want [n_pages, heads_kv, page_size, head_dim], contiguous in the last "
                             "dimension, k and v alike")
    for t, name in ((k_scale, "k_scale"), (v_scale, "v_scale")):
        if (t is not None) != e4m3:
            raise ValueError("k_scale and v_scale come together")
        if e4m3:
            _dense(t, (*k.shape[:3], k.shape[3] // EAD_FMT_BLOCK), T.uint8, name)
    c = EadKvCache(EAD_FMT_E4M3 if e4m3 else EAD_FMT_BF16, k.shape[1], k.shape[3], k.shape[2], k.shape[0], 0,
                   *strides(k), _ptr(k), _ptr(v), _ptr(k_scale), _ptr(v_scale))
    c.held = (k, v, k_scale, v_scale)
    c.ref = C.byref(c)
    return c


def ead_kv_batch(page_table, new_start, kv_len=None, *, n_tokens, max_new, max_len) -> EadKvBatch:
    """Describes one step's batch: device int32 tensors ``page_table`` ``[B, entries]``, ``new_start``
    ``[B + 1]``, ``kv_len`` ``[B]`` (borrowed; the description keeps them alive) and what the host knows
    of them.  ``kv_len`` may be omitted for reading."""
    i32 = _t().int32
    B = page_table.shape[0]
    if page_table.dtype is not i32 or page_table.dim() != 2 or (page_table.stride(1) != 1 and page_table.shape[1] > 1):
        raise ValueError("page_table: want int32 [B, entries] with contiguous rows")
    _dense(new_start, (B + 1,), i32, "new_start")
    if kv_len is not None:
        _dense(kv_len, (B,), i32, "kv_len")
    c = EadKvBatch(B, int(n_tokens), int(max_new), int(max_len), _ptr(new_start), _ptr(kv_len), _ptr(page_table),
                   max(page_table.stride(0) if B > 1 else page_table.shape[1], 1), 0)
    c.held = (page_table, new_start, kv_len)
    c.ref = C.byref(c)
    return c


def ead_kv_write(cache: EadKvCache, batch: EadKvBatch, k_new, v_new, *, status=None, device=0, stream=0) -> None:
    """Writes the step's keys and values, bf16 ``[n_tokens, heads_kv, head_dim]``, into the cache."""
    shape = (batch.n_tokens, cache.heads_kv, cache.head_dim)
    stride = _rows3(k_new, shape, "k_new")
    if _rows3(v_new, shape, "v_new") != stride:
        raise ValueError("k_new and v_new: want the same row stride")
    rc = lib().ead_kv_write(cache.ref, batch.ref, k_new.data_ptr(), v_new.data_ptr(), stride, _ptr(status), device,
                            stream)
    if rc:
        _check(rc, "ead_kv_write")


def ead_kv_read(cache: EadKvCache, batch: EadKvBatch, k_out, v_out, *, first=None, status=None, device=0,
                stream=0) -> None:
    """Reads tokens back as bf16 ``[n_tokens, heads_kv, head_dim]``; ``first``: int32 ``[B]``, first positions."""
    shape = (batch.n_tokens, cache.heads_kv, cache.head_dim)
    stride = _rows3(k_out, shape, "k_out")
    if _rows3(v_out, shape, "v_out") != stride:
        raise ValueError("k_out and v_out: want the same row stride")
    if first is not None:
        _dense(first, (batch.B,), _t().int32, "first")
    rc = lib().ead_kv_read(cache.ref, batch.ref, _ptr(first), k_out.data_ptr(), v_out.data_ptr(), stride,
                           _ptr(status), device, stream)
    if rc:
        _check(rc, "ead_kv_read")


def ead_kv_attention(cache: EadKvCache, batch: EadKvBatch, q, out, *, scale, workspace, window=0, sinks=0, lse=None,
                     status=None, device=0, stream=0) -> None:
    """Attention of the step's new tokens over the paged cache; ``q`` and ``out`` are bf16
    ``[n_tokens, heads_q, head_dim]``, ``lse`` float ``[n_tokens, heads_q]``; ``workspace`` is a zero-filled
    buffer of ``EAD_KV_WORKSPACE_BYTES`` that calls which may overlap must not share."""
    heads_q = q.shape[1]
    shape = (batch.n_tokens, heads_q, cache.head_dim)
    q_stride, out_stride = _rows3(q, shape, "q"), _rows3(out, shape, "out")
    if lse is not None:
        _dense(lse, shape[:2], _t().float32, "lse")
    if workspace.nbytes < EAD_KV_WORKSPACE_BYTES:
        raise ValueError("workspace: want EAD_KV_WORKSPACE_BYTES bytes")
    rc = lib().ead_kv_attention(cache.ref, batch.ref, q.data_ptr(), q_stride, heads_q, scale, window, sinks,
                                out.data_ptr(), out_stride, _ptr(lse), workspace.data_ptr(), _ptr(status), device,
                                stream)
    if rc:
        _check(rc, "ead_kv_attention")


def ead_kv_wait_limit(ns: int) -> None:
    """Limit of the attention kernels' bounded waits; negative: the default."""
    _check(lib().ead_kv_wait_limit(ns), "ead_kv_wait_limit")


def ead_plan_chunk(n_new, kv_len, *, heads_per_kv, max_new=None, window=0, sinks=0) -> dict:
    a = (C.c_int64 * 2)()
    _check(lib().ead_plan_chunk(n_new, kv_len, n_new if max_new is None else max_new, heads_per_kv, window, sinks, a),
           "ead_plan_chunk")
    return dict(units=a[0], cost=a[1])


def ead_add_rmsnorm(x, weight, out, *, residual=None, residual_out=None, out_scale=None, eps=1e-6, device=0,
                    stream=0) -> None:
    """``out = norm(x + residual) * weight`` over bf16 rows ``[n, H]``, ``residual_out = x + residual``; with
    ``out_scale`` (uint8 ``[n, H / 32]``) the output is 8-bit (``torch.float8_e4m3fn`` or ``torch.uint8``)."""
    T = _t()
    bf16 = (T.bfloat16,)
    n, H = shape = x.shape
    x_stride = _rows2(x, shape, "x", bf16)
    _dense(weight, (H,), T.bfloat16, "weight")
    out_stride = _rows2(out, shape, "out", bf16 if out_scale is None else (T.float8_e4m3fn, T.uint8))
    r_stride = ro_stride = 0
    if residual is not None:
        r_stride = _rows2(residual, shape, "residual", bf16)
    if residual_out is not None:
        ro_stride = _rows2(residual_out, shape, "residual_out", bf16)
    if out_scale is not None:
        _dense(out_scale, (n, H // EAD_FMT_BLOCK), T.uint8, "out_scale")
    rc = lib().ead_add_rmsnorm(x.data_ptr(), x_stride, _ptr(residual), r_stride, _ptr(residual_out), ro_stride,
                               weight.data_ptr(), eps, n, H, EAD_FMT_BF16 if out_scale is None else EAD_FMT_E4M3,
                               out.data_ptr(), out_stride, _ptr(out_scale), device, stream)
    if rc:
        _check(rc, "ead_add_rmsnorm")


def ead_destroy(ctx) -> None:
    if ctx:
        lib().ead_destroy(ctx)

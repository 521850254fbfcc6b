"""Python binding of the C ABI in include/bkv.h (argument marshalling only).

Each ``bkv_*`` function has the C function's name and meaning; tensors are
torch tensors whose device pointers are handed to the library, and the CUDA
stream defaults to torch's current stream.  Nothing here computes: every step
of the method runs in libbkv.so, and this module raises if the library cannot
be loaded (there is no other implementation to fall back on).
"""
from __future__ import annotations

import ctypes
import os
import threading

import torch

from . import _build

BKV_OK = 0
BKV_EINVAL = -1
BKV_ENOMEM = -2
BKV_ECUDA = -3
BKV_ETIMEOUT = -4
BKV_ESTATE = -5
BKV_EBOUNDS = -6

KERNEL_NAMES = ("fps_init", "update", "qobs", "score", "select_gather", "keep_all", "cfps", "rope_stage",
                "attend", "attend_merge", "attend_weights", "evict", "pack4", "unpack4", "attend4")


# bkv_config.flags options (include/bkv.h)
BKV_F_NONE = 0
BKV_F_MEAN_AGG = 1
BKV_F_CONTINUAL_FPS = 2
BKV_F_CAUSAL_WINDOW = 4


class BkvConfig(ctypes.Structure):
    _fields_ = [
        ("n_layers", ctypes.c_int32), ("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("n_beacons", ctypes.c_int32),
        ("window", ctypes.c_int32), ("n_prefix", ctypes.c_int32), ("capacity", ctypes.c_int32),
        ("rope_theta", ctypes.c_double), ("flags", ctypes.c_uint32),
    ]


class BkvError(RuntimeError):
    def __init__(self, code: int, where: str, detail: str = ""):
        self.code = code
        super().__init__(f"{where}: {bkv_strerror(code)} ({code})" + (f": {detail}" if detail else ""))


_lib = None
_lock = threading.Lock()
_P = ctypes.c_void_p
_streams: dict = {}  # stream handle of every live context, for outputs allocated on its behalf


def load_library(path: str | None = None, build: bool = True):
    """Load libbkv.so (building it in-tree first if it is missing or stale).  With the environment
    variable BKV_CHECKED=1 the process uses the bounds-checked flavour libbkv_checked.so instead."""
    global _lib
    with _lock:
        if _lib is not None and path is None:
            return _lib
        checked = os.environ.get("BKV_CHECKED") == "1"
        default = _build.LIB_PATH_CHECKED if checked else _build.LIB_PATH
        p = path or (_build.build(checked=checked) if build else default)
        if not os.path.exists(p):
            raise RuntimeError(f"libbkv.so not found at {p}; run __graft_entry__.build()")
        lib = ctypes.CDLL(p)
        sig = {
            "bkv_create": (ctypes.c_int, [ctypes.POINTER(BkvConfig), _P, ctypes.POINTER(_P)]),
            "bkv_destroy": (None, [_P]),
            "bkv_set_stream": (ctypes.c_int, [_P, _P]),
            "bkv_init_beacons": (ctypes.c_int, [_P, _P, ctypes.c_int32]),
            "bkv_update_beacons": (ctypes.c_int, [_P, _P, ctypes.c_int32, _P]),
            "bkv_update_beacons_seq": (ctypes.c_int, [_P, _P, ctypes.c_int32, _P]),
            "bkv_compress": (ctypes.c_int, [_P, _P, _P, ctypes.c_int32, ctypes.c_int32, ctypes.c_int64, _P, _P,
                                            _P, _P]),
            "bkv_compress_ragged": (ctypes.c_int, [_P, _P, _P, _P, ctypes.c_int32, _P, _P, _P, _P, _P]),
            "bkv_attend": (ctypes.c_int, [_P, _P, ctypes.c_int32, _P, _P, _P, ctypes.c_double, _P, _P, _P]),
            "bkv_attend_shared": (ctypes.c_int, [_P, _P, ctypes.c_int32, _P, _P, _P, ctypes.c_int32, ctypes.c_int32,
                                                 _P, _P, _P, ctypes.c_double, _P, _P, _P]),
            "bkv_attend_window": (ctypes.c_int, [_P, _P, ctypes.c_int32, _P, _P, _P, ctypes.c_int32, ctypes.c_int32,
                                                 ctypes.c_double, _P, _P]),
            "bkv_attend_reserve": (ctypes.c_int, [_P, ctypes.c_int32, ctypes.c_int32, ctypes.c_int]),
            "bkv_evict": (ctypes.c_int, [_P, _P, _P, _P, _P, ctypes.c_int32, _P, _P, _P, ctypes.c_int32, _P, _P]),
            "bkv_pack4": (ctypes.c_int, [_P, _P, _P, ctypes.c_int32, _P, _P, _P, _P, _P]),
            "bkv_unpack4": (ctypes.c_int, [_P, _P, _P, _P, ctypes.c_int32, _P, _P, _P, _P]),
            "bkv_attend4": (ctypes.c_int, [_P, _P, ctypes.c_int32, _P, _P, _P, _P, ctypes.c_double, _P, _P, _P]),
            "bkv_attend4_reserve": (ctypes.c_int, [_P, ctypes.c_int32, ctypes.c_int]),
            "bkv_evict4": (ctypes.c_int, [_P, _P, _P, _P, _P, _P, ctypes.c_int32, _P, _P, _P, _P, ctypes.c_int32, _P,
                                          _P]),
            "bkv_get_state": (ctypes.c_int, [_P, _P, _P, _P]),
            "bkv_set_state": (ctypes.c_int, [_P, _P, _P, _P]),
            "bkv_get_cfps_state": (ctypes.c_int, [_P, _P, _P]),
            "bkv_set_cfps_state": (ctypes.c_int, [_P, _P, _P]),
            "bkv_sync": (ctypes.c_int, [_P]),
            "bkv_selftest_wait_timeout": (ctypes.c_int, [_P, ctypes.c_int64]),
            "bkv_selftest_bounds": (ctypes.c_int, [_P]),
            "bkv_checked_build": (ctypes.c_int, []),
            "bkv_debug_fail_alloc": (ctypes.c_int, [ctypes.c_int32]),
            "bkv_compress_static": (ctypes.c_int, [ctypes.POINTER(BkvConfig), _P, _P, _P, _P, ctypes.c_int32,
                                                   ctypes.c_int32, ctypes.c_int64, _P, _P, _P, _P, _P, _P,
                                                   ctypes.c_char_p, ctypes.c_size_t]),
            "bkv_profile_enable": (ctypes.c_int, [_P, ctypes.c_int]),
            "bkv_profile_read": (ctypes.c_int, [_P, _P, _P, ctypes.c_int32]),
            "bkv_strerror": (ctypes.c_char_p, [ctypes.c_int]),
            "bkv_last_error": (ctypes.c_char_p, [_P]),
            "bkv_version": (ctypes.c_char_p, []),
        }
        for name, (res, args) in sig.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        if path is None:
            _lib = lib
        return lib


def _l():
    return _lib if _lib is not None else load_library()


def _ptr(t: torch.Tensor | None, dtype: torch.dtype, name: str, device=None):
    if t is None:
        return None
    if t.dtype is dtype and t.is_cuda and t.is_contiguous():
        return t.data_ptr()
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    raise ValueError(f"{name} must be contiguous")


def _ptr_any(t: torch.Tensor | None, dtype: torch.dtype, name: str):
    """Pointer of a CUDA or host tensor (the state copies take their direction from the pointer)."""
    if t is None:
        return None
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream) -> ctypes.c_void_p:
    if stream is None:
        if not torch.cuda.is_available():
            return ctypes.c_void_p(0)
        stream = torch.cuda.current_stream()
    handle = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    return ctypes.c_void_p(handle)


def _expect(t: torch.Tensor | None, n: int, name: str) -> None:
    """The C ABI receives bare pointers and trusts the sizes that the shape implies: a tensor of the
    wrong element count is a ValueError here instead of an out-of-bounds access on the device."""
    if t is not None and t.numel() != n:
        raise ValueError(f"{name} has {t.numel()} elements; the configured shape needs {n}")


def _arg(t: torch.Tensor | None, dtype: torch.dtype, n: int, name: str):
    """_expect and _ptr in one, for the calls of a decode step: a step's host time is what its small calls take."""
    if t is None:
        return None
    if t.dtype is dtype and t.is_cuda and t.is_contiguous() and t.numel() == n:
        return t.data_ptr()
    _expect(t, n, name)
    return _ptr(t, dtype, name)


def _check(rc: int, where: str, ctx=None) -> None:
    if rc != BKV_OK:
        detail = _l().bkv_last_error(ctx).decode() if ctx is not None else ""
        raise BkvError(rc, where, detail)


# ---------------------------------------------------------------- C-ABI mirror
def bkv_version() -> str:
    return _l().bkv_version().decode()


def bkv_strerror(code: int) -> str:
    return _l().bkv_strerror(int(code)).decode()


def bkv_last_error(ctx) -> str:
    return _l().bkv_last_error(ctx).decode()


def bkv_create(cfg: BkvConfig, stream=None) -> ctypes.c_void_p:
    out = ctypes.c_void_p()
    handle = _stream(stream)
    _check(_l().bkv_create(ctypes.byref(cfg), handle, ctypes.byref(out)), "bkv_create")
    _streams[out.value] = handle.value or 0
    return out


def bkv_destroy(ctx) -> None:
    if ctx:
        _streams.pop(ctx.value, None)
        _l().bkv_destroy(ctx)


def bkv_set_stream(ctx, stream=None) -> None:
    handle = _stream(stream)
    _check(_l().bkv_set_stream(ctx, handle), "bkv_set_stream", ctx)
    _streams[ctx.value] = handle.value or 0


def bkv_init_beacons(ctx, q_init: torch.Tensor, n_init: int) -> None:
    _check(_l().bkv_init_beacons(ctx, _ptr(q_init, torch.bfloat16, "q_init"), int(n_init)), "bkv_init_beacons", ctx)


def bkv_update_beacons(ctx, q_new: torch.Tensor, n_new: int, assign_out: torch.Tensor | None = None) -> None:
    _check(_l().bkv_update_beacons(ctx, _ptr(q_new, torch.bfloat16, "q_new"), int(n_new),
                                   _ptr(assign_out, torch.int32, "assign_out")), "bkv_update_beacons", ctx)


def bkv_update_beacons_seq(ctx, q_steps: torch.Tensor, n_steps: int, assign_out: torch.Tensor | None = None) -> None:
    _check(_l().bkv_update_beacons_seq(ctx, _ptr(q_steps, torch.bfloat16, "q_steps"), int(n_steps),
                                       _ptr(assign_out, torch.int32, "assign_out")), "bkv_update_beacons_seq", ctx)


def bkv_compress(ctx, K: torch.Tensor, V: torch.Tensor, L: int, budget: int, t_pos: int,
                 q_recent: torch.Tensor | None, recent_pos, kept_idx_out: torch.Tensor,
                 scores_out: torch.Tensor | None = None) -> None:
    pos = (ctypes.c_int64 * max(1, len(recent_pos)))(*[int(p) for p in recent_pos])
    _check(_l().bkv_compress(ctx, _ptr(K, torch.bfloat16, "K"), _ptr(V, torch.bfloat16, "V"), int(L), int(budget),
                             int(t_pos), _ptr(q_recent, torch.bfloat16, "q_recent"), ctypes.cast(pos, _P),
                             _ptr(kept_idx_out, torch.int32, "kept_idx_out"),
                             _ptr(scores_out, torch.float32, "scores_out")), "bkv_compress", ctx)


def bkv_compress_ragged(ctx, K: torch.Tensor, V: torch.Tensor, L: torch.Tensor, budget: int, t_pos, q_recent,
                        recent_pos, kept_idx_out: torch.Tensor, scores_out: torch.Tensor | None = None) -> None:
    """L: int32 device tensor, one cache length per instance; t_pos: one position per batch row;
    recent_pos: one list of window positions per batch row (see include/bkv.h)."""
    tp = (ctypes.c_int64 * max(1, len(t_pos)))(*[int(p) for p in t_pos])
    flat = [int(p) for row in recent_pos for p in row]
    rp = (ctypes.c_int64 * max(1, len(flat)))(*flat)
    _check(_l().bkv_compress_ragged(ctx, _ptr(K, torch.bfloat16, "K"), _ptr(V, torch.bfloat16, "V"),
                                    _ptr(L, torch.int32, "L"), int(budget), ctypes.cast(tp, _P),
                                    _ptr(q_recent, torch.bfloat16, "q_recent"), ctypes.cast(rp, _P),
                                    _ptr(kept_idx_out, torch.int32, "kept_idx_out"),
                                    _ptr(scores_out, torch.float32, "scores_out")), "bkv_compress_ragged", ctx)


def bkv_attend_reserve(ctx, n_q: int, n_groups: int = 0, weights: bool = False) -> None:
    _check(_l().bkv_attend_reserve(ctx, int(n_q), int(n_groups), int(bool(weights))), "bkv_attend_reserve", ctx)


def bkv_attend(ctx, q: torch.Tensor, n_q: int, K: torch.Tensor, V: torch.Tensor, length: torch.Tensor, scale: float,
               o: torch.Tensor, lse_out: torch.Tensor | None = None, weights: torch.Tensor | None = None) -> None:
    bf16, f32 = torch.bfloat16, torch.float32
    _check(_l().bkv_attend(ctx, _ptr(q, bf16, "q"), int(n_q), _ptr(K, bf16, "K"), _ptr(V, bf16, "V"),
                           _ptr(length, torch.int32, "length"), float(scale), _ptr(o, bf16, "o"),
                           _ptr(lse_out, f32, "lse_out"), _ptr(weights, f32, "weights")), "bkv_attend", ctx)


def bkv_attend_shared(ctx, q: torch.Tensor, n_q: int, Kp: torch.Tensor, Vp: torch.Tensor, prefix_len: torch.Tensor,
                      n_groups: int, prefix_capacity: int, K: torch.Tensor, V: torch.Tensor, length: torch.Tensor,
                      scale: float, o: torch.Tensor, lse_out: torch.Tensor | None = None,
                      weights: torch.Tensor | None = None) -> None:
    bf16, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    _check(_l().bkv_attend_shared(ctx, _ptr(q, bf16, "q"), int(n_q), _ptr(Kp, bf16, "Kp"), _ptr(Vp, bf16, "Vp"),
                                  _ptr(prefix_len, i32, "prefix_len"), int(n_groups), int(prefix_capacity),
                                  _ptr(K, bf16, "K"), _ptr(V, bf16, "V"), _ptr(length, i32, "length"), float(scale),
                                  _ptr(o, bf16, "o"), _ptr(lse_out, f32, "lse_out"), _ptr(weights, f32, "weights")),
           "bkv_attend_shared", ctx)


def bkv_attend_window(ctx, q: torch.Tensor, n_q: int, K: torch.Tensor, V: torch.Tensor, length: torch.Tensor,
                      window: int, n_sink: int, scale: float, o: torch.Tensor,
                      lse_out: torch.Tensor | None = None) -> None:
    bf16 = torch.bfloat16
    _check(_l().bkv_attend_window(ctx, _ptr(q, bf16, "q"), int(n_q), _ptr(K, bf16, "K"), _ptr(V, bf16, "V"),
                                  _ptr(length, torch.int32, "length"), int(window), int(n_sink), float(scale),
                                  _ptr(o, bf16, "o"), _ptr(lse_out, torch.float32, "lse_out")), "bkv_attend_window",
           ctx)


def bkv_evict(ctx, K: torch.Tensor, V: torch.Tensor, weights: torch.Tensor, L: torch.Tensor, budget: int,
              K_out: torch.Tensor, V_out: torch.Tensor, weights_out: torch.Tensor, capacity_out: int,
              kept_idx_out: torch.Tensor, len_out: torch.Tensor | None = None) -> None:
    bf16, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    _check(_l().bkv_evict(ctx, _ptr(K, bf16, "K"), _ptr(V, bf16, "V"), _ptr(weights, f32, "weights"),
                          _ptr(L, i32, "L"), int(budget), _ptr(K_out, bf16, "K_out"), _ptr(V_out, bf16, "V_out"),
                          _ptr(weights_out, f32, "weights_out"), int(capacity_out), _ptr(kept_idx_out, i32, "kept"),
                          _ptr(len_out, i32, "len_out")), "bkv_evict", ctx)


def bkv_pack4(ctx, K: torch.Tensor, V: torch.Tensor, n_rows: int, first: torch.Tensor | None, length: torch.Tensor,
              K4: torch.Tensor, V4: torch.Tensor, S4: torch.Tensor) -> None:
    bf16, u8, i32 = torch.bfloat16, torch.uint8, torch.int32
    _check(_l().bkv_pack4(ctx, _ptr(K, bf16, "K"), _ptr(V, bf16, "V"), int(n_rows), _ptr(first, i32, "first"),
                          _ptr(length, i32, "length"), _ptr(K4, u8, "K4"), _ptr(V4, u8, "V4"),
                          _ptr(S4, torch.float16, "S4")), "bkv_pack4", ctx)


def bkv_unpack4(ctx, K4: torch.Tensor, V4: torch.Tensor, S4: torch.Tensor, n_rows: int, first: torch.Tensor | None,
                length: torch.Tensor, K: torch.Tensor, V: torch.Tensor) -> None:
    bf16, u8, i32 = torch.bfloat16, torch.uint8, torch.int32
    _check(_l().bkv_unpack4(ctx, _ptr(K4, u8, "K4"), _ptr(V4, u8, "V4"), _ptr(S4, torch.float16, "S4"), int(n_rows),
                            _ptr(first, i32, "first"), _ptr(length, i32, "length"), _ptr(K, bf16, "K"),
                            _ptr(V, bf16, "V")), "bkv_unpack4", ctx)


def bkv_attend4(ctx, q: torch.Tensor, n_q: int, K4: torch.Tensor, V4: torch.Tensor, S4: torch.Tensor,
                length: torch.Tensor, scale: float, o: torch.Tensor, lse_out: torch.Tensor | None = None,
                weights: torch.Tensor | None = None) -> None:
    bf16, f32, u8 = torch.bfloat16, torch.float32, torch.uint8
    _check(_l().bkv_attend4(ctx, _ptr(q, bf16, "q"), int(n_q), _ptr(K4, u8, "K4"), _ptr(V4, u8, "V4"),
                            _ptr(S4, torch.float16, "S4"), _ptr(length, torch.int32, "length"), float(scale),
                            _ptr(o, bf16, "o"), _ptr(lse_out, f32, "lse_out"), _ptr(weights, f32, "weights")),
           "bkv_attend4", ctx)


def bkv_attend4_reserve(ctx, n_q: int, weights: bool = False) -> None:
    _check(_l().bkv_attend4_reserve(ctx, int(n_q), int(bool(weights))), "bkv_attend4_reserve", ctx)


def bkv_evict4(ctx, K4: torch.Tensor, V4: torch.Tensor, S4: torch.Tensor, weights: torch.Tensor, L: torch.Tensor,
               budget: int, K4_out: torch.Tensor, V4_out: torch.Tensor, S4_out: torch.Tensor,
               weights_out: torch.Tensor, capacity_out: int, kept_idx_out: torch.Tensor,
               len_out: torch.Tensor | None = None) -> None:
    u8, f16, f32, i32 = torch.uint8, torch.float16, torch.float32, torch.int32
    _check(_l().bkv_evict4(ctx, _ptr(K4, u8, "K4"), _ptr(V4, u8, "V4"), _ptr(S4, f16, "S4"),
                           _ptr(weights, f32, "weights"), _ptr(L, i32, "L"), int(budget), _ptr(K4_out, u8, "K4_out"),
                           _ptr(V4_out, u8, "V4_out"), _ptr(S4_out, f16, "S4_out"),
                           _ptr(weights_out, f32, "weights_out"), int(capacity_out), _ptr(kept_idx_out, i32, "kept"),
                           _ptr(len_out, i32, "len_out")), "bkv_evict4", ctx)


def bkv_get_state(ctx, centroids=None, sums=None, counts=None) -> None:
    """Tensors may live on the device or the host; host results are valid after bkv_sync."""
    _check(_l().bkv_get_state(ctx, _ptr_any(centroids, torch.float32, "centroids"),
                              _ptr_any(sums, torch.float64, "sums"), _ptr_any(counts, torch.int64, "counts")),
           "bkv_get_state", ctx)


def bkv_set_state(ctx, centroids, sums, counts) -> None:
    _check(_l().bkv_set_state(ctx, _ptr_any(centroids, torch.float32, "centroids"),
                              _ptr_any(sums, torch.float64, "sums"), _ptr_any(counts, torch.int64, "counts")),
           "bkv_set_state", ctx)


def bkv_get_cfps_state(ctx, buffers=None, sizes=None) -> None:
    _check(_l().bkv_get_cfps_state(ctx, _ptr_any(buffers, torch.bfloat16, "buffers"),
                                   _ptr_any(sizes, torch.int32, "sizes")), "bkv_get_cfps_state", ctx)


def bkv_set_cfps_state(ctx, buffers, sizes) -> None:
    _check(_l().bkv_set_cfps_state(ctx, _ptr_any(buffers, torch.bfloat16, "buffers"),
                                   _ptr_any(sizes, torch.int32, "sizes")), "bkv_set_cfps_state", ctx)


def bkv_sync(ctx) -> None:
    _check(_l().bkv_sync(ctx), "bkv_sync", ctx)


def bkv_selftest_wait_timeout(ctx, limit_ns: int) -> int:
    """Runs one device wait that is meant to expire after limit_ns (see
    include/bkv.h) and returns the status code bkv_sync reports for it
    (BKV_ETIMEOUT when the expiry path works); raises on other errors."""
    rc = _l().bkv_selftest_wait_timeout(ctx, int(limit_ns))
    if rc not in (BKV_OK, BKV_ETIMEOUT):
        _check(rc, "bkv_selftest_wait_timeout", ctx)
    return rc


def bkv_selftest_bounds(ctx) -> int:
    """Runs one checked out-of-range store (see include/bkv.h) and returns the status code bkv_sync
    reports for it: BKV_EBOUNDS in a checked build, BKV_OK otherwise; raises on other errors."""
    rc = _l().bkv_selftest_bounds(ctx)
    if rc not in (BKV_OK, BKV_EBOUNDS):
        _check(rc, "bkv_selftest_bounds", ctx)
    return rc


def bkv_checked_build() -> bool:
    return bool(_l().bkv_checked_build())


def bkv_debug_fail_alloc(nth: int) -> None:
    """Arms (nth > 0) or disarms (0) the allocation-failure hook of bkv_create (include/bkv.h)."""
    _check(_l().bkv_debug_fail_alloc(int(nth)), "bkv_debug_fail_alloc")


def bkv_profile_enable(ctx, on: bool = True) -> None:
    _check(_l().bkv_profile_enable(ctx, int(bool(on))), "bkv_profile_enable", ctx)


def bkv_profile_read(ctx) -> dict:
    """{kernel name: (total ms, launches)} since the previous read (syncs the stream)."""
    n = len(KERNEL_NAMES)
    ms = (ctypes.c_double * n)()
    cnt = (ctypes.c_int64 * n)()
    _check(_l().bkv_profile_read(ctx, ctypes.cast(ms, _P), ctypes.cast(cnt, _P), n), "bkv_profile_read", ctx)
    return {KERNEL_NAMES[k]: (ms[k], cnt[k]) for k in range(n)}


def bkv_compress_static(cfg: BkvConfig, centroids, counts, K, V, L: int, budget: int, t_pos: int, q_recent,
                        recent_pos, kept_idx_out, scores_out=None, dev_status=None, stream=None) -> None:
    """Context-free compress that allocates no device memory (see include/bkv.h).

    For callers that cannot allocate on the device, e.g. an engine whose KV
    page allocator owns all of HBM.  Scratch lives in a fixed 16 MiB array
    inside the library; concurrent calls on different streams race on it.
    Every tensor's element count is checked against the sizes cfg implies
    before any pointer reaches the library."""
    c = cfg
    n_inst = c.n_layers * c.batch * c.n_kv_heads
    if n_inst < 1 or c.head_dim < 1 or c.capacity < 1 or budget < 1 or c.window < 0 or c.n_beacons < 0:
        raise ValueError("cfg must describe at least one instance of head_dim, capacity and budget >= 1")
    _expect(K, n_inst * c.capacity * c.head_dim, "K")
    _expect(V, n_inst * c.capacity * c.head_dim, "V")
    _expect(kept_idx_out, n_inst * int(budget), "kept_idx_out")
    _expect(scores_out, n_inst * c.capacity, "scores_out")
    _expect(q_recent, c.n_layers * c.batch * c.n_q_heads * c.window * c.head_dim, "q_recent")
    _expect(centroids, n_inst * c.n_beacons * c.head_dim, "centroids")
    _expect(counts, n_inst * c.n_beacons, "counts")
    if dev_status is not None and dev_status.numel() < 1:
        raise ValueError("dev_status must hold one int32")
    if recent_pos is None:
        recent_pos = []
    if c.window > 0 and len(recent_pos) != c.window:
        raise ValueError(f"recent_pos has {len(recent_pos)} positions; the window is {c.window}")
    pos = (ctypes.c_int64 * max(1, len(recent_pos)))(*[int(p) for p in recent_pos])
    msg = ctypes.create_string_buffer(256)
    rc = _l().bkv_compress_static(
        ctypes.byref(cfg), _ptr(centroids, torch.float32, "centroids"), _ptr(counts, torch.int64, "counts"),
        _ptr(K, torch.bfloat16, "K"), _ptr(V, torch.bfloat16, "V"), int(L), int(budget), int(t_pos),
        _ptr(q_recent, torch.bfloat16, "q_recent"), ctypes.cast(pos, _P), _ptr(kept_idx_out, torch.int32, "kept"),
        _ptr(scores_out, torch.float32, "scores_out"), _ptr(dev_status, torch.int32, "dev_status"),
        _stream(stream), msg, ctypes.sizeof(msg))
    if rc != BKV_OK:
        raise BkvError(rc, "bkv_compress_static", msg.value.decode())


# ---------------------------------------------------------------- convenience
class BeaconKV:
    """Owns one context for a model shape and allocates outputs with torch.

    Example::
        bk = BeaconKV(n_layers=36, batch=16, n_q_heads=32, n_kv_heads=8, head_dim=128,
                      n_beacons=8, window=8, capacity=4224, rope_theta=1e6)
        bk.init_beacons(q_init)                       # [L, B, Hq, n_init, d] bf16
        bk.update(q_new)                              # [L, B, Hq, n_new, d] bf16
        kept = bk.compress(K, V, L=4224, budget=4096, t_pos=4223, q_recent=q, recent_pos=[...])
    """

    def __init__(self, *, n_layers, batch, n_q_heads, n_kv_heads, head_dim, n_beacons, window, capacity,
                 rope_theta=0.0, n_prefix=0, stream=None, mean_agg=False, continual_fps=False, causal_window=False):
        flags = ((BKV_F_MEAN_AGG if mean_agg else BKV_F_NONE) | (BKV_F_CONTINUAL_FPS if continual_fps else BKV_F_NONE)
                 | (BKV_F_CAUSAL_WINDOW if causal_window else BKV_F_NONE))
        self.cfg = BkvConfig(n_layers, batch, n_q_heads, n_kv_heads, head_dim, n_beacons, window, n_prefix,
                             capacity, float(rope_theta), flags)
        self.ctx = bkv_create(self.cfg, stream)
        self.n_inst = n_layers * batch * n_kv_heads
        self._layer = (batch, n_q_heads, head_dim, batch * n_kv_heads, batch * n_kv_heads * capacity)

    @classmethod
    def for_workload(cls, wl, stream=None, capacity=None, mean_agg=False, continual_fps=False,
                     causal_window=False) -> "BeaconKV":
        return cls(n_layers=wl.n_layers, batch=wl.batch, n_q_heads=wl.n_q_heads, n_kv_heads=wl.n_kv_heads,
                   head_dim=wl.head_dim, n_beacons=wl.n_beacons, window=wl.window,
                   capacity=capacity or wl.capacity, rope_theta=wl.rope_theta, n_prefix=wl.n_prefix, stream=stream,
                   mean_agg=mean_agg, continual_fps=continual_fps, causal_window=causal_window)

    def close(self):
        if self.ctx:
            bkv_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:  # noqa: BLE001 - interpreter shutdown
            pass

    # The C ABI receives bare pointers and trusts the sizes that the context's shape implies (_expect).
    _expect = staticmethod(_expect)

    def _rows(self, q: torch.Tensor, name: str) -> int:
        """Queries per query head of a [n_layers, batch, n_q_heads, n, head_dim] block."""
        c = self.cfg
        if q.dim() < 2 or q.shape[-1] != c.head_dim:
            raise ValueError(f"{name} must end in [n, head_dim = {c.head_dim}], got {tuple(q.shape)}")
        n = q.shape[-2]
        self._expect(q, c.n_layers * c.batch * c.n_q_heads * n * c.head_dim, name)
        return n

    def init_beacons(self, q_init: torch.Tensor):
        bkv_init_beacons(self.ctx, q_init, self._rows(q_init, "q_init"))

    def update(self, q_new: torch.Tensor, assign_out: torch.Tensor | None = None):
        n_new = self._rows(q_new, "q_new")
        c = self.cfg
        self._expect(assign_out, c.n_layers * c.batch * c.n_q_heads * n_new, "assign_out")
        bkv_update_beacons(self.ctx, q_new, n_new, assign_out)

    def update_seq(self, q_steps: torch.Tensor, assign_out: torch.Tensor | None = None):
        """Decode steps in order: q_steps is [n_steps, n_layers, batch, n_q_heads, head_dim]."""
        c = self.cfg
        per_step = c.n_layers * c.batch * c.n_q_heads
        if q_steps.dim() < 2 or q_steps.shape[-1] != c.head_dim or q_steps.numel() % (per_step * c.head_dim):
            raise ValueError(f"q_steps must be [n_steps, n_layers, batch, n_q_heads, head_dim = {c.head_dim}], "
                             f"got {tuple(q_steps.shape)}")
        n_steps = q_steps.numel() // (per_step * c.head_dim)
        self._expect(assign_out, per_step * n_steps, "assign_out")
        bkv_update_beacons_seq(self.ctx, q_steps, n_steps, assign_out)

    def compress(self, K, V, *, L, budget, t_pos, q_recent, recent_pos, kept_out=None, scores_out=None):
        c = self.cfg
        per_head = c.n_layers * c.batch * c.n_kv_heads
        self._expect(K, per_head * c.capacity * c.head_dim, "K")
        self._expect(V, per_head * c.capacity * c.head_dim, "V")
        self._expect(q_recent, c.n_layers * c.batch * c.n_q_heads * c.window * c.head_dim, "q_recent")
        if len(recent_pos) != c.window:
            raise ValueError(f"recent_pos has {len(recent_pos)} positions; the window is {c.window}")
        self._expect(kept_out, per_head * budget, "kept_out")
        self._expect(scores_out, per_head * c.capacity, "scores_out")
        if kept_out is None:
            kept_out = torch.empty(c.n_layers, c.batch, c.n_kv_heads, budget, dtype=torch.int32, device=K.device)
        bkv_compress(self.ctx, K, V, L, budget, t_pos, q_recent, recent_pos, kept_out, scores_out)
        return kept_out

    def compress_ragged(self, K, V, *, L, budget, t_pos, q_recent, recent_pos, kept_out=None, scores_out=None):
        """Per-instance cache lengths: L is an int32 CUDA tensor [n_layers, batch, n_kv_heads]; t_pos and
        recent_pos hold one position (one list of window positions) per batch row."""
        c = self.cfg
        per_head = c.n_layers * c.batch * c.n_kv_heads
        self._expect(K, per_head * c.capacity * c.head_dim, "K")
        self._expect(V, per_head * c.capacity * c.head_dim, "V")
        self._expect(L, per_head, "L")
        self._expect(q_recent, c.n_layers * c.batch * c.n_q_heads * c.window * c.head_dim, "q_recent")
        if len(t_pos) != c.batch:
            raise ValueError(f"t_pos has {len(t_pos)} positions; the batch is {c.batch}")
        if len(recent_pos) != c.batch or any(len(r) != c.window for r in recent_pos):
            raise ValueError(f"recent_pos must hold {c.batch} lists of {c.window} positions")
        self._expect(kept_out, per_head * budget, "kept_out")
        self._expect(scores_out, per_head * c.capacity, "scores_out")
        if kept_out is None:
            kept_out = torch.empty(c.n_layers, c.batch, c.n_kv_heads, budget, dtype=torch.int32, device=K.device)
        bkv_compress_ragged(self.ctx, K, V, L, budget, t_pos, q_recent, recent_pos, kept_out, scores_out)
        return kept_out

    # ------------------------------------------------------------ attention over the caches
    def _new(self, like: torch.Tensor, shape, dtype, shape2, dtype2):
        """Two new outputs, from the allocator pool of the context's stream (their memory may have been freed
        by work that is only ordered on that stream)."""
        device = like.device
        stream = _streams[self.ctx.value]
        if torch._C._cuda_getCurrentRawStream(device.index) == stream:
            return torch.empty(shape, dtype=dtype, device=device), torch.empty(shape2, dtype=dtype2, device=device)
        with torch.cuda.stream(torch.cuda.ExternalStream(stream, device=device)):
            return torch.empty(shape, dtype=dtype, device=device), torch.empty(shape2, dtype=dtype2, device=device)

    def reserve_attend(self, *, n_q: int = 1, n_groups: int = 0, weights: bool = False):
        """Workspace for attend (n_groups = 0) or attend_shared with n_q queries per head; needed once
        before the first call of that size (bkv_attend_reserve)."""
        bkv_attend_reserve(self.ctx, n_q, n_groups, weights)

    def _attend_args(self, q, K, V, length, weights, o_out, lse_out):
        batch, heads, d, lens, rows_kv = self._layer
        shape = q.shape
        if len(shape) != 4 or shape[0] != batch or shape[1] != heads or shape[3] != d:
            raise ValueError(f"q must be [batch = {batch}, n_q_heads = {heads}, n_q, head_dim = {d}], got "
                             f"{tuple(shape)}")
        expect = self._expect
        expect(K, rows_kv * d, "K")
        expect(V, rows_kv * d, "V")
        expect(length, lens, "length")
        expect(weights, rows_kv, "weights")
        if not q.is_cuda:
            raise TypeError("q must be a CUDA tensor")
        n_q = shape[2]
        if o_out is None and lse_out is None:
            o_out, lse_out = self._new(q, shape, torch.bfloat16, shape[:3], torch.float32)
        elif o_out is None:
            expect(lse_out, q.numel() // d, "lse_out")
            o_out, _ = self._new(q, shape, torch.bfloat16, 0, torch.float32)
        else:
            expect(o_out, q.numel(), "o_out")
            if lse_out is None:
                lse_out, _ = self._new(q, shape[:3], torch.float32, 0, torch.float32)
            else:
                expect(lse_out, q.numel() // d, "lse_out")
        return n_q, o_out, lse_out

    def attend(self, q, K, V, *, length, scale=None, weights=None, o_out=None, lse_out=None):
        """Attention of one layer's newest queries over its caches (bkv_attend): q [batch, n_q_heads, n_q,
        head_dim], K and V [batch, n_kv_heads, capacity, head_dim], length int32 [batch, n_kv_heads];
        weights fp32 [batch, n_kv_heads, capacity] is added to.  o_out and lse_out share no memory with q or the
        caches.  Returns (o, lse)."""
        n_q, o, lse = self._attend_args(q, K, V, length, weights, o_out, lse_out)
        bkv_attend(self.ctx, q, n_q, K, V, length, scale or 0.0, o, lse, weights)
        return o, lse

    def attend_shared(self, q, Kp, Vp, K, V, *, prefix_len, length, scale=None, weights=None, o_out=None,
                      lse_out=None):
        """attend for sequences that continue a shared prefix (bkv_attend_shared): Kp and Vp [n_groups,
        n_kv_heads, prefix_capacity, head_dim], prefix_len int32 [n_groups].  Returns (o, lse)."""
        c = self.cfg
        n_q, o, lse = self._attend_args(q, K, V, length, weights, o_out, lse_out)
        if Kp.dim() != 4 or Kp.shape[1] != c.n_kv_heads or Kp.shape[3] != c.head_dim:
            raise ValueError(f"Kp must be [n_groups, n_kv_heads = {c.n_kv_heads}, prefix_capacity, head_dim = "
                             f"{c.head_dim}], got {tuple(Kp.shape)}")
        groups, pcap = Kp.shape[0], Kp.shape[2]
        self._expect(Vp, Kp.numel(), "Vp")
        self._expect(prefix_len, groups, "prefix_len")
        bkv_attend_shared(self.ctx, q, n_q, Kp, Vp, prefix_len, groups, pcap, K, V, length, scale or 0.0, o, lse,
                          weights)
        return o, lse

    def _outputs(self, q, o_out, lse_out):
        """n_q, the pointer of q, and the outputs of an attention call, new where they are not given."""
        batch, heads, d = self._layer[:3]
        shape = q.shape
        if len(shape) != 4 or shape[0] != batch or shape[1] != heads or shape[3] != d:
            raise ValueError(f"q must be [batch = {batch}, n_q_heads = {heads}, n_q, head_dim = {d}], got "
                             f"{tuple(shape)}")
        if q.dtype is not torch.bfloat16 or not q.is_cuda or not q.is_contiguous():
            _ptr(q, torch.bfloat16, "q")
        n_q = shape[2]
        if o_out is None and lse_out is None:
            o, lse = self._new(q, shape, torch.bfloat16, shape[:3], torch.float32)
            return n_q, q.data_ptr(), o, lse, o.data_ptr(), lse.data_ptr()
        if o_out is None:
            o_out, _ = self._new(q, shape, torch.bfloat16, 0, torch.float32)
        elif lse_out is None:
            lse_out, _ = self._new(q, shape[:3], torch.float32, 0, torch.float32)
        n = batch * heads * n_q
        return (n_q, q.data_ptr(), o_out, lse_out, _arg(o_out, torch.bfloat16, n * d, "o_out"),
                _arg(lse_out, torch.float32, n, "lse_out"))

    def attend_window(self, q, K, V, *, length, window, n_sink=0, scale=None, o_out=None, lse_out=None):
        """attend where a query sees the `window` newest rows up to its own and the first `n_sink` rows
        (bkv_attend_window); the reservation is that of attend.  Returns (o, lse)."""
        _, _, d, lens, rows = self._layer
        kp, vp = _arg(K, torch.bfloat16, rows * d, "K"), _arg(V, torch.bfloat16, rows * d, "V")
        lp = _arg(length, torch.int32, lens, "length")
        n_q, qp, o, lse, op, ep = self._outputs(q, o_out, lse_out)
        rc = _lib.bkv_attend_window(self.ctx, qp, n_q, kp, vp, lp, window, n_sink, scale or 0.0, op, ep)
        if rc:
            _check(rc, "bkv_attend_window", self.ctx)
        return o, lse

    # ------------------------------------------------------------ caches in 4 bits
    def _cache4(self, K4, V4, S4, rows, suffix=""):
        d, u8 = self.cfg.head_dim, torch.uint8
        return (_arg(K4, u8, rows * (d // 2), "K4" + suffix), _arg(V4, u8, rows * (d // 2), "V4" + suffix),
                _arg(S4, torch.float16, rows * (d // 8), "S4" + suffix))

    def _rows4(self, K, V, first, length):
        """Pointers of K, V, first and length, and n_rows."""
        c, shape = self.cfg, K.shape
        batch, _, d, lens, _ = self._layer
        if len(shape) != 4 or shape[0] != batch or shape[1] != c.n_kv_heads or shape[3] != d:
            raise ValueError(f"K must be [batch = {batch}, n_kv_heads = {c.n_kv_heads}, n_rows, head_dim = {d}], got "
                             f"{tuple(shape)}")
        n, bf16, i32 = lens * shape[2] * d, torch.bfloat16, torch.int32
        return (_arg(K, bf16, n, "K"), _arg(V, bf16, n, "V"), _arg(first, i32, lens, "first"),
                _arg(length, i32, lens, "length"), shape[2])

    def pack4(self, K, V, K4, V4, S4, *, length, first=None):
        """Writes rows of one layer into its 4-bit caches (bkv_pack4): row i of K and V [batch, n_kv_heads, n_rows,
        head_dim] becomes row first + i of its cache, for first + i < length.  K4 and V4 are uint8 [batch,
        n_kv_heads, capacity, head_dim / 2], S4 fp16 [batch, n_kv_heads, capacity, 2, head_dim / 32, 2]; first
        (None: 0) and length int32 [batch, n_kv_heads]."""
        kp, vp, fp, lp, n = self._rows4(K, V, first, length)
        k4, v4, s4 = self._cache4(K4, V4, S4, self._layer[4])
        rc = _lib.bkv_pack4(self.ctx, kp, vp, n, fp, lp, k4, v4, s4)
        if rc:
            _check(rc, "bkv_pack4", self.ctx)

    def unpack4(self, K4, V4, S4, K_out, V_out, *, length, first=None):
        """The inverse of pack4 (bkv_unpack4): row first + i of each cache, below its length, to row i of K_out and
        V_out; their other rows keep what they held."""
        kp, vp, fp, lp, n = self._rows4(K_out, V_out, first, length)
        k4, v4, s4 = self._cache4(K4, V4, S4, self._layer[4])
        rc = _lib.bkv_unpack4(self.ctx, k4, v4, s4, n, fp, lp, kp, vp)
        if rc:
            _check(rc, "bkv_unpack4", self.ctx)

    def reserve_attend4(self, *, n_q: int = 1, weights: bool = False):
        """Workspace for attend4 with n_q queries per head (bkv_attend4_reserve)."""
        bkv_attend4_reserve(self.ctx, n_q, weights)

    def attend4(self, q, K4, V4, S4, *, length, scale=None, weights=None, o_out=None, lse_out=None):
        """attend over one layer's 4-bit caches, which are those of pack4 (bkv_attend4: made for up to some 16 query
        rows per KV head; with more, attend over bf16 caches is faster).  Returns (o, lse)."""
        _, _, _, lens, rows = self._layer
        k4, v4, s4 = self._cache4(K4, V4, S4, rows)
        lp, wp = _arg(length, torch.int32, lens, "length"), _arg(weights, torch.float32, rows, "weights")
        n_q, qp, o, lse, op, ep = self._outputs(q, o_out, lse_out)
        rc = _lib.bkv_attend4(self.ctx, qp, n_q, k4, v4, s4, lp, scale or 0.0, op, ep, wp)
        if rc:
            _check(rc, "bkv_attend4", self.ctx)
        return o, lse

    def evict4(self, K4, V4, S4, weights, *, L, budget, K4_out=None, V4_out=None, S4_out=None, weights_out=None,
               kept_out=None, len_out=None):
        """evict for 4-bit caches of all layers (bkv_evict4), in place or, with all of K4_out, V4_out, S4_out and
        weights_out, into other caches.  Returns (kept rows, new lengths)."""
        given = (K4_out is not None) + (V4_out is not None) + (S4_out is not None) + (weights_out is not None)
        if given == 0:
            K4_out, V4_out, S4_out, weights_out = K4, V4, S4, weights
        elif given != 4:
            raise ValueError("K4_out, V4_out, S4_out and weights_out come together or not at all")
        n_inst, f32, i32 = self.n_inst, torch.float32, torch.int32
        cap_out = weights_out.numel() // n_inst
        rows = n_inst * self.cfg.capacity
        k4, v4, s4 = self._cache4(K4, V4, S4, rows)
        ko, vo, so = (k4, v4, s4) if given == 0 else self._cache4(K4_out, V4_out, S4_out, n_inst * cap_out, "_out")
        wp, wo = _arg(weights, f32, rows, "weights"), _arg(weights_out, f32, n_inst * cap_out, "weights_out")
        lp = _arg(L, i32, n_inst, "L")
        kept_out, len_out = self._evict_outputs(K4, budget, kept_out, len_out)
        rc = _lib.bkv_evict4(self.ctx, k4, v4, s4, wp, lp, budget, ko, vo, so, wo, cap_out,
                             _arg(kept_out, i32, n_inst * budget, "kept_out"), _arg(len_out, i32, n_inst, "len_out"))
        if rc:
            _check(rc, "bkv_evict4", self.ctx)
        return kept_out, len_out

    def _evict_outputs(self, K, budget, kept_out, len_out):
        """The outputs of an eviction, new where they are not given."""
        if not K.is_cuda:
            raise TypeError("K must be a CUDA tensor")
        if kept_out is None or len_out is None:
            c, i32 = self.cfg, torch.int32
            shape = (c.n_layers, c.batch, c.n_kv_heads)
            kept, length = self._new(K, shape + (max(0, budget) if kept_out is None else 0,), i32, shape, i32)
            kept_out = kept if kept_out is None else kept_out
            len_out = length if len_out is None else len_out
        return kept_out, len_out

    def evict(self, K, V, weights, *, L, budget, K_out=None, V_out=None, weights_out=None, kept_out=None,
              len_out=None):
        """Eviction by accumulated weight (bkv_evict), in place or, with K_out, V_out and weights_out of
        [n_layers, batch, n_kv_heads, capacity_out] rows, into another cache.  L: int32 CUDA tensor
        [n_layers, batch, n_kv_heads]; len_out may be L.  A window that the context's limit on G * window refuses
        is taken by a context of its own with n_q_heads = n_kv_heads.  Returns (kept rows, new lengths)."""
        c = self.cfg
        given = (K_out is not None) + (V_out is not None) + (weights_out is not None)
        if given == 0:
            K_out, V_out, weights_out = K, V, weights
        elif given != 3:
            raise ValueError("K_out, V_out and weights_out come together or not at all")
        n_inst, d = self.n_inst, c.head_dim
        rows = n_inst * c.capacity
        cap_out = weights_out.numel() // n_inst
        rows_out = n_inst * cap_out
        self._expect(K, rows * d, "K")
        self._expect(V, rows * d, "V")
        self._expect(K_out, rows_out * d, "K_out")
        self._expect(V_out, rows_out * d, "V_out")
        self._expect(weights, rows, "weights")
        self._expect(L, n_inst, "L")
        self._expect(weights_out, rows_out, "weights_out")
        self._expect(kept_out, n_inst * budget, "kept_out")
        self._expect(len_out, n_inst, "len_out")
        kept_out, len_out = self._evict_outputs(K, budget, kept_out, len_out)
        bkv_evict(self.ctx, K, V, weights, L, budget, K_out, V_out, weights_out, cap_out, kept_out, len_out)
        return kept_out, len_out

    def state(self):
        c = self.cfg
        dev = torch.device("cuda", torch.cuda.current_device())
        cent = torch.empty(self.n_inst, c.n_beacons, c.head_dim, dtype=torch.float32, device=dev)
        sums = torch.empty(self.n_inst, c.n_beacons, c.head_dim, dtype=torch.float64, device=dev)
        counts = torch.empty(self.n_inst, c.n_beacons, dtype=torch.int64, device=dev)
        bkv_get_state(self.ctx, cent, sums, counts)
        return cent, sums, counts

    def set_state(self, cent, sums, counts):
        c = self.cfg
        self._expect(cent, self.n_inst * c.n_beacons * c.head_dim, "centroids")
        self._expect(sums, self.n_inst * c.n_beacons * c.head_dim, "sums")
        self._expect(counts, self.n_inst * c.n_beacons, "counts")
        bkv_set_state(self.ctx, cent, sums, counts)

    def cfps_state(self):
        """Continual FPS buffers: (bf16 [L, B, Hq, n_beacons + window, d], int32 sizes [L, B, Hq])."""
        c = self.cfg
        dev = torch.device("cuda", torch.cuda.current_device())
        buf = torch.empty(c.n_layers, c.batch, c.n_q_heads, c.n_beacons + c.window, c.head_dim, dtype=torch.bfloat16,
                          device=dev)
        sizes = torch.empty(c.n_layers, c.batch, c.n_q_heads, dtype=torch.int32, device=dev)
        bkv_get_cfps_state(self.ctx, buf, sizes)
        return buf, sizes

    def set_cfps_state(self, buf, sizes):
        c = self.cfg
        heads = c.n_layers * c.batch * c.n_q_heads
        self._expect(buf, heads * (c.n_beacons + c.window) * c.head_dim, "buffers")
        self._expect(sizes, heads, "sizes")
        bkv_set_cfps_state(self.ctx, buf, sizes)

    def sync(self):
        bkv_sync(self.ctx)

"""Thin ctypes binding of libtessera.so: argument marshalling only.

Every step of the path runs inside the library's kernels.  torch appears here
only as the owner of device memory and of the current stream.  Importing this
module fails loudly when the library has not been built; there is no fallback.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtessera.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        "libtessera.so is missing: build it with `python -m paper_2609_32999_b200.build` "
        "(nvcc, sm_100a).  This package has no CPU or eager fallback.")
_lib = ctypes.CDLL(LIB_PATH)

OK = 0
INVALID_ARG, UNSORTED_POSITIONS, UNIT_OVERLAP, UNCOVERED_POSITION = -1, -2, -3, -4
PAGE_OUT_OF_RANGE, OUT_OF_PAGES, UNSUPPORTED_SHAPE, CUDA_ERROR, DEVICE_TIMEOUT = -5, -6, -7, -8, -9
PLAN_HOST_ONLY = 1
FUSE_ROPE = 1

_I32P = ctypes.POINTER(ctypes.c_int32)


class ModelCfg(ctypes.Structure):
    _fields_ = [("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("rope_theta", ctypes.c_double), ("inv_freq", ctypes.POINTER(ctypes.c_double)),
                ("rope_pairing", ctypes.c_int32), ("sm_scale", ctypes.c_float)]


class ComposeDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("seq_len", _I32P), ("unit_off", _I32P), ("unit_len", _I32P),
                ("unit_cached_pos", _I32P), ("unit_cached_stride", _I32P), ("unit_target_pos", _I32P),
                ("unit_page_off", _I32P), ("unit_pages", _I32P), ("recompute_off", _I32P),
                ("recompute_pos", _I32P), ("free_pages", _I32P), ("n_free", ctypes.c_int32),
                ("unit_src_offset", _I32P), ("num_source_pages", ctypes.c_int32), ("unit_target_stride", _I32P),
                ("unit_retain_page_off", _I32P), ("unit_retain_pages", _I32P), ("retain_pool_pages", ctypes.c_int32)]


class PlanInfo(ctypes.Structure):
    _fields_ = [("total_tokens", ctypes.c_int64), ("n_q", ctypes.c_int64), ("cached_tokens", ctypes.c_int64),
                ("qk_pairs", ctypes.c_int64), ("gather_bytes", ctypes.c_int64), ("attn_flops", ctypes.c_int64),
                ("n_rope_rows", ctypes.c_int32), ("n_gather_items", ctypes.c_int32),
                ("n_attn_items", ctypes.c_int32), ("attn_kernel", ctypes.c_int32),
                ("retained_tokens", ctypes.c_int64), ("attn_mma_pairs", ctypes.c_int64)]


class FreshRows(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("q_out", ctypes.c_void_p),
                ("q_row", ctypes.c_int64), ("k_row", ctypes.c_int64), ("v_row", ctypes.c_int64),
                ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("eps", ctypes.c_float)]


class DecodeDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("block_table", ctypes.c_void_p),
                ("seq_len", ctypes.c_void_p), ("num_pool_pages", ctypes.c_int32), ("window", ctypes.c_int32),
                ("n_sink", ctypes.c_int32)]


EXPORTS = ["tessera_plan_create", "tessera_plan_create_windowed", "tessera_plan_destroy", "tessera_plan_block_table", "tessera_plan_get_info",
           "tessera_plan_status", "tessera_kv_compose", "tessera_kv_compose_from", "tessera_kv_compose_from_fp8", "tessera_kv_retain_fp8", "tessera_rope_shift", "tessera_rope_fresh", "tessera_extend_write", "tessera_partial_prefill_attn", "tessera_kv_compose_k8", "tessera_partial_prefill_attn_k8",
           "tessera_composed_prefill_host", "tessera_composed_prefill_host_tier", "tessera_rope_shift_static", "tessera_selftest_bounded_wait", "tessera_last_error",
           "tessera_kv_retain_kv4", "tessera_kv_compose_from_kv4", "tessera_extend_write_norm", "tessera_decode_write", "tessera_decode_write_kv4",
           "tessera_decode_workspace_bytes", "tessera_decode_attn", "tessera_decode_attn_kv4",
           "tessera_launch_count"]

_vp = ctypes.c_void_p
_lib.tessera_plan_create.argtypes = [ctypes.POINTER(ModelCfg), ctypes.POINTER(ComposeDesc), ctypes.c_int32,
                                     ctypes.c_uint32, ctypes.POINTER(_vp), _vp]
_lib.tessera_plan_create_windowed.argtypes = [ctypes.POINTER(ModelCfg), ctypes.POINTER(ComposeDesc), ctypes.c_int32,
                                              ctypes.c_int32, ctypes.c_int32, ctypes.c_uint32, ctypes.POINTER(_vp), _vp]
_lib.tessera_plan_destroy.argtypes = [_vp]
_lib.tessera_plan_block_table.argtypes = [_vp, ctypes.POINTER(_I32P), ctypes.POINTER(_I32P), ctypes.POINTER(_I32P)]
_lib.tessera_plan_get_info.argtypes = [_vp, ctypes.POINTER(PlanInfo)]
_lib.tessera_plan_status.argtypes = [_vp, _I32P, _vp]
_lib.tessera_kv_compose.argtypes = [_vp, _vp, _vp, ctypes.c_uint32, _vp]
_lib.tessera_kv_compose_from.argtypes = [_vp, _vp, _vp, _vp, _vp, ctypes.c_uint32, _vp]
_lib.tessera_kv_compose_from_fp8.argtypes = [_vp, _vp, _vp, ctypes.c_float, ctypes.c_float, _vp, _vp, ctypes.c_uint32, _vp]
_lib.tessera_kv_retain_fp8.argtypes = [_vp, _vp, _vp, _vp, _vp, ctypes.c_float, ctypes.c_float, ctypes.c_uint32, _vp]
_lib.tessera_rope_shift.argtypes = [_vp, _vp, _vp]
_lib.tessera_rope_fresh.argtypes = [_vp, _vp, _vp, _vp]
_lib.tessera_extend_write.argtypes = [_vp] * 9
_lib.tessera_partial_prefill_attn.argtypes = [_vp] * 9
_lib.tessera_kv_compose_k8.argtypes = [_vp, _vp, _vp, _vp, _vp, ctypes.c_float, ctypes.c_uint32, _vp]
_lib.tessera_partial_prefill_attn_k8.argtypes = [_vp, _vp, ctypes.c_float, _vp, _vp, ctypes.c_float, _vp, _vp, _vp, _vp, _vp]
_lib.tessera_composed_prefill_host.argtypes = [_vp] * 9
_lib.tessera_composed_prefill_host_tier.argtypes = [_vp, _vp, _vp, ctypes.c_int32, ctypes.c_float, ctypes.c_float,
                                                    _vp, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_int32, _vp]
_lib.tessera_rope_shift_static.argtypes = [ctypes.POINTER(ModelCfg), _vp, ctypes.c_int64, _vp, _vp, ctypes.c_int32,
                                           _I32P, ctypes.c_int32, _vp]
_lib.tessera_selftest_bounded_wait.argtypes = [ctypes.c_int64, _I32P, ctypes.POINTER(ctypes.c_int64), _vp]
_lib.tessera_kv_retain_kv4.argtypes = _lib.tessera_kv_compose_from_kv4.argtypes = [_vp, _vp, _vp, _vp, _vp, ctypes.c_uint32, _vp]
# (structures by address: ctypes takes an integer in half the time it takes to check a typed pointer)
_lib.tessera_extend_write_norm.argtypes = [_vp] * 7
_lib.tessera_decode_write.argtypes = _lib.tessera_decode_write_kv4.argtypes = [_vp] * 6
_lib.tessera_decode_workspace_bytes.argtypes = [_vp, ctypes.POINTER(ctypes.c_int64)]
_lib.tessera_decode_attn.argtypes = _lib.tessera_decode_attn_kv4.argtypes = [_vp] * 8 + [ctypes.c_int64, _vp]
_lib.tessera_last_error.argtypes = [ctypes.c_char_p, ctypes.c_int32]
_lib.tessera_launch_count.argtypes = []
_lib.tessera_launch_count.restype = ctypes.c_int64
for _n in EXPORTS[:-1]:
    getattr(_lib, _n).restype = ctypes.c_int32


class TesseraError(RuntimeError):
    def __init__(self, status: int, text: str):
        super().__init__("tessera status %d: %s" % (status, text))
        self.status = status


class ArgumentError(TesseraError, ValueError):
    """A tensor of the wrong kind, refused before the library is called."""

    def __init__(self, text: str):
        super().__init__(INVALID_ARG, text)


def last_error() -> str:
    buf = ctypes.create_string_buffer(512)
    _lib.tessera_last_error(buf, 512)
    return buf.value.decode("utf-8", "replace")


def _check(st: int) -> None:
    if st != OK:
        raise TesseraError(st, last_error())


def launch_count() -> int:
    return int(_lib.tessera_launch_count())


def _arr(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32))


def _ptr(a: np.ndarray):
    return a.ctypes.data_as(_I32P)


def _dev(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _current_device() -> int:
    import torch
    return torch._C._cuda_getDevice()


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        # the handle alone: torch.cuda.current_stream() builds a Stream object, 3.3 us of an 8 us call
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()) or None
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream or None


def _frequencies(sh, inv_freq) -> Optional[np.ndarray]:
    """Rotary frequencies as the library reads them: head_dim / 2 numbers."""
    if inv_freq is None:
        return None
    inv = np.ascontiguousarray(inv_freq, dtype=np.float64)
    if inv.size < sh.head_dim // 2:
        raise ArgumentError("inv_freq: %d numbers, a head_dim of %d takes %d" % (inv.size, sh.head_dim, sh.head_dim // 2))
    return inv


def _model_cfg(sh, inv: Optional[np.ndarray]) -> ModelCfg:
    return ModelCfg(sh.num_q_heads, sh.num_kv_heads, sh.head_dim, sh.page_size, float(sh.rope_theta),
                    None if inv is None else inv.ctypes.data_as(ctypes.POINTER(ctypes.c_double)),
                    int(sh.rope_pairing), float(sh.sm_scale))


def _expect(what: str, t, index: int, dtype, shape, rows: bool = False) -> int:
    """Device, type and shape of a tensor; contiguous, or (rows) with heads side by side inside rows any distance apart: returned in
    elements, 0 where the tensor is contiguous."""
    if t.dtype is dtype and t.shape == shape and t.get_device() == index and t.is_contiguous():
        return 0
    if t.dtype is not dtype or t.shape != shape or t.get_device() != index:
        raise ArgumentError("%s: expected %s of %s on device %d, got %s of %s on device %d"
                            % (what, tuple(shape), dtype, index, tuple(t.shape), t.dtype, t.get_device()))
    if not (rows and t.stride()[1:] == (shape[2], 1) and t.stride(0) >= shape[1] * shape[2]):
        raise ArgumentError("%s: strides %s" % (what, tuple(t.stride())))
    return t.stride(0)


def _expect_pool(what: str, t, index: int, dtype, shape, pinned: bool = False) -> None:
    """A contiguous pool of at least shape[0] pages on the device or (pinned) in page-locked host memory.  What is None the library
    refuses by itself."""
    if t is None or (t.dtype is dtype and t.shape == shape and t.get_device() == index and t.is_contiguous()):
        return
    there = t.get_device() == index or (pinned and t.device.type == "cpu" and t.is_pinned())
    if not (there and t.dtype is dtype and t.dim() == len(shape) and t.shape[0] >= shape[0] and t.shape[1:] == shape[1:] and t.is_contiguous()):
        raise ArgumentError("%s: expected %s (or more pages) of %s, contiguous, on device %d, got %s of %s on %s"
                            % (what, tuple(shape), dtype, index, tuple(t.shape), t.dtype, t.device))


def _fresh_rows(sh, n: int, index: int, bfloat16, q, q_out, k, v, q_weight, k_weight, eps) -> FreshRows:
    hq, h, d = sh.num_q_heads, sh.num_kv_heads, sh.head_dim
    q_row = 0
    if q is not None:
        q_row = _expect("q", q, index, bfloat16, (n, hq, d), rows=True)
        _expect("q_out", q_out, index, bfloat16, (n, hq, d))
    k_row, v_row = _expect("k_new", k, index, bfloat16, (n, h, d), rows=True), _expect("v_new", v, index, bfloat16, (n, h, d), rows=True)
    if q_weight is not None:
        _expect("q_weight", q_weight, index, bfloat16, (d,))
    if k_weight is not None:
        _expect("k_weight", k_weight, index, bfloat16, (d,))
    return FreshRows(_dev(q), k.data_ptr(), v.data_ptr(), None if q is None else q_out.data_ptr(), q_row, k_row, v_row, _dev(q_weight), _dev(k_weight), eps)


class Plan:
    """tessera_plan_create / tessera_plan_destroy with host arrays taken from a Workload-like
    object (anything with the descriptor's field names and a `.shape` model description).  With `window` > 0
    its attention calls see the last `window` positions and the first `n_sink` (tessera_plan_create_windowed)."""

    def __init__(self, w, host_only: bool = False, stream=None, inv_freq=None, window: int = 0, n_sink: int = 0):
        sh = w.shape
        self._keep = [_arr(getattr(w, f)) for f in
                      ("seq_len", "unit_off", "unit_len", "unit_cached_pos", "unit_cached_stride",
                       "unit_target_pos", "unit_page_off", "unit_pages", "recompute_off", "recompute_pos",
                       "free_pages")]
        a = self._keep
        self._inv = _frequencies(sh, inv_freq)
        cfg = _model_cfg(sh, self._inv)
        self.shape = sh
        opt = [None if getattr(w, f, None) is None else _arr(getattr(w, f))
               for f in ("unit_src_offset", "unit_target_stride", "unit_retain_page_off", "unit_retain_pages")]
        op = [None if x is None else _ptr(x) for x in opt]
        desc = ComposeDesc(len(a[0]), *[_ptr(x) for x in a[:11]], len(a[10]), op[0],
                           int(getattr(w, "num_source_pages", 0) or 0), op[1], op[2], op[3],
                           int(getattr(w, "retain_pool_pages", 0) or 0))
        self._opt = opt
        self._h = _vp()
        self.host_only = host_only
        self._row = (sh.page_size, sh.num_kv_heads, sh.head_dim)
        self._pool = (int(w.num_pool_pages),) + self._row
        self._sources = (desc.num_source_pages,) + self._row
        self._pool4, self._sources4 = pool4_shape(sh, self._pool[0]), pool4_shape(sh, self._sources[0])
        self._cache = (desc.retain_pool_pages,) + self._row if desc.retain_pool_pages > 0 else self._pool
        args = (PLAN_HOST_ONLY if host_only else 0, ctypes.byref(self._h), None if host_only else _stream(stream))
        if window == 0 and n_sink == 0:
            st = _lib.tessera_plan_create(ctypes.byref(cfg), ctypes.byref(desc), int(w.num_pool_pages), *args)
        else:
            st = _lib.tessera_plan_create_windowed(ctypes.byref(cfg), ctypes.byref(desc), int(w.num_pool_pages), int(window), int(n_sink), *args)
        _check(st)
        self.batch = len(a[0])
        self.info = PlanInfo()
        _check(_lib.tessera_plan_get_info(self._h, ctypes.byref(self.info)))
        # share of the tensor-core (row, key) products that is not an algorithmic (query row, key) pair
        pairs = self.info.qk_pairs * sh.num_q_heads
        self.masked_mma_fraction = 1.0 - pairs / self.info.attn_mma_pairs if self.info.attn_mma_pairs else 0.0

    def block_table(self):
        """(page_off, pages, src_slot) as numpy copies of the plan's host tables."""
        po, pg, ss = _I32P(), _I32P(), _I32P()
        _check(_lib.tessera_plan_block_table(self._h, ctypes.byref(po), ctypes.byref(pg), ctypes.byref(ss)))
        page_off = np.ctypeslib.as_array(po, shape=(self.batch + 1,)).copy()
        n_pages, n_tok = int(page_off[-1]), int(self.info.total_tokens)
        pages = np.ctypeslib.as_array(pg, shape=(n_pages,)).copy() if n_pages else np.zeros(0, np.int32)
        src = np.ctypeslib.as_array(ss, shape=(n_tok,)).copy() if n_tok else np.zeros(0, np.int32)
        return page_off, pages, src

    def status(self, stream=None) -> int:
        detail = ctypes.c_int32(0)
        st = _lib.tessera_plan_status(self._h, ctypes.byref(detail), _stream(stream))
        if st not in (OK, DEVICE_TIMEOUT):
            _check(st)
        return int(detail.value)

    def kv_compose(self, k_pool, v_pool, fuse_rope: bool = True, stream=None) -> None:
        _check(_lib.tessera_kv_compose(self._h, _dev(k_pool), _dev(v_pool), FUSE_ROPE if fuse_rope else 0,
                                       _stream(stream)))

    def kv_compose_from(self, k_src, v_src, k_pool, v_pool, fuse_rope: bool = True, stream=None) -> None:
        """Sources in a separate pool (pinned host tensors or device tensors), destinations in the pools."""
        _check(_lib.tessera_kv_compose_from(self._h, _dev(k_src), _dev(v_src), _dev(k_pool), _dev(v_pool),
                                            FUSE_ROPE if fuse_rope else 0, _stream(stream)))

    def kv_compose_from_fp8(self, k_src8, v_src8, k_scale: float, v_scale: float, k_pool, v_pool,
                            fuse_rope: bool = True, stream=None) -> None:
        """Sources are e4m3 codes (uint8 or float8_e4m3fn tensors) standing for code * scale."""
        _check(_lib.tessera_kv_compose_from_fp8(self._h, _dev(k_src8), _dev(v_src8), k_scale, v_scale, _dev(k_pool),
                                                _dev(v_pool), FUSE_ROPE if fuse_rope else 0, _stream(stream)))

    def kv_retain_fp8(self, k_src, v_src, k_dst8, v_dst8, k_scale: float, v_scale: float, fuse_rope: bool = True,
                      stream=None) -> None:
        """16-bit source pools -> e4m3 destination pools (the plan's destination pages index the 8-bit pools)."""
        _check(_lib.tessera_kv_retain_fp8(self._h, _dev(k_src), _dev(v_src), _dev(k_dst8), _dev(v_dst8), k_scale, v_scale,
                                          FUSE_ROPE if fuse_rope else 0, _stream(stream)))

    def _tier4(self, k_src, v_src, source_dtype, sources, k_dst, v_dst, dtype, pool, stream):
        """Checks the pools of a 4-bit tier call; returns the stream's handle.  (A plan that serves no such call the library refuses.)"""
        if self.host_only or self._sources[0] <= 0:
            return None
        index = _current_device()                                      # (the library refuses a current device that is not the plan's)
        _expect_pool("k source", k_src, index, source_dtype, sources, pinned=True)
        _expect_pool("v source", v_src, index, source_dtype, sources, pinned=True)
        _expect_pool("k destination", k_dst, index, dtype, pool, pinned=True)
        _expect_pool("v destination", v_dst, index, dtype, pool, pinned=True)
        return _stream(stream)

    def kv_retain_kv4(self, k_src, v_src, k_dst4, v_dst4, fuse_rope: bool = True, stream=None) -> None:
        """16-bit source pools -> 4-bit pools (pool4_shape); the plan's destination pages index the 4-bit pools.  Pools live on the plan's device,
        the current one, or in page-locked host memory, and may have more pages than the plan counts."""
        import torch
        st = self._tier4(k_src, v_src, torch.bfloat16, self._sources, k_dst4, v_dst4, torch.uint8, self._pool4, stream)
        _check(_lib.tessera_kv_retain_kv4(self._h, _dev(k_src), _dev(v_src), _dev(k_dst4), _dev(v_dst4), FUSE_ROPE if fuse_rope else 0, st))

    def kv_compose_from_kv4(self, k_src4, v_src4, k_pool, v_pool, fuse_rope: bool = True, stream=None) -> None:
        """Sources in 4-bit pools (pool4_shape), destinations in the 16-bit pools, keys rotated on the way.  Pools as for kv_retain_kv4."""
        import torch
        st = self._tier4(k_src4, v_src4, torch.uint8, self._sources4, k_pool, v_pool, torch.bfloat16, self._pool, stream)
        _check(_lib.tessera_kv_compose_from_kv4(self._h, _dev(k_src4), _dev(v_src4), _dev(k_pool), _dev(v_pool), FUSE_ROPE if fuse_rope else 0, st))

    def rope_shift(self, k_pool, stream=None) -> None:
        _check(_lib.tessera_rope_shift(self._h, _dev(k_pool), _stream(stream)))

    def rope_fresh(self, q, k_new, stream=None) -> None:
        """Rotate fresh q / k_new rows in place for their target positions (either may be None)."""
        _check(_lib.tessera_rope_fresh(self._h, _dev(q), _dev(k_new), _stream(stream)))

    def extend_write(self, k_pool, v_pool, q, k_new_raw, v_new, k_cache=None, v_cache=None, stream=None) -> None:
        """Fused write side of the extend pass: rotate q in place, write rotated K / V rows to their slots
        and the raw rows of captured units to k_cache / v_cache (attention then runs with k_new = v_new = None)."""
        _check(_lib.tessera_extend_write(self._h, _dev(k_pool), _dev(v_pool), _dev(q), _dev(k_new_raw), _dev(v_new),
                                         _dev(k_cache), _dev(v_cache), _stream(stream)))

    def extend_write_norm(self, k_pool, v_pool, q, q_out, k_new_raw, v_new, q_weight=None, k_weight=None, eps: float = 1e-6, k_cache=None,
                          v_cache=None, stream=None) -> None:
        """extend_write with per-head norms of q and k before the rotation, q written to q_out (q itself, or another tensor); q, k_new_raw and
        v_new may be slices [n_q, heads, D] of a fused projection.  q None: keys and values alone.  All tensors live on the plan's device, the
        current one; cache pools may be page-locked host memory."""
        from torch import bfloat16
        index = -1 if self.host_only else _current_device()            # (the library refuses a current device that is not the plan's)
        _expect_pool("k_pool", k_pool, index, bfloat16, self._pool)
        _expect_pool("v_pool", v_pool, index, bfloat16, self._pool)
        if self.info.retained_tokens > 0:
            _expect_pool("k_cache", k_cache, index, bfloat16, self._cache, pinned=True)
            _expect_pool("v_cache", v_cache, index, bfloat16, self._cache, pinned=True)
        rows = _fresh_rows(self.shape, int(self.info.n_q), index, bfloat16, q, q_out, k_new_raw, v_new, q_weight, k_weight, eps)
        _check(_lib.tessera_extend_write_norm(self._h, _dev(k_pool), _dev(v_pool), ctypes.addressof(rows), _dev(k_cache), _dev(v_cache), _stream(stream)))

    def partial_prefill_attn(self, k_pool, v_pool, q, k_new, v_new, out, lse=None, stream=None) -> None:
        _check(_lib.tessera_partial_prefill_attn(self._h, _dev(k_pool), _dev(v_pool), _dev(q), _dev(k_new),
                                                 _dev(v_new), _dev(out), _dev(lse), _stream(stream)))

    def kv_compose_k8(self, k_src, v_src, k_pool8, v_pool, k_scale: float, fuse_rope: bool = True, stream=None) -> None:
        """16-bit source pools -> keys as e4m3 codes in k_pool8 (rotated on the way), values into the 16-bit v_pool."""
        _check(_lib.tessera_kv_compose_k8(self._h, _dev(k_src), _dev(v_src), _dev(k_pool8), _dev(v_pool), float(k_scale),
                                          FUSE_ROPE if fuse_rope else 0, _stream(stream)))

    def partial_prefill_attn_k8(self, k_pool8, k_scale: float, v_pool, q, q_scale: float, k_new, v_new, out, lse=None,
                                stream=None) -> None:
        """Attention over 8-bit (e4m3) key pages: q is quantised by the call, k_pool8 holds codes."""
        _check(_lib.tessera_partial_prefill_attn_k8(self._h, _dev(k_pool8), float(k_scale), _dev(v_pool), _dev(q),
                                                    float(q_scale), _dev(k_new), _dev(v_new), _dev(out), _dev(lse),
                                                    _stream(stream)))

    def composed_prefill_host(self, k_pool, v_pool, q_host, k_new_host, v_new_host, out_host, lse_host=None,
                              stream=None) -> None:
        _check(_lib.tessera_composed_prefill_host(self._h, _dev(k_pool), _dev(v_pool), _dev(q_host),
                                                  _dev(k_new_host), _dev(v_new_host), _dev(out_host),
                                                  _dev(lse_host), _stream(stream)))

    def composed_prefill_host_tier(self, k_src_host, v_src_host, k_pool, v_pool, q, k_new, v_new, out, lse=None,
                                   src_format: int = 0, k_scale: float = 1.0, v_scale: float = 1.0,
                                   reader_blocks: int = 0, stream=None) -> None:
        """Cached units in pinned host pools (bf16, or e4m3 codes with src_format=1), pulled over the link
        chunk by chunk by a small reader launch while attention of the chunks already there runs."""
        _check(_lib.tessera_composed_prefill_host_tier(self._h, _dev(k_src_host), _dev(v_src_host), int(src_format),
                                                       float(k_scale), float(v_scale), _dev(k_pool), _dev(v_pool),
                                                       _dev(q), _dev(k_new), _dev(v_new), _dev(out), _dev(lse),
                                                       int(reader_blocks), _stream(stream)))

    def destroy(self) -> None:
        if self._h:
            h, self._h = self._h, _vp()        # the plan is gone even when its memory could not be released
            _check(_lib.tessera_plan_destroy(h))

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def pool4_shape(shape, num_pages: int):
    """Shape of a 4-bit pool (uint8) of num_pages pages."""
    return (int(num_pages), shape.num_kv_heads, shape.page_size * (shape.head_dim // 2 + 8))


class Decode:
    """The step after the first token (tessera_decode_*): one new token a request.

    block_table [batch, max_pages] and seq_lens [batch] are int32 device tensors that the caller goes on updating in place;
    they are read by every call when it runs on the GPU, so a step may be captured into a graph.  seq_lens counts the new
    token, whose position is seq_lens - 1; 0 leaves a place out.  `workspace` (uint8, all zeros before its first use; made
    here by default) must not be shared by calls that can overlap on the GPU: use a Decode for each stream or concurrent graph.
    Keep the object as long as graphs that captured its calls.  Without `workspace` it cannot be made while a graph is captured.
    All tensors live on the device of block_table, which is the current one during the calls."""

    def __init__(self, shape, block_table, seq_lens, num_pool_pages: int, window: int = 0, n_sink: int = 0, inv_freq=None, workspace=None):
        import torch
        # (the frequencies here, once: 64 powers in every call's host time otherwise)
        d = shape.head_dim
        self._inv = _frequencies(shape, [float(shape.rope_theta) ** (-2.0 * m / d) for m in range(d // 2)] if inv_freq is None else inv_freq)
        if block_table.device.type != "cuda" or block_table.dim() != 2:
            raise ValueError("block_table: a [batch, max_pages] tensor on a CUDA device")
        self.shape, self.batch, self.device = shape, int(seq_lens.shape[0]), block_table.device
        self._index = block_table.get_device()
        self._current, self._raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
        self._bf16, self._f32, self._u8 = torch.bfloat16, torch.float32, torch.uint8
        _expect("block_table", block_table, self._index, torch.int32, (self.batch, int(block_table.shape[1])))
        _expect("seq_lens", seq_lens, self._index, torch.int32, (self.batch,))
        self._cfg = _model_cfg(shape, self._inv)
        self.block_table, self.seq_lens, self.num_pool_pages = block_table, seq_lens, int(num_pool_pages)
        self._desc = DecodeDesc(self.batch, int(block_table.shape[1]), _dev(block_table), _dev(seq_lens), self.num_pool_pages, int(window), int(n_sink))
        self._args = ctypes.addressof(self._cfg), ctypes.addressof(self._desc)
        need = ctypes.c_int64(0)
        with torch.cuda.device(self.device):
            _check(_lib.tessera_decode_workspace_bytes(self._args[0], ctypes.byref(need)))
            if workspace is None:
                if torch.cuda.is_current_stream_capturing():
                    raise ValueError("a graph is being captured: make the Decode before, or pass a zeroed workspace")
                workspace = torch.zeros(need.value, dtype=torch.uint8, device=self.device)
                torch.cuda.current_stream().synchronize()           # (zeros now, for calls on whatever stream)
        self.workspace = workspace
        _expect("workspace", self.workspace, self._index, torch.uint8, (int(self.workspace.numel()),))
        self._pool = (self.num_pool_pages, shape.page_size, shape.num_kv_heads, d)
        self._pool4 = pool4_shape(shape, self.num_pool_pages)
        self._q, self._lse = (self.batch, shape.num_q_heads, d), (self.batch, shape.num_q_heads)

    def _pools(self, k_pool, v_pool, dtype, shape, stream):
        """Checks the pools and the current device; returns the stream's handle."""
        if self._current() != self._index:
            raise ValueError("the current device is not %s" % self.device)
        _expect("k_pool", k_pool, self._index, dtype, shape)
        _expect("v_pool", v_pool, self._index, dtype, shape)
        return self._raw_stream(self._index) if stream is None else _stream(stream)

    def _write(self, call, k_pool, v_pool, q, q_out, k_new, v_new, q_weight, k_weight, eps, stream) -> None:
        rows = _fresh_rows(self.shape, self.batch, self._index, self._bf16, q, q_out, k_new, v_new, q_weight, k_weight, eps)
        _check(call(*self._args, k_pool.data_ptr(), v_pool.data_ptr(), ctypes.addressof(rows), stream))

    def write(self, k_pool, v_pool, q, q_out, k_new, v_new, q_weight=None, k_weight=None, eps: float = 1e-6, stream=None) -> None:
        """The new tokens' un-rotated rows: q (normalised with q_weight, rotated) to q_out, k (likewise) and v to their slots.  q, k_new and v_new
        may be slices [batch, heads, D] of a fused projection; q None: keys and values alone."""
        st = self._pools(k_pool, v_pool, self._bf16, self._pool, stream)
        self._write(_lib.tessera_decode_write, k_pool, v_pool, q, q_out, k_new, v_new, q_weight, k_weight, eps, st)

    def write_kv4(self, k_pool4, v_pool4, q, q_out, k_new, v_new, q_weight=None, k_weight=None, eps: float = 1e-6, stream=None) -> None:
        """write() into 4-bit pools (pool4_shape)."""
        st = self._pools(k_pool4, v_pool4, self._u8, self._pool4, stream)
        self._write(_lib.tessera_decode_write_kv4, k_pool4, v_pool4, q, q_out, k_new, v_new, q_weight, k_weight, eps, st)

    def _attn(self, call, k_pool, v_pool, q, out, lse, stream) -> None:
        _expect("q", q, self._index, self._bf16, self._q)
        _expect("out", out, self._index, self._bf16, self._q)
        if lse is not None:
            _expect("lse", lse, self._index, self._f32, self._lse)
        _check(call(*self._args, k_pool.data_ptr(), v_pool.data_ptr(), q.data_ptr(), out.data_ptr(), _dev(lse), self.workspace.data_ptr(),
                    self.workspace.numel(), stream))

    def attn(self, k_pool, v_pool, q, out, lse=None, stream=None) -> None:
        """Attention of the rotated q [batch, H_q, D] over the requests' 16-bit pages."""
        st = self._pools(k_pool, v_pool, self._bf16, self._pool, stream)
        self._attn(_lib.tessera_decode_attn, k_pool, v_pool, q, out, lse, st)

    def attn_kv4(self, k_pool4, v_pool4, q, out, lse=None, stream=None) -> None:
        """Attention of the rotated q [batch, H_q, D] over the requests' 4-bit pages (pool4_shape)."""
        st = self._pools(k_pool4, v_pool4, self._u8, self._pool4, stream)
        self._attn(_lib.tessera_decode_attn_kv4, k_pool4, v_pool4, q, out, lse, st)


def selftest_bounded_wait(max_cycles: int, stream=None):
    """tessera_selftest_bounded_wait: returns (status, code, [cycles first wait, cycles second wait, success mask])."""
    code = ctypes.c_int32(0)
    cyc = (ctypes.c_int64 * 3)()
    st = _lib.tessera_selftest_bounded_wait(int(max_cycles), ctypes.byref(code), cyc, _stream(stream))
    return int(st), int(code.value), [int(x) for x in cyc]


STATIC_MAX_SHIFTS = 512


def rope_shift_static(shape, k_pool, slots, slot_shift, shifts, stream=None, inv_freq=None,
                      num_pool_slots: Optional[int] = None) -> None:
    """tessera_rope_shift_static: rotate the listed pool slots in place without any device
    allocation.  `slots` / `slot_shift` are int32 device tensors, `shifts` a host int32 sequence;
    `num_pool_slots` (default: every row of k_pool) bounds the slot ids the kernel accepts."""
    inv = _frequencies(shape, inv_freq)
    cfg = _model_cfg(shape, inv)
    sh = _arr(shifts)
    if num_pool_slots is None:
        num_pool_slots = int(k_pool.shape[0]) * int(k_pool.shape[1])
    _check(_lib.tessera_rope_shift_static(ctypes.byref(cfg), _dev(k_pool), int(num_pool_slots), _dev(slots),
                                          _dev(slot_shift), int(slots.numel()), _ptr(sh), len(sh), _stream(stream)))


def plan_create_status(w, host_only: bool = True) -> int:
    """Status code of tessera_plan_create for `w` (the plan, if any, is destroyed at once)."""
    try:
        Plan(w, host_only=host_only).destroy()
        return OK
    except TesseraError as e:
        return e.status

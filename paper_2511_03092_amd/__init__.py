"""SnapStream hot path on MI355X: Python binding of libsnapstream.so.

Argument marshalling only.  Every step of compression and decoding runs in the
HIP kernels of ``libsnapstream.so`` (built in-tree by ``build.py``); torch is
used for device memory and the current stream.  If the library is missing the
first call raises -- there is no other implementation behind these names.

Functions keep the C names (include/snapstream.h):
    snap_compress, snap_prefill, snap_prefill_attn, snap_cache_append, snap_decode_attn, snap_decode_step,
    snap_decode_step_noalloc, snap_advance, snap_debug_checks,
    snap_rope, snap_paged_append, snap_paged_decode_attn, snap_paged_decode_step, snap_paged_evict,
    snap_paged_decode_workspace, snap_paged_evict_workspace, snap_compress_workspace, snap_prefill_workspace, snap_decode_workspace, snap_status_str
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsnapstream.so")
# the same library built with the device-side invariant checks (build.py --debug)
DEBUG_LIB_PATH = os.path.join(_HERE, "libsnapstream_debug.so")

SNAP_OK, SNAP_ERR_INVALID_ARG, SNAP_ERR_UNSUPPORTED, SNAP_ERR_WORKSPACE, SNAP_ERR_HIP = range(5)
SNAP_F32, SNAP_BF16, SNAP_FP8_E4M3 = 0, 1, 2
SNAP_POOL_MAX, SNAP_POOL_AVG = 0, 1
SNAP_NORM_CAND, SNAP_NORM_ROW = 0, 1
SNAP_FP8_SCALES_GIVEN, SNAP_FP8_SCALES_AMAX = 0, 1
SNAP_KV_AUTO, SNAP_KV_STREAM, SNAP_KV_KEEP = 0, 1, 2
SNAP_ROPE_HALVES, SNAP_ROPE_PAIRS = 0, 1
SNAP_ROPE_PLAIN, SNAP_ROPE_DIVIDE, SNAP_ROPE_BY_TURNS, SNAP_ROPE_BY_INDEX = 0, 1, 2, 3

EXPORTED = ["snap_compress_workspace", "snap_decode_workspace", "snap_prefill_workspace", "snap_compress",
            "snap_prefill", "snap_prefill_attn", "snap_cache_append",
            "snap_decode_attn", "snap_decode_step", "snap_decode_step_noalloc", "snap_advance", "snap_debug_checks",
            "snap_rope", "snap_paged_append", "snap_paged_decode_workspace", "snap_paged_decode_attn",
            "snap_paged_decode_step", "snap_paged_evict_workspace", "snap_paged_evict",
            "snap_status_str", "snap_last_error"]


class SnapParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "n_q_heads", "n_kv_heads", "d_qk", "d_v", "v_in_k", "sink", "recent", "topk",
        "obs_window", "pool_kernel", "pool", "norm", "in_dtype", "kv_dtype")] + [("sm_scale", ctypes.c_float),
                                                                                  ("fp8_scales", ctypes.c_int32),
                                                                                  ("fp8_qk", ctypes.c_int32),
                                                                                  ("kv_reuse", ctypes.c_int32)]


class SnapCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("n_slots", ctypes.c_int32)]


class SnapRopeParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("rot_start", "rot_dim", "layout", "rule")] + [
        (n, ctypes.c_float) for n in ("base", "factor", "low_turns", "high_turns")] + [
        ("orig_len", ctypes.c_int32), ("amplitude", ctypes.c_float)]


class SnapRopeHeads(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("y", ctypes.c_void_p), ("x_stride", ctypes.c_int64 * 3),
                ("y_stride", ctypes.c_int64 * 3), ("n_heads", ctypes.c_int32)]


class SnapPagedCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("token", ctypes.c_void_p), ("weight", ctypes.c_void_p),
                ("page_table", ctypes.c_void_p), ("n_slots", ctypes.c_int32), ("n_pages", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("max_pages", ctypes.c_int32)]


class SnapError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"snapstream: {msg} (status {status})")
        self.status = status


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded HIP library; raises if it has not been built."""
    global _lib
    if _lib is None:
        _lib = load(LIB_PATH)
    return _lib


def use_library(path: str) -> ctypes.CDLL:
    """Route every call of this module to the library at `path` (the release
    or the debug build); returns the library that was in use."""
    global _lib
    prev = lib()
    _lib = load(path)
    return prev


def load(path: str) -> ctypes.CDLL:
    """Load one build of the library and declare its entry points."""
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with `python -m paper_2511_03092_amd.build` "
                          "(there is no fallback implementation)")
    # torch first: its HIP runtime is then the process's libamdhip64.so.7, and
    # the library binds to that same runtime (the one that owns the device
    # memory passed in).  Loaded before torch, the library would bring in the
    # system's runtime beside torch's, and its launches would not see torch's
    # device state.
    import torch  # noqa: F401
    L = ctypes.CDLL(path)
    P, vp, i32, sz = ctypes.POINTER(SnapParams), ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    C = ctypes.POINTER(SnapCache)
    L.snap_compress_workspace.argtypes = [P, i32, i32]
    L.snap_compress_workspace.restype = sz
    L.snap_decode_workspace.argtypes = [P, i32]
    L.snap_decode_workspace.restype = sz
    L.snap_compress.argtypes = [P, C, vp, vp, i32, vp, vp, i32, vp, vp, vp, vp, vp, vp, sz, vp]
    L.snap_compress.restype = ctypes.c_int
    L.snap_prefill_workspace.argtypes = [P, i32, i32]
    L.snap_prefill_workspace.restype = sz
    L.snap_prefill.argtypes = [P, C, vp, vp, i32, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.snap_prefill.restype = ctypes.c_int
    L.snap_prefill_attn.argtypes = [P, i32, vp, i32, vp, vp, vp, vp, vp, sz, vp]
    L.snap_prefill_attn.restype = ctypes.c_int
    L.snap_cache_append.argtypes = [P, C, vp, i32, vp, vp, vp, vp]
    L.snap_cache_append.restype = ctypes.c_int
    L.snap_decode_attn.argtypes = [P, C, vp, vp, i32, vp, vp, vp, i32, vp, sz, vp]
    L.snap_decode_attn.restype = ctypes.c_int
    L.snap_decode_step.argtypes = [P, C, vp, vp, i32, vp, vp, vp, vp, vp, i32, vp, sz, vp]
    L.snap_decode_step.restype = ctypes.c_int
    L.snap_decode_step_noalloc.argtypes = [P, C, vp, vp, i32, vp, vp, vp, vp, vp, i32, vp]
    L.snap_decode_step_noalloc.restype = ctypes.c_int
    L.snap_advance.argtypes = [vp, i32, i32, vp, vp]
    L.snap_advance.restype = ctypes.c_int
    L.snap_status_str.argtypes = [ctypes.c_int]
    L.snap_status_str.restype = ctypes.c_char_p
    L.snap_last_error.argtypes = []
    L.snap_last_error.restype = ctypes.c_char_p
    R, H, PC = ctypes.POINTER(SnapRopeParams), ctypes.POINTER(SnapRopeHeads), ctypes.POINTER(SnapPagedCache)
    L.snap_rope.argtypes = [R, i32, i32, i32, i32, vp, i32, vp, vp, H, H, vp]
    L.snap_rope.restype = ctypes.c_int
    L.snap_paged_append.argtypes = [P, PC, vp, vp, i32, vp, vp, i32, vp, vp, vp, vp, vp, vp]
    L.snap_paged_append.restype = ctypes.c_int
    L.snap_paged_decode_workspace.argtypes = [P, i32, i32, i32]
    L.snap_paged_decode_workspace.restype = sz
    L.snap_paged_decode_attn.argtypes = [P, PC, vp, i32, vp, i32, vp, vp, i32, i32, vp, sz, vp]
    L.snap_paged_decode_attn.restype = ctypes.c_int
    L.snap_paged_decode_step.argtypes = [P, PC, vp, vp, i32, vp, i32, vp, vp, vp, vp, i32, i32, vp, sz, vp]
    L.snap_paged_decode_step.restype = ctypes.c_int
    L.snap_paged_evict_workspace.argtypes = [P, i32, i32]
    L.snap_paged_evict_workspace.restype = sz
    L.snap_paged_evict.argtypes = [P, PC, vp, vp, vp, i32, vp, i32, vp, vp, sz, vp]
    L.snap_paged_evict.restype = ctypes.c_int
    L.snap_debug_checks.argtypes = [ctypes.POINTER(ctypes.c_uint32), i32]
    L.snap_debug_checks.restype = ctypes.c_int
    return L


@dataclass
class Params:
    """Hyper-parameters (snap_params); dtypes use the SNAP_* codes."""
    n_q_heads: int
    n_kv_heads: int
    d_qk: int
    d_v: int
    sink: int
    recent: int
    topk: int
    obs_window: int
    pool_kernel: int
    pool: int = SNAP_POOL_MAX
    norm: int = SNAP_NORM_CAND
    v_in_k: bool = False
    in_dtype: int = SNAP_BF16
    kv_dtype: int = SNAP_BF16
    sm_scale: float = 0.0
    fp8_scales: int = SNAP_FP8_SCALES_GIVEN
    fp8_qk: int = 0
    kv_reuse: int = SNAP_KV_AUTO

    @property
    def budget(self) -> int:
        return self.sink + self.recent + self.topk

    def c(self) -> SnapParams:
        return SnapParams(self.n_q_heads, self.n_kv_heads, self.d_qk, self.d_v, int(self.v_in_k), self.sink,
                          self.recent, self.topk, self.obs_window, self.pool_kernel, self.pool, self.norm,
                          self.in_dtype, self.kv_dtype, float(self.sm_scale), int(self.fp8_scales),
                          int(self.fp8_qk), int(self.kv_reuse))


def _ptr(t) -> int | None:
    return None if t is None else t.data_ptr()


def _stream(stream) -> int | None:
    if stream is not None:
        return stream
    import torch
    return torch.cuda.current_stream().cuda_stream


def _check(status: int):
    if status != SNAP_OK:
        L = lib()
        raise SnapError(status, (L.snap_last_error() or b"").decode() or L.snap_status_str(status).decode())


def cache_struct(k, v=None, k_scale=None, v_scale=None) -> SnapCache:
    return SnapCache(_ptr(k), _ptr(v), _ptr(k_scale), _ptr(v_scale), int(k.shape[0]))


def snap_status_str(status: int) -> str:
    return lib().snap_status_str(status).decode()


def snap_compress_workspace(p: Params, n_seq: int, max_len: int) -> int:
    return int(lib().snap_compress_workspace(ctypes.byref(p.c()), n_seq, max_len))


def snap_decode_workspace(p: Params, n: int) -> int:
    return int(lib().snap_decode_workspace(ctypes.byref(p.c()), n))


def snap_compress(p: Params, cache: SnapCache, pos, n_topk, slot_ids, lengths, q_obs, k, v, workspace,
                  sel_out=None, pooled_out=None, stream=None):
    n_seq, max_len = int(k.shape[0]), int(k.shape[2])
    _check(lib().snap_compress(ctypes.byref(p.c()), ctypes.byref(cache), _ptr(pos), _ptr(n_topk), n_seq,
                               _ptr(slot_ids), _ptr(lengths), max_len, _ptr(q_obs), _ptr(k), _ptr(v),
                               _ptr(sel_out), _ptr(pooled_out), _ptr(workspace),
                               workspace.numel() * workspace.element_size(), _stream(stream)))


def snap_prefill_workspace(p: Params, n_seq: int, max_len: int) -> int:
    return int(lib().snap_prefill_workspace(ctypes.byref(p.c()), n_seq, max_len))


def snap_prefill(p: Params, cache: SnapCache, pos, n_topk, slot_ids, lengths, q, k, v, out, workspace,
                 sel_out=None, pooled_out=None, stream=None):
    n_seq, max_len = int(k.shape[0]), int(k.shape[2])
    _check(lib().snap_prefill(ctypes.byref(p.c()), ctypes.byref(cache), _ptr(pos), _ptr(n_topk), n_seq,
                              _ptr(slot_ids), _ptr(lengths), max_len, _ptr(q), _ptr(k), _ptr(v), _ptr(out),
                              _ptr(sel_out), _ptr(pooled_out), _ptr(workspace),
                              workspace.numel() * workspace.element_size(), _stream(stream)))


def snap_prefill_attn(p: Params, lengths, q, k, v, out, workspace, stream=None):
    n_seq, max_len = int(k.shape[0]), int(k.shape[2])
    _check(lib().snap_prefill_attn(ctypes.byref(p.c()), n_seq, _ptr(lengths), max_len, _ptr(q), _ptr(k), _ptr(v),
                                   _ptr(out), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                   _stream(stream)))


def snap_cache_append(p: Params, cache: SnapCache, pos, slot_ids, k_new, v_new=None, stream=None):
    _check(lib().snap_cache_append(ctypes.byref(p.c()), ctypes.byref(cache), _ptr(pos), int(k_new.shape[0]),
                                   _ptr(slot_ids), _ptr(k_new), _ptr(v_new), _stream(stream)))


def snap_decode_attn(p: Params, cache: SnapCache, pos, n_topk, slot_ids, q, out, workspace, stream=None):
    import torch
    out_dtype = SNAP_BF16 if out.dtype == torch.bfloat16 else SNAP_F32
    _check(lib().snap_decode_attn(ctypes.byref(p.c()), ctypes.byref(cache), _ptr(pos), _ptr(n_topk),
                                  int(q.shape[0]), _ptr(slot_ids), _ptr(q), _ptr(out), out_dtype,
                                  _ptr(workspace), workspace.numel() * workspace.element_size(),
                                  _stream(stream)))


def snap_decode_step(p: Params, cache: SnapCache, pos, n_topk, slot_ids, q, k_new, v_new, out, workspace,
                     stream=None):
    import torch
    out_dtype = SNAP_BF16 if out.dtype == torch.bfloat16 else SNAP_F32
    _check(lib().snap_decode_step(ctypes.byref(p.c()), ctypes.byref(cache), _ptr(pos), _ptr(n_topk),
                                  int(q.shape[0]), _ptr(slot_ids), _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(out),
                                  out_dtype, _ptr(workspace), workspace.numel() * workspace.element_size(),
                                  _stream(stream)))


def snap_decode_step_noalloc(p: Params, cache: SnapCache, pos, n_topk, slot_ids, q, k_new, v_new, out, stream=None):
    import torch
    out_dtype = SNAP_BF16 if out.dtype == torch.bfloat16 else SNAP_F32
    _check(lib().snap_decode_step_noalloc(ctypes.byref(p.c()), ctypes.byref(cache), _ptr(pos), _ptr(n_topk),
                                          int(q.shape[0]), _ptr(slot_ids), _ptr(q), _ptr(k_new), _ptr(v_new),
                                          _ptr(out), out_dtype, _stream(stream)))


def snap_advance(pos, slot_ids, stream=None):
    _check(lib().snap_advance(_ptr(pos), int(pos.shape[0]), int(slot_ids.shape[0]), _ptr(slot_ids),
                              _stream(stream)))


@dataclass(frozen=True)
class RopeParams:
    """Rotary positions (snap_rope_params)."""
    rot_start: int
    rot_dim: int
    layout: int = SNAP_ROPE_HALVES
    rule: int = SNAP_ROPE_PLAIN
    base: float = 10000.0
    factor: float = 1.0
    low_turns: float = 1.0
    high_turns: float = 32.0
    orig_len: int = 0
    amplitude: float = 1.0

    def __post_init__(self):  # frozen: the structure is built once
        object.__setattr__(self, "_struct", SnapRopeParams(
            self.rot_start, self.rot_dim, self.layout, self.rule, self.base, self.factor, self.low_turns,
            self.high_turns, self.orig_len, self.amplitude))

    def c(self) -> SnapRopeParams:
        return self._struct


def _bad(msg: str):
    raise SnapError(SNAP_ERR_INVALID_ARG, msg)


def _want(t, name: str, dtype, shape: tuple, index: int):
    """t is a contiguous tensor of this type, shape and device index (the library sees only its address)."""
    if t is None:
        _bad(f"{name} is None")
    if t.dtype is not dtype or t.shape != shape or t.get_device() != index or not t.is_contiguous():
        _bad(f"{name} must be a contiguous {dtype} {tuple(shape)} tensor on device {index} (got {t.dtype} "
             f"{tuple(t.shape)}, strides {t.stride()}, on {t.device})")


def _launch(index: int, stream, fn, *args):
    """One library call on the tensors' device (a launch goes to the current one) and its current stream."""
    import torch
    if index < 0:
        _bad("tensors must be on the GPU")
    if stream is None:
        stream = torch._C._cuda_getCurrentRawStream(index)
    if torch.cuda.current_device() == index:
        status = fn(*args, stream)
    else:
        with torch.cuda.device(index):
            status = fn(*args, stream)
    if status:
        _check(status)


_i64x3 = ctypes.c_int64 * 3


def _rope_heads(x, y, name: str):
    if y is None:
        y = x
    xs, ys = x.stride(), y.stride()
    if len(xs) != 4 or y.shape != x.shape or y.dtype is not x.dtype or y.get_device() != x.get_device():
        _bad(f"{name} and its output must be [n, heads, tokens, d] of one shape, type and device "
             f"(got {tuple(x.shape)} {x.dtype} on {x.device}, {tuple(y.shape)} {y.dtype} on {y.device})")
    if xs[3] != 1 or ys[3] != 1:
        _bad(f"{name}: the last dimension must be contiguous")
    return SnapRopeHeads(x.data_ptr(), y.data_ptr(), _i64x3(*xs[:3]), _i64x3(*ys[:3]), x.shape[1])


def snap_rope(r: RopeParams, q, k=None, q_out=None, k_out=None, pos=None, slot_ids=None, lengths=None, stream=None):
    """Rotates q [n, heads, tokens, d] and k (any strides but the last) into q_out / k_out, or in place."""
    import torch
    if q is None:
        _bad("q is None")
    dtype, index = q.dtype, q.get_device()
    if dtype is not torch.bfloat16 and dtype is not torch.float32:
        _bad(f"q must be bfloat16 or float32 (got {dtype})")
    hq, hk = _rope_heads(q, q_out, "q"), None
    n, _, tokens, d = q.shape
    if k is not None:
        hk = _rope_heads(k, k_out, "k")
        if k.shape[0] != n or k.shape[2] != tokens or k.shape[3] != d or k.dtype is not dtype or k.get_device() != index:
            _bad(f"q and k differ in more than their heads (got {tuple(q.shape)} {dtype}, {tuple(k.shape)} {k.dtype})")
    n_slots = 0
    if pos is None:
        slot_ids = None
    else:
        n_slots = pos.numel()
        _want(pos, "pos", torch.int32, (n_slots,), index)
        _want(slot_ids, "slot_ids", torch.int32, (n,), index)
    if lengths is not None:
        _want(lengths, "lengths", torch.int32, (n,), index)
    if n == 0 or tokens == 0:
        return
    _launch(index, stream, lib().snap_rope, ctypes.byref(r.c()), SNAP_BF16 if dtype is torch.bfloat16 else SNAP_F32, n,
            tokens, d, _ptr(pos), n_slots, _ptr(slot_ids), _ptr(lengths), ctypes.byref(hq),
            None if hk is None else ctypes.byref(hk))


def paged_cache_struct(k, v, page_table, token=None, weight=None, k_scale=None, v_scale=None) -> SnapPagedCache:
    """The handle of a paged cache: k [n_pages, n_kv_heads, page_size, d_qk], v likewise (None for a latent cache),
    page_table [n_slots, max_pages], token and weight [n_pages, n_kv_heads, page_size].  It holds the tensors."""
    import torch
    if k is None:
        _bad("k is None")
    if k.dim() != 4 or k.dtype not in (torch.float32, torch.bfloat16, torch.uint8):
        _bad(f"k must be [n_pages, n_kv_heads, page_size, d] float32, bfloat16 or uint8 (got {tuple(k.shape)} {k.dtype})")
    index, pages = k.get_device(), k.shape[:3]
    _want(k, "k", k.dtype, k.shape, index)
    if v is not None:
        if v.dim() != 4:
            _bad(f"v must be [n_pages, n_kv_heads, page_size, d_v] (got {tuple(v.shape)})")
        _want(v, "v", k.dtype, pages + v.shape[3:], index)
    if page_table is None or page_table.dim() != 2:
        _bad("page_table must be [n_slots, max_pages]")
    _want(page_table, "page_table", torch.int32, page_table.shape, index)
    slots = int(page_table.shape[0])
    for t, name, dtype, shape in ((token, "token", torch.int32, pages), (weight, "weight", torch.float32, pages),
                                  (k_scale, "k_scale", torch.float32, (slots, pages[1])),
                                  (v_scale, "v_scale", torch.float32, (slots, pages[1]))):
        if t is not None:
            _want(t, name, dtype, shape, index)
    c = SnapPagedCache(_ptr(k), _ptr(v), _ptr(k_scale), _ptr(v_scale), _ptr(token), _ptr(weight), _ptr(page_table), slots,
                       int(k.shape[0]), int(k.shape[2]), int(page_table.shape[1]))
    c.tensors = (k, v, page_table, token, weight, k_scale, v_scale)
    c.index, c.slots_shape, c.i32 = index, (slots,), torch.int32
    c.in_dtype = torch.float32 if k.dtype is torch.float32 else torch.bfloat16
    c.kind = ({torch.float32: SNAP_F32, torch.bfloat16: SNAP_BF16, torch.uint8: SNAP_FP8_E4M3}[k.dtype], int(k.shape[1]),
              int(k.shape[3]), None if v is None else int(v.shape[3]))
    c.rows_max, c.params = c.max_pages * c.page_size, (None, None)
    return c


def _paged(p: Params, cache: SnapPagedCache, rows, pos, slot_ids):
    """Checks what every paged call shares; the number of sequences and the parameters' structure."""
    if cache is None or slot_ids is None:
        _bad("cache or slot_ids is None")
    values, params = tuple(vars(p).values()), cache.params
    if params[0] != values:  # (the same parameters as the last call's: the same structure)
        kind = (p.kv_dtype, p.n_kv_heads, p.d_qk, None if p.v_in_k else p.d_v)
        if cache.kind != kind:
            _bad(f"the cache (type, heads, widths {cache.kind}) is not that of the parameters ({kind})")
        cache.params = params = (values, p.c())
    n, index = slot_ids.shape[0], cache.index
    _want(slot_ids, "slot_ids", cache.i32, (n,), index)
    _want(rows, "rows", cache.i32, cache.slots_shape, index)
    if pos is not None:
        _want(pos, "pos", cache.i32, cache.slots_shape, index)
    return n, ctypes.byref(params[1])


def _strides(t, name: str, dtype, shape: tuple, index: int):
    st = t.stride()
    if t.dtype is not dtype or t.shape != shape or t.get_device() != index or st[3] != 1:
        _bad(f"{name} must be a {dtype} {tuple(shape)} tensor on device {index} whose rows are contiguous (got {t.dtype} "
             f"{tuple(t.shape)}, strides {st}, on {t.device})")
    return _i64x3(*st[:3])


def snap_paged_append(p: Params, cache: SnapPagedCache, rows, pos, slot_ids, k_new, v_new=None, lengths=None,
                      weight_new=None, stream=None):
    """Stores k_new [n, n_kv_heads, tokens, d_qk] and v_new (any strides but the last) behind the rows held."""
    import torch
    (n, cp), index, heads = _paged(p, cache, rows, pos, slot_ids), cache.index, p.n_kv_heads
    if k_new is None or k_new.dim() != 4 or (v_new is None) != bool(p.v_in_k):
        _bad("k_new must be [n, n_kv_heads, tokens, d_qk], with v_new unless the values are in the keys")
    tokens = k_new.shape[2]
    ks = _strides(k_new, "k_new", cache.in_dtype, (n, heads, tokens, p.d_qk), index)
    vs = None if v_new is None else _strides(v_new, "v_new", cache.in_dtype, (n, heads, tokens, p.d_v), index)
    if lengths is not None:
        _want(lengths, "lengths", cache.i32, (n,), index)
    if weight_new is not None:
        _want(weight_new, "weight_new", torch.float32, (n, heads, tokens), index)
    if n == 0 or tokens == 0:
        return
    _launch(index, stream, lib().snap_paged_append, cp, ctypes.byref(cache), _ptr(rows), _ptr(pos), n, _ptr(slot_ids),
            _ptr(lengths), tokens, _ptr(k_new), ks, _ptr(v_new), vs, _ptr(weight_new))


def snap_paged_decode_workspace(p: Params, n: int, max_rows: int, weigh: bool = False) -> int:
    return int(lib().snap_paged_decode_workspace(ctypes.byref(p.c()), n, max_rows, int(weigh)))


def snap_paged_evict_workspace(p: Params, n: int, max_rows: int) -> int:
    return int(lib().snap_paged_evict_workspace(ctypes.byref(p.c()), n, max_rows))


def _bytes(workspace, index: int) -> int:
    if workspace is None:
        return 0
    if workspace.get_device() != index or not workspace.is_contiguous():
        _bad(f"workspace must be contiguous on device {index} (got {workspace.device})")
    return workspace.numel() * workspace.element_size()


def _paged_io(p: Params, cache: SnapPagedCache, n: int, q, out) -> int:
    """Checks queries and output; the output's type code."""
    import torch
    _want(q, "q", cache.in_dtype, (n, p.n_q_heads, p.d_qk), cache.index)
    if out is None:
        _bad("out is None")
    bf16 = out.dtype is torch.bfloat16
    _want(out, "out", torch.bfloat16 if bf16 else torch.float32, (n, p.n_q_heads, p.d_v), cache.index)
    return SNAP_BF16 if bf16 else SNAP_F32


def snap_paged_decode_attn(p: Params, cache: SnapPagedCache, rows, slot_ids, q, out, workspace, max_rows=None,
                           weigh: bool = False, stream=None):
    """Attention of one new token per sequence (stored already); max_rows bounds their rows (default: the table's)."""
    (n, cp), index = _paged(p, cache, rows, None, slot_ids), cache.index
    od = _paged_io(p, cache, n, q, out)
    _launch(index, stream, lib().snap_paged_decode_attn, cp, ctypes.byref(cache), _ptr(rows), n, _ptr(slot_ids),
            cache.rows_max if max_rows is None else max_rows, _ptr(q), _ptr(out), od, int(weigh), _ptr(workspace),
            _bytes(workspace, index))


def snap_paged_decode_step(p: Params, cache: SnapPagedCache, rows, pos, slot_ids, q, k_new, v_new, out, workspace,
                           max_rows=None, weigh: bool = False, stream=None):
    """Stores one token per sequence (k_new [n, n_kv_heads, 1, d_qk], or without the 1) and attends it."""
    (n, cp), index = _paged(p, cache, rows, pos, slot_ids), cache.index
    od = _paged_io(p, cache, n, q, out)
    if (v_new is None) != bool(p.v_in_k):
        _bad("v_new must be given unless the values are in the keys")
    heads = (n, p.n_kv_heads) if k_new is not None and k_new.dim() == 3 else (n, p.n_kv_heads, 1)
    _want(k_new, "k_new", cache.in_dtype, heads + (p.d_qk,), index)
    if v_new is not None:
        _want(v_new, "v_new", cache.in_dtype, heads + (p.d_v,), index)
    _launch(index, stream, lib().snap_paged_decode_step, cp, ctypes.byref(cache), _ptr(rows), _ptr(pos), n, _ptr(slot_ids),
            cache.rows_max if max_rows is None else max_rows, _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(out), od, int(weigh),
            _ptr(workspace), _bytes(workspace, index))


def snap_paged_evict(p: Params, cache: SnapPagedCache, rows, pos, slot_ids, rows_out, workspace, max_rows=None,
                     kept_out=None, stream=None):
    """Cuts slots back to the budget; rows_out [n_slots] gets the rows they then hold."""
    if pos is None:
        _bad("pos is None")
    (n, cp), index = _paged(p, cache, rows, pos, slot_ids), cache.index
    _want(rows_out, "rows_out", cache.i32, cache.slots_shape, index)
    if kept_out is not None:
        _want(kept_out, "kept_out", cache.i32, (n, p.n_kv_heads, p.budget), index)
    _launch(index, stream, lib().snap_paged_evict, cp, ctypes.byref(cache), _ptr(rows), _ptr(pos), _ptr(rows_out), n,
            _ptr(slot_ids), cache.rows_max if max_rows is None else max_rows, _ptr(kept_out), _ptr(workspace),
            _bytes(workspace, index))


def snap_debug_checks(reset: bool = True) -> int:
    """The invariant bits the debug build's kernels recorded (waits for the
    device); raises SnapError on a release build."""
    flags = ctypes.c_uint32(0)
    _check(lib().snap_debug_checks(ctypes.byref(flags), int(reset)))
    return int(flags.value)


def workspace(nbytes: int, device="cuda"):
    """A 256-byte aligned device buffer (torch's allocator aligns to 512)."""
    import torch
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)

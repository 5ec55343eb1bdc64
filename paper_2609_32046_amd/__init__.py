"""MI355X receiver-conditioned KV selection: Python binding of ``libcacheback.so``.

Argument marshalling only.  Every step of the path runs in the HIP kernels
behind the C ABI declared in ``include/cacheback.h`` and
``include/cacheback_cache.h``; this module converts
torch tensors (or raw integer device pointers) to pointers, passes the current
HIP stream, and turns status codes into exceptions.  torch is used for device
memory and streams only.

There is no CPU fallback: importing this package raises if the HIP library
has not been built (``python paper_2609_32046_amd/build.py``).
"""
from __future__ import annotations

import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcacheback.so")

CB_F32, CB_BF16 = 0, 1
STATUS = {0: "CB_OK", -1: "CB_ERR_NULL", -2: "CB_ERR_SHAPE", -3: "CB_ERR_DTYPE",
          -4: "CB_ERR_RATIO", -5: "CB_ERR_WORKSPACE", -6: "CB_ERR_ALIGN", -7: "CB_ERR_HIP",
          -8: "CB_ERR_TIMEOUT", -9: "CB_ERR_PAGES"}

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build the HIP library first "
        "(python paper_2609_32046_amd/build.py).  There is no CPU fallback.")

_lib = ctypes.CDLL(LIB_PATH)


class cb_layout(ctypes.Structure):
    _fields_ = [("layers", ctypes.c_int32), ("q_heads", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("q_len", ctypes.c_int32), ("senders", ctypes.c_int32),
                ("seq_len", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("scale", ctypes.c_float)]


_vp, _i64, _sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t
_lib.cb_score_workspace_bytes.argtypes = [ctypes.POINTER(cb_layout)]
_lib.cb_score_workspace_bytes.restype = _sz
_lib.cb_score.argtypes = [_vp, _vp, ctypes.POINTER(cb_layout), _vp, _vp, _vp, _sz, _vp]
_lib.cb_score.restype = ctypes.c_int
_lib.cb_keep_count.argtypes = [_i64, ctypes.c_double]
_lib.cb_keep_count.restype = _i64
_lib.cb_select.argtypes = [_vp, _i64, _i64, ctypes.c_double, _vp, ctypes.POINTER(_i64), _vp]
_lib.cb_select.restype = ctypes.c_int
_lib.cb_select_workspace_bytes.argtypes = [_i64, _i64]
_lib.cb_select_workspace_bytes.restype = _sz
_lib.cb_select_ws.argtypes = [_vp, _i64, _i64, ctypes.c_double, _vp, ctypes.POINTER(_i64), _vp,
                              _sz, _vp]
_lib.cb_select_ws.restype = ctypes.c_int
_lib.cb_select_status.argtypes = [_i64, _i64, _vp, _sz, _vp]
_lib.cb_select_status.restype = ctypes.c_int
_lib.cb_compact.argtypes = [_vp, _vp, _vp, ctypes.POINTER(cb_layout), _i64, _vp, _vp, _vp]
_lib.cb_compact.restype = ctypes.c_int
_lib.cb_pipeline.argtypes = [_vp, _vp, _vp, ctypes.POINTER(cb_layout), ctypes.c_double, _vp, _vp,
                             _vp, _vp, _vp, _vp, _sz, ctypes.POINTER(_i64), _vp]
_lib.cb_pipeline.restype = ctypes.c_int
_lib.cb_pipeline_noalloc.argtypes = [_vp, _vp, _vp, ctypes.POINTER(cb_layout), ctypes.c_double,
                                     _vp, _vp, _vp, _vp, _vp, ctypes.POINTER(_i64), _vp]
_lib.cb_pipeline_noalloc.restype = ctypes.c_int
_lib.cb_score_status.argtypes = [ctypes.POINTER(cb_layout), _vp, _sz, _vp]
_lib.cb_score_status.restype = ctypes.c_int
_lib.cb_set_wait_limit.argtypes = [ctypes.c_uint32]
_lib.cb_set_wait_limit.restype = ctypes.c_uint32
_lib.cb_position_workspace_bytes.argtypes = [ctypes.POINTER(cb_layout)]
_lib.cb_position_workspace_bytes.restype = _sz
_lib.cb_position_score.argtypes = [_vp, _vp, ctypes.POINTER(cb_layout), ctypes.c_double,
                                   ctypes.c_double, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.cb_position_score.restype = ctypes.c_int
_lib.cb_position_status.argtypes = [ctypes.POINTER(cb_layout), _vp, _sz, _vp]
_lib.cb_position_status.restype = ctypes.c_int
_lib.cb_budget_fanout.argtypes = [_i64, _i64]
_lib.cb_budget_fanout.restype = _i64
_lib.cb_budget_chain.argtypes = [_i64, _i64, _i64, ctypes.c_int, _i64]
_lib.cb_budget_chain.restype = _i64
_lib.cb_spans_workspace_bytes.argtypes = [_i64, _i64, ctypes.c_int32]
_lib.cb_spans_workspace_bytes.restype = _sz
_lib.cb_select_spans.argtypes = [_vp, _i64, _i64, _i64, _i64, ctypes.c_int32, _vp,
                                 ctypes.POINTER(_i64), _vp, _sz, _vp]
_lib.cb_select_spans.restype = ctypes.c_int
_lib.cb_gather_rows.argtypes = [_vp, _i64, _i64, _i64, _vp, _i64, _vp, _vp]
_lib.cb_gather_rows.restype = ctypes.c_int


class _rope(ctypes.Structure):
    _fields_ = [("rotary_dim", ctypes.c_int32), ("scaling", ctypes.c_int32),
                ("base", ctypes.c_double), ("factor", ctypes.c_double),
                ("original_len", ctypes.c_double), ("fast_turns", ctypes.c_double),
                ("slow_turns", ctypes.c_double)]


class cb_rows(ctypes.Structure):
    dev = None   # device of its tensors, where rows() made it
    _fields_ = [("x", _vp), ("out", _vp), ("pos", _vp), ("frm", _vp), ("size", _i64 * 3),
                ("in_stride", _i64 * 3), ("out_stride", _i64 * 3), ("pos_stride", _i64 * 3),
                ("from_stride", _i64 * 3)]


class cb_cache(ctypes.Structure):
    dev = None   # device of its tensors, where cache() made it
    _fields_ = [("layers", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("page_len", ctypes.c_int32),
                ("pages", ctypes.c_int32), ("seqs", ctypes.c_int32), ("width", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("pool", _vp), ("refs", _vp), ("table", _vp),
                ("lens", _vp)]


_i32, _pc = ctypes.c_int32, ctypes.POINTER(cb_cache)
for _name, _args, _res in [
        ("cb_rotary_frequencies", [ctypes.POINTER(_rope), _vp, ctypes.POINTER(ctypes.c_double)], ctypes.c_int),
        ("cb_rotary", [ctypes.POINTER(cb_rows), _i32, _i32, _vp, _i32, ctypes.c_double, _i32, _i32, _i32, _vp],
         ctypes.c_int),
        ("cb_cache_page_bytes", [_pc], _sz),
        ("cb_cache_status", [_vp, _vp], ctypes.c_int),
        ("cb_cache_extend", [_pc, _vp, _vp, _i32, _vp, _vp], ctypes.c_int),
        ("cb_cache_free", [_pc, _vp, _i32, _vp], ctypes.c_int),
        ("cb_cache_fork_workspace_bytes", [_pc, _i32], _sz),
        ("cb_cache_fork", [_pc, _vp, _vp, _i32, _i32, _vp, _vp, _sz, _vp], ctypes.c_int),
        ("cb_cache_compact_workspace_bytes", [_pc, _i32], _sz),
        ("cb_cache_compact", [_pc, _vp, _vp, _i32, _vp, ctypes.POINTER(_i64), _i64, _vp, _vp, _vp, _sz, _vp],
         ctypes.c_int),
        ("cb_cache_write", [_pc, _i32, _i32, _vp, _i32, _vp, _vp, _i64, _vp, _vp,
                            ctypes.POINTER(_i64), _i32, _vp], ctypes.c_int),
        ("cb_cache_read", [_pc, _i32, _i32, _vp, _i32, _vp, _vp, _i64, _vp, _vp,
                           ctypes.POINTER(_i64), _i32, _vp], ctypes.c_int),
        ("cb_cache_attend_workspace_bytes", [_pc, _i32, _i32, _i32, _i64, _i64], _sz),
        ("cb_cache_attend", [_pc, _i32, _i32, _vp, _i32, _vp, ctypes.POINTER(_i64), _i32, _vp, _i64,
                             _i32, _i64, ctypes.c_double, _vp, ctypes.POINTER(_i64), _vp, _i32, _vp, _sz,
                             _vp], ctypes.c_int)]:
    getattr(_lib, _name).argtypes = _args
    getattr(_lib, _name).restype = _res
_lib.cb_status_string.argtypes = [ctypes.c_int]
_lib.cb_status_string.restype = ctypes.c_char_p


class CBError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS.get(status, status)} "
                         f"({_lib.cb_status_string(status).decode()})")


def _check(status: int, where: str) -> int:
    if status < 0:
        raise CBError(status, where)
    return status


def _ptr(x):
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _stream(stream):
    if stream is None:
        import torch

        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def layout(layers, q_heads, kv_heads, head_dim, q_len, seq_len, senders=1, dtype=CB_BF16,
           scale=0.0) -> cb_layout:
    if isinstance(dtype, str):
        dtype = {"f32": CB_F32, "bf16": CB_BF16}[dtype]
    return cb_layout(layers, q_heads, kv_heads, head_dim, q_len, senders, seq_len, dtype, scale)


def layout_of(w, scale=0.0) -> cb_layout:
    """cb_layout for a workload description with the usual attribute names."""
    return layout(w.layers, w.q_heads, w.kv_heads, w.head_dim, w.q_len, w.seq_len,
                  w.senders, w.dtype, scale)


def cb_score_workspace_bytes(lay: cb_layout) -> int:
    n = _lib.cb_score_workspace_bytes(ctypes.byref(lay))
    if n == 0:
        raise CBError(-2, "cb_score_workspace_bytes")
    return n


def cb_score(q, k, lay: cb_layout, importance, row_lse=None, ws=None, ws_bytes=None,
             stream=None) -> None:
    if ws_bytes is None:
        ws_bytes = ws.numel() * ws.element_size() if ws is not None and not isinstance(ws, int) else 0
    _check(_lib.cb_score(_ptr(q), _ptr(k), ctypes.byref(lay), _ptr(importance), _ptr(row_lse),
                         _ptr(ws), ws_bytes, _stream(stream)), "cb_score")


def cb_keep_count(T: int, keep_ratio: float) -> int:
    return _check(int(_lib.cb_keep_count(int(T), float(keep_ratio))), "cb_keep_count")


def cb_select(importance, units: int, T: int, keep_ratio: float, idx, stream=None) -> int:
    keep = _i64(0)
    _check(_lib.cb_select(_ptr(importance), int(units), int(T), float(keep_ratio), _ptr(idx),
                          ctypes.byref(keep), _stream(stream)), "cb_select")
    return keep.value


def cb_select_workspace_bytes(units: int, T: int) -> int:
    """Scratch bytes of cb_select_ws for these rows (0: rows are not split)."""
    return _lib.cb_select_workspace_bytes(int(units), int(T))


def cb_select_ws(importance, units: int, T: int, keep_ratio: float, idx, ws, ws_bytes=None,
                 stream=None) -> int:
    keep = _i64(0)
    _check(_lib.cb_select_ws(_ptr(importance), int(units), int(T), float(keep_ratio), _ptr(idx),
                             ctypes.byref(keep), _ptr(ws), _nbytes(ws, ws_bytes),
                             _stream(stream)), "cb_select_ws")
    return keep.value


def cb_select_status(units: int, T: int, ws, ws_bytes=None, stream=None) -> int:
    """Synchronises the stream and returns 0 (CB_OK) or -8 (CB_ERR_TIMEOUT)
    for the last cb_select_ws call on ``ws``; argument errors raise."""
    st = _lib.cb_select_status(int(units), int(T), _ptr(ws), _nbytes(ws, ws_bytes),
                               _stream(stream))
    if st not in (0, -8):
        _check(st, "cb_select_status")
    return st


def cb_compact(k, v, idx, lay: cb_layout, keep: int, k_out, v_out, stream=None) -> None:
    _check(_lib.cb_compact(_ptr(k), _ptr(v), _ptr(idx), ctypes.byref(lay), int(keep),
                           _ptr(k_out), _ptr(v_out), _stream(stream)), "cb_compact")


def cb_pipeline(q, k, v, lay: cb_layout, keep_ratio: float, importance, idx, k_out, v_out,
                ws, row_lse=None, ws_bytes=None, stream=None) -> int:
    if ws_bytes is None:
        ws_bytes = ws.numel() * ws.element_size() if not isinstance(ws, int) else 0
    keep = _i64(0)
    _check(_lib.cb_pipeline(_ptr(q), _ptr(k), _ptr(v), ctypes.byref(lay), float(keep_ratio),
                            _ptr(importance), _ptr(row_lse), _ptr(idx), _ptr(k_out), _ptr(v_out),
                            _ptr(ws), ws_bytes, ctypes.byref(keep), _stream(stream)),
           "cb_pipeline")
    return keep.value


def cb_score_status(lay: cb_layout, ws, ws_bytes=None, stream=None) -> int:
    """Synchronises the stream and returns the status word of the last score
    call on ``ws``: 0 (CB_OK) or -8 (CB_ERR_TIMEOUT); argument errors raise."""
    if ws_bytes is None:
        ws_bytes = ws.numel() * ws.element_size() if not isinstance(ws, int) else 0
    st = _lib.cb_score_status(ctypes.byref(lay), _ptr(ws), ws_bytes, _stream(stream))
    if st not in (0, -8):
        _check(st, "cb_score_status")
    return st


def _nbytes(ws, ws_bytes):
    if ws_bytes is not None:
        return ws_bytes
    return ws.numel() * ws.element_size() if ws is not None and not isinstance(ws, int) else 0


def cb_position_workspace_bytes(lay: cb_layout) -> int:
    n = _lib.cb_position_workspace_bytes(ctypes.byref(lay))
    if n == 0:
        raise CBError(-2, "cb_position_workspace_bytes")
    return n


def cb_position_score(q, k, lay: cb_layout, score, ws, p=2.0, alpha=2.0, qscore=None, corr=None,
                      importance=None, ws_bytes=None, stream=None) -> None:
    _check(_lib.cb_position_score(_ptr(q), _ptr(k), ctypes.byref(lay), float(p), float(alpha),
                                  _ptr(score), _ptr(qscore), _ptr(corr), _ptr(importance),
                                  _ptr(ws), _nbytes(ws, ws_bytes), _stream(stream)),
           "cb_position_score")


def cb_position_status(lay: cb_layout, ws, ws_bytes=None, stream=None) -> int:
    st = _lib.cb_position_status(ctypes.byref(lay), _ptr(ws), _nbytes(ws, ws_bytes),
                                 _stream(stream))
    if st not in (0, -8):
        _check(st, "cb_position_status")
    return st


def cb_budget_fanout(T: int, r: int) -> int:
    return _check(int(_lib.cb_budget_fanout(int(T), int(r))), "cb_budget_fanout")


def cb_budget_chain(T_old: int, T_new: int, r: int, relative: bool, B_max: int = 0) -> int:
    return _check(int(_lib.cb_budget_chain(int(T_old), int(T_new), int(r), int(bool(relative)),
                                           int(B_max))), "cb_budget_chain")


def cb_spans_workspace_bytes(senders: int, T: int, width: int = 16) -> int:
    n = _lib.cb_spans_workspace_bytes(int(senders), int(T), int(width))
    if n == 0:
        raise CBError(-2, "cb_spans_workspace_bytes")
    return n


def cb_select_spans(score, senders: int, T: int, budget: int, idx, ws, n_latent: int = 40,
                    width: int = 16, ws_bytes=None, stream=None) -> int:
    count = _i64(0)
    _check(_lib.cb_select_spans(_ptr(score), int(senders), int(T), int(budget), int(n_latent),
                                int(width), _ptr(idx), ctypes.byref(count), _ptr(ws),
                                _nbytes(ws, ws_bytes), _stream(stream)), "cb_select_spans")
    return count.value


def cb_gather_rows(rows, senders: int, T: int, row_bytes: int, idx, count: int, out,
                   stream=None) -> None:
    _check(_lib.cb_gather_rows(_ptr(rows), int(senders), int(T), int(row_bytes), _ptr(idx),
                               int(count), _ptr(out), _stream(stream)), "cb_gather_rows")


def cb_set_wait_limit(polls: int) -> int:
    return int(_lib.cb_set_wait_limit(int(polls)))


def cb_pipeline_noalloc(q, k, v, lay: cb_layout, keep_ratio: float, importance, idx, k_out, v_out,
                        row_lse=None, stream=None) -> int:
    """cb_pipeline with the library's own per-device workspace (no ws)."""
    keep = _i64(0)
    _check(_lib.cb_pipeline_noalloc(_ptr(q), _ptr(k), _ptr(v), ctypes.byref(lay),
                                    float(keep_ratio), _ptr(importance), _ptr(row_lse), _ptr(idx),
                                    _ptr(k_out), _ptr(v_out), ctypes.byref(keep), _stream(stream)),
           "cb_pipeline_noalloc")
    return keep.value


def cb_status_string(status: int) -> str:
    return _lib.cb_status_string(int(status)).decode()


class Buffers:
    """Device buffers for one layout and keep ratio (torch allocations)."""

    def __init__(self, lay: cb_layout, keep_ratio: float, device="cuda"):
        import torch

        self.lay = lay
        S, L, Hkv, T = lay.senders, lay.layers, lay.kv_heads, lay.seq_len
        self.units = S * L * Hkv
        self.keep = cb_keep_count(T, keep_ratio)
        self.keep_ratio = keep_ratio
        dt = torch.bfloat16 if lay.dtype == CB_BF16 else torch.float32
        self.importance = torch.empty((S, L, Hkv, T), dtype=torch.float32, device=device)
        self.row_lse = torch.empty((S, L, lay.q_heads, lay.q_len), dtype=torch.float32,
                                   device=device)
        self.idx = torch.empty((S, L, Hkv, self.keep), dtype=torch.int32, device=device)
        self.k_out = torch.empty((L, Hkv, S * self.keep, lay.head_dim), dtype=dt, device=device)
        self.v_out = torch.empty_like(self.k_out)
        self.ws = torch.empty(cb_score_workspace_bytes(lay), dtype=torch.uint8, device=device)
        # cb_select_ws scratch for the staged calls (None: rows are not split)
        nsel = cb_select_workspace_bytes(self.units, T)
        self.sel_ws = torch.empty(nsel, dtype=torch.uint8, device=device) if nsel else None


def run_steps(q, k, v, buf: Buffers, want_lse=True, stream=None) -> None:
    """cb_score -> cb_select_ws -> cb_compact on one stream, into ``buf`` (the
    selection splits rows as cb_pipeline does, where it can)."""
    cb_score(q, k, buf.lay, buf.importance, buf.row_lse if want_lse else None, buf.ws,
             stream=stream)
    cb_select_ws(buf.importance, buf.units, buf.lay.seq_len, buf.keep_ratio, buf.idx, buf.sel_ws,
                 stream=stream)
    cb_compact(k, v, buf.idx, buf.lay, buf.keep, buf.k_out, buf.v_out, stream=stream)


def run_pipeline(q, k, v, buf: Buffers, want_lse=True, stream=None) -> None:
    """The fused entry point cb_pipeline, into ``buf``."""
    keep = cb_pipeline(q, k, v, buf.lay, buf.keep_ratio, buf.importance, buf.idx, buf.k_out,
                       buf.v_out, buf.ws, row_lse=buf.row_lse if want_lse else None,
                       stream=stream)
    assert keep == buf.keep


class PositionBuffers:
    """Device buffers of the position-level path for one layout (torch
    allocations): scores, Q, C, importance and the two workspaces."""

    def __init__(self, lay: cb_layout, device="cuda", span_width=16):
        import torch

        S, L, Hkv, T = lay.senders, lay.layers, lay.kv_heads, lay.seq_len
        self.lay = lay
        self.score = torch.empty((S, T), dtype=torch.float32, device=device)
        self.qscore = torch.empty_like(self.score)
        self.corr = torch.empty_like(self.score)
        self.importance = torch.empty((S, L, Hkv, T), dtype=torch.float32, device=device)
        self.ws = torch.empty(cb_position_workspace_bytes(lay), dtype=torch.uint8, device=device)
        self.span_ws = torch.empty(cb_spans_workspace_bytes(S, T, span_width), dtype=torch.uint8,
                                   device=device)


# ---------------------------------------------------------------------------
# The receiver's side: rotary positions, the paged four-bit cache, attention


_S3, _S4 = _i64 * 3, _i64 * 4
_byref = ctypes.byref
_torch = None
_raw_stream = None


def _lazy_torch():
    global _torch, _raw_stream
    if _torch is None:
        import torch

        # the current stream's handle without a Stream object (a microsecond a call)
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda dev: torch.cuda.current_stream(dev).cuda_stream)
        _torch = torch
    return _torch


def _now(stream):
    """(current device, stream as an integer): looked up once a call, as these calls take some
    microseconds in all."""
    torch = _torch or _lazy_torch()
    dev = torch.cuda.current_device()
    if stream is None:
        return dev, _raw_stream(dev)
    return dev, stream if isinstance(stream, int) else stream.cuda_stream


def _cache_now(c, where, stream):
    """_now for a call on a cache, which has to be the current device's."""
    dev, s = _now(stream)
    if c.dev != dev and c.dev is not None:
        raise CBError(-2, f"{where}: the cache is on device {c.dev}, the current one is {dev}")
    return dev, s


def _refuse(where, x, what, status=-2):
    raise CBError(status, f"{where}: {what} (got {tuple(x.shape)} {x.dtype} on {x.device})")


def _ints(x, where, dev, n=None):
    """Address of a contiguous int32 list (of n entries) on the current device; None for None."""
    if x is None:
        return None
    if x.dtype is not _torch.int32:
        _refuse(where, x, "an int32 list is wanted", -3)
    if x.dim() != 1 or (n is not None and x.shape[0] != n) or not x.is_contiguous():
        _refuse(where, x, f"a contiguous list of {'any' if n is None else n} entries is wanted")
    if x.get_device() != dev:
        _refuse(where, x, "not on the current device")
    return x.data_ptr()


def _scratch(ws, ws_bytes, where, dev):
    """Address and size of a call's scratch."""
    if ws is None or isinstance(ws, int):
        return ws, ws_bytes or 0
    if ws.get_device() != dev or not ws.is_contiguous():
        _refuse(where, ws, "scratch is not contiguous on the current device")
    return ws.data_ptr(), ws.numel() * ws.element_size() if ws_bytes is None else ws_bytes


def _float_kind(x, where):
    if x.dtype is _torch.bfloat16:
        return CB_BF16
    if x.dtype is _torch.float32:
        return CB_F32
    _refuse(where, x, "float32 or bfloat16 is wanted", -3)


def _row_strides(x, where, dev):
    """Strides of all axes but the last, whose values have to be contiguous."""
    if x.get_device() != dev:
        _refuse(where, x, "not on the current device")
    st = x.stride()
    if st[-1] != 1 and x.shape[-1] > 1:
        _refuse(where, x, "the values of a row are not contiguous")
    return st[:-1]


def cb_rotary_frequencies(rotary_dim: int, base: float = 10000.0, scaling: str = "none",
                          factor: float = 1.0, original_len: float = 0.0,
                          fast_turns: float = 0.0, slow_turns: float = 0.0):
    """(turns per position of every pair, as a host list; amplitude).  scaling:
    "none", "linear" or "yarn"."""
    import array

    kinds = {"none": 0, "linear": 1, "yarn": 2}
    if scaling not in kinds:
        raise CBError(-2, f"cb_rotary_frequencies: scaling {scaling!r}")
    rotary_dim = max(-1, min(int(rotary_dim), 1 << 20))
    r = _rope(rotary_dim, kinds[scaling], float(base), float(factor), float(original_len),
              float(fast_turns), float(slow_turns))
    freq, amp = array.array("d", bytes(8 * max(0, min(rotary_dim, 1024) // 2 + 1))), ctypes.c_double(0.0)
    _check(_lib.cb_rotary_frequencies(ctypes.byref(r), freq.buffer_info()[0], ctypes.byref(amp)),
           "cb_rotary_frequencies")
    return list(freq[:rotary_dim // 2]), amp.value


def rows(x, out, pos, frm=None) -> cb_rows:
    """Rows of one tensor for cb_rotary: x and out [a][b][c][D] (out may be x), int32 positions
    `pos` and earlier ones `frm` of shapes that broadcast to [a][b][c].  The struct keeps its
    tensors."""
    where, torch = "rows", _torch or _lazy_torch()
    dev = torch.cuda.current_device()
    kind = _float_kind(x, where)
    if x.dim() != 4 or out.shape != x.shape or x.shape[3] > 1024:
        _refuse(where, out, f"rows [a][b][c][D <= 1024] and their like are wanted, {tuple(x.shape)} given")
    if out.dtype is not x.dtype:
        _refuse(where, out, f"{x.dtype} is wanted", -3)
    r = cb_rows(x=x.data_ptr(), out=out.data_ptr(), size=_S3(*x.shape[:3]),
                in_stride=_S3(*_row_strides(x, where, dev)),
                out_stride=_S3(*_row_strides(out, where, dev)))
    r.tensors = (x, out, pos, frm)
    r.kind, r.head_dim, r.dev = kind, x.shape[3], dev
    for p, name, stride in ((pos, "pos", "pos_stride"), (frm, "frm", "from_stride")):
        if p is not None:
            if p.dtype is not torch.int32:
                _refuse(where, p, "int32 positions are wanted", -3)
            if p.get_device() != dev:
                _refuse(where, p, "not on the current device")
            try:
                q = p.expand(x.shape[:3])
            except RuntimeError:
                _refuse(where, p, f"positions do not fit rows {tuple(x.shape[:3])}")
            setattr(r, name, q.data_ptr())
            setattr(r, stride, _S3(*q.stride()))
    return r


def cb_rotary(parts, freq, amplitude: float = 1.0, interleaved: bool = False,
              transpose: bool = False, stream=None) -> None:
    """Rotates the rows of one or two tensors (`rows`) by the frequencies `freq` (device, float64,
    one a pair)."""
    where = "cb_rotary"
    if isinstance(parts, cb_rows):
        parts = (parts,)
    n = len(parts)
    if not 1 <= n <= 2:
        raise CBError(-2, f"{where}: one or two tensors")
    a = parts[0]
    if n == 2:
        if parts[1].kind != a.kind:
            raise CBError(-3, f"{where}: tensors of unlike types")
        if parts[1].head_dim != a.head_dim:
            raise CBError(-2, f"{where}: rows of unlike widths")
    dev, s = _now(stream)
    for r in parts:
        if r.dev != dev:
            raise CBError(-2, f"{where}: rows on device {r.dev}, the current one is {dev}")
    if freq.dtype is not _torch.float64:
        _refuse(where, freq, "float64 frequencies are wanted", -3)
    if freq.dim() != 1 or freq.shape[0] > 512 or not freq.is_contiguous() or freq.get_device() != dev:
        _refuse(where, freq, "a contiguous list of at most 512 on the current device is wanted")
    _check(_lib.cb_rotary((cb_rows * 2)(*parts) if n == 2 else _byref(a), n, a.head_dim,
                          freq.data_ptr(), 2 * freq.shape[0], amplitude, interleaved, transpose,
                          a.kind, s), where)


def cache(pool, refs, table, lens, head_dim: int, page_len: int) -> cb_cache:
    """Descriptor of a paged four-bit cache over the caller's tensors: pool uint8
    [pages][layers][kv_heads][unit], int32 refs [pages], table [seqs][width], lens [seqs].  It keeps
    them."""
    where, D, P, torch = "cache", int(head_dim), int(page_len), _torch or _lazy_torch()
    dev = torch.cuda.current_device()
    if pool.dtype is not torch.uint8 or table.dtype is not torch.int32:
        _refuse(where, pool, f"a uint8 pool and int32 tables are wanted, {table.dtype} given", -3)
    if pool.dim() != 4 or pool.shape[3] != P * (D + D // 16) or table.dim() != 2 or \
            max(*pool.shape, *table.shape) > 0x7fffffff:
        _refuse(where, pool, f"a pool [pages][layers][kv_heads][{P * (D + D // 16)}] is wanted")
    for t in (pool, table):
        if not t.is_contiguous() or t.get_device() != dev:
            _refuse(where, t, "not contiguous on the current device")
    c = cb_cache(pool.shape[1], pool.shape[2], D, P, pool.shape[0], table.shape[0], table.shape[1],
                 0, pool.data_ptr(), _ints(refs, where, dev, pool.shape[0]), table.data_ptr(),
                 _ints(lens, where, dev, table.shape[0]))
    c.tensors, c.dev = (pool, refs, table, lens), dev
    if _lib.cb_cache_page_bytes(_byref(c)) == 0:
        raise CBError(-2, where)
    return c


class Cache:
    """Device buffers of a paged four-bit cache (torch allocations), empty, and its descriptor
    `desc`."""

    def __init__(self, layers, kv_heads, head_dim, page_len, pages, seqs, width, device="cuda"):
        import torch

        i32 = dict(dtype=torch.int32, device=device)
        self.pool = torch.empty((pages, layers, kv_heads, page_len * (head_dim + head_dim // 16)),
                                dtype=torch.uint8, device=device)
        self.refs = torch.zeros(pages, **i32)
        self.table = torch.full((seqs, width), -1, **i32)
        self.lens = torch.zeros(seqs, **i32)
        self.status = torch.zeros(1, **i32)
        self.desc = cache(self.pool, self.refs, self.table, self.lens, head_dim, page_len)


def cb_cache_page_bytes(c: cb_cache) -> int:
    return _lib.cb_cache_page_bytes(_byref(c))


def cb_cache_status(status, stream=None) -> int:
    """Synchronises the stream and returns 0 (CB_OK), -9 (CB_ERR_PAGES: pages lacked) or -2
    (CB_ERR_SHAPE: an invalid entry) for the last call that wrote `status`."""
    dev, s = _now(stream)
    return _lib.cb_cache_status(_ints(status, "cb_cache_status", dev, 1), s)


def cb_cache_extend(c: cb_cache, seqs, add, status, stream=None) -> None:
    where = "cb_cache_extend"
    dev, s = _cache_now(c, where, stream)
    n = seqs.numel()
    _check(_lib.cb_cache_extend(_byref(c), _ints(seqs, where, dev), _ints(add, where, dev, n), n,
                                _ints(status, where, dev, 1), s), where)


def cb_cache_free(c: cb_cache, seqs, stream=None) -> None:
    where = "cb_cache_free"
    dev, s = _cache_now(c, where, stream)
    _check(_lib.cb_cache_free(_byref(c), _ints(seqs, where, dev), seqs.numel(), s), where)


def cb_cache_fork_workspace_bytes(c: cb_cache, n: int) -> int:
    return _lib.cb_cache_fork_workspace_bytes(_byref(c), n)


def cb_cache_fork(c: cb_cache, parents, children, status, ws, copy: bool = False, ws_bytes=None,
                  stream=None) -> None:
    where = "cb_cache_fork"
    dev, s = _cache_now(c, where, stream)
    n = parents.numel()
    _check(_lib.cb_cache_fork(_byref(c), _ints(parents, where, dev), _ints(children, where, dev, n),
                              n, copy, _ints(status, where, dev, 1),
                              *_scratch(ws, ws_bytes, where, dev), s), where)


def cb_cache_compact_workspace_bytes(c: cb_cache, n: int) -> int:
    return _lib.cb_cache_compact_workspace_bytes(_byref(c), n)


def cb_cache_compact(c: cb_cache, src, dst, idx, status, ws, counts=None, ws_bytes=None,
                     stream=None) -> None:
    """idx: int32 [n][layers or 1][kv_heads or 1][keep]; an axis of one serves all."""
    where = "cb_cache_compact"
    dev, s = _cache_now(c, where, stream)
    n = src.numel()
    if idx.dtype is not _torch.int32:
        _refuse(where, idx, "int32 positions are wanted", -3)
    shape = idx.shape
    if len(shape) != 4 or shape[0] != n or shape[1] not in (1, c.layers) or \
            shape[2] not in (1, c.kv_heads):
        _refuse(where, idx, f"lists [{n}][{c.layers} or 1][{c.kv_heads} or 1][keep] are wanted")
    st = _row_strides(idx, where, dev)
    stride = _S3(st[0], 0 if shape[1] == 1 else st[1], 0 if shape[2] == 1 else st[2])
    _check(_lib.cb_cache_compact(_byref(c), _ints(src, where, dev), _ints(dst, where, dev, n), n,
                                 idx.data_ptr(), stride, shape[3], _ints(counts, where, dev, n),
                                 _ints(status, where, dev, 1), *_scratch(ws, ws_bytes, where, dev),
                                 s), where)


def _cache_rows(fn, where, c, k, v, seqs, start, counts, layer, stream):
    dev, s = _cache_now(c, where, stream)
    kind, shape = _float_kind(k, where), k.shape
    if len(shape) != 5 or shape[2] != c.kv_heads or shape[4] != c.head_dim or v.shape != shape or \
            (shape[0] | shape[1] | shape[2]) >> 31 or not 0 <= layer < 4096:
        _refuse(where, v, f"rows [layers][n][{c.kv_heads}][rows][{c.head_dim}] are wanted, keys and "
                          f"values alike, {tuple(shape)} at layer {layer} given")
    if v.dtype is not k.dtype:
        _refuse(where, v, f"{k.dtype} is wanted", -3)
    st, sv = _row_strides(k, where, dev), _row_strides(v, where, dev)
    if st != sv and any(a != b and size > 1 for a, b, size in zip(st, sv, shape)):   # of axes that are walked
        _refuse(where, v, "keys and values of unlike strides")
    n = shape[1]
    _check(fn(_byref(c), layer, shape[0], _ints(seqs, where, dev, n), n, _ints(start, where, dev, n),
              _ints(counts, where, dev, n), shape[3], k.data_ptr(), v.data_ptr(), _S4(*st), kind, s),
           where)


def cb_cache_write(c: cb_cache, k, v, seqs=None, start=None, counts=None, layer: int = 0,
                   stream=None) -> None:
    """k, v [layers][n][kv_heads][rows][D] into the cache, from `layer` on."""
    _cache_rows(_lib.cb_cache_write, "cb_cache_write", c, k, v, seqs, start, counts, layer, stream)


def cb_cache_read(c: cb_cache, k, v, seqs=None, start=None, counts=None, layer: int = 0,
                  stream=None) -> None:
    """The cache's values into k, v [layers][n][kv_heads][rows][D]."""
    _cache_rows(_lib.cb_cache_read, "cb_cache_read", c, k, v, seqs, start, counts, layer, stream)


def cb_cache_attend_workspace_bytes(c: cb_cache, layers: int, n: int, q_heads: int,
                                    q_len: int, longest: int = 0) -> int:
    """Scratch bytes of cb_cache_attend (0: it needs none)."""
    return _lib.cb_cache_attend_workspace_bytes(_byref(c), layers, n, q_heads, q_len, longest)


def cb_cache_attend(c: cb_cache, q, out, ws=None, lse=None, seqs=None, q_lens=None,
                    causal: bool = True, scale: float = 0.0, layer: int = 0, ws_bytes=None,
                    stream=None, longest: int = 0) -> None:
    """q, out [layers][n][q_heads][q_len][D]; lse [layers][n][q_heads][q_len] fp32.  longest: the
    longest of the sequences, where the host knows it (scratch asked for with the same)."""
    where = "cb_cache_attend"
    dev, s = _cache_now(c, where, stream)
    kind, shape = _float_kind(q, where), q.shape
    if len(shape) != 5 or shape[4] != c.head_dim or out.shape != shape or \
            (shape[0] | shape[1] | shape[2]) >> 31 or not 0 <= layer < 4096:
        _refuse(where, out, f"rows [layers][n][q_heads][q_len][{c.head_dim}] and their like are wanted, "
                            f"{tuple(shape)} at layer {layer} given")
    if out.dtype is not q.dtype:
        _refuse(where, out, f"{q.dtype} is wanted", -3)
    qs, os_ = _row_strides(q, where, dev), _row_strides(out, where, dev)
    if lse is not None and (lse.dtype is not _torch.float32 or lse.shape != shape[:4] or
                            not lse.is_contiguous() or lse.get_device() != dev):
        _refuse(where, lse, f"contiguous float32 {tuple(shape[:4])} on the current device is wanted")
    n = shape[1]
    _check(_lib.cb_cache_attend(_byref(c), layer, shape[0], _ints(seqs, where, dev, n), n,
                                q.data_ptr(), _S4(*qs), shape[2], _ints(q_lens, where, dev, n),
                                shape[3], causal, longest, scale, out.data_ptr(), _S4(*os_),
                                None if lse is None else lse.data_ptr(), kind,
                                *_scratch(ws, ws_bytes, where, dev), s), where)


__all__ = ["cb_layout", "layout", "layout_of", "cb_score_workspace_bytes", "cb_score",
           "cb_keep_count", "cb_select", "cb_compact", "cb_status_string", "CBError",
           "cb_pipeline", "cb_score_status", "cb_set_wait_limit", "cb_position_workspace_bytes",
           "cb_position_score", "cb_position_status", "cb_budget_fanout", "cb_budget_chain",
           "cb_spans_workspace_bytes", "cb_select_spans", "cb_gather_rows", "PositionBuffers",
           "cb_pipeline_noalloc", "cb_select_workspace_bytes", "cb_select_ws", "cb_select_status",
           "cb_rotary_frequencies", "cb_rows", "rows", "cb_rotary", "cb_cache", "cache", "Cache",
           "cb_cache_page_bytes", "cb_cache_status", "cb_cache_extend", "cb_cache_free",
           "cb_cache_fork_workspace_bytes", "cb_cache_fork", "cb_cache_compact_workspace_bytes",
           "cb_cache_compact", "cb_cache_write", "cb_cache_read",
           "cb_cache_attend_workspace_bytes", "cb_cache_attend",
           "Buffers", "run_steps", "run_pipeline", "CB_F32", "CB_BF16",
           "LIB_PATH"]

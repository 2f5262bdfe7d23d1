"""Thin ctypes binding of ``libdart.so`` (declared in ``include/dart.h``).

Argument marshalling only: every step of the reduction runs in the library's CUDA kernels.
There is no CPU fallback; if the library is missing the first use raises.  The module-level
functions carry the C names; :class:`Dart` wraps a context for torch tensors (torch supplies
device memory and streams, nothing else).
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import threading
from typing import Optional

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libdart.so")

DART_OK = 0
DART_ERR_NULL, DART_ERR_BAD_SHAPE, DART_ERR_ALIGN, DART_ERR_ALIAS = -1, -2, -3, -4
DART_ERR_CUDA, DART_ERR_NOMEM, DART_ERR_TIMEOUT, DART_ERR_CHECK, DART_ERR_UNSUPPORTED = -5, -6, -7, -8, -9
DART_FLAG_HOST_STAGING = 1
DART_PATH_AUTO, DART_PATH_STAGED, DART_PATH_FUSED, DART_PATH_TWO_PASS, DART_PATH_RESIDENT, DART_PATH_SPLIT, DART_PATH_PAIRED = 0, 1, 2, 3, 4, 5, 6
DART_PATH_FLOW = 7
DART_RETAIN_AUTO, DART_RETAIN_SERIAL, DART_RETAIN_LISTS, DART_RETAIN_BANDS, DART_RETAIN_FUSED = 0, 1, 2, 3, 4
DART_RETAIN_RANKED = 5
DART_RULE_QUOTAS, DART_RULE_GLOBAL, DART_RULE_UNION = 0, 1, 2
DART_PIVOTS_BY_SCORE, DART_PIVOTS_MIXED, DART_PIVOTS_RANDOM = 0, 1, 2

EXPORTS = (
    "dart_create", "dart_destroy", "dart_set_shape", "dart_reduce", "dart_reduce_ex", "dart_reduce_host",
    "dart_status", "dart_status_detail", "dart_last_cuda_error", "dart_workspace_bytes", "dart_launch_count",
    "dart_profile_enable", "dart_profile_read", "dart_strerror", "dart_version", "dart_pivots_static",
    "dart_gather_rows", "dart_norm_rope", "dart_cache_append", "dart_attend_workspace", "dart_attend",
)
DART_STATIC_MAX_ROWS = 262144
DART_BF16, DART_FP16 = 0, 1


class dart_desc(ctypes.Structure):
    _fields_ = [("B_max", ctypes.c_int32), ("S_max", ctypes.c_int32), ("d", ctypes.c_int32),
                ("P_max", ctypes.c_int32), ("Kp_max", ctypes.c_int32), ("device", ctypes.c_int32),
                ("flags", ctypes.c_uint32)]


class dart_opts(ctypes.Structure):
    _fields_ = [("norm_kind", ctypes.c_int32), ("pivot_smallest", ctypes.c_int32), ("path", ctypes.c_int32),
                ("wait_limit", ctypes.c_int32), ("sweep_lag", ctypes.c_int32),
                ("test_withhold_pivots", ctypes.c_int32), ("retention", ctypes.c_int32), ("rule", ctypes.c_int32),
                ("cosine_on_hidden", ctypes.c_int32), ("text_pivots", ctypes.c_int32), ("pivots_in", ctypes.c_void_p),
                ("cu_seqlens", ctypes.c_void_p), ("resident_split", ctypes.c_int32), ("pivot_source", ctypes.c_int32),
                ("n_text_pivots", ctypes.c_int32), ("seed", ctypes.c_uint64), ("sample_base", ctypes.c_int32),
                ("tune", ctypes.c_int32)]


class dart_debug(ctypes.Structure):
    _fields_ = [("l1", ctypes.c_void_p), ("ssq", ctypes.c_void_p), ("pivot_idx", ctypes.c_void_p),
                ("sim", ctypes.c_void_p), ("eps", ctypes.c_void_p), ("keep", ctypes.c_void_p),
                ("owner", ctypes.c_void_p)]


class dart_rope(ctypes.Structure):
    _fields_ = [("inv_freq", ctypes.c_void_p), ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("n_axes", ctypes.c_int32),
                ("section", ctypes.c_int32 * 3)]


class dart_cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("n_pages", ctypes.c_int32), ("n_heads", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("device", ctypes.c_int32)]


class dart_attend_args(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("out", ctypes.c_void_p), ("lse", ctypes.c_void_p), ("q_stride", ctypes.c_int64),
                ("out_stride", ctypes.c_int64), ("n_rows", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("n_seq", ctypes.c_int32), ("n_groups", ctypes.c_int32), ("cu_q", ctypes.c_void_p), ("table", ctypes.c_void_p),
                ("kv_len", ctypes.c_void_p), ("cu_group", ctypes.c_void_p), ("prefix_table", ctypes.c_void_p),
                ("prefix_len", ctypes.c_void_p), ("table_stride", ctypes.c_int32), ("prefix_stride", ctypes.c_int32),
                ("scale", ctypes.c_float), ("wait_limit", ctypes.c_int32), ("status", ctypes.c_void_p),
                ("test_withhold", ctypes.c_int32)]


class DartError(RuntimeError):
    def __init__(self, code: int, what: str):
        self.code = code
        super().__init__("%s: %s (%d)" % (what, dart_strerror(code), code))


_lib = None


def lib() -> ctypes.CDLL:
    """Load libdart.so (once).  Raises if it has not been built: there is no other code path."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("%s is missing: build it with `python -m paper_2502_11494_b200.build`; "
                               "the reduction has no fallback path" % LIB_PATH)
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64p, i32p = ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p
        L.dart_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(dart_desc)]
        L.dart_destroy.argtypes = [vp]
        L.dart_set_shape.argtypes = [vp, i32, i32]
        L.dart_reduce.argtypes = [vp, vp, vp, i32, i32, i32, i32, vp, i32p, i64p, vp]
        L.dart_reduce_ex.argtypes = [vp, vp, vp, i64p, i32, i32, i32, i32, vp, i32p, i64p,
                                     ctypes.POINTER(dart_opts), ctypes.POINTER(dart_debug), vp]
        L.dart_reduce_host.argtypes = [vp, vp, vp, i32, i32, i32, i32, vp, i32p, i64p]
        L.dart_status.argtypes = [vp]
        L.dart_status_detail.argtypes = [vp, ctypes.POINTER(ctypes.c_int32)]
        L.dart_last_cuda_error.argtypes = [vp]
        L.dart_workspace_bytes.argtypes = [vp]
        L.dart_workspace_bytes.restype = ctypes.c_size_t
        L.dart_launch_count.argtypes = [vp]
        L.dart_launch_count.restype = ctypes.c_int64
        L.dart_profile_enable.argtypes = [vp, i32]
        L.dart_profile_read.argtypes = [vp, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_int32),
                                        ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(ctypes.c_int)]
        L.dart_pivots_static.argtypes = [vp, i32, i32, i32, i32, i32, i32, i32p, i32, vp]
        L.dart_gather_rows.argtypes = [vp, i32p, i32, i32, i32, i32, vp, i32, vp]
        i64, f32 = ctypes.c_int64, ctypes.c_float
        L.dart_norm_rope.argtypes = [vp, i64, i32, vp, i64, i32, i32, i32, i32, vp, vp, f32, ctypes.POINTER(dart_rope), vp, i64,
                                     vp, i64, vp, i64, i32, vp]
        L.dart_cache_append.argtypes = [ctypes.POINTER(dart_cache), vp, i64, vp, i64, i32, i32, vp, vp, i32, vp, i32, vp, vp, f32,
                                        ctypes.POINTER(dart_rope), vp, i64, vp, vp]
        L.dart_attend_workspace.argtypes = [ctypes.POINTER(dart_cache), ctypes.POINTER(dart_attend_args)]
        L.dart_attend_workspace.restype = ctypes.c_size_t
        L.dart_attend.argtypes = [ctypes.POINTER(dart_cache), ctypes.POINTER(dart_attend_args), vp, ctypes.c_size_t, vp]
        L.dart_strerror.argtypes = [i32]
        L.dart_strerror.restype = ctypes.c_char_p
        L.dart_version.argtypes = []
        _lib = L
    return _lib


# ---- the C entry points under their own names (raw pointers as ints) ---------------------------

def dart_strerror(code: int) -> str:
    return lib().dart_strerror(code).decode()


def dart_version() -> int:
    return lib().dart_version()


def dart_create(B_max, S_max, d, P_max, Kp_max, device=0, flags=0):
    """-> (return code, context handle)."""
    h = ctypes.c_void_p()
    desc = dart_desc(B_max, S_max, d, P_max, Kp_max, device, flags)
    rc = lib().dart_create(ctypes.byref(h), ctypes.byref(desc))
    return rc, h


def dart_destroy(ctx) -> int:
    return lib().dart_destroy(ctx)


def dart_set_shape(ctx, B, S) -> int:
    return lib().dart_set_shape(ctx, B, S)


def dart_reduce(ctx, hidden, keys, vis_offset, n_vis, n_pivot, n_keep, out_hidden, out_idx, out_pos, stream) -> int:
    return lib().dart_reduce(ctx, hidden, keys, vis_offset, n_vis, n_pivot, n_keep, out_hidden, out_idx, out_pos, stream)


def dart_reduce_ex(ctx, hidden, keys, pos_in, vis_offset, n_vis, n_pivot, n_keep, out_hidden, out_idx, out_pos,
                   opts: Optional[dart_opts], dbg: Optional[dart_debug], stream) -> int:
    return lib().dart_reduce_ex(ctx, hidden, keys, pos_in, vis_offset, n_vis, n_pivot, n_keep, out_hidden, out_idx,
                                out_pos, ctypes.byref(opts) if opts is not None else None,
                                ctypes.byref(dbg) if dbg is not None else None, stream)


def dart_reduce_host(ctx, hidden, keys, vis_offset, n_vis, n_pivot, n_keep, out_hidden, out_idx, out_pos) -> int:
    return lib().dart_reduce_host(ctx, hidden, keys, vis_offset, n_vis, n_pivot, n_keep, out_hidden, out_idx, out_pos)


def dart_pivots_static(keys, B, S, d, vis_offset, n_vis, n_pivot, pivot_idx, device, stream) -> int:
    """Context-free, allocation-free pivot selection (raw device pointers); see include/dart.h."""
    return lib().dart_pivots_static(keys, B, S, d, vis_offset, n_vis, n_pivot, pivot_idx, device, stream)


def dart_gather_rows(src, idx, B, S, S_out, row_bytes, out, device, stream) -> int:
    """Context-free row gather by a packed index list (raw device pointers); see include/dart.h."""
    return lib().dart_gather_rows(src, idx, B, S, S_out, row_bytes, out, device, stream)


def dart_norm_rope(q, q_stride, n_q_heads, k, k_stride, n_k_heads, n_rows, head_dim, dtype, q_weight, k_weight, eps,
                   rope: Optional[dart_rope], pos, pos_stride, q_out, qo_stride, k_out, ko_stride, device, stream) -> int:
    """Norm of each head and position rotation of queries and keys (raw device pointers); see include/dart.h."""
    return lib().dart_norm_rope(q, q_stride, n_q_heads, k, k_stride, n_k_heads, n_rows, head_dim, dtype, q_weight, k_weight,
                                eps, rope, pos, pos_stride, q_out, qo_stride, k_out, ko_stride, device, stream)


def dart_cache_append(cache: Optional[dart_cache], k, k_stride, v, v_stride, n_seq, n_rows, cu_rows, idx, S, table, table_stride,
                      start, k_weight, eps, rope: Optional[dart_rope], pos, pos_stride, status, stream) -> int:
    """Rows of keys and values into the pages of a cache (raw device pointers); see include/dart.h."""
    return lib().dart_cache_append(cache, k, k_stride, v, v_stride, n_seq, n_rows, cu_rows, idx, S, table, table_stride, start,
                                   k_weight, eps, rope, pos, pos_stride, status, stream)


def dart_attend_workspace(cache: Optional[dart_cache], args: Optional[dart_attend_args]) -> int:
    return lib().dart_attend_workspace(cache, args)


def dart_attend(cache: Optional[dart_cache], args: Optional[dart_attend_args], workspace, workspace_bytes, stream) -> int:
    """Attention over a paged cache, with prefixes that groups of sequences share (raw device pointers); see include/dart.h."""
    return lib().dart_attend(cache, args, workspace, workspace_bytes, stream)


def dart_status(ctx) -> int:
    return lib().dart_status(ctx)


def dart_status_detail(ctx):
    """-> (return code, [which wait, task index, CTA]) of the last error that dart_status reported."""
    d = (ctypes.c_int32 * 11)()
    rc = lib().dart_status_detail(ctx, d)
    return rc, list(d)


def dart_last_cuda_error(ctx) -> int:
    return lib().dart_last_cuda_error(ctx)


def dart_workspace_bytes(ctx) -> int:
    return lib().dart_workspace_bytes(ctx)


def dart_launch_count(ctx) -> int:
    return lib().dart_launch_count(ctx)


def dart_profile_enable(ctx, on: bool) -> int:
    return lib().dart_profile_enable(ctx, int(on))


def dart_profile_read(ctx):
    """-> (return code, {kernel name: (milliseconds, launches)}) accumulated since the last read."""
    cap = 16
    ms = (ctypes.c_float * cap)()
    n_l = (ctypes.c_int32 * cap)()
    names = (ctypes.c_char_p * cap)()
    n = ctypes.c_int(cap)
    rc = lib().dart_profile_read(ctx, ms, n_l, names, ctypes.byref(n))
    return rc, {names[k].decode(): (float(ms[k]), int(n_l[k])) for k in range(n.value)} if rc == 0 else {}


# ---- torch convenience wrapper --------------------------------------------------------------------

def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _made_for(stream):
    """Where tensors are made that a call on ``stream`` writes or reads: the allocator hands out memory whose last user is of the stream that is
    current, and may still be at work there."""
    if stream is None:
        return contextlib.nullcontext()
    import torch

    return torch.cuda.stream(stream)


class Dart:
    """A reduction context bound to one CUDA device.  ``reduce`` enqueues on torch's current stream, or on ``stream``."""

    def __init__(self, B_max, S_max, d, P_max, Kp_max, device=0, flags=0):
        rc, self._h = dart_create(B_max, S_max, d, P_max, Kp_max, device, flags)
        if rc != DART_OK:
            self._h = None
            raise DartError(rc, "dart_create")
        self.B_max, self.S_max, self.d, self.P_max, self.Kp_max, self.device = B_max, S_max, d, P_max, Kp_max, device

    def close(self):
        if getattr(self, "_h", None) is not None:
            dart_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def handle(self):
        return self._h

    def reduce(self, hidden, keys, vis_offset, n_vis, n_pivot, n_keep, pos_in=None, out=None, opts=None,
               debug=False, stream=None):
        """hidden/keys: [B, S, d] bf16 CUDA tensors.  Returns (out_hidden, out_idx, out_pos[, dbg dict])."""
        import torch

        B, S, d = hidden.shape
        if not (hidden.is_cuda and hidden.is_contiguous() and hidden.dtype == torch.bfloat16):
            raise ValueError("hidden must be a contiguous bf16 CUDA tensor")
        if keys is not None and not (keys.is_cuda and keys.is_contiguous() and keys.dtype == torch.bfloat16
                                     and keys.shape == hidden.shape):
            raise ValueError("keys must be a contiguous bf16 CUDA tensor shaped like hidden")
        if d != self.d:
            raise ValueError("row width %d differs from the context's %d" % (d, self.d))
        rc = dart_set_shape(self._h, B, S)
        if rc != DART_OK:
            raise DartError(rc, "dart_set_shape")
        S_out = S - n_vis + n_keep
        dev = hidden.device
        if out is None:
            if not (0 < n_keep <= n_vis <= S):
                raise DartError(DART_ERR_BAD_SHAPE, "dart_reduce")
            with _made_for(stream):
                out = (torch.empty((B, S_out, d), dtype=torch.bfloat16, device=dev),
                       torch.empty((B, S_out), dtype=torch.int32, device=dev),
                       torch.empty((B, S_out), dtype=torch.int64, device=dev))
        oh, oi, op = out
        dbg_t, dbg_s = None, None
        if debug:
            with _made_for(stream):
                dbg_t = {
                    "l1": torch.empty((B, n_vis), dtype=torch.float32, device=dev),
                    "ssq": torch.empty((B, n_vis), dtype=torch.float32, device=dev),
                    "pivot_idx": torch.empty((B, n_pivot), dtype=torch.int32, device=dev),
                    "sim": torch.empty((B, n_pivot, n_vis), dtype=torch.float32, device=dev),
                    "eps": torch.empty((B, n_pivot), dtype=torch.float32, device=dev),
                    "keep": torch.empty((B, n_vis), dtype=torch.uint8, device=dev),
                    "owner": torch.empty((B, n_vis), dtype=torch.int32, device=dev),
                }
            dbg_s = dart_debug(**{k: v.data_ptr() for k, v in dbg_t.items()})
        st = stream if stream is not None else torch.cuda.current_stream(dev)
        rc = dart_reduce_ex(self._h, _ptr(hidden), _ptr(keys), _ptr(pos_in), vis_offset, n_vis, n_pivot, n_keep,
                            _ptr(oh), _ptr(oi), _ptr(op), opts, dbg_s, ctypes.c_void_p(st.cuda_stream))
        if rc != DART_OK:
            raise DartError(rc, "dart_reduce_ex")
        return (oh, oi, op, dbg_t) if debug else (oh, oi, op)

    def status(self) -> int:
        return dart_status(self._h)


# ---- around the reduction: rotated rows, the paged cache -------------------------------------------
# (One token of a few sequences takes the GPU 3 us: the checks below ask a tensor for as little as they can.)

_CODES = {}      # torch dtypes -> DART_*
_raw_stream = None


def _with_torch():
    """torch, once: the current stream of a device as a number, and the types that rows may have."""
    global _raw_stream
    import torch

    _CODES.update({torch.bfloat16: DART_BF16, torch.float16: DART_FP16})
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
    return torch


def _code(dtype):
    if not _CODES:
        _with_torch()
    if dtype not in _CODES:
        raise ValueError("rows must be bf16 or fp16")
    return _CODES[dtype]


def _on(stream, device, index):
    """The stream of a call as a number: the caller's, or the device's current one."""
    if stream is None:
        return _raw_stream(index)
    if stream.device != device:
        raise ValueError("the stream must be of the rows' device")
    return stream.cuda_stream


def _head_rows(t, name, dtype, device, n_rows, D):
    """Rows [n_rows, heads, D] with the heads of a row side by side -> (address, values from row to row, heads)."""
    shape, stride = t.shape, t.stride()
    if len(shape) != 3 or t.dtype is not dtype or t.device != device or shape[0] != n_rows or shape[2] != D:
        raise ValueError("%s must be [%d rows, heads, %d] of type %s on %s" % (name, n_rows, D, dtype, device))
    h = shape[1]
    if (stride[2] != 1 and D > 1) or (stride[1] != D and h > 1):
        raise ValueError("%s: the heads of a row must lie side by side" % name)
    return t.data_ptr(), stride[0] if n_rows > 1 else h * D, h


def _vector(t, name, size, dtype, device):
    if t is None:
        return None
    if t.dtype is not dtype or t.device != device or t.shape != (size,) or not t.is_contiguous():
        raise ValueError("%s must be a contiguous vector of %d values of type %s on %s" % (name, size, dtype, device))
    return t.data_ptr()


class Rope:
    """A position rotation: the first ``2 * len(inv_freq)`` elements of a head turn by ``pos * inv_freq``, pairs being
    ``(i, i + half)`` or, ``interleaved``, ``(2i, 2i + 1)``.  ``sections``: pairs per position axis (vision tokens in time,
    height and width).  Positions [axes, N] have rows of their own: ``pos.expand(3, N)`` of text tokens is to be made contiguous."""

    def __init__(self, inv_freq, interleaved=False, sections=None):
        import torch

        if not (inv_freq.is_cuda and inv_freq.dtype == torch.float32 and inv_freq.dim() == 1 and inv_freq.is_contiguous()):
            raise ValueError("inv_freq must be a contiguous fp32 CUDA vector")
        self.inv_freq, self.axes, self.device = inv_freq, len(sections) if sections is not None else 1, inv_freq.device
        if not 1 <= self.axes <= 3:
            raise ValueError("one to three sections")
        self._int64 = torch.int64
        self._c = dart_rope(inv_freq.data_ptr(), 2 * inv_freq.numel(), int(interleaved), self.axes,
                            tuple(int(n) for n in sections) + (0,) * (3 - self.axes) if sections is not None else (0, 0, 0))

    def at(self, pos, n_rows, device):
        """(struct, address, stride) for rows at ``pos`` ([n_rows], or [axes, n_rows]; None where the callee has its own)."""
        if device != self.device:
            raise ValueError("inv_freq and the rows must be on the same device")
        if pos is None:
            return self._c, None, 0
        shape, stride = pos.shape, pos.stride()
        if (pos.dtype is not self._int64 or pos.device != device or shape[-1] != n_rows or (n_rows > 1 and stride[-1] != 1)
                or (shape[0] if len(shape) == 2 else 1) != self.axes or not 1 <= len(shape) <= 2):
            raise ValueError("pos must be int64 [%s%d] on the rows' device" % ("%d, " % self.axes if self.axes > 1 else "", n_rows))
        return self._c, pos.data_ptr(), stride[0] if self.axes > 1 else n_rows


_NO_ROPE = (None, None, 0)
_NO_ROWS = (None, 0, 0)


def norm_rope(q, k, pos=None, rope=None, q_weight=None, k_weight=None, eps=1e-6, out=None, stream=None):
    """Norm of each head (``q_weight`` / ``k_weight`` [D], None: no norm) and rotation of queries [N, Hq, D] and keys [N, Hk, D]
    (either may be None) in one pass.  ``pos``: int64 [N], or [axes, N].  ``out``: (q_out, k_out), which may be q and k
    themselves; made for ``stream`` if None.  Returns (q_out, k_out).

    The keys are what ``Dart.reduce`` scores (bf16): ``reduce(hidden, keys)`` where they are as wide as the hidden rows; with fewer key heads
    ``reduce(keys, None)``, and ``dart_gather_rows`` packs the hidden rows by its index list."""
    one = q if q is not None else k
    if one is None:
        raise ValueError("queries or keys are needed")
    dtype, dev, shape = one.dtype, one.device, one.shape
    code, index = _code(dtype), dev.index
    if index is None:
        raise ValueError("rows must be CUDA tensors")
    n, D = shape[0], shape[-1]
    st = _on(stream, dev, index)
    if out is None:
        with _made_for(stream):
            out = tuple(t.new_empty(t.shape) if t is not None else None for t in (q, k))
    q_out, k_out = out
    qa = _head_rows(q, "q", dtype, dev, n, D) if q is not None else _NO_ROWS
    ka = _head_rows(k, "k", dtype, dev, n, D) if k is not None else _NO_ROWS
    qo = _head_rows(q_out, "q_out", dtype, dev, n, D) if q is not None else _NO_ROWS
    ko = _head_rows(k_out, "k_out", dtype, dev, n, D) if k is not None else _NO_ROWS
    if qo[2] != qa[2] or ko[2] != ka[2]:
        raise ValueError("outputs must have the heads of their inputs")
    if rope is None:
        turn = _NO_ROPE
    elif pos is None:
        raise ValueError("a rotation needs positions")
    else:
        turn = rope.at(pos, n, dev)
    rc = lib().dart_norm_rope(qa[0], qa[1], qa[2], ka[0], ka[1], ka[2], n, D, code, _vector(q_weight, "q_weight", D, dtype, dev),
                              _vector(k_weight, "k_weight", D, dtype, dev), eps, turn[0], turn[1], turn[2], qo[0], qo[1], ko[0], ko[1], index,
                              st)
    if rc != DART_OK:
        raise DartError(rc, "dart_norm_rope")
    return out


class PagedCache:
    """A cache of keys and values in pages: two tensors [pages, heads, page_size, head_dim], the caller's.  A sequence's token
    number s lies in page ``table[sequence, s // page_size]``.  ``append`` fills pages of any size and head_dim up to 256 (a multiple of
    8); ``attend`` reads head_dim 64 and 128 and page_size 16 to 1024, a power of two, and refuses others."""

    def __init__(self, k, v):
        torch = _with_torch()
        if not (k.is_cuda and k.dim() == 4 and k.shape == v.shape and k.dtype == v.dtype and k.device == v.device
                and k.is_contiguous() and v.is_contiguous()):
            raise ValueError("k and v must be contiguous CUDA tensors [pages, heads, page_size, head_dim] of one type and device")
        self.k, self.v, self.device, self.dtype = k, v, k.device, k.dtype
        self.heads, self.head_dim, self._index = k.shape[1], k.shape[3], k.device.index
        self._status = torch.zeros(4, dtype=torch.int32, device=k.device)
        with torch.cuda.device(k.device):  # (cleared before a call on another stream reports; a capture clears it by itself)
            if not torch.cuda.is_current_stream_capturing():
                torch.cuda.current_stream().synchronize()
        self._status_at, self._int32, self._torch = self._status.data_ptr(), torch.int32, torch
        self._lock = threading.Lock()  # held by a launch, and by status() from its waiting to its clearing
        self._c = dart_cache(k.data_ptr(), v.data_ptr(), k.shape[0], k.shape[1], k.shape[2], k.shape[3], _code(k.dtype), self._index)

    def _ints(self, t, name, size=None):
        if t is None:
            return None
        if t.dtype is not self._int32 or t.device != self.device or not t.is_contiguous() or (size is not None and t.shape != (size,)):
            raise ValueError("%s must be contiguous int32%s on %s" % (name, " [%d]" % size if size is not None else "", self.device))
        return t.data_ptr()

    def _table(self, t, name, stream=None):
        """(address, entries from row to row, rows, what has to live until the launch).  The rows of a view are as wide as its stride for the
        kernels, which look at lengths against that: a view whose last row ends beyond its memory is copied."""
        shape, stride = t.shape, t.stride()
        if (t.dtype is not self._int32 or t.device != self.device or len(shape) != 2 or (shape[1] > 1 and stride[1] != 1)
                or (shape[0] > 1 and stride[0] < shape[1])):
            raise ValueError("%s must be int32 [sequences, pages] on %s" % (name, self.device))
        if shape[0] > 1 and stride[0] > shape[1] and 4 * (t.storage_offset() + shape[0] * stride[0]) > t.untyped_storage().nbytes():
            with _made_for(stream):
                t = t.contiguous()
            stride = t.stride()
        return t.data_ptr(), stride[0] if shape[0] > 1 else shape[1], shape[0], t

    def append(self, k, v, table, start=None, cu_rows=None, idx=None, S=0, pos=None, rope=None, k_weight=None, eps=1e-6, stream=None):
        """Rows of keys and values [N, heads, D] behind the ``start`` tokens that each sequence already has.  ``cu_rows``
        [sequences + 1]: ragged numbers of rows (None: equally many).  ``idx`` (a reduction's out_idx, flat or [B, S_out]): take row
        b * S + idx[n] for packed row n.  The keys are normalised (``k_weight``) and rotated (``rope``, at ``pos`` or at the slots)
        on the way; a slot is the number in the sequence's own pages, so that tokens behind a shared prefix need ``pos``."""
        dev, dtype, D = self.device, self.dtype, self.head_dim
        tp, ts, n_seq, table = self._table(table, "table", stream)
        rows = k.shape[0]
        ka, va = _head_rows(k, "k", dtype, dev, rows, D), _head_rows(v, "v", dtype, dev, rows, D)
        if ka[2] != self.heads or va[2] != self.heads:
            raise ValueError("k and v must have the cache's heads")
        n = rows
        if idx is not None:
            n = idx.numel()
            if S < 1 or rows != n_seq * S:
                raise ValueError("with idx, k and v hold S rows per sequence")
        if rope is None:
            turn = _NO_ROPE
        else:
            if pos is not None and rope.axes == 1 and pos.dim() > 1:
                with _made_for(stream):  # (positions that lie apart are copied)
                    pos = pos.reshape(-1)
            turn = rope.at(pos, n, dev)
        args = (self._c, ka[0], ka[1], va[0], va[1], n_seq, n, self._ints(cu_rows, "cu_rows", n_seq + 1), self._ints(idx, "idx"), S, tp, ts,
                self._ints(start, "start", n_seq), _vector(k_weight, "k_weight", D, dtype, dev), eps, turn[0], turn[1], turn[2], self._status_at,
                _on(stream, dev, self._index))
        with self._lock:
            rc = lib().dart_cache_append(*args)
        if rc != DART_OK:
            raise DartError(rc, "dart_cache_append")

    def attend(self, q, table, kv_len, cu_q=None, prefix=None, scale=None, out=None, lse=None, wait_limit=0, stream=None):
        """Attention of query rows [N, Hq, D] over the cached tokens of their sequences: ``kv_len`` own tokens in the pages of
        ``table`` [sequences, pages], the rows' own new tokens the last of them, and with ``prefix`` = (table [groups, pages],
        lengths [groups], cu_group [groups + 1]) the tokens that a group of sequences shares.  ``cu_q`` [sequences + 1]: ragged
        numbers of rows (None: one row per sequence).  ``scale``: None for 1 / sqrt(D).  Returns ``out`` (made if None); ``lse``, a
        fp32 tensor [N, Hq], is filled if given.  Keys and values of visible tokens must be finite; a query that holds a NaN or an
        infinity has a row of NaN."""
        if stream is not None:  # (what is made below is made for that stream)
            _on(stream, self.device, self._index)
            with self._torch.cuda.stream(stream):
                return self.attend(q, table, kv_len, cu_q, prefix, scale, out, lse, wait_limit)
        dev, dtype, D = self.device, self.dtype, self.head_dim
        n = q.shape[0]
        qa = _head_rows(q, "q", dtype, dev, n, D)
        if out is None:
            out = q.new_empty(q.shape)
        oa = _head_rows(out, "out", dtype, dev, n, D)
        if oa[2] != qa[2]:
            raise ValueError("out must have q's heads")
        if lse is not None and not (lse.dtype is self._torch.float32 and lse.shape == q.shape[:2] and lse.is_contiguous() and lse.device == dev):
            raise ValueError("lse must be contiguous fp32 [rows, heads] on the rows' device")
        tp, ts, n_seq, table = self._table(table, "table")
        if prefix is not None:
            pp, ps, groups, ptable = self._table(prefix[0], "prefix table")
            pl, cg = self._ints(prefix[1], "prefix lengths", groups), self._ints(prefix[2], "cu_group", groups + 1)
        else:
            pp, ps, groups, ptable, pl, cg = None, 0, 0, None, None, None
        a = dart_attend_args(qa[0], oa[0], lse.data_ptr() if lse is not None else None, qa[1], oa[1], n, qa[2], n_seq, groups,
                             self._ints(cu_q, "cu_q", n_seq + 1), tp, self._ints(kv_len, "kv_len", n_seq), cg, pp, pl, ts, ps,
                             D ** -0.5 if scale is None else scale, wait_limit, self._status_at)
        L = lib()
        # (made for this call on its stream: the allocator keeps it apart from other streams' and graphs' calls)
        need = L.dart_attend_workspace(self._c, a)
        ws = self._torch.empty(need, dtype=self._torch.uint8, device=dev) if need else None
        with self._lock:
            rc = L.dart_attend(self._c, a, ws.data_ptr() if need else None, need, _raw_stream(self._index))
        if rc != DART_OK:
            raise DartError(rc, "dart_attend")
        return out

    def status(self) -> int:
        """DART_OK, or what a kernel found wrong since the last reading (a page or an index out of range, a wait that gave up), in any call
        and on any stream: the caller tells them apart by reading in between.  Waits for the device; reading clears it, and calls of other threads
        wait until it has (replays of captured graphs do not: read between them)."""
        with self._lock:
            self._torch.cuda.synchronize(self.device)
            code = int(self._status[0].item())
            if code:
                self._status.zero_()
                self._torch.cuda.synchronize(self.device)  # (before a call on another stream reports)
        return code

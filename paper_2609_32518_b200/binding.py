"""Binding of libunstep.so: same names as the C ABI, argument marshalling only.

A call goes through the native marshalling module (csrc/marshal.cpp) when all its arguments have
exactly the expected form; the module answers None for anything else, before anything is launched,
and the general path in ctypes takes over and raises what there is to raise.  Where the module cannot
be built or loaded (no host compiler, no headers), every call takes the general path."""

from __future__ import annotations

import ctypes
from ctypes import c_char_p, c_double, c_float, c_int, c_int32, c_int64, c_void_p, POINTER

from . import build as _build

EXPORTS = ("unstep_rope_table", "unstep_rope_kv_append", "unstep_window_attn",
           "unstep_window_attn_noalloc", "unstep_rope_kv_append_sink", "unstep_window_attn_sink",
           "unstep_rmsnorm_rope_kv_append", "unstep_window_attn_plan", "unstep_window_attn_plan_clusters",
           "unstep_rotary_table", "unstep_rotary_apply", "unstep_rotary_kv_append_q8", "unstep_kv_read_q8",
           "unstep_window_attn_q8", "unstep_window_attn_q8_way", "unstep_attn_workers", "unstep_attn_clusters",
           "unstep_selftest_wait_limit", "unstep_shutdown", "unstep_strerror", "unstep_poll_status", "unstep_launch_count")


class UnstepError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {strerror(code)} ({code})")


class Shape(ctypes.Structure):
    """Mirror of unstep_shape_t."""
    _fields_ = [("batch", c_int32), ("heads", c_int32), ("head_dim", c_int32),
                ("chunk_frames", c_int32), ("grid_h", c_int32), ("grid_w", c_int32),
                ("ring_frames", c_int32), ("band_t", c_int32), ("band_h", c_int32),
                ("band_w", c_int32), ("rope_base", c_double)]

    @classmethod
    def make(cls, batch, heads, chunk_frames, grid_h, grid_w, ring_frames, head_dim=128,
             bands=(44, 42, 42), rope_base=10000.0):
        return cls(batch, heads, head_dim, chunk_frames, grid_h, grid_w, ring_frames,
                   bands[0], bands[1], bands[2], rope_base)

    @property
    def tokens_per_frame(self):
        return self.grid_h * self.grid_w

    @property
    def chunk_tokens(self):
        return self.chunk_frames * self.grid_h * self.grid_w

    @property
    def rotated_dims(self):
        return self.band_t + self.band_h + self.band_w


class Rope(ctypes.Structure):
    """Mirror of unstep_rope_t: layout and scaling of a model's rotary positions.  The axes are (frame, row, column)."""
    _fields_ = [("half", c_int32), ("trained", c_int32 * 3), ("factor", c_double * 3), ("beta_slow", c_double),
                ("beta_fast", c_double), ("magnitude", c_double)]

    @classmethod
    def make(cls, half=False, factor=(1.0, 1.0, 1.0), trained=(0, 0, 0), beta=(1.0, 32.0), magnitude=1.0):
        return cls(int(half), (c_int32 * 3)(*trained), (c_double * 3)(*factor), beta[0], beta[1], magnitude)


_lib = None
_fast = None   # the native marshalling module, bound to the functions of _lib, or a _NoMarshal


class _NoMarshal:
    """Stands in for the marshalling module: no call is of its form."""

    def __getattr__(self, name):
        return lambda *args: None


def lib() -> ctypes.CDLL:
    """Load (building first if stale) the CUDA library; raises if that is impossible."""
    global _lib
    if _lib is None:
        import os
        path = _build.build(variant=os.environ.get("UNSTEP_LIB_VARIANT", ""))
        L = ctypes.CDLL(path)
        L.unstep_rope_table.restype = c_int
        L.unstep_rope_table.argtypes = [POINTER(Shape), c_int32, c_void_p, c_void_p, c_void_p]
        L.unstep_rope_kv_append.restype = c_int
        L.unstep_rope_kv_append.argtypes = [POINTER(Shape), POINTER(c_int32), c_void_p, c_void_p,
                                            c_void_p, c_void_p, c_void_p, c_int64, c_void_p,
                                            c_void_p, c_void_p, c_void_p]
        L.unstep_window_attn.restype = c_int
        L.unstep_window_attn.argtypes = [POINTER(Shape), POINTER(c_int32), c_int32, c_void_p,
                                         c_void_p, c_void_p, c_void_p, c_void_p]
        L.unstep_window_attn_noalloc.restype = c_int
        L.unstep_window_attn_noalloc.argtypes = L.unstep_window_attn.argtypes
        L.unstep_rope_kv_append_sink.restype = c_int
        L.unstep_rope_kv_append_sink.argtypes = [POINTER(Shape), c_int32, POINTER(c_int32), c_void_p,
                                                 c_void_p, c_void_p, c_void_p, c_void_p, c_int64,
                                                 c_void_p, c_void_p, c_void_p, c_void_p]
        L.unstep_window_attn_sink.restype = c_int
        L.unstep_window_attn_sink.argtypes = [POINTER(Shape), c_int32, POINTER(c_int32), c_int32, c_int32,
                                              c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]
        L.unstep_rmsnorm_rope_kv_append.restype = c_int
        L.unstep_rmsnorm_rope_kv_append.argtypes = [POINTER(Shape), c_int32, POINTER(c_int32), c_void_p,
                                                    c_void_p, c_void_p, c_void_p, c_void_p, c_float,
                                                    c_void_p, c_void_p, c_int64, c_void_p, c_void_p,
                                                    c_void_p, c_void_p]
        L.unstep_window_attn_plan.restype = c_int
        L.unstep_window_attn_plan.argtypes = [POINTER(Shape), c_int32, POINTER(c_int32), c_int32, c_int32,
                                              c_int32, POINTER(c_int32), c_int32, POINTER(c_int32)]
        L.unstep_window_attn_plan_clusters.restype = c_int
        L.unstep_window_attn_plan_clusters.argtypes = [POINTER(Shape), c_int32, POINTER(c_int32), c_int32, c_int32,
                                                       c_int32, POINTER(c_int32), POINTER(c_int32), c_int32,
                                                       POINTER(c_int32)]
        L.unstep_rotary_table.restype = c_int
        L.unstep_rotary_table.argtypes = [POINTER(Shape), POINTER(Rope), c_int32, c_void_p, c_void_p, c_void_p]
        L.unstep_rotary_apply.restype = c_int
        L.unstep_rotary_apply.argtypes = [POINTER(Shape), POINTER(Rope), c_int32, c_void_p, c_void_p, c_void_p,
                                          c_int64, c_void_p, c_void_p]
        L.unstep_rotary_kv_append_q8.restype = c_int
        L.unstep_rotary_kv_append_q8.argtypes = [POINTER(Shape), POINTER(Rope), c_int32, POINTER(c_int32)] + \
            [c_void_p] * 5 + [c_float, c_void_p, c_void_p, c_int64] + [c_void_p] * 6
        L.unstep_kv_read_q8.restype = c_int
        L.unstep_kv_read_q8.argtypes = [POINTER(Shape), c_int32, POINTER(c_int32), c_int32] + [c_void_p] * 7
        L.unstep_window_attn_q8.restype = c_int
        L.unstep_window_attn_q8.argtypes = [POINTER(Shape), c_int32, POINTER(c_int32), c_int32, c_int32] + \
            [c_void_p] * 7
        L.unstep_window_attn_q8_way.restype = c_int
        L.unstep_window_attn_q8_way.argtypes = [POINTER(Shape), c_int32, POINTER(c_int32), c_int32, c_int32, c_int32,
                                                POINTER(c_int32)]
        L.unstep_attn_clusters.restype = c_int
        L.unstep_attn_clusters.argtypes = [POINTER(c_int32)]
        L.unstep_attn_workers.restype = c_int
        L.unstep_attn_workers.argtypes = [POINTER(c_int32), POINTER(c_int32)]
        L.unstep_selftest_wait_limit.restype = c_int
        L.unstep_selftest_wait_limit.argtypes = [c_int64, c_void_p]
        L.unstep_shutdown.restype = None
        L.unstep_shutdown.argtypes = []
        L.unstep_strerror.restype = c_char_p
        L.unstep_strerror.argtypes = [c_int]
        L.unstep_poll_status.restype = c_int
        L.unstep_poll_status.argtypes = []
        L.unstep_launch_count.restype = c_int64
        L.unstep_launch_count.argtypes = []
        _lib = L
    return _lib


def _native():
    global _fast
    if _fast is None:
        L = lib()
        try:
            mod = _build.load_marshal()
        except (ImportError, OSError, RuntimeError) as e:
            import warnings
            warnings.warn(f"calls are marshalled by ctypes, 8-10 us each: {e}", RuntimeWarning, stacklevel=3)
            _fast = _NoMarshal()
            return _fast
        mod.bind(Shape, Rope, *(ctypes.cast(f, c_void_p).value for f in (
            L.unstep_rope_table, L.unstep_rope_kv_append_sink, L.unstep_rmsnorm_rope_kv_append,
            L.unstep_window_attn, L.unstep_window_attn_noalloc, L.unstep_window_attn_sink, L.unstep_rotary_table,
            L.unstep_rotary_apply, L.unstep_rotary_kv_append_q8, L.unstep_kv_read_q8, L.unstep_window_attn_q8)))
        _fast = mod
    return _fast


def strerror(code: int) -> str:
    return lib().unstep_strerror(int(code)).decode()


def _stream_ptr(stream):
    if stream is None:
        import torch
        stream = torch.cuda.current_stream()
    return c_void_p(int(getattr(stream, "cuda_stream", stream)))


def _dev_ptr(t, dtype, numel, name):
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name}: expected a CUDA tensor")
    if t.dtype != dtype or not t.is_contiguous() or t.numel() != numel:
        raise ValueError(f"{name}: expected contiguous {dtype} with {numel} elements, got "
                         f"{t.dtype} {tuple(t.shape)}")
    return c_void_p(t.data_ptr())


def _here_ptr(t, dtype, numel, name):
    """_dev_ptr of a tensor on the current device, where the call is enqueued."""
    import torch
    ptr = _dev_ptr(t, dtype, numel, name)
    if t.device.index != torch.cuda.current_device():
        raise ValueError(f"{name}: on {t.device}, the current device is cuda:{torch.cuda.current_device()}")
    return ptr


def _starts(shape: Shape, start_frame):
    vals = [int(s) for s in start_frame]
    if len(vals) != shape.batch:
        raise ValueError("start_frame needs one entry per stream")
    return (c_int32 * len(vals))(*vals)


def _check(rc: int, where: str):
    if rc != 0:
        raise UnstepError(rc, where)


def rope_table(shape: Shape, start_frame: int, cos, sin, stream=None):
    """unstep_rope_table: fill float32 cos/sin [L, 64] for the chunk starting at start_frame."""
    rc = (_fast or _native()).rope_table(
        shape, start_frame, cos, sin, stream)
    if rc is None:
        _general_rope_table(shape, start_frame, cos, sin, stream)
    elif rc:
        raise UnstepError(rc, "unstep_rope_table")


def _general_rope_table(shape, start_frame, cos, sin, stream):
    import torch
    n = shape.chunk_tokens * 64
    _check(lib().unstep_rope_table(ctypes.byref(shape), int(start_frame),
                                   _dev_ptr(cos, torch.float32, n, "cos"),
                                   _dev_ptr(sin, torch.float32, n, "sin"), _stream_ptr(stream)),
           "unstep_rope_table")


def rope_kv_append(shape: Shape, start_frame, q_in, k_in, v_in, cos, sin, q_out, ring_k, ring_v,
                   table_stream_stride: int = 0, stream=None):
    """unstep_rope_kv_append: rotate q/k, write k/v of the chunk into ring slots."""
    rc = (_fast or _native()).append(
        shape, 0, start_frame, q_in, k_in, v_in, cos, sin, q_out, ring_k, ring_v, table_stream_stride, stream)
    if rc is None:
        _general_rope_kv_append(shape, start_frame, q_in, k_in, v_in, cos, sin, q_out, ring_k, ring_v,
                                table_stream_stride, stream)
    elif rc:
        raise UnstepError(rc, "unstep_rope_kv_append")


def _general_rope_kv_append(shape, start_frame, q_in, k_in, v_in, cos, sin, q_out, ring_k, ring_v,
                            table_stream_stride, stream):
    import torch
    bf = torch.bfloat16
    n = shape.batch * shape.chunk_tokens * shape.heads * shape.head_dim
    nr = shape.batch * shape.ring_frames * shape.tokens_per_frame * shape.heads * shape.head_dim
    ntab = shape.chunk_tokens * 64 + (shape.batch - 1) * int(table_stream_stride)
    _check(lib().unstep_rope_kv_append(
        ctypes.byref(shape), _starts(shape, start_frame), _dev_ptr(q_in, bf, n, "q_in"),
        _dev_ptr(k_in, bf, n, "k_in"), _dev_ptr(v_in, bf, n, "v_in"),
        _dev_ptr(cos, torch.float32, ntab, "cos"), _dev_ptr(sin, torch.float32, ntab, "sin"),
        int(table_stream_stride), _dev_ptr(q_out, bf, n, "q_out"),
        _dev_ptr(ring_k, bf, nr, "ring_k"), _dev_ptr(ring_v, bf, nr, "ring_v"),
        _stream_ptr(stream)), "unstep_rope_kv_append")


def window_attn(shape: Shape, start_frame, window_frames: int, q_rot, ring_k, ring_v, out,
                stream=None):
    """unstep_window_attn: attention of the chunk's queries over the retained window."""
    rc = (_fast or _native()).attn(
        shape, start_frame, window_frames, q_rot, ring_k, ring_v, out, stream)
    if rc is None:
        _general_window_attn(shape, start_frame, window_frames, q_rot, ring_k, ring_v, out, stream)
    elif rc:
        raise UnstepError(rc, "unstep_window_attn")


def _general_window_attn(shape, start_frame, window_frames, q_rot, ring_k, ring_v, out, stream):
    import torch
    bf = torch.bfloat16
    n = shape.batch * shape.chunk_tokens * shape.heads * shape.head_dim
    nr = shape.batch * shape.ring_frames * shape.tokens_per_frame * shape.heads * shape.head_dim
    _check(lib().unstep_window_attn(
        ctypes.byref(shape), _starts(shape, start_frame), int(window_frames),
        _dev_ptr(q_rot, bf, n, "q_rot"), _dev_ptr(ring_k, bf, nr, "ring_k"),
        _dev_ptr(ring_v, bf, nr, "ring_v"), _dev_ptr(out, bf, n, "out"), _stream_ptr(stream)),
        "unstep_window_attn")


def window_attn_noalloc(shape: Shape, start_frame, window_frames: int, q_rot, ring_k, ring_v, out,
                        stream=None):
    """unstep_window_attn_noalloc: the same attention for callers that must not allocate device
    memory (a process whose memory is owned by a framework allocator, a latency-critical loop,
    a deployment with a fixed footprint).  Its scratch is a fixed ~40 MB array inside the
    library; all calls on a device share it, so calls that may overlap on the GPU must be
    serialised by the caller.  Raises UnstepError(-5) when the problem exceeds the array."""
    rc = (_fast or _native()).attn_noalloc(
        shape, start_frame, window_frames, q_rot, ring_k, ring_v, out, stream)
    if rc is None:
        _general_window_attn_noalloc(shape, start_frame, window_frames, q_rot, ring_k, ring_v, out, stream)
    elif rc:
        raise UnstepError(rc, "unstep_window_attn_noalloc")


def _general_window_attn_noalloc(shape, start_frame, window_frames, q_rot, ring_k, ring_v, out, stream):
    import torch
    bf = torch.bfloat16
    n = shape.batch * shape.chunk_tokens * shape.heads * shape.head_dim
    nr = shape.batch * shape.ring_frames * shape.tokens_per_frame * shape.heads * shape.head_dim
    _check(lib().unstep_window_attn_noalloc(
        ctypes.byref(shape), _starts(shape, start_frame), int(window_frames),
        _dev_ptr(q_rot, bf, n, "q_rot"), _dev_ptr(ring_k, bf, nr, "ring_k"),
        _dev_ptr(ring_v, bf, nr, "ring_v"), _dev_ptr(out, bf, n, "out"), _stream_ptr(stream)),
        "unstep_window_attn_noalloc")


def rope_kv_append_sink(shape: Shape, sink_frames: int, start_frame, q_in, k_in, v_in, cos, sin, q_out,
                        cache_k, cache_v, table_stream_stride: int = 0, stream=None):
    """unstep_rope_kv_append_sink: the append with a sink prefix of `sink_frames` slots."""
    rc = (_fast or _native()).append(
        shape, sink_frames, start_frame, q_in, k_in, v_in, cos, sin, q_out, cache_k, cache_v,
        table_stream_stride, stream)
    if rc is None:
        _general_rope_kv_append_sink(shape, sink_frames, start_frame, q_in, k_in, v_in, cos, sin, q_out,
                                     cache_k, cache_v, table_stream_stride, stream)
    elif rc:
        raise UnstepError(rc, "unstep_rope_kv_append_sink")


def _general_rope_kv_append_sink(shape, sink_frames, start_frame, q_in, k_in, v_in, cos, sin, q_out, cache_k,
                                 cache_v, table_stream_stride, stream):
    import torch
    bf = torch.bfloat16
    n = shape.batch * shape.chunk_tokens * shape.heads * shape.head_dim
    nr = (shape.batch * (shape.ring_frames + int(sink_frames)) * shape.tokens_per_frame * shape.heads
          * shape.head_dim)
    ntab = shape.chunk_tokens * 64 + (shape.batch - 1) * int(table_stream_stride)
    _check(lib().unstep_rope_kv_append_sink(
        ctypes.byref(shape), int(sink_frames), _starts(shape, start_frame),
        _dev_ptr(q_in, bf, n, "q_in"), _dev_ptr(k_in, bf, n, "k_in"), _dev_ptr(v_in, bf, n, "v_in"),
        _dev_ptr(cos, torch.float32, ntab, "cos"), _dev_ptr(sin, torch.float32, ntab, "sin"),
        int(table_stream_stride), _dev_ptr(q_out, bf, n, "q_out"), _dev_ptr(cache_k, bf, nr, "cache_k"),
        _dev_ptr(cache_v, bf, nr, "cache_v"), _stream_ptr(stream)), "unstep_rope_kv_append_sink")


def rmsnorm_rope_kv_append(shape: Shape, sink_frames: int, start_frame, q_in, k_in, v_in, gain_q, gain_k,
                           eps: float, cos, sin, q_out, cache_k, cache_v, table_stream_stride: int = 0,
                           stream=None):
    """unstep_rmsnorm_rope_kv_append: RMSNorm of q and k, rotation and cache write in one kernel."""
    rc = (_fast or _native()).norm_append(
        shape, sink_frames, start_frame, q_in, k_in, v_in, gain_q, gain_k, eps, cos, sin, q_out, cache_k,
        cache_v, table_stream_stride, stream)
    if rc is None:
        _general_rmsnorm_rope_kv_append(shape, sink_frames, start_frame, q_in, k_in, v_in, gain_q, gain_k,
                                        eps, cos, sin, q_out, cache_k, cache_v, table_stream_stride, stream)
    elif rc:
        raise UnstepError(rc, "unstep_rmsnorm_rope_kv_append")


def _general_rmsnorm_rope_kv_append(shape, sink_frames, start_frame, q_in, k_in, v_in, gain_q, gain_k, eps,
                                    cos, sin, q_out, cache_k, cache_v, table_stream_stride, stream):
    import torch
    bf = torch.bfloat16
    n = shape.batch * shape.chunk_tokens * shape.heads * shape.head_dim
    nr = (shape.batch * (shape.ring_frames + int(sink_frames)) * shape.tokens_per_frame * shape.heads
          * shape.head_dim)
    ntab = shape.chunk_tokens * 64 + (shape.batch - 1) * int(table_stream_stride)
    ng = shape.heads * shape.head_dim
    _check(lib().unstep_rmsnorm_rope_kv_append(
        ctypes.byref(shape), int(sink_frames), _starts(shape, start_frame),
        _dev_ptr(q_in, bf, n, "q_in"), _dev_ptr(k_in, bf, n, "k_in"), _dev_ptr(v_in, bf, n, "v_in"),
        _dev_ptr(gain_q, torch.float32, ng, "gain_q"), _dev_ptr(gain_k, torch.float32, ng, "gain_k"),
        c_float(eps), _dev_ptr(cos, torch.float32, ntab, "cos"), _dev_ptr(sin, torch.float32, ntab, "sin"),
        int(table_stream_stride), _dev_ptr(q_out, bf, n, "q_out"), _dev_ptr(cache_k, bf, nr, "cache_k"),
        _dev_ptr(cache_v, bf, nr, "cache_v"), _stream_ptr(stream)), "unstep_rmsnorm_rope_kv_append")


def window_attn_sink(shape: Shape, sink_frames: int, start_frame, recent_frames: int, sink_attend: int,
                     q_rot, cache_k, cache_v, out, stream=None):
    """unstep_window_attn_sink: attention over sink frames + the recent window."""
    rc = (_fast or _native()).attn_sink(
        shape, sink_frames, start_frame, recent_frames, sink_attend, q_rot, cache_k, cache_v, out, stream)
    if rc is None:
        _general_window_attn_sink(shape, sink_frames, start_frame, recent_frames, sink_attend, q_rot, cache_k,
                                  cache_v, out, stream)
    elif rc:
        raise UnstepError(rc, "unstep_window_attn_sink")


def _general_window_attn_sink(shape, sink_frames, start_frame, recent_frames, sink_attend, q_rot, cache_k,
                              cache_v, out, stream):
    import torch
    bf = torch.bfloat16
    n = shape.batch * shape.chunk_tokens * shape.heads * shape.head_dim
    nr = (shape.batch * (shape.ring_frames + int(sink_frames)) * shape.tokens_per_frame * shape.heads
          * shape.head_dim)
    _check(lib().unstep_window_attn_sink(
        ctypes.byref(shape), int(sink_frames), _starts(shape, start_frame), int(recent_frames),
        int(sink_attend), _dev_ptr(q_rot, bf, n, "q_rot"), _dev_ptr(cache_k, bf, nr, "cache_k"),
        _dev_ptr(cache_v, bf, nr, "cache_v"), _dev_ptr(out, bf, n, "out"), _stream_ptr(stream)),
        "unstep_window_attn_sink")


def rotary_table(shape: Shape, rope: Rope, start_frame: int, cos, sin, stream=None):
    """unstep_rotary_table: fill float32 cos/sin [L, R/2] for the chunk starting at start_frame, R the dims that the
    bands of the shape rotate."""
    rc = (_fast or _native()).rotary_table(shape, rope, start_frame, cos, sin, stream)
    if rc is None:
        _general_rotary_table(shape, rope, start_frame, cos, sin, stream)
    elif rc:
        raise UnstepError(rc, "unstep_rotary_table")


def _rope(rope):
    if not isinstance(rope, Rope):
        raise TypeError("rope: expected a Rope")
    return ctypes.byref(rope)


def _general_rotary_table(shape, rope, start_frame, cos, sin, stream):
    import torch
    n = shape.chunk_tokens * (shape.rotated_dims // 2)
    _check(lib().unstep_rotary_table(ctypes.byref(shape), _rope(rope), int(start_frame),
                                     _here_ptr(cos, torch.float32, n, "cos"),
                                     _here_ptr(sin, torch.float32, n, "sin"), _stream_ptr(stream)),
           "unstep_rotary_table")


def _rotary_table_numel(shape, table_stream_stride):
    return shape.chunk_tokens * (shape.rotated_dims // 2) + (shape.batch - 1) * int(table_stream_stride)


def rotary_apply(shape: Shape, rope: Rope, x, cos, sin, y, transposed: bool = False, table_stream_stride: int = 0,
                 stream=None):
    """unstep_rotary_apply: rotate x [B, L, Hn, 128] into y; transposed: its backward pass."""
    rc = (_fast or _native()).rotary_apply(shape, rope, x, cos, sin, y, transposed, table_stream_stride, stream)
    if rc is None:
        _general_rotary_apply(shape, rope, x, cos, sin, y, transposed, table_stream_stride, stream)
    elif rc:
        raise UnstepError(rc, "unstep_rotary_apply")


def _general_rotary_apply(shape, rope, x, cos, sin, y, transposed, table_stream_stride, stream):
    import torch
    n = shape.batch * shape.chunk_tokens * shape.heads * shape.head_dim
    ntab = _rotary_table_numel(shape, table_stream_stride)
    _check(lib().unstep_rotary_apply(
        ctypes.byref(shape), _rope(rope), int(bool(transposed)), _here_ptr(x, torch.bfloat16, n, "x"),
        _here_ptr(cos, torch.float32, ntab, "cos"), _here_ptr(sin, torch.float32, ntab, "sin"),
        int(table_stream_stride), _here_ptr(y, torch.bfloat16, n, "y"), _stream_ptr(stream)), "unstep_rotary_apply")


def _cache8_ptrs(shape, sink_frames, cache_k, scale_k, cache_v, scale_v):
    import torch
    n = (shape.batch * (shape.ring_frames + int(sink_frames)) * shape.tokens_per_frame * shape.heads
         * shape.head_dim)
    codes, scales = torch.float8_e4m3fn, torch.float8_e8m0fnu
    return (_here_ptr(cache_k, codes, n, "cache_k"), _here_ptr(scale_k, scales, n // 32, "scale_k"),
            _here_ptr(cache_v, codes, n, "cache_v"), _here_ptr(scale_v, scales, n // 32, "scale_v"))


def rotary_kv_append_q8(shape: Shape, rope: Rope, sink_frames: int, start_frame, q_in, k_in, v_in, cos, sin, q_out,
                        cache_k, scale_k, cache_v, scale_v, gain_q=None, gain_k=None, eps: float = 0.0,
                        table_stream_stride: int = 0, stream=None):
    """unstep_rotary_kv_append_q8: (RMSNorm and) rotation of q and k, k and v quantised into the cache.  cache_k,
    cache_v: float8_e4m3fn [B, sink + C, T, Hn, 128], scale_k, scale_v: float8_e8m0fnu [B, sink + C, T, Hn, 4]."""
    rc = (_fast or _native()).append_q8(
        shape, rope, sink_frames, start_frame, q_in, k_in, v_in, cos, sin, q_out, cache_k, scale_k, cache_v, scale_v,
        gain_q, gain_k, eps, table_stream_stride, stream)
    if rc is None:
        _general_rotary_kv_append_q8(shape, rope, sink_frames, start_frame, q_in, k_in, v_in, cos, sin, q_out, cache_k,
                                     scale_k, cache_v, scale_v, gain_q, gain_k, eps, table_stream_stride, stream)
    elif rc:
        raise UnstepError(rc, "unstep_rotary_kv_append_q8")


def _general_rotary_kv_append_q8(shape, rope, sink_frames, start_frame, q_in, k_in, v_in, cos, sin, q_out, cache_k,
                                 scale_k, cache_v, scale_v, gain_q, gain_k, eps, table_stream_stride, stream):
    import torch
    bf = torch.bfloat16
    n = shape.batch * shape.chunk_tokens * shape.heads * shape.head_dim
    ntab = _rotary_table_numel(shape, table_stream_stride)
    ng = shape.heads * shape.head_dim
    gains = [None if g is None else _here_ptr(g, torch.float32, ng, name)
             for g, name in ((gain_q, "gain_q"), (gain_k, "gain_k"))]
    _check(lib().unstep_rotary_kv_append_q8(
        ctypes.byref(shape), _rope(rope), int(sink_frames), _starts(shape, start_frame),
        _here_ptr(q_in, bf, n, "q_in"), _here_ptr(k_in, bf, n, "k_in"), _here_ptr(v_in, bf, n, "v_in"), *gains,
        c_float(eps), _here_ptr(cos, torch.float32, ntab, "cos"), _here_ptr(sin, torch.float32, ntab, "sin"),
        int(table_stream_stride), _here_ptr(q_out, bf, n, "q_out"),
        *_cache8_ptrs(shape, sink_frames, cache_k, scale_k, cache_v, scale_v), _stream_ptr(stream)),
        "unstep_rotary_kv_append_q8")


def kv_read_q8(shape: Shape, sink_frames: int, first_frame, n_frames: int, cache_k, scale_k, cache_v, scale_v, out_k,
               out_v, stream=None):
    """unstep_kv_read_q8: frames [first_frame[b], first_frame[b] + n_frames) of an 8-bit cache as bf16
    [B, n_frames, T, Hn, 128]."""
    rc = (_fast or _native()).read_q8(
        shape, sink_frames, first_frame, n_frames, cache_k, scale_k, cache_v, scale_v, out_k, out_v, stream)
    if rc is None:
        _general_kv_read_q8(shape, sink_frames, first_frame, n_frames, cache_k, scale_k, cache_v, scale_v, out_k, out_v,
                            stream)
    elif rc:
        raise UnstepError(rc, "unstep_kv_read_q8")


def _general_kv_read_q8(shape, sink_frames, first_frame, n_frames, cache_k, scale_k, cache_v, scale_v, out_k, out_v,
                        stream):
    import torch
    n = shape.batch * int(n_frames) * shape.tokens_per_frame * shape.heads * shape.head_dim
    _check(lib().unstep_kv_read_q8(
        ctypes.byref(shape), int(sink_frames), _starts(shape, first_frame), int(n_frames),
        *_cache8_ptrs(shape, sink_frames, cache_k, scale_k, cache_v, scale_v),
        _here_ptr(out_k, torch.bfloat16, n, "out_k"), _here_ptr(out_v, torch.bfloat16, n, "out_v"),
        _stream_ptr(stream)), "unstep_kv_read_q8")


def window_attn_q8(shape: Shape, sink_frames: int, start_frame, recent_frames: int, sink_attend: int, q_rot, cache_k,
                   scale_k, cache_v, scale_v, out, stream=None):
    """unstep_window_attn_q8: attention over sink frames + the recent window of an 8-bit cache."""
    rc = (_fast or _native()).attn_q8(
        shape, sink_frames, start_frame, recent_frames, sink_attend, q_rot, cache_k, scale_k, cache_v, scale_v, out,
        stream)
    if rc is None:
        _general_window_attn_q8(shape, sink_frames, start_frame, recent_frames, sink_attend, q_rot, cache_k, scale_k,
                                cache_v, scale_v, out, stream)
    elif rc:
        raise UnstepError(rc, "unstep_window_attn_q8")


def _general_window_attn_q8(shape, sink_frames, start_frame, recent_frames, sink_attend, q_rot, cache_k, scale_k,
                            cache_v, scale_v, out, stream):
    import torch
    bf = torch.bfloat16
    n = shape.batch * shape.chunk_tokens * shape.heads * shape.head_dim
    _check(lib().unstep_window_attn_q8(
        ctypes.byref(shape), int(sink_frames), _starts(shape, start_frame), int(recent_frames), int(sink_attend),
        _here_ptr(q_rot, bf, n, "q_rot"), *_cache8_ptrs(shape, sink_frames, cache_k, scale_k, cache_v, scale_v),
        _here_ptr(out, bf, n, "out"), _stream_ptr(stream)), "unstep_window_attn_q8")


def window_attn_q8_way(shape: Shape, sink_frames: int, start_frame, recent_frames: int, sink_attend: int,
                       max_workers: int) -> str:
    """unstep_window_attn_q8_way: how window_attn_q8 is run on a device of max_workers SMs: "few", "tiles" or
    "unpacked" (as "tiles" where the buffer for that cannot be made or does not hold the window of a head).  Host only."""
    way = c_int32(-1)
    _check(lib().unstep_window_attn_q8_way(ctypes.byref(shape), int(sink_frames), _starts(shape, start_frame),
                                           int(recent_frames), int(sink_attend), int(max_workers), ctypes.byref(way)),
           "unstep_window_attn_q8_way")
    return ("few", "tiles", "unpacked")[way.value]


def window_attn_plan(shape: Shape, start_frame, recent_frames: int, max_workers: int, sink_frames: int = 0,
                     sink_attend: int = 0, clusters=None):
    """unstep_window_attn_plan_clusters: the segments of one attention launch as rows of 10 ints (worker,
    stream, head, query pair, query tiles, first key tile, end key tile, tiles of the item, parts, scratch
    slot, -1 for a whole item or a part of a cluster).  `clusters`: the limits as attn_clusters() returns
    them, None for a device that runs no clusters.  Host only."""
    n = c_int32(0)
    starts = _starts(shape, start_frame)
    if clusters is not None:
        if len(clusters) != 9:
            raise ValueError("clusters needs 9 entries")
        clusters = (c_int32 * 9)(*clusters)
    args = (ctypes.byref(shape), int(sink_frames), starts, int(recent_frames), int(sink_attend),
            int(max_workers), clusters)
    where = "unstep_window_attn_plan_clusters"
    _check(lib().unstep_window_attn_plan_clusters(*args, None, 0, ctypes.byref(n)), where)
    buf = (c_int32 * (10 * max(n.value, 1)))()
    _check(lib().unstep_window_attn_plan_clusters(*args, buf, n.value, ctypes.byref(n)), where)
    return [tuple(buf[10 * i:10 * i + 10]) for i in range(n.value)]


def attn_workers():
    """unstep_attn_workers: (workers of a full-size attention launch, thread blocks per worker)."""
    a, b = c_int32(0), c_int32(0)
    _check(lib().unstep_attn_workers(ctypes.byref(a), ctypes.byref(b)), "unstep_attn_workers")
    return a.value, b.value


def attn_clusters():
    """unstep_attn_clusters: how many clusters of n blocks of the attention over a bf16 cache run at the same time, at
    index n (2 .. 8)."""
    buf = (c_int32 * 9)()
    _check(lib().unstep_attn_clusters(buf), "unstep_attn_clusters")
    return list(buf)


def selftest_wait_limit(limit_cycles: int, stream=None):
    """unstep_selftest_wait_limit: make a bounded device-side wait run out (diagnostic)."""
    _check(lib().unstep_selftest_wait_limit(int(limit_cycles), _stream_ptr(stream)),
           "unstep_selftest_wait_limit")


def shutdown():
    """unstep_shutdown: free the scratch buffers the attention calls created."""
    lib().unstep_shutdown()


def poll_status() -> int:
    return int(lib().unstep_poll_status())


def launch_count() -> int:
    return int(lib().unstep_launch_count())

"""Python binding of libhs (checkpoint-aligned restore-and-resume, sm_103a).

Argument marshalling only: every function forwards to the C entry point of
the same name in ``libhs.so`` (declared in ``include/hs.h``, ``include/hs_attn.h`` and ``include/hs_kv8.h``); all GPU
work
runs in the library's kernels.  Tensors are accepted wherever the C call
takes a pointer (their ``data_ptr()`` is passed); plain ints are passed as
addresses.  A non-OK status raises ``HsError``.

The library is built in-tree by ``paper_2609_15030_gb300.build.build()``.
If ``libhs.so`` is missing, every call raises: there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import os
import threading
from array import array

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libhs.so")

HS_OK = 0
HS_ERR_INVALID_ARG = 1
HS_ERR_MISALIGNED = 2
HS_ERR_UNSUPPORTED = 3
HS_ERR_CUDA = 4
HS_ERR_DEVICE_CHECK = 5
HS_ERR_TOO_LARGE = 6

HS_DEVERR_NONE = 0
HS_DEVERR_BLOCK_OOB = 1
HS_DEVERR_MISALIGNED = 2
HS_DEVERR_NULL = 3
HS_DEVERR_TIMEOUT = 4
HS_DEVERR_LENGTH = 5

HS_MAX_BATCH = 384
HS_CHUNK = 64
HS_SHORT_SEGMENT = 8
HS_NOALLOC_SCRATCH_BYTES = 16 << 20

HS_LINATTN_AUTO = 0
HS_LINATTN_RECURRENT = 1
HS_LINATTN_CHUNKED_TC = 2
HS_LINATTN_SINGLE_TOKEN = 3

HS_BF16 = 0
HS_FP16 = 1

HS_KV8_GROUP = 16
HS_ROPE_HALF = 0
HS_ROPE_INTERLEAVED = 1
HS_ROPE_PLAIN = 0
HS_ROPE_LINEAR = 1
HS_ROPE_BASE = 2
HS_ROPE_TURNS = 3
HS_ROPE_INDEX = 4
HS_ROPE_MAX_PAIRS = 64

EXPORTED = ("hs_status_string", "hs_version", "hs_align_prefix", "hs_restore_kv_pages",
            "hs_save_kv_pages", "hs_restore_kv_page_slices", "hs_save_kv_page_slices",
            "hs_restore_state", "hs_checkpoint_states", "hs_linattn_prefill_from_state",
            "hs_linattn_num_checkpoints", "hs_linattn_prefill_packed", "hs_restore_request",
            "hs_test_prefill_stalled", "hs_linattn_prefill_scan", "hs_linattn_scan_workspace_bytes",
            "hs_linattn_prefill_scan_noalloc", "hs_kv_append", "hs_attn_prefill",
            "hs_attn_prefill_workspace_bytes", "hs_attn_decode", "hs_attn_decode_workspace_bytes",
            "hs_attn_decode_shared", "hs_attn_decode_shared_workspace_bytes",
            "hs_test_attn_stalled", "hs_rope_plan", "hs_rope_apply", "hs_kv8_block_bytes",
            "hs_kv8_append", "hs_kv8_append_rope", "hs_kv8_decode", "hs_kv8_decode_workspace_bytes",
            "hs_kv8_read", "hs_test_kv8_stalled")


class HsError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {hs_status_string(status)}")


class hs_linattn_shape(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_heads", C.c_int32), ("d_k", C.c_int32),
                ("d_v", C.c_int32), ("max_tokens", C.c_int64), ("kernel", C.c_int32),
                ("reserved", C.c_int32)]


class hs_attn_shape(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("page_size", C.c_int32), ("dtype", C.c_int32),
                ("num_blocks", C.c_int64), ("max_pages", C.c_int64), ("q_stride", C.c_int64),
                ("o_stride", C.c_int64), ("scale", C.c_float), ("unsplit", C.c_int32)]


class hs_rope(C.Structure):
    _fields_ = [("dims", C.c_int32), ("layout", C.c_int32), ("amplitude", C.c_double),
                ("theta", C.c_double * HS_ROPE_MAX_PAIRS)]


_lock = threading.Lock()
_lib = None


def load() -> C.CDLL:
    """Load libhs.so; raises if it has not been built (no fallback path exists)."""
    global _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(LIB_PATH):
                raise RuntimeError(f"{LIB_PATH} not found: build it with "
                                   "paper_2609_15030_gb300.build.build()")
            L = C.CDLL(LIB_PATH)
            vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
            L.hs_status_string.argtypes = [C.c_int]
            L.hs_status_string.restype = C.c_char_p
            L.hs_version.argtypes = []
            L.hs_version.restype = i32
            L.hs_align_prefix.argtypes = [i64, i64, vp, i32, i32, vp, vp, vp]
            L.hs_restore_kv_pages.argtypes = [vp, vp, i32, vp, i32, i64, i64, vp, vp]
            L.hs_save_kv_pages.argtypes = [vp, vp, i32, vp, i32, i64, i64, vp, vp]
            L.hs_restore_request.argtypes = [vp, vp, i32, vp, i32, i64, i64, vp, vp, i32, i64, vp, vp]
            for name in ("hs_restore_kv_page_slices", "hs_save_kv_page_slices"):
                getattr(L, name).argtypes = [vp, vp, i32, vp, i32, i64, i32, i64, i64, i64, vp, vp]
            L.hs_restore_state.argtypes = [vp, vp, i32, i64, vp, vp]
            L.hs_checkpoint_states.argtypes = [vp, vp, i32, i64, vp, vp]
            L.hs_linattn_prefill_from_state.argtypes = [C.POINTER(hs_linattn_shape), vp, vp, vp,
                                                        vp, vp, vp, vp, vp, i32, vp, vp, vp]
            L.hs_linattn_num_checkpoints.argtypes = [i32, vp, vp, i32, vp]
            L.hs_linattn_prefill_packed.argtypes = [C.POINTER(hs_linattn_shape), vp, vp, vp, vp,
                                                    vp, vp, vp, vp, vp, i32, vp, vp, vp]
            L.hs_test_prefill_stalled.argtypes = L.hs_linattn_prefill_from_state.argtypes
            L.hs_linattn_prefill_scan.argtypes = [C.POINTER(hs_linattn_shape), vp, vp, vp, vp, vp,
                                                  vp, vp, vp, i32, vp, vp, i64, vp, vp]
            L.hs_linattn_scan_workspace_bytes.argtypes = [C.POINTER(hs_linattn_shape), vp, vp, vp]
            L.hs_linattn_prefill_scan_noalloc.argtypes = [C.POINTER(hs_linattn_shape), vp, vp, vp,
                                                          vp, vp, vp, vp, vp, i32, vp, vp, vp]
            ash = C.POINTER(hs_attn_shape)
            L.hs_kv_append.argtypes = [ash, vp, vp, i64, vp, i64, vp, vp, vp]
            L.hs_attn_prefill.argtypes = [ash, vp, vp, vp, vp, vp, vp, vp, vp, vp, i64, vp, vp]
            L.hs_test_attn_stalled.argtypes = L.hs_attn_prefill.argtypes
            L.hs_attn_prefill_workspace_bytes.argtypes = [ash, vp, vp, vp]
            L.hs_attn_decode.argtypes = [ash, vp, vp, vp, vp, i64, vp, vp, vp, i64, vp, vp]
            L.hs_attn_decode_workspace_bytes.argtypes = [ash, i64, vp]
            L.hs_attn_decode_shared.argtypes = [ash, vp, vp, vp, i64, vp, vp, i64, vp, vp, vp, i64,
                                                vp, vp]
            L.hs_attn_decode_shared_workspace_bytes.argtypes = [ash, i64, i64, vp]
            rp, f64 = C.POINTER(hs_rope), C.c_double
            L.hs_rope_plan.argtypes = [i32, i32, f64, i32, f64, i64, f64, f64, f64, rp]
            L.hs_rope_apply.argtypes = [ash, rp, vp, vp, i64, vp, i64, vp, i64, vp, i64, vp]
            L.hs_kv8_block_bytes.argtypes = [ash, vp]
            L.hs_kv8_append.argtypes = L.hs_kv_append.argtypes
            L.hs_kv8_append_rope.argtypes = [ash, rp, vp, vp, vp, i64, vp, vp, i64, vp, i64, vp, vp, vp]
            L.hs_kv8_decode.argtypes = L.hs_attn_decode.argtypes
            L.hs_test_kv8_stalled.argtypes = L.hs_attn_decode.argtypes
            L.hs_kv8_decode_workspace_bytes.argtypes = [ash, i64, vp]
            L.hs_kv8_read.argtypes = [ash, vp, vp, vp, i64, vp, i64, vp, vp, vp]
            for name in EXPORTED[2:]:
                getattr(L, name).restype = C.c_int
            _lib = L
    return _lib


# Every call below is a decode step's host time: with the conversions written out per
# element (ctypes arrays from int() of each entry, the torch stream object) a call of nine
# problems spent 11 us in this module and 3.3 us in the library, launch included.

def _ptr(x):
    if x is None:
        return None
    try:
        return x.data_ptr()
    except AttributeError:
        pass
    if isinstance(x, int):
        return x
    if hasattr(x, "ctypes"):           # numpy (host arrays)
        return x.ctypes.data
    raise TypeError(f"cannot pass {type(x)} as a pointer")


def _host_array(code, ctype, values, n: int):
    """A host array of n integers (its address, and the object that owns it).  Lists and tuples
    of n integers in range go through array.array, in C; anything else (other containers,
    floats, values beyond the type, another length) through int() and ctypes as they always
    have."""
    if type(values) is list or type(values) is tuple:
        try:
            a = array(code, values)
            if len(a) == n > 0:
                return a.buffer_info()[0], a
        except (TypeError, OverflowError):
            pass
    c = (ctype * max(n, 1))(*[int(x) for x in values])
    return C.addressof(c), c


def _i64(values, n: int):
    return _host_array("q", C.c_int64, values, n)


def _i32(values, n: int):
    return _host_array("i", C.c_int32, values, n)


_current_stream = None


def _bind_current_stream():
    """The function that returns the current torch stream's handle: torch's raw-handle query
    (0.3 us) where this torch has it, else through the stream object (3 us)."""
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is None:
        return lambda: torch.cuda.current_stream().cuda_stream
    device = torch.cuda.current_device
    return lambda: raw(device())


def _stream(s):
    global _current_stream
    if s is None:
        if _current_stream is None:
            _current_stream = _bind_current_stream()
        return _current_stream()
    if isinstance(s, int):
        return s
    return s.cuda_stream


def _check(rc: int, where: str):
    if rc != HS_OK:
        raise HsError(rc, where)


def hs_status_string(status: int) -> str:
    return load().hs_status_string(int(status)).decode()


def hs_version() -> int:
    return load().hs_version()


def ptr_array(tensors, device):
    """Device int64 tensor holding the data pointers of ``tensors`` (a device pointer array)."""
    import torch
    return torch.tensor([_ptr(t) for t in tensors], dtype=torch.int64, device=device)


def hs_align_prefix(N: int, hit_len: int, avail, page_size: int):
    """Strict-prefix alignment; returns (c, n_pages, tail)."""
    av = (C.c_int64 * len(avail))(*[int(a) for a in avail]) if len(avail) else None
    c, npg, tail = C.c_int64(), C.c_int64(), C.c_int64()
    rc = (_lib or load()).hs_align_prefix(
        int(N), int(hit_len), C.cast(av, C.c_void_p) if av else None, len(avail), int(page_size),
        C.addressof(c), C.addressof(npg), C.addressof(tail))
    _check(rc, "hs_align_prefix")
    return c.value, npg.value, tail.value


def hs_restore_kv_pages(staging_layers, cache_layers, n_layers: int, block_table, n_pages: int,
                        page_bytes: int, num_blocks: int, d_err=None, stream=None):
    rc = (_lib or load()).hs_restore_kv_pages(
        _ptr(staging_layers), _ptr(cache_layers), int(n_layers), _ptr(block_table), int(n_pages),
        int(page_bytes), int(num_blocks), _ptr(d_err), _stream(stream))
    _check(rc, "hs_restore_kv_pages")


def hs_restore_request(staging_layers, cache_layers, n_layers: int, block_table, n_pages: int,
                       page_bytes: int, num_blocks: int, src_slots, dst_slots, n_slots: int,
                       floats_each: int, d_err=None, stream=None):
    rc = (_lib or load()).hs_restore_request(
        _ptr(staging_layers), _ptr(cache_layers), int(n_layers), _ptr(block_table), int(n_pages),
        int(page_bytes), int(num_blocks), _ptr(src_slots), _ptr(dst_slots), int(n_slots),
        int(floats_each), _ptr(d_err), _stream(stream))
    _check(rc, "hs_restore_request")


def hs_save_kv_pages(cache_layers, staging_layers, n_layers: int, block_table, n_pages: int,
                     page_bytes: int, num_blocks: int, d_err=None, stream=None):
    rc = (_lib or load()).hs_save_kv_pages(
        _ptr(cache_layers), _ptr(staging_layers), int(n_layers), _ptr(block_table), int(n_pages),
        int(page_bytes), int(num_blocks), _ptr(d_err), _stream(stream))
    _check(rc, "hs_save_kv_pages")


def hs_restore_kv_page_slices(staging_layers, cache_layers, n_layers: int, block_table,
                              n_pages: int, page_bytes: int, rows: int, col_off: int,
                              col_bytes: int, num_blocks: int, d_err=None, stream=None):
    rc = (_lib or load()).hs_restore_kv_page_slices(
        _ptr(staging_layers), _ptr(cache_layers), int(n_layers), _ptr(block_table), int(n_pages),
        int(page_bytes), int(rows), int(col_off), int(col_bytes), int(num_blocks), _ptr(d_err),
        _stream(stream))
    _check(rc, "hs_restore_kv_page_slices")


def hs_save_kv_page_slices(cache_layers, staging_layers, n_layers: int, block_table, n_pages: int,
                           page_bytes: int, rows: int, col_off: int, col_bytes: int,
                           num_blocks: int, d_err=None, stream=None):
    rc = (_lib or load()).hs_save_kv_page_slices(
        _ptr(cache_layers), _ptr(staging_layers), int(n_layers), _ptr(block_table), int(n_pages),
        int(page_bytes), int(rows), int(col_off), int(col_bytes), int(num_blocks), _ptr(d_err),
        _stream(stream))
    _check(rc, "hs_save_kv_page_slices")


def hs_restore_state(src_slots, dst_slots, n: int, floats_each: int, d_err=None, stream=None):
    rc = (_lib or load()).hs_restore_state(
        _ptr(src_slots), _ptr(dst_slots), int(n), int(floats_each), _ptr(d_err), _stream(stream))
    _check(rc, "hs_restore_state")


def hs_checkpoint_states(live_states, ckpt_slots, n: int, floats_each: int, d_err=None,
                         stream=None):
    rc = (_lib or load()).hs_checkpoint_states(
        _ptr(live_states), _ptr(ckpt_slots), int(n), int(floats_each), _ptr(d_err),
        _stream(stream))
    _check(rc, "hs_checkpoint_states")


def make_shape(batch, n_heads, d_k, d_v, max_tokens, kernel=HS_LINATTN_AUTO):
    return hs_linattn_shape(int(batch), int(n_heads), int(d_k), int(d_v), int(max_tokens),
                            int(kernel), 0)


def _prefill_call(name, shape, q, k, v, log_g, o, state, pos0, n_tokens, ckpt_interval,
                  ckpt_slots, d_err, stream):
    B = int(shape.batch)
    p0, keep_p0 = _i64(pos0, B)
    nt, keep_nt = _i32(n_tokens, B)
    rc = getattr(_lib or load(), name)(
        C.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(log_g), _ptr(o), _ptr(state), p0, nt,
        int(ckpt_interval), _ptr(ckpt_slots), _ptr(d_err), _stream(stream))
    _check(rc, name)


def hs_linattn_prefill_from_state(shape: hs_linattn_shape, q, k, v, log_g, o, state, pos0,
                                  n_tokens, ckpt_interval: int, ckpt_slots=None, d_err=None,
                                  stream=None):
    """pos0 / n_tokens: host sequences (ints) of length shape.batch."""
    _prefill_call("hs_linattn_prefill_from_state", shape, q, k, v, log_g, o, state, pos0,
                  n_tokens, ckpt_interval, ckpt_slots, d_err, stream)


def hs_test_prefill_stalled(shape: hs_linattn_shape, q, k, v, log_g, o, state, pos0, n_tokens,
                            ckpt_interval: int, ckpt_slots=None, d_err=None, stream=None):
    """Failure-detection hook (include/hs_test.h): the tensor-core prefill with one wait that
    nothing completes; each CTA's bounded wait runs out and it reports HS_DEVERR_TIMEOUT."""
    _prefill_call("hs_test_prefill_stalled", shape, q, k, v, log_g, o, state, pos0, n_tokens,
                  ckpt_interval, ckpt_slots, d_err, stream)


def hs_linattn_scan_workspace_bytes(shape: hs_linattn_shape, pos0, n_tokens) -> int:
    """Bytes of workspace hs_linattn_prefill_scan needs for these arguments."""
    B = int(shape.batch)
    p0, keep_p0 = _i64(pos0, B)
    nt, keep_nt = _i32(n_tokens, B)
    out = C.c_int64()
    rc = (_lib or load()).hs_linattn_scan_workspace_bytes(
        C.byref(shape), p0, nt, C.addressof(out))
    _check(rc, "hs_linattn_scan_workspace_bytes")
    return out.value


def hs_linattn_prefill_scan(shape: hs_linattn_shape, q, k, v, log_g, o, state, pos0, n_tokens,
                            ckpt_interval: int, ckpt_slots, workspace, workspace_bytes: int,
                            d_err=None, stream=None):
    """Segment-parallel prefill (same arguments as hs_linattn_prefill_from_state plus a device
    workspace of hs_linattn_scan_workspace_bytes bytes)."""
    B = int(shape.batch)
    p0, keep_p0 = _i64(pos0, B)
    nt, keep_nt = _i32(n_tokens, B)
    rc = (_lib or load()).hs_linattn_prefill_scan(
        C.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(log_g), _ptr(o), _ptr(state), p0, nt,
        int(ckpt_interval), _ptr(ckpt_slots), _ptr(workspace), int(workspace_bytes), _ptr(d_err),
        _stream(stream))
    _check(rc, "hs_linattn_prefill_scan")


def hs_linattn_prefill_scan_noalloc(shape: hs_linattn_shape, q, k, v, log_g, o, state, pos0,
                                    n_tokens, ckpt_interval: int, ckpt_slots=None, d_err=None,
                                    stream=None):
    """hs_linattn_prefill_scan with the library's fixed per-device workspace of
    HS_NOALLOC_SCRATCH_BYTES, for callers that cannot allocate device memory at this point (a
    serving engine whose HBM is already handed to its KV-cache pool).  Allocates nothing: the
    host arrays below are ctypes buffers.  Calls that overlap on the GPU share the workspace
    and race; the first call on a device does a one-time set-up and belongs before any stream
    capture."""
    B = int(shape.batch)
    p0, keep_p0 = _i64(pos0, B)
    nt, keep_nt = _i32(n_tokens, B)
    rc = (_lib or load()).hs_linattn_prefill_scan_noalloc(
        C.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(log_g), _ptr(o), _ptr(state), p0, nt,
        int(ckpt_interval), _ptr(ckpt_slots), _ptr(d_err), _stream(stream))
    _check(rc, "hs_linattn_prefill_scan_noalloc")


def hs_linattn_prefill_packed(shape: hs_linattn_shape, q, k, v, log_g, o, state, pos0, n_tokens,
                              cu_rows, ckpt_interval: int, ckpt_slots=None, d_err=None,
                              stream=None):
    """Packed token layout: token t of problem b is row cu_rows[b] + t.  pos0 / n_tokens /
    cu_rows: host sequences of length batch, batch, batch + 1."""
    B = int(shape.batch)
    p0, keep_p0 = _i64(pos0, B)
    nt, keep_nt = _i32(n_tokens, B)
    cu, keep_cu = _i64(cu_rows, B + 1)
    rc = (_lib or load()).hs_linattn_prefill_packed(
        C.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(log_g), _ptr(o), _ptr(state), p0, nt, cu,
        int(ckpt_interval), _ptr(ckpt_slots), _ptr(d_err), _stream(stream))
    _check(rc, "hs_linattn_prefill_packed")


def hs_linattn_num_checkpoints(pos0, n_tokens, ckpt_interval: int) -> int:
    B = len(pos0)
    p0, keep_p0 = _i64(pos0, B)
    nt, keep_nt = _i32(n_tokens, B)
    tot = C.c_int64()
    rc = (_lib or load()).hs_linattn_num_checkpoints(
        B, p0, nt, int(ckpt_interval), C.addressof(tot))
    _check(rc, "hs_linattn_num_checkpoints")
    return tot.value


def make_attn_shape(batch, n_heads, n_kv_heads, head_dim, page_size, num_blocks, max_pages,
                    dtype=HS_BF16, scale=None, q_stride=0, o_stride=0, unsplit=False):
    """scale=None: head_dim ** -0.5."""
    return hs_attn_shape(int(batch), int(n_heads), int(n_kv_heads), int(head_dim), int(page_size),
                         int(dtype), int(num_blocks), int(max_pages), int(q_stride), int(o_stride),
                         float(head_dim) ** -0.5 if scale is None else float(scale), int(unsplit))


def hs_kv_append(shape: hs_attn_shape, k, v, kv_stride: int, slots, n_rows: int, cache, d_err=None,
                 stream=None):
    """slots: device int64, block * page_size + row in the page; negative: the row is skipped."""
    rc = (_lib or load()).hs_kv_append(
        C.byref(shape), _ptr(k), _ptr(v), int(kv_stride), _ptr(slots), int(n_rows), _ptr(cache),
        _ptr(d_err), _stream(stream))
    _check(rc, "hs_kv_append")


def hs_attn_prefill_workspace_bytes(shape: hs_attn_shape, pos0, n_tokens) -> int:
    B = int(shape.batch)
    p0, keep_p0 = _i64(pos0, B)
    nt, keep_nt = _i32(n_tokens, B)
    out = C.c_int64()
    rc = (_lib or load()).hs_attn_prefill_workspace_bytes(C.byref(shape), p0, nt, C.addressof(out))
    _check(rc, "hs_attn_prefill_workspace_bytes")
    return out.value


def _attn_prefill_call(name, shape, q, cache, block_table, o, lse, pos0, n_tokens, cu_rows, workspace,
                       workspace_bytes, d_err, stream):
    B = int(shape.batch)
    p0, keep_p0 = _i64(pos0, B)
    nt, keep_nt = _i32(n_tokens, B)
    cu, keep_cu = _i64(cu_rows, B + 1)
    rc = getattr(_lib or load(), name)(
        C.byref(shape), _ptr(q), _ptr(cache), _ptr(block_table), _ptr(o), _ptr(lse), p0, nt, cu,
        _ptr(workspace), int(workspace_bytes), _ptr(d_err), _stream(stream))
    _check(rc, name)


def hs_attn_prefill(shape: hs_attn_shape, q, cache, block_table, o, lse, pos0, n_tokens, cu_rows,
                    workspace=None, workspace_bytes: int = 0, d_err=None, stream=None):
    """Causal attention of packed tails over the paged cache.  pos0 / n_tokens / cu_rows: host
    sequences of length batch, batch, batch + 1; lse may be None."""
    _attn_prefill_call("hs_attn_prefill", shape, q, cache, block_table, o, lse, pos0, n_tokens, cu_rows,
                       workspace, workspace_bytes, d_err, stream)


def hs_test_attn_stalled(shape: hs_attn_shape, q, cache, block_table, o, lse, pos0, n_tokens, cu_rows,
                         workspace=None, workspace_bytes: int = 0, d_err=None, stream=None):
    """Failure-detection hook (include/hs_test.h): hs_attn_prefill with one wait per CTA that nothing
    completes; it reports HS_DEVERR_TIMEOUT."""
    _attn_prefill_call("hs_test_attn_stalled", shape, q, cache, block_table, o, lse, pos0, n_tokens,
                       cu_rows, workspace, workspace_bytes, d_err, stream)


def hs_attn_decode_workspace_bytes(shape: hs_attn_shape, max_kv_len: int) -> int:
    out = C.c_int64()
    rc = (_lib or load()).hs_attn_decode_workspace_bytes(C.byref(shape), int(max_kv_len),
                                                         C.addressof(out))
    _check(rc, "hs_attn_decode_workspace_bytes")
    return out.value


def hs_attn_decode(shape: hs_attn_shape, q, cache, block_table, kv_len, max_kv_len: int, o, lse=None,
                   workspace=None, workspace_bytes: int = 0, d_err=None, stream=None):
    """One decode step; kv_len: device int32 [batch], the token of the step counted in."""
    rc = (_lib or load()).hs_attn_decode(
        C.byref(shape), _ptr(q), _ptr(cache), _ptr(block_table), _ptr(kv_len), int(max_kv_len),
        _ptr(o), _ptr(lse), _ptr(workspace), int(workspace_bytes), _ptr(d_err), _stream(stream))
    _check(rc, "hs_attn_decode")


def hs_attn_decode_shared_workspace_bytes(shape: hs_attn_shape, prefix_len: int,
                                          max_kv_len: int) -> int:
    out = C.c_int64()
    rc = (_lib or load()).hs_attn_decode_shared_workspace_bytes(
        C.byref(shape), int(prefix_len), int(max_kv_len), C.addressof(out))
    _check(rc, "hs_attn_decode_shared_workspace_bytes")
    return out.value


def hs_attn_decode_shared(shape: hs_attn_shape, q, cache, prefix_table, prefix_len: int, block_table,
                          kv_len, max_kv_len: int, o, lse=None, workspace=None,
                          workspace_bytes: int = 0, d_err=None, stream=None):
    """One decode step of requests behind one cached prefix; kv_len and block_table: of the keys
    behind it."""
    rc = (_lib or load()).hs_attn_decode_shared(
        C.byref(shape), _ptr(q), _ptr(cache), _ptr(prefix_table), int(prefix_len),
        _ptr(block_table), _ptr(kv_len), int(max_kv_len), _ptr(o), _ptr(lse), _ptr(workspace),
        int(workspace_bytes), _ptr(d_err), _stream(stream))
    _check(rc, "hs_attn_decode_shared")


def hs_rope_plan(dims: int, layout: int, base: float, scaling: int = HS_ROPE_PLAIN, factor: float = 1.0,
                 context: int = 1, low: float = 1.0, high: float = 32.0,
                 amplitude: float = 1.0) -> hs_rope:
    """The angles of rotary positions (host only); context, low and high: HS_ROPE_TURNS and
    HS_ROPE_INDEX alone."""
    out = hs_rope()
    rc = (_lib or load()).hs_rope_plan(int(dims), int(layout), float(base), int(scaling), float(factor),
                                       int(context), float(low), float(high), float(amplitude),
                                       C.byref(out))
    _check(rc, "hs_rope_plan")
    return out


def hs_rope_apply(shape: hs_attn_shape, rope: hs_rope, q, k, in_stride: int, pos, n_rows: int, q_out,
                  q_out_stride: int, k_out, k_out_stride: int, stream=None):
    """pos: device int64 [n_rows].  q and q_out, or k and k_out, may be None; in place is fine."""
    rc = (_lib or load()).hs_rope_apply(
        C.byref(shape), C.byref(rope), _ptr(q), _ptr(k), int(in_stride), _ptr(pos), int(n_rows),
        _ptr(q_out), int(q_out_stride), _ptr(k_out), int(k_out_stride), _stream(stream))
    _check(rc, "hs_rope_apply")


def hs_kv8_block_bytes(shape: hs_attn_shape) -> int:
    """Bytes of one block (page) of the 8-bit cache, its scales included."""
    out = C.c_int64()
    rc = (_lib or load()).hs_kv8_block_bytes(C.byref(shape), C.addressof(out))
    _check(rc, "hs_kv8_block_bytes")
    return out.value


def hs_kv8_append(shape: hs_attn_shape, k, v, kv_stride: int, slots, n_rows: int, cache, d_err=None,
                  stream=None):
    """slots as in hs_kv_append; the rows of a group of 16 tokens stand within 16 rows, none but skipped
    ones among them."""
    rc = (_lib or load()).hs_kv8_append(
        C.byref(shape), _ptr(k), _ptr(v), int(kv_stride), _ptr(slots), int(n_rows), _ptr(cache),
        _ptr(d_err), _stream(stream))
    _check(rc, "hs_kv8_append")


def hs_kv8_append_rope(shape: hs_attn_shape, rope: hs_rope, q, k, v, in_stride: int, pos, slots,
                       n_rows: int, q_out, q_out_stride: int, cache, d_err=None, stream=None):
    """hs_rope_apply of q and hs_kv8_append of the turned k, and of v; q and q_out may be None."""
    rc = (_lib or load()).hs_kv8_append_rope(
        C.byref(shape), C.byref(rope), _ptr(q), _ptr(k), _ptr(v), int(in_stride), _ptr(pos),
        _ptr(slots), int(n_rows), _ptr(q_out), int(q_out_stride), _ptr(cache), _ptr(d_err),
        _stream(stream))
    _check(rc, "hs_kv8_append_rope")


def hs_kv8_decode_workspace_bytes(shape: hs_attn_shape, max_kv_len: int) -> int:
    out = C.c_int64()
    rc = (_lib or load()).hs_kv8_decode_workspace_bytes(C.byref(shape), int(max_kv_len),
                                                        C.addressof(out))
    _check(rc, "hs_kv8_decode_workspace_bytes")
    return out.value


def _kv8_decode_call(name, shape, q, cache, block_table, kv_len, max_kv_len, o, lse, workspace,
                     workspace_bytes, d_err, stream):
    rc = getattr(_lib or load(), name)(
        C.byref(shape), _ptr(q), _ptr(cache), _ptr(block_table), _ptr(kv_len), int(max_kv_len),
        _ptr(o), _ptr(lse), _ptr(workspace), int(workspace_bytes), _ptr(d_err), _stream(stream))
    _check(rc, name)


def hs_kv8_decode(shape: hs_attn_shape, q, cache, block_table, kv_len, max_kv_len: int, o, lse=None,
                  workspace=None, workspace_bytes: int = 0, d_err=None, stream=None):
    """One decode step over the 8-bit cache; kv_len: device int32 [batch], the token of the step
    counted in."""
    _kv8_decode_call("hs_kv8_decode", shape, q, cache, block_table, kv_len, max_kv_len, o, lse, workspace,
                     workspace_bytes, d_err, stream)


def hs_test_kv8_stalled(shape: hs_attn_shape, q, cache, block_table, kv_len, max_kv_len: int, o, lse=None,
                        workspace=None, workspace_bytes: int = 0, d_err=None, stream=None):
    """Failure-detection hook (include/hs_test.h): hs_kv8_decode with one wait per warp that nothing
    completes; it reports HS_DEVERR_TIMEOUT."""
    _kv8_decode_call("hs_test_kv8_stalled", shape, q, cache, block_table, kv_len, max_kv_len, o, lse,
                     workspace, workspace_bytes, d_err, stream)


def hs_kv8_read(shape: hs_attn_shape, cache, block_table, kv_len, max_kv_len: int, out, out_blocks: int,
                out_table, d_err=None, stream=None):
    """The first kv_len[b] tokens of each request read back into 16-bit pages; kv_len: device int32
    [batch]."""
    rc = (_lib or load()).hs_kv8_read(
        C.byref(shape), _ptr(cache), _ptr(block_table), _ptr(kv_len), int(max_kv_len), _ptr(out),
        int(out_blocks), _ptr(out_table), _ptr(d_err), _stream(stream))
    _check(rc, "hs_kv8_read")

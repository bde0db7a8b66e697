"""Thin ctypes binding of libdash (include/dash.h), same names as the C ABI.

Argument marshalling only: shapes, raw device pointers and the current HIP
stream are taken from torch tensors and passed through; every step of the
computation runs in the library's HIP kernels.  If libdash.so is missing this
module raises -- there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
import struct

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libdash.so")

DASH_SCHED_ATOMIC, DASH_SCHED_NAIVE, DASH_SCHED_DESCENDING = 0, 1, 2
DASH_SCHED_SHIFT, DASH_SCHED_SYMSHIFT, DASH_SCHED_AUTO, DASH_SCHED_PARTIALS, DASH_SCHED_SPLIT = 3, 4, 5, 6, 7
SCHEDULES = {"atomic": 0, "naive": 1, "descending": 2, "shift": 3, "symshift": 4, "auto": 5, "partials": 6,
             "split": 7}
DASH_OK, DASH_ERR_INVALID_ARG, DASH_ERR_UNSUPPORTED = 0, -1, -2
DASH_ERR_HIP, DASH_ERR_TIMEOUT, DASH_ERR_NO_DEVICE = -3, -4, -5
DASH_FLAG_POISON_COUNTERS = 1
DASH_TICKETS_AUTO, DASH_TICKETS_HEAD_MAJOR, DASH_TICKETS_CHAIN_MAJOR = 0, 1, 2
DASH_PLACEMENT_AUTO, DASH_PLACEMENT_GLOBAL, DASH_PLACEMENT_XCD = 0, 1, 2

# every symbol include/dash.h declares
EXPORTS = ("dash_attn_fwd", "dash_attn_fwd_ex", "dash_attn_bwd", "dash_bwd_workspace_size",
           "dash_attn_bwd_ex", "dash_attn_bwd_noalloc", "dash_bwd_check", "dash_resolve_schedule", "dash_schedule_table",
           "dash_bwd_placement", "dash_mfma_peak", "dash_last_error", "dash_release_workspace",
           "dash_auto_schedule", "dash_model_makespan", "dash_kv_append", "dash_attn_decode",
           "dash_decode_workspace_size", "dash_attn_packed_fwd", "dash_attn_packed_bwd",
           "dash_packed_workspace_size", "dash_packed_fwd_workspace_size", "dash_kv_read", "dash_rotary",
           "dash_rotary_frequencies", "dash_attn_prefix_decode", "dash_prefix_decode_workspace_size")
DASH_CACHE_BF16, DASH_CACHE_E4M3, DASH_CACHE_MXFP4, DASH_CACHE_MXFP8 = 0, 1, 4, 8
ROTARY_SCALINGS = {"plain": 0, "linear": 1, "base": 2, "parts": 3}


class DashError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"libdash error {code}: {msg}")
        self.code = code


class dash_bwd_options_t(ctypes.Structure):
    _fields_ = [("spin_limit", ctypes.c_int), ("flags", ctypes.c_int),
                ("witness", ctypes.c_void_p), ("partials", ctypes.c_void_p),
                ("dq_accum", ctypes.c_void_p), ("event_main_begin", ctypes.c_void_p),
                ("event_main_end", ctypes.c_void_p), ("max_workgroups", ctypes.c_int),
                ("ticket_order", ctypes.c_int), ("placement", ctypes.c_int),
                ("wait_stats", ctypes.c_void_p)]


_VP, _CI, _I64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64


class dash_paged_cache_t(ctypes.Structure):
    _fields_ = [("batch", _CI), ("heads_q", _CI), ("heads_kv", _CI), ("d", _CI), ("pages", _CI), ("page_size", _CI),
                ("table_width", _CI), ("cache_type", _CI), ("k_cache", _VP), ("v_cache", _VP),
                ("k_page_stride", _I64), ("k_head_stride", _I64), ("k_row_stride", _I64),
                ("v_page_stride", _I64), ("v_head_stride", _I64), ("v_row_stride", _I64),
                ("block_table", _VP), ("table_stride", _I64), ("lens", _VP), ("k_scale", _VP), ("v_scale", _VP),
                ("k_mx", _VP), ("v_mx", _VP)]


class dash_append_t(ctypes.Structure):
    _fields_ = [("tokens", _CI), ("cu", _VP), ("k", _VP), ("v", _VP), ("q", _VP), ("q_out", _VP), ("k_out", _VP),
                ("k_row_stride", _I64), ("k_head_stride", _I64), ("v_row_stride", _I64), ("v_head_stride", _I64),
                ("q_row_stride", _I64), ("q_head_stride", _I64), ("q_out_row_stride", _I64),
                ("q_out_head_stride", _I64), ("k_out_row_stride", _I64), ("k_out_head_stride", _I64),
                ("inv_freq", _VP), ("rotary_dim", _CI), ("interleaved", _CI)]


class dash_read_t(ctypes.Structure):
    _fields_ = [("rows", _CI), ("cu", _VP), ("first", _VP), ("k_out", _VP), ("v_out", _VP), ("k_row_stride", _I64),
                ("k_head_stride", _I64), ("v_row_stride", _I64), ("v_head_stride", _I64)]


class dash_rotary_t(ctypes.Structure):
    _fields_ = [("rows", _CI), ("heads_q", _CI), ("heads_k", _CI), ("d", _CI), ("positions", _VP), ("cu", _VP), ("start", _VP),
                ("batch", _CI), ("q", _VP), ("k", _VP), ("q_out", _VP), ("k_out", _VP),
                ("q_row_stride", _I64), ("q_head_stride", _I64), ("k_row_stride", _I64), ("k_head_stride", _I64),
                ("q_out_row_stride", _I64), ("q_out_head_stride", _I64), ("k_out_row_stride", _I64), ("k_out_head_stride", _I64),
                ("inv_freq", _VP), ("rotary_dim", _CI), ("interleaved", _CI), ("amplitude", ctypes.c_float), ("backward", _CI)]


class dash_packed_t(ctypes.Structure):
    _fields_ = [("batch", _CI), ("heads_q", _CI), ("heads_kv", _CI), ("d", _CI), ("causal", _CI), ("total_q", _CI),
                ("total_k", _CI), ("scale", ctypes.c_float), ("cu_q", _VP), ("cu_k", _VP)]
    _fields_ += [(f"{t}_{s}_stride", _I64) for t in ("q", "k", "v", "o", "do", "dq", "dk", "dv") for s in ("row", "head")]


def _packer(cls):
    """A function from a C struct's values, by position, to its bytes, in a third of the time
    that ctypes takes for its fields.  Pointers are ints here, 0 for none."""
    code = {_CI: "i", ctypes.c_float: "f", _I64: "q", _VP: "P"}
    fmt = struct.Struct("@" + "".join(code[t] for _, t in cls._fields_))
    for i, (name, t) in enumerate(cls._fields_):  # the same layout
        head = struct.calcsize("@" + "".join(code[u] for _, u in cls._fields_[:i]) + "0" + code[t])
        assert getattr(cls, name).offset == head and fmt.size <= ctypes.sizeof(cls)

    def pack(*values):
        try:
            return fmt.pack(*values)
        except (struct.error, OverflowError) as e:
            _bad(f"{cls.__name__}: {e}")
    return pack


_pack_cache, _pack_append, _pack_packed, _pack_read, _pack_rotary = map(
    _packer, (dash_paged_cache_t, dash_append_t, dash_packed_t, dash_read_t, dash_rotary_t))
_lib = None


def load():
    """Load libdash.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise DashError(DASH_ERR_NO_DEVICE, f"{LIB_PATH} is not built (run __graft_entry__.build())")
        lib = ctypes.CDLL(LIB_PATH)
        vp, ci, cf, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
        ip = ctypes.POINTER(ctypes.c_int)
        lib.dash_attn_fwd.argtypes = [vp] * 5 + [ci] * 5
        lib.dash_attn_fwd_ex.argtypes = [vp] * 5 + [ci] * 5 + [cf, vp]
        lib.dash_attn_bwd.argtypes = [vp] * 9 + [ci] * 6
        lib.dash_attn_bwd_ex.argtypes = ([vp] * 9 + [ci] * 6 + [cf, vp, sz,
                                         ctypes.POINTER(dash_bwd_options_t), vp])
        lib.dash_attn_bwd_noalloc.argtypes = [vp] * 9 + [ci] * 6 + [cf, vp, vp]
        lib.dash_bwd_workspace_size.argtypes = [ci] * 5
        lib.dash_bwd_workspace_size.restype = sz
        lib.dash_bwd_check.argtypes = [vp, vp]
        lib.dash_resolve_schedule.argtypes = [ci] * 3
        lib.dash_schedule_table.argtypes = [ci] * 6 + [ip] * 5
        lib.dash_bwd_placement.argtypes = [ci] * 6
        lib.dash_mfma_peak.argtypes = [ci, ctypes.POINTER(ctypes.c_double)]
        dp = ctypes.POINTER(ctypes.c_double)
        lib.dash_auto_schedule.argtypes = [ci] * 6 + [ip, dp]
        lib.dash_model_makespan.argtypes = [ci] * 9 + [ctypes.c_double, ctypes.c_double, dp]
        # (the structs as void pointers: bytes are one as well)
        lib.dash_kv_append.argtypes = [vp, vp, vp, vp]
        lib.dash_attn_decode.argtypes = [vp, vp, _I64, _I64, vp, _I64, _I64, vp, cf, vp,
                                         sz, vp, vp]
        lib.dash_decode_workspace_size.argtypes = [ci] * 6
        lib.dash_attn_packed_bwd.argtypes = [vp] * 11 + [sz, vp, vp]
        lib.dash_packed_workspace_size.argtypes = [ci] * 6
        lib.dash_packed_workspace_size.restype = sz
        lib.dash_attn_packed_fwd.argtypes = [vp] * 7 + [sz, vp]
        lib.dash_packed_fwd_workspace_size.argtypes = [ci] * 6
        lib.dash_packed_fwd_workspace_size.restype = sz
        lib.dash_decode_workspace_size.restype = sz
        lib.dash_kv_read.argtypes = [vp, vp, vp, vp]
        lib.dash_rotary.argtypes = [vp, vp, vp]
        lib.dash_rotary_frequencies.argtypes = [ci, ctypes.c_double, ci] + [ctypes.c_double] * 4 + [vp, ctypes.POINTER(cf)]
        lib.dash_attn_prefix_decode.argtypes = [vp, vp, ci, vp, vp, _I64, _I64, vp, _I64, _I64, vp, cf, vp, sz, vp, vp]
        lib.dash_prefix_decode_workspace_size.argtypes = [ci] * 7
        lib.dash_prefix_decode_workspace_size.restype = sz
        lib.dash_last_error.restype = ctypes.c_char_p
        lib.dash_release_workspace.restype = None
        for f in ("dash_attn_fwd", "dash_attn_fwd_ex", "dash_attn_bwd", "dash_attn_bwd_ex", "dash_attn_bwd_noalloc",
                  "dash_bwd_check", "dash_resolve_schedule", "dash_schedule_table", "dash_bwd_placement",
                  "dash_mfma_peak", "dash_auto_schedule", "dash_model_makespan", "dash_kv_append", "dash_attn_decode",
                  "dash_attn_packed_fwd", "dash_attn_packed_bwd", "dash_kv_read", "dash_rotary", "dash_rotary_frequencies",
                  "dash_attn_prefix_decode"):
            getattr(lib, f).restype = ci
        _lib = lib
    return _lib


def _check(rc: int):
    if rc != DASH_OK:
        raise DashError(rc, load().dash_last_error().decode())
    return rc


def _sched(s) -> int:
    return SCHEDULES[s] if isinstance(s, str) else int(s)


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is None:
        import torch
        return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    return ctypes.c_void_p(stream if isinstance(stream, int) else stream.cuda_stream)


def _shape(q):
    if q.dim() != 4:
        raise DashError(DASH_ERR_INVALID_ARG, "tensors must be [B, H, N, d]")
    return tuple(int(x) for x in q.shape)


def _require(ts, dtype_name):
    import torch
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype_name]
    for t in ts:
        if t.dtype != dt or not t.is_contiguous() or not t.is_cuda:
            raise DashError(DASH_ERR_INVALID_ARG, f"expected contiguous {dtype_name} device tensors")


def dash_last_error() -> str:
    return load().dash_last_error().decode()


def dash_release_workspace():
    load().dash_release_workspace()


def dash_resolve_schedule(schedule, d: int, causal: bool) -> int:
    return load().dash_resolve_schedule(_sched(schedule), d, int(causal))


def dash_auto_schedule(B: int, H: int, N: int, d: int, causal: bool, workers: int = 0):
    """(schedule, predicted ms) that DASH_SCHED_AUTO runs for this shape."""
    s, ms = ctypes.c_int(), ctypes.c_double()
    _check(load().dash_auto_schedule(B, H, N, d, int(causal), workers, ctypes.byref(s), ctypes.byref(ms)))
    return s.value, ms.value


def dash_model_makespan(schedule, B: int, H: int, N: int, d: int, causal: bool, workers: int, c: float, r: float,
                        ticket_order: int = DASH_TICKETS_AUTO, max_heads: int = 0) -> float:
    """Makespan of the DAG model with block-step costs c (compute) and r (reduction)."""
    m = ctypes.c_double()
    _check(load().dash_model_makespan(_sched(schedule), B, H, N, d, int(causal), workers, ticket_order,
                                      max_heads, c, r, ctypes.byref(m)))
    return m.value


def dash_bwd_workspace_size(B: int, H: int, N: int, d: int, schedule="shift") -> int:
    return int(load().dash_bwd_workspace_size(B, H, N, d, _sched(schedule)))


def dash_attn_fwd(q, k, v, o, lse, causal: bool, scale=None, stream=None):
    """O and L of attention into o (bf16) and lse (fp32) on the current stream."""
    B, H, N, d = _shape(q)
    _require((q, k, v, o), "bf16")
    _require((lse,), "f32")
    s = 0.0 if scale is None else float(scale)  # 0: the library's default 1/sqrt(d)
    _check(load().dash_attn_fwd_ex(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), B, H, N, d,
                                   int(causal), s, _stream(stream)))


def dash_attn_bwd(q, k, v, o, dO, lse, dq, dk, dv, causal: bool, schedule, scale=None,
                  workspace=None, options: dash_bwd_options_t | None = None, stream=None):
    """Backward into dq, dk, dv.  With ``workspace`` (a device uint8 tensor of at
    least dash_bwd_workspace_size bytes) the call is asynchronous on the
    current stream; without it the library's own workspace is used and the
    call synchronizes and reports wait timeouts."""
    B, H, N, d = _shape(q)
    _require((q, k, v, o, dO, dq, dk, dv), "bf16")
    _require((lse,), "f32")
    lib = load()
    if workspace is None and options is None and scale is None:
        _check(lib.dash_attn_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(dO), _ptr(lse),
                                 _ptr(dq), _ptr(dk), _ptr(dv), B, H, N, d, int(causal),
                                 _sched(schedule)))
        return
    if workspace is None:
        raise DashError(DASH_ERR_INVALID_ARG, "scale/options need an explicit workspace")
    s = 0.0 if scale is None else float(scale)  # 0: the library's default 1/sqrt(d)
    opt = ctypes.byref(options) if options is not None else None
    _check(lib.dash_attn_bwd_ex(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(dO), _ptr(lse),
                                _ptr(dq), _ptr(dk), _ptr(dv), B, H, N, d, int(causal),
                                _sched(schedule), s, _ptr(workspace), workspace.numel(), opt,
                                _stream(stream)))


def dash_attn_bwd_noalloc(q, k, v, o, dO, lse, dq, dk, dv, causal: bool, schedule, scale=None, status=None,
                          stream=None):
    """Backward into dq, dk, dv on the library's fixed per-device scratch: no
    allocation, asynchronous on the current stream.  ``status``: optional
    device int32 tensor (one element) that receives 0, or 1 after a wait
    timeout, once the stream has run the call."""
    B, H, N, d = _shape(q)
    _require((q, k, v, o, dO, dq, dk, dv), "bf16")
    _require((lse,), "f32")
    if status is not None and (not status.is_cuda or status.dtype.itemsize != 4):
        raise DashError(DASH_ERR_INVALID_ARG, "status must be a device int32 tensor")
    s = 0.0 if scale is None else float(scale)
    _check(load().dash_attn_bwd_noalloc(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(dO), _ptr(lse),
                                        _ptr(dq), _ptr(dk), _ptr(dv), B, H, N, d, int(causal),
                                        _sched(schedule), s, _ptr(status), _stream(stream)))


def dash_bwd_check(workspace, stream=None) -> int:
    """Synchronize and return the status of the last backward on ``workspace``
    (DASH_OK or DASH_ERR_TIMEOUT) without raising."""
    return load().dash_bwd_check(_ptr(workspace), _stream(stream))


def dash_bwd_placement(B: int, H: int, N: int, d: int, causal: bool, schedule="auto") -> int:
    """The placement AUTO picks on the current device (DASH_PLACEMENT_GLOBAL / _XCD)."""
    rc = load().dash_bwd_placement(B, H, N, d, int(causal), _sched(schedule))
    if rc < 0:
        _check(rc)
    return rc


def dash_mfma_peak(iters: int = 0) -> float:
    """Measured bf16 dense MFMA throughput of the current device in TFLOP/s."""
    out = ctypes.c_double(0.0)
    _check(load().dash_mfma_peak(int(iters), ctypes.byref(out)))
    return out.value


def dash_schedule_table(schedule, N: int, d: int, causal: bool, placement=DASH_PLACEMENT_GLOBAL, heads: int = 1) -> dict:
    """The schedule the kernels follow for one head of a call of ``heads`` (= B*H)
    heads under ``placement`` (host computation)."""
    lib = load()
    geo = (ctypes.c_int * 6)()
    _check(lib.dash_schedule_table(_sched(schedule), heads, N, d, int(causal), placement, geo, None, None, None, None))
    t_r, t_c, br, chains, bc, grp = list(geo)
    cap = t_r + 1
    chain_len = np.zeros(chains, np.int32)
    task_kv = np.full(chains * cap, -1, np.int32)
    task_q = np.full(chains * cap, -1, np.int32)
    rank = np.zeros(t_r * t_c, np.int32)
    p = lambda a: a.ctypes.data_as(ctypes.POINTER(ctypes.c_int))
    _check(lib.dash_schedule_table(_sched(schedule), heads, N, d, int(causal), placement, geo, p(chain_len), p(task_kv),
                                   p(task_q), p(rank)))
    return dict(t_r=t_r, t_c=t_c, br=br, chains=chains, bc=bc, group=grp, chain_len=chain_len,
                task_kv=task_kv.reshape(chains, cap), task_q=task_q.reshape(chains, cap),
                rank=rank.reshape(t_r, t_c))


# ----------------------------------------------------------------- sequences of different lengths
# These calls are short on the GPU, so their checks are written to be quick: the
# strides go into the C structs by position, and the raw stream is asked for.
def _bad(msg: str):
    raise DashError(DASH_ERR_INVALID_ARG, msg)


def _rows(name, t, dtype, dev, rows, heads, d):
    """A [rows, heads, d] tensor on GPU `dev` whose heads are contiguous: its pointer and strides."""
    if t.dtype is not dtype or t.get_device() != dev or t.shape != (rows, heads, d):
        _bad(f"{name} must be a {dtype} [{rows}, {heads}, {d}] tensor on cuda:{dev}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    row, head, one = t.stride()
    if one != 1 and d > 1:
        _bad(f"{name}: the last dimension must be contiguous")
    return t.data_ptr(), row, head


_NONE = (0, 0, 0)  # of a tensor that is not there


def _flat(name, t, dtype, dev, *shape):
    """A contiguous tensor of this shape on GPU `dev`, or None: its pointer (0 for None).  A
    vector may have further dimensions of 1."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous() or t.shape != shape and (
            len(shape) > 1 or t.numel() != shape[0] or t.numel() not in (1, *t.shape)):
        _bad(f"{name} must be a contiguous {dtype} {list(shape)} tensor on cuda:{dev}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _gpu(t):
    """The number of a tensor's GPU."""
    dev = t.get_device()
    if dev < 0:
        _bad("expected device tensors")
    return dev


def _space(workspace, need, like, dev, stream):
    """A call's workspace (allocated beside `like` if there is none, behind the current
    stream's work): pointer, bytes and tensor."""
    import torch
    if workspace is None:
        if stream is not None:
            _bad("a call on an explicit stream needs an explicit workspace")
        need = need if need > 256 else 256
        workspace = like.new_empty(need, dtype=torch.uint8)
        return workspace.data_ptr(), need, workspace
    return _flat("workspace", workspace, torch.uint8, dev, *workspace.shape), workspace.numel(), workspace


def _call(f, dev, stream, *args):
    """f(*args, stream) with GPU `dev` current, as the library launches on the current one."""
    import torch
    if torch._C._cuda_getDevice() != dev:
        with torch.cuda.device(dev):
            return _call(f, dev, stream, *args)
    if stream is None:
        stream = torch._C._cuda_getCurrentRawStream(dev)
    elif not isinstance(stream, int):
        stream = stream.cuda_stream
    _check(f(*args, stream))


def _cache(k_cache, v_cache, block_table, lens, k_scale, v_scale, heads_q, dev):
    """dash_paged_cache_t of [pages, heads_kv, page_size, d] caches (any strides, contiguous rows), and its
    d: bfloat16; float8_e4m3fn with a scale per head or none, or with a scale byte per 32 components
    (uint8 [pages, heads_kv, page_size, d / 32]); or uint8 [..., d / 2], two e2m1 each, with scale bytes."""
    import torch
    dt, u8 = k_cache.dtype, torch.uint8
    if k_cache.dim() != 4 or k_cache.shape != v_cache.shape or v_cache.dtype is not dt or v_cache.get_device() != dev:
        _bad("k_cache and v_cache must be [pages, heads_kv, page_size, d] tensors alike")
    pages, heads_kv, page, d = k_cache.shape
    if dt is torch.bfloat16:
        kind = DASH_CACHE_BF16
    elif dt is torch.float8_e4m3fn:
        kind = DASH_CACHE_E4M3 if (k_scale is None or k_scale.dtype is not u8) and (v_scale is None or v_scale.dtype is not u8) else DASH_CACHE_MXFP8
    elif dt is u8:
        kind, d = DASH_CACHE_MXFP4, 2 * d
    else:
        _bad("caches must be bfloat16, float8_e4m3fn or (MXFP4) uint8")
    (kp, kh, kr, k1), (vp, vh, vr, v1) = k_cache.stride(), v_cache.stride()
    if k1 != 1 or v1 != 1:
        _bad("the last dimension of the caches must be contiguous")
    batch = lens.numel()
    if block_table.dtype is not torch.int32 or block_table.get_device() != dev or block_table.dim() != 2:
        _bad(f"block_table must be an int32 [batch, width] tensor on cuda:{dev}")
    rows, width = block_table.shape
    row, one = block_table.stride()
    if rows != batch or (width > 1 and one != 1):
        _bad("block_table must be [batch, width] with contiguous rows")
    ks = vs = kx = vx = 0
    if kind >= DASH_CACHE_MXFP4:
        if k_scale is None or v_scale is None:
            _bad("a microscaled cache needs k_scale and v_scale")
        kx = _flat("k_scale", k_scale, u8, dev, pages, heads_kv, page, d // 32)
        vx = _flat("v_scale", v_scale, u8, dev, pages, heads_kv, page, d // 32)
    else:
        ks, vs = _flat("k_scale", k_scale, torch.float32, dev, heads_kv), _flat("v_scale", v_scale, torch.float32, dev, heads_kv)
    return _pack_cache(
        batch, heads_q, heads_kv, d, pages, page, width, kind, k_cache.data_ptr(), v_cache.data_ptr(), kp, kh, kr, vp, vh, vr,
        block_table.data_ptr(), row if batch > 1 else width, _flat("lens", lens, torch.int32, dev, batch), ks, vs, kx, vx), d


def dash_kv_append(k, v, k_cache, v_cache, block_table, lens, cu=None, q=None, q_out=None, k_out=None, inv_freq=None,
                   interleaved: bool = False, k_scale=None, v_scale=None, status=None, stream=None):
    """New keys and values (bf16 [tokens, heads_kv, d]) into a paged cache behind the
    ``lens`` rows that each sequence has, keys and queries rotated by their place
    (``inv_freq``: fp32, one per rotated pair).  ``cu``: int32 [batch + 1], where each
    sequence's tokens begin (rows before cu[0] and from cu[-1] on are left alone); without it every
    sequence gets one token.  The rotated
    queries go to ``q_out`` and, if given, the rotated keys to ``k_out``.
    A microscaled cache (float8_e4m3fn, or uint8 for MXFP4, with uint8 ``k_scale`` and ``v_scale``
    [pages, heads_kv, page_size, d / 32]) gets its scale bytes too.
    The rotation by ``inv_freq`` has no amplitude: with frequencies that come with one, dash_rotary (``start`` = lens)
    goes before this call, which then gets none.
    ``status``: optional int32 that a token without a page, or a row between offsets that do
    not rise, sets to 1."""
    import torch
    if k.dim() != 3:
        _bad("k must be [tokens, heads_kv, d]")
    if (q is None) != (q_out is None):
        _bad("q and q_out come together")
    if q is not None and q.dim() != 3:
        _bad("q must be [tokens, heads_q, d]")
    dev = _gpu(k_cache)
    tokens, heads_kv, d = k.shape
    heads_q = heads_kv if q is None else q.shape[1]
    c, cd = _cache(k_cache, v_cache, block_table, lens, k_scale, v_scale, heads_q, dev)
    bf, i32 = torch.bfloat16, torch.int32
    if k_cache.shape[1] != heads_kv or cd != d:
        _bad("k and k_cache must have the same heads and head dim")
    none = (0, 0, 0)
    kp, *ks = _rows("k", k, bf, dev, tokens, heads_kv, d)
    vp, *vs = _rows("v", v, bf, dev, tokens, heads_kv, d)
    qp, *qs = none if q is None else _rows("q", q, bf, dev, tokens, heads_q, d)
    qo, *qos = none if q is None else _rows("q_out", q_out, bf, dev, tokens, heads_q, d)
    ko, *kos = none if k_out is None else _rows("k_out", k_out, bf, dev, tokens, heads_kv, d)
    rot = 0 if inv_freq is None else 2 * inv_freq.numel()
    x = _pack_append(tokens, _flat("cu", cu, i32, dev, lens.numel() + 1), kp, vp, qp, qo, ko, *ks, *vs, *qs, *qos, *kos,
                     _flat("inv_freq", inv_freq, torch.float32, dev, rot // 2), rot, interleaved)
    _call(load().dash_kv_append, dev, stream, c, x, _flat("status", status, i32, dev, 1))


def dash_decode_workspace_size(batch: int, heads_q: int, heads_kv: int, d: int, page_size: int, table_width: int) -> int:
    return int(load().dash_decode_workspace_size(batch, heads_q, heads_kv, d, page_size, table_width))


def dash_attn_decode(q, k_cache, v_cache, block_table, lens, o, lse=None, scale=None, k_scale=None, v_scale=None,
                     workspace=None, status=None, stream=None):
    """Attention of one query token per sequence (q: bf16 [batch, heads_q, d]) over its
    ``lens`` cached keys into o and, if given, lse (fp32 [batch, heads_q]).
    ``workspace``: a uint8 device tensor of dash_decode_workspace_size bytes (without
    it one is allocated).  ``status``: optional int32 that a length or a
    page out of range sets to 1."""
    import torch
    if q.dim() != 3:
        _bad("q must be [batch, heads_q, d]")
    dev = _gpu(k_cache)
    batch, heads_q, d = q.shape
    c, cd = _cache(k_cache, v_cache, block_table, lens, k_scale, v_scale, heads_q, dev)
    _, heads_kv, page, _ = k_cache.shape
    if lens.numel() != batch or cd != d:
        _bad("q, lens and the caches must have the same batch and head dim")
    lib = load()
    need = 0 if workspace is not None else lib.dash_decode_workspace_size(batch, heads_q, heads_kv, d, page, block_table.shape[1])
    ws, size, workspace = _space(workspace, need, q, dev, stream)
    _call(lib.dash_attn_decode, dev, stream, c, *_rows("q", q, torch.bfloat16, dev, batch, heads_q, d),
          *_rows("o", o, torch.bfloat16, dev, batch, heads_q, d), _flat("lse", lse, torch.float32, dev, batch, heads_q),
          0.0 if scale is None else scale, ws, size, _flat("status", status, torch.int32, dev, 1))


def attn_decode(q, k_cache, v_cache, block_table, lens, scale=None, k_scale=None, v_scale=None, workspace=None,
                status=None):
    """dash_attn_decode into a new o."""
    import torch
    o = torch.empty_like(q, memory_format=torch.contiguous_format)
    dash_attn_decode(q, k_cache, v_cache, block_table, lens, o, None, scale, k_scale, v_scale, workspace, status)
    return o


def dash_prefix_decode_workspace_size(batch: int, heads_q: int, heads_kv: int, d: int, page_size: int, table_width: int,
                                      prefix_width: int) -> int:
    return int(load().dash_prefix_decode_workspace_size(batch, heads_q, heads_kv, d, page_size, table_width, prefix_width))


def dash_attn_prefix_decode(q, k_cache, v_cache, block_table, lens, prefix_table, prefix_len, o, lse=None, scale=None,
                            k_scale=None, v_scale=None, workspace=None, status=None, stream=None):
    """dash_attn_decode for a batch whose sequences share their first ``prefix_len`` keys (int32, one
    element, on the device), in the pages ``prefix_table`` (int32 [width]), read once for all of
    them.  ``lens`` and ``block_table`` count the shared keys as dash_attn_decode does."""
    import torch
    if q.dim() != 3:
        _bad("q must be [batch, heads_q, d]")
    dev = _gpu(k_cache)
    batch, heads_q, d = q.shape
    c, cd = _cache(k_cache, v_cache, block_table, lens, k_scale, v_scale, heads_q, dev)
    _, heads_kv, page, _ = k_cache.shape
    if lens.numel() != batch or cd != d:
        _bad("q, lens and the caches must have the same batch and head dim")
    if prefix_table.dim() != 1:
        _bad("prefix_table must be int32 [width]")
    width = prefix_table.numel()
    pt, pl = _flat("prefix_table", prefix_table, torch.int32, dev, width), _flat("prefix_len", prefix_len, torch.int32, dev, prefix_len.numel())
    if prefix_len.numel() != 1:
        _bad("prefix_len must be one int32")
    lib = load()
    need = 0 if workspace is not None else lib.dash_prefix_decode_workspace_size(batch, heads_q, heads_kv, d, page, block_table.shape[1], width)
    ws, size, workspace = _space(workspace, need, q, dev, stream)
    _call(lib.dash_attn_prefix_decode, dev, stream, c, pt, width, pl, *_rows("q", q, torch.bfloat16, dev, batch, heads_q, d),
          *_rows("o", o, torch.bfloat16, dev, batch, heads_q, d), _flat("lse", lse, torch.float32, dev, batch, heads_q),
          0.0 if scale is None else scale, ws, size, _flat("status", status, torch.int32, dev, 1))


def attn_prefix_decode(q, k_cache, v_cache, block_table, lens, prefix_table, prefix_len, scale=None, k_scale=None, v_scale=None,
                       workspace=None, status=None):
    """dash_attn_prefix_decode into a new o."""
    import torch
    o = torch.empty_like(q, memory_format=torch.contiguous_format)
    dash_attn_prefix_decode(q, k_cache, v_cache, block_table, lens, prefix_table, prefix_len, o, None, scale, k_scale, v_scale,
                            workspace, status)
    return o


def dash_kv_read(k_cache, v_cache, block_table, lens, cu, k_out=None, v_out=None, first=None, k_scale=None, v_scale=None,
                 status=None, stream=None):
    """Keys and values of a paged cache of any type as packed bf16 rows into ``k_out`` and ``v_out``
    ([rows, heads_kv, d], either may be None): rows cu[s] .. cu[s+1]-1 (``cu``: int32 [batch + 1]) receive
    sequence s's keys ``first``[s] .. (int32 [batch]; None: from its first).  Rows of no sequence are left alone.
    ``status``: optional int32 that a key behind ``lens`` or in no page, or a row between offsets that do not rise, sets
    to 1; its row is left alone."""
    import torch
    dev = _gpu(k_cache)
    heads_kv = k_cache.shape[1] if k_cache.dim() == 4 else 0
    c, d = _cache(k_cache, v_cache, block_table, lens, k_scale, v_scale, heads_kv, dev)
    out = k_out if k_out is not None else v_out
    if out is None or out.dim() != 3:
        _bad("k_out or v_out must be [rows, heads_kv, d]")
    rows, batch = out.shape[0], lens.numel()
    bf, i32 = torch.bfloat16, torch.int32
    kp, k0, k1 = _NONE if k_out is None else _rows("k_out", k_out, bf, dev, rows, heads_kv, d)
    vp, v0, v1 = _NONE if v_out is None else _rows("v_out", v_out, bf, dev, rows, heads_kv, d)
    x = _pack_read(rows, _flat("cu", cu, i32, dev, batch + 1), _flat("first", first, i32, dev, batch), kp, vp, k0, k1, v0, v1)
    _call(load().dash_kv_read, dev, stream, c, x, _flat("status", status, i32, dev, 1))


def kv_read(k_cache, v_cache, block_table, lens, cu, rows: int, first=None, k_scale=None, v_scale=None, status=None):
    """dash_kv_read into new k and v of ``rows`` rows.  Rows that no key is read into hold whatever the memory held."""
    import torch
    if k_cache.dim() != 4:
        _bad("k_cache and v_cache must be [pages, heads_kv, page_size, d] tensors alike")
    _, heads, _, d = k_cache.shape
    if k_cache.dtype is torch.uint8:
        d *= 2
    k = k_cache.new_empty((rows, heads, d), dtype=torch.bfloat16)
    v = torch.empty_like(k)
    dash_kv_read(k_cache, v_cache, block_table, lens, cu, k, v, first, k_scale, v_scale, status)
    return k, v


# ----------------------------------------------------------------- rotary positions
def dash_rotary(q, k, q_out, k_out, inv_freq, positions=None, cu=None, start=None, interleaved: bool = False,
                amplitude: float = 1.0, backward: bool = False, status=None, stream=None):
    """Queries and keys (bf16 [rows, heads, d], either may be None) turned by their positions into q_out and
    k_out (which may be q and k): ``positions`` (int32 [rows]), or ``start``[s] + t - ``cu``[s] for row t of
    sequence s (int32 [batch], None: 0, and [batch + 1]).  Pair i turns by position * ``inv_freq``[i] (fp32), times
    ``amplitude``.  ``backward``: q and k are gradients of rotated ones, turned back.  Rows of no sequence are left alone.
    ``status``: optional int32 that a row between offsets that do not rise sets to 1."""
    import torch
    if (q is None) != (q_out is None) or (k is None) != (k_out is None):
        _bad("q and q_out, k and k_out come together")
    one = k if q is None else q
    if one is None or one.dim() != 3 or (k is not None and k.dim() != 3):
        _bad("q and k must be [rows, heads, d]")
    if (positions is None) == (cu is None) or (start is not None and cu is None):
        _bad("either positions, or cu (and start)")
    if inv_freq is None:
        _bad("inv_freq must be given")
    if -1e-37 < amplitude < 1e-37:  # (0 in the struct is 1)
        _bad("amplitude must not be 0")
    dev = _gpu(one)
    rows, _, d = one.shape
    bf, i32 = torch.bfloat16, torch.int32
    hq = qp = q0 = q1 = qo = q2 = q3 = hk = kp = k0 = k1 = ko = k2 = k3 = 0
    if q is not None:
        hq = q.shape[1]
        qp, q0, q1 = _rows("q", q, bf, dev, rows, hq, d)
        qo, q2, q3 = _rows("q_out", q_out, bf, dev, rows, hq, d)
    if k is not None:
        hk = k.shape[1]
        kp, k0, k1 = _rows("k", k, bf, dev, rows, hk, d)
        ko, k2, k3 = _rows("k_out", k_out, bf, dev, rows, hk, d)
    batch = at = first = place = 0
    if cu is None:
        place = _flat("positions", positions, i32, dev, rows)
    else:
        if cu.dim() != 1 or cu.numel() < 1:
            _bad("cu must be int32 [batch + 1]")
        batch = cu.numel() - 1
        at, first = _flat("cu", cu, i32, dev, batch + 1), _flat("start", start, i32, dev, batch)
    n = inv_freq.numel()
    x = _pack_rotary(rows, hq, hk, d, place, at, first, batch, qp, kp, qo, ko, q0, q1, k0, k1, q2, q3, k2, k3,
                     _flat("inv_freq", inv_freq, torch.float32, dev, n), 2 * n, interleaved, amplitude, backward)
    _call(load().dash_rotary, dev, stream, x, _flat("status", status, i32, dev, 1))


def rotary(q, k, inv_freq, positions=None, cu=None, start=None, interleaved: bool = False, amplitude: float = 1.0,
           backward: bool = False):
    """dash_rotary into new tensors.  Rows that no sequence holds have whatever the memory held."""
    import torch
    q_out = None if q is None else torch.empty_like(q, memory_format=torch.contiguous_format)
    k_out = None if k is None else torch.empty_like(k, memory_format=torch.contiguous_format)
    dash_rotary(q, k, q_out, k_out, inv_freq, positions, cu, start, interleaved, amplitude, backward)
    return q_out, k_out


def dash_rotary_frequencies(rotary_dim: int, base: float = 10000.0, scaling="plain", factor: float = 1.0, original: float = 0.0,
                            fast: float = 32.0, slow: float = 1.0):
    """(inv_freq, amplitude) of a context stretched by ``factor`` from ``original`` positions: a host fp32
    array [rotary_dim / 2] and a number.  ``scaling``: "plain", "linear", "base" or "parts"."""
    out, amplitude = np.empty(max(rotary_dim // 2, 1), np.float32), ctypes.c_float()
    _check(load().dash_rotary_frequencies(rotary_dim, base, ROTARY_SCALINGS.get(scaling, scaling if isinstance(scaling, int) else -1),
                                          factor, original, fast, slow, out.ctypes.data, ctypes.byref(amplitude)))
    return out, amplitude.value


# ----------------------------------------------------------------- packed attention
_NO_STRIDES = (0,) * 8


def _packed(q, k, v, o, cu_q, cu_k, causal, scale, dev, *rest):
    """dash_packed_t of a packed call; `rest`: strides of the backward's tensors.  Returns
    it with the pointers of q, k, v, o."""
    import torch
    if q.dim() != 3 or k.dim() != 3:
        _bad("q and k must be [tokens, heads, d]")
    (tq, hq, d), (tk, hkv, _) = q.shape, k.shape
    if cu_q.dim() != 1 or cu_q.numel() < 1:
        _bad("cu_q must be int32 [batch + 1]")
    n = cu_q.numel()
    if cu_k is None and tk != tq:
        _bad("without cu_k, k must have as many rows as q")
    bf, i32 = torch.bfloat16, torch.int32
    qp, q0, q1 = _rows("q", q, bf, dev, tq, hq, d)
    kp, k0, k1 = _rows("k", k, bf, dev, tk, hkv, d)
    vp, v0, v1 = _rows("v", v, bf, dev, tk, hkv, d)
    op, o0, o1 = _rows("o", o, bf, dev, tq, hq, d)
    return _pack_packed(n - 1, hq, hkv, d, causal, tq, tk, 0.0 if scale is None else scale, _flat("cu_q", cu_q, i32, dev, n),
                        _flat("cu_k", cu_k, i32, dev, n), q0, q1, k0, k1, v0, v1, o0, o1, *(rest or _NO_STRIDES)), qp, kp, vp, op


def dash_packed_fwd_workspace_size(batch: int, total_q: int, total_k: int, heads_q: int, heads_kv: int, d: int) -> int:
    return int(load().dash_packed_fwd_workspace_size(batch, total_q, total_k, heads_q, heads_kv, d))


def dash_attn_packed_fwd(q, k, v, o, lse, cu_q, cu_k=None, causal: bool = True, scale=None, workspace=None, stream=None):
    """O and L of attention over packed sequences into o (bf16 [total_q, heads_q, d]) and
    lse (fp32 [heads_q, total_q]); q like o, k and v [total_k, heads_kv, d], any row and
    head strides.  ``cu_q``, ``cu_k``: int32 [batch + 1], where each sequence's queries and
    keys begin (the same without ``cu_k``); a causal mask is aligned to the last key.
    ``workspace``: None, or a uint8 device tensor of dash_packed_fwd_workspace_size bytes with
    which a call of few rows is split over its keys."""
    import torch
    dev = _gpu(q)
    p, qp, kp, vp, op = _packed(q, k, v, o, cu_q, cu_k, causal, scale, dev)
    ws, size = (0, 0) if workspace is None else _space(workspace, 0, q, dev, stream)[:2]
    _call(load().dash_attn_packed_fwd, dev, stream, p, qp, kp, vp, op,
          _flat("lse", lse, torch.float32, dev, q.shape[1], q.shape[0]), ws, size)


def attn_packed_fwd(q, k, v, cu_q, cu_k=None, causal: bool = True, scale=None):
    """dash_attn_packed_fwd into a new o and lse.  Rows that belong to no sequence (before
    cu_q[0], from cu_q[-1] on) hold whatever the memory held."""
    import torch
    dev = _gpu(q)
    if q.dim() != 3 or k.dim() != 3:
        _bad("q and k must be [tokens, heads, d]")
    (tq, hq, d), (tk, hkv, _) = q.shape, k.shape
    o = torch.empty_like(q, memory_format=torch.contiguous_format)
    lse = q.new_empty((hq, tq), dtype=torch.float32)
    n = load().dash_packed_fwd_workspace_size(cu_q.numel() - 1, tq, tk, hq, hkv, d)
    dash_attn_packed_fwd(q, k, v, o, lse, cu_q, cu_k, causal, scale, _space(None, n, q, dev, None)[2] if n else None)
    return o, lse


def dash_packed_workspace_size(batch: int, total_q: int, total_k: int, heads_q: int, heads_kv: int, d: int) -> int:
    return int(load().dash_packed_workspace_size(batch, total_q, total_k, heads_q, heads_kv, d))


def dash_attn_packed_bwd(q, k, v, o, dO, lse, dq, dk, dv, cu_q, cu_k=None, causal: bool = True, scale=None,
                         workspace=None, status=None, stream=None):
    """Backward of dash_attn_packed_fwd into dq (like q), dk and dv (like k), from its o
    and lse.  ``workspace``: a uint8 device tensor of dash_packed_workspace_size bytes
    (without it one is allocated).  ``status``: optional int32 that receives 0, or 1
    for offsets that do not rise (or after a wait timeout)."""
    import torch
    dev = _gpu(q)
    if q.dim() != 3 or k.dim() != 3:
        _bad("q and k must be [tokens, heads, d]")
    (tq, hq, d), (tk, hkv, _) = q.shape, k.shape
    bf = torch.bfloat16
    do, *dos = _rows("dO", dO, bf, dev, tq, hq, d)
    a, *dqs = _rows("dq", dq, bf, dev, tq, hq, d)
    b, *dks = _rows("dk", dk, bf, dev, tk, hkv, d)
    c, *dvs = _rows("dv", dv, bf, dev, tk, hkv, d)
    p, qp, kp, vp, op = _packed(q, k, v, o, cu_q, cu_k, causal, scale, dev, *dos, *dqs, *dks, *dvs)
    lib = load()
    need = 0 if workspace is not None else lib.dash_packed_workspace_size(cu_q.numel() - 1, tq, tk, hq, hkv, d)
    ws, size, workspace = _space(workspace, need, q, dev, stream)
    _call(lib.dash_attn_packed_bwd, dev, stream, p, qp, kp, vp, op, do,
          _flat("lse", lse, torch.float32, dev, hq, tq), a, b, c, ws, size, _flat("status", status, torch.int32, dev, 1))


def attn_packed_bwd(q, k, v, o, dO, lse, cu_q, cu_k=None, causal: bool = True, scale=None, workspace=None):
    """dash_attn_packed_bwd into new dq, dk and dv.  Rows that belong to no sequence hold
    whatever the memory held: of a padded batch, take the sequences' rows alone, or give
    dash_attn_packed_bwd gradients filled with zeros."""
    import torch
    dq, dk, dv = (torch.empty_like(t, memory_format=torch.contiguous_format) for t in (q, k, v))
    dash_attn_packed_bwd(q, k, v, o, dO, lse, dq, dk, dv, cu_q, cu_k, causal, scale, workspace)
    return dq, dk, dv


# ----------------------------------------------------------------- helpers
def new_workspace(B, H, N, d, schedule="shift"):
    import torch
    n = dash_bwd_workspace_size(B, H, N, d, schedule)
    return torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")


def attn_fwd(q, k, v, causal: bool, scale=None):
    import torch
    B, H, N, d = _shape(q)
    o = torch.empty_like(q)
    lse = torch.empty((B, H, N), dtype=torch.float32, device=q.device)
    dash_attn_fwd(q, k, v, o, lse, causal, scale)
    return o, lse


def attn_bwd(q, k, v, o, dO, lse, causal: bool, schedule="auto", scale=None, workspace=None,
             options=None):
    import torch
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    dash_attn_bwd(q, k, v, o, dO, lse, dq, dk, dv, causal, schedule, scale, workspace, options)
    return dq, dk, dv

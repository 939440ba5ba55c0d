"""GB300 mixed prefill/decode paged attention: Python binding of the C ABI.

Thin ctypes marshalling over ``_build/libfnpu.so`` (declared in
``include/fnpu.h``); every step of the computation runs in the library's CUDA
kernels. Functions carry the C names without the ``fnpu_`` prefix:

    kv_append(desc, k_new, v_new, slot_mapping, k_cache, v_cache, stream=None)
    mixed_attn_plan(desc, query_len, context_len, phase, block_table, opts=None, stream=None)
    mixed_attn_replan(plan, query_len, context_len, phase, block_table, opts=None, stream=None)
    mixed_attn_run(plan, q, k_cache, v_cache, out, lse, stream=None)
    rope(desc, inv_freq, positions, x, out=None, stream=None)
    rope_append(desc, rope, inv_freq, positions, q, k_new, v_new, slot_mapping, q_out, k_cache, v_cache, kv_format=0)
    kv_read(desc, slots, k_cache, v_cache, k_out, v_out, kv_format=0)
    kv8_attn_plan(desc, kv_format, query_len, context_len, phase, block_table, opts=None, stream=None)
    check(stream=None), plan_check(plan, stream=None), status_str(code)

Device arguments are CUDA torch tensors (torch supplies device memory and
streams only) or raw integer device addresses; host metadata are numpy arrays.
There is no CPU fallback: if the library is missing, importing the binding's
entry points raises.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional

import numpy as np

from . import build as _build

FNPU_OK = 0
FNPU_EINVAL = -1
FNPU_EUNSUPPORTED = -2
FNPU_ECUDA = -3
FNPU_EDEVICE_TIMEOUT = -4
FNPU_ENOMEM = -5
FNPU_EDEVICE_RANGE = -6

PLAN_SEPARATE_LAUNCHES = 1
PLAN_NO_TCGEN05 = 2
PLAN_GREEN_CONTEXTS = 4
PLAN_FUSED_APPEND = 8

# cache formats of rope_append, kv_read and kv8_attn_plan
KV_BF16 = 0
KV_INT8_BLOCK = 1
KV_E4M3_BLOCK = 2

EXPORTED = (
    "fnpu_kv_append", "fnpu_mixed_attn_plan", "fnpu_mixed_attn_plan_ex", "fnpu_mixed_attn_run",
    "fnpu_plan_check", "fnpu_check", "fnpu_plan_destroy", "fnpu_plan_info", "fnpu_status_str",
    "fnpu_version", "fnpu_decode_attn_noalloc", "fnpu_last_cuda_error", "fnpu_plan_phase_ms",
    "fnpu_dispatch_next_share", "fnpu_mla_expand", "fnpu_mixed_attn_replan",
    "fnpu_plan_decode_share", "fnpu_mixed_step", "fnpu_rope", "fnpu_rope_append", "fnpu_kv_read",
    "fnpu_kv8_block_bytes", "fnpu_kv8_attn_plan",
)


class FnpuError(RuntimeError):
    def __init__(self, code: int, what: str):
        msg = f"{what}: {status_str(code)} ({code})"
        if code == FNPU_ECUDA:
            msg += f" [{last_cuda_error()}]"
        super().__init__(msg)
        self.code = code


class AttnDesc(ctypes.Structure):
    _fields_ = [("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim_qk", ctypes.c_int32), ("head_dim_v", ctypes.c_int32),
                ("block_size", ctypes.c_int32), ("num_blocks", ctypes.c_int32),
                ("v_in_k_latent", ctypes.c_int32), ("softmax_scale", ctypes.c_float),
                ("kv_fp8", ctypes.c_int32)]


class PlanOpts(ctypes.Structure):
    _fields_ = [("decode_split_keys", ctypes.c_int32), ("decode_share_pct", ctypes.c_int32),
                ("num_sms", ctypes.c_int32), ("flags", ctypes.c_int32)]


class RopeDesc(ctypes.Structure):
    _fields_ = [("rotary_dim", ctypes.c_int32), ("rotary_offset", ctypes.c_int32),
                ("interleaved", ctypes.c_int32), ("inverse", ctypes.c_int32),
                ("num_axes", ctypes.c_int32), ("pair_axis", ctypes.c_void_p)]


_lib = None


def lib_path() -> str:
    return _build.LIB


def load(build_if_missing: bool = True):
    """Load the CUDA library (building it first if it is absent or stale)."""
    global _lib
    if _lib is not None:
        return _lib
    if build_if_missing:
        _build.build()
    if not os.path.exists(_build.LIB):
        raise ImportError(f"CUDA library {_build.LIB} is missing; run __graft_entry__.build()")
    lib = ctypes.CDLL(_build.LIB)
    P, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    lib.fnpu_kv_append.argtypes = [ctypes.POINTER(AttnDesc), P, P, P, i32, P, P, P]
    lib.fnpu_mixed_attn_plan.argtypes = [ctypes.POINTER(AttnDesc), i32, P, P, P, P, i32, P,
                                         ctypes.POINTER(P)]
    lib.fnpu_mixed_attn_plan_ex.argtypes = [ctypes.POINTER(AttnDesc), i32, P, P, P, P, i32,
                                            ctypes.POINTER(PlanOpts), P, ctypes.POINTER(P)]
    lib.fnpu_mixed_attn_replan.argtypes = [P, i32, P, P, P, P, i32, ctypes.POINTER(PlanOpts), P]
    lib.fnpu_mixed_attn_run.argtypes = [P, P, P, P, P, P, P]
    lib.fnpu_mixed_step.argtypes = [P, P, P, P, P, P, P, P, P, P]
    lib.fnpu_plan_decode_share.argtypes = [P, ctypes.POINTER(i32)]
    lib.fnpu_mla_expand.argtypes = [ctypes.POINTER(AttnDesc), P, P, i32, P, P, P, P, P, P]
    lib.fnpu_plan_check.argtypes = [P, P]
    lib.fnpu_check.argtypes = [P]
    lib.fnpu_plan_destroy.argtypes = [P]
    lib.fnpu_plan_destroy.restype = None
    lib.fnpu_plan_info.argtypes = [P, ctypes.POINTER(i32), ctypes.POINTER(i32), ctypes.POINTER(i32),
                                   ctypes.POINTER(i64)]
    lib.fnpu_decode_attn_noalloc.argtypes = [ctypes.POINTER(AttnDesc), i32, P, P, i32, i32, i32,
                                             P, P, P, P, P, P]
    lib.fnpu_last_cuda_error.argtypes = []
    lib.fnpu_last_cuda_error.restype = ctypes.c_char_p
    lib.fnpu_status_str.argtypes = [ctypes.c_int]
    lib.fnpu_status_str.restype = ctypes.c_char_p
    lib.fnpu_plan_phase_ms.argtypes = [P, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_float)]
    lib.fnpu_dispatch_next_share.argtypes = [i32, ctypes.c_float, ctypes.c_float, ctypes.c_float,
                                             ctypes.POINTER(i32)]
    RP, i64p = ctypes.POINTER(RopeDesc), ctypes.POINTER(i64)
    lib.fnpu_rope.argtypes = [RP, P, P, P, i64, i32, i32, i32, P, i64, P]
    lib.fnpu_rope_append.argtypes = [ctypes.POINTER(AttnDesc), i32, RP, P, P, P, i64, P, i64, P, i64, P, i32, P, P, P, P]
    lib.fnpu_kv_read.argtypes = [ctypes.POINTER(AttnDesc), i32, P, i32, P, P, P, P, P]
    lib.fnpu_kv8_block_bytes.argtypes = [ctypes.POINTER(AttnDesc), i32, i64p]
    lib.fnpu_kv8_attn_plan.argtypes = [ctypes.POINTER(AttnDesc), i32, i32, P, P, P, P, i32, ctypes.POINTER(PlanOpts), P,
                                       ctypes.POINTER(P)]
    for name in ("fnpu_rope", "fnpu_rope_append", "fnpu_kv_read", "fnpu_kv8_block_bytes", "fnpu_kv8_attn_plan"):
        getattr(lib, name).restype = ctypes.c_int
    for name in ("fnpu_kv_append", "fnpu_mixed_attn_plan", "fnpu_mixed_attn_plan_ex",
                 "fnpu_mixed_attn_run", "fnpu_plan_check", "fnpu_check", "fnpu_plan_info",
                 "fnpu_version", "fnpu_decode_attn_noalloc", "fnpu_plan_phase_ms",
                 "fnpu_dispatch_next_share", "fnpu_mla_expand", "fnpu_mixed_attn_replan",
                 "fnpu_plan_decode_share"):
        getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def last_cuda_error() -> str:
    return load().fnpu_last_cuda_error().decode()


def status_str(code: int) -> str:
    return load().fnpu_status_str(int(code)).decode()


def _dptr(x) -> Optional[int]:
    """Device address of a CUDA tensor / raw int / None."""
    if x is None or isinstance(x, int):
        return x
    try:  # a tensor as it should be, first
        if x.is_cuda and x.is_contiguous():
            return x.data_ptr()
    except AttributeError:
        pass
    if hasattr(x, "data_ptr"):
        if not x.is_cuda:
            raise ValueError("expected a CUDA tensor")
        if not x.is_contiguous():
            raise ValueError("expected a contiguous tensor")
        return x.data_ptr()
    raise TypeError(f"cannot take a device address of {type(x)!r}")


def _tptr(x) -> Optional[int]:
    """``_dptr`` of what is known to be a tensor, but for one that it refuses."""
    if x.is_cuda and x.is_contiguous():
        return x.data_ptr()
    return _dptr(x)


_raw_stream = None  # (device index) -> raw handle of torch's current stream
_current_device = None  # () -> index of the current device


def _current_stream() -> int:
    """Raw handle of torch's current stream on the current device, without
    building a Stream object for it (3.1 us a call, against 0.6)."""
    global _raw_stream, _current_device
    if _raw_stream is None:
        import torch
        torch.cuda.current_device()  # (torch's own start, before its inner functions are called)
        _current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
        get = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        _raw_stream = get or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)
    return _raw_stream(_current_device())


def _stream(stream) -> Optional[int]:
    if stream is None:
        return _current_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _np(a, dtype) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a), dtype=dtype)


def _host_ptr(a: np.ndarray) -> int:
    """Address of a contiguous array's first element; through the buffer
    protocol where it is writable and not empty (a third of the time)."""
    try:
        return ctypes.addressof(ctypes.c_char.from_buffer(a))
    except (TypeError, ValueError):
        return a.ctypes.data


def _step_meta(query_len, context_len, phase, block_table):
    """The metadata arrays of a plan, converted and checked against each other,
    and their addresses (the arrays own the memory: keep them for the call)."""
    ql, cl = _np(query_len, np.int32), _np(context_len, np.int32)
    ph, bt = _np(phase, np.uint8), _np(block_table, np.int32)
    if bt.ndim != 2 or not (ql.shape == cl.shape == ph.shape) or bt.shape[0] != ql.shape[0]:
        raise ValueError("metadata shapes disagree")
    return (ql, cl, ph, bt), (_host_ptr(ql), _host_ptr(cl), _host_ptr(ph), _host_ptr(bt), bt.shape[1])


# bytes of one block of the FP8 cache format (16 slots, 4 kv heads, d = 128):
# K or V codes [16 * 4 * 128] then fp32 scales [16 * 4]
FP8_BLOCK_BYTES = 16 * 4 * 128 + 16 * 4 * 4


def mla_expand(desc: AttnDesc, latent_cache, slots, w_uk, w_uv, workspace, k_out, v_out, stream=None,
               num_rows: Optional[int] = None) -> None:
    """Per-head keys [n, Hq, 192] and values [n, Hq, 128] of latent rows
    (``fnpu_mla_expand``): MLA prefill without absorption."""
    if num_rows is None:
        num_rows = int(slots.shape[0])
    rc = load().fnpu_mla_expand(ctypes.byref(desc), _dptr(latent_cache), _dptr(slots), int(num_rows), _dptr(w_uk),
                                _dptr(w_uv), _dptr(workspace), _dptr(k_out), _dptr(v_out), _stream(stream))
    if rc != FNPU_OK:
        raise FnpuError(rc, "fnpu_mla_expand")


def make_desc(num_q_heads, num_kv_heads, head_dim_qk, head_dim_v, block_size, num_blocks,
              latent=False, softmax_scale=0.0, kv_fp8=False) -> AttnDesc:
    return AttnDesc(num_q_heads, num_kv_heads, head_dim_qk, head_dim_v, block_size, num_blocks,
                    int(bool(latent)), float(softmax_scale), int(bool(kv_fp8)))


def kv_append(desc: AttnDesc, k_new, v_new, slot_mapping, k_cache, v_cache, stream=None,
              num_tokens: Optional[int] = None) -> None:
    """Store new K/V rows into their paged slots (``fnpu_kv_append``)."""
    if num_tokens is None:
        num_tokens = int(slot_mapping.shape[0])
    rc = load().fnpu_kv_append(ctypes.byref(desc), _dptr(k_new), _dptr(v_new), _dptr(slot_mapping),
                               int(num_tokens), _dptr(k_cache), _dptr(v_cache), _stream(stream))
    if rc != FNPU_OK:
        raise FnpuError(rc, "fnpu_kv_append")


class Plan:
    """Owner of an ``fnpu_plan*``; destroyed with the object."""

    def __init__(self, handle: int, desc: AttnDesc, num_tokens: int, kv_format: int = KV_BF16):
        self.handle = handle
        self.desc = desc
        self.num_tokens = num_tokens
        self.kv_format = kv_format
        self.shape = bytes(desc)  # as planned, whatever becomes of ``desc``
        self.pools = None if kv_format == KV_BF16 else _layout(self.shape, kv_format)[4]

    def info(self) -> dict:
        pi, di, la = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
        ws = ctypes.c_int64()
        rc = load().fnpu_plan_info(self.handle, ctypes.byref(pi), ctypes.byref(di), ctypes.byref(la),
                                   ctypes.byref(ws))
        if rc != FNPU_OK:
            raise FnpuError(rc, "fnpu_plan_info")
        return {"prefill_items": pi.value, "decode_items": di.value, "launches_per_run": la.value,
                "workspace_bytes": ws.value}

    def destroy(self) -> None:
        if self.handle:
            load().fnpu_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def mixed_attn_plan(desc: AttnDesc, query_len, context_len, phase, block_table,
                    opts: Optional[PlanOpts] = None, stream=None) -> Plan:
    """Build the phase-aware work list of one step (``fnpu_mixed_attn_plan_ex``)."""
    arrays, addr = _step_meta(query_len, context_len, phase, block_table)
    ql = arrays[0]
    out = ctypes.c_void_p()
    rc = load().fnpu_mixed_attn_plan_ex(ctypes.byref(desc), ql.shape[0], *addr,
                                        None if opts is None else ctypes.byref(opts), _stream(stream),
                                        ctypes.byref(out))
    if rc != FNPU_OK:
        raise FnpuError(rc, "fnpu_mixed_attn_plan")
    return Plan(out.value, desc, int(ql.sum()))


def mixed_attn_replan(plan: Plan, query_len, context_len, phase, block_table,
                      opts: Optional[PlanOpts] = None, stream=None) -> None:
    """Rebuild ``plan`` for a new step's metadata, reusing its streams, events,
    staging and workspace (``fnpu_mixed_attn_replan``)."""
    arrays, addr = _step_meta(query_len, context_len, phase, block_table)
    ql = arrays[0]
    rc = load().fnpu_mixed_attn_replan(plan.handle, ql.shape[0], *addr, None if opts is None else ctypes.byref(opts),
                                       _stream(stream))
    if rc != FNPU_OK:
        raise FnpuError(rc, "fnpu_mixed_attn_replan")
    plan.num_tokens = int(ql.sum())


def mixed_attn_run(plan: Plan, q, k_cache, v_cache, out, lse, stream=None) -> None:
    """Attention of every planned query (``fnpu_mixed_attn_run``)."""
    kp, vp = (_dptr(k_cache), _dptr(v_cache)) if plan.pools is None else _pool_addresses(plan.pools, k_cache, v_cache)
    rc = load().fnpu_mixed_attn_run(plan.handle, _dptr(q), kp, vp, _dptr(out), _dptr(lse), _stream(stream))
    if rc != FNPU_OK:
        raise FnpuError(rc, "fnpu_mixed_attn_run")


def mixed_step(plan: Plan, k_new, v_new, slot_mapping, q, k_cache, v_cache, out, lse, stream=None) -> None:
    """Append of the step's new rows and attention of every planned query in
    one call (``fnpu_mixed_step``; the same results as ``kv_append`` then
    ``mixed_attn_run``)."""
    kp, vp = (_dptr(k_cache), _dptr(v_cache)) if plan.pools is None else _pool_addresses(plan.pools, k_cache, v_cache)
    rc = load().fnpu_mixed_step(plan.handle, _dptr(k_new), _dptr(v_new), _dptr(slot_mapping), _dptr(q), kp, vp,
                                _dptr(out), _dptr(lse), _stream(stream))
    if rc != FNPU_OK:
        raise FnpuError(rc, "fnpu_mixed_step")


def decode_attn_noalloc(desc: AttnDesc, context_len, block_table, max_context_len: int, q,
                        k_cache, v_cache, out, lse, split_keys: int = 0, stream=None) -> None:
    """Decode attention with the library's fixed scratch and no allocation
    (``fnpu_decode_attn_noalloc``); context_len and block_table are device
    int32 tensors."""
    rc = load().fnpu_decode_attn_noalloc(ctypes.byref(desc), int(context_len.shape[0]),
                                         _dptr(context_len), _dptr(block_table),
                                         int(block_table.shape[1]), int(max_context_len),
                                         int(split_keys), _dptr(q), _dptr(k_cache), _dptr(v_cache),
                                         _dptr(out), _dptr(lse), _stream(stream))
    if rc != FNPU_OK:
        raise FnpuError(rc, "fnpu_decode_attn_noalloc")


def plan_check(plan: Plan, stream=None) -> int:
    return int(load().fnpu_plan_check(plan.handle, _stream(stream)))


def check(stream=None) -> int:
    return int(load().fnpu_check(_stream(stream)))


def version() -> int:
    return int(load().fnpu_version())


def plan_phase_ms(plan: Plan) -> tuple:
    """(prefill_ms, decode_ms) of the last co-located run of `plan`."""
    a, b = ctypes.c_float(), ctypes.c_float()
    rc = load().fnpu_plan_phase_ms(plan.handle, ctypes.byref(a), ctypes.byref(b))
    if rc != FNPU_OK:
        raise FnpuError(rc, "fnpu_plan_phase_ms")
    return a.value, b.value


def plan_decode_share(plan: Plan) -> int:
    """Decode share (percent of SMs) a co-located plan uses."""
    out = ctypes.c_int32()
    rc = load().fnpu_plan_decode_share(plan.handle, ctypes.byref(out))
    if rc != FNPU_OK:
        raise FnpuError(rc, "fnpu_plan_decode_share")
    return out.value


def dispatch_next_share(share_pct: int, prefill_ms: float, decode_ms: float, tolerance: float = 0.05) -> int:
    """Decode share (percent of SMs) for the next step of a serving loop."""
    out = ctypes.c_int32()
    rc = load().fnpu_dispatch_next_share(int(share_pct), float(prefill_ms), float(decode_ms), float(tolerance),
                                         ctypes.byref(out))
    if rc != FNPU_OK:
        raise FnpuError(rc, "fnpu_dispatch_next_share")
    return out.value


def make_rope(rotary_dim: int, rotary_offset: int = 0, interleaved: bool = False, inverse: bool = False, num_axes: int = 1,
              pair_axis=None) -> RopeDesc:
    """Descriptor of a rotation (``fnpu_rope_desc``); ``pair_axis``: the axis
    of each of the rotary_dim / 2 pairs (all 0 by default)."""
    axis = None if pair_axis is None else _np(pair_axis, np.uint8).copy()
    if axis is not None and axis.shape != (rotary_dim // 2,):
        raise ValueError("pair_axis has an entry for each of the rotary_dim / 2 pairs")
    d = RopeDesc(int(rotary_dim), int(rotary_offset), int(bool(interleaved)), int(bool(inverse)), int(num_axes),
                 None if axis is None else axis.ctypes.data)
    d._axis = axis  # (the descriptor holds its address)
    return d


_dtypes = None  # (rows, positions, frequencies, slots, 8-bit pools): torch's dtypes, looked up once


def _types():
    global _dtypes
    if _dtypes is None:
        import torch
        _dtypes = (torch.bfloat16, torch.int32, torch.float32, torch.int64, torch.uint8)
    return _dtypes


def _rows(x, shape):
    """Address and token stride of bf16 rows of that shape, [tokens, heads, d], whose
    tokens may lie apart (a slice of a fused projection's output)."""
    if not x.is_cuda:
        raise ValueError("expected a CUDA tensor")
    if x.dtype is not (_dtypes or _types())[0]:
        raise TypeError("rows are bf16")
    if x.shape != shape:
        raise ValueError(f"expected rows of shape {tuple(shape)}, not {tuple(x.shape)}")
    n, h, d = shape
    s, t, u = x.stride()
    if ((u != 1 and d > 1) or (t != d and h > 1)) and n:
        raise ValueError("the heads and columns of a token must be contiguous")
    return x.data_ptr(), s if n > 1 else h * d  # (of one token any stride may be reported)


@functools.lru_cache(maxsize=64)
def _layout(shape: bytes, kv_format: int):
    """What a descriptor, given as its bytes, and a cache format ask of a call's tensors:
    (query heads, kv heads, d_qk, d_v, pools), the last (type, elements of k_cache, of
    v_cache or None where there is none), or None for a cache that the library refuses."""
    desc = AttnDesc.from_buffer_copy(shape)
    heads, slots, pools = desc.num_kv_heads, desc.num_blocks * desc.block_size, None
    if kv_format == KV_BF16 and not desc.kv_fp8:
        pools = (_types()[0], slots * heads * desc.head_dim_qk, None if desc.v_in_k_latent else slots * heads * desc.head_dim_v)
    elif kv_format in (KV_INT8_BLOCK, KV_E4M3_BLOCK) and not desc.kv_fp8 and not desc.v_in_k_latent:
        n = slots * heads * desc.head_dim_qk + desc.num_blocks * ((heads + 3) // 4 * 16)  # codes; fp32 scales of a block
        pools = (_types()[4], n, n)
    return desc.num_q_heads, heads, desc.head_dim_qk, desc.head_dim_v, pools


def _pool_addresses(pools, k_cache, v_cache):
    """The addresses of both pools, which (where they are tensors) are of the format's type
    and hold every block that the descriptor speaks of: slots up to there are written and
    read."""
    if pools is not None:
        dtype, k, v = pools
        try:  # tensors as they should be, first
            if (not isinstance(k_cache, int) and k_cache.dtype is dtype and k_cache.numel() >= k and v is not None and
                    v_cache.dtype is dtype and v_cache.numel() >= v):
                return _tptr(k_cache), _tptr(v_cache)
        except AttributeError:
            pass
        for x, n in ((k_cache, k), (v_cache, v)):
            if isinstance(x, int) or x is None or n is None:
                continue
            if getattr(x, "dtype", None) is not dtype:
                raise TypeError(f"the pools of this cache are {dtype} tensors")
            if x.numel() < n:
                raise ValueError(f"a pool of this descriptor has {n} elements, not {x.numel()}")
    return _dptr(k_cache), _dptr(v_cache)


def _check_positions(desc: RopeDesc, inv_freq, positions, n: int) -> None:
    if inv_freq.numel() != desc.rotary_dim >> 1 or positions.numel() != desc.num_axes * n:
        raise ValueError("inv_freq is [rotary_dim / 2] and positions are [num_axes, tokens]")
    types = _dtypes or _types()
    if inv_freq.dtype is not types[2] or positions.dtype is not types[1]:
        raise TypeError("inv_freq is fp32 and positions are int32")


def rope(desc: RopeDesc, inv_freq, positions, x, out=None, stream=None) -> None:
    """Rotate rows x [n, heads, head_dim] into ``out`` (default: in place);
    ``positions`` int32 [num_axes, n], ``inv_freq`` fp32 (``fnpu_rope``)."""
    n, h, d = x.shape
    out = x if out is None else out
    _check_positions(desc, inv_freq, positions, n)
    (xp, xs), (op, os_) = _rows(x, x.shape), _rows(out, x.shape)
    rc = load().fnpu_rope(ctypes.byref(desc), _tptr(inv_freq), _tptr(positions), xp, xs, h, d, n, op, os_, _stream(stream))
    if rc != FNPU_OK:
        raise FnpuError(rc, "fnpu_rope")


def rope_append(desc: AttnDesc, rope: Optional[RopeDesc], inv_freq, positions, q, k_new, v_new, slot_mapping, q_out,
                k_cache, v_cache, kv_format: int = KV_BF16, stream=None) -> None:
    """Rotate the step's queries into ``q_out`` and its keys into their cache
    slots, and store its values (``fnpu_rope_append``); q, k_new and v_new are
    [n, heads, d], their tokens possibly apart. ``rope`` None: rows as they are."""
    n = slot_mapping.numel()
    fp, pp = None, None
    if rope is not None:
        _check_positions(rope, inv_freq, positions, n)
        fp, pp = _tptr(inv_freq), _tptr(positions)
    bf16, _, _, int64, _ = _dtypes or _types()
    if slot_mapping.dtype is not int64:
        raise TypeError("slot_mapping is int64")
    hq, h, d, dv, pools = _layout(bytes(desc), kv_format)
    kc, vc = _pool_addresses(pools, k_cache, v_cache)
    qp, qs, op, vp, vs = None, 0, None, None, 0
    if q is not None:
        qp, qs = _rows(q, (n, hq, d))
        if q_out is None or q_out.dtype is not bf16 or q_out.shape != q.shape:
            raise ValueError("q_out is bf16, of the shape of q")
        op = _tptr(q_out)
    kp, ks = _rows(k_new, (n, h, d))
    if v_new is not None:
        vp, vs = _rows(v_new, (n, h, dv))
    rc = (_lib or load()).fnpu_rope_append(ctypes.byref(desc), int(kv_format), None if rope is None else ctypes.byref(rope), fp, pp,
                                           qp, qs, kp, ks, vp, vs, _tptr(slot_mapping), n, op, kc, vc, _stream(stream))
    if rc != FNPU_OK:
        raise FnpuError(rc, "fnpu_rope_append")


def kv_read(desc: AttnDesc, slots, k_cache, v_cache, k_out, v_out, kv_format: int = KV_BF16, stream=None) -> None:
    """The rows that ``slots`` store, as bf16 (``fnpu_kv_read``)."""
    bf16, _, _, int64, _ = _dtypes or _types()
    if slots.dtype is not int64:
        raise TypeError("slots are int64")
    _, h, d, dv, pools = _layout(bytes(desc), kv_format)
    kc, vc = _pool_addresses(pools, k_cache, v_cache)
    rows = slots.shape[0] * h
    if k_out.dtype is not bf16 or k_out.numel() != rows * d or (
            v_out is not None and (v_out.dtype is not bf16 or v_out.numel() != rows * dv)):
        raise ValueError("k_out and v_out are bf16 [n, Hkv, d]")
    rc = (_lib or load()).fnpu_kv_read(ctypes.byref(desc), int(kv_format), _tptr(slots), slots.shape[0], kc, vc, _tptr(k_out),
                                       _dptr(v_out), _stream(stream))
    if rc != FNPU_OK:
        raise FnpuError(rc, "fnpu_kv_read")


def kv8_block_bytes(desc: AttnDesc, kv_format: int) -> int:
    """Bytes of one block of each pool in an 8-bit block format."""
    out = ctypes.c_int64()
    rc = load().fnpu_kv8_block_bytes(ctypes.byref(desc), int(kv_format), ctypes.byref(out))
    if rc != FNPU_OK:
        raise FnpuError(rc, "fnpu_kv8_block_bytes")
    return out.value


def kv8_attn_plan(desc: AttnDesc, kv_format: int, query_len, context_len, phase, block_table,
                  opts: Optional[PlanOpts] = None, stream=None) -> Plan:
    """A plan over an 8-bit block cache (``fnpu_kv8_attn_plan``)."""
    arrays, addr = _step_meta(query_len, context_len, phase, block_table)
    ql = arrays[0]
    out = ctypes.c_void_p()
    rc = load().fnpu_kv8_attn_plan(ctypes.byref(desc), int(kv_format), ql.shape[0], *addr,
                                   None if opts is None else ctypes.byref(opts), _stream(stream), ctypes.byref(out))
    if rc != FNPU_OK:
        raise FnpuError(rc, "fnpu_kv8_attn_plan")
    return Plan(out.value, desc, int(ql.sum()), int(kv_format))

"""ctypes binding of libdifa.so: argument marshalling only, same names as include/difa.h.

PyTorch is used for device memory and streams; every step of the operator runs in the HIP
library.  There is no fallback: if the library is missing, importing this module fails.
"""
import ctypes
import os
import struct

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("DIFA_LIBRARY", os.path.join(HERE, "libdifa.so"))   # override: another build of the same ABI

DIFA_OK, DIFA_ERR_INVALID_ARG, DIFA_ERR_UNSUPPORTED, DIFA_ERR_ALLOC, DIFA_ERR_HIP = range(5)
DIFA_HEAD_FULL, DIFA_HEAD_ARROW, DIFA_HEAD_CACHE, DIFA_HEAD_ARROW_RESIDUAL = 0, 1, 2, 3
DIFA_ITEM_ADD_RESIDUAL = 1
DIFA_DTYPE_BF16, DIFA_DTYPE_F32 = 0, 1
DIFA_LAYOUT_BHND, DIFA_LAYOUT_BNHD = 0, 1
DIFA_FLAG_BLOCK_BAND = 1
DIFA_FLAG_IMAGE_FIRST = 2
DIFA_ROPE_HALVES, DIFA_ROPE_INVERSE = 1, 2
DIFA_ACT_NONE, DIFA_ACT_GELU_TANH, DIFA_ACT_GELU_ERF, DIFA_ACT_SILU = range(4)


class difa_plan_desc_t(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("layout", ctypes.c_int32), ("max_tokens", ctypes.c_int32),
                ("softmax_scale", ctypes.c_float), ("device", ctypes.c_int32), ("flags", ctypes.c_uint32)]


class difa_work_item_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("bh", "q_tile", "kv0_end", "nm0_end", "kv1_begin", "kv1_end", "nm1_begin", "nm1_end",
                 "window", "n_tiles", "flags")]


class difa_segment_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("bh", "q_tile", "kv0_end", "nm0_end", "kv1_begin", "kv1_end", "nm1_begin", "nm1_end",
                 "window", "pos_begin", "pos_end", "part_slot", "merge_idx", "n_parts", "first_slot", "flags")]


class difa_merge_item_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("bh", "q_tile", "first_slot", "n_parts")]


class difa_rope_desc_t(ctypes.Structure):
    _fields_ = [("axes", ctypes.c_int32), ("dims", ctypes.c_int32 * 4), ("theta", ctypes.c_float)]


class difa_qkv_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q", "k", "v")] + \
               [(n, ctypes.c_int64) for n in ("stride_b", "stride_n", "stride_h")] + \
               [(n, ctypes.c_void_p) for n in ("q_weight", "k_weight")] + [("n_tokens", ctypes.c_int32)]


class difa_qkv_grad_t(ctypes.Structure):
    _fields_ = difa_qkv_t._fields_[:-1]


class difa_linear_desc_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "rows", "n", "k", "activation")] + \
               [(n, ctypes.c_int64) for n in ("x_stride_b", "x_stride_n", "w_stride", "out_stride_b", "out_stride_n",
                                              "residual_stride_b", "residual_stride_n", "gate_stride_b")]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2503_22796_amd.build` "
                          "(there is no fallback path)")
    L = ctypes.CDLL(LIB_PATH)
    vp, i32, i32p = ctypes.c_void_p, ctypes.c_int32, ctypes.POINTER(ctypes.c_int32)
    L.difa_plan_create.restype = ctypes.c_int
    L.difa_plan_create.argtypes = [ctypes.POINTER(difa_plan_desc_t), ctypes.POINTER(vp)]
    L.difa_joint_attention.restype = ctypes.c_int
    L.difa_joint_attention.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, i32, vp, vp]
    L.difa_joint_attention_static.restype = ctypes.c_int
    L.difa_joint_attention_static.argtypes = L.difa_joint_attention.argtypes
    L.difa_joint_attention_residual.restype = ctypes.c_int
    L.difa_joint_attention_residual.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, vp, vp]
    L.difa_residual_store.restype = ctypes.c_int
    L.difa_residual_store.argtypes = [vp, vp, vp, vp, i32, vp]
    L.difa_plan_destroy.restype = ctypes.c_int
    L.difa_plan_destroy.argtypes = [vp]
    L.difa_plan_describe.restype = ctypes.c_int
    L.difa_plan_describe.argtypes = [vp, ctypes.POINTER(difa_plan_desc_t)]
    L.difa_status_string.restype = ctypes.c_char_p
    L.difa_status_string.argtypes = [ctypes.c_int]
    L.difa_last_error.restype = ctypes.c_char_p
    L.difa_last_error.argtypes = [vp]
    L.difa_tile_shape.restype = i32
    L.difa_tile_shape.argtypes = [i32, i32, i32p, i32p]
    L.difa_worklist_build.restype = ctypes.c_int
    L.difa_worklist_build.argtypes = [i32, i32, vp, vp, i32, i32, i32, i32, i32, ctypes.c_uint32, vp, i32, i32p, vp, i32p]
    L.difa_schedule_build.restype = ctypes.c_int
    L.difa_schedule_build.argtypes = [vp, i32, i32, i32, vp, i32, vp, i32p, vp, i32, i32p, i32p]
    L.difa_plan_timing_enable.restype = ctypes.c_int
    L.difa_plan_timing_enable.argtypes = [vp, i32]
    L.difa_plan_timing_read.restype = ctypes.c_int
    L.difa_plan_timing_read.argtypes = [vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double),
                                        ctypes.POINTER(ctypes.c_int64), i32]
    L.difa_plan_solve.restype = ctypes.c_int
    L.difa_plan_solve.argtypes = [vp, vp, ctypes.c_double, i32, i32, ctypes.c_double, ctypes.c_double, vp,
                                  ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double)]
    L.difa_head_rse.restype = ctypes.c_int
    L.difa_head_rse.argtypes = [vp, vp, vp, i32, vp, vp]
    L.difa_plan_die_speeds.restype = ctypes.c_int
    L.difa_plan_die_speeds.argtypes = [vp, ctypes.POINTER(ctypes.c_double), i32, i32p, i32p, i32p]
    L.difa_plan_timing_read_head_rse.restype = ctypes.c_int
    L.difa_plan_timing_read_head_rse.argtypes = [vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64), i32]
    L.difa_device_info.restype = ctypes.c_int
    L.difa_device_info.argtypes = [i32, i32p, i32p, i32p, i32p, ctypes.c_char_p, i32]
    L.difa_probe_mfma_rate.restype = ctypes.c_int
    L.difa_probe_mfma_rate.argtypes = [vp, ctypes.c_int64, i32, i32, vp, vp, ctypes.POINTER(ctypes.c_double),
                                       ctypes.POINTER(ctypes.c_double)]
    i64, u32, f32 = ctypes.c_int64, ctypes.c_uint32, ctypes.c_float
    for name, args in (
            ("difa_rope_table", [vp, vp, vp, i32, vp, vp]),
            ("difa_rotate", [vp, vp, vp, vp, vp, vp, i32, i32, u32, vp]),
            ("difa_qk_norm_rotate", [vp, vp, vp, vp, i32, f32, u32, vp, vp, vp, vp]),
            ("difa_qk_norm_rotate_workspace", [vp, i32, i32, ctypes.POINTER(i64)]),
            ("difa_qk_norm_rotate_backward", [vp, vp, vp, vp, i32, f32, u32, vp, vp, vp, vp, vp, vp, i64, vp]),
            ("difa_linear_workspace", [vp, i32, i32, i32, i32, ctypes.POINTER(i64)]),
            ("difa_linear", [vp, vp, vp, vp, vp, vp, vp, vp, vp, i64, vp])):
        getattr(L, name).restype = ctypes.c_int
        getattr(L, name).argtypes = args
    return L


lib = _load()


class DifaError(RuntimeError):
    def __init__(self, status, text):
        super().__init__(f"difa status {status} ({lib.difa_status_string(status).decode()}): {text}")
        self.status = status


def difa_status_string(status: int) -> str:
    return lib.difa_status_string(int(status)).decode()


def difa_last_error(plan=None) -> str:
    return lib.difa_last_error(plan).decode()


def difa_tile_shape(head_dim: int, dtype: int = DIFA_DTYPE_BF16):
    bm, bn = ctypes.c_int32(0), ctypes.c_int32(0)
    if lib.difa_tile_shape(head_dim, dtype, ctypes.byref(bm), ctypes.byref(bn)) != 0:
        raise DifaError(DIFA_ERR_UNSUPPORTED, "difa_tile_shape: unsupported head_dim/dtype")
    return bm.value, bn.value


def _i32(a):
    return None if a is None else np.ascontiguousarray(np.asarray(a, dtype=np.int32))


def difa_worklist_build(batch, heads, head_plan, window, n_text, n_img, bm, bn, n_xcd=1, flags=0):
    """Returns (status, items as a numpy structured array, CACHE-head indices)."""
    hp, win = _i32(head_plan), _i32(window)
    n_items, n_copy = ctypes.c_int32(0), ctypes.c_int32(0)
    copy_heads = np.zeros(max(int(heads), 1), dtype=np.int32)
    st = lib.difa_worklist_build(batch, heads, hp.ctypes.data if hp is not None else None,
                                 win.ctypes.data if win is not None else None, n_text, n_img, bm, bn, n_xcd,
                                 flags, None, 0, ctypes.byref(n_items), None, ctypes.byref(n_copy))
    if st != DIFA_OK:
        return st, None, None
    items = (difa_work_item_t * max(n_items.value, 1))()
    st = lib.difa_worklist_build(batch, heads, hp.ctypes.data, win.ctypes.data if win is not None else None,
                                 n_text, n_img, bm, bn, n_xcd, flags, ctypes.cast(items, ctypes.c_void_p), n_items.value,
                                 ctypes.byref(n_items), copy_heads.ctypes.data, ctypes.byref(n_copy))
    arr = np.frombuffer(items, dtype=np.dtype([(n, np.int32) for n, _ in difa_work_item_t._fields_]),
                        count=n_items.value).copy()
    return st, arr, copy_heads[:n_copy.value].copy()


def difa_schedule_build(items, n_wg, n_xcd):
    """items: structured array as difa_worklist_build returns.  Returns (status, segments, wg_begin,
    merge items, number of scratch slots); the arrays are numpy structured / int32 arrays."""
    items = np.ascontiguousarray(items)
    n = len(items)
    seg_cap, merge_cap = n + 2 * n_wg, 2 * n_wg
    segs = (difa_segment_t * max(seg_cap, 1))()
    merges = (difa_merge_item_t * max(merge_cap, 1))()
    wg_begin = np.zeros(n_wg + 1, dtype=np.int32)
    n_segs, n_merges, n_slots = ctypes.c_int32(0), ctypes.c_int32(0), ctypes.c_int32(0)
    st = lib.difa_schedule_build(items.ctypes.data if n else None, n, n_wg, n_xcd, ctypes.cast(segs, ctypes.c_void_p),
                                 seg_cap, wg_begin.ctypes.data, ctypes.byref(n_segs),
                                 ctypes.cast(merges, ctypes.c_void_p), merge_cap, ctypes.byref(n_merges),
                                 ctypes.byref(n_slots))
    if st != DIFA_OK:
        return st, None, None, None, 0
    sa = np.frombuffer(segs, dtype=np.dtype([(n_, np.int32) for n_, _ in difa_segment_t._fields_]),
                       count=n_segs.value).copy()
    ma = np.frombuffer(merges, dtype=np.dtype([(n_, np.int32) for n_, _ in difa_merge_item_t._fields_]),
                       count=n_merges.value).copy()
    return st, sa, wg_begin, ma, n_slots.value


def difa_plan_create(batch, heads, head_dim, dtype=DIFA_DTYPE_BF16, layout=DIFA_LAYOUT_BHND,
                     max_tokens=1, softmax_scale=0.0, device=0, flags=0):
    desc = difa_plan_desc_t(batch, heads, head_dim, dtype, layout, max_tokens, softmax_scale, device, flags)
    plan = ctypes.c_void_p()
    st = lib.difa_plan_create(ctypes.byref(desc), ctypes.byref(plan))
    if st != DIFA_OK:
        raise DifaError(st, difa_last_error(None))
    plan.desc = desc
    return plan


def difa_plan_destroy(plan):
    st = lib.difa_plan_destroy(plan)
    if st != DIFA_OK:
        raise DifaError(st, "difa_plan_destroy")


def difa_plan_describe(plan):
    """What the plan object was created with, as a difa_plan_desc_t."""
    desc = difa_plan_desc_t()
    st = lib.difa_plan_describe(plan, ctypes.byref(desc))
    if st != DIFA_OK:
        raise DifaError(st, "difa_plan_describe")
    return desc


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def difa_joint_attention_static(plan, q, k, v, out, cache, head_plan, n_text, n_img, window, stream=None):
    """difa_joint_attention with the library's file-scope device array as scratch (no allocation anywhere)."""
    return difa_joint_attention(plan, q, k, v, out, cache, head_plan, n_text, n_img, window, stream=stream,
                                _entry=lib.difa_joint_attention_static)


def difa_joint_attention(plan, q, k, v, out, cache, head_plan, n_text, n_img, window, stream=None, _entry=None):
    """q, k, v, out, cache: torch tensors on the plan's device (cache may be None).

    `stream`: a torch.cuda.Stream, a raw hipStream_t integer, or None for torch's current stream.
    """
    import torch
    hp, win = _i32(head_plan), _i32(window)
    if stream is None:
        stream = torch.cuda.current_stream(q.device).cuda_stream
    elif hasattr(stream, "cuda_stream"):
        stream = stream.cuda_stream
    st = (_entry or lib.difa_joint_attention)(plan, _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(cache),
                                  hp.ctypes.data if hp is not None else None, int(n_text), int(n_img),
                                  win.ctypes.data if win is not None else None, ctypes.c_void_p(stream))
    if st != DIFA_OK:
        raise DifaError(st, difa_last_error(plan))


def difa_joint_attention_residual(plan, q, k, v, out, cache, residual, head_plan, n_text, n_img, window, stream=None):
    """difa_joint_attention with the kept differences of the DIFA_HEAD_ARROW_RESIDUAL heads (`residual`, may be None)."""
    import torch
    hp, win = _i32(head_plan), _i32(window)
    if stream is None:
        stream = torch.cuda.current_stream(q.device).cuda_stream
    elif hasattr(stream, "cuda_stream"):
        stream = stream.cuda_stream
    st = lib.difa_joint_attention_residual(plan, _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(cache), _ptr(residual),
                                           hp.ctypes.data if hp is not None else None, int(n_text), int(n_img),
                                           win.ctypes.data if win is not None else None, ctypes.c_void_p(stream))
    if st != DIFA_OK:
        raise DifaError(st, difa_last_error(plan))


def difa_residual_store(plan, o_full, o_arrow, residual, n_tokens, stream=None):
    """residual = o_full - o_arrow, element by element (device tensors of the plan's shape and dtype), asynchronous."""
    import torch
    s = stream if stream is not None else torch.cuda.current_stream(o_full.device).cuda_stream
    st = lib.difa_residual_store(plan, _ptr(o_full), _ptr(o_arrow), _ptr(residual), int(n_tokens), ctypes.c_void_p(s))
    if st != DIFA_OK:
        raise DifaError(st, difa_last_error(plan))


def difa_plan_timing_enable(plan, enable=True):
    st = lib.difa_plan_timing_enable(plan, 1 if enable else 0)
    if st != DIFA_OK:
        raise DifaError(st, "difa_plan_timing_enable")


def difa_plan_timing_read(plan, reset=True):
    """Returns (attention kernel ms, copy kernel ms, attention launches) accumulated so far."""
    a, c, n = ctypes.c_double(0), ctypes.c_double(0), ctypes.c_int64(0)
    st = lib.difa_plan_timing_read(plan, ctypes.byref(a), ctypes.byref(c), ctypes.byref(n), 1 if reset else 0)
    if st != DIFA_OK:
        raise DifaError(st, difa_last_error(plan))
    return a.value, c.value, n.value


def difa_device_info(device=0):
    """What the runtime reports for the device: a dict with compute_units, clock_khz, memory_clock_khz, l2_bytes, arch."""
    cu, clk, mclk, l2 = (ctypes.c_int32(0) for _ in range(4))
    arch = ctypes.create_string_buffer(64)
    st = lib.difa_device_info(int(device), ctypes.byref(cu), ctypes.byref(clk), ctypes.byref(mclk), ctypes.byref(l2),
                              arch, 64)
    if st != DIFA_OK:
        raise DifaError(st, "difa_device_info")
    return {"compute_units": cu.value, "clock_khz": clk.value, "memory_clock_khz": mclk.value, "l2_bytes": l2.value,
            "arch": arch.value.decode()}


def difa_probe_mfma_rate(data, waves_per_simd=1, rounds=50000, stream=None):
    """Sustained dense bf16 MFMA rate on the operand bits of `data` (a bf16 device tensor).
    Returns (TFLOP/s, milliseconds)."""
    import torch
    assert data.is_cuda and data.dtype == torch.bfloat16 and data.is_contiguous()
    scratch = torch.zeros(1, dtype=torch.float32, device=data.device)
    t, ms = ctypes.c_double(0), ctypes.c_double(0)
    s = stream if stream is not None else torch.cuda.current_stream(data.device).cuda_stream
    with torch.cuda.device(data.device):
        st = lib.difa_probe_mfma_rate(ctypes.c_void_p(data.data_ptr()), int(data.numel()), int(waves_per_simd),
                                      int(rounds), ctypes.c_void_p(scratch.data_ptr()), ctypes.c_void_p(s),
                                      ctypes.byref(t), ctypes.byref(ms))
    if st != DIFA_OK:
        raise DifaError(st, "difa_probe_mfma_rate")
    return t.value, ms.value


def difa_head_rse(plan, y_m, y_o, n_tokens, rse_out, stream=None):
    """rse_out[h] = sum (y_m - y_o)^2 / sum (y_o - mean y_o)^2 per head; device tensors, asynchronous."""
    import torch
    s = stream if stream is not None else torch.cuda.current_stream(y_m.device).cuda_stream
    st = lib.difa_head_rse(plan, ctypes.c_void_p(y_m.data_ptr()), ctypes.c_void_p(y_o.data_ptr()), int(n_tokens),
                           ctypes.c_void_p(rse_out.data_ptr()), ctypes.c_void_p(s))
    if st != DIFA_OK:
        raise DifaError(st, difa_last_error(plan))


def difa_plan_die_speeds(plan):
    """(relative die speeds, launches averaged, schedules made again)"""
    sp = (ctypes.c_double * 16)()
    n, samples, retunes = ctypes.c_int32(0), ctypes.c_int32(0), ctypes.c_int32(0)
    st = lib.difa_plan_die_speeds(plan, sp, 16, ctypes.byref(n), ctypes.byref(samples), ctypes.byref(retunes))
    if st != DIFA_OK:
        raise DifaError(st, difa_last_error(plan))
    return [float(sp[i]) for i in range(n.value)], samples.value, retunes.value


def difa_plan_timing_read_head_rse(plan, reset=True):
    """Returns (milliseconds, calls) of difa_head_rse accumulated while timing was enabled."""
    a, n = ctypes.c_double(0), ctypes.c_int64(0)
    st = lib.difa_plan_timing_read_head_rse(plan, ctypes.byref(a), ctypes.byref(n), 1 if reset else 0)
    if st != DIFA_OK:
        raise DifaError(st, difa_last_error(plan))
    return a.value, n.value


def difa_plan_solve(influence, latency, latency_full, delta, c):
    """Eq. 2 for one layer.  influence [H, M], latency [M] (host).  Returns (status, choice [H] with -1 = full
    attention, total latency, total influence)."""
    infl = np.ascontiguousarray(influence, dtype=np.float64)
    lat = np.ascontiguousarray(latency, dtype=np.float64)
    H, M = infl.shape
    assert lat.shape == (M,)
    choice = np.full(H, -2, dtype=np.int32)
    tl, ti = ctypes.c_double(0), ctypes.c_double(0)
    st = lib.difa_plan_solve(infl.ctypes.data, lat.ctypes.data, float(latency_full), H, M, float(delta), float(c),
                             choice.ctypes.data, ctypes.byref(tl), ctypes.byref(ti))
    return st, choice, tl.value, ti.value


# ------------------------------------------------------------------ around the attention of a layer
# These calls take a few microseconds on the device, so their descriptions are packed, not built field by field.
_QKV = struct.Struct("3Q3q2Qi4x")
_QKV_GRAD = struct.Struct("3Q3q2Q")
_LINEAR = struct.Struct("5i4x8q")
_ROPE = struct.Struct("5if")
assert (_QKV.size, _QKV_GRAD.size, _LINEAR.size, _ROPE.size) == tuple(
    ctypes.sizeof(c) for c in (difa_qkv_t, difa_qkv_grad_t, difa_linear_desc_t, difa_rope_desc_t))


def _stream(stream, fit):
    return fit.current_stream(fit.device) if stream is None else getattr(stream, "cuda_stream", stream)


def _addr(t):
    return None if t is None else t.data_ptr()


def _check(st, plan):
    if st != DIFA_OK:
        raise DifaError(st, difa_last_error(plan))


def _refuse(text):
    raise DifaError(DIFA_ERR_INVALID_ARG, text)


class _Fit:
    """A plan object's description in torch's terms: what tensors of its calls are compared with before their addresses are used."""
    __slots__ = ("batch", "heads", "head_dim", "bnhd", "dtype", "device", "row", "f32", "current_stream")

    def __init__(self, desc):
        import torch                              # not at the module's top: its host-only calls do without
        self.batch, self.heads, self.head_dim, self.device = desc.batch, desc.heads, desc.head_dim, desc.device
        self.bnhd = desc.layout == DIFA_LAYOUT_BNHD
        self.dtype = torch.bfloat16 if desc.dtype == DIFA_DTYPE_BF16 else torch.float32
        self.row = (self.head_dim,)
        self.f32 = torch.float32
        # the current stream's number without an object around it
        self.current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda d: torch.cuda.current_stream(d).cuda_stream)


def _fit(plan):
    try:
        return plan.fit
    except AttributeError:                        # the first call; or a handle from elsewhere, whose object may change
        if not hasattr(plan, "desc"):
            return _Fit(difa_plan_describe(plan))
        plan.fit = _Fit(plan.desc)
        return plan.fit


def _int32(*sizes):
    for n in sizes:
        if not -2 ** 31 <= n < 2 ** 31:           # ctypes would take the lowest 32 bits
            _refuse("sizes must fit 32 bits")


def _elsewhere():
    _refuse("tensors must be on the plan's device")


def _on_device(fit, *tensors):
    device = fit.device
    for t in tensors:
        if t is not None and t.get_device() != device:
            _elsewhere()


def _bytes(workspace):
    if workspace is None:
        return 0
    if not workspace.is_contiguous():
        _refuse("workspace must be contiguous")
    return workspace.numel() * workspace.element_size()


def difa_rope_table(plan, positions, dims, theta, table, stream=None):
    """table [rows, head_dim / 2, 2] (fp32): cosines and sines for `positions` [rows, axes] (fp32), axis a with dims[a] features."""
    fit, shape, to = _fit(plan), positions.shape, table.shape
    if len(shape) != 2 or not 1 <= shape[1] <= 4 or len(dims) != shape[1]:
        _refuse("positions must be [rows, axes] with 1 to 4 axes, and dims one number per axis")
    f32 = fit.f32
    if positions.dtype is not f32 or table.dtype is not f32 or not positions.is_contiguous() or not table.is_contiguous() or \
            len(to) != 3 or to[0] != shape[0] or 2 * to[1] != fit.head_dim or to[2] != 2:
        _refuse("positions and table [rows, head_dim / 2, 2] must be contiguous fp32 tensors")
    device = fit.device
    if positions.get_device() != device or table.get_device() != device:
        _elsewhere()
    try:
        desc = _ROPE.pack(shape[1], *dims, *(0,) * (4 - shape[1]), theta)
    except (struct.error, OverflowError):
        _refuse("dims must be whole numbers of 32 bits, theta a number of fp32")
    _check(lib.difa_rope_table(plan, desc, positions.data_ptr(), shape[0], table.data_ptr(), _stream(stream, fit)), plan)


def _table_batch(fit, table, n_tokens):
    """Batch entries of a table [n_tokens, head_dim / 2, 2] or [batch, n_tokens, head_dim / 2, 2]."""
    if table is None:
        return 1
    shape = table.shape
    if table.dtype is not fit.f32 or not table.is_contiguous() or len(shape) not in (3, 4) or \
            shape[-1] != 2 or 2 * shape[-2] != fit.head_dim or shape[-3] != n_tokens:
        _refuse("table must be a contiguous fp32 tensor [(batch,) tokens, head_dim / 2, 2]")
    return shape[0] if len(shape) == 4 else 1


def _joint(fit, n_tokens, *tensors):
    """Joint tensors of a call: contiguous, of the plan's shape, layout and element type."""
    dtype = fit.dtype
    shape = (fit.batch, n_tokens, fit.heads, fit.head_dim) if fit.bnhd else (fit.batch, fit.heads, n_tokens, fit.head_dim)
    for t in tensors:
        if t is not None and (t.shape != shape or t.dtype is not dtype or not t.is_contiguous()):
            _refuse(f"joint tensors must be contiguous, of the plan's element type and shape {shape}")


def difa_rotate(plan, q, k, q_out, k_out, table, n_tokens, flags=0, stream=None):
    """q_out, k_out: q and k (plan layout, n_tokens tokens; k and k_out may be None) turned by the table's angles."""
    fit = _fit(plan)
    if not 0 <= flags < 2 ** 32:
        _refuse("unknown flag bits")
    table_batch = _table_batch(fit, table, n_tokens)
    _joint(fit, n_tokens, q, k, q_out, k_out)
    _on_device(fit, q, k, q_out, k_out, table)
    _check(lib.difa_rotate(plan, q.data_ptr(), _addr(k), q_out.data_ptr(), _addr(k_out), table.data_ptr(),
                           table_batch, int(n_tokens), int(flags), _stream(stream, fit)), plan)


def _qkv(fit, stream, grad=False):
    """The C structure of a stream (q, k, v, q_weight, k_weight), and its tokens (0 for a stream that is None or empty): q, k, v
    [batch, tokens, heads, head_dim] views with the same strides and contiguous features, v and the weights may be None."""
    if stream is None:
        return None, 0
    q, k, v, qw, kw = stream
    shape = q.shape
    if len(shape) == 4 and shape[1] == 0:
        return None, 0
    st, dtype = q.stride(), fit.dtype
    if len(st) != 4 or st[3] != 1 or k.stride() != st or k.shape != shape or q.dtype is not dtype or k.dtype is not dtype or \
            (v is not None and (v.stride() != st or v.shape != shape or v.dtype is not dtype)):
        _refuse("q, k and v of a stream must be [batch, tokens, heads, head_dim] of the plan's element type, with the same strides and contiguous features")
    batch, tokens, heads, head_dim = shape
    if batch != fit.batch or heads != fit.heads or head_dim != fit.head_dim:
        _refuse("streams must have the plan's batch, heads and head_dim")
    if grad:
        dtype = fit.f32
    row = fit.row
    if (qw is not None and (qw.shape != row or qw.dtype is not dtype or qw.stride() != (1,))) or \
            (kw is not None and (kw.shape != row or kw.dtype is not dtype or kw.stride() != (1,))):
        _refuse("norm weights must be contiguous, one value per feature, of the plan's element type, and their gradients fp32")
    sb, sn, sh, _ = st
    fields = (q.data_ptr(), k.data_ptr(), 0 if v is None else v.data_ptr(), sb, sn, sh, 0 if qw is None else qw.data_ptr(),
              0 if kw is None else kw.data_ptr())
    return (_QKV_GRAD.pack(*fields) if grad else _QKV.pack(*fields, tokens)), tokens


def difa_qk_norm_rotate(plan, text, image, q_out, k_out, v_out, table=None, eps=1e-6, flags=0, stream=None):
    """Norms and turns both streams' queries and keys and gathers them, and v, into the joint tensors.

    text, image: (q, k, v, q_weight, k_weight) of the stream, or None; table: one row per joint token, or None."""
    fit = _fit(plan)
    if not 0 <= flags < 2 ** 32:
        _refuse("unknown flag bits")
    t, nt = _qkv(fit, text)
    i, ni = _qkv(fit, image)
    n = nt + ni
    _joint(fit, n, q_out, k_out, v_out)
    table_batch = _table_batch(fit, table, n)
    _on_device(fit, q_out, k_out, v_out, table, *(text if nt else ()), *(image if ni else ()))
    _check(lib.difa_qk_norm_rotate(plan, t, i, _addr(table), table_batch, float(eps), int(flags),
                                   q_out.data_ptr(), k_out.data_ptr(), _addr(v_out), _stream(stream, fit)), plan)


def difa_qk_norm_rotate_workspace(plan, n_text, n_img):
    """Bytes of workspace that the weight gradients take."""
    size = ctypes.c_int64(0)
    _int32(n_text, n_img)
    _check(lib.difa_qk_norm_rotate_workspace(plan, int(n_text), int(n_img), ctypes.byref(size)), plan)
    return size.value


def difa_qk_norm_rotate_backward(plan, text, image, dq, dk, dv, text_grad, image_grad, workspace=None, table=None, eps=1e-6,
                                 flags=0, stream=None):
    """Gradients of difa_qk_norm_rotate.  text_grad, image_grad: (dq, dk, dv, dq_weight, dk_weight) to be written, laid out
    as a stream is (dv, the weights may be None; the weights' are fp32); workspace: a byte tensor."""
    fit = _fit(plan)
    if not 0 <= flags < 2 ** 32:
        _refuse("unknown flag bits")
    t, nt = _qkv(fit, text)
    i, ni = _qkv(fit, image)
    n = nt + ni
    _joint(fit, n, dq, dk, dv)
    table_batch = _table_batch(fit, table, n)
    tg, tn = _qkv(fit, text_grad if nt else None, grad=True)
    ig, in_ = _qkv(fit, image_grad if ni else None, grad=True)
    if tn not in (0, nt) or in_ not in (0, ni):
        _refuse("a stream's gradients must have its tokens")
    size = _bytes(workspace)
    _on_device(fit, dq, dk, dv, table, workspace, *(text if nt else ()), *(image if ni else ()), *(text_grad if tn else ()), *(image_grad if in_ else ()))
    _check(lib.difa_qk_norm_rotate_backward(plan, t, i, _addr(table), table_batch, float(eps), int(flags),
                                            dq.data_ptr(), dk.data_ptr(), _addr(dv), tg, ig,
                                            _addr(workspace), size, _stream(stream, fit)), plan)


def difa_linear_workspace(plan, batch, rows, n, k):
    """Bytes of workspace that difa_linear can use for these sizes (zero-filled once by the caller); 0: none.  bf16 rows that do not
    start at multiples of 16 bytes though k is a multiple of eight (slices of a wider tensor) are copied where the workspace has
    16384 + 2 (batch * rows + n) * (k rounded up to 64) bytes."""
    size = ctypes.c_int64(0)
    _int32(batch, rows, n, k)
    _check(lib.difa_linear_workspace(plan, int(batch), int(rows), int(n), int(k), ctypes.byref(size)), plan)
    return size.value


def difa_linear(plan, x, w, out, bias=None, activation=DIFA_ACT_NONE, gate=None, residual=None, workspace=None, stream=None):
    """out = residual + gate * act(x w^T + bias).  x [(batch,) rows, k], out and residual [(batch,) rows, n]: views with
    contiguous features; w [n, k]; bias [n]; gate [n] or [batch, n]; workspace: a byte tensor, zeros before its first use."""
    fit = _fit(plan)
    shape, to, (n, k), dtype = x.shape, out.shape, w.shape, fit.dtype
    st, of, ws = x.stride(), out.stride(), w.stride()
    lead = len(st) - 1
    if lead not in (1, 2) or shape[lead] != k or len(to) != lead + 1 or to[lead] != n or to[0] != shape[0] or to[lead - 1] != shape[lead - 1]:
        _refuse("x must be [(batch,) rows, k], w [n, k], out and residual [(batch,) rows, n]")
    batch, rows = (shape[0], shape[1]) if lead == 2 else (1, shape[0])
    dense = (k == 1 or (st[lead] == 1 and ws[1] == 1)) and (n == 1 or of[lead] == 1)
    same = x.dtype is dtype and w.dtype is dtype and out.dtype is dtype
    rf, gate_stride = of, 0
    if bias is not None:
        if bias.shape != (n,):
            _refuse("bias must be [n]")
        dense, same = dense and (n == 1 or bias.stride(0) == 1), same and bias.dtype is dtype
    if gate is not None:
        if gate.shape != (n,) and gate.shape != (batch, n):
            _refuse("gate must be [n] or [batch, n]")
        gs = gate.stride()
        dense, same = dense and (n == 1 or gs[-1] == 1), same and gate.dtype is dtype
        gate_stride = gs[0] if len(gs) == 2 else 0
    if residual is not None:
        if residual.shape != to:
            _refuse("residual must have the shape of out")
        rf = residual.stride()
        dense, same = dense and (n == 1 or rf[lead] == 1), same and residual.dtype is dtype
    if not dense:
        _refuse("features must be contiguous")
    if not same:
        _refuse("tensors must have the plan's element type")
    size = _bytes(workspace)
    _on_device(fit, x, w, out, bias, gate, residual, workspace)
    if lead == 1:
        st, of, rf = (0, st[0]), (0, of[0]), (0, rf[0])
    try:
        desc = _LINEAR.pack(batch, rows, n, k, activation, st[0], st[1], ws[0] if n > 1 else k, of[0], of[1], rf[0], rf[1], gate_stride)
    except struct.error:
        _refuse("sizes and the activation must be whole numbers of 32 bits")
    _check(lib.difa_linear(plan, desc, x.data_ptr(), w.data_ptr(), _addr(bias), _addr(gate), _addr(residual),
                           out.data_ptr(), _addr(workspace), size, _stream(stream, fit)), plan)

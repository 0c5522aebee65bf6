"""ctypes binding of ``libnsp.so``: the same entry points as ``include/nsp.h``, argument marshalling only.

Every step of the path runs inside the CUDA library; torch is used here for device memory and streams. There is
no fallback: if the library has not been built (``python -m paper_2609_22755_b200.build``) importing the symbols
raises, and on a machine without a B200 the compute calls return ``NSP_ERR_CUDA`` / ``NSP_ERR_UNSUPPORTED``.
"""
from __future__ import annotations

import ctypes
import struct
from pathlib import Path

import numpy as np

NSP_OK = 0
NSP_ERR_INVALID_ARG = 1
NSP_ERR_UNSUPPORTED = 2
NSP_ERR_ALLOC = 3
NSP_ERR_CUDA = 4
NSP_ERR_DEVICE_TIMEOUT = 5
NSP_ERR_WORKSPACE = 6
NSP_ERR_DEVICE_ASSERT = 7
NSP_ERR_INFEASIBLE = 8
NSP_BF16 = 0
NSP_F32 = 1
NSP_MAX_RUNS = 32
NSP_PLAN_DETERMINISTIC_DQ = 1
NSP_PLAN_ROUNDED_DQ = 2
NSP_ROPE_HALF, NSP_ROPE_INTERLEAVED = 0, 1
NSP_ROPE_PLAIN, NSP_ROPE_LINEAR, NSP_ROPE_BASE, NSP_ROPE_PARTS = 0, 1, 2, 3
NSP_ROPE_MAX_TENSORS, NSP_ROPE_MAX_ROT, NSP_ROPE_MAX_HEAD_DIM = 64, 512, 1024
NSP_NORM_LAYER, NSP_NORM_RMS = 0, 1
NSP_NORM_MAX_DIM = 16384
NSP_ACT_SILU, NSP_ACT_GELU = 0, 1
NSP_GLU_MAX_DIM = 1048576

EXPORTS = [
    "nsp_plan_tiles", "nsp_plan_sizes", "nsp_plan_get", "nsp_attn_fwd", "nsp_attn_bwd", "nsp_device_status",
    "nsp_launch_count", "nsp_plan_destroy", "nsp_status_string", "nsp_plan_set_profiling", "nsp_plan_kernel_ms",
    "nsp_attn_bwd_static", "nsp_recompute_mark", "nsp_plan_recompute_ws_bytes", "nsp_attn_bwd_recompute",
    "nsp_cost_table", "nsp_route_sp_tree", "nsp_a2a_gather_heads", "nsp_a2a_scatter_heads",
    "nsp_selftest_wait_timeout", "nsp_a2a_gather_heads_to", "nsp_plan_set_wait_limit",
    "nsp_plan_step_host_ws_bytes", "nsp_attn_step_host", "nsp_trim", "nsp_plan_pair_items",
    "nsp_rope_frequencies", "nsp_rope", "nsp_norm_fwd", "nsp_norm_bwd_ws_bytes", "nsp_norm_bwd",
    "nsp_glu_fwd", "nsp_glu_bwd_ws_bytes", "nsp_glu_bwd", "nsp_glu_status",
]
CHECKED_EXPORTS = ["nsp_checked_withhold_load", "nsp_checked_withhold_pair_load", "nsp_checked_withhold_glu_load"]  # libnsp_checked.so only
NSP_COST_BUCKETS = 16
NSP_STATIC_WS_BYTES = 32 * 1024 * 1024
KERNEL_FWD, KERNEL_BWD_PRE, KERNEL_BWD_MAIN, KERNEL_BWD_POST, KERNEL_BWD_FIRST, KERNEL_FWD_FIRST = 0, 1, 2, 3, 4, 5

import os

# NSP_LIBRARY names another build of the same library (for instance the checked build, libnsp_checked.so, whose
# kernels verify every index they compute); the default is the library built next to this file.
LIB_PATH = Path(os.environ.get("NSP_LIBRARY", Path(__file__).resolve().parent / "libnsp.so"))
_lib = None


class NspError(RuntimeError):
    def __init__(self, code: int, what: str):
        self.code = code
        super().__init__(f"{what}: {status_string(code)} (code {code})")


class PlanOpts(ctypes.Structure):
    _fields_ = [("bm", ctypes.c_int32), ("bn", ctypes.c_int32), ("order_version", ctypes.c_int32),
                ("flags", ctypes.c_int32)]


class RopeTensor(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("y", ctypes.c_void_p), ("positions", ctypes.c_void_p), ("tokens", ctypes.c_int64),
                ("x_token_stride", ctypes.c_int64), ("x_head_stride", ctypes.c_int64), ("y_token_stride", ctypes.c_int64),
                ("y_head_stride", ctypes.c_int64), ("heads", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class RopeScaling(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("scale", ctypes.c_double), ("trained_tokens", ctypes.c_double),
                ("fast_turns", ctypes.c_double), ("slow_turns", ctypes.c_double)]


class Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("outer_stride", ctypes.c_int64), ("inner_stride", ctypes.c_int64)]


class Matrix(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("row_stride", ctypes.c_int64)]


def lib() -> ctypes.CDLL:
    """Load the CUDA library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not LIB_PATH.exists():
            raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2609_22755_b200.build` "
                              "(there is no CPU fallback)")
        L = ctypes.CDLL(str(LIB_PATH))
        vp, i32p, i64p = ctypes.c_void_p, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int64)
        L.nsp_plan_tiles.argtypes = [vp, vp, vp, ctypes.c_int32, ctypes.c_int32, vp, vp, ctypes.POINTER(vp)]
        L.nsp_plan_tiles.restype = ctypes.c_int
        L.nsp_plan_sizes.argtypes = [vp, i64p, i64p, i64p, ctypes.POINTER(ctypes.c_size_t), ctypes.POINTER(ctypes.c_size_t)]
        L.nsp_plan_sizes.restype = ctypes.c_int
        L.nsp_plan_get.argtypes = [vp, ctypes.c_int, vp, ctypes.c_int64, i64p]
        L.nsp_plan_get.restype = ctypes.c_int
        L.nsp_plan_pair_items.argtypes = [vp, ctypes.c_int, i64p, i64p]
        L.nsp_plan_pair_items.restype = ctypes.c_int
        L.nsp_attn_fwd.argtypes = [vp, vp, vp, vp, vp, vp, ctypes.c_float, vp, ctypes.c_size_t, vp]
        L.nsp_attn_fwd.restype = ctypes.c_int
        L.nsp_attn_bwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_int, ctypes.c_int, ctypes.c_float,
                                   vp, ctypes.c_size_t, vp]
        L.nsp_attn_bwd.restype = ctypes.c_int
        L.nsp_attn_bwd_static.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_int, ctypes.c_int,
                                          ctypes.c_float, vp]
        L.nsp_attn_bwd_static.restype = ctypes.c_int
        L.nsp_recompute_mark.argtypes = [vp, vp, vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int64, vp, i64p]
        L.nsp_recompute_mark.restype = ctypes.c_int
        L.nsp_plan_recompute_ws_bytes.argtypes = [vp, ctypes.POINTER(ctypes.c_size_t)]
        L.nsp_plan_recompute_ws_bytes.restype = ctypes.c_int
        L.nsp_attn_bwd_recompute.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_int, ctypes.c_int,
                                             ctypes.c_float, vp, ctypes.c_size_t, vp]
        L.nsp_attn_bwd_recompute.restype = ctypes.c_int
        L.nsp_cost_table.argtypes = [vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                     vp, vp, ctypes.c_double, vp]
        L.nsp_cost_table.restype = ctypes.c_int
        L.nsp_route_sp_tree.argtypes = [vp, vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                        ctypes.c_int64, ctypes.c_int32, vp, vp, vp, vp, i32p]
        L.nsp_route_sp_tree.restype = ctypes.c_int
        for f in (L.nsp_a2a_gather_heads, L.nsp_a2a_scatter_heads):
            f.argtypes = [vp, vp, ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                          ctypes.c_int32, vp, vp]
            f.restype = ctypes.c_int
        L.nsp_a2a_gather_heads_to.argtypes = [vp, vp, vp, vp, ctypes.c_int32, ctypes.c_int64, ctypes.c_int32, ctypes.c_int32,
                                              ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, vp, vp]
        L.nsp_a2a_gather_heads_to.restype = ctypes.c_int
        L.nsp_plan_step_host_ws_bytes.argtypes = [vp, ctypes.c_int, ctypes.c_int, ctypes.POINTER(ctypes.c_size_t)]
        L.nsp_plan_step_host_ws_bytes.restype = ctypes.c_int
        L.nsp_attn_step_host.argtypes = [vp] * 10 + [ctypes.c_int, ctypes.c_int, ctypes.c_float, vp, ctypes.c_size_t, vp]
        L.nsp_attn_step_host.restype = ctypes.c_int
        L.nsp_plan_set_wait_limit.argtypes = [vp, ctypes.c_int64]
        L.nsp_plan_set_wait_limit.restype = ctypes.c_int
        L.nsp_rope_frequencies.argtypes = [ctypes.c_int32, ctypes.c_double, ctypes.POINTER(RopeScaling), vp,
                                           ctypes.POINTER(ctypes.c_float)]
        L.nsp_rope.argtypes = [vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, vp, ctypes.c_float,
                               ctypes.c_int32, vp]
        rows = vp  # packed Rows
        L.nsp_norm_fwd.argtypes = [rows, vp, vp, rows, vp, vp, ctypes.c_int64] + [ctypes.c_int32] * 5 + [ctypes.c_float, vp]
        L.nsp_norm_bwd_ws_bytes.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.POINTER(ctypes.c_size_t)]
        L.nsp_norm_bwd.argtypes = [rows, rows, vp, vp, vp, rows, vp, vp, ctypes.c_int64] + [ctypes.c_int32] * 5 + [
            vp, ctypes.c_size_t, vp]
        matrix = vp  # a packed Matrix
        L.nsp_glu_fwd.argtypes = [matrix] * 6 + [ctypes.c_int64] + [ctypes.c_int32] * 3 + [vp]
        L.nsp_glu_bwd_ws_bytes.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(ctypes.c_size_t)]
        L.nsp_glu_bwd.argtypes = [matrix] * 9 + [ctypes.c_int64] + [ctypes.c_int32] * 3 + [vp, ctypes.c_size_t, vp]
        L.nsp_glu_status.argtypes = [i32p]
        for f in (L.nsp_glu_fwd, L.nsp_glu_bwd_ws_bytes, L.nsp_glu_bwd, L.nsp_glu_status):
            f.restype = ctypes.c_int
        for f in (L.nsp_rope_frequencies, L.nsp_rope, L.nsp_norm_fwd, L.nsp_norm_bwd_ws_bytes, L.nsp_norm_bwd):
            f.restype = ctypes.c_int
        if hasattr(L, "nsp_checked_withhold_load"):
            L.nsp_checked_withhold_load.argtypes = [vp, ctypes.c_int]
            L.nsp_checked_withhold_load.restype = ctypes.c_int
            L.nsp_checked_withhold_pair_load.argtypes = [vp, ctypes.c_int]
            L.nsp_checked_withhold_pair_load.restype = ctypes.c_int
            L.nsp_checked_withhold_glu_load.argtypes = [ctypes.c_int]
            L.nsp_checked_withhold_glu_load.restype = ctypes.c_int
        L.nsp_selftest_wait_timeout.argtypes = [vp, ctypes.c_int64, vp]
        L.nsp_selftest_wait_timeout.restype = ctypes.c_int
        L.nsp_device_status.argtypes = [vp, i32p]
        L.nsp_device_status.restype = ctypes.c_int
        L.nsp_launch_count.argtypes = []
        L.nsp_launch_count.restype = ctypes.c_int64
        L.nsp_plan_destroy.argtypes = [vp]
        L.nsp_plan_destroy.restype = ctypes.c_int
        L.nsp_trim.argtypes = []
        L.nsp_trim.restype = ctypes.c_int
        L.nsp_plan_set_profiling.argtypes = [vp, ctypes.c_int]
        L.nsp_plan_set_profiling.restype = ctypes.c_int
        L.nsp_plan_kernel_ms.argtypes = [vp, ctypes.c_int, ctypes.POINTER(ctypes.c_float)]
        L.nsp_plan_kernel_ms.restype = ctypes.c_int
        L.nsp_status_string.argtypes = [ctypes.c_int]
        L.nsp_status_string.restype = ctypes.c_char_p
        _lib = L
    return _lib


def status_string(code: int) -> str:
    return lib().nsp_status_string(int(code)).decode()


def launch_count() -> int:
    return int(lib().nsp_launch_count())


def nsp_trim():
    """Give back the memory kept from destroyed plans."""
    rc = lib().nsp_trim()
    if rc != NSP_OK:
        raise NspError(rc, "nsp_trim")


def _i32(a):
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32))


def _ptr(t):
    """Address of a torch tensor / numpy array (host metadata only) / int / None. Tensor arguments of the compute
    calls are validated by _check_tensors before they get here."""
    if t is None or isinstance(t, int):
        return t
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return t.data_ptr()


def _check_tensors(what, plan, specs):
    """Refuse buffers the kernels would read or write out of bounds: every tensor must be a contiguous CUDA tensor
    of the stated dtype with at least the plan's element count. specs: (name, tensor, allowed dtypes, min elements).
    Sizes of zero need no buffer at all."""
    import torch

    tensor, here = torch.Tensor, None
    for name, t, dtypes, need in specs:
        if need == 0:
            continue
        if not isinstance(t, tensor) or not t.is_cuda or not t.is_contiguous():
            raise NspError(NSP_ERR_INVALID_ARG, f"{what}: {name} must be a contiguous CUDA tensor")
        if t.dtype not in dtypes:
            raise NspError(NSP_ERR_INVALID_ARG, f"{what}: {name} has dtype {t.dtype}")
        if t.numel() < need:
            raise NspError(NSP_ERR_INVALID_ARG, f"{what}: {name} holds {t.numel()} elements, the plan needs {need}")
        if here is None:
            here = torch.cuda.current_device()
        if t.get_device() != here:
            raise NspError(NSP_ERR_INVALID_ARG, f"{what}: {name} is on {t.device}, not on the current device")


def _fwd_specs(plan, q, k, v, o, lse):
    import torch

    bf, f32 = (torch.bfloat16,), (torch.float32,)
    return [("q", q, bf, plan.q_elems), ("k", k, bf, plan.kv_elems), ("v", v, bf, plan.kv_elems),
            ("o", o, bf, plan.q_elems), ("lse", lse, f32, plan.lse_elems)]


def _bwd_specs(plan, q, k, v, o, d_o, lse, dq, dk, dv, dq_dtype, dkv_dtype):
    import torch

    bf, f32 = (torch.bfloat16,), (torch.float32,)
    return _fwd_specs(plan, q, k, v, o, lse) + [
        ("d_o", d_o, bf, plan.q_elems), ("dq", dq, f32 if dq_dtype == NSP_F32 else bf, plan.q_elems),
        ("dk", dk, f32 if dkv_dtype == NSP_F32 else bf, plan.kv_elems),
        ("dv", dv, f32 if dkv_dtype == NSP_F32 else bf, plan.kv_elems)]


def _check_ws(what, ws):
    import torch

    if ws is not None and (not isinstance(ws, torch.Tensor) or not ws.is_cuda or not ws.is_contiguous()):
        raise NspError(NSP_ERR_WORKSPACE, f"{what}: the workspace must be a contiguous CUDA tensor")


def _stream_ptr(stream):
    """Address of a stream (None: the current one; its handle is asked for directly where torch has that call, which is not a
    public one: building a Stream object around it costs 3 us of a call)."""
    if stream is None:
        import torch

        direct = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        return direct(torch.cuda.current_device()) if direct else torch.cuda.current_stream().cuda_stream
    return stream if isinstance(stream, int) else stream.cuda_stream


class Plan:
    """Owner of an ``nsp_plan_t*``."""

    def __init__(self, handle, n_seg):
        self.handle = handle
        self.n_seg = n_seg
        q, kv, l = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64()
        fw, bw = ctypes.c_size_t(), ctypes.c_size_t()
        rc = lib().nsp_plan_sizes(handle, ctypes.byref(q), ctypes.byref(kv), ctypes.byref(l), ctypes.byref(fw),
                                  ctypes.byref(bw))
        if rc != NSP_OK:
            raise NspError(rc, "nsp_plan_sizes")
        self.q_elems, self.kv_elems, self.lse_elems = q.value, kv.value, l.value
        self.fwd_ws_bytes, self.bwd_ws_bytes = fw.value, bw.value

    def destroy(self):
        if self.handle:
            lib().nsp_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def nsp_plan_tiles(cu_seqlens, hq, hkv, head_dim=128, opts=None, stream=None) -> Plan:
    cu, hq_, hkv_ = _i32(cu_seqlens), _i32(hq), _i32(hkv)
    n_seg = len(hq_)
    if len(cu) != n_seg + 1 or len(hkv_) != n_seg:
        raise NspError(NSP_ERR_INVALID_ARG, "nsp_plan_tiles(argument shapes)")
    o = None
    if opts is not None:
        o = PlanOpts(*opts)
    handle = ctypes.c_void_p()
    rc = lib().nsp_plan_tiles(_ptr(cu), _ptr(hq_), _ptr(hkv_), n_seg, head_dim, ctypes.byref(o) if o else None,
                              _stream_ptr(stream), ctypes.byref(handle))
    if rc != NSP_OK:
        raise NspError(rc, "nsp_plan_tiles")
    return Plan(handle, n_seg)


def nsp_plan_get(plan: Plan, pass_: int) -> np.ndarray:
    """The device work list as an int32 array [n_items, 4] = (seg, head, tile, cost)."""
    n = ctypes.c_int64()
    rc = lib().nsp_plan_get(plan.handle, pass_, None, 0, ctypes.byref(n))
    if rc != NSP_OK:
        raise NspError(rc, "nsp_plan_get")
    out = np.zeros((max(n.value, 1), 4), np.int32)
    rc = lib().nsp_plan_get(plan.handle, pass_, _ptr(out), n.value, ctypes.byref(n))
    if rc != NSP_OK:
        raise NspError(rc, "nsp_plan_get")
    return out[: n.value]


def nsp_plan_pair_items(plan: Plan, dkv_dtype: int = NSP_F32):
    """(items on pairs of thread blocks, items on single ones) of the backward main kernels with dK / dV of that type."""
    pairs, left = ctypes.c_int64(), ctypes.c_int64()
    rc = lib().nsp_plan_pair_items(plan.handle, int(dkv_dtype), ctypes.byref(pairs), ctypes.byref(left))
    if rc != NSP_OK:
        raise NspError(rc, "nsp_plan_pair_items")
    return pairs.value, left.value


def nsp_attn_fwd(plan: Plan, q, k, v, o, lse, softmax_scale, ws=None, stream=None):
    _check_tensors("nsp_attn_fwd", plan, _fwd_specs(plan, q, k, v, o, lse))
    _check_ws("nsp_attn_fwd", ws)
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    rc = lib().nsp_attn_fwd(plan.handle, _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), float(softmax_scale), _ptr(ws),
                            ws_bytes, _stream_ptr(stream))
    if rc != NSP_OK:
        raise NspError(rc, "nsp_attn_fwd")


def nsp_attn_bwd(plan: Plan, q, k, v, o, d_o, lse, dq, dk, dv, softmax_scale, ws, dq_dtype=None, dkv_dtype=None,
                 stream=None):
    import torch

    if dq_dtype is None:
        dq_dtype = NSP_F32 if dq.dtype == torch.float32 else NSP_BF16
    if dkv_dtype is None:
        dkv_dtype = NSP_F32 if dk.dtype == torch.float32 else NSP_BF16
    if dq_dtype not in (NSP_BF16, NSP_F32) or dkv_dtype not in (NSP_BF16, NSP_F32):
        raise NspError(NSP_ERR_INVALID_ARG, "nsp_attn_bwd: gradient dtype")
    _check_tensors("nsp_attn_bwd", plan, _bwd_specs(plan, q, k, v, o, d_o, lse, dq, dk, dv, dq_dtype, dkv_dtype))
    _check_ws("nsp_attn_bwd", ws)
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    rc = lib().nsp_attn_bwd(plan.handle, _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(d_o), _ptr(lse), _ptr(dq), _ptr(dk),
                            _ptr(dv), dq_dtype, dkv_dtype, float(softmax_scale), _ptr(ws), ws_bytes,
                            _stream_ptr(stream))
    if rc != NSP_OK:
        raise NspError(rc, "nsp_attn_bwd")


def nsp_plan_step_host_ws_bytes(plan: Plan, dq_dtype=NSP_BF16, dkv_dtype=NSP_F32) -> int:
    n = ctypes.c_size_t()
    rc = lib().nsp_plan_step_host_ws_bytes(plan.handle, int(dq_dtype), int(dkv_dtype), ctypes.byref(n))
    if rc != NSP_OK:
        raise NspError(rc, "nsp_plan_step_host_ws_bytes")
    return int(n.value)


def nsp_attn_step_host(plan: Plan, h_q, h_k, h_v, h_do, h_o, h_lse, h_dq, h_dk, h_dv, softmax_scale, dev_ws, stream=None):
    """Forward + backward with host tensors in and out (CPU torch tensors, pinned for asynchronous copies); dev_ws is
    a CUDA uint8 tensor of at least nsp_plan_step_host_ws_bytes. Returns (host-to-device, device-to-host) bytes."""
    import torch

    bf, f32 = (torch.bfloat16,), (torch.float32,)
    dq_dtype = NSP_F32 if h_dq.dtype == torch.float32 else NSP_BF16
    dkv_dtype = NSP_F32 if h_dk.dtype == torch.float32 else NSP_BF16
    specs = [("h_q", h_q, bf, plan.q_elems), ("h_k", h_k, bf, plan.kv_elems), ("h_v", h_v, bf, plan.kv_elems),
             ("h_do", h_do, bf, plan.q_elems), ("h_o", h_o, bf, plan.q_elems), ("h_lse", h_lse, f32, plan.lse_elems),
             ("h_dq", h_dq, f32 + bf, plan.q_elems), ("h_dk", h_dk, f32 + bf, plan.kv_elems),
             ("h_dv", h_dv, (h_dk.dtype,), plan.kv_elems)]
    for name, t, dtypes, need in specs:
        if need == 0:
            continue
        if not isinstance(t, torch.Tensor) or t.is_cuda or not t.is_contiguous() or t.dtype not in dtypes or t.numel() < need:
            raise NspError(NSP_ERR_INVALID_ARG, f"nsp_attn_step_host: {name} must be a contiguous host tensor of "
                                                f"{need} elements of {dtypes}")
    _check_ws("nsp_attn_step_host", dev_ws)
    ws_bytes = 0 if dev_ws is None else dev_ws.numel() * dev_ws.element_size()
    rc = lib().nsp_attn_step_host(plan.handle, _ptr(h_q), _ptr(h_k), _ptr(h_v), _ptr(h_do), _ptr(h_o), _ptr(h_lse),
                                  _ptr(h_dq), _ptr(h_dk), _ptr(h_dv), dq_dtype, dkv_dtype, float(softmax_scale),
                                  _ptr(dev_ws), ws_bytes, _stream_ptr(stream))
    if rc != NSP_OK:
        raise NspError(rc, "nsp_attn_step_host")
    size = lambda t: t.numel() * t.element_size()
    return (sum(size(t) for t in (h_q, h_k, h_v, h_do)), sum(size(t) for t in (h_o, h_lse, h_dq, h_dk, h_dv)))


def nsp_recompute_mark(cu_seqlens, hq, level, budget_bytes: int, head_dim: int = 128):
    """Save / recompute marking of a shard's segments under an activation budget (host only); returns
    (flags uint8 [n_seg], bytes of the saved segments)."""
    import numpy as np

    cu = np.ascontiguousarray(cu_seqlens, dtype=np.int32)
    hq = np.ascontiguousarray(hq, dtype=np.int32)
    level = np.ascontiguousarray(level, dtype=np.int32)
    n = len(hq)
    if cu.shape != (n + 1,) or level.shape != (n,):
        raise ValueError("cu_seqlens needs n_seg + 1 entries, hq and level n_seg")
    flags = np.zeros(max(n, 1), dtype=np.uint8)
    saved = ctypes.c_int64()
    vp = ctypes.c_void_p
    rc = lib().nsp_recompute_mark(cu.ctypes.data_as(vp), hq.ctypes.data_as(vp), level.ctypes.data_as(vp), n,
                                  int(head_dim), int(budget_bytes), flags.ctypes.data_as(vp), ctypes.byref(saved))
    if rc != NSP_OK:
        raise NspError(rc, "nsp_recompute_mark")
    return flags[:n], int(saved.value)


def nsp_cost_table(lengths, n_levels, hq, hkv, head_dim, tcomp_ns, link_gbs, other_ns_per_token):
    """Cost table [n_samples, n_levels] (int64 ns per covered GPU) from profiled coefficients (host only)."""
    import numpy as np

    lengths = np.ascontiguousarray(lengths, dtype=np.int32)
    tcomp = np.ascontiguousarray(tcomp_ns, dtype=np.float64)
    link = np.ascontiguousarray(link_gbs, dtype=np.float64)
    if tcomp.shape != (n_levels, NSP_COST_BUCKETS) or link.shape != (n_levels,):
        raise ValueError("tcomp_ns must be [n_levels, NSP_COST_BUCKETS], link_gbs [n_levels]")
    out = np.zeros((len(lengths), n_levels), dtype=np.int64)
    vp = ctypes.c_void_p
    rc = lib().nsp_cost_table(lengths.ctypes.data_as(vp), len(lengths), int(n_levels), int(hq), int(hkv), int(head_dim),
                              tcomp.ctypes.data_as(vp), link.ctypes.data_as(vp), float(other_ns_per_token),
                              out.ctypes.data_as(vp))
    if rc != NSP_OK:
        raise NspError(rc, "nsp_cost_table")
    return out


def nsp_route_sp_tree(lengths, cost, n_levels, prefix_k, beam_w, b_tok, monotone=False):
    """Algorithm 1 (host only). Returns (level[n], index[n], load[P], tok[P] in 1/P tokens, feasible) or raises
    NspError(NSP_ERR_INFEASIBLE)."""
    import numpy as np

    lengths = np.ascontiguousarray(lengths, dtype=np.int32)
    cost = np.ascontiguousarray(cost, dtype=np.int64)
    n = len(lengths)
    if cost.shape != (n, n_levels):
        raise ValueError("cost must be [n_samples, n_levels]")
    P = 1 << (n_levels - 1)
    level = np.zeros(max(n, 1), np.int32)
    index = np.zeros(max(n, 1), np.int32)
    load = np.zeros(P, np.int64)
    tok = np.zeros(P, np.int64)
    feas = ctypes.c_int32()
    vp = ctypes.c_void_p
    rc = lib().nsp_route_sp_tree(lengths.ctypes.data_as(vp), cost.ctypes.data_as(vp), n, int(n_levels), int(prefix_k),
                                 int(beam_w), int(b_tok), int(bool(monotone)), level.ctypes.data_as(vp),
                                 index.ctypes.data_as(vp), load.ctypes.data_as(vp), tok.ctypes.data_as(vp),
                                 ctypes.byref(feas))
    if rc != NSP_OK:
        raise NspError(rc, "nsp_route_sp_tree")
    return level[:n], index[:n], load, tok, bool(feas.value)


def _a2a(fn_name, src, dst, tokens, heads, heads_per_block, head_dim, first_head, stream):
    import torch

    dtype = NSP_F32 if src.dtype == torch.float32 else NSP_BF16
    if dst.dtype != src.dtype:
        raise ValueError("source and destination must have the same dtype")
    fh = np.ascontiguousarray(first_head, dtype=np.int32)  # refuses heads that a C int would wrap
    rc = getattr(lib(), fn_name)(_ptr(src), _ptr(dst), int(tokens), int(heads), int(heads_per_block), len(fh), int(head_dim),
                                 dtype, _ptr(fh), _stream_ptr(stream))
    if rc != NSP_OK:
        raise NspError(rc, fn_name)


def nsp_a2a_gather_heads(src, dst, tokens, heads, heads_per_block, head_dim, first_head, stream=None):
    """[tokens, heads, D] -> [len(first_head)][tokens, heads_per_block, D] (device tensors, flat or shaped)."""
    _a2a("nsp_a2a_gather_heads", src, dst, tokens, heads, heads_per_block, head_dim, first_head, stream)


def nsp_a2a_gather_heads_to(src, dst_tensors, dst_row, sample_off, tokens, heads, heads_per_block, head_dim, first_head,
                            stream=None):
    """The head gather fused with the exchange: block p is stored into dst_tensors[p] (the receiving GPU's packed
    attention buffer, or a local stand-in) at the rows dst_row[p, j] (device int64 [n_blocks, n_samples]) for the
    samples whose rows in src are given by sample_off (device int64 [n_samples + 1])."""
    import numpy as np
    import torch

    dtype = NSP_F32 if src.dtype == torch.float32 else NSP_BF16
    n = len(dst_tensors)
    fh = np.ascontiguousarray(first_head, dtype=np.int32)
    if len(fh) != n or any(t.dtype != src.dtype or not t.is_cuda for t in dst_tensors):
        raise ValueError("one destination tensor of the source's dtype per block")
    if dst_row.dtype != torch.int64 or sample_off.dtype != torch.int64 or not dst_row.is_cuda or not sample_off.is_cuda:
        raise ValueError("dst_row and sample_off are int64 device tensors")
    n_samples = sample_off.numel() - 1
    if dst_row.numel() != n * n_samples:
        raise ValueError("dst_row holds one row per (block, sample)")
    bases = (ctypes.c_void_p * n)(*[t.data_ptr() for t in dst_tensors])
    rc = lib().nsp_a2a_gather_heads_to(_ptr(src), bases, _ptr(dst_row.contiguous()), _ptr(sample_off.contiguous()),
                                       n_samples, int(tokens), int(heads), int(heads_per_block), n, int(head_dim), dtype,
                                       fh.ctypes.data_as(ctypes.c_void_p), _stream_ptr(stream))
    if rc != NSP_OK:
        raise NspError(rc, "nsp_a2a_gather_heads_to")


def nsp_a2a_scatter_heads(src, dst, tokens, heads, heads_per_block, head_dim, first_head, stream=None):
    """[len(first_head)][tokens, heads_per_block, D] -> [tokens, heads, D], adding blocks that share a head."""
    _a2a("nsp_a2a_scatter_heads", src, dst, tokens, heads, heads_per_block, head_dim, first_head, stream)


def nsp_plan_recompute_ws_bytes(plan: Plan) -> int:
    n = ctypes.c_size_t()
    rc = lib().nsp_plan_recompute_ws_bytes(plan.handle, ctypes.byref(n))
    if rc != NSP_OK:
        raise NspError(rc, "nsp_plan_recompute_ws_bytes")
    return int(n.value)


def nsp_attn_bwd_recompute(plan: Plan, recompute, q, k, v, o, d_o, lse, dq, dk, dv, softmax_scale, ws, dq_dtype=None,
                           dkv_dtype=None, stream=None):
    """nsp_attn_bwd with per-segment flags (uint8 [n_seg], host): o and lse of a flagged segment are never read."""
    import numpy as np
    import torch

    recompute = np.ascontiguousarray(recompute, dtype=np.uint8)
    if recompute.shape != (plan.n_seg,):
        raise ValueError("recompute must have one entry per segment")
    if dq_dtype is None:
        dq_dtype = NSP_F32 if dq.dtype == torch.float32 else NSP_BF16
    if dkv_dtype is None:
        dkv_dtype = NSP_F32 if dk.dtype == torch.float32 else NSP_BF16
    _check_tensors("nsp_attn_bwd_recompute", plan,
                   _bwd_specs(plan, q, k, v, o, d_o, lse, dq, dk, dv, dq_dtype, dkv_dtype))
    _check_ws("nsp_attn_bwd_recompute", ws)
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    rc = lib().nsp_attn_bwd_recompute(plan.handle, recompute.ctypes.data_as(ctypes.c_void_p), _ptr(q), _ptr(k), _ptr(v),
                                      _ptr(o), _ptr(d_o), _ptr(lse), _ptr(dq), _ptr(dk), _ptr(dv), dq_dtype, dkv_dtype,
                                      float(softmax_scale), _ptr(ws), ws_bytes, _stream_ptr(stream))
    if rc != NSP_OK:
        raise NspError(rc, "nsp_attn_bwd_recompute")


def nsp_selftest_wait_timeout(plan: Plan, limit_clk: int = 1_000_000, stream=None):
    """Let one bounded device-side wait run out on purpose; the plan's status word then holds NSP_ERR_DEVICE_TIMEOUT."""
    rc = lib().nsp_selftest_wait_timeout(plan.handle, int(limit_clk), _stream_ptr(stream))
    if rc != NSP_OK:
        raise NspError(rc, "nsp_selftest_wait_timeout")


def nsp_plan_set_wait_limit(plan: Plan, sm_clocks: int):
    rc = lib().nsp_plan_set_wait_limit(plan.handle, int(sm_clocks))
    if rc != NSP_OK:
        raise NspError(rc, "nsp_plan_set_wait_limit")


def nsp_checked_withhold_load(plan: Plan, enable: bool):
    """Checked build only: the next forward launch leaves out one V tile load (failure-detection test)."""
    if not hasattr(lib(), "nsp_checked_withhold_load"):
        raise NspError(NSP_ERR_UNSUPPORTED, "nsp_checked_withhold_load (needs libnsp_checked.so)")
    rc = lib().nsp_checked_withhold_load(plan.handle, int(bool(enable)))
    if rc != NSP_OK:
        raise NspError(rc, "nsp_checked_withhold_load")


def nsp_checked_withhold_pair_load(plan: Plan, load: int):
    """Checked build only: later backward launches on CTA pairs leave out one tile load (1 .. 5, see nsp.h; 0: none)."""
    if not hasattr(lib(), "nsp_checked_withhold_pair_load"):
        raise NspError(NSP_ERR_UNSUPPORTED, "nsp_checked_withhold_pair_load (needs libnsp_checked.so)")
    rc = lib().nsp_checked_withhold_pair_load(plan.handle, int(load))
    if rc != NSP_OK:
        raise NspError(rc, "nsp_checked_withhold_pair_load")


def nsp_checked_withhold_glu_load(load: int):
    """Checked build only: later nsp_glu launches leave out one tile load (1: of A, 2: of B, 0: none)."""
    if not hasattr(lib(), "nsp_checked_withhold_glu_load"):
        raise NspError(NSP_ERR_UNSUPPORTED, "nsp_checked_withhold_glu_load (needs libnsp_checked.so)")
    rc = lib().nsp_checked_withhold_glu_load(int(load))
    if rc != NSP_OK:
        raise NspError(rc, "nsp_checked_withhold_glu_load")


def nsp_device_status(plan: Plan):
    out = (ctypes.c_int32 * 4)()
    rc = lib().nsp_device_status(plan.handle, out)
    if rc != NSP_OK:
        raise NspError(rc, "nsp_device_status")
    return tuple(out)


def nsp_plan_set_profiling(plan: Plan, enable: bool):
    rc = lib().nsp_plan_set_profiling(plan.handle, int(bool(enable)))
    if rc != NSP_OK:
        raise NspError(rc, "nsp_plan_set_profiling")


def nsp_plan_kernel_ms(plan: Plan, kernel_id: int) -> float:
    ms = ctypes.c_float()
    rc = lib().nsp_plan_kernel_ms(plan.handle, kernel_id, ctypes.byref(ms))
    if rc != NSP_OK:
        raise NspError(rc, "nsp_plan_kernel_ms")
    return float(ms.value)


def nsp_attn_bwd_static(plan: Plan, q, k, v, o, d_o, lse, dq, dk, dv, softmax_scale, dq_dtype=None, dkv_dtype=None,
                        stream=None):
    """nsp_attn_bwd for callers that may not allocate: no workspace argument, the scratch is a fixed array inside
    the library (at most NSP_STATIC_WS_BYTES; larger batches raise NSP_ERR_WORKSPACE). Calls sharing a device
    must not overlap. Make the first call on a device outside any stream capture."""
    import torch

    if dq_dtype is None:
        dq_dtype = NSP_F32 if dq.dtype == torch.float32 else NSP_BF16
    if dkv_dtype is None:
        dkv_dtype = NSP_F32 if dk.dtype == torch.float32 else NSP_BF16
    _check_tensors("nsp_attn_bwd_static", plan,
                   _bwd_specs(plan, q, k, v, o, d_o, lse, dq, dk, dv, dq_dtype, dkv_dtype))
    rc = lib().nsp_attn_bwd_static(plan.handle, _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(d_o), _ptr(lse), _ptr(dq),
                                   _ptr(dk), _ptr(dv), dq_dtype, dkv_dtype, float(softmax_scale), _stream_ptr(stream))
    if rc != NSP_OK:
        raise NspError(rc, "nsp_attn_bwd_static")


# ---- token-wise operators around the attention
# The small calls of these last about as long as the checks around them: structures are packed at once (struct) instead of field by
# field, every attribute of a tensor is asked for once, and what is needed of torch is looked up once (an import statement inside a
# function costs 0.2 us each time).
_INT32_MAX = 2 ** 31 - 1
_ROPE_TENSOR, _ROWS, _MATRIX = (struct.Struct(f) for f in ("=QQQqqqqqii", "=Qqq", "=Qq"))


class _Torch:
    """Filled at the first call (the host-only functions of this module need no torch)."""

    ready = False

    @classmethod
    def fill(cls):
        import torch

        cls.bf16, cls.f32, cls.i64 = torch.bfloat16, torch.float32, torch.int64
        cls.Tensor, cls.current_device = torch.Tensor, torch.cuda.current_device
        cls.raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        cls.code = {torch.bfloat16: NSP_BF16, torch.float32: NSP_F32}
        cls.both, cls.only_f32 = (torch.float32, torch.bfloat16), (torch.float32,)
        cls.ready = True


def _refuse(what, why, code=NSP_ERR_INVALID_ARG):
    raise NspError(code, f"{what}: {why}")


def _on_device(what, names, tensors):
    """The current device; refuses tensors that are not on it (None is left out)."""
    if not _Torch.ready:
        _Torch.fill()
    here = None
    for t in tensors:
        if t is None:
            continue
        at = t.get_device() if isinstance(t, _Torch.Tensor) else -1
        if at != here:
            name = names[[x is t for x in tensors].index(True) % len(names)]
            if at < 0:
                _refuse(what, f"{name} must be a CUDA tensor")
            current = _Torch.current_device()
            if at != current:
                _refuse(what, f"{name} is on {t.device}, not on the current device")
            here = current
    return here


def _stream_on(here, stream):
    """As _stream_ptr, with the current device known."""
    if stream is None and here is not None and _Torch.raw_stream:
        return _Torch.raw_stream(here)
    return _stream_ptr(stream)


def _dtype_of(what, name, dtype):
    code = _Torch.code.get(dtype)
    if code is None:
        _refuse(what, f"{name} has dtype {dtype}")
    return code


def nsp_rope_frequencies(rot_dim, base=10000.0, kind=NSP_ROPE_PLAIN, scale=1.0, trained_tokens=0.0, fast_turns=32.0,
                         slow_turns=1.0):
    """(radians per position float64 [rot_dim / 2], magnitude) of rotary positions (host only); kind: NSP_ROPE_PLAIN, or how
    they are scaled for contexts `scale` times the trained ones (see nsp.h)."""
    out = np.zeros(max(int(rot_dim) // 2, 1), np.float64)
    m = ctypes.c_float()
    sc = RopeScaling(int(kind), float(scale), float(trained_tokens), float(fast_turns), float(slow_turns))
    rc = lib().nsp_rope_frequencies(int(rot_dim), float(base), ctypes.byref(sc), _ptr(out), ctypes.byref(m))
    if rc != NSP_OK:
        raise NspError(rc, "nsp_rope_frequencies")
    return out, float(m.value)


def nsp_rope(xs, ys, positions, inv_freq, layout=NSP_ROPE_HALF, magnitude=1.0, inverse=False, stream=None):
    """Rotate the heads of xs (a tensor [tokens, heads, head_dim], or a list of them with one head_dim) by their positions into
    ys (of the same shapes and types; x itself: in place), all in one launch. positions: int64 CUDA tensor [tokens], a list of
    them, or None (0, 1, 2, ...). inv_freq: float64 [rot_dim / 2] on the host. inverse: the gradient's way back."""
    what = "nsp_rope"
    if not _Torch.ready:
        _Torch.fill()
    if isinstance(xs, _Torch.Tensor):
        xs, ys = [xs], [ys]
    if not isinstance(positions, (list, tuple)):
        positions = [positions] * len(xs)
    if len(ys) != len(xs) or len(positions) != len(xs):
        _refuse(what, "as many outputs and positions as inputs")
    freq = np.ascontiguousarray(inv_freq, dtype=np.float64)
    if freq.ndim != 1 or len(freq) == 0:
        _refuse(what, "inv_freq holds one frequency per rotated pair")
    if len(xs) > NSP_ROPE_MAX_TENSORS:
        _refuse(what, f"more than {NSP_ROPE_MAX_TENSORS} tensors", NSP_ERR_UNSUPPORTED)
    if not xs:
        return
    here = _on_device(what, ("x", "y", "positions"), [t for group in zip(xs, ys, positions) for t in group])
    packed, head_dim, known = [], xs[0].shape[-1], None
    for x, y, pos in zip(xs, ys, positions):
        shape, dtype, sx, sy = x.shape, x.dtype, x.stride(), y.stride()
        if len(shape) != 3 or shape[2] != head_dim or y.shape != shape or y.dtype != dtype:
            _refuse(what, "x and y are [tokens, heads, head_dim] of one shape and type, with one head_dim in all")
        if head_dim > 1 and (sx[2] != 1 or sy[2] != 1):
            _refuse(what, "the elements of a head must be contiguous")
        tokens, heads = shape[0], shape[1]
        if heads > _INT32_MAX or head_dim > NSP_ROPE_MAX_HEAD_DIM:  # the library takes them in 32 bits
            _refuse(what, f"x has shape {tuple(shape)}", NSP_ERR_UNSUPPORTED)
        if pos is None:
            at = 0
        else:
            if pos is not known or tokens != known_tokens:
                if pos.dtype != _Torch.i64 or pos.shape != (tokens,) or not pos.is_contiguous():
                    _refuse(what, "positions must be a contiguous int64 tensor with one entry per token")
                known, known_tokens, known_at = pos, tokens, pos.data_ptr()
            at = known_at
        if tokens * heads * head_dim == 0:
            continue
        packed.append(_ROPE_TENSOR.pack(x.data_ptr(), y.data_ptr(), at, tokens, sx[0], sx[1], sy[0], sy[1], heads, _dtype_of(what, "x", dtype)))
    rc = lib().nsp_rope(b"".join(packed), len(packed), head_dim, 2 * len(freq), int(layout), freq.tobytes(), float(magnitude),
                        1 if inverse else 0, _stream_on(here, stream))
    if rc != NSP_OK:
        raise NspError(rc, what)


def _rows(what, name, t, shape, dtype):
    """A packed nsp_rows_t of a tensor [rows, dim] or [outer, inner, dim] of that shape and type, with contiguous last axis."""
    if t.shape != shape or t.dtype != dtype:
        _refuse(what, f"{name} must have x's shape and type")
    strides = t.stride()
    if strides[-1] != 1 and shape[-1] > 1:
        _refuse(what, f"the last axis of {name} must be contiguous")
    return _ROWS.pack(t.data_ptr(), strides[0], strides[1] if len(strides) == 3 else 0)


def _norm_shape(what, x):
    """(outer, inner, dim, dtype code) of x."""
    shape = x.shape
    if len(shape) == 2:
        outer, inner, dim = shape[0], 1, shape[1]
    elif len(shape) == 3:
        outer, inner, dim = shape
    else:
        _refuse(what, "x must be [rows, dim] or [outer, inner, dim]")
    if inner > _INT32_MAX or dim > NSP_NORM_MAX_DIM:  # the library takes them in 32 bits
        _refuse(what, f"x has shape {tuple(shape)}", NSP_ERR_UNSUPPORTED)
    return outer, inner, dim, _dtype_of(what, "x", x.dtype)


def _norm_vector(what, name, t, n, dtypes):
    """Address of a contiguous tensor of n elements of these types; None: a null pointer."""
    if t is None:
        return None
    if t.numel() != n or t.dtype not in dtypes or not t.is_contiguous():
        _refuse(what, f"{name} must be contiguous, with {n} elements of {dtypes}")
    return t.data_ptr()


def nsp_norm_fwd(x, weight, bias, y, mean, rstd, eps=1e-5, kind=NSP_NORM_LAYER, stream=None):
    """Layer norm or RMS norm of the rows of x [rows, dim] or [outer, inner, dim] into y (x itself: in place). weight, bias [dim]
    (bf16 or fp32, None = 1 and 0); mean, rstd: fp32, one entry per row, for the backward pass (None: not wanted)."""
    what = "nsp_norm_fwd"
    here = _on_device(what, ("x", "y", "weight", "bias", "mean", "rstd"), (x, y, weight, bias, mean, rstd))
    outer, inner, dim, dtype = _norm_shape(what, x)
    rows, both, f32 = outer * inner, _Torch.both, _Torch.only_f32
    rx, ry = _rows(what, "x", x, x.shape, x.dtype), _rows(what, "y", y, x.shape, x.dtype)
    w, b = _norm_vector(what, "weight", weight, dim, both), _norm_vector(what, "bias", bias, dim, both)
    if weight is not None and bias is not None and weight.dtype != bias.dtype:
        _refuse(what, "weight and bias have one type")
    m, r = _norm_vector(what, "mean", mean, rows, f32), _norm_vector(what, "rstd", rstd, rows, f32)
    if rows == 0 or dim == 0:
        return
    one = weight if weight is not None else bias
    w_dtype = NSP_BF16 if one is not None and one.dtype == _Torch.bf16 else NSP_F32
    rc = lib().nsp_norm_fwd(rx, w, b, ry, m, r, outer, inner, dim, dtype, w_dtype, int(kind), float(eps), _stream_on(here, stream))
    if rc != NSP_OK:
        raise NspError(rc, what)


def nsp_norm_bwd_ws_bytes(rows, dim) -> int:
    n = ctypes.c_size_t()
    rc = lib().nsp_norm_bwd_ws_bytes(int(rows), int(dim), ctypes.byref(n))
    if rc != NSP_OK:
        raise NspError(rc, "nsp_norm_bwd_ws_bytes")
    return int(n.value)


def nsp_norm_bwd(x, dy, weight, mean, rstd, dx, dweight, dbias, ws, kind=NSP_NORM_LAYER, stream=None):
    """Backward pass of nsp_norm_fwd: dx of x's shape and type (x or dy itself: in place), dweight and dbias fp32 [dim]
    (overwritten; None: not wanted). ws: a CUDA tensor of at least nsp_norm_bwd_ws_bytes(rows, dim) bytes (None where neither
    is wanted)."""
    what = "nsp_norm_bwd"
    here = _on_device(what, ("x", "dy", "dx", "weight", "mean", "rstd", "dweight", "dbias", "ws"),
                      (x, dy, dx, weight, mean, rstd, dweight, dbias, ws))
    outer, inner, dim, dtype = _norm_shape(what, x)
    rows, both, f32 = outer * inner, _Torch.both, _Torch.only_f32
    rx, rdy, rdx = (_rows(what, name, t, x.shape, x.dtype) for name, t in (("x", x), ("dy", dy), ("dx", dx)))
    w = _norm_vector(what, "weight", weight, dim, both)
    dw, db = _norm_vector(what, "dweight", dweight, dim, f32), _norm_vector(what, "dbias", dbias, dim, f32)
    if rstd is None or (mean is None and kind == NSP_NORM_LAYER):
        _refuse(what, "the forward pass's statistics are needed")
    m, r = _norm_vector(what, "mean", mean, rows, f32), _norm_vector(what, "rstd", rstd, rows, f32)
    _check_ws(what, ws)
    if dim == 0:
        return
    w_dtype = NSP_BF16 if weight is not None and weight.dtype == _Torch.bf16 else NSP_F32
    rc = lib().nsp_norm_bwd(rx, rdy, w, m, r, rdx, dw, db, outer if rows else 0, inner if rows else 1, dim, dtype, w_dtype, int(kind),
                            None if ws is None else ws.data_ptr(), 0 if ws is None else ws.numel() * ws.element_size(),
                            _stream_on(here, stream))
    if rc != NSP_OK:
        raise NspError(rc, what)


def _matrix(what, name, t, rows, cols):
    """A packed nsp_matrix_t of a bf16 tensor [rows, cols] with contiguous rows (None: a null pointer)."""
    if t is None:
        return None
    if t.dtype != _Torch.bf16:
        _refuse(what, f"{name} has dtype {t.dtype}")
    strides = t.stride()
    if t.shape != (rows, cols) or (cols > 1 and strides[1] != 1):
        _refuse(what, f"{name} must be [{rows}, {cols}] with contiguous rows")
    return _MATRIX.pack(t.data_ptr(), strides[0])


def _glu_sizes(what, x, w_gate):
    sx, sw = x.shape, w_gate.shape
    if len(sx) != 2 or len(sw) != 2:
        _refuse(what, "x is [rows, d_model], w_gate and w_up are [d_ff, d_model]")
    if sx[1] > NSP_GLU_MAX_DIM or sw[0] > NSP_GLU_MAX_DIM:  # the library takes them in 32 bits
        _refuse(what, f"d_model {sx[1]}, d_ff {sw[0]}", NSP_ERR_UNSUPPORTED)
    return sx[0], sx[1], sw[0]


def nsp_glu_fwd(x, w_gate, w_up, h, g=None, u=None, act=NSP_ACT_SILU, stream=None):
    """h = act(x w_gate^T) * (x w_up^T), bf16 tensors x [rows, d_model], w_gate and w_up [d_ff, d_model], h [rows, d_ff]; g and u
    (as h): the two projections, for the backward pass."""
    what = "nsp_glu_fwd"
    here = _on_device(what, ("x", "w_gate", "w_up", "h", "g", "u"), (x, w_gate, w_up, h, g, u))
    rows, d, f = _glu_sizes(what, x, w_gate)
    rc = lib().nsp_glu_fwd(_matrix(what, "x", x, rows, d), _matrix(what, "w_gate", w_gate, f, d), _matrix(what, "w_up", w_up, f, d),
                           _matrix(what, "h", h, rows, f), _matrix(what, "g", g, rows, f), _matrix(what, "u", u, rows, f), rows, d, f,
                           int(act), _stream_on(here, stream))
    if rc != NSP_OK:
        raise NspError(rc, what)


def nsp_glu_bwd_ws_bytes(rows, d_model, d_ff) -> int:
    n = ctypes.c_size_t()
    rc = lib().nsp_glu_bwd_ws_bytes(int(rows), int(d_model), int(d_ff), ctypes.byref(n))
    if rc != NSP_OK:
        raise NspError(rc, "nsp_glu_bwd_ws_bytes")
    return int(n.value)


def nsp_glu_bwd(dh, x, w_gate, w_up, g, u, dx, dw_gate, dw_up, ws, act=NSP_ACT_SILU, stream=None):
    """Backward pass of nsp_glu_fwd from dh and the g, u it saved: dx (None: not wanted), dw_gate and dw_up (both None: not
    wanted), overwritten. ws: a CUDA tensor of at least nsp_glu_bwd_ws_bytes(rows, d_model, d_ff) bytes."""
    what = "nsp_glu_bwd"
    here = _on_device(what, ("dh", "x", "w_gate", "w_up", "g", "u", "dx", "dw_gate", "dw_up", "ws"),
                      (dh, x, w_gate, w_up, g, u, dx, dw_gate, dw_up, ws))
    rows, d, f = _glu_sizes(what, x, w_gate)
    _check_ws(what, ws)
    rc = lib().nsp_glu_bwd(_matrix(what, "dh", dh, rows, f), _matrix(what, "x", x, rows, d), _matrix(what, "w_gate", w_gate, f, d),
                           _matrix(what, "w_up", w_up, f, d), _matrix(what, "g", g, rows, f), _matrix(what, "u", u, rows, f),
                           _matrix(what, "dx", dx, rows, d), _matrix(what, "dw_gate", dw_gate, f, d), _matrix(what, "dw_up", dw_up, f, d),
                           rows, d, f, int(act), None if ws is None else ws.data_ptr(),
                           0 if ws is None else ws.numel() * ws.element_size(), _stream_on(here, stream))
    if rc != NSP_OK:
        raise NspError(rc, what)


def nsp_glu_status():
    """The record of the nsp_glu calls on the current device, (code, tile, where, aux); code 0 = healthy. Synchronises."""
    out = (ctypes.c_int32 * 4)()
    rc = lib().nsp_glu_status(out)
    if rc != NSP_OK:
        raise NspError(rc, "nsp_glu_status")
    return tuple(out)
